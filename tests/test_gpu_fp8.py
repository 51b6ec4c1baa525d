"""The 8-bit floating-point stores, their product and the linear layer on it, against the float64 references
in fp8_ref."""
import numpy as np
import pytest
import torch

import fp8_ref as F
import ops_ref as R
from paper_2404_14712_amd._lib import Fp8LinearDesc

pytestmark = pytest.mark.gpu


def _data(rows, n, dtype, seed, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(rows, n, generator=g, dtype=torch.float64)
    if spread:
        t = t * torch.exp((torch.rand(rows, 1, generator=g, dtype=torch.float64) * 2 - 1) * spread)
    return t.float().to(R.TORCH[dtype])


def _bytes(n, fill=0xA5):
    return torch.full((max(n, 1),), fill, dtype=torch.uint8, device="cuda")


def _pack(lib, x, tile=1, both=False, ldx=None, rows_only=True):
    rows, n = x.shape
    s = _bytes(lib.orbit_fp8_bytes(rows, n)) if rows_only else None
    st = _bytes(lib.orbit_fp8_bytes(n, rows)) if both else None
    code = R.CODE["bf16" if x.dtype == torch.bfloat16 else "f32"]
    ld = ldx or -(-n // 8) * 8
    wide = torch.full((rows, ld), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, :n] = x.cuda()
    lib.orbit_fp8_pack(code, rows, n, tile, wide, ld, s, st)
    return s, st


def _check_store(s, x, tile):
    rows, n = x.shape
    codes, E, val = F.pack_ref(x.double().numpy(), tile)
    wide, groups, at, _ = F.layout(rows, n)
    b = s.cpu().numpy()
    got = b[:rows * wide].reshape(rows, wide)
    np.testing.assert_array_equal(got[:, :n], codes)
    assert not got[:, n:].any()
    ge = b[at:at + rows * groups].reshape(rows, groups)
    np.testing.assert_array_equal(ge[:, :E.shape[1]], E)
    assert not ge[:, E.shape[1]:].any()
    return val


SHAPES = [(1, 8), (1, 1024), (3, 130), (128, 128), (129, 257), (300, 1000), (37, 1), (1000, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_store_bits(lib, rows, n, tile, dtype):
    """Codes, E and values bit for bit, in both orientations, over many binades; padding zero, strides, and what lies
    past the row left alone."""
    x = _data(rows, n, dtype, rows + n, spread=80.0)
    if rows > 2:
        x[1] = 0.0
        x[2, ::3] = -0.0
    for both, only, ld in ((True, True, None), (False, True, -(-n // 8) * 8 + 16), (True, False, None)):
        s, st = _pack(lib, x, tile, both, ld, only)
        if only:
            val = _check_store(s, x, tile)
            ldx = -(-n // 8) * 8 + 8
            back = torch.full((rows, ldx), 7.0, dtype=x.dtype, device="cuda")
            lib.orbit_fp8_unpack(R.CODE[dtype], rows, n, s, back, ldx)
            np.testing.assert_array_equal(back[:, :n].double().cpu().numpy(), val)
            assert (back[:, n:] == 7.0).all()
        if both:
            _check_store(st, x.t().contiguous(), tile)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_store_extremes(lib, dtype):
    """The largest and smallest finite values, ties, infinities and NaN, each in its place only."""
    big = torch.finfo(R.TORCH[dtype]).max
    x = torch.zeros(9, 256, dtype=torch.float64)
    x[0, :5] = torch.tensor([big, -big, 1e30, 1.0, 1e38], dtype=torch.float64)
    x[1, :4] = torch.tensor([1e-45, -1e-40, 2.0 ** -126, 2.0 ** -133], dtype=torch.float64)
    x[2] = torch.arange(256, dtype=torch.float64) * 1.0625            # ties among them
    x[3, :6] = torch.tensor([float("inf"), 1.0, float("nan"), -2.0, float("-inf"), 448.0], dtype=torch.float64)
    x[4] = float("nan")
    x[5, 128:] = float("inf")
    x[6, :127] = 2.0 ** -8
    x[7] = torch.linspace(-464, 464, 256, dtype=torch.float64)
    x[8, 200] = -3.0
    x = x.to(R.TORCH[dtype])
    for tile in (1, 128):
        s, st = _pack(lib, x, tile, True)
        val = _check_store(s, x, tile)
        _check_store(st, x.t().contiguous(), tile)
        back = torch.empty(9, 256, dtype=x.dtype, device="cuda")
        lib.orbit_fp8_unpack(R.CODE[dtype], 9, 256, s, back, 256)
        np.testing.assert_array_equal(back.double().cpu().numpy(), val)


def test_every_code_reads_back(lib):
    """All 256 codes at the smallest, a middle and the largest E."""
    wide, groups, at, size = F.layout(3, 256)
    b = np.zeros(size, np.uint8)
    b[:768] = np.tile(np.arange(256, dtype=np.uint8), 3)
    b[at:at + 12].reshape(3, 4)[:, :2] = [[10, 10], [127, 127], [246, 246]]
    for dtype in ("f32", "bf16"):
        back = torch.empty(3, 256, dtype=R.TORCH[dtype], device="cuda")
        lib.orbit_fp8_unpack(R.CODE[dtype], 3, 256, torch.from_numpy(b).cuda(), back, 256)
        v = np.append(F.e4m3_values(), np.nan)
        v = np.concatenate([v, -v])
        for i, e in enumerate((10, 127, 246)):
            np.testing.assert_array_equal(back[i].double().cpu().numpy(), v * 2.0 ** (e - 127))


# ---------------------------------------------------------------------------
# the product
# ---------------------------------------------------------------------------
def _slices(a, b, k0):
    """Per (m, n): the sum over steps of k0 of the largest |a b| of the step."""
    K = a.shape[1]
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64)
    for k in range(0, K, k0):
        out += (a[:, None, k:k + k0] * b[None, :, k:k + k0]).abs().amax(-1)
    return out


def _bound(a, b, ref, exact, dtype):
    """float32 results: every addition rounds a partial sum of at most sum |a b| by half a step. bf16 results: the
    instruction keeps the bits of a product down to 2^-13 of the largest of its step (of 64, or 128 of thin
    products, taken as 128 here), so each of the 128 loses less than that; the result is rounded once more."""
    K = a.shape[1]
    s = a.abs() @ b.abs().t()
    err = (K + 24) * F.U32 * s
    if not exact:
        err = err + 128 * 2.0 ** -13 * _slices(a, b, 128) + F.HALF["bf16"] * (ref.abs() + err)
    return err


GEMMS = [(1, 8, 8), (1, 128, 128), (7, 136, 1000), (16, 4096, 1024), (17, 40, 130), (33, 264, 2056), (64, 512, 300),
         (65, 8, 64), (100, 200, 129), (128, 128, 128), (150, 768, 1000), (257, 520, 513), (300, 1000, 2056),
         (515, 264, 4100), (40, 16, 20000), (130, 136, 9000)]


@pytest.mark.parametrize("form", ["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("M,N,K", GEMMS)
def test_gemm(lib, M, N, K, form):
    dtype = form.split("-")[0]
    exact = form != "bf16"
    x, w = _data(M, K, dtype, M + K, spread=3.0), _data(N, K, dtype, N + K)
    bias = _data(1, N, dtype, 5)[0]
    a, _ = _pack(lib, x)
    b, _ = _pack(lib, w, 128)
    va, vb = F.values(x.double()), F.values(w.double(), 128)
    ref = va @ vb.t()
    out_t = torch.float32 if exact else torch.bfloat16
    code = R.CODE[dtype]
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    ldc = N + 8
    C = torch.full((M, ldc), 3.0, dtype=out_t, device="cuda")
    lib.orbit_fp8_gemm(code, M, N, K, a, b, C, ldc, int(exact), None, 0, ws)
    err = (C[:, :N].double().cpu() - ref).abs()
    bound = _bound(va, vb, ref, exact, dtype)
    assert (err <= bound).all(), float((err / bound.clamp(min=1e-300)).max())
    assert (C[:, N:] == 3.0).all()
    # with a bias, onto what was there (float32), the same bits whatever the workspace held
    D = torch.full((M, ldc), 3.0, dtype=out_t, device="cuda")
    ws.fill_(0)
    lib.orbit_fp8_gemm(code, M, N, K, a, b, D, ldc, int(exact), bias.cuda(), int(exact), ws)
    ref2 = ref + bias.double() + (3.0 if exact else 0.0)
    err = (D[:, :N].double().cpu() - ref2).abs()
    bound = bound + 4 * F.U32 * (ref.abs() + bias.double().abs() + 3) + (0 if exact else F.HALF["bf16"] * ref2.abs())
    assert (err <= bound).all()
    E = torch.full((M, ldc), 3.0, dtype=out_t, device="cuda")
    lib.orbit_fp8_gemm(code, M, N, K, a, b, E, ldc, int(exact), bias.cuda(), int(exact), ws)
    assert torch.equal(D, E)


@pytest.mark.parametrize("form", ["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("M,N,K", [(16, 264, 1024), (16, 136, 4200), (24, 4104, 260), (30, 72, 2048), (30, 72, 2049), (32, 4096, 130),
                                   (9, 8200, 512), (3, 1032, 9000), (700, 1400, 520), (1030, 1032, 513), (2000, 4200, 300), (130, 72, 260)])
def test_gemm_kernels(lib, M, N, K, form):
    """As above, at the sizes where one kernel, tile or number of parts gives way to another."""
    test_gemm(lib, M, N, K, form)


@pytest.mark.parametrize("M", [5, 200])
def test_gemm_keeps_small_products(lib, M):
    """float32 results keep what a float32 sum can hold of a product beside a far larger one, at every place of a
    step of 128 (the 8-bit instruction alone drops what is 2^-14 of it)."""
    K, N = 256, 128
    x, w = torch.zeros(M, K), torch.zeros(N, K)
    x[:, 0], w[:, 0] = 256.0, 256.0
    for n in range(1, N):
        w[n, n] = 2.0 ** -4
    x[:, 1:N] = 2.0 ** -3
    a, _ = _pack(lib, x)
    b, _ = _pack(lib, w)
    C = torch.empty(M, N, device="cuda")
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    lib.orbit_fp8_gemm(0, M, N, K, a, b, C, N, 1, None, 0, ws)
    ref = F.values(x.double()) @ F.values(w.double()).t()
    assert ref[0, 5] == 65536 + 2.0 ** -7 and torch.equal(C.double().cpu(), ref)


@pytest.mark.parametrize("M,dtype", [(3, "bf16"), (3, "f32"), (140, "bf16"), (140, "f32"), (300, "bf16")])
def test_gemm_non_finite(lib, M, dtype):
    """A NaN or an infinity of an operand reaches its row (column) of the result and nothing else; far scales."""
    N, K = 264, 300
    x, w = _data(M, K, dtype, 1), _data(N, K, dtype, 2)
    x[1, 290], w[70, 5] = float("inf"), float("nan")
    a, _ = _pack(lib, x)
    b, _ = _pack(lib, w, 128)
    C = torch.empty(M, N, dtype=x.dtype, device="cuda")
    lib.orbit_fp8_gemm(R.CODE[dtype], M, N, K, a, b, C, N, 0, None, 0, _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K)))
    bad = torch.isnan(C).cpu()
    want = torch.zeros(M, N, dtype=torch.bool)
    want[1], want[:, 70] = True, True
    assert torch.equal(bad, want)
    # scales at the ends of E's range meet in the middle
    x2, w2 = (_data(M, K, "f32", 3) * 2.0 ** 100).to(x.dtype), (_data(N, K, "f32", 4) * 2.0 ** -100).to(x.dtype)
    a, _ = _pack(lib, x2)
    b, _ = _pack(lib, w2, 128)
    lib.orbit_fp8_gemm(R.CODE[dtype], M, N, K, a, b, C, N, 0, None, 0, _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K)))
    va, vb = F.values(x2.double()), F.values(w2.double(), 128)
    ref = va @ vb.t()
    assert ((C.double().cpu() - ref).abs() <= _bound(va, vb, ref, dtype == "f32", dtype)).all()


# ---------------------------------------------------------------------------
# the linear layer
# ---------------------------------------------------------------------------
LINEARS = [("bf16", 1, 64, 8), ("f32", 3, 136, 40), ("bf16", 150, 1000, 264), ("f32", 70, 256, 520), ("bf16", 300, 520, 1000),
           ("f32", 129, 8, 136)]


class _Linear:
    def __init__(self, lib, dtype, rows, i, o, pad=0, seed=0):
        self.lib, self.code, self.pad = lib, R.CODE[dtype], pad
        self.x, self.dy = _data(rows, i, dtype, seed + 1, 2.0), _data(rows, o, dtype, seed + 2, 2.0)
        self.w, self.b = (_data(i, o, dtype, seed + 3) * 0.1).to(R.TORCH[dtype]), _data(1, o, dtype, seed + 4)[0]
        self.rows, self.i, self.o = rows, i, o
        self.desc = Fp8LinearDesc(rows, i, o, self.code)
        dt = R.TORCH[dtype]
        wide = lambda t: torch.nn.functional.pad(t, (0, pad), value=9.0).cuda()
        self.gx, self.gdy, self.gb = wide(self.x), wide(self.dy), self.b.cuda()
        self.ws_, self.wt = _pack(lib, self.w, 128, True)
        self.y = torch.full((rows, o + pad), 5.0, dtype=dt, device="cuda")
        self.dx = torch.full((rows, i + pad), 5.0, dtype=dt, device="cuda")
        self.dw, self.db = torch.full((i, o), 5.0, device="cuda"), torch.full((o,), 5.0, device="cuda")
        self.saved = _bytes(lib.orbit_fp8_linear_saved_bytes(self.desc))
        self.ws = _bytes(lib.orbit_fp8_linear_workspace_bytes(self.desc))

    def fwd(self, saved=True, bias=True):
        p = self.pad
        self.lib.orbit_fp8_linear_fwd(self.desc, self.gx, self.i + p, self.wt, self.gb if bias else None, self.y, self.o + p,
                                      self.saved if saved else None, self.ws)

    def bwd(self, accumulate=0, dx=True, db=True):
        p = self.pad
        self.lib.orbit_fp8_linear_bwd(self.desc, self.saved, self.ws_ if dx else None, self.gdy, self.o + p,
                                      self.dx if dx else None, self.i + p, self.dw, self.db if db else None, accumulate, self.ws)


@pytest.mark.parametrize("dtype,rows,i,o", LINEARS)
def test_linear(lib, dtype, rows, i, o):
    t = _Linear(lib, dtype, rows, i, o, pad=8)
    t.fwd()
    t.ws.fill_(0x3C)
    t.bwd()
    d = lambda v: v.double().cpu()
    x, dy, w, b = d(t.x), d(t.dy), d(t.w), d(t.b)
    qx, qw, qdy = F.values(x), F.values(w, 128), F.values(dy)
    qxt, qdyt = F.values(x.t().contiguous()), F.values(dy.t().contiguous())
    ex = dtype == "f32"
    y = qx @ qw
    err = (d(t.y)[:, :o] - y - b).abs()
    bound = _bound(qx, qw.t(), y, ex, dtype) + 4 * F.U32 * (y.abs() + b.abs()) + (0 if ex else F.HALF["bf16"] * (y + b).abs())
    assert (err <= bound).all()
    dx = qdy @ qw.t()
    assert ((d(t.dx)[:, :i] - dx).abs() <= _bound(qdy, qw, dx, ex, dtype)).all()
    dw = qxt @ qdyt.t()
    assert ((d(t.dw) - dw).abs() <= _bound(qxt, qdyt, dw, True, dtype)).all()
    assert ((d(t.db) - dy.sum(0)).abs() <= (rows + 4) * F.U32 * dy.abs().sum(0)).all()
    assert (t.y[:, o:] == 5.0).all() and (t.dx[:, i:] == 5.0).all()
    # the reference's own gradients are these (its autograd function)
    xr, wr, br = (v.clone().requires_grad_(True) for v in (x, w, b))
    F.Fp8Linear.apply(xr, wr, br).backward(dy)
    assert torch.equal(xr.grad, dx) and torch.equal(wr.grad, dw)
    # inference: the same y; without dx and db: the same dw; accumulated on what is there
    y0, dx0, dw0, db0 = t.y.clone(), t.dx.clone(), t.dw.clone(), t.db.clone()
    t.fwd(saved=False)
    t.bwd(dx=False, db=False)
    assert torch.equal(t.y, y0) and torch.equal(t.dw, dw0) and torch.equal(t.db, db0)
    t.bwd(accumulate=1)
    assert ((t.dw - 2 * dw0).abs() <= 2 * F.U32 * (2 * dw0).abs()).all() and torch.equal(t.dx, dx0)
    assert ((t.db - 2 * db0).abs() <= 2 * F.U32 * (2 * db0).abs()).all()
    t.fwd(bias=False)
    assert ((d(t.y)[:, :o] - y).abs() <= _bound(qx, qw.t(), y, ex, dtype)).all()


def test_linear_graph_and_streams(lib):
    """Two layers on two streams at once, and captured into graphs that are replayed with eager work between."""
    a, b = _Linear(lib, "bf16", 260, 520, 264), _Linear(lib, "bf16", 70, 1000, 136, seed=9)
    outs = lambda t: [t.y, t.dx, t.dw, t.db]
    want = []
    for t in (a, b):
        t.fwd()
        t.bwd()
        want += [o.clone() for o in outs(t)]
    torch.cuda.synchronize()
    for o in outs(a) + outs(b):
        o.zero_()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s, t in ((s1, a), (s2, b)):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            t.fwd()
            t.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs(a) + outs(b), want))
    graphs = []
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.fwd()
            t.bwd()
        graphs.append(g)
    gen = torch.Generator().manual_seed(4)
    for _ in range(3):
        for g, t in zip(graphs, (a, b)):
            t.gx.copy_(torch.randn(t.gx.shape, generator=gen).to(t.gx.dtype))
            g.replay()
            torch.cuda.synchronize()
            got = [o.clone() for o in outs(t)]
            t.fwd()
            t.bwd()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, outs(t)))


@pytest.mark.parametrize("M,N,K", [(4096, 2056, 4104), (3500, 3336, 64), (3500, 3336, 129), (3500, 3336, 700), (3500, 3336, 1030),
                                   (2000, 8200, 2056)])
def test_full_size(lib, M, N, K):
    """Products of many tiles, of every length of the pipeline's start and end, against float64 on the device."""
    ld = -(-K // 8) * 8
    x, w = (torch.nn.functional.pad(_data(r, K, "bf16", i), (0, ld - K)).cuda() for i, r in ((1, M), (2, N)))
    a, b = _bytes(lib.orbit_fp8_bytes(M, K)), _bytes(lib.orbit_fp8_bytes(N, K))
    lib.orbit_fp8_pack(1, M, K, 1, x, ld, a)
    lib.orbit_fp8_pack(1, N, K, 128, w, ld, b)
    va, vb = torch.zeros(M, ld, device="cuda"), torch.zeros(N, ld, device="cuda")
    lib.orbit_fp8_unpack(0, M, K, a, va, ld)
    lib.orbit_fp8_unpack(0, N, K, b, vb, ld)
    ref = va.double() @ vb.double().t()
    s = va.abs().double() @ vb.abs().double().t()
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    C = torch.empty(M, N, device="cuda")
    lib.orbit_fp8_gemm(1, M, N, K, a, b, C, N, 1, None, 0, ws)
    assert ((C.double() - ref).abs() <= (K + 24) * F.U32 * s).all()
    # errors of independent roundings: far below that
    assert float((C.double() - ref).norm() / ref.norm()) < 4 * F.U32 * max(1.0, K / 16) ** 0.5
    H = torch.full((M, N + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    bias = _data(1, N, "bf16", 3).cuda()
    lib.orbit_fp8_gemm(1, M, N, K, a, b, H, N + 8, 0, bias, 0, ws)
    assert (H[:, N:] == 3.0).all()
    H, ref = H[:, :N].double(), ref + bias.double()
    assert float((H - ref).norm() / ref.norm()) < F.HALF["bf16"]
    # the largest product of a step is at most va.max vb.max: each of K loses less than 2^-13 of it
    lost = K * 2.0 ** -13 * va.abs().amax(1, keepdim=True).double() * vb.abs().amax(1).double()
    assert ((H - ref).abs() <= lost + F.HALF["bf16"] * ref.abs() * 1.01).all()


def test_beyond_32_bits(lib):
    """Codes, input and results whose offsets pass 2^31 and 2^32 bytes."""
    M, N, K, ld, ldc = 530000, 16, 4100, 4104, 4104
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(M, ld, dtype=torch.bfloat16, device="cuda", generator=g)
    w = torch.randn(N, ld, dtype=torch.bfloat16, device="cuda", generator=g)
    a, b = _bytes(lib.orbit_fp8_bytes(M, K)), _bytes(lib.orbit_fp8_bytes(N, K))
    lib.orbit_fp8_pack(1, M, K, 1, x, ld, a)
    lib.orbit_fp8_pack(1, N, K, 1, w, ld, b)
    back = torch.empty_like(x)
    lib.orbit_fp8_unpack(1, M, K, a, back, ld)
    sel = torch.cat([torch.arange(5), torch.arange(M // 2 - 130, M // 2 + 130), torch.arange(M - 300, M)]).cuda()
    va, vx = back[sel, :K].double(), x[sel, :K].double()
    assert ((va - vx).abs() <= 2.0 ** -4 * vx.abs() + 2.0 ** -10 * vx.abs().amax(1, keepdim=True) / 128).all()
    vb = F.values(w[:, :K].double().cpu()).cuda()
    ref, s = va @ vb.t(), va.abs() @ vb.abs().t()
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    del x, back
    C = torch.zeros(M, ldc, dtype=torch.bfloat16, device="cuda")
    lib.orbit_fp8_gemm(1, M, N, K, a, b, C, ldc, 0, None, 0, ws)
    lost = 64 * 2.0 ** -13 * va.abs().amax(1, keepdim=True) * vb.abs().amax(1) * -(-K // 64)
    assert ((C[sel, :N].double() - ref).abs() <= lost + F.HALF["bf16"] * ref.abs() * 1.01).all()
    assert float((C[sel, :N].double() - ref).norm() / ref.norm()) < F.HALF["bf16"]
    assert not C[sel, N:].any()
    del C
    D = torch.zeros(M, 2056, device="cuda")
    lib.orbit_fp8_gemm(1, M, N, K, a, b, D, 2056, 1, None, 0, ws)
    assert ((D[sel, :N].double() - ref).abs() <= (K + 24) * F.U32 * s).all() and not D[sel, N:].any()


def test_products_on_two_streams(lib):
    """The same stores read by products of every kernel that run side by side, each with its own workspace."""
    N, K = 3336, 1100
    cases = [(4096, 0), (4096, 1), (600, 0), (100, 1), (20, 0), (3, 1)]
    b, _ = _pack(lib, _data(N, K, "bf16", 2))
    runs = []
    for M, f32 in cases:
        a, _ = _pack(lib, _data(M, K, "bf16", M))
        runs.append((M, f32, a, [_bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K)) for _ in range(3)],
                     [torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda") for _ in range(3)]))
    call = lambda r, i, s: lib.orbit_fp8_gemm(1, r[0], N, K, r[2], b, r[4][i], N, r[1], None, 0, r[3][i], s)
    for r in runs:
        call(r, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i, s in enumerate(streams):
            for r in runs if i else runs[::-1]:
                call(r, i + 1, s)
    torch.cuda.synchronize()
    for r in runs:
        assert torch.equal(r[4][0], r[4][1]) and torch.equal(r[4][0], r[4][2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_full_size_float32_results(lib, dtype):
    """Products of many tiles with a bias, onto what was there, with gaps between rows; a NaN stays in its row and an
    infinity's in its column, bit for bit."""
    M, N, K, ldc = 2950, 2840, 700, 2856
    code = R.CODE[dtype]
    x, w = _data(M, K, dtype, 1), _data(N, K, dtype, 2)
    bias, c0 = _data(1, N, dtype, 3), _data(M, ldc, "f32", 4)
    va, vb = F.values(x.double()).cuda(), F.values(w.double()).cuda()
    ref, s = va @ vb.t(), va.abs() @ vb.abs().t()
    ref, s = ref + bias.double().cuda() + c0[:, :N].double().cuda(), s + bias.abs().double().cuda() + c0[:, :N].abs().double().cuda()
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    out = []
    for spoil in (False, True):
        if spoil:
            x[1234, 5], w[2000, 7] = float("nan"), float("inf")
        (a, _), (b, _) = _pack(lib, x), _pack(lib, w)
        C = c0.cuda()
        lib.orbit_fp8_gemm(code, M, N, K, a, b, C, ldc, 1, bias.cuda(), 1, ws)
        assert torch.equal(C[:, N:].cpu(), c0[:, N:])
        out.append(C[:, :N])
    clean, spoilt = out
    assert ((clean.double() - ref).abs() <= (K + 32) * F.U32 * s).all()
    hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    hit[1234], hit[:, 2000] = True, True
    assert torch.isnan(spoilt[hit]).all() and torch.equal(spoilt[~hit], clean[~hit])


def test_full_size_non_finite(lib):
    """The same for bf16 results."""
    M, N, K = 2950, 2840, 260
    x, w = _data(M, K, "bf16", 1), _data(N, K, "bf16", 2)
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    out = []
    for spoil in (False, True):
        if spoil:
            x[2949, 5], w[0, 259] = float("-inf"), float("nan")
        (a, _), (b, _) = _pack(lib, x), _pack(lib, w)
        C = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        lib.orbit_fp8_gemm(1, M, N, K, a, b, C, N, 0, None, 0, ws)
        out.append(C)
    hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    hit[2949], hit[:, 0] = True, True
    assert torch.isnan(out[1][hit]).all() and torch.equal(out[1][~hit], out[0][~hit]) and torch.isfinite(out[0]).all()


@pytest.mark.parametrize("f32", [0, 1])
def test_rows_of_results_far_apart(lib, f32):
    """130 x 33000, wide enough for the large tiles, whole and with rows 2^24 apart, where offsets pass 31 bits."""
    M, N, K, ldc = 130, 33000, 300, 1 << 24
    (a, _), (b, _) = _pack(lib, _data(M, K, "bf16", 1)), _pack(lib, _data(N, K, "bf16", 2))
    t = torch.float32 if f32 else torch.bfloat16
    ws = _bytes(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
    C, D = torch.empty(M, N, dtype=t, device="cuda"), torch.zeros(M, ldc, dtype=t, device="cuda")
    lib.orbit_fp8_gemm(1, M, N, K, a, b, C, N, f32, None, 0, ws)
    lib.orbit_fp8_gemm(1, M, N, K, a, b, D, ldc, f32, None, 0, ws)
    va, vb = torch.zeros(M, 304, device="cuda"), torch.zeros(N, 304, device="cuda")
    lib.orbit_fp8_unpack(0, M, K, a, va, 304)
    lib.orbit_fp8_unpack(0, N, K, b, vb, 304)
    ref = va.double() @ vb.double().t()
    bound = 2.0 ** -22 if f32 else F.HALF["bf16"]
    for R_ in (C, D[:, :N]):
        assert float((R_.double() - ref).norm() / ref.norm()) < bound
    assert not D[:, N:].any()
