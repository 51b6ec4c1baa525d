"""The 8-bit activation store on the GPU against its 64-bit definition: codes,
steps and values bit for bit, GELU and weight gradients within float32 rounding."""
import numpy as np
import pytest
import torch

import ops_ref as R

pytestmark = pytest.mark.gpu
DT = ["bf16", "f32"]


def _matrix(rows, n, dtype, seed=0):
    """Rows of sizes from 2^-140 to 2^120, a zero row, and values at the rounding's borders."""
    r = np.random.default_rng([seed, rows, n])
    x = r.standard_normal((rows, n)) * np.exp2(r.integers(-6, 7, (rows, 1)))
    k = np.arange(rows)
    x[k % 7 == 3] *= 2.0 ** -60
    x[k % 11 == 5] *= 2.0 ** 110
    x[k % 13 == 6] *= 2.0 ** -130           # float32 subnormals
    x[k % 17 == 8] = 0.0
    x[k % 5 == 2, :8] = [1.0, 127.5 / 64, 0.5 / 64, 1.5 / 64, -2.5 / 64, 63.5 / 64, -1.0, -127.5 / 64]
    return torch.from_numpy(x.astype(np.float32)).to(R.TORCH[dtype])


def _packed(lib, x, ld=None, dtype="bf16"):
    rows, n = x.shape
    ld = ld or n
    buf = torch.full((rows, ld), 7.0, dtype=x.dtype, device="cuda")
    buf[:, :n] = x.cuda()
    nb = lib.orbit_act8_bytes(rows, n)
    store = torch.full((nb + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    lib.orbit_act8_pack(R.CODE[dtype], rows, n, buf, ld, store[:nb])
    return store[:nb], store


SHAPES = [(1, 8), (1, 24), (3, 40), (1, 1024), (5, 32), (257, 1000), (64, 2056), (2, 16384), (70000, 8), (513, 640)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("pad", [0, 24])
def test_pack_unpack_bitwise(lib, rows, n, pad, dtype):
    x = _matrix(rows, n, dtype)
    store, whole = _packed(lib, x, n + pad, dtype)
    codes, E, val = R.act8_ref(x.double().numpy())
    at, groups, nb = R.store_layout(rows, n)
    got = whole.cpu().numpy()
    np.testing.assert_array_equal(got[:rows * n].view(np.int8).reshape(rows, n), codes)
    np.testing.assert_array_equal(got[at:at + rows * groups].reshape(rows, groups), E)
    assert (got[rows * n:at] == 0x5A).all() and (got[at + rows * groups:] == 0x5A).all()
    out = torch.full((rows + 2, n + pad), 3.0, dtype=R.TORCH[dtype], device="cuda")
    lib.orbit_act8_unpack(R.CODE[dtype], rows, n, store, out, n + pad)
    o = out.cpu().double().numpy()
    np.testing.assert_array_equal(o[:rows, :n], val)
    assert (o[rows:] == 3.0).all() and (o[:, n:] == 3.0).all()


@pytest.mark.parametrize("dtype", DT)
def test_extremes_and_non_finite(lib, dtype):
    big = torch.finfo(R.TORCH[dtype]).max
    x = torch.randn(10, 72, dtype=torch.float64, generator=torch.Generator().manual_seed(1)).float()
    x[1, 5] = float("inf")
    x[2, 40] = float("nan")
    x[3, 71] = -float("inf")
    x[4, 0], x[4, 1] = big, -big            # the type's largest and lowest value
    x[5, :] = torch.finfo(torch.float32).tiny
    x[6, :] = 2.0 ** -149
    x[7, 33] = -float("nan")
    x = x.to(R.TORCH[dtype])
    store, _ = _packed(lib, x, dtype=dtype)
    _, _, val = R.act8_ref(x.double().numpy())
    u, g = (torch.empty(10, 72, dtype=R.TORCH[dtype], device="cuda") for _ in range(2))
    lib.orbit_act8_unpack(R.CODE[dtype], 10, 72, store, u, 72, g, 72)
    got = u.cpu().double().numpy()
    np.testing.assert_array_equal(got, val)
    assert np.isnan(got[1, :32]).all() and np.isnan(got[2, 32:64]).all() and np.isnan(got[3, 64:]).all()
    assert np.isfinite(got[4]).all() and np.isfinite(got[1, 32:]).all()
    np.testing.assert_array_equal(np.isnan(g.cpu().float().numpy()), np.isnan(val))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,n,pad,with_u", [(1, 8, 0, True), (33, 1000, 8, True), (300, 4096, 0, False), (7, 40, 0, False)])
def test_unpack_gelu(lib, rows, n, pad, with_u, dtype):
    x = torch.randn(rows, n, generator=torch.Generator().manual_seed(rows)).mul_(3.0).to(R.TORCH[dtype])
    store, _ = _packed(lib, x, dtype=dtype)
    _, _, val = R.act8_ref(x.double().numpy())
    u = torch.empty(rows, n + pad, dtype=R.TORCH[dtype], device="cuda") if with_u else None
    g = torch.empty(rows, n + pad, dtype=R.TORCH[dtype], device="cuda")
    lib.orbit_act8_unpack(R.CODE[dtype], rows, n, store, u, n + pad, g, n + pad)
    if with_u:
        np.testing.assert_array_equal(u[:, :n].cpu().double().numpy(), val)
    val = torch.from_numpy(val)
    ref = R.gelu_ref(val)
    # u/2 (1 + erf): erf off by 1.5e-7 and 8 roundings of float32; then the storage type's rounding
    tol = R.HALF[dtype] * ref.abs() + val.abs() * (0.75e-7 + 8 * R.U32)
    err = (g[:, :n].cpu().double() - ref).abs()
    assert (err <= tol).all(), float((err - tol).max())


def test_unpack_two_leading_dimensions(lib):
    """x without gaps beside a GELU with them, and the other way round."""
    rows, n = 19, 96
    x = torch.randn(rows, n, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    store, _ = _packed(lib, x)
    ref = torch.empty(2, rows, n, dtype=torch.bfloat16, device="cuda")
    lib.orbit_act8_unpack(1, rows, n, store, ref[0], n, ref[1], n)
    for lx, lg in ((n, n + 40), (n + 8, n)):
        u = torch.full((rows, lx), 4.0, dtype=torch.bfloat16, device="cuda")
        g = torch.full((rows, lg), 4.0, dtype=torch.bfloat16, device="cuda")
        lib.orbit_act8_unpack(1, rows, n, store, u, lx, g, lg)
        assert torch.equal(u[:, :n], ref[0]) and torch.equal(g[:, :n], ref[1])
        assert bool((u[:, n:] == 4).all()) and bool((g[:, n:] == 4).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,K,N", [(1, 8, 8), (1, 64, 40), (31, 40, 200), (100, 1000, 72), (513, 256, 1024), (2048, 520, 136)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_weight_grad(lib, rows, K, N, accumulate, dtype):
    g = torch.Generator().manual_seed(rows + K)
    x = torch.randn(rows, K, generator=g).to(R.TORCH[dtype])
    ld = N + 16
    dy = torch.randn(rows, ld, generator=g).to(R.TORCH[dtype])
    store, _ = _packed(lib, x, dtype=dtype)
    _, _, val = R.act8_ref(x.double().numpy())
    val, d = torch.from_numpy(val), dy[:, :N].double()
    dw0, db0 = torch.randn(K, N, generator=g), torch.randn(N, generator=g)
    dw, db = dw0.cuda(), db0.cuda()
    nb = lib.orbit_act8_weight_grad_workspace_bytes(R.CODE[dtype], rows, K, N)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    lib.orbit_act8_weight_grad(R.CODE[dtype], rows, K, N, store, dy.cuda(), ld, dw, db, accumulate, ws)
    ref_w = val.t() @ d + (dw0.double() if accumulate else 0)
    ref_b = d.sum(0) + (db0.double() if accumulate else 0)
    # one float32 rounding per addition, in any order, and a few per product (float32
    # operands are split into bf16 parts: 6 partial products)
    S = (rows + 16) * R.U32
    tol_w = S * (val.abs().t() @ d.abs()) + R.U32 * 4 * ref_w.abs()
    tol_b = S * d.abs().sum(0) + R.U32 * 4 * ref_b.abs()
    assert ((dw.cpu().double() - ref_w).abs() <= tol_w).all()
    assert ((db.cpu().double() - ref_b).abs() <= tol_b).all()
    # without a bias gradient, and bitwise the same
    again = dw0.cuda()
    lib.orbit_act8_weight_grad(R.CODE[dtype], rows, K, N, store, dy.cuda(), ld, again, None, accumulate, ws)
    assert torch.equal(again, dw) or ((again - dw).abs().cpu().double() <= 2 * tol_w).all()


@pytest.mark.parametrize("n", [32768, 32776])
def test_far_offsets(lib, n):
    """A store past 2^31 bytes, its values past 2^32: the last rows read back as they were."""
    rows = 70000
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, n, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
    x[0] = 1.0
    store = torch.empty(lib.orbit_act8_bytes(rows, n), dtype=torch.uint8, device="cuda")
    lib.orbit_act8_pack(1, rows, n, x, n, store)
    out = torch.full((rows, n), 9.0, dtype=torch.bfloat16, device="cuda")
    lib.orbit_act8_unpack(1, rows, n, store, out, n)
    _, _, val = R.act8_ref(x[-3:].double().cpu().numpy())
    np.testing.assert_array_equal(out[-3:].double().cpu().numpy(), val)
    assert bool((out[0] == 1.0).all()) and not bool(out[1:-3].any())


def test_rows_far_apart(lib):
    """Rows of a few columns 2^30 bytes apart: offsets of a block's rows pass 31 bits."""
    rows, n, ld = 4, 40, 1 << 29
    x = torch.zeros((rows - 1) * ld + n, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(rows, n, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    for r in range(rows):
        x[r * ld:r * ld + n] = v[r].cuda()
    store = torch.empty(lib.orbit_act8_bytes(rows, n), dtype=torch.uint8, device="cuda")
    lib.orbit_act8_pack(1, rows, n, x, ld, store)
    _, _, val = R.act8_ref(v.double().numpy())
    x.zero_()
    lib.orbit_act8_unpack(1, rows, n, store, x, ld)
    for r in range(rows):
        np.testing.assert_array_equal(x[r * ld:r * ld + n].cpu().double().numpy(), val[r])
        assert r + 1 == rows or not bool(x[r * ld + n:(r + 1) * ld].any())


def test_side_stream_and_graph(lib):
    """Pack, read back and the weight gradient on another stream and captured into a graph,
    replayed with eager work in between: every replay gives the eager result for its inputs."""
    rows, K, N = 300, 264, 512
    g = torch.Generator().manual_seed(4)
    x, dy = (torch.empty(rows, w, dtype=torch.bfloat16, device="cuda") for w in (K, N))
    store = torch.empty(lib.orbit_act8_bytes(rows, K), dtype=torch.uint8, device="cuda")
    u, ge = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.zeros(K, N, device="cuda"), torch.zeros(N, device="cuda")
    ws = torch.empty(lib.orbit_act8_weight_grad_workspace_bytes(1, rows, K, N), dtype=torch.uint8, device="cuda")

    def step():
        lib.orbit_act8_pack(1, rows, K, x, K, store)
        lib.orbit_act8_unpack(1, rows, K, store, u, K, ge, K)
        lib.orbit_act8_weight_grad(1, rows, K, N, store, dy, N, dw, db, 0, ws)

    def fresh():
        x.copy_(torch.randn(rows, K, generator=g).to(torch.bfloat16))
        dy.copy_(torch.randn(rows, N, generator=g).to(torch.bfloat16))

    fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    outs = (u, ge, dw, db, store)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        fresh()
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got[:4], outs[:4]):
            assert torch.equal(a, b)
