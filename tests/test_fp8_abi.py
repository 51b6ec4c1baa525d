"""Host-side checks of the 8-bit floating-point and rotary entry points: sizes, refusals, and
the 64-bit references the GPU tests compare with (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_ref as F
from paper_2404_14712_amd import _lib as L

BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    return L.OrbitLib()


@pytest.mark.parametrize("rows,n", [(1, 1), (1, 128), (3, 129), (257, 1000), (8192, 4096), (5, 513)])
def test_store_bytes(lib, rows, n):
    assert lib.orbit_fp8_bytes(rows, n) == F.layout(rows, n)[3]


def _refuses(lib, f, ok, bad, status=L.ORBIT_E_ARG):
    for what, (i, v) in bad:
        a = list(ok)
        a[i] = v
        assert f(*a) == status and what in lib.last_error(), (what, i, v, lib.last_error())


def test_pack_refusals(lib):
    assert lib.orbit_fp8_bytes(0, 8) == 0 and lib.orbit_fp8_bytes(8, -1) == 0
    assert lib.orbit_fp8_bytes(1 << 27, 128) == 0 and lib.orbit_fp8_bytes((1 << 27) - 1, 128) > 0
    assert lib.orbit_fp8_bytes(1 << 60, 1 << 60) == 0
    c = lib.lib
    ok = (1, 4, 40, 1, 0x100, 40, 0x200, BIG, 0x300, BIG, None)
    need, need_t = F.layout(4, 40)[3], F.layout(40, 4)[3]
    _refuses(lib, c.orbit_fp8_pack, ok, [
        ("dtype", (0, 7)), ("bad sizes", (1, 0)), ("bad sizes", (2, -3)), ("tile_rows", (3, 2)), ("x is NULL", (4, None)),
        ("16-byte", (4, 0x108)), ("ldx", (5, 32)), ("ldx", (5, 44)), ("store is not", (6, 0x204)), ("store of", (7, need - 1)),
        ("store_t of", (9, need_t - 1)), ("alias", (8, 0x200)), ("alias", (6, 0x100)), ("alias", (8, 0x100))])
    assert c.orbit_fp8_pack(1, 4, 40, 1, 0x100, 40, None, 0, None, 0, None) == L.ORBIT_E_ARG and "both" in lib.last_error()
    assert c.orbit_fp8_pack(1, 1 << 27, 128, 1, 0x100, 128, 0x200, BIG, None, 0, None) == L.ORBIT_E_UNSUPPORTED
    # a transposed store pads the rows of X to 128
    assert c.orbit_fp8_pack(1, 16, 1 << 29, 1, 0x100, 1 << 29, None, 0, 0x200, BIG, None) == L.ORBIT_E_UNSUPPORTED
    assert c.orbit_fp8_pack(1, 7, 1 << 31, 1, 0x100, 1 << 31, 0x200, BIG, None, 0, None) == L.ORBIT_E_UNSUPPORTED
    assert "2^24 tiles" in lib.last_error()
    un = (1, 4, 40, 0x100, BIG, 0x200, 40, None)
    _refuses(lib, c.orbit_fp8_unpack, un, [
        ("dtype", (0, 2)), ("bad sizes", (1, -1)), ("bad sizes", (2, 0)), ("store is NULL", (3, None)),
        ("store of", (4, need - 1)), ("x is NULL", (5, None)), ("16-byte", (5, 0x202)), ("ldx", (6, 36)), ("alias", (5, 0x100))])


def test_gemm_refusals(lib):
    c = lib.lib
    a, b = F.layout(5, 100)[3], F.layout(16, 100)[3]
    ok = (1, 5, 16, 100, 0x1000, a, 0x2000, b, 0x3000, 16, 0, 0x4000, 0, 0x5000, BIG, None)
    _refuses(lib, c.orbit_fp8_gemm, ok, [
        ("dtype", (0, 3)), ("bad sizes", (1, 0)), ("bad sizes", (2, 12)), ("bad sizes", (3, 0)), ("A is NULL", (4, None)),
        ("A of", (5, a - 1)), ("B is not", (6, 0x2008)), ("B of", (7, b - 1)), ("C is NULL", (8, None)), ("ldc", (9, 8)),
        ("ldc", (9, 20)), ("c_f32", (10, 2)), ("bias is not", (11, 0x4001)), ("accumulate", (12, 2)),
        ("accumulate needs", (12, 1)), ("alias", (8, 0x1000)), ("alias", (13, 0x3000))])
    for i, v in ((3, 1 << 22), (2, 1 << 26)):
        x = list(ok)
        x[i] = v
        assert c.orbit_fp8_gemm(*x) == L.ORBIT_E_UNSUPPORTED
    assert lib.orbit_fp8_gemm_workspace_bytes(8192, 12, 128) == 0 and "multiple" in lib.last_error()
    # a product that splits K needs its workspace
    need = lib.orbit_fp8_gemm_workspace_bytes(128, 128, 1 << 16)
    assert need > 0
    big = (1, 128, 128, 1 << 16, 0x1000, BIG, 0x2000, BIG, 0x3000, 128, 0, None, 0, None, BIG, None)
    assert c.orbit_fp8_gemm(*big) == L.ORBIT_E_ARG and "workspace" in lib.last_error()
    assert c.orbit_fp8_gemm(*big[:13], 0x5000, need - 1, None) == L.ORBIT_E_ARG and "workspace" in lib.last_error()


def test_linear_refusals(lib):
    c, r = lib.lib, ctypes.byref
    for bad in ((0, 8, 8, 1), (4, 12, 8, 1), (4, 8, 20, 1), (4, 8, 8, 5)):
        d = L.Fp8LinearDesc(*bad)
        assert lib.orbit_fp8_linear_saved_bytes(d) == 0 and lib.orbit_fp8_linear_workspace_bytes(d) == 0
        assert c.orbit_fp8_linear_fwd(r(d), 0x100, 8, 0x200, BIG, None, 0x300, 8, None, 0x400, BIG, None) == L.ORBIT_E_ARG
    assert lib.orbit_fp8_linear_saved_bytes(L.Fp8LinearDesc(1 << 22, 8, 8, 1)) == 0
    d = L.Fp8LinearDesc(5, 16, 24, 1)
    assert lib.orbit_fp8_linear_saved_bytes(d) == F.layout(16, 5)[3]
    wt, w = F.layout(24, 16)[3], F.layout(16, 24)[3]
    fwd = (r(d), 0x100, 16, 0x200, wt, 0x300, 0x400, 24, 0x500, 0x600, BIG, None)
    _refuses(lib, c.orbit_fp8_linear_fwd, fwd, [
        ("x is NULL", (1, None)), ("ldx", (2, 8)), ("w_t is NULL", (3, None)), ("w_t of", (4, wt - 1)), ("bias is not", (5, 0x301)),
        ("y is NULL", (6, None)), ("ldy", (7, 20)), ("saved is not", (8, 0x501)), ("ws is NULL", (9, None)),
        ("workspace", (10, 16)), ("alias", (6, 0x100))])
    bwd = (r(d), 0x100, 0x200, w, 0x300, 24, 0x400, 16, 0x500, 0x600, 0, 0x700, BIG, None)
    _refuses(lib, c.orbit_fp8_linear_bwd, bwd, [
        ("saved is NULL", (1, None)), ("w is NULL", (2, None)), ("w of", (3, w - 1)), ("dy is NULL", (4, None)),
        ("lddy", (5, 16)), ("lddx", (7, 12)), ("dw is NULL", (8, None)), ("db is not", (9, 0x601)), ("accumulate", (10, -1)),
        ("ws is NULL", (11, None)), ("workspace", (12, 8)), ("alias", (6, 0x300))])


def _rope(**kw):
    v = dict(tokens=12, q_heads=4, k_heads=2, head_dim=64, dtype=1, axis=[0] * 16 + [1] * 16, axes=2, pos_rows=6)
    v.update(kw)
    return L.QkRopeDesc.of(**v)


def test_rope_refusals(lib):
    c, r = lib.lib, ctypes.byref
    p, g = L.QkRopeParams(0x10, 0x20, 0x30, 0x40), L.QkRopeGrads(0x50, 0x60, 0x70, 0x80)

    def fwd(d, p=p, pos=0x100, freq=0x200, src=0x300, lds=384, dst=0x400, ldd=384, mean=0x500, rstd=0x600):
        return c.orbit_qk_rope_fwd(r(d), r(p) if p else None, pos, freq, src, lds, dst, ldd, mean, rstd, None)

    def bwd(d, p=p, pos=0x100, freq=0x200, src=0x300, lds=384, mean=0x500, rstd=0x600, dy=0x700, lddy=384, dx=0x800,
            lddx=384, g=g, acc=0, ws=0x900, n=BIG):
        return c.orbit_qk_rope_bwd(r(d), r(p) if p else None, pos, freq, src, lds, mean, rstd, dy, lddy, dx, lddx,
                                   r(g) if g else None, acc, ws, n, None)

    for kw, what, st in ((dict(tokens=0), "positive", 1), (dict(k_heads=0), "positive", 1), (dict(head_dim=96), "head_dim", 2),
                         (dict(dtype=4), "dtype", 1), (dict(axes=0), "axes", 1), (dict(axes=5), "axes", 1),
                         (dict(axes=1), "axis[16]", 1), (dict(pos_rows=5), "pos_rows", 1), (dict(pos_rows=0), "pos_rows", 1),
                         (dict(eps=0.0), "eps", 1), (dict(norm=2), "norm", 1), (dict(near=3), "near", 1),
                         (dict(tokens=1 << 24, pos_rows=1), "too many", 2),
                         (dict(tokens=1 << 20, pos_rows=1, q_heads=1 << 20), "too many", 2)):
        d = _rope(**kw)
        assert fwd(d) == st and what in lib.last_error(), (kw, lib.last_error())
        assert bwd(d) == st and what in lib.last_error(), (kw, lib.last_error())
        assert lib.orbit_qk_rope_bwd_workspace_bytes(d) == 0
    d = _rope()
    for kw, what in ((dict(p=None), "params"), (dict(pos=None), "pos is NULL"), (dict(freq=0x202), "freq is not"),
                     (dict(src=None), "src"), (dict(dst=None), "dst"), (dict(lds=376), "leading"), (dict(ldd=388), "leading"),
                     (dict(dst=0x300, ldd=392), "dst may be src"), (dict(mean=None), "go together"),
                     (dict(p=L.QkRopeParams(0x10, 0x20, None, 0x40)), "kn_g"), (dict(p=L.QkRopeParams(0x10, 0, 0x30, 0x40)), "qn_b")):
        assert fwd(d, **kw) == 1 and what in lib.last_error(), (kw, lib.last_error())
    for kw, what in ((dict(p=None), "params"), (dict(src=None), "src"), (dict(mean=None), "mean"), (dict(rstd=0x601), "rstd"),
                     (dict(dy=None), "dy"), (dict(dx=None), "dx"), (dict(lddy=8), "leading"), (dict(lds=380), "leading"),
                     (dict(dx=0x700, lddx=392), "dx may be dy"), (dict(dx=0x300), "alias"), (dict(g=None), "grads"),
                     (dict(g=L.QkRopeGrads(0x50, 0x60, 0x70, None)), "grads.kn_b"), (dict(acc=2), "accumulate"),
                     (dict(ws=None), "ws"), (dict(n=64), "workspace")):
        assert bwd(d, **kw) == 1 and what in lib.last_error(), (kw, lib.last_error())
    assert lib.orbit_qk_rope_bwd_workspace_bytes(_rope(norm=False)) == 0
    with pytest.raises(ValueError):
        _rope(axis=[0] * 129)


def test_block_opt_refusals(lib):
    r = ctypes.byref
    d = L.BlockDesc(2, 6, 64, 2, 32, 64, 1, 1e-5, 1)
    none, act8 = L.BlockExt(0, 0, 0, 1.0), L.BlockExt(1, 0, 0, 1.0)
    rope = L.BlockRope.of([0] * 8 + [1] * 8, 2, 6, 0x100, 0x200)
    stores = {n: 0x1000 for n in L.BLOCK_FP8_STORES}
    q = lambda o, e=none: (lib.orbit_vit_block_opt_saved_bytes(d, e, o), lib.orbit_vit_block_opt_workspace_bytes(d, e, o))
    # with nothing asked for the sizes are the block's; stores of inputs are smaller than the inputs
    plain = q(L.BlockOpt.of())
    assert plain == (lib.orbit_vit_block_saved_bytes(d), lib.orbit_vit_block_workspace_bytes(d))
    wide = L.BlockDesc(2, 256, 512, 4, 64, 1024, 1, 1e-5, 1)
    opt8 = L.BlockOpt.of(fp8=stores)
    assert lib.orbit_vit_block_opt_saved_bytes(wide, none, opt8) < lib.orbit_vit_block_saved_bytes(wide)
    assert q(L.BlockOpt.of(rope)) [0] == plain[0]
    assert q(opt8, act8) == (0, 0) and "act8" in lib.last_error()
    assert q(L.BlockOpt.of(L.BlockRope.of([0] * 15 + [2], 2, 6, 0x100, 0x200))) == (0, 0) and "axis[15]" in lib.last_error()
    assert q(L.BlockOpt.of(L.BlockRope.of([0] * 16, 1, 5, 0x100, 0x200))) == (0, 0) and "pos_rows" in lib.last_error()

    def call(o, ws=1 << 40):
        p = L.BlockParams(*[0x4000 + 0x100 * i for i in range(16)])
        g = L.BlockGrads(*[0x8000 + 0x100 * i for i in range(16)])
        f = lib.lib.orbit_vit_block_opt_fwd(r(d), r(none), r(o) if o else None, r(p), None, 0x100, 0x200, 0x300, 0x400, ws, None)
        m = lib.last_error()
        b = lib.lib.orbit_vit_block_opt_bwd(r(d), r(none), r(o) if o else None, r(p), None, 0x100, 0x300, 0x200, 0x500, r(g),
                                            None, 0, 0x400, ws, None)
        return f, b, m + lib.last_error()

    for o, what in ((None, "opt is NULL"), (L.BlockOpt.of(L.BlockRope.of([0] * 16, 1, 6, None, 0x200)), "rope.pos"),
                    (L.BlockOpt.of(L.BlockRope.of([0] * 16, 1, 6, 0x100, 0x204)), "rope.freq"),
                    (L.BlockOpt.of(fp8=dict(stores, w_fc2_t=None)), "fp8.w_fc2_t")):
        f, b, m = call(o)
        assert f == b == L.ORBIT_E_ARG and m.count(what) == 2, (what, m)
    f, b, m = call(L.BlockOpt.of(rope, stores), 16)
    assert f == b == L.ORBIT_E_ARG and m.count("workspace") == 2


def test_store_reference_by_brute_force():
    """Each value is the nearest of those the scale offers; half the scale would not hold the block's largest."""
    r = np.random.default_rng(5)
    x = (r.standard_normal((40, 150)) * np.exp(r.uniform(-30, 30, (40, 1)))).astype(np.float32).astype(np.float64)
    x[0] = 0.0
    x[1, :128], x[2, :128] = 448.0 * 2.0 ** -9, np.nextafter(np.float32(448.0 * 2.0 ** -9), np.float32(1))
    code, E, val = F.pack_ref(x)
    grid = np.concatenate([-F.e4m3_values()[::-1], F.e4m3_values()])
    for i in range(len(x)):
        for b in range(2):
            t, s = x[i, 128 * b:128 * b + 128], 2.0 ** (int(E[i, b]) - 127)
            best = np.abs(t[:, None] - grid[None] * s).min(1)
            np.testing.assert_array_equal(np.abs(t - val[i, 128 * b:128 * b + 128]), best)
            assert np.abs(t).max() <= 448 * s and (E[i, b] == 10 or np.abs(t).max() > 224 * s)
    assert E[2, 0] == E[1, 0] + 1 == 119
    # tiles: one scale, and the transpose holds the same values
    _, Et, vt = F.pack_ref(x, 128)
    assert (Et == Et[0]).all()
    np.testing.assert_array_equal(F.pack_ref(x.T, 128)[2].T, vt)
    c, E, v = F.pack_ref(np.array([[np.inf, -np.inf, np.nan, 1.0, -0.0, 3.4e38]]))
    assert list(c[0, :3]) == [0x7F] * 3 and E[0, 0] == 246 and v[0, 5] == 448 * 2.0 ** 119 and c[0, 4] == 0x80


@pytest.mark.parametrize("near", [False, True])
def test_rope_reference_by_differences(near):
    """The reference's gradient against differences, and the turn against complex numbers."""
    g = torch.Generator().manual_seed(3)
    src = torch.randn(4, 3, 8, generator=g, dtype=torch.float64)
    p = {k: torch.randn(8, generator=g, dtype=torch.float64) for k in ("qn_g", "qn_b", "kn_g", "kn_b")}
    pos, freq, axis = torch.randn(2, 2, generator=g) * 3, torch.rand(4, generator=g), [0, 1, 1, 0]
    dy = torch.randn(4, 3, 8, generator=g, dtype=torch.float64)
    f = lambda s: (F.rope_ref(s, p, pos, freq, axis, near, 2, True) * dy).sum()
    s = src.clone().requires_grad_(True)
    f(s).backward()
    for i in (0, 17, 40, 95):
        e = torch.zeros(96, dtype=torch.float64)
        e[i] = 1e-6
        num = (f(src + e.reshape(src.shape)) - f(src - e.reshape(src.shape))) / 2e-6
        assert abs(float(num - s.grad.reshape(-1)[i])) < 1e-7
    t = F.turn(src, pos, freq, axis, near)
    for tok in range(4):
        for i in range(4):
            a, b = (2 * i, 2 * i + 1) if near else (i, i + 4)
            z = complex(src[tok, 1, a], src[tok, 1, b]) * np.exp(1j * float(pos[tok % 2, axis[i]].double() * freq[i].double()))
            assert abs(z - complex(t[tok, 1, a], t[tok, 1, b])) < 1e-12


def test_pass_refuses_positions_the_kernels_cannot_read(lib):
    """ViTPass hands positions and frequencies on as pointers to packed float32 on its device."""
    from paper_2404_14712_amd.model import PassDims, Rope, ViTPass
    z = PassDims(mode="blocks", dtype="f32", B=1, L=6, d=64, blocks=1, heads=2, head_dim=32, mlp=64)
    E = lambda *s: torch.zeros(*s)
    block = {"w_qkv": E(64, 192), "b_qkv": E(192), "w_proj": E(64, 64), "b_proj": E(64), "w_fc1": E(64, 64), "b_fc1": E(64),
             "w_fc2": E(64, 64), "b_fc2": E(64)}
    block.update({n + s: E(w) for n, w in (("ln1", 64), ("ln2", 64), ("qn", 32), ("kn", 32)) for s in ("_g", "_b")})
    make = lambda r: ViTPass(lib, z, {"blocks": [block]}, device="cpu", rope=r)
    pos, freq, axis = torch.rand(6, 2), torch.rand(16), [0] * 8 + [1] * 8
    p = make(Rope(pos, freq, axis))
    assert p.opts[0].rope.contents.pos == pos.data_ptr() and p.opts[0].rope.contents.freq == freq.data_ptr()
    for bad, what in ((Rope(pos.double(), freq, axis), "pos"), (Rope(pos.long(), freq, axis), "pos"),
                      (Rope(torch.rand(2, 6).t(), freq, axis), "pos"), (Rope(torch.rand(1, 2).expand(6, 2), freq, axis), "pos"),
                      (Rope(torch.rand(12), freq, axis), "pos"), (Rope(pos.to("meta"), freq, axis), "pos"),
                      (Rope(pos, freq.double(), axis), "freq"), (Rope(pos, torch.rand(32)[::2], axis), "freq"),
                      (Rope(pos, freq.to("meta"), axis), "freq"), (Rope(pos.numpy(), freq, axis), "pos")):
        with pytest.raises(ValueError, match="rope." + what):
            make(bad)
    for bad in (Rope(pos, freq, axis[:15]), Rope(pos, freq[:8], axis[:8])):
        with pytest.raises(ValueError, match="16 pairs"):
            make(bad)
    for bad, what in ((Rope(torch.rand(4, 2), freq, axis), "pos_rows"), (Rope(pos, freq, [2] * 16), "axis")):
        with pytest.raises(ValueError, match=what):
            make(bad)


def test_stores_of_2_24_tiles_are_refused(lib):
    """The limit of a store that pack can write holds wherever a store is named: its size, and reading it back (rows
    of 2^33 columns would be a launch of 2^32 threads)."""
    c = lib.lib
    for n in (1 << 31, (1 << 33) - 5, 1 << 33, (1 << 34) - 128):
        assert lib.orbit_fp8_bytes(1, n) == 0 and lib.orbit_fp8_bytes(1, (1 << 31) - 128) > 0
        assert c.orbit_fp8_unpack(1, 1, n, 0x100, BIG, 0x200, 1 << 34, None) == L.ORBIT_E_UNSUPPORTED
        assert "2^24 tiles" in lib.last_error()
        assert c.orbit_fp8_pack(1, 1, n, 1, 0x100, 1 << 34, 0x200, BIG, None, 0, None) == L.ORBIT_E_UNSUPPORTED
        assert "2^24 tiles" in lib.last_error()
    # just below both limits: the store is checked, not refused
    n = (1 << 31) - 128
    assert c.orbit_fp8_unpack(1, 1, n, 0x100, F.layout(1, n)[3] - 1, 0x200, n, None) == L.ORBIT_E_ARG and "store of" in lib.last_error()


def test_grid_rope_written_out():
    from paper_2404_14712_amd.model import grid_rope
    r = grid_rope(2, 3, 32, theta=16.0, device="cpu")
    assert r.pos.tolist() == [[0, 0], [0, 1], [0, 2], [1, 0], [1, 1], [1, 2]] and r.pos.dtype == torch.float32
    assert r.axis == [0] * 8 + [1] * 8 and not r.near
    want = [1.0, 2.0 ** -0.5, 0.5, 2.0 ** -1.5, 0.25, 2.0 ** -2.5, 0.125, 2.0 ** -3.5] * 2
    assert r.freq.dtype == torch.float32 and all(abs(float(f) - w) <= F.U32 * w for f, w in zip(r.freq, want))
