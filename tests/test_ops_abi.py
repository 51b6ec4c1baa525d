"""Host-side checks of the 8-bit store's and the gated norms' entry points: sizes, refusals and the
64-bit references the GPU tests compare with (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import ops_ref as R
from paper_2404_14712_amd import _lib as L


@pytest.fixture(scope="module")
def lib():
    return L.OrbitLib()


@pytest.mark.parametrize("rows,n", [(1, 8), (1, 32), (3, 40), (257, 1000), (8192, 4096)])
def test_act8_bytes(lib, rows, n):
    assert lib.orbit_act8_bytes(rows, n) == R.store_layout(rows, n)[2]


def test_act8_refusals(lib):
    c = lib.lib
    big = 1 << 50
    assert lib.orbit_act8_bytes(0, 8) == 0 and lib.orbit_act8_bytes(4, 12) == 0 and lib.orbit_act8_bytes(4, -8) == 0
    assert lib.orbit_act8_bytes(1 << 40, 8) == 0
    ok = (1, 4, 40, 0x100, 40, 0x200, big, None)
    bad = {"dtype": (7,) + ok[1:], "bad sizes": (1, 4, 36) + ok[3:], "x is NULL": ok[:3] + (None,) + ok[4:],
           "16-byte": ok[:3] + (0x108,) + ok[4:], "ldx": ok[:4] + (32,) + ok[5:], "store is NULL": ok[:5] + (None, big, None),
           "smaller": ok[:6] + (R.store_layout(4, 40)[2] - 1, None)}
    for what, args in bad.items():
        assert c.orbit_act8_pack(*args) == L.ORBIT_E_ARG and what in lib.last_error(), (what, lib.last_error())
    assert c.orbit_act8_pack(1, 1 << 39, 1 << 20, 0x100, 1 << 20, 0x200, big, None) == L.ORBIT_E_UNSUPPORTED
    assert c.orbit_act8_pack(*ok[:4], 44, *ok[5:]) == L.ORBIT_E_ARG and "ldx" in lib.last_error()
    un = (1, 4, 40, 0x100, big, 0x200, 40, 0x300, 40, None)
    bad = {"both NULL": un[:5] + (None, 0, None, 0, None), "alias": un[:7] + (0x200, 40, None),
           "ldx": un[:6] + (36,) + un[7:], "ldgelu": un[:8] + (8, None), "store is NULL": un[:3] + (None,) + un[4:],
           "gelu is not": un[:7] + (0x301,) + un[8:]}
    for what, args in bad.items():
        assert c.orbit_act8_unpack(*args) == L.ORBIT_E_ARG and what in lib.last_error(), (what, lib.last_error())
    assert lib.orbit_act8_weight_grad_workspace_bytes(1, 4, 36, 8) == 0
    assert lib.orbit_act8_weight_grad_workspace_bytes(1, 4, 40, 8) > 0
    wg = (1, 4, 40, 16, 0x100, big, 0x200, 16, 0x300, 0x400, 0, 0x500, big, None)
    bad = {"bad sizes": (1, 4, 40, 12) + wg[4:], "dy is NULL": wg[:6] + (None,) + wg[7:], "lddy": wg[:7] + (8,) + wg[8:],
           "dw is NULL": wg[:8] + (None,) + wg[9:], "accumulate": wg[:10] + (2,) + wg[11:],
           "workspace": wg[:12] + (16, None), "store of": wg[:5] + (100,) + wg[6:]}
    for what, args in bad.items():
        assert c.orbit_act8_weight_grad(*args) == L.ORBIT_E_ARG and what in lib.last_error(), (what, lib.last_error())


def _desc(**kw):
    v = dict(rows=8, n=64, gate_rows=2, post_norm=1, pre_norm=1, scale=1.0, eps=1e-5, dtype=1)
    v.update(kw)
    return L.GatedNormDesc(*[v[k] for k, _ in L.GatedNormDesc._fields_])


PARAMS = {"gate": 0x1000, "post_g": 0x1100, "post_b": 0x1200, "pre_g": 0x1300, "pre_b": 0x1400}


def _fwd(lib, desc=None, params=None, x=0x100, f=0x200, store=None, store_bytes=0, y=0x300, h=0x400, stats=0x500):
    p = lib._struct(L.GatedNormParams, PARAMS if params is None else params)
    return lib.lib.orbit_gated_norm_fwd(ctypes.byref(desc or _desc()), ctypes.byref(p), x, f, store, store_bytes, y, h,
                                        stats, None)


def _bwd(lib, desc=None, params=None, grads=None, f=0x100, store=None, store_bytes=0, y=0x200, stats=0x300, dh=0x400,
         dy=0x500, dx=0x600, df=0x700, accumulate=0, ws=0x800, ws_bytes=1 << 40):
    p = lib._struct(L.GatedNormParams, PARAMS if params is None else params)
    g = lib._struct(L.GatedNormGrads, PARAMS if grads is None else grads)
    return lib.lib.orbit_gated_norm_bwd(ctypes.byref(desc or _desc()), ctypes.byref(p), f, store, store_bytes, y, stats,
                                        dh, dy, dx, df, ctypes.byref(g), accumulate, ws, ws_bytes, None)


def test_gated_norm_refusals(lib):
    for kw, what in ((dict(rows=0), "sizes"), (dict(n=60), "sizes"), (dict(gate_rows=3), "gate_rows"),
                     (dict(gate_rows=-1), "gate_rows"), (dict(post_norm=2), "post_norm"), (dict(pre_norm=-1), "pre_norm"),
                     (dict(eps=0.0), "eps"), (dict(dtype=3), "dtype")):
        assert _fwd(lib, _desc(**kw)) == L.ORBIT_E_ARG and what in lib.last_error()
        assert _bwd(lib, _desc(**kw)) == L.ORBIT_E_ARG and what in lib.last_error()
        assert lib.orbit_gated_norm_bwd_workspace_bytes(_desc(**kw)) == 0
    assert _fwd(lib, _desc(n=16392)) == L.ORBIT_E_UNSUPPORTED
    assert lib.orbit_gated_norm_bwd_workspace_bytes(_desc(n=16392)) == 0
    for k in PARAMS:
        less = dict(PARAMS)
        del less[k]
        assert _fwd(lib, params=less) == L.ORBIT_E_ARG and k in lib.last_error()
        assert _bwd(lib, grads=less) == L.ORBIT_E_ARG and k in lib.last_error()
    for kw, what in ((dict(x=None), "x is NULL"), (dict(y=0x308), "y is not"), (dict(f=None), "both NULL"),
                     (dict(y=0x100), "alias"), (dict(h=0x300), "alias"), (dict(h=None), "h is NULL"),
                     (dict(stats=None), "stats"), (dict(store=0x600, store_bytes=64), "smaller")):
        assert _fwd(lib, **kw) == L.ORBIT_E_ARG and what in lib.last_error(), (kw, lib.last_error())
    for kw, what in ((dict(f=None), "both NULL"), (dict(y=None), "y is NULL"), (dict(dh=None), "dh is NULL"),
                     (dict(df=None), "df is NULL"), (dict(dx=0x700), "alias"), (dict(dx=0x200), "alias"),
                     (dict(dx=0x400), "alias"), (dict(df=0x500), "alias"), (dict(dx=0x100), "alias"),
                     (dict(accumulate=2), "accumulate"), (dict(ws=None), "ws is NULL"), (dict(ws_bytes=8), "workspace"),
                     (dict(f=None, store=0x900, store_bytes=8), "smaller"), (dict(stats=None), "stats")):
        assert _bwd(lib, **kw) == L.ORBIT_E_ARG and what in lib.last_error(), (kw, lib.last_error())
    assert _bwd(lib, _desc(pre_norm=0), dy=None) == L.ORBIT_E_ARG and "dy is NULL" in lib.last_error()


def test_act8_reference_by_brute_force():
    """Every value is the nearest of the 255 the chosen step offers, and half that step would not reach the
    largest: the two properties the store is defined by."""
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((40, 40)) * np.exp(rng.uniform(-30, 30, (40, 1)))).astype(np.float32)
    x[0] = 0.0
    x[1, :32] = 127.5 / 64          # the border at which the step doubles
    x[2, :32] = np.float32(127.4999 / 64)
    codes, E, val = R.act8_ref(x)
    for r in range(x.shape[0]):
        for g in range(2):
            t, step = x[r, 32 * g:32 * g + 32].astype(np.float64), 2.0 ** (int(E[r, g]) - 133)
            grid = np.arange(-127, 128) * step
            best = np.abs(t[:, None] - grid[None]).min(1)
            np.testing.assert_array_equal(np.abs(t - val[r, 32 * g:32 * g + 32]), best)
            assert best.max() <= step / 2
            if E[r, g] > 7:
                assert np.abs(t).max() >= 127.5 * step / 2
    assert E[1, 0] == E[2, 0] + 1 == 128


def test_gated_norm_reference_by_differences():
    """The float64 gradients against central differences of the forward formula."""
    g = torch.Generator().manual_seed(3)
    z = dict(rows=6, n=16, gate_rows=3, post_norm=1, pre_norm=1, scale=0.7, eps=1e-5)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    p = {"gate": rnd(3, 16), "post_g": rnd(16), "post_b": rnd(16), "pre_g": rnd(16), "pre_b": rnd(16)}
    x, f, dh, dy = (rnd(6, 16) for _ in range(4))
    y, _ = R.gated_norm_ref(z, p, x, f)
    dx, df, gp = R.gated_norm_grad_ref(z, p, f, y, dh, dy)

    def value(p, x, f):
        y, h = R.gated_norm_ref(z, p, x, f)
        return float((dh * h).sum() + (dy * y).sum())

    e = 1e-5
    for name, grad in dict(gp, x=dx, f=df).items():
        v = rnd(*grad.shape)
        args = lambda s: (dict(p, **{name: p[name] + s * e * v}) if name in p else p, x + s * e * v if name == "x" else x,
                          f + s * e * v if name == "f" else f)
        num = (value(*args(1)) - value(*args(-1))) / (2 * e)
        assert abs(num - float((grad * v).sum())) <= 1e-6 * max(1.0, abs(num)), name


def _bdesc(**kw):
    v = dict(B=2, L=20, d=64, heads=2, head_dim=32, mlp=128, qk_norm=1, eps=1e-5, dtype=1)
    v.update(kw)
    return L.BlockDesc(*[v[k] for k, _ in L.BlockDesc._fields_])


def test_block_ext_sizes(lib):
    """The plain form asks for what the plain calls ask for; 8-bit stores take under a quarter of the
    bytes at the workloads' sizes."""
    import synth
    for c in synth.CONFIGS.values():
        d = L.BlockDesc(c.B, c.L, c.d, c.heads, c.head_dim, c.mlp, c.qk_norm, c.eps, 1 if c.dtype == "bf16" else 0)
        plain = L.BlockExt(0, 0, 0, 1.0)
        full = lib.orbit_vit_block_saved_bytes(d)
        assert lib.orbit_vit_block_ext_saved_bytes(d, plain) == full
        assert lib.orbit_vit_block_ext_workspace_bytes(d, plain) == lib.orbit_vit_block_workspace_bytes(d)
        small = lib.orbit_vit_block_ext_saved_bytes(d, L.BlockExt(1, 0, 0, 1.0))
        assert 0 < small < full / 4, c.name
        gated = L.BlockExt(1, 1, c.B, 0.5)
        assert small < lib.orbit_vit_block_ext_saved_bytes(d, gated) < full / 3
        assert lib.orbit_vit_block_ext_saved_bytes(d, L.BlockExt(0, 1, c.B, 0.5)) > full


def test_block_ext_refusals(lib):
    d = _bdesc()
    for ext, what in (((2, 0, 0, 1.0), "act8"), ((0, 3, 0, 1.0), "post_norm"), ((0, 0, 3, 1.0), "gate_rows"),
                      ((0, 0, -1, 1.0), "gate_rows")):
        e = L.BlockExt(*ext)
        assert lib.orbit_vit_block_ext_saved_bytes(d, e) == 0 and what in lib.last_error()
        assert lib.orbit_vit_block_ext_workspace_bytes(d, e) == 0
    assert lib.orbit_vit_block_ext_saved_bytes(_bdesc(d=60), L.BlockExt(1, 0, 0, 1.0)) == 0

    def fwd(e, drop=(), ws_bytes=1 << 40, y=0x200):
        p = L.BlockParams(*[0x1000 + 0x100 * i for i in range(16)])
        ep = L.BlockExtParams(*[None if n in drop else 0x4000 + 0x100 * i for i, n in enumerate(L.BLOCK_EXT_PARAMS)])
        return lib.lib.orbit_vit_block_ext_fwd(ctypes.byref(d), ctypes.byref(e) if e else None, ctypes.byref(p),
                                               ctypes.byref(ep), 0x100, y, None, 0x300, ws_bytes, None)

    def bwd(e, drop=(), ws_bytes=1 << 40):
        p = L.BlockParams(*[0x1000 + 0x100 * i for i in range(16)])
        ep = L.BlockExtParams(*[0x4000 + 0x100 * i for i in range(6)])
        g = L.BlockGrads(*[0x5000 + 0x100 * i for i in range(16)])
        eg = L.BlockExtGrads(*[None if n in drop else 0x7000 + 0x100 * i for i, n in enumerate(L.BLOCK_EXT_PARAMS)])
        return lib.lib.orbit_vit_block_ext_bwd(ctypes.byref(d), ctypes.byref(e), ctypes.byref(p), ctypes.byref(ep), 0x100,
                                               None, 0x200, 0x300, ctypes.byref(g), ctypes.byref(eg), 0, 0x400, ws_bytes,
                                               None)

    full = L.BlockExt(1, 1, 2, 0.5)
    assert fwd(None) == L.ORBIT_E_ARG and "ext is NULL" in lib.last_error()
    assert fwd(full, y=0x100) == L.ORBIT_E_ARG and "alias" in lib.last_error()
    assert fwd(full, ws_bytes=64) == L.ORBIT_E_ARG and "workspace" in lib.last_error()
    assert bwd(full, ws_bytes=64) == L.ORBIT_E_ARG and "workspace" in lib.last_error()
    # the plain call's workspace is too small for the extended one
    assert fwd(full, ws_bytes=lib.orbit_vit_block_workspace_bytes(d)) == L.ORBIT_E_ARG
    for n in L.BLOCK_EXT_PARAMS:
        assert fwd(full, drop=(n,)) == L.ORBIT_E_ARG and n in lib.last_error()
        assert bwd(full, drop=(n,)) == L.ORBIT_E_ARG and f"grads.{n}" in lib.last_error()


@pytest.mark.parametrize("post,gates", [(1, 2), (0, 1), (1, 0), (0, 0)])
def test_block_ext_reference_by_autograd(post, gates):
    """The written-out gradients equal autograd's of the forward when nothing is rounded."""
    g = torch.Generator().manual_seed(6)
    B, Lq, d, H, F = 2, 5, 16, 2, 24
    rnd = lambda *s: 0.4 * torch.randn(*s, generator=g, dtype=torch.float64)
    p = {"w_qkv": rnd(d, 3 * d), "b_qkv": rnd(3 * d), "w_proj": rnd(d, d), "b_proj": rnd(d), "w_fc1": rnd(d, F),
         "b_fc1": rnd(F), "w_fc2": rnd(F, d), "b_fc2": rnd(d)}
    for n, w in (("ln1", d), ("ln2", d), ("qn", d // H), ("kn", d // H), ("post1", d), ("post2", d)):
        if post or not n.startswith("post"):
            p.update({n + "_g": 1 + rnd(w), n + "_b": rnd(w)})
    if gates:
        p.update(gate1=rnd(gates, d), gate2=rnd(gates, d))
    z = dict(n=d, gate_rows=gates, post_norm=post, scale=0.7)
    x, dy = rnd(B, Lq, d), rnd(B, Lq, d)
    leaf = {k: v.clone().requires_grad_(True) for k, v in p.items()}
    xl = x.clone().requires_grad_(True)
    y, _ = R.block_ext_forward(xl, leaf, H, z)
    y.backward(dy)
    _, c = R.block_ext_forward(x, p, H, z)
    dx, gr = R.block_ext_backward(x, p, H, z, c, dy, lambda t: t)
    assert torch.allclose(dx, xl.grad, rtol=1e-9, atol=1e-11)
    assert set(gr) == set(p)
    for k in p:
        assert torch.allclose(gr[k], leaf[k].grad, rtol=1e-9, atol=1e-11), k


@pytest.mark.parametrize("checkpoint,kept", [(False, "full"), (None, "full"), (0, "full"), (True, None), (1, None),
                                             (np.True_, None), ("act8", "small")])
def test_pass_checkpoint_values(lib, checkpoint, kept):
    """What a pass keeps of its blocks: any value but "act8" counts by its truth."""
    from paper_2404_14712_amd.model import PassDims, ViTPass
    dims = PassDims("blocks", "bf16", 1, 4, 64, 1, 2, 32, 128)
    vp = ViTPass(lib, dims, {"blocks": [{}]}, device="cpu", checkpoint=checkpoint)
    want = {"full": lambda: lib.orbit_vit_block_saved_bytes(vp.bdesc),
            "small": lambda: lib.orbit_vit_block_ext_saved_bytes(vp.bdesc, L.BlockExt(1, 0, 0, 1.0))}
    got = [None if s is None else s.numel() for s in vp.saved]
    assert got == [want[kept]() if kept else None]


def test_pass_checkpoint_refusal(lib):
    from paper_2404_14712_amd.model import PassDims, ViTPass
    with pytest.raises(ValueError, match="checkpoint"):
        ViTPass(lib, PassDims("blocks", "bf16", 1, 4, 64, 1, 2, 32, 128), {"blocks": [{}]}, device="cpu",
                checkpoint="full")


def test_refusals_of_the_largest_sizes(lib):
    """Sizes whose launches or offsets would not fit are refused before anything is launched."""
    c, big = lib.lib, 1 << 50
    edge = (1 << 34) // 1024
    assert lib.orbit_act8_bytes(edge, 1024) == 0 and lib.orbit_act8_bytes(edge - 1, 1024) > 0
    assert c.orbit_act8_pack(1, edge, 1024, 0x100, 1024, 0x200, big, None) == L.ORBIT_E_UNSUPPORTED
    assert c.orbit_act8_unpack(1, edge, 1024, 0x200, big, 0x100, 1024, None, 0, None) == L.ORBIT_E_UNSUPPORTED
    wg = (1, 4, 40, 16, 0x100, big, 0x200, 16, 0x300, 0x400, 0, 0x500, big, None)
    assert c.orbit_act8_weight_grad(*wg[:7], 1 << 25, *wg[8:]) == L.ORBIT_E_UNSUPPORTED and "lddy" in lib.last_error()
    assert c.orbit_act8_weight_grad(*wg[:2], 1 << 25, *wg[3:]) == L.ORBIT_E_UNSUPPORTED and "K=" in lib.last_error()
    assert lib.orbit_act8_weight_grad_workspace_bytes(1, 4, 1 << 25, 16) == 0
    for rows, n in ((1 << 26, 8), ((1 << 26) - 63, 8)):
        d = _desc(rows=rows, n=n, gate_rows=1)
        assert _fwd(lib, d) == L.ORBIT_E_UNSUPPORTED and "rows" in lib.last_error()
        assert _bwd(lib, d) == L.ORBIT_E_UNSUPPORTED
        assert lib.orbit_gated_norm_bwd_workspace_bytes(d) == 0
    assert lib.orbit_gated_norm_bwd_workspace_bytes(_desc(rows=(1 << 26) - 64, n=8, gate_rows=1)) > 0
