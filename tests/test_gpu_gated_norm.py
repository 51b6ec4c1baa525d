"""Gated norms on the GPU, forward and backward, against the formulas in 64 bits
(bounds derived in ops_ref) and against differences of the forward."""
import numpy as np
import pytest
import torch

import ops_ref as R
from paper_2404_14712_amd._lib import GatedNormDesc

pytestmark = pytest.mark.gpu


def _case(rows, n, gates, post, pre, dtype, seed=0, scale=0.5, mean=0.0):
    g = torch.Generator().manual_seed(seed + rows * 131 + n)
    dt = R.TORCH[dtype]
    rnd = lambda *s, std=1.0, m=0.0: (torch.randn(*s, generator=g) * std + m).to(dt)
    z = dict(rows=rows, n=n, gate_rows=gates, post_norm=post, pre_norm=pre, scale=scale, eps=1e-5)
    p = {}
    if gates:
        p["gate"] = rnd(gates, n, std=0.3, m=0.4)
    if post:
        p.update(post_g=rnd(n, std=0.1, m=1.0), post_b=rnd(n, std=0.1))
    if pre:
        p.update(pre_g=rnd(n, std=0.1, m=1.0), pre_b=rnd(n, std=0.1))
    return z, p, {k: rnd(rows, n, m=mean if k in "xf" else 0.0) for k in ("x", "f", "dh", "dy")}


def _desc(z, dtype):
    return GatedNormDesc(z["rows"], z["n"], z["gate_rows"], z["post_norm"], z["pre_norm"], z["scale"], z["eps"],
                         R.CODE[dtype])


def _d(p):
    return {k: v.cuda() for k, v in p.items()}


def _64(p):
    return {k: v.double() for k, v in p.items()}


def _forward(lib, z, p, t, dtype, f8=0):
    """f8: 0 no store, 1 f also into a store, 2 f read from the store."""
    rows, n = z["rows"], z["n"]
    x, f = t["x"].cuda(), t["f"].cuda()
    y = torch.full((rows + 1, n), 5.0, dtype=x.dtype, device="cuda")
    h = torch.full((rows + 1, n), 5.0, dtype=x.dtype, device="cuda") if z["pre_norm"] else None
    stats = torch.full((rows + 1, 4), 5.0, device="cuda")
    store = torch.zeros(lib.orbit_act8_bytes(rows, n), dtype=torch.uint8, device="cuda") if f8 else None
    if f8 == 2:
        lib.orbit_act8_pack(R.CODE[dtype], rows, n, f, n, store)
    lib.orbit_gated_norm_fwd(_desc(z, dtype), _d(p), x, None if f8 == 2 else f, store, y, h, stats)
    assert bool((y[rows] == 5).all()) and bool((stats[rows] == 5).all()) and (h is None or bool((h[rows] == 5).all()))
    return y[:rows], h[:rows] if h is not None else None, stats[:rows], store


def _within(got, ref, tol, what):
    err = (got.cpu().double() - ref).abs()
    assert bool((err <= tol).all()), f"{what}: off by {float(err.max()):.3e}, {float((err / tol.clamp(min=1e-300)).max()):.2f} of the bound"


def _check_forward(lib, z, p, t, dtype, f8=0):
    y, h, stats, store = _forward(lib, z, p, t, dtype, f8)
    f = t["f"].double()
    if f8 == 2:
        f = torch.from_numpy(R.act8_ref(f.numpy())[2])
    ry, rh, ty, th = R.gated_norm_tol(z, _64(p), t["x"].double(), f, R.HALF[dtype])
    _within(y, ry, ty, "y")
    if z["pre_norm"]:
        _within(h, rh, th, "h")
    if f8 == 1:
        back = torch.empty_like(y)
        lib.orbit_act8_unpack(R.CODE[dtype], z["rows"], z["n"], store, back, z["n"])
        np.testing.assert_array_equal(back.cpu().double().numpy(), R.act8_ref(f.numpy())[2])
    return y, h, stats, store


def _grads(p):
    return {k: torch.full(v.shape, 2.0, device="cuda") for k, v in p.items()}


def _backward(lib, z, p, t, y, stats, dtype, store=None, accumulate=0, dy=True, dx=True):
    rows, n = z["rows"], z["n"]
    ws = torch.full((lib.orbit_gated_norm_bwd_workspace_bytes(_desc(z, dtype)),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((2, rows + 1, n), 5.0, dtype=y.dtype, device="cuda")
    g = _grads(p)
    lib.orbit_gated_norm_bwd(_desc(z, dtype), _d(p), None if store is not None else t["f"].cuda(), store, y, stats,
                             t["dh"].cuda() if z["pre_norm"] else None, t["dy"].cuda() if dy else None,
                             out[0, :rows] if dx else None, out[1, :rows], g, accumulate, ws)
    assert bool((out[:, rows] == 5).all())
    return out[0, :rows], out[1, :rows], g


def _check_backward(lib, z, p, t, dtype, f8=0, accumulate=0, dy=True):
    y, _, stats, store = _forward(lib, z, p, t, dtype, f8)
    f = t["f"].double()
    if f8:
        f = torch.from_numpy(R.act8_ref(f.numpy())[2])
        if f8 == 1:  # the store's f has statistics of its own
            _, _, stats, _ = _forward(lib, z, p, t, dtype, 2)
    # the backward takes y as stored: statistics of that y
    y64 = y.cpu().double()
    if z["pre_norm"]:
        mu = y64.mean(-1)
        rs = 1.0 / torch.sqrt(((y64 - mu[:, None]) ** 2).mean(-1) + z["eps"])
        stats = stats.clone()
        stats[:, 2], stats[:, 3] = mu.float().cuda(), rs.float().cuda()
    dx, df, g = _backward(lib, z, p, t, y, stats, dtype, store if f8 else None, accumulate, dy)
    dy64 = t["dy"].double() if dy else None
    rx, rf, rg = R.gated_norm_grad_ref(z, _64(p), f, y64, t["dh"].double(), dy64)
    tx, tf, tg = R.gated_norm_grad_tol(z, _64(p), f, y64, t["dh"].double(), dy64, R.HALF[dtype])
    _within(dx, rx, tx, "dx")
    _within(df, rf, tf, "df")
    assert set(g) == set(rg)
    for k in g:
        ref = rg[k] + (2.0 if accumulate else 0.0)
        _within(g[k], ref, tg[k] + 4 * R.U32 * ref.abs(), k)
    return dx, df, g


SHAPES = [(1, 8, 1), (1, 2048, 1), (3, 40, 3), (4, 512, 2), (7, 1000, 1), (6, 1032, 3), (37, 2056, 0), (10, 4104, 2),
          (5, 8200, 1), (3, 16384, 3), (515, 128, 5), (300, 1024, 4),
          (9, 520, 0), (5, 8192, 1), (2, 12288, 2), (3, 12296, 1), (1100, 1040, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,gates", SHAPES)
@pytest.mark.parametrize("f8", [0, 1, 2])
def test_forward(lib, rows, n, gates, f8, dtype):
    z, p, t = _case(rows, n, gates, 1, 1, dtype)
    _check_forward(lib, z, p, t, dtype, f8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,gates", SHAPES)
@pytest.mark.parametrize("f8", [0, 1])
def test_backward(lib, rows, n, gates, f8, dtype):
    z, p, t = _case(rows, n, gates, 1, 1, dtype, seed=1)
    _check_backward(lib, z, p, t, dtype, f8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre,gates", [(0, 0, 0), (0, 0, 2), (0, 1, 0), (0, 1, 2), (1, 0, 0), (1, 0, 2), (1, 1, 0)])
@pytest.mark.parametrize("n", [264, 8200])
def test_parts(lib, post, pre, gates, n, dtype):
    """Each norm and the gate alone and in pairs, accumulating."""
    z, p, t = _case(18, n, gates, post, pre, dtype, seed=2, scale=-1.25)
    _check_forward(lib, z, p, t, dtype, 1)
    for f8 in (0, 1):
        _check_backward(lib, z, p, t, dtype, f8, accumulate=1)
    if pre:
        _check_backward(lib, z, p, t, dtype, 0, dy=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre,gates", [(0, 1, 0), (1, 0, 1), (0, 1, 4)])
@pytest.mark.parametrize("rows,n", [(1100, 8200), (2000, 4104)])
def test_one_norm_over_many_turns(lib, rows, n, post, pre, gates, dtype):
    """One norm alone, rows of several waves and chunks of several turns: a turn's wave sums are read
    before the next turn's overwrite them, every time."""
    z, p, t = _case(rows, n, gates, post, pre, dtype, seed=18)
    dx, df, g = _check_backward(lib, z, p, t, dtype)
    y, _, stats, _ = _forward(lib, z, p, t, dtype)
    for _ in range(3):
        dx2, df2, g2 = _backward(lib, z, p, t, y, stats, dtype)
        dx3, df3, g3 = _backward(lib, z, p, t, y, stats, dtype)
        assert torch.equal(dx2, dx3) and torch.equal(df2, df3) and all(torch.equal(g2[k], g3[k]) for k in g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gate_per_row_and_hard_rows(lib, dtype):
    """A gate row for each token; rows far from zero, constant rows, empty (zero) rows."""
    z, p, t = _case(33, 328, 33, 1, 1, dtype, seed=5, mean=50.0)
    for k in ("x", "f"):
        t[k][3] = 0.0
        t[k][4] = 7.0
    t["f"][6] = 0.0
    _check_forward(lib, z, p, t, dtype)
    _check_backward(lib, z, p, t, dtype)


def test_streamed_rows(lib):
    """From 96 MB of tensors on bf16 rows are loaded non-temporally: the same results, checked on some rows."""
    z, p, t = _case(6144, 2056, 3, 1, 1, "bf16", seed=14)
    y, h, stats, _ = _forward(lib, z, p, t, "bf16")
    pick = torch.tensor([0, 1, 2047, 2048, 4096, 6143])
    zs = dict(z, rows=len(pick), gate_rows=len(pick))
    ps = dict(_64(p), gate=p["gate"].double()[pick // 2048])
    ry, rh, ty, th = R.gated_norm_tol(zs, ps, t["x"].double()[pick], t["f"].double()[pick], R.HALF["bf16"])
    _within(y[pick.cuda()], ry, ty, "y")
    _within(h[pick.cuda()], rh, th, "h")
    dx, df, g = _backward(lib, z, p, t, y, stats, "bf16")
    rx, rf, rg = R.gated_norm_grad_ref(z, _64(p), t["f"].double(), y.cpu().double(), t["dh"].double(), t["dy"].double())
    tx, tf, tg = R.gated_norm_grad_tol(z, _64(p), t["f"].double(), y.cpu().double(), t["dh"].double(), t["dy"].double(),
                                       R.HALF["bf16"])
    # in the 2-norm: the outputs' own rounding, at most 2^-8 of each value, and the statistics of the unrounded y,
    # whose mean and deviation the rounding of 2056 values (2^-8 each at most, of either sign) moves far less
    slack = 2.0 ** -8
    assert float((dx.cpu().double() - rx).norm()) <= slack * float(rx.norm())
    assert float((df.cpu().double() - rf).norm()) <= slack * float(rf.norm())
    for k in g:
        assert float((g[k].cpu().double() - rg[k]).norm()) <= slack * float(rg[k].norm()), k


@pytest.mark.parametrize("f8", [0, 1])
def test_far_offsets(lib, f8):
    """Tensors of 4.6 GB: rows past 2^31 values give what the same rows give alone."""
    rows, n, last = 140000, 16384, 3
    z, p, t = _case(last, n, 1, 1, 1, "bf16", seed=15)
    small = _forward(lib, z, p, t, "bf16", 2 if f8 else 0)
    sdx, sdf, _ = _backward(lib, z, p, t, small[0], small[2], "bf16", small[3])
    P = _d(p)
    big = {k: torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda") for k in ("x", "f", "dh", "dy")}
    for k in big:
        big[k][-last:] = t[k].cuda()
    zb = dict(z, rows=rows)
    store = None
    if f8:
        store = torch.empty(lib.orbit_act8_bytes(rows, n), dtype=torch.uint8, device="cuda")
        lib.orbit_act8_pack(1, rows, n, big["f"], n, store)
    f = None if f8 else big["f"]
    y, h = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    stats = torch.empty(rows, 4, device="cuda")
    lib.orbit_gated_norm_fwd(_desc(zb, "bf16"), P, big["x"], f, store, y, h, stats)
    assert torch.equal(y[-last:], small[0]) and torch.equal(h[-last:], small[1])
    assert torch.equal(stats[-last:], small[2])
    ws = torch.empty(lib.orbit_gated_norm_bwd_workspace_bytes(_desc(zb, "bf16")), dtype=torch.uint8, device="cuda")
    dx, df = h, torch.empty_like(h)
    lib.orbit_gated_norm_bwd(_desc(zb, "bf16"), P, f, store, y, stats, big["dh"], big["dy"], dx, df, _grads(p), 0, ws)
    assert torch.equal(dx[-last:], sdx) and torch.equal(df[-last:], sdf)


def test_two_streams_at_once(lib):
    """Calls in flight on two streams, each with its own buffers, give what they give alone."""
    cases = [_case(900, 2056, 3, 1, 1, "bf16", seed=s) for s in (16, 17)]
    runs = []
    for z, p, t in cases:
        y, _, stats, _ = _forward(lib, z, p, t, "bf16")
        alone = _backward(lib, z, p, t, y, stats, "bf16")
        D = {k: v.cuda() for k, v in t.items()}
        ws = torch.empty(lib.orbit_gated_norm_bwd_workspace_bytes(_desc(z, "bf16")), dtype=torch.uint8, device="cuda")
        runs.append((z, _d(p), D, y, stats, torch.empty_like(y), torch.empty_like(y), _grads(p), ws, alone, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for z, P, D, y, stats, dx, df, g, ws, _, s in runs:
            lib.orbit_gated_norm_bwd(_desc(z, "bf16"), P, D["f"], None, y, stats, D["dh"], D["dy"], dx, df, g, 0, ws, stream=s)
    torch.cuda.synchronize()
    for _, _, _, _, _, dx, df, g, _, alone, _ in runs:
        assert torch.equal(dx, alone[0]) and torch.equal(df, alone[1]) and all(torch.equal(g[k], alone[2][k]) for k in g)


def test_many_rows(lib):
    """More rows than chunks of one size: ragged last chunks per gate row."""
    z, p, t = _case(3 * 1371, 72, 3, 1, 1, "f32", seed=6)
    _check_forward(lib, z, p, t, "f32", 2)
    _check_backward(lib, z, p, t, "f32", 1)


def test_non_finite_rows_stay_in_their_rows(lib):
    z, p, t = _case(9, 256, 1, 1, 1, "bf16", seed=7)
    t["f"][2, 17] = float("nan")
    t["x"][5, 3] = float("inf")
    y, h, _, store = _forward(lib, z, p, t, "bf16", 1)
    bad = [2, 5]
    good = [i for i in range(9) if i not in bad]
    assert bool(torch.isfinite(y[good]).all()) and bool(torch.isfinite(h[good]).all())
    assert bool(torch.isnan(h[bad]).all())


def test_no_dx_and_aliases(lib):
    """dx left out; dx over dy and df over dh give the same bits as separate buffers."""
    z, p, t = _case(50, 1096, 2, 1, 1, "bf16", seed=8)
    y, _, stats, _ = _forward(lib, z, p, t, "bf16")
    dx, df, g = _backward(lib, z, p, t, y, stats, "bf16")
    _, df2, g2 = _backward(lib, z, p, t, y, stats, "bf16", dx=False)
    assert torch.equal(df, df2) and all(torch.equal(g[k], g2[k]) for k in g)
    dy, dh, f = t["dy"].cuda(), t["dh"].cuda(), t["f"].cuda()
    ws = torch.empty(lib.orbit_gated_norm_bwd_workspace_bytes(_desc(z, "bf16")), dtype=torch.uint8, device="cuda")
    g3 = _grads(p)
    lib.orbit_gated_norm_bwd(_desc(z, "bf16"), _d(p), f, None, y, stats, dh, dy, dy, dh, g3, 0, ws)
    assert torch.equal(dy, dx) and torch.equal(dh, df) and all(torch.equal(g[k], g3[k]) for k in g)
    dy, dh = t["dy"].cuda(), t["dh"].cuda()
    lib.orbit_gated_norm_bwd(_desc(z, "bf16"), _d(p), f, None, y, stats, dh, dy, dy, f, g3, 0, ws)
    assert torch.equal(dy, dx) and torch.equal(f, df)


def test_store_read_equals_its_values(lib):
    """Forward and backward from the store are bitwise those from the values it stands for."""
    for dtype in ("bf16", "f32"):
        z, p, t = _case(70, 2056, 2, 1, 1, dtype, seed=9)
        y, h, stats, store = _forward(lib, z, p, t, dtype, 2)
        f = torch.empty(70, 2056, dtype=R.TORCH[dtype], device="cuda")
        lib.orbit_act8_unpack(R.CODE[dtype], 70, 2056, store, f, 2056)
        t2 = dict(t, f=f.cpu())
        y2, h2, stats2, _ = _forward(lib, z, p, t2, dtype)
        assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(stats, stats2)
        a, b = _backward(lib, z, p, t, y, stats, dtype, store), _backward(lib, z, p, t2, y, stats, dtype)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][k], b[2][k]) for k in a[2])


def test_gradients_against_differences(lib):
    """Directional derivatives of <dh, h> + <dy, y> by central differences of the float32 forward."""
    z, p, t = _case(40, 512, 4, 1, 1, "f32", seed=10)

    def value(p, t):
        y, h, _, _ = _forward(lib, z, p, t, "f32")
        return float((t["dy"].double() * y.cpu().double()).sum() + (t["dh"].double() * h.cpu().double()).sum())

    y, _, stats, _ = _forward(lib, z, p, t, "f32")
    dx, df, g = _backward(lib, z, p, t, y, stats, "f32")
    grads = dict({k: v.cpu() for k, v in g.items()}, x=dx.cpu(), f=df.cpu())
    gen = torch.Generator().manual_seed(11)
    e = 2.0 ** -8
    for name, gr in grads.items():
        v = torch.randn(gr.shape, generator=gen)
        at = lambda s: (dict(p, **{name: p[name] + s * e * v}), t) if name in p else (p, dict(t, **{name: t[name] + s * e * v}))
        num = (value(*at(1)) - value(*at(-1))) / (2 * e)
        ana = float((gr.double() * v.double()).sum())
        # e^2 times third derivatives of order one (the norms' curvature) over the terms' sizes,
        # and the forward's float32 rounding (2^-22 of each of 2 x 20480 terms, at random) over e
        size = float((gr.double() * v.double()).norm())
        noise = 2.0 ** -22 * (2 * 20480) ** 0.5 * 4 / e
        assert abs(num - ana) <= 16 * e * e * size * 20 + noise, (name, num, ana)


@pytest.mark.parametrize("f8", [0, 1])
def test_side_stream_and_graph(lib, f8):
    """Forward and backward on another stream and captured, replayed with eager work between."""
    z, p, t = _case(260, 1040, 4, 1, 1, "bf16", seed=12)
    P, D = _d(p), {k: v.cuda() for k, v in t.items()}
    gen = torch.Generator().manual_seed(13)
    y, h, dx, df = (torch.empty_like(D["x"]) for _ in range(4))
    stats = torch.empty(260, 4, device="cuda")
    store = torch.empty(lib.orbit_act8_bytes(260, 1040), dtype=torch.uint8, device="cuda") if f8 else None
    g = _grads(p)
    desc = _desc(z, "bf16")
    ws = torch.empty(lib.orbit_gated_norm_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def step():
        lib.orbit_gated_norm_fwd(desc, P, D["x"], D["f"], store, y, h, stats)
        lib.orbit_gated_norm_bwd(desc, P, None if f8 else D["f"], store, y, stats, D["dh"], D["dy"], dx, df, g, 0, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outs = [y, h, stats, dx, df, *g.values()]
    for _ in range(4):
        for k in D:
            D[k].copy_(torch.randn(260, 1040, generator=gen).to(torch.bfloat16))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
