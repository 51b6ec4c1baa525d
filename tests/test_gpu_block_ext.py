"""The block with gated norms and / or saved tensors in 8 bits, through its entry
points and through ViTPass, against the 64-bit reference in ops_ref."""
import numpy as np
import pytest
import torch

import ops_ref as R
from helpers import TOL, check, host
from paper_2404_14712_amd._lib import BlockDesc, BlockExt

pytestmark = pytest.mark.gpu

# dtype, B, L, d, heads, head_dim, mlp, qk_norm: ragged token counts, a shard (A != d), no QK norm, one token
CASES = [("f32", 2, 37, 128, 4, 32, 512, 1), ("f32", 1, 70, 256, 2, 64, 264, 0), ("bf16", 2, 37, 256, 4, 64, 1024, 1),
         ("bf16", 1, 600, 512, 2, 128, 512, 1), ("bf16", 2, 45, 512, 4, 64, 520, 0), ("f32", 2, 1, 64, 2, 32, 128, 1)]
EXTS = {"gated": dict(post_norm=1, gates="B", scale=0.5), "gate": dict(post_norm=0, gates=1, scale=1.0),
        "post": dict(post_norm=1, gates=0, scale=1.0), "scale": dict(post_norm=0, gates=0, scale=0.25),
        "plain": dict(post_norm=0, gates=0, scale=1.0)}


def _make(case, ext, seed=0):
    dtype, B, L, d, H, dh, F, qk = case
    A = H * dh
    gates = B if ext["gates"] == "B" else ext["gates"]
    g = torch.Generator().manual_seed(100 * seed + d + L)
    dt = R.TORCH[dtype]
    rnd = lambda *s, std=0.05, m=0.0: (torch.randn(*s, generator=g) * std + m).to(dt)
    p = {"w_qkv": rnd(d, 3 * A), "b_qkv": rnd(3 * A), "w_proj": rnd(A, d), "b_proj": rnd(d), "w_fc1": rnd(d, F),
         "b_fc1": rnd(F), "w_fc2": rnd(F, d), "b_fc2": rnd(d)}
    for n, w in (("ln1", d), ("ln2", d), ("qn", dh), ("kn", dh)) + ((("post1", d), ("post2", d)) if ext["post_norm"] else ()):
        p.update({n + "_g": rnd(w, m=1.0), n + "_b": rnd(w)})
    if gates:
        p.update(gate1=rnd(gates, d, std=0.2, m=0.5), gate2=rnd(gates, d, std=0.2, m=0.5))
    x, dy = rnd(B, L, d, std=1.0), rnd(B, L, d, std=1.0)
    z = dict(n=d, gate_rows=gates, post_norm=ext["post_norm"], scale=ext["scale"])
    return z, p, x, dy


def _desc(case):
    dtype, B, L, d, H, dh, F, qk = case
    return BlockDesc(B, L, d, H, dh, F, qk, 1e-5, R.CODE[dtype])


def _run(lib, case, z, p, x, dy, act8, keep=True, fill=0xFF, accumulate=0, start=0.0):
    """keep: pass `saved` (else the backward recomputes)."""
    desc, ext = _desc(case), BlockExt(act8, z["post_norm"], z["gate_rows"], z["scale"])
    P = {k: v.cuda() for k, v in p.items()}
    x, dy = x.cuda(), dy.cuda()
    byt = lambda n: torch.full((n,), fill, dtype=torch.uint8, device="cuda")
    ws = byt(lib.orbit_vit_block_ext_workspace_bytes(desc, ext))
    saved = byt(lib.orbit_vit_block_ext_saved_bytes(desc, ext)) if keep else None
    y, dx = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    g = {k: torch.full(v.shape, start, dtype=torch.float32, device="cuda") for k, v in p.items()}
    lib.orbit_vit_block_ext_fwd(desc, ext, P, x, y, saved, ws)
    ws.fill_(255 - fill)
    lib.orbit_vit_block_ext_bwd(desc, ext, P, x, saved, dy, dx, g, accumulate, ws)
    torch.cuda.synchronize()
    return y, dx, g


def _ref(case, z, p, x, dy, keep):
    qk = bool(case[7])
    P = {k: v.double() for k, v in p.items()}
    y, c = R.block_ext_forward(x.double(), P, case[4], z, qk)
    dx, g = R.block_ext_backward(x.double(), P, case[4], z, c, dy.double(), keep, qk)
    return y, dx, g


@pytest.mark.parametrize("ext", ["gated", "gate", "post", "scale"])
@pytest.mark.parametrize("case", CASES)
def test_block_gated(lib, case, ext):
    z, p, x, dy = _make(case, EXTS[ext])
    y, dx, g = _run(lib, case, z, p, x, dy, 0)
    ry, rdx, rg = _ref(case, z, p, x, dy, lambda t: t)
    tol = TOL[case[0]]
    check("y", host(y), ry.numpy(), tol)
    check("dx", host(dx), rdx.numpy(), tol)
    floor = rg["ln1_b"].numpy()
    for k in g:
        if case[0] == "bf16" and k in ("qn_g", "qn_b", "kn_g", "kn_b"):
            continue  # sums that nearly cancel: their bf16 storage floor lies at the bound itself
        check(f"d{k}", host(g[k]), rg[k].numpy(), tol, floor_ref=floor)
    # the backward that recomputes, and the sums added to what was there
    y2, dx2, g2 = _run(lib, case, z, p, x, dy, 0, keep=False, fill=0)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)
    if case[0] == "f32":
        _, _, g3 = _run(lib, case, z, p, x, dy, 0, accumulate=1, start=0.5)
        for k in g:
            assert (g3[k] - 0.5 - g[k]).abs().max() <= 4 * R.U32 * (0.5 + float(g[k].abs().max())), k


@pytest.mark.parametrize("case", CASES)
def test_block_plain_is_the_plain_call(lib, case):
    z, p, x, dy = _make(case, EXTS["plain"])
    y, dx, g = _run(lib, case, z, p, x, dy, 0)
    desc = _desc(case)
    P = {k: v.cuda() for k, v in p.items()}
    ws = torch.empty(lib.orbit_vit_block_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    saved = torch.empty(lib.orbit_vit_block_saved_bytes(desc), dtype=torch.uint8, device="cuda")
    y2, dx2 = torch.empty_like(y), torch.empty_like(dx)
    g2 = {k: torch.empty_like(v) for k, v in g.items()}
    lib.orbit_vit_block_fwd(desc, P, x.cuda(), y2, saved, ws)
    lib.orbit_vit_block_bwd(desc, P, x.cuda(), saved, dy.cuda(), dx2, g2, 0, ws)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)


@pytest.mark.parametrize("ext", ["gated", "gate", "plain"])
@pytest.mark.parametrize("case", CASES)
def test_block_act8(lib, case, ext):
    """The forward as without the stores; the backward's gradients those of the 64-bit formulas at the
    stored values. A value whose float32 or bf16 rounding differs from the reference's may be stored one
    step aside: such steps are fewer and no larger than the rounding of all the others, whose effect is
    max|reference at the stores - exact|, so a share of that effect is allowed beside the type's bound:
    half for float32 (about 1 value in 1000 moves), three halves for bf16 (about 1 in 8 moves, and the
    rest carry bf16's own rounding of up to a quarter step)."""
    dtype = case[0]
    z, p, x, dy = _make(case, EXTS[ext], seed=1)
    y, dx, g = _run(lib, case, z, p, x, dy, 1)
    ry, rdx, rg = _ref(case, z, p, x, dy, R.act8_values)
    _, edx, eg = _ref(case, z, p, x, dy, lambda t: t)
    tol = TOL[dtype]
    check("y", host(y), ry.numpy(), tol)
    y0, dx0, g0 = _run(lib, case, z, p, x, dy, 0)
    assert torch.equal(y, y0)
    floor = float(rg["ln1_b"].abs().max())
    share = 0.5 if dtype == "f32" else 1.5
    for k, got, ref, ex in [("x", dx, rdx, edx)] + [(k, g[k], rg[k], eg[k]) for k in g]:
        if k in ("qn_g", "qn_b", "kn_g", "kn_b"):
            continue
        size = max(float(ex.abs().max()), 1e-3 * floor)
        noise = float((ref - ex).abs().max())
        err = float((torch.from_numpy(host(got)) - ref).abs().max())
        assert err <= share * noise + tol * size, (k, err / size, noise / size)
        assert noise <= 0.1 * size, (k, noise / size)
    # recomputing instead of reading the stores: the gradients without their rounding, bit for bit those
    # of the block that keeps full tensors
    _, dx1, g1 = _run(lib, case, z, p, x, dy, 1, keep=False)
    assert torch.equal(dx1, dx0) and all(torch.equal(g1[k], g0[k]) for k in g)
    # scratch contents do not matter
    _, dx4, g4 = _run(lib, case, z, p, x, dy, 1, fill=0)
    assert torch.equal(dx, dx4) and all(torch.equal(g[k], g4[k]) for k in g)


def test_block_act8_graph(lib):
    """Forward and backward captured, replayed with eager work in between."""
    case = ("bf16", 2, 100, 256, 4, 64, 512, 1)
    z, p, x, dy = _make(case, EXTS["gated"], seed=2)
    desc, ext = _desc(case), BlockExt(1, 1, 2, 0.5)
    P, x, dy = {k: v.cuda() for k, v in p.items()}, x.cuda(), dy.cuda()
    ws = torch.empty(lib.orbit_vit_block_ext_workspace_bytes(desc, ext), dtype=torch.uint8, device="cuda")
    saved = torch.empty(lib.orbit_vit_block_ext_saved_bytes(desc, ext), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    g = {k: torch.zeros(v.shape, device="cuda") for k, v in p.items()}

    def step():
        lib.orbit_vit_block_ext_fwd(desc, ext, P, x, y, saved, ws)
        lib.orbit_vit_block_ext_bwd(desc, ext, P, x, saved, dy, dx, g, 0, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outs = [y, dx, *g.values()]
    gen = torch.Generator().manual_seed(3)
    for _ in range(3):
        x.copy_(torch.randn(x.shape, generator=gen).to(x.dtype))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def _model(lib, checkpoint, gated):
    """The tiny float32 model's pass with the given residual form."""
    import dataclasses

    import synth
    from paper_2404_14712_amd.model import PassDims, ViTPass
    c = synth.CONFIGS["tiny"]
    D = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    blocks = [dict(synth.block_params(c, i)) for i in range(c.blocks)]
    dims = PassDims(mode="full", dtype="f32", B=c.B, L=c.L, d=c.d, blocks=c.blocks, heads=c.heads, head_dim=c.head_dim,
                    mlp=c.mlp, V=c.V, grid=c.grid, agg_heads=c.agg_heads, agg_head_dim=c.agg_head_dim)
    if gated:
        dims = dataclasses.replace(dims, post_norm=1, gate_rows=c.B, res_scale=0.5)
        r = np.random.default_rng(4)
        for b in blocks:
            for s in "12":
                b["post%s_g" % s], b["post%s_b" % s] = 1 + 0.1 * r.standard_normal(c.d), 0.1 * r.standard_normal(c.d)
                b["gate%s" % s] = 0.5 + 0.1 * r.standard_normal((c.B, c.d))
    params = {"embed": synth.embed_params(c), "agg": synth.agg_params(c), "head": synth.head_params(c), "blocks": blocks}
    P = lambda q: {k: (None if v is None else D(v)) for k, v in q.items()}
    params = {k: [P(b) for b in v] if k == "blocks" else P(v) for k, v in params.items()}
    vp = ViTPass(lib, dims, params, checkpoint=checkpoint)
    loss = float(vp.forward_backward({"img": D(synth.image(c)), "tgt": D(synth.target(c))}).item())
    flat = torch.cat([v.flatten() for part in ("embed", "agg", "head") for v in vp.grads[part].values()] +
                     [v.flatten() for b in vp.grads["blocks"] for v in b.values()])
    return vp, loss, flat.double()


@pytest.mark.parametrize("gated", [False, True])
def test_model_pass(lib, gated):
    """The whole model: 8-bit stores leave the loss and turn the gradient by their rounding only; recomputing
    gives the gradients of full tensors bit for bit."""
    vp, loss, g = _model(lib, False, gated)
    vr, loss_r, gr = _model(lib, True, gated)
    v8, loss8, g8 = _model(lib, "act8", gated)
    assert loss == loss_r and torch.equal(g, gr)
    assert loss8 == loss
    # each stored value is off by at most 2^-7 of its group's largest, uncorrelated: relative errors well under that
    assert float((g8 - g).norm()) <= 2.0 ** -7 * float(g.norm())
    assert float((g8 - g).norm()) > 0
    assert v8.saved[0].numel() * 3 < vp.saved[0].numel()


def test_model_pass_refuses_unknown_checkpoint(lib):
    with pytest.raises(ValueError, match="checkpoint"):
        _model(lib, "int4", False)
