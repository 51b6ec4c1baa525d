"""The block with rotary positions and / or 8-bit products, through its entry points and through ViTPass,
against the float64 reference in fp8_ref."""
import numpy as np
import pytest
import torch

import fp8_ref as F
import ops_ref as R
from helpers import TOL, check, host
from paper_2404_14712_amd._lib import BLOCK_FP8_WEIGHTS, BlockDesc, BlockExt, BlockOpt, BlockRope

pytestmark = pytest.mark.gpu

# dtype, B, L, d, heads, head_dim, mlp, qk_norm: ragged token counts, a shard (A != d), no QK norm, one token
CASES = [("f32", 2, 37, 128, 4, 32, 512, 1), ("f32", 1, 70, 256, 2, 64, 264, 0), ("bf16", 2, 37, 256, 4, 64, 1024, 1),
         ("bf16", 1, 300, 512, 2, 128, 512, 1), ("bf16", 2, 45, 512, 4, 64, 520, 0), ("f32", 2, 1, 64, 2, 32, 128, 1)]
EXTS = {"plain": dict(post_norm=0, gate_rows=0, scale=1.0), "gated": dict(post_norm=1, gate_rows=1, scale=0.5),
        "scale": dict(post_norm=0, gate_rows=0, scale=0.25)}


class _Block:
    def __init__(self, lib, case, fp8, rope, ext="plain", seed=0):
        dtype, B, L, d, H, dh, mlp, qk = case
        self.lib, self.case, self.fp8, self.z = lib, case, fp8, EXTS[ext]
        A = H * dh
        g = torch.Generator().manual_seed(100 * seed + d + L)
        dt = R.TORCH[dtype]
        rnd = lambda *s, std=0.05, m=0.0: (torch.randn(*s, generator=g) * std + m).to(dt)
        p = {"w_qkv": rnd(d, 3 * A), "b_qkv": rnd(3 * A), "w_proj": rnd(A, d), "b_proj": rnd(d), "w_fc1": rnd(d, mlp),
             "b_fc1": rnd(mlp), "w_fc2": rnd(mlp, d), "b_fc2": rnd(d)}
        for n, w in (("ln1", d), ("ln2", d), ("qn", dh), ("kn", dh)) + \
                ((("post1", d), ("post2", d)) if self.z["post_norm"] else ()):
            p.update({n + "_g": rnd(w, m=1.0), n + "_b": rnd(w)})
        if self.z["gate_rows"]:
            p.update(gate1=rnd(1, d, std=0.2, m=0.5), gate2=rnd(1, d, std=0.2, m=0.5))
        self.p = p
        self.x, self.dy = rnd(B, L, d, std=1.0), rnd(B, L, d, std=1.0)
        self.rope = None
        if rope:
            axis = [i % 2 for i in range(dh // 2)]
            self.rope = (torch.randn(L, 2, generator=g) * 9, torch.rand(dh // 2, generator=g), axis, rope == "near")
        self.desc = BlockDesc(B, L, d, H, dh, mlp, qk, 1e-5, R.CODE[dtype])
        self.ext = BlockExt(0, self.z["post_norm"], self.z["gate_rows"], self.z["scale"])
        self.P = {k: v.cuda() for k, v in p.items()}
        self.gx, self.gdy = self.x.cuda(), self.dy.cuda()
        self.keep = [None, None]
        r = None
        if rope:
            pos, freq, axis, near = self.rope
            self.keep = [pos.cuda(), freq.cuda()]
            r = BlockRope.of(axis, 2, L, *self.keep, near)
        self.w8 = {} if fp8 else None
        if fp8:
            for n in BLOCK_FP8_WEIGHTS:
                i, o = p[n].shape
                for t, s in (("", (i, o)), ("_t", (o, i))):
                    self.w8[n + t] = torch.empty(lib.orbit_fp8_bytes(*s), dtype=torch.uint8, device="cuda")
                lib.orbit_fp8_pack(R.CODE[dtype], i, o, 128, self.P[n], o, self.w8[n], self.w8[n + "_t"])
        self.opt = BlockOpt.of(r, self.w8)

    def run(self, keep=True, fill=0xFF, accumulate=0, start=0.0):
        lib, a = self.lib, (self.desc, self.ext, self.opt)
        byt = lambda n: torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        ws = byt(lib.orbit_vit_block_opt_workspace_bytes(*a))
        saved = byt(lib.orbit_vit_block_opt_saved_bytes(*a)) if keep else None
        y, dx = torch.full_like(self.gx, 9.0), torch.full_like(self.gx, 9.0)
        g = {k: torch.full(v.shape, start, dtype=torch.float32, device="cuda") for k, v in self.p.items()}
        lib.orbit_vit_block_opt_fwd(*a, self.P, self.gx, y, saved, ws)
        ws.fill_(255 - fill)
        lib.orbit_vit_block_opt_bwd(*a, self.P, self.gx, saved, self.gdy, dx, g, accumulate, ws)
        torch.cuda.synchronize()
        return y, dx, g

    def ref(self, fp8=None):
        P = {k: v.double().requires_grad_(True) for k, v in self.p.items()}
        x = self.x.double().requires_grad_(True)
        y = F.block_ref(x, P, self.case[4], bool(self.case[7]), self.fp8 if fp8 is None else fp8, self.rope, self.z)
        y.backward(self.dy.double())
        return y.detach(), x.grad, {k: torch.zeros_like(v) if v.grad is None else v.grad for k, v in P.items()}


@pytest.mark.parametrize("ext", ["plain", "gated"])
@pytest.mark.parametrize("near", ["half", "near"])
@pytest.mark.parametrize("case", CASES)
def test_block_rope(lib, case, near, ext):
    b = _Block(lib, case, False, near, ext)
    y, dx, g = b.run()
    ry, rdx, rg = b.ref()
    tol = TOL[case[0]]
    check("y", host(y), ry.numpy(), tol)
    check("dx", host(dx), rdx.numpy(), tol)
    floor = rg["ln1_b"].numpy()
    for k in g:
        if case[0] == "bf16" and k in ("qn_g", "qn_b", "kn_g", "kn_b"):
            continue  # sums that nearly cancel: their bf16 storage floor lies at the bound itself
        check(f"d{k}", host(g[k]), rg[k].numpy(), tol, floor_ref=floor)
    y2, dx2, g2 = b.run(keep=False, fill=0)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)


@pytest.mark.parametrize("ext", ["plain", "gated", "scale"])
@pytest.mark.parametrize("rope", [None, "half"])
@pytest.mark.parametrize("case", CASES)
def test_block_fp8(lib, case, rope, ext):
    """The 64-bit formulas with their 8-bit products. What the codes' rounding does to a tensor is noise =
    |reference - exact| in the 2-norm. A value whose own rounding differs from the reference's may take the next
    code: in bf16 2^-8 / 2^-4 = 1 / 16 of all, in float32 about 2^-22 / 2^-4 = 2^-18 (70 x 256 values, seven packed
    tensors deep: one in every second block). One moved value, a step of up to 2^-3 of it, changes its row's next
    outputs, sums of n terms, by 2^-3 / sqrt(n) of their size, which moves 2^-3 / sqrt(n) / 2^-4 = 2 / sqrt(n) of
    their codes (1 in 8 at n = 256), and attention carries that into every row: further layers are then rounded
    anew, and two independent roundings differ by sqrt(2) noise. So sqrt(2) noise is allowed beside the type's
    bound in either type; the products themselves are held to their last bits in test_gpu_fp8.py."""
    dtype = case[0]
    b = _Block(lib, case, True, rope, ext, seed=1)
    y, dx, g = b.run()
    ry, rdx, rg = b.ref()
    ey, edx, eg = b.ref(fp8=False)
    share = 2.0 ** 0.5
    floor = float(eg["ln1_b"].norm())
    for k, got, ref, ex in [("y", y, ry, ey), ("x", dx, rdx, edx)] + [(k, g[k], rg[k], eg[k]) for k in g]:
        if k in ("qn_g", "qn_b", "kn_g", "kn_b"):
            continue
        size = max(float(ex.norm()), 1e-3 * floor)
        noise = float((ref - ex).norm())
        err = float((torch.from_numpy(host(got)) - ref).norm())
        assert err <= share * noise + TOL[dtype] * size, (k, err / size, noise / size)
        assert noise <= 0.25 * size, (k, noise / size)
    # the backward that recomputes, scratch contents, and sums added to what was there
    y2, dx2, g2 = b.run(keep=False, fill=0)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)
    _, _, g3 = b.run(accumulate=1, start=0.5)
    for k in g:
        assert (g3[k] - 0.5 - g[k]).abs().max() <= 8 * F.U32 * (0.5 + float(g[k].abs().max())), k


@pytest.mark.parametrize("case", CASES)
def test_block_without_options_is_the_extended_call(lib, case):
    b = _Block(lib, case, False, None, "gated")
    y, dx, g = b.run()
    ws = torch.empty(lib.orbit_vit_block_ext_workspace_bytes(b.desc, b.ext), dtype=torch.uint8, device="cuda")
    saved = torch.empty(lib.orbit_vit_block_ext_saved_bytes(b.desc, b.ext), dtype=torch.uint8, device="cuda")
    y2, dx2 = torch.empty_like(y), torch.empty_like(dx)
    g2 = {k: torch.empty_like(v) for k, v in g.items()}
    lib.orbit_vit_block_ext_fwd(b.desc, b.ext, b.P, b.gx, y2, saved, ws)
    lib.orbit_vit_block_ext_bwd(b.desc, b.ext, b.P, b.gx, saved, b.gdy, dx2, g2, 0, ws)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)


def test_rope_of_zero_frequencies_is_the_block_without(lib):
    """Turned by nothing: the norm's kernel differs from the block's own, the values by their last bits only."""
    case = ("f32", 2, 37, 128, 4, 32, 512, 1)
    b, c = _Block(lib, case, False, "half"), _Block(lib, case, False, None)
    b.keep[1].zero_()
    c.P = b.P = {k: v for k, v in b.P.items()}
    c.gx, c.gdy = b.gx, b.gdy
    for got, want in zip(b.run()[:2], c.run()[:2]):
        assert float((got - want).norm()) <= 1e-5 * float(want.norm())


def test_block_graph(lib):
    """Forward and backward with both options captured, replayed with eager work in between."""
    b = _Block(lib, ("bf16", 2, 100, 256, 4, 64, 512, 1), True, "half", "gated", seed=2)
    a = (b.desc, b.ext, b.opt)
    ws = torch.empty(lib.orbit_vit_block_opt_workspace_bytes(*a), dtype=torch.uint8, device="cuda")
    saved = torch.empty(lib.orbit_vit_block_opt_saved_bytes(*a), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(b.gx), torch.empty_like(b.gx)
    g = {k: torch.zeros(v.shape, device="cuda") for k, v in b.p.items()}

    def step():
        for n in BLOCK_FP8_WEIGHTS:
            i, o = b.p[n].shape
            lib.orbit_fp8_pack(1, i, o, 128, b.P[n], o, b.w8[n], b.w8[n + "_t"])
        lib.orbit_vit_block_opt_fwd(*a, b.P, b.gx, y, saved, ws)
        lib.orbit_vit_block_opt_bwd(*a, b.P, b.gx, saved, b.gdy, dx, g, 0, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outs = [y, dx, *g.values()]
    gen = torch.Generator().manual_seed(3)
    for _ in range(3):
        b.gx.copy_(torch.randn(b.gx.shape, generator=gen).to(b.gx.dtype))
        b.P["w_fc1"].copy_((torch.randn(b.P["w_fc1"].shape, generator=gen) * 0.05).to(b.gx.dtype))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, outs))


def _model(lib, checkpoint=False, fp8=False, rope=False):
    import synth
    from paper_2404_14712_amd.model import PassDims, ViTPass, grid_rope
    c = synth.CONFIGS["tiny"]
    D = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    P = lambda q: {k: (None if v is None else D(v)) for k, v in q.items()}
    dims = PassDims(mode="full", dtype="f32", B=c.B, L=c.L, d=c.d, blocks=c.blocks, heads=c.heads, head_dim=c.head_dim,
                    mlp=c.mlp, V=c.V, grid=c.grid, agg_heads=c.agg_heads, agg_head_dim=c.agg_head_dim)
    params = {"embed": P(synth.embed_params(c)), "agg": P(synth.agg_params(c)), "head": P(synth.head_params(c)),
              "blocks": [P(synth.block_params(c, i)) for i in range(c.blocks)]}
    r = grid_rope(c.grid[0] // 4, c.grid[1] // 4, c.head_dim) if rope else None
    vp = ViTPass(lib, dims, params, checkpoint=checkpoint, fp8=fp8, rope=r)
    run = lambda: vp.forward_backward({"img": D(synth.image(c)), "tgt": D(synth.target(c))})
    loss = float(run().item())
    flat = lambda: torch.cat([v.flatten() for part in ("embed", "agg", "head") for v in vp.grads[part].values()] +
                             [v.flatten() for b in vp.grads["blocks"] for v in b.values()]).double()
    return vp, run, loss, flat


def test_model_pass(lib):
    """The whole model with either and both: recomputing gives the same bits, 8-bit products turn the gradient by
    their rounding (2^-4 / sqrt(3) of a value at most, of random sign, several layers deep), rotary positions matter."""
    _, _, l0, g0 = _model(lib)
    for fp8, rope in ((True, False), (False, True), (True, True)):
        _, _, l1, g1 = _model(lib, False, fp8, rope)
        _, _, l2, g2 = _model(lib, True, fp8, rope)
        assert l1 == l2 and torch.equal(g1(), g2())
        d = float((g1() - g0()).norm() / g0().norm())
        assert 0 < d < 0.25 if not rope else d > 0, d
    with pytest.raises(ValueError, match="act8"):
        _model(lib, "act8", True)


def test_model_pass_takes_new_weights(lib):
    """The gradient is that of the weights as they are at the call (the stores are packed by every pass)."""
    vp, run, l0, flat = _model(lib, fp8=True, rope=True)
    w = vp.params["blocks"][0]["w_fc1"]
    before = w.clone()
    w.mul_(1.5)
    l1 = float(run().item())
    assert l1 != l0
    w.copy_(before)
    assert float(run().item()) == l0


def test_full_size_block(lib):
    """A 115M-scale block with both options: recompute, and against the same block in full precision."""
    case = ("bf16", 1, 2048, 1024, 16, 64, 4096, 1)
    b, c = _Block(lib, case, True, "half"), _Block(lib, case, False, "half")
    y, dx, g = b.run()
    y2, dx2, g2 = b.run(keep=False)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)
    yf, dxf, gf = c.run()
    # e4m3 rounds a value by 2^-4 at most, 2.6% in the root mean square; both operands, a few products deep
    for k, u, v in [("y", y, yf), ("dx", dx, dxf)] + [(k, g[k], gf[k]) for k in g if not k.startswith(("qn", "kn"))]:
        if k == "b_qkv":
            continue  # its key part vanishes but for rounding
        assert float((u.double() - v.double()).norm()) <= 0.15 * float(v.double().norm()), k


def test_block_fp8_of_many_tokens(lib):
    """Enough tokens that every product of the block takes the tiles for large ones, with each of their epilogues:
    the samples are the same in parts that take the small tiles. Sums in another order round some bf16 values to
    their neighbours, 2^-8 away, and such a value takes the next code one time in 2^-4 / 2^-8 = 16, moving by up to
    2^-3. Were every value so moved, that is 2^-3 / sqrt(16) = 2^-5 in the root mean square for an operand, and a row
    passes four products forward and four back with two operands that moved at most: sqrt(16) 2^-5 = 2^-3. A row
    that were wrong or lost differs by its own size."""
    case = ("bf16", 48, 257, 1024, 16, 64, 4096, 1)
    big = _Block(lib, case, True, None)
    y, dx, g = big.run()
    part = _Block(lib, (case[0], 6) + case[2:], True, None)
    part.P, part.w8, part.opt = big.P, big.w8, big.opt
    rows = lambda t: t.double().norm(dim=-1)
    total = {k: torch.zeros_like(v) for k, v in g.items()}
    for i in range(0, 48, 6):
        part.gx, part.gdy = big.gx[i:i + 6].contiguous(), big.gdy[i:i + 6].contiguous()
        py, pdx, pg = part.run()
        for got, want in ((y[i:i + 6], py), (dx[i:i + 6], pdx)):
            assert (rows(got.double() - want.double()) <= 2.0 ** -3 * rows(want)).all()
        for k in total:
            total[k] += pg[k]
    for k in g:
        if k not in ("b_qkv", "qn_g", "qn_b", "kn_g", "kn_b"):  # sums that cancel
            assert float((g[k] - total[k]).norm()) <= 2.0 ** -3 * float(total[k].norm()), k


def test_block_fp8_of_many_float32_tokens(lib):
    """The same samples in float32, where the products of all four layers have more than 512 tiles of 128 x 128 (97 x 8
    at the least) and those of the parts have not (13 x 32 at the most). The bound is the one above: a float32 sum in
    another order moves few values to the next code at first (2^-22 / 2^-4 = 2^-18 of them), but a row that holds one
    is 2^-3 / sqrt(1024) = 2^-8 of its size off, as a bf16 rounding is, and goes on as such a row does."""
    case = ("f32", 48, 257, 1024, 16, 64, 4096, 1)
    big = _Block(lib, case, True, None)
    y, dx, g = big.run()
    part = _Block(lib, (case[0], 6) + case[2:], True, None)
    part.P, part.w8, part.opt = big.P, big.w8, big.opt
    rows = lambda t: t.double().norm(dim=-1)
    total = {k: torch.zeros_like(v) for k, v in g.items()}
    for i in range(0, 48, 6):
        part.gx, part.gdy = big.gx[i:i + 6].contiguous(), big.gdy[i:i + 6].contiguous()
        py, pdx, pg = part.run()
        for got, want in ((y[i:i + 6], py), (dx[i:i + 6], pdx)):
            assert (rows(got.double() - want.double()) <= 2.0 ** -3 * rows(want)).all()
        for k in total:
            total[k] += pg[k]
    for k in g:
        if k not in ("b_qkv", "qn_g", "qn_b", "kn_g", "kn_b"):  # sums that cancel
            assert float((g[k] - total[k]).norm()) <= 2.0 ** -3 * float(total[k].norm()), k


def _qk_terms(b, fp8):
    """What each token and head adds to the gradients of the norms of q and k, float64 [tokens, heads, head_dim]."""
    dtype, B, L, d, H, dh, mlp, qk = b.case
    P = {k: v.double() for k, v in b.p.items()}
    P.update({k: P[k].expand(B * L, H, dh).clone().requires_grad_(True) for k in ("qn_g", "qn_b", "kn_g", "kn_b")})
    y = F.block_ref(b.x.double(), P, H, True, fp8, b.rope, b.z)
    y.backward(b.dy.double())
    return {k: P[k].grad for k in ("qn_g", "qn_b", "kn_g", "kn_b")}


@pytest.mark.parametrize("fp8,rope", [(False, "half"), (False, "near"), (True, None), (True, "half")])
@pytest.mark.parametrize("case", [c for c in CASES if c[7]])
def test_gradients_of_the_norms_of_q_and_k(lib, case, fp8, rope):
    """Sums over tokens and heads whose terms nearly cancel, so that they are held to the terms: roundings of terms
    are independent and add in squares, each of at most the type's bound of its size. 8-bit codes move a term by
    noise = |reference - exact|, two independent roundings by sqrt(2) of that. The bounds are four and twice those: a
    sum over 32 columns and more is off by a quarter more than expected at most. A gradient that were missing or of
    another sign differs by about sqrt(sum of the squares of its terms)."""
    b = _Block(lib, case, fp8, rope, seed=3)
    _, _, g = b.run()
    ref, ex = _qk_terms(b, fp8), _qk_terms(b, False)
    floor = float(b.ref(fp8=False)[2]["ln1_b"].norm())
    for k in ref:
        got = torch.from_numpy(host(g[k]))
        err = float((got - ref[k].sum((0, 1))).norm())
        size, noise = float(ex[k].norm()), float((ref[k] - ex[k]).norm())
        if size <= 1e-9 * floor:  # a softmax of one key
            assert err <= TOL[case[0]] * floor, (k, err / floor)
        else:
            assert err <= 4 * TOL[case[0]] * size + 2 * 2.0 ** 0.5 * noise, (k, err / size, noise / size)


@pytest.mark.parametrize("ext", ["plain", "scale", "gate"])
@pytest.mark.parametrize("case", CASES)
def test_block_rope_act8(lib, case, ext):
    """Rotary positions with the saved tensors in 8 bits: the forward as without the stores, bit for bit, and the
    gradients of the formulas at the stored values (each store passes the gradient straight through). A value whose
    own rounding differs from the reference's may be stored a step aside: half of max|reference - exact| is allowed
    for that in float32, three halves in bf16, beside the type's bound."""
    dtype, B, L, d, H, dh, mlp, qk = case
    b = _Block(lib, case, False, "half", "plain" if ext == "gate" else ext, seed=4)
    if ext == "gate":
        gen = torch.Generator().manual_seed(6)
        b.z = dict(post_norm=0, gate_rows=1, scale=1.0)
        for n in ("gate1", "gate2"):
            b.p[n] = (torch.randn(1, d, generator=gen) * 0.2 + 0.5).to(R.TORCH[dtype])
            b.P[n] = b.p[n].cuda()
    b.ext = BlockExt(0, 0, b.z["gate_rows"], b.z["scale"])
    y0, _, _ = b.run()
    b.ext = BlockExt(1, 0, b.z["gate_rows"], b.z["scale"])
    y, dx, g = b.run()
    assert torch.equal(y, y0)

    def grads(keep):
        """Autograd of the block whose kept tensors take the values keep() makes of the exact ones."""
        P = {k: v.double().requires_grad_(True) for k, v in b.p.items()}
        x = b.x.double().requires_grad_(True)
        T, A = B * L, H * dh
        gate = lambda s: P["gate" + s].expand(T, d) if b.z["gate_rows"] else 1.0
        heads = lambda t: t.reshape(B, L, H, dh).transpose(1, 2).contiguous()

        def chain(kept):
            # exact with kept None; else each kept tensor is replaced, the gradient going on through the formula
            c = {}

            def at(n, t):
                c[n] = t.detach()
                return t if kept is None else t + (keep(kept[n]) - t).detach()

            xf = x.reshape(T, d)
            qkv = at("qkv", R.ln_ref(xf, P["ln1_g"], P["ln1_b"], 1e-5) @ P["w_qkv"] + P["b_qkv"])
            t = qkv[:, :2 * A].reshape(T, 2 * H, dh)
            if qk:
                t = torch.cat([R.ln_ref(t[:, :H], P["qn_g"], P["qn_b"], 1e-5), R.ln_ref(t[:, H:], P["kn_g"], P["kn_b"], 1e-5)], 1)
            t = F.turn(t, *b.rope)
            q, k, v = heads(t[:, :H]), heads(t[:, H:]), heads(qkv[:, 2 * A:])
            o = torch.softmax(q @ k.transpose(-1, -2).contiguous() / dh ** 0.5, -1) @ v
            o = at("o", o.transpose(1, 2).reshape(T, A))
            x1 = xf + b.z["scale"] * gate("1") * at("f1", o @ P["w_proj"] + P["b_proj"])
            u = at("u", R.ln_ref(x1, P["ln2_g"], P["ln2_b"], 1e-5) @ P["w_fc1"] + P["b_fc1"])
            f2 = at("f2", R.gelu_ref(u) @ P["w_fc2"] + P["b_fc2"])
            return x1 + b.z["scale"] * gate("2") * f2, c

        exact, c = chain(None)
        chain(c)[0].backward(b.dy.double().reshape(T, d))
        return exact.detach().reshape(B, L, d), x.grad, {k: torch.zeros_like(v) if v.grad is None else v.grad for k, v in P.items()}

    ry, rdx, rg = grads(R.act8_values)
    _, edx, eg = grads(lambda t: t)
    tol, share = TOL[dtype], 0.5 if dtype == "f32" else 1.5
    check("y", host(y), ry.numpy(), tol)
    floor = float(rg["ln1_b"].abs().max())
    for k, got, ref, exact in [("x", dx, rdx, edx)] + [(k, g[k], rg[k], eg[k]) for k in g]:
        if k in ("qn_g", "qn_b", "kn_g", "kn_b"):
            continue  # sums that nearly cancel
        size = max(float(exact.abs().max()), 1e-3 * floor)
        noise = float((ref - exact).abs().max())
        err = float((torch.from_numpy(host(got)) - ref).abs().max())
        assert err <= share * noise + tol * size, (k, err / size, noise / size)
        assert noise <= 0.1 * size, (k, noise / size)
    # scratch contents do not matter
    _, dx2, g2 = b.run(fill=0)
    assert torch.equal(dx, dx2) and all(torch.equal(g[k], g2[k]) for k in g)


def test_pass_with_rope_against_the_reference(lib):
    """Two blocks of a ViTPass on a grid of 3 x 5 patches, with positions and frequencies written out here."""
    from paper_2404_14712_amd.model import PassDims, ViTPass, grid_rope
    rows, cols, d, H, dh = 3, 5, 128, 2, 64
    case = ("f32", 2, rows * cols, d, H, dh, 256, 1)
    blocks = [_Block(lib, case, False, None, seed=s) for s in (7, 8)]
    z = PassDims(mode="blocks", dtype="f32", B=2, L=rows * cols, d=d, blocks=2, heads=H, head_dim=dh, mlp=256)
    vp = ViTPass(lib, z, {"blocks": [b.P for b in blocks]}, rope=grid_rope(rows, cols, dh, theta=50.0))
    dx = vp.forward_backward({"x": blocks[0].gx, "dy": blocks[0].gdy})
    pos = torch.tensor([[float(r), float(c)] for r in range(rows) for c in range(cols)])
    freq = torch.tensor([50.0 ** (-(i % 16) / 16) for i in range(32)])
    rope = (pos, freq, [0] * 16 + [1] * 16, False)
    x = blocks[0].x.double().requires_grad_(True)
    P = [{k: v.double().requires_grad_(True) for k, v in b.p.items()} for b in blocks]
    y = F.block_ref(F.block_ref(x, P[0], H, True, False, rope), P[1], H, True, False, rope)
    y.backward(blocks[0].dy.double())
    check("y", host(vp.xs[-1]), y.detach().numpy(), TOL["f32"])
    check("dx", host(dx), x.grad.numpy(), TOL["f32"])
    for i, p in enumerate(P):
        for k in p:
            check(f"d{k}", host(vp.grads["blocks"][i][k]), p[k].grad.numpy(), TOL["f32"], floor_ref=p["ln1_b"].grad.numpy())
