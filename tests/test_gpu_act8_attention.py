"""The attention's gradients of a block whose saved tensors are in 8 bits: those of the softmax of the
stored q and k, whatever the size of the scores."""
import pytest
import torch

import ops_ref as R
from helpers import TOL, check, host
from paper_2404_14712_amd._lib import BlockDesc, BlockExt

GATED = dict(post_norm=1, gates=2, scale=0.5)
PLAIN = dict(post_norm=0, gates=0, scale=1.0)
# dtype, B, L, heads, head_dim, QK norm, largest score, deviation of a component common to all keys, residual form
CASES = [("f32", 2, 70, 2, 64, 1, 20, 0.0, PLAIN), ("f32", 1, 129, 2, 32, 1, 45, 0.0, GATED),
         ("f32", 2, 70, 2, 64, 1, 20, 2.0, PLAIN), ("f32", 1, 150, 2, 128, 0, 20, 2.0, PLAIN),
         ("f32", 2, 70, 2, 64, 0, 90, 0.0, GATED), ("f32", 1, 200, 2, 64, 0, 450, 0.0, PLAIN),
         ("bf16", 2, 70, 2, 64, 0, 20, 0.0, GATED), ("bf16", 1, 300, 2, 128, 0, 90, 0.0, PLAIN),
         ("bf16", 1, 200, 2, 64, 0, 450, 0.0, PLAIN), ("f32", 3, 1, 2, 32, 1, 6, 2.0, GATED)]


def _scores(qkv, p, H, qk):
    """float64 q, k through their norms: the largest |score| and the largest |q| |k| / sqrt(head_dim)."""
    q, k, _ = (R._heads(t, H) for t in qkv.chunk(3, -1))
    if qk:
        q, k = R.ln_ref(q, p["qn_g"], p["qn_b"], 1e-5), R.ln_ref(k, p["kn_g"], p["kn_b"], 1e-5)
    root = q.shape[-1] ** 0.5
    return (float((q @ k.transpose(-1, -2).contiguous()).abs().max()) / root,
            float(q.norm(dim=-1).max() * k.norm(dim=-1).max()) / root)


def _make(case):
    """A block whose largest |score| is the case's: without the norms q's and k's weights are scaled,
    with them the norms' gains and shifts."""
    dtype, B, L, H, dh, qk, top, common, ext = case
    d, F, A = 128, 264, H * dh
    g = torch.Generator().manual_seed(int(top) + 10 * L + dh)
    dt = R.TORCH[dtype]
    rnd = lambda *s, std=0.05, m=0.0: torch.randn(*s, generator=g) * std + m
    p = {"w_qkv": rnd(d, 3 * A), "b_qkv": rnd(3 * A), "w_proj": rnd(A, d), "b_proj": rnd(d), "w_fc1": rnd(d, F),
         "b_fc1": rnd(F), "w_fc2": rnd(F, d), "b_fc2": rnd(d)}
    for n, w in (("ln1", d), ("ln2", d), ("qn", dh), ("kn", dh)) + ((("post1", d), ("post2", d)) if ext["post_norm"] else ()):
        p.update({n + "_g": rnd(w, m=1.0), n + "_b": rnd(w)})
    if ext["gates"]:
        gates = ext["gates"] if B * L % ext["gates"] == 0 else 1
        p.update(gate1=rnd(gates, d, std=0.2, m=0.5), gate2=rnd(gates, d, std=0.2, m=0.5))
    p["kn_b" if qk else "b_qkv"][slice(None) if qk else slice(A, 2 * A)] += common * torch.randn(dh if qk else A, generator=g)
    x, dy = rnd(B, L, d, std=1.0).to(dt), rnd(B, L, d, std=1.0).to(dt)
    z = dict(n=d, gate_rows=p["gate1"].shape[0] if ext["gates"] else 0, post_norm=ext["post_norm"], scale=ext["scale"])
    h1 = R.ln_ref(x.double(), p["ln1_g"].double(), p["ln1_b"].double(), 1e-5)
    s, _ = _scores(h1 @ p["w_qkv"].double() + p["b_qkv"].double(), {k: v.double() for k, v in p.items()}, H, qk)
    r = (top / s) ** 0.5
    for k in ("qn_g", "qn_b", "kn_g", "kn_b"):
        p[k] *= r if qk else 1.0
    if not qk:
        p["w_qkv"][:, :2 * A] *= r
        p["b_qkv"][:2 * A] *= r
    return z, {k: v.to(dt) for k, v in p.items()}, x, dy


def _stored(lib, case, z, d, F, saved):
    """What the block's stores read back as, in their order: q|k|v, o, f1, u and, with a gate or norm, f2."""
    dtype, B, L, H, dh = case[:5]
    A, T, at, out = H * dh, B * L, 0, []
    for n in (3 * A, A, d, F) + ((d,) if z["post_norm"] or z["gate_rows"] else ()):
        size = R.store_layout(T, n)[2]
        t = torch.empty(T, n, dtype=R.TORCH[dtype], device="cuda")
        lib.orbit_act8_unpack(R.CODE[dtype], T, n, saved[at:at + size], t, n)
        out.append(t.cpu().double().reshape(B, L, n))
        at += size
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_gradients_at_large_scores(lib, case):
    """Every gradient against the 64-bit formulas at the values that the forward's stores hold. Beside the
    type's bound: a score is a float32 sum of head_dim products, off by at most (head_dim + 8) U32 |q| |k| /
    sqrt(head_dim); the probability's and its normaliser's errors together are twice that, and it enters
    dS = P (dP - D) through P and D, and dq, dk, dv once each: four times that of a gradient's size."""
    dtype, B, L, H, dh, qk, top, common, _ = case
    z, p, x, dy = _make(case)
    d, F = x.shape[-1], p["w_fc1"].shape[1]
    desc = BlockDesc(B, L, d, H, dh, F, qk, 1e-5, R.CODE[dtype])
    ext = BlockExt(1, z["post_norm"], z["gate_rows"], z["scale"])
    P = {k: v.cuda() for k, v in p.items()}
    ws = torch.full((lib.orbit_vit_block_ext_workspace_bytes(desc, ext),), 0xFF, dtype=torch.uint8, device="cuda")
    saved = torch.full((lib.orbit_vit_block_ext_saved_bytes(desc, ext),), 0xFF, dtype=torch.uint8, device="cuda")
    xd, dyd = x.cuda(), dy.cuda()
    y, dx = torch.empty_like(xd), torch.empty_like(xd)
    g = {k: torch.zeros(v.shape, device="cuda") for k, v in p.items()}
    lib.orbit_vit_block_ext_fwd(desc, ext, P, xd, y, saved, ws)
    kept = _stored(lib, case, z, d, F, saved)
    ws.fill_(0xFF)
    lib.orbit_vit_block_ext_bwd(desc, ext, P, xd, saved, dyd, dx, g, 0, ws)
    p64 = {k: v.double() for k, v in p.items()}
    _, c = R.block_ext_forward(x.double(), p64, H, z, bool(qk))
    s, size = _scores(kept[0], p64, H, qk)
    assert 0.8 * top <= s <= 1.25 * top
    it = iter(kept)
    rdx, rg = R.block_ext_backward(x.double(), p64, H, z, c, dy.double(), lambda t: next(it, t), bool(qk))
    tol = TOL[dtype] + 4 * 2 * (dh + 8) * R.U32 * size
    floor = rg["ln1_b"].numpy()
    check("dx", host(dx), rdx.numpy(), tol)
    for k in g:
        check(f"d{k}", host(g[k]), rg[k].numpy(), tol, floor_ref=floor)
    if not qk:  # a softmax does not see a shift of all keys: the gradient of their bias vanishes
        A = H * dh
        db = host(g["b_qkv"])
        assert abs(db[A:2 * A]).max() <= tol * abs(db[:A]).max()


@pytest.mark.parametrize("case", [c for c in CASES if not c[5]])
def test_reference_is_of_a_softmax(case):
    """The 64-bit formulas at stored values: the gradient of the keys' bias vanishes."""
    _, _, _, H, dh, _, _, _, _ = case
    z, p, x, dy = _make(case)
    p = {k: v.double() for k, v in p.items()}
    _, c = R.block_ext_forward(x.double(), p, H, z, False)
    _, g = R.block_ext_backward(x.double(), p, H, z, c, dy.double(), R.act8_values, False)
    A = H * dh
    assert float(g["b_qkv"][A:2 * A].abs().max()) <= 1e-9 * float(g["b_qkv"][:A].abs().max())


def test_reference_of_one_token():
    """One token per sample: its probability is 1 whatever is stored, and nothing reaches q and k."""
    case = CASES[-1]
    z, p, x, dy = _make(case)
    p = {k: v.double() for k, v in p.items()}
    _, c = R.block_ext_forward(x.double(), p, case[3], z, True)
    _, g = R.block_ext_backward(x.double(), p, case[3], z, c, dy.double(), R.act8_values, True)
    A = case[3] * case[4]
    assert float(g["b_qkv"][:2 * A].abs().max()) <= 1e-12 * float(g["b_qkv"][2 * A:].abs().max())
    # and v receives the projection's input gradient as it is
    assert torch.allclose(g["b_qkv"][2 * A:], p["w_proj"] @ g["b_proj"], rtol=1e-12, atol=1e-12)
