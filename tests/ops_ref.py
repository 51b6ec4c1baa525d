"""64-bit references of the 8-bit activation store and the gated norms."""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24              # half a step of float32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": 0, "bf16": 1}
GROUP = 32


def store_layout(rows, n):
    at = -(-rows * n // 256) * 256
    groups = -(-n // GROUP)
    return at, groups, -(-(at + rows * groups) // 256) * 256


def act8_ref(x):
    """x [rows, n] float64 -> (codes int8 [rows, n], E uint8 [rows, groups], values float64)."""
    x = np.asarray(x, np.float64)
    rows, n = x.shape
    groups = -(-n // GROUP)
    codes, E, val = np.zeros((rows, n), np.int8), np.zeros((rows, groups), np.uint8), np.full((rows, n), np.nan)
    for g in range(groups):
        t = x[:, g * GROUP:(g + 1) * GROUP]
        top = np.abs(t).max(axis=1)
        fine = np.isfinite(top)
        safe = np.where(fine, top, 0.0)
        m, e = np.frexp(safe)                       # safe = m 2^e, m in [1/2, 1) or 0
        k = e - 7 + (m * 128.0 >= 127.5)            # the smallest step that keeps the codes within 127
        k = np.where(safe > 0, np.clip(k, -126, 121), -126)
        step = np.ldexp(1.0, k)
        with np.errstate(invalid="ignore"):
            q = np.clip(np.rint(t / step[:, None]), -127, 127)
        codes[fine, g * GROUP:(g + 1) * GROUP] = q[fine].astype(np.int8)
        E[:, g] = np.where(fine, k + 133, 0)
        val[:, g * GROUP:(g + 1) * GROUP] = np.where(fine[:, None], q * step[:, None], np.nan)
    return codes, E, val


def gelu_ref(u):
    u = torch.as_tensor(u, dtype=torch.float64)
    return u * 0.5 * torch.erfc(-u / 2.0 ** 0.5)


def ln_ref(t, g, b, eps):
    mu = t.mean(-1, keepdim=True)
    v = ((t - mu) ** 2).mean(-1, keepdim=True)
    return (t - mu) / torch.sqrt(v + eps) * g + b


def gated_norm_ref(z, p, x, f):
    """z: dict rows, n, gate_rows, post_norm, pre_norm, scale, eps; float64 tensors -> y, h (or None)."""
    t = ln_ref(f, p["post_g"], p["post_b"], z["eps"]) if z["post_norm"] else f
    if z["gate_rows"]:
        t = p["gate"].repeat_interleave(z["rows"] // z["gate_rows"], 0) * t
    y = x + z["scale"] * t
    return y, (ln_ref(y, p["pre_g"], p["pre_b"], z["eps"]) if z["pre_norm"] else None)


def gated_norm_grad_ref(z, p, f, y, dh, dy):
    """Gradients by autograd in float64: dx, df and those of the parameters, the pre norm
    taken at the given y and the branch at the given f."""
    p = {k: v.detach().clone().requires_grad_(True) for k, v in p.items()}
    f = f.detach().clone().requires_grad_(True)
    y = y.detach().clone().requires_grad_(True)
    val = (dy * y).sum() if dy is not None else torch.zeros((), dtype=torch.float64)
    if z["pre_norm"]:
        val = val + (dh * ln_ref(y, p["pre_g"], p["pre_b"], z["eps"])).sum()
    val.backward()
    t = y.grad
    branch, _ = gated_norm_ref(dict(z, pre_norm=0), p, torch.zeros_like(f), f)
    (branch * t).sum().backward()
    return t, f.grad, {k: v.grad for k, v in p.items()}


def gated_norm_tol(z, p, x, f, half):
    """Error bounds of y and h: `half` of the output's type for its rounding and float32 arithmetic
    inside. A row's sums run over at most 64 values of a thread, then 8 levels, so a mean is off by at
    most 72 U32 mean|.| and a variance by a few times that relative to itself; 256 U32 covers the
    chain of a norm (mean, variance, reciprocal root, gain and shift) relative to the terms' sizes."""
    K = 256 * U32

    def norm(t, g, b):
        mu = t.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt(((t - mu) ** 2).mean(-1, keepdim=True) + z["eps"])
        th = (t - mu) * r
        return th, r, (th.abs() + r * t.abs().mean(-1, keepdim=True)) * g.abs() + b.abs()

    size = f.abs()
    if z["post_norm"]:
        size = norm(f, p["post_g"], p["post_b"])[2]
    if z["gate_rows"]:
        size = size * p["gate"].abs().repeat_interleave(z["rows"] // z["gate_rows"], 0)
    y, h = gated_norm_ref(z, p, x, f)
    ey = K * (x.abs() + abs(z["scale"]) * size)
    ty = half * y.abs() + ey
    if h is None:
        return y, None, ty, None
    yh, r, sz = norm(y, p["pre_g"], p["pre_b"])
    moved = r * (ey + ey.mean(-1, keepdim=True)) + yh.abs() * r * torch.sqrt((ey ** 2).mean(-1, keepdim=True))
    return y, h, ty, half * h.abs() + K * sz + p["pre_g"].abs() * moved


def gated_norm_grad_tol(z, p, f, y, dh, dy, half):
    """Bounds of dx, df and the parameter gradients' errors: the sizes of the terms of each formula times
    512 U32 for the arithmetic of a row (as above, twice over), and for sums over rows one more U32 per
    row, whatever their order."""
    K = 512 * U32
    rows = z["rows"]

    def norm(t):
        mu = t.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt(((t - mu) ** 2).mean(-1, keepdim=True) + z["eps"])
        return (t - mu) * r, r, r * mu.abs()

    size_t = dy.abs() if dy is not None else torch.zeros_like(f)
    S = (rows + 512) * U32
    tol = {}
    if z["pre_norm"]:
        yh, r, off = norm(y)
        ya = yh.abs() + off
        w = (dh * p["pre_g"]).abs()
        size_t = size_t + r * (w + w.mean(-1, keepdim=True) + ya * (w * ya).mean(-1, keepdim=True))
        tol["pre_g"], tol["pre_b"] = S * (dh.abs() * ya).sum(0), S * dh.abs().sum(0)
    t, df, _ = gated_norm_grad_ref(z, p, f, y, dh, dy)
    size_g = torch.ones_like(f) * abs(z["scale"])
    if z["gate_rows"]:
        size_g = size_g * p["gate"].abs().repeat_interleave(rows // z["gate_rows"], 0)
    w = size_g * size_t

    def per_gate(v):
        return v.reshape(z["gate_rows"], -1, z["n"]).sum(1)

    if z["post_norm"]:
        fh, r, off = norm(f)
        fa = fh.abs() + off
        tol["post_g"], tol["post_b"] = S * (w * fa).sum(0), S * w.sum(0)
        if z["gate_rows"]:
            tol["gate"] = abs(z["scale"]) * S * per_gate(size_t * (fa * p["post_g"].abs() + p["post_b"].abs()))
        w = w * p["post_g"].abs()
        w = r * (w + w.mean(-1, keepdim=True) + fa * (w * fa).mean(-1, keepdim=True))
    elif z["gate_rows"]:
        tol["gate"] = abs(z["scale"]) * S * per_gate(size_t * f.abs())
    return half * t.abs() + K * size_t, half * df.abs() + K * w, tol


# ---------------------------------------------------------------------------
# transformer block with gated norms, and with saved tensors in 8 bits
# ---------------------------------------------------------------------------
def act8_values(t):
    """The values a store of t (float64, last axis the columns) reads back as."""
    return torch.from_numpy(act8_ref(t.reshape(-1, t.shape[-1]).numpy())[2]).reshape(t.shape)


def _heads(t, H):
    B, L, A = t.shape
    return t.reshape(B, L, H, A // H).permute(0, 2, 1, 3)


def _merge(t):
    B, H, L, dh = t.shape
    return t.permute(0, 2, 1, 3).reshape(B, L, H * dh)


def block_ext_forward(x, p, H, z, qk=True, eps=1e-5):
    """x [B, L, d] float64 -> y and what the backward reads (z as in gated_norm_ref)."""
    B, L, d = x.shape
    gn = lambda sub, pre, res, f: gated_norm_ref(
        dict(z, rows=B * L, pre_norm=pre, eps=eps),
        {"gate": p.get(f"gate{sub}"), "post_g": p.get(f"post{sub}_g"), "post_b": p.get(f"post{sub}_b"),
         "pre_g": p["ln2_g"], "pre_b": p["ln2_b"]}, res.reshape(B * L, d), f.reshape(B * L, d))
    c = {"h1": ln_ref(x, p["ln1_g"], p["ln1_b"], eps)}
    c["qkv"] = c["h1"] @ p["w_qkv"] + p["b_qkv"]
    q, k, v = (_heads(t, H) for t in c["qkv"].chunk(3, -1))
    if qk:
        q, k = ln_ref(q, p["qn_g"], p["qn_b"], eps), ln_ref(k, p["kn_g"], p["kn_b"], eps)
    sc = q @ k.transpose(-1, -2).contiguous() / q.shape[-1] ** 0.5
    c["lse"] = torch.logsumexp(sc, -1, keepdim=True)
    c["o"] = _merge(torch.exp(sc - c["lse"]) @ v)
    c["f1"] = c["o"] @ p["w_proj"] + p["b_proj"]
    x1, h2 = gn(1, 1, x, c["f1"])
    c["x1"], c["h2"] = x1.reshape(x.shape), h2.reshape(x.shape)
    c["u"] = c["h2"] @ p["w_fc1"] + p["b_fc1"]
    c["f2"] = gelu_ref(c["u"]) @ p["w_fc2"] + p["b_fc2"]
    return gn(2, 0, c["x1"], c["f2"])[0].reshape(x.shape), c


def block_ext_backward(x, p, H, z, c, dy, keep, qk=True, eps=1e-5):
    """Gradients from the tensors `keep(t)` makes of the forward's (identity: the exact gradients;
    act8_values: those of 8-bit stores). The softmax is that of the kept q and k, and the o of its
    backward their softmax's; f2's statistics are the forward's."""
    B, L, d = x.shape
    T = B * L
    flat = lambda t: t.reshape(T, -1)
    g = {}

    def ln_back(t, gain, dh):
        mu = t.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt(((t - mu) ** 2).mean(-1, keepdim=True) + eps)
        th, w = (t - mu) * r, dh * gain
        n = t.shape[-1]
        return (r * (w - w.mean(-1, keepdim=True) - th * (w * th).mean(-1, keepdim=True)),
                (dh * th).reshape(-1, n).sum(0), dh.reshape(-1, n).sum(0))

    def branch_back(sub, f, t, stats_of):
        """gradient of f through scale gate (LN f): statistics taken from stats_of."""
        gate = torch.ones(1, d, dtype=torch.float64)
        if z["gate_rows"]:
            gate = p[f"gate{sub}"]
        G = gate.shape[0]
        rows = gate.repeat_interleave(T // G, 0)
        w = z["scale"] * rows * t
        if not z["post_norm"]:
            if z["gate_rows"]:
                g[f"gate{sub}"] = z["scale"] * (t * f).reshape(G, -1, d).sum(1)
            return w
        mu = stats_of.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt(((stats_of - mu) ** 2).mean(-1, keepdim=True) + eps)
        fh = (f - mu) * r
        g[f"post{sub}_g"], g[f"post{sub}_b"] = (w * fh).sum(0), w.sum(0)
        if z["gate_rows"]:
            g[f"gate{sub}"] = z["scale"] * (t * (fh * p[f"post{sub}_g"] + p[f"post{sub}_b"])).reshape(G, -1, d).sum(1)
        w = w * p[f"post{sub}_g"]
        return r * (w - w.mean(-1, keepdim=True) - fh * (w * fh).mean(-1, keepdim=True))

    qkv, o, f1, u, f2 = (keep(c[k]) for k in ("qkv", "o", "f1", "u", "f2"))
    # x1 and h2 as formed again from x and the kept f1
    t1 = flat(f1)
    if z["post_norm"]:
        t1 = ln_ref(t1, p["post1_g"], p["post1_b"], eps)
    if z["gate_rows"]:
        t1 = t1 * p["gate1"].repeat_interleave(T // z["gate_rows"], 0)
    x1 = flat(x) + z["scale"] * t1
    h2 = ln_ref(x1, p["ln2_g"], p["ln2_b"], eps)
    dyf = flat(dy)
    df2 = branch_back(2, flat(f2), dyf, flat(c["f2"]))
    ge, uf = gelu_ref(flat(u)), flat(u)
    g["w_fc2"], g["b_fc2"] = ge.t() @ df2, df2.sum(0)
    phi = torch.exp(-uf * uf / 2) / (2 * np.pi) ** 0.5
    du = (df2 @ p["w_fc2"].t()) * (0.5 * torch.erfc(-uf / 2 ** 0.5) + uf * phi)
    g["w_fc1"], g["b_fc1"] = h2.t() @ du, du.sum(0)
    dx1, g["ln2_g"], g["ln2_b"] = ln_back(x1, p["ln2_g"], du @ p["w_fc1"].t())
    dx1 = dx1 + dyf
    df1 = branch_back(1, flat(f1), dx1, flat(f1))
    g["w_proj"], g["b_proj"] = flat(o).t() @ df1, df1.sum(0)
    dO = (df1 @ p["w_proj"].t()).reshape(B, L, -1)
    q0, k0, v = (_heads(t, H) for t in qkv.chunk(3, -1))
    q, k = q0, k0
    if qk:
        q, k = ln_ref(q0, p["qn_g"], p["qn_b"], eps), ln_ref(k0, p["kn_g"], p["kn_b"], eps)
    dh = q.shape[-1]
    P = torch.softmax(q @ k.transpose(-1, -2).contiguous() / dh ** 0.5, -1)
    dOh, oh = _heads(dO, H), P @ v
    dS = P * (dOh @ v.transpose(-1, -2).contiguous() - (dOh * oh).sum(-1, keepdim=True)) / dh ** 0.5
    dq, dk, dv = dS @ k, dS.transpose(-1, -2).contiguous() @ q, P.transpose(-1, -2).contiguous() @ dOh
    for name in ("qn_g", "qn_b", "kn_g", "kn_b"):
        g[name] = torch.zeros(dh, dtype=torch.float64)
    if qk:
        dq, g["qn_g"], g["qn_b"] = ln_back(q0, p["qn_g"], dq)
        dk, g["kn_g"], g["kn_b"] = ln_back(k0, p["kn_g"], dk)
    dqkv = flat(torch.cat([_merge(dq), _merge(dk), _merge(dv)], -1))
    g["w_qkv"], g["b_qkv"] = flat(c["h1"]).t() @ dqkv, dqkv.sum(0)
    dx, g["ln1_g"], g["ln1_b"] = ln_back(flat(x), p["ln1_g"], dqkv @ p["w_qkv"].t())
    return (dx + dx1).reshape(x.shape), g
