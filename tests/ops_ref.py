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
