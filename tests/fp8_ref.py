"""Plain float64 references of the 8-bit floating-point stores, products and linear
layers, of the rotary positions and of the block with them (CPU, torch)."""
from __future__ import annotations

import numpy as np
import torch

import ops_ref as R

BLOCK = 128
U32 = 2.0 ** -24          # half a step of float32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # half a step of the type
NAN_CODE = 0x7F


def e4m3_values():
    """The values of codes 0 .. 126."""
    v = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    return np.array(v[:127])


def layout(rows, n):
    """(wide, groups, offset of E, bytes) of a store."""
    wide, groups = -(-n // BLOCK) * BLOCK, -(-n // (4 * BLOCK)) * 4
    at = -(-rows * wide // 256) * 256
    return wide, groups, at, -(-(at + rows * groups) // 256) * 256


def pack_ref(x, tile=1):
    """x [rows, n] (float values) -> codes [rows, n] uint8, E [rows, blocks] uint8, values float64."""
    x = np.asarray(x, np.float64)
    rows, n = x.shape
    nb = -(-n // BLOCK)
    fine = np.isfinite(x)
    mag = np.zeros((-(-rows // tile) * tile, nb * BLOCK))
    mag[:rows, :n] = np.where(fine, np.abs(x), 0.0)
    top = mag.reshape(-1, tile, nb, BLOCK).max((1, 3))
    m, e = np.frexp(top)                      # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    k = np.clip(np.where(top > 0, e - 9 + (m > 0.875), -117), -117, 119)
    k = np.repeat(k, tile, 0)[:rows]
    step = np.ldexp(1.0, np.repeat(k, BLOCK, 1)[:, :n].astype(np.int64))
    u = np.minimum(np.where(fine, np.abs(x), 0.0) / step, 448.0)
    table = e4m3_values()
    mid = 0.5 * (table[1:] + table[:-1])
    low = np.searchsorted(mid, u)             # mid[low - 1] < u <= mid[low]
    tie = (low < 126) & (u == mid[np.minimum(low, 125)]) & (low % 2 == 1)
    code = low + tie
    val = np.where(fine, table[code] * step * np.where(np.signbit(x), -1.0, 1.0), np.nan)
    code = np.where(fine, code | np.where(np.signbit(x), 0x80, 0), NAN_CODE).astype(np.uint8)
    return code, (k + 127).astype(np.uint8), val


def values(t, tile=1):
    """The values that the store of a float64 tensor [rows, n] reads back as."""
    return torch.from_numpy(pack_ref(t.detach().numpy(), tile)[2])


class Fp8Linear(torch.autograd.Function):
    """y = Q(x) Qw + b with the gradients of orbit_fp8_linear_bwd, float64."""

    @staticmethod
    def forward(ctx, x, w, b):
        qw = values(w, BLOCK)
        ctx.save_for_backward(x, qw)
        return values(x) @ qw + b

    @staticmethod
    def backward(ctx, dy):
        x, qw = ctx.saved_tensors
        qxt, qdyt = values(x.t().contiguous()), values(dy.t().contiguous())
        return values(dy) @ qw.t(), qxt @ qdyt.t(), dy.sum(0)


def linear(x, w, b, fp8):
    return Fp8Linear.apply(x, w, b) if fp8 else x @ w + b


def turn(t, pos, freq, axis, near):
    """[tokens, heads, D] float64 turned by the tokens' angles."""
    ang = pos.double()[:, list(axis)] * freq.double()
    ang = ang.repeat(t.shape[0] // pos.shape[0], 1)[:, None]
    c, s = torch.cos(ang), torch.sin(ang)
    D = t.shape[-1]
    a, b = (t[..., 0::2], t[..., 1::2]) if near else (t[..., :D // 2], t[..., D // 2:])
    x, y = a * c - b * s, a * s + b * c
    return torch.stack([x, y], -1).reshape(t.shape) if near else torch.cat([x, y], -1)


def rope_ref(src, p, pos, freq, axis, near, q_heads, norm, eps=1e-5):
    """src [tokens, heads, D] float64 -> the same, normed and turned."""
    if norm:
        q, k = src[:, :q_heads], src[:, q_heads:]
        src = torch.cat([R.ln_ref(q, p["qn_g"], p["qn_b"], eps), R.ln_ref(k, p["kn_g"], p["kn_b"], eps)], 1)
    return turn(src, pos, freq, axis, near)


def pair_sum(t, near):
    """|t| of each value plus that of the other of its pair."""
    t = t.abs()
    D = t.shape[-1]
    if near:
        s = t[..., 0::2] + t[..., 1::2]
        return torch.stack([s, s], -1).reshape(t.shape)
    s = t[..., :D // 2] + t[..., D // 2:]
    return torch.cat([s, s], -1)


def block_ref(x, p, heads, qk, fp8, rope, ext=None, eps=1e-5):
    """The block's output [B, L, d] float64 (autograd gives its gradients). rope: None or (pos, freq, axis, near);
    ext: None or dict(post_norm, gate_rows, scale)."""
    B, L, d = x.shape
    T = B * L
    e = ext or dict(post_norm=0, gate_rows=0, scale=1.0)

    def branch(sub, f):
        if e["post_norm"]:
            f = R.ln_ref(f, p[f"post{sub}_g"], p[f"post{sub}_b"], eps)
        if e["gate_rows"]:
            f = f * p[f"gate{sub}"].repeat_interleave(T // e["gate_rows"], 0)
        return e["scale"] * f

    xf = x.reshape(T, d)
    qkv = linear(R.ln_ref(xf, p["ln1_g"], p["ln1_b"], eps), p["w_qkv"], p["b_qkv"], fp8)
    A = qkv.shape[1] // 3
    D = A // heads
    qk_ = qkv[:, :2 * A].reshape(T, 2 * heads, D)
    if qk:
        qk_ = torch.cat([R.ln_ref(qk_[:, :heads], p["qn_g"], p["qn_b"], eps),
                         R.ln_ref(qk_[:, heads:], p["kn_g"], p["kn_b"], eps)], 1)
    if rope is not None:
        qk_ = turn(qk_, *rope)
    h = lambda t: t.reshape(B, L, heads, D).transpose(1, 2).contiguous()
    q, k, v = h(qk_[:, :heads]), h(qk_[:, heads:]), h(qkv[:, 2 * A:])
    P = torch.softmax(q @ k.transpose(-1, -2).contiguous() / D ** 0.5, -1)
    o = (P @ v).transpose(1, 2).reshape(T, A)
    x1 = xf + branch(1, linear(o, p["w_proj"], p["b_proj"], fp8))
    u = linear(R.ln_ref(x1, p["ln2_g"], p["ln2_b"], eps), p["w_fc1"], p["b_fc1"], fp8)
    y = x1 + branch(2, linear(0.5 * u * torch.erfc(-u * 0.5 ** 0.5), p["w_fc2"], p["b_fc2"], fp8))
    return y.reshape(x.shape)
