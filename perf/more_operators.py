"""Speed of the 8-bit floating-point products and of the rotary positions: what a
block's linear layers and its queries and keys go through, each case one pass
through the public entry points.

A case is a dict of plain sizes. `listed()` gives the named ones, `draw(rng)`
more of the same ranges, `prepare` what a program holds before the call, `run`
one pass (in plain torch, or through the library where `own` is true), `exact`
the same outputs in float64.

The 8-bit floating-point store of a matrix X[rows, n]: blocks of 128 consecutive
columns of a row, or tiles of 128 x 128, share a power of two. With a the bit
pattern of the largest finite |x| of a block as a float32,
E = min(246, max(10, ((a + 0x1fffff) >> 23) - 8)) and the codes are
e4m3(x 2^(127 - E)), nearest even, within +-448 (only the largest float32 values
end there); infinities and NaN become the NaN code. A value reads back as
code 2^(E - 127). In memory: code bytes [rows, n up to a multiple of 128] (zeros
past n), from the next multiple of 256 on one byte E per 128 columns [rows, number
of blocks up to a multiple of 4], the whole a multiple of 256 bytes.

The product of two stores A[M, K], B[N, K]: C = A B^T + bias. A linear layer
y = x W + b with W [in, out] in 128 x 128 tiles: y = Q(x) Q(W) + b,
dx = Q(dy) Q(W)^T, dw = Qt(x)^T Qt(dy), db the column sums of dy, with Q in
blocks along a row and Qt in blocks along the rows of a column.

Rotary positions with several axes: pair i of a head's D values turns by
pos[token % pos_rows, axis[i]] freq[i], after the head's LayerNorm where there is
one. The pair is (i, i + D/2), or (2i, 2i + 1) where `near`.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BLOCK = 128


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _named(name, c):
    return dict(c, name=name) if name else c


def _pack(name, dtype, rows, n, tile, both, pad=0):
    return _named(name, {"kind": "pack", "dtype": dtype, "rows": rows, "n": n, "tile": tile, "both": both, "pad": pad})


def _gemm(name, dtype, M, N, K, f32_out, bias):
    return _named(name, {"kind": "gemm", "dtype": dtype, "M": M, "N": N, "K": K, "f32_out": f32_out, "bias": bias})


def _linear(name, dtype, rows, n_in, n_out):
    return _named(name, {"kind": "linear", "dtype": dtype, "rows": rows, "n_in": n_in, "n_out": n_out})


def _rope(name, kind, dtype, tokens, pos_rows, q_heads, k_heads, head_dim, norm, axes, near):
    return _named(name, {"kind": kind, "dtype": dtype, "tokens": tokens, "pos_rows": pos_rows, "q_heads": q_heads,
                         "k_heads": k_heads, "head_dim": head_dim, "norm": norm, "axes": axes, "near": near})


def listed():
    return [
        # one token's activation packed and read back: what the calls cost
        _pack("pack-token", "bf16", 1, 1024, 1, False),
        # an output gradient of a 10B-scale shard, for the input's and for the
        # weight's gradient: both orientations from one read
        _pack("pack-grad-10b", "bf16", 4096, 8192, 1, True),
        # a float32 weight inside a wider buffer, odd sizes, in 128 x 128 tiles
        _pack("pack-weight-ragged-f32", "f32", 1000, 2056, 128, True, 24),
        # one token through a 115M-scale layer: weights read once
        _gemm("gemm-token", "bf16", 1, 4096, 1024, False, True),
        # a regional crop's token count and odd widths
        _gemm("gemm-ragged", "bf16", 1770, 1000, 2056, True, True),
        # fc1 of a 10B-scale shard, forward
        _gemm("gemm-fc1-10b", "bf16", 4096, 4096, 8192, False, True),
        # a training step of a float32 layer on a small crop
        _linear("linear-ragged-f32", "f32", 150, 1000, 768),
        # a training step of fc1 of a 10B-scale shard: three products
        _linear("linear-fc1-10b", "bf16", 4096, 8192, 4096),
        # a single token of a 115M-scale block
        _rope("rope-token", "rope", "bf16", 1, 1, 16, 16, 64, True, 2, False),
        # q and k of a 115M-scale block: 4 samples of a 32 x 64 patch grid
        _rope("rope-115m", "rope", "bf16", 8192, 2048, 16, 16, 64, True, 2, False),
        # the backward on a 10B-scale shard
        _rope("rope-grad-10b", "rope_grad", "bf16", 4096, 2048, 8, 8, 128, True, 2, False),
        # a sequence of fields in float32: time, latitude and longitude, keys
        # shared by query heads, no norm, neighbouring pairs, ragged counts
        _rope("rope-grad-video-f32", "rope_grad", "f32", 1770, 885, 12, 4, 64, False, 3, True),
    ]


def _logint(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case of the listed ones' ranges."""
    while True:
        kind = rng.choice(["pack", "gemm", "gemm", "linear", "linear", "rope", "rope_grad"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = _logint(rng, 1, 8192)
        if kind == "pack":
            c = _pack(None, dtype, rows, 8 * _logint(rng, 1, 1024), rng.choice([1, 1, 128]), rng.choice([True, False]),
                      8 * rng.choice([0, 0, rng.randint(1, 64)]))
        elif kind == "gemm":
            c = _gemm(None, dtype, rows, 8 * _logint(rng, 16, 1024), _logint(rng, 128, 8192),
                      dtype == "f32" or rng.choice([True, False, False]), rng.choice([True, False]))
        elif kind == "linear":
            c = _linear(None, dtype, rows, 8 * _logint(rng, 32, 1024), 8 * _logint(rng, 32, 1024))
        else:
            dims = [32, 64, 64, 128, 128, 192, 256]
            k_heads = _logint(rng, 1, 32)
            q_heads = k_heads * rng.choice([1, 1, 1, 2, 4])
            samples = rng.choice([1, 1, 2, 4])
            c = _rope(None, kind, dtype, samples * max(1, rows // samples), max(1, rows // samples), q_heads, k_heads,
                      rng.choice(dims), rng.choice([True, True, False]), rng.randint(1, 4), rng.choice([True, False]))
        w = work(c)
        if w["bytes"] <= 4.0e8 and w["flops"] <= 8.2e11:
            return c


# ---------------------------------------------------------------------------
# the store, in integer and elementary operations
# ---------------------------------------------------------------------------
def _blocks(x, tile):
    """[rows, n] -> [row blocks, tile, column blocks, 128], zeros behind the edges."""
    rows, n = x.shape
    x = torch.nn.functional.pad(x, (0, -n % BLOCK, 0, -rows % tile))
    return x.reshape(-(-rows // tile), tile, -(-n // BLOCK), BLOCK)


def _quantise(x, tile):
    """Scaled e4m3 values [rows, n] (NaN where x is not finite) and E [rows, blocks] of a float32 matrix."""
    rows, n = x.shape
    t = _blocks(x, tile)
    fine = torch.isfinite(t)
    top = torch.where(fine, t.abs(), 0.0).amax((1, 3), keepdim=True)
    E = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(10, 246)
    up = ((254 - E) << 23).view(torch.float32)  # 2^(127 - E)
    v = torch.where(fine, (t * up).clamp(-448.0, 448.0), 0.0)
    # the step of e4m3 at |v|: 2^(floor(log2 |v|) - 3), 2^-9 below 2^-6
    k = ((v.abs().view(torch.int32) >> 23) - 127).clamp(min=-6) - 3
    v = torch.round(v * ((127 - k) << 23).view(torch.float32)) * ((127 + k) << 23).view(torch.float32)
    v = torch.where(fine, v, float("nan"))
    E = E.expand(-1, tile, -1, 1).reshape(-1, E.shape[2])[:rows]
    return v.reshape(-1, v.shape[2] * BLOCK)[:rows, :n], E


def _scale(E, n):
    return (E << 23).view(torch.float32).repeat_interleave(BLOCK, 1)[:, :n]  # 2^(E - 127)


def _rounded(x, tile):
    """The values that the store of a float32 matrix stands for."""
    v, E = _quantise(x, tile)
    return v * _scale(E, x.shape[1])


def _places(rows, n):
    """Code columns, offset of the E bytes, E columns, bytes of a store."""
    wide, groups = -(-n // BLOCK) * BLOCK, -(-n // (4 * BLOCK)) * 4
    at = -(-rows * wide // 256) * 256
    return wide, at, groups, -(-(at + rows * groups) // 256) * 256


def _new_store(rows, n):
    return torch.zeros(_places(rows, n)[3], dtype=torch.uint8, device="cuda")


def _store_of(x, tile):
    """A store of a float32 matrix, laid out as the library reads it."""
    rows, n = x.shape
    v, E = _quantise(x, tile)
    wide, at, groups, _ = _places(rows, n)
    s = _new_store(rows, n)
    s[:rows * wide].view(rows, wide)[:, :n] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    s[at:at + rows * groups].view(rows, groups)[:, :E.shape[1]] = E.to(torch.uint8)
    return s


def _parts(store, rows, n):
    """Codes [rows, n] and E [rows, blocks] (int32) of a store."""
    wide, at, groups, _ = _places(rows, n)
    codes = store[:rows * wide].view(rows, wide)[:, :n]
    return codes, store[at:at + rows * groups].view(rows, groups)[:, :wide // BLOCK].to(torch.int32)


def _values(store, rows, n):
    """The float32 values of a store, from its bytes."""
    codes, E = _parts(store, rows, n)
    c = codes.to(torch.int32)
    e, m = (c >> 3) & 15, (c & 7).float()
    # subnormal: m 2^-9; else (8 + m) 2^(e - 10)
    v = torch.where(e == 0, m * 2.0 ** -9, (m + 8.0) * ((e + 117) << 23).view(torch.float32))
    v = torch.where((c & 127) == 127, float("nan"), v)
    return torch.where(c > 127, -v, v) * _scale(E, n)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _code(c):
    return 1 if c["dtype"] == "bf16" else 0


class _Rand:
    """Normal tensors from one seeded generator on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(7919 * int(seed) + 41)

    def __call__(self, shape, dtype, std=1.0, mean=0.0):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(std).add_(mean).to(dtype)

    def activation(self, rows, n, dtype, std=1.0):
        """Normal, a few channels far larger, rows of different size."""
        t = torch.randn((rows, n), generator=self.g, device="cuda", dtype=torch.float32).mul_(std)
        ch = torch.rand(n, generator=self.g, device="cuda")
        t.mul_(torch.where(ch < 0.01, 12.0, 1.0))
        return t.mul_(torch.rand((rows, 1), generator=self.g, device="cuda").add_(0.5)).to(dtype)


def _axis(c):
    """The axis of each of a head's pairs: runs of about equal length."""
    half, axes = c["head_dim"] // 2, c["axes"]
    return [min(i * axes // half, axes - 1) for i in range(half)]


def _frequencies(c):
    """10000^(-j / n) for the j-th of an axis' n pairs."""
    ax = _axis(c)
    out = []
    for i, a in enumerate(ax):
        out.append(10000.0 ** (-(i - ax.index(a)) / ax.count(a)))
    return torch.tensor(out, dtype=torch.float32)


def _positions(c, r):
    """The last axis walks fastest over a grid; the first carries hours of a long record."""
    n, axes = c["pos_rows"], c["axes"]
    side = max(1, int(round(n ** (1.0 / max(1, min(2, axes))))))
    t = torch.arange(n, device="cuda")
    cols = [t % side, t // side % side, t // (side * side)][:axes]
    while len(cols) < axes:
        cols.append(t)
    pos = torch.stack(cols[::-1], -1).float()
    if axes >= 3:
        pos[:, 0] += torch.rand((), generator=r.g, device="cuda").mul_(90000.0).floor_()
    return pos.contiguous()


def prepare(case, seed):
    c, r = case, _Rand(seed)
    dt, kind = _dt(c), c["kind"]
    E = lambda *shape: torch.empty(*shape, dtype=dt, device="cuda")
    F = lambda *shape: torch.zeros(*shape, dtype=torch.float32, device="cuda")
    s = {"c": c}
    if kind == "pack":
        rows, n = c["rows"], c["n"]
        s["x"] = r.activation(rows, n + c["pad"], dt)[:, :n]
        s.update(store=_new_store(rows, n), back=E(rows, n))
        if c["both"]:
            s.update(store_t=_new_store(n, rows), back_t=E(n, -(-rows // 8) * 8)[:, :rows])
    elif kind == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        s["a"] = _store_of(r.activation(M, K, dt).float(), 1)
        s["b"] = _store_of(r((N, K), dt, 0.02).float(), 128)
        s["bias"] = r((N,), dt, 0.1) if c["bias"] else None
        s["out"] = F(M, N) if c["f32_out"] else E(M, N)
    elif kind == "linear":
        rows, i, o = c["rows"], c["n_in"], c["n_out"]
        s["x"], s["dy"] = r.activation(rows, i, dt), r.activation(rows, o, dt, 0.01)
        s["w"] = r((i, o), dt, 0.02)
        s["bias"] = r((o,), dt, 0.1)
        # the weight in both orientations, packed once per optimiser step
        s["w_store"], s["wt_store"] = _store_of(s["w"].float(), 128), _store_of(s["w"].float().t(), 128)
        s.update(y=E(rows, o), dx=E(rows, i), dw=F(i, o), db=F(o))
    else:
        T, D, heads = c["tokens"], c["head_dim"], c["q_heads"] + c["k_heads"]
        s["src"] = r.activation(T, heads * D, dt)
        s["pos"], s["freq"] = _positions(c, r), _frequencies(c).cuda()
        s["p"] = {k: r((D,), dt, 0.02, 1.0 if k.endswith("g") else 0.0) for k in ("qn_g", "qn_b", "kn_g", "kn_b")} \
            if c["norm"] else {}
        s["out"] = E(T, heads * D)
        if kind == "rope":
            s.update(mean=F(T, heads), rstd=F(T, heads))
        else:
            # the forward's statistics, as a program has them
            h = s["src"].double().view(T, heads, D)
            s.update(mean=h.mean(-1).float(), rstd=(h.var(-1, unbiased=False) + EPS).rsqrt().float())
            s["dy"] = r((T, heads * D), dt)
            s["grads"] = {k: F(D) for k in s["p"]}
    return s


# ---------------------------------------------------------------------------
# one pass, in plain operations
# ---------------------------------------------------------------------------
def _turn(c, t, pos, freq, back):
    """[tokens, heads, D] turned by the tokens' angles, or back by them. Angles in 64 bits."""
    half = c["head_dim"] // 2
    angle = pos.double()[:, _axis(c)] * freq.double()
    co, si = torch.cos(angle).to(t.dtype), torch.sin(angle).to(t.dtype)
    rep = t.shape[0] // pos.shape[0]
    co, si = co.repeat(rep, 1)[:, None], si.repeat(rep, 1)[:, None]
    if back:
        si = -si
    if c["near"]:
        a, b = t[..., 0::2], t[..., 1::2]
        return torch.stack([a * co - b * si, a * si + b * co], -1).reshape(t.shape)
    a, b = t[..., :half], t[..., half:]
    return torch.cat([a * co - b * si, a * si + b * co], -1)


def _per_head(c, p, q, k):
    """The queries' parameter for the query heads, the keys' for the key heads: [heads, D]."""
    return torch.cat([p[q].expand(c["q_heads"], -1), p[k].expand(c["k_heads"], -1)])


def _plain(s):
    c = s["c"]
    dt, kind = _dt(c), c["kind"]
    if kind == "pack":
        x = s["x"].float()
        out = {"x": _rounded(x, c["tile"]).to(dt)}
        if c["both"]:
            out["xt"] = _rounded(x.t(), c["tile"]).to(dt)
        return out
    if kind == "gemm":
        y = _values(s["a"], c["M"], c["K"]) @ _values(s["b"], c["N"], c["K"]).t()
        if c["bias"]:
            y = y + s["bias"].float()
        return y if c["f32_out"] else y.to(dt)
    if kind == "linear":
        x, dy = s["x"].float(), s["dy"].float()
        w = _values(s["w_store"], c["n_in"], c["n_out"])
        y = _rounded(x, 1) @ w + s["bias"].float()
        dx = _rounded(dy, 1) @ w.t()
        dw = _rounded(x.t(), 1) @ _rounded(dy.t(), 1).t()
        return {"y": y.to(dt), "dx": dx.to(dt), "dw": dw, "db": dy.double().sum(0).float()}
    T, D, heads = c["tokens"], c["head_dim"], c["q_heads"] + c["k_heads"]
    p = {k: v.float() for k, v in s["p"].items()}
    src = s["src"].float().view(T, heads, D)
    if kind == "rope":
        if c["norm"]:
            d = src - src.mean(-1, keepdim=True)
            src = d * torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
            src = src * _per_head(c, p, "qn_g", "kn_g") + _per_head(c, p, "qn_b", "kn_b")
        return _turn(c, src, s["pos"], s["freq"], False).reshape(T, -1).to(dt)
    g = _turn(c, s["dy"].float().view(T, heads, D), s["pos"], s["freq"], True)
    grads = {}
    if c["norm"]:
        h = (src - s["mean"][..., None]) * s["rstd"][..., None]
        q = c["q_heads"]
        for name, part in (("qn", slice(0, q)), ("kn", slice(q, heads))):
            grads[name + "_g"] = (g[:, part] * h[:, part]).double().sum((0, 1)).float()
            grads[name + "_b"] = g[:, part].double().sum((0, 1)).float()
        w = g * _per_head(c, p, "qn_g", "kn_g")
        g = s["rstd"][..., None] * (w - w.mean(-1, keepdim=True) - h * (w * h).mean(-1, keepdim=True))
    return {"d": g.reshape(T, -1).to(dt), "grads": grads}


# ---------------------------------------------------------------------------
# one pass through the library
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2404_14712_amd import load
    from paper_2404_14712_amd._lib import Fp8LinearDesc, QkRopeDesc

    lib, c = load(), s["c"]
    code, kind = _code(c), c["kind"]
    room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    if kind == "pack":
        rows, n = c["rows"], c["n"]
        lib.orbit_fp8_pack(code, rows, n, c["tile"], s["x"], n + c["pad"], s["store"], s.get("store_t"))
        lib.orbit_fp8_unpack(code, rows, n, s["store"], s["back"], n)
        out = {"x": s["back"]}
        if c["both"]:
            lib.orbit_fp8_unpack(code, n, rows, s["store_t"], s["back_t"], s["back_t"].stride(0))
            out["xt"] = s["back_t"]
        return out
    if kind == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        ws = room(lib.orbit_fp8_gemm_workspace_bytes(M, N, K))
        lib.orbit_fp8_gemm(code, M, N, K, s["a"], s["b"], s["out"], N, c["f32_out"], s["bias"], 0, ws)
        return s["out"]
    if kind == "linear":
        desc = Fp8LinearDesc(c["rows"], c["n_in"], c["n_out"], code)
        saved, ws = room(lib.orbit_fp8_linear_saved_bytes(desc)), room(lib.orbit_fp8_linear_workspace_bytes(desc))
        lib.orbit_fp8_linear_fwd(desc, s["x"], c["n_in"], s["wt_store"], s["bias"], s["y"], c["n_out"], saved, ws)
        lib.orbit_fp8_linear_bwd(desc, saved, s["w_store"], s["dy"], c["n_out"], s["dx"], c["n_in"], s["dw"], s["db"],
                                 0, ws)
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    n = (c["q_heads"] + c["k_heads"]) * c["head_dim"]
    desc = QkRopeDesc.of(c["tokens"], c["q_heads"], c["k_heads"], c["head_dim"], code, axis=_axis(c), axes=c["axes"],
                         pos_rows=c["pos_rows"], norm=c["norm"], near=c["near"], eps=EPS)
    if kind == "rope":
        lib.orbit_qk_rope_fwd(desc, s["p"], s["pos"], s["freq"], s["src"], n, s["out"], n, s["mean"], s["rstd"])
        return s["out"]
    ws = room(lib.orbit_qk_rope_bwd_workspace_bytes(desc))
    lib.orbit_qk_rope_bwd(desc, s["p"], s["pos"], s["freq"], s["src"], n, s["mean"], s["rstd"], s["dy"], n, s["out"], n,
                          s["grads"], 0, ws)
    return {"d": s["out"], "grads": s["grads"]}


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ---------------------------------------------------------------------------
# the work of one pass
# ---------------------------------------------------------------------------
def work(case):
    c, kind = case, case["kind"]
    e = 2.0 if c["dtype"] == "bf16" else 4.0
    if kind == "pack":
        # x read and each store written, each store read and its values written
        v, two = float(c["rows"]) * c["n"], 2.0 if c["both"] else 1.0
        return {"bytes": v * (e + two * (e + 2.0 * (1.0 + 1.0 / BLOCK))), "flops": 8.0 * v}
    if kind == "gemm":
        M, N, K = float(c["M"]), float(c["N"]), float(c["K"])
        by = (M + N) * K * (1.0 + 1.0 / BLOCK) + M * N * (4.0 if c["f32_out"] else e) + (N * e if c["bias"] else 0.0)
        return {"bytes": by, "flops": 2.0 * M * N * K}
    if kind == "linear":
        # x, dy, the weight in both orientations and the bias read; y, dx, dw, db written
        T, i, o = float(c["rows"]), float(c["n_in"]), float(c["n_out"])
        by = 2.0 * T * (i + o) * e + 2.0 * i * o * (1.0 + 1.0 / BLOCK) + o * e + 4.0 * (i + 1.0) * o
        return {"bytes": by, "flops": 6.0 * T * i * o}
    T, D, heads = float(c["tokens"]), float(c["head_dim"]), float(c["q_heads"] + c["k_heads"])
    par = (4.0 * D if c["norm"] else 0.0)
    small = 4.0 * c["pos_rows"] * c["axes"] + 2.0 * D
    if kind == "rope":
        return {"bytes": 2.0 * T * heads * D * e + small + par * e + (8.0 * T * heads if c["norm"] else 0.0),
                "flops": 14.0 * T * heads * D}
    reads = 3.0 if c["norm"] else 2.0
    return {"bytes": reads * T * heads * D * e + small + par * (e + 4.0) + (8.0 * T * heads if c["norm"] else 0.0),
            "flops": 20.0 * T * heads * D}


# ---------------------------------------------------------------------------
# float64 reference
# ---------------------------------------------------------------------------
def _power64(k):
    """2^k in float64, exactly (a power function may be off by a rounding, which decides ties)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4m3_table():
    """The 127 values of the format that are not negative, by code."""
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    return torch.tensor(v[:127], dtype=torch.float64, device="cuda")


def _nearest64(x, tile):
    """The values that the store of a finite float64 matrix stands for: the
    smallest step 2^k, -117 <= k <= 119, with 448 2^k at least a block's largest,
    and of the format's values the nearest, on ties the even code."""
    table = _e4m3_table()
    middle = 0.5 * (table[1:] + table[:-1])
    out = torch.empty_like(x)
    n = x.shape[1]
    for a in range(0, n, BLOCK):
        t = x[:, a:a + BLOCK]
        top = t.abs().amax(1)
        if tile > 1:
            top = torch.cat([part.amax().expand(len(part)) for part in top.split(tile)])
        m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
        step = _power64((e - 9 + (m > 0.875)).clamp(-117, 119))[:, None]
        u = (t.abs() / step).clamp(max=448.0)
        low = torch.bucketize(u, middle)            # first middle not below u
        tie = (low < 126) & (u == middle[low.clamp(max=125)]) & (low % 2 == 1)
        out[:, a:a + BLOCK] = table[low + tie] * step * torch.sign(t)
    return out


def _values64(store, rows, n):
    """The values of a store, from its bytes."""
    codes, E = _parts(store, rows, n)
    v = torch.cat([_e4m3_table(), torch.full((1,), math.nan, dtype=torch.float64, device="cuda")])
    v = torch.cat([v, -v])[codes.long()]
    return v * _power64(E - 127).repeat_interleave(BLOCK, 1)[:, :n]


def _complex_turn(c, t, pos, freq):
    """[tokens, heads, D] float64, each pair as a complex number times e^(i angle)."""
    angle = pos.double()[:, _axis(c)] * freq.double()
    z = torch.polar(torch.ones_like(angle), angle).repeat(t.shape[0] // pos.shape[0], 1)[:, None]
    half = c["head_dim"] // 2
    pair = (t.unflatten(-1, (half, 2)) if c["near"] else t.unflatten(-1, (2, half)).transpose(-1, -2)).contiguous()
    w = torch.view_as_real(torch.view_as_complex(pair) * z)
    return (w if c["near"] else w.transpose(-1, -2)).reshape(t.shape)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    kind = c["kind"]
    if kind == "pack":
        out = {"x": _nearest64(s["x"].double(), c["tile"])}
        if c["both"]:
            out["xt"] = _nearest64(s["x"].double().t(), c["tile"])
        return out
    if kind == "gemm":
        y = _values64(s["a"], c["M"], c["K"]) @ _values64(s["b"], c["N"], c["K"]).t()
        return y + s["bias"].double() if c["bias"] else y
    if kind == "linear":
        x, dy, w = s["x"].double(), s["dy"].double(), _nearest64(s["w"].double(), 128)
        return {"y": _nearest64(x, 1) @ w + s["bias"].double(), "dx": _nearest64(dy, 1) @ w.t(),
                "dw": _nearest64(x.t(), 1) @ _nearest64(dy.t(), 1).t(), "db": dy.sum(0)}
    T, D, q = c["tokens"], c["head_dim"], c["q_heads"]
    p = {k: v.double().requires_grad_(True) for k, v in s["p"].items()}
    src = s["src"].double().view(T, -1, D).requires_grad_(True)

    def whole(t):
        if c["norm"]:
            ln = torch.nn.functional.layer_norm
            t = torch.cat([ln(t[:, :q], (D,), p["qn_g"], p["qn_b"], EPS), ln(t[:, q:], (D,), p["kn_g"], p["kn_b"], EPS)], 1)
        return _complex_turn(c, t, s["pos"], s["freq"]).reshape(T, -1)

    if kind == "rope":
        with torch.no_grad():
            return whole(src)
    (whole(src) * s["dy"].double()).sum().backward()
    return {"d": src.grad.reshape(T, -1), "grads": {k: v.grad for k, v in p.items()}}
