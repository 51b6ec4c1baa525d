// LayerNorm over each head of q and k, then rotary positions with several axes,
// in one pass, and its backward. HBM-bound: a head is read and written once.
//
// A token's angles are the same for all its heads, so a block takes a few tokens,
// forms their cosines and sines once in LDS and passes all their heads of q (or of
// k, blockIdx.y) by them. A lane holds 8 columns of a head's first half and the 8
// across, which are whole pairs in either arrangement; dh / 16 lanes (the next
// power of two) hold a head, and its statistics go over them by lane moves.
//
// Angles: a position times a frequency is exact in 64 bits (24 bits each). It is
// brought within pi / 4 there, and the rest's sine and cosine are Taylor sums in
// 32 bits, so that far positions lose nothing.
#include <algorithm>

#include "gemm_args.h"
#include "lanes.h"
#include "rope.h"
#include "rowbuf.h"

namespace orbit {
namespace {

struct RopeArgs {
  const void* src; int64_t lds;
  const void* dy; int64_t lddy;   // backward only
  void* dst; int64_t ldd;         // dx in the backward
  const void *g[2], *b[2];        // gain and shift of q's and of k's norm
  const float *pos, *freq;
  float *mean, *rstd;             // [T, heads of q and k]
  float* part;                    // [2][gridDim.x][2][dh] sums for the gains and shifts
  int T, heads[2], axes, pos_rows, tb;  // tb: tokens of a block
  float eps;
  RopeAxes ax;
};

constexpr int kRopeBwdBlocks = 256;

template <int DH> struct RopeShape {
  static constexpr int CH = DH / 16, G = pow2_ceil(CH), NG = 256 / G, HALF = DH / 2;
};

// sine and cosine of a 64-bit angle, below about 2^50
ORBIT_DEV float2 rope_cos_sin(double x) {
  // n quarter turns off, with pi / 2 in two parts
  const double n = rint(x * 0.63661977236758134308);
  double r = fma(-n, 1.57079632679489661923, x);
  r = fma(-n, 6.12323399573676588614e-17, r);
  const int q = (int)(n - 4.0 * floor(n * 0.25));
  const float f = (float)r, z = f * f;
  // Taylor sums: the first terms left out are 1.8e-9 (sine) and 1.4e-10 of one at pi / 4
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(s, z, 8.3333333e-3f);
  s = fmaf(s, z, -0.16666667f);
  s = fmaf(s * z, f, f);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(c, z, -1.3888889e-3f);
  c = fmaf(c, z, 4.1666667e-2f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.0f);
  const float co = q & 1 ? s : c, si = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -co : co, q >= 2 ? -si : si);
}

// Cosines and sines of a block's tokens t0 .. t0 + nt - 1, nt DH / 2 <= 256 kRopeAngles:
// tab[token][pair]. A thread's loads are issued before its rows' (load), the angles
// formed when these are on their way (store).
constexpr int kRopeAngles = 4;
template <int DH>
struct RopeTable {
  static constexpr int HALF = RopeShape<DH>::HALF;
  float p[kRopeAngles], f[kRopeAngles];
  ORBIT_DEV void load(const RopeArgs& a, int t0, int nt) {
#pragma unroll
    for (int k = 0; k < kRopeAngles; ++k) {
      const int i = threadIdx.x + 256 * k, tl = i / HALF, pair = i - tl * HALF;
      p[k] = f[k] = 0.f;
      if (tl < nt) {
        // every axis' position, so that none waits for the pair's axis
        const float* pr = a.pos + (int64_t)((unsigned)(t0 + tl) % (unsigned)a.pos_rows) * a.axes;
        const int ax = a.ax.axis[pair];
        const float p0 = pr[0], p1 = a.axes > 1 ? pr[1] : 0.f, p2 = a.axes > 2 ? pr[2] : 0.f, p3 = a.axes > 3 ? pr[3] : 0.f;
        f[k] = a.freq[pair];
        p[k] = ax == 0 ? p0 : ax == 1 ? p1 : ax == 2 ? p2 : p3;
      }
    }
  }
  ORBIT_DEV void store(int nt, float2* tab) const {
#pragma unroll
    for (int k = 0; k < kRopeAngles; ++k) {
      const int i = threadIdx.x + 256 * k;
      if (i < nt * HALF) tab[i] = rope_cos_sin((double)p[k] * (double)f[k]);
    }
  }
};

// the 16 values v of a lane (8 of the first half, 8 of the second) turned by the
// token's angles, or back by them
template <int DH, bool NEAR, bool BACK>
ORBIT_DEV void rope_turn(float* v, const float2* tab, int li) {
  if constexpr (NEAR) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 cs = tab[h * (DH / 4) + li * 4 + i];
        const float si = BACK ? -cs.y : cs.y, x = v[8 * h + 2 * i], y = v[8 * h + 2 * i + 1];
        v[8 * h + 2 * i] = x * cs.x - y * si;
        v[8 * h + 2 * i + 1] = x * si + y * cs.x;
      }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 cs = tab[li * 8 + i];
      const float si = BACK ? -cs.y : cs.y, x = v[i], y = v[8 + i];
      v[i] = x * cs.x - y * si;
      v[8 + i] = x * si + y * cs.x;
    }
  }
}

// sum over G consecutive lanes (2, 4, 8 or 16), in each of them
template <int G, int STEP = 0> ORBIT_DEV float group_sum(float v) {
  if constexpr ((1 << STEP) == G) {
    return v;
  } else {
    float a, b;
    wave_pair<STEP>(v, a, b);
    return group_sum<G, STEP + 1>(a + b);
  }
}
template <int CTRL> ORBIT_DEV float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// sum over the wave's lanes with the same place in their group of G
template <int G> ORBIT_DEV float place_sum(float v) {
  if constexpr (G <= 8) v = dpp_add<0x128>(v);  // rotated by 8 within 16 lanes
  if constexpr (G <= 4) v = dpp_add<0x124>(v);  // and by 4
  if constexpr (G <= 2) v = dpp_add<0x4E>(v);   // the quad's other pair
  float a, b;
  wave_pair<4>(v, a, b);
  wave_pair<5>(a + b, a, b);
  return a + b;
}

// one lane's part of a row as stored
template <typename T, int DH>
struct RopeRow {
  U128 lo[sizeof(T) / 2], hi[sizeof(T) / 2];
  ORBIT_DEV void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      lo[i] = ld128(p + i * 4);
      hi[i] = ld128(p + DH / 2 + i * 4);
    }
  }
  ORBIT_DEV void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) lo[i] = hi[i] = zero128();
  }
  ORBIT_DEV void get(float* v) const {
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      unpack(lo[i], v + i * E, (T*)nullptr);
      unpack(hi[i], v + 8 + i * E, (T*)nullptr);
    }
  }
};
template <typename T, int DH> ORBIT_DEV void rope_store(T* p, const float* v) {
  st8(p, v);
  st8(p + DH / 2, v + 8);
}

template <typename T, int DH, bool NORM, bool NEAR>
__global__ void __launch_bounds__(256) rope_fwd_kernel(RopeArgs a) {
  using Z = RopeShape<DH>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float2* tab = reinterpret_cast<float2*>(smem);
  const int li = threadIdx.x % Z::G, grp = threadIdx.x / Z::G;
  const bool lv = li < Z::CH;
  const int sel = blockIdx.y, heads = a.heads[sel], nh = a.heads[0] + a.heads[1], h0 = sel ? a.heads[0] : 0;
  const int t0 = blockIdx.x * a.tb, nt = min(a.tb, a.T - t0), rows = nt * heads;
  float g[16], b[16];
  if (NORM && lv) {
    const T* pg = static_cast<const T*>(a.g[sel]) + li * 8;
    const T* pb = static_cast<const T*>(a.b[sel]) + li * 8;
    ld8(pg, g); ld8(pg + DH / 2, g + 8);
    ld8(pb, b); ld8(pb + DH / 2, b + 8);
  }
  RopeTable<DH> table;
  table.load(a, t0, nt);
  auto fetch = [&](RopeRow<T, DH>& w, int r) {
    w.zero();
    if (r < rows && lv) {
      const int tl = r / heads, j = r - tl * heads;
      w.load(static_cast<const T*>(a.src) + (int64_t)(t0 + tl) * a.lds + (h0 + j) * DH + li * 8);
    }
  };
  RopeRow<T, DH> cur;
  fetch(cur, grp);
  table.store(nt, tab);
  __syncthreads();
  // every group runs the same number of rows (lane moves); the next row's loads are in
  // flight while one is worked on
#pragma unroll 1
  for (int first = 0; first < rows; first += Z::NG) {
    const int r = first + grp;
    RopeRow<T, DH> nxt;
    fetch(nxt, r + Z::NG);
    const bool on = r < rows;
    const int tl = on ? r / heads : 0, j = r - tl * heads;
    float v[16];
    cur.get(v);
    if (NORM) {
      // the mean's own rounding is summed with the squares and taken off too
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += v[i];
      const float m = group_sum<Z::G>(s) / (float)DH;
      float d = 0.f, q = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[i] = lv ? v[i] - m : 0.f;
        d += v[i];
        q = fmaf(v[i], v[i], q);
      }
      d = group_sum<Z::G>(d) / (float)DH;
      q = group_sum<Z::G>(q) / (float)DH;
      const float rs = rsqrtf(fmaxf(fmaf(-d, d, q), 0.f) + a.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = fmaf((v[i] - d) * rs, g[i], b[i]);
      if (on && li == 0 && a.mean) {
        const int64_t at = (int64_t)(t0 + tl) * nh + h0 + j;
        a.mean[at] = m + d;
        a.rstd[at] = rs;
      }
    }
    if (on && lv) {
      rope_turn<DH, NEAR, false>(v, tab + tl * Z::HALF, li);
      rope_store<T, DH>(static_cast<T*>(a.dst) + (int64_t)(t0 + tl) * a.ldd + (h0 + j) * DH + li * 8, v);
    }
    cur = nxt;
  }
}

// dx = rstd (w - mean(w) - x^ mean(w x^)) with w the turned-back gradient times the
// gain; a block walks its share of the tokens and leaves one partial row of each sum
template <typename T, int DH, bool NORM, bool NEAR>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) rope_bwd_kernel(RopeArgs a) {
  using Z = RopeShape<DH>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float2* tab = reinterpret_cast<float2*>(smem);
  const int li = threadIdx.x % Z::G, grp = threadIdx.x / Z::G;
  const bool lv = li < Z::CH;
  const int sel = blockIdx.y, heads = a.heads[sel], nh = a.heads[0] + a.heads[1], h0 = sel ? a.heads[0] : 0;
  float g[16], sg[16], sb[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) g[i] = sg[i] = sb[i] = 0.f;
  if (NORM && lv) {
    const T* pg = static_cast<const T*>(a.g[sel]) + li * 8;
    ld8(pg, g); ld8(pg + DH / 2, g + 8);
  }
  for (int t0 = blockIdx.x * a.tb; t0 < a.T; t0 += gridDim.x * a.tb) {
    const int nt = min(a.tb, a.T - t0), rows = nt * heads;
    struct Row {
      RopeRow<T, DH> d, x;
      float mu, rs;
    };
    // a row's loads; past the last row nothing
    auto fetch = [&](Row& w, int r) {
      w.d.zero();
      w.x.zero();
      w.mu = w.rs = 0.f;
      if (r < rows) {
        const int tl = r / heads, j = r - tl * heads;
        if (NORM) {
          const int64_t at = (int64_t)(t0 + tl) * nh + h0 + j;
          w.mu = a.mean[at];
          w.rs = a.rstd[at];
        }
        if (lv) {
          w.d.load(static_cast<const T*>(a.dy) + (int64_t)(t0 + tl) * a.lddy + (h0 + j) * DH + li * 8);
          if (NORM) w.x.load(static_cast<const T*>(a.src) + (int64_t)(t0 + tl) * a.lds + (h0 + j) * DH + li * 8);
        }
      }
    };
    RopeTable<DH> table;
    table.load(a, t0, nt);
    Row cur;
    fetch(cur, grp);
    __syncthreads();  // the table's readers of the tokens before are done
    table.store(nt, tab);
    __syncthreads();
    // every group runs the same number of rows (lane moves); the next row's loads are
    // in flight while one is worked on
#pragma unroll 1
    for (int first = 0; first < rows; first += Z::NG) {
      const int r = first + grp;
      Row nxt;
      fetch(nxt, r + Z::NG);
      const bool on = r < rows;
      const int tl = on ? r / heads : 0, j = r - tl * heads;
      float v[16];
      cur.d.get(v);
      rope_turn<DH, NEAR, true>(v, tab + tl * Z::HALF, lv ? li : 0);
      if (NORM) {
        float xh[16], s1 = 0.f, s2 = 0.f;
        cur.x.get(xh);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          xh[i] = (xh[i] - cur.mu) * cur.rs;
          sg[i] = fmaf(v[i], xh[i], sg[i]);
          sb[i] += v[i];
          v[i] *= g[i];
          s1 += v[i];
          s2 = fmaf(v[i], xh[i], s2);
        }
        s1 = group_sum<Z::G>(s1) / (float)DH;
        s2 = group_sum<Z::G>(s2) / (float)DH;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = cur.rs * (v[i] - s1 - xh[i] * s2);
      }
      if (on && lv) rope_store<T, DH>(static_cast<T*>(a.dst) + (int64_t)(t0 + tl) * a.ldd + (h0 + j) * DH + li * 8, v);
      cur = nxt;
    }
  }
  if (!NORM) return;
  // the groups of a wave, the waves in order through LDS
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    sg[i] = place_sum<Z::G>(sg[i]);
    sb[i] = place_sum<Z::G>(sb[i]);
  }
  __syncthreads();
  float* sm = reinterpret_cast<float*>(smem);  // [4][2][DH]
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < Z::CH) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = (i >> 3) * (DH / 2) + li * 8 + (i & 7);
      sm[(wave * 2 + 0) * DH + c] = sg[i];
      sm[(wave * 2 + 1) * DH + c] = sb[i];
    }
  }
  __syncthreads();
  float* out = a.part + ((int64_t)sel * gridDim.x + blockIdx.x) * 2 * DH;
  for (int e = threadIdx.x; e < 2 * DH; e += 256) out[e] = (sm[e] + sm[2 * DH + e]) + (sm[4 * DH + e] + sm[6 * DH + e]);
}

// Tokens of a block: about four heads for every group of lanes, no more than the
// table's, and fewer where blocks would be short. Blocks that leave partial sums pay
// for them at their end: 256 each for q and k (4096 tokens of 8 + 8 heads of 128:
// 14.4 us; 512: 15.7, 1024: 18.1), else up to 1024 (8192 tokens of 16 + 16 heads of
// 64 forward: 14.8 us; 512: 16.5).
int rope_tb(const RopeDims& z, bool sums) {
  const int ng = 256 / pow2_ceil(z.dh / 16), most = std::max(z.qh, z.kh);
  const int64_t full = cdiv((int64_t)4 * ng, most), few = cdiv(z.T, sums ? kRopeBwdBlocks : 1024);
  return (int)std::max<int64_t>(1, std::min<int64_t>({full, few, 256 * kRopeAngles / (z.dh / 2)}));
}
int rope_bwd_blocks(const RopeDims& z) {
  const int64_t n = cdiv(z.T, rope_tb(z, z.norm));
  return (int)(z.norm ? std::min<int64_t>(kRopeBwdBlocks, n) : n);
}

RopeArgs rope_args(const RopeDims& z, const RopeParams& p, const float* pos, const float* freq, const void* src,
                   int64_t lds, bool sums) {
  RopeArgs a{};
  a.src = src; a.lds = lds;
  a.g[0] = p.qn_g; a.g[1] = p.kn_g; a.b[0] = p.qn_b; a.b[1] = p.kn_b;
  a.pos = pos; a.freq = freq;
  a.T = z.T; a.heads[0] = z.qh; a.heads[1] = z.kh; a.axes = z.axes; a.pos_rows = z.pos_rows; a.tb = rope_tb(z, sums);
  a.eps = z.eps;
  a.ax = z.ax;
  return a;
}

template <typename T, int DH, bool BWD>
orbit_status rope_run(const RopeDims& z, const RopeArgs& a, hipStream_t s) {
  const double v = (double)z.T * (z.qh + z.kh) * DH;
  KernelInfo ki{BWD ? (sizeof(T) == 2 ? "rope_bwd<bf16>" : "rope_bwd<f32>") : (sizeof(T) == 2 ? "rope_fwd<bf16>" : "rope_fwd<f32>"),
                (BWD ? 20.0 : 14.0) * v, (BWD && z.norm ? 3.0 : 2.0) * v * sizeof(T)};
  const dim3 grid((unsigned)(BWD ? rope_bwd_blocks(z) : (int)cdiv(z.T, a.tb)), 2), block(256);
  const size_t lds = std::max<size_t>((size_t)a.tb * (DH / 2) * sizeof(float2), BWD ? 8 * DH * sizeof(float) : 0);
#define ROPE(N, R) \
  if (z.norm == N && z.near == R) return launch(ki, BWD ? rope_bwd_kernel<T, DH, N, R> : rope_fwd_kernel<T, DH, N, R>, grid, block, lds, s, a)
  ROPE(true, false); ROPE(true, true); ROPE(false, false); ROPE(false, true);
#undef ROPE
  return ORBIT_E_ARG;
}

template <bool BWD>
orbit_status rope_pick(const RopeDims& z, const RopeArgs& a, hipStream_t s) {
#define DIMS(TT)                                                    \
  switch (z.dh) {                                                   \
    case 32: return rope_run<TT, 32, BWD>(z, a, s);                 \
    case 64: return rope_run<TT, 64, BWD>(z, a, s);                 \
    case 128: return rope_run<TT, 128, BWD>(z, a, s);               \
    case 192: return rope_run<TT, 192, BWD>(z, a, s);               \
    case 256: return rope_run<TT, 256, BWD>(z, a, s);               \
  }
  if (z.dt == ORBIT_BF16) { DIMS(bf16) } else { DIMS(float) }
#undef DIMS
  set_error("rope: head_dim %d unsupported", z.dh);
  return ORBIT_E_UNSUPPORTED;
}

}  // namespace

orbit_status rope_fwd(const RopeDims& z, const RopeParams& p, const float* pos, const float* freq, const void* src,
                      int64_t lds, void* dst, int64_t ldd, float* mean, float* rstd, hipStream_t s) {
  RopeArgs a = rope_args(z, p, pos, freq, src, lds, false);
  a.dst = dst; a.ldd = ldd; a.mean = mean; a.rstd = rstd;
  return rope_pick<false>(z, a, s);
}

size_t rope_bwd_ws_bytes(const RopeDims& z) {
  return z.norm ? align_up((size_t)4 * rope_bwd_blocks(z) * z.dh * sizeof(float)) : 0;
}

orbit_status rope_bwd(const RopeDims& z, const RopeParams& p, const float* pos, const float* freq, const void* src,
                      int64_t lds, const float* mean, const float* rstd, const void* dy, int64_t lddy, void* dx,
                      int64_t lddx, const RopeGrads& g, int accumulate, void* ws, ColFinal* fin, hipStream_t s) {
  RopeArgs a = rope_args(z, p, pos, freq, src, lds, z.norm);
  a.dy = dy; a.lddy = lddy; a.dst = dx; a.ldd = lddx;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = static_cast<float*>(ws);
  ORBIT_TRY(rope_pick<true>(z, a, s));
  if (!z.norm) return ORBIT_OK;
  ColFinal own;
  ColFinal& f = fin ? *fin : own;
  const int blocks = rope_bwd_blocks(z);
  float* outs[2][2] = {{g.qn_g, g.qn_b}, {g.kn_g, g.kn_b}};
  for (int k = 0; k < 2; ++k)
    for (int i = 0; i < 2; ++i)
      f.add(a.part + ((int64_t)k * blocks * 2 + i) * z.dh, 2 * z.dh, blocks, z.dh, outs[k][i]);
  return fin ? ORBIT_OK : own.run(accumulate, s);
}

}  // namespace orbit
