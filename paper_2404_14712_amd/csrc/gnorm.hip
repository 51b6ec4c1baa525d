// Gated norms, forward and backward (gnorm.h). HBM-bound: a row's values stay
// in registers between the passes over it, so every tensor is read and written
// once; statistics and parameter gradients are float32.
#include <algorithm>
#include <type_traits>

#include "act8.h"
#include "gnorm.h"
#include "lanes.h"
#include "rowbuf.h"

namespace orbit {
namespace {

struct GnFwd {
  const void *x, *f, *gate, *post_g, *post_b, *pre_g, *pre_b;
  void *y, *h;
  const uint8_t *fc, *fe;  // the store that f is read from (f null)
  uint8_t *qc, *qe;        // the store that receives f (may be null)
  float* stats;
  int rows, n, groups, rpg, tpr;  // rpg: rows per gate row
  int post, pre;
  float scale, eps;
};

// 8 codes of a store and their group's E
struct Raw8Q {
  u32v2 q;
  uint32_t e;
  ORBIT_DEV void renew() { asm volatile("" : "+v"(q)); }
  ORBIT_DEV void get4(int h, float* f) const { act8_decode4(q[h], e, f); }
  // piece at column col of row r; `on`: a row of n columns is there
  ORBIT_DEV void load(const uint8_t* codes, const uint8_t* exps, int64_t r, int n, int groups, uint32_t col, bool on) {
    const RowBuf bq(codes, r * n, on ? n : 0), be(exps, r * groups, on ? groups : 0);
    q = __builtin_amdgcn_raw_buffer_load_b64(bq.r, col, 0, 0);
    // where nothing is read: any E but 0, which stands for NaN
    e = __builtin_amdgcn_raw_buffer_load_b8(be.r, col >> 5, 0, 0) | (on && col < (uint32_t)n ? 0u : 7u);
  }
};

// A block's G = blockDim / tpr groups of tpr threads take a row each; thread t of
// a group owns the NCH 8-column pieces t + c tpr, so that a quad holds the 32
// columns of a group of the store. Statistics: each thread's own mean (pairwise
// sums of 8 values, pieces and waves as differences from the first: a constant's
// mean is that constant) and squared deviations, merged pairwise over the wave,
// then over the row's waves through LDS with one barrier. The mean is subtracted
// before anything is scaled: v r - mean r would round at the mean's size. y is
// written rounded to the storage type, h and the statistics come from its float32
// value: h then carries one rounding instead of two, and the backward's (rounded
// y - mean) differs from the exact one by y's rounding alone.
//
// Many independent rows per CU (16 waves: at most 128 registers) hide the two
// reductions of a row; 4096 x 8192 in bf16 moves 268 MB in 59 us (4.5 TB/s; a
// copy of that size 5.3). One block per CU that kept the parameter vectors in
// registers and loaded its next row ahead took 85 us, 20 waves with their
// spills 76. STREAM: x and f are loaded non-temporally.
template <typename T, int NCH, bool F8, bool STREAM>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) gnorm_fwd_kernel(GnFwd a) {
  constexpr int AUX = STREAM ? 2 : 0;
  __shared__ float2 red[2][8];  // [norm][wave]
  __shared__ float counts[8];
  const int tpr = a.tpr, G = (int)blockDim.x / tpr, wpg = tpr >> 6;
  const int q = __builtin_amdgcn_readfirstlane((int)threadIdx.x / tpr);
  const int t = (int)threadIdx.x - q * tpr, wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const int n = a.n, row_bytes = n * (int)sizeof(T);
  const int64_t r = (int64_t)blockIdx.x * G + q;
  const bool rv = r < a.rows, post = a.post, pre = a.pre;
  uint32_t col[NCH];
  bool on[NCH];
  int own = 0;  // values of this thread
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = 8u * (uint32_t)(t + c * tpr);
    on[c] = col[c] < (uint32_t)n;
    own += on[c] ? 8 : 0;
  }
  auto row = [&](const void* p, int64_t at, bool there) { return RowBuf(p, at * row_bytes, there ? row_bytes : 0); };
  // an absent gain or gate is 1: its zeros or-ed with the bits of 1
  auto vec = [&](const RowBuf& b, int c, uint32_t bits) {
    Raw8<T> v;
    v.load(b, col[c] * (uint32_t)sizeof(T));
    v.or_bits(bits);
    return v;
  };
  Raw8<T> x[NCH];
  float v[NCH][8];
  {
    std::conditional_t<F8, Raw8Q, Raw8<T>> f[NCH];
    const RowBuf bx = row(a.x, r, rv), bf = row(a.f, F8 ? 0 : r, !F8 && rv);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      x[c].template load<AUX>(bx, col[c] * (uint32_t)sizeof(T));
      if constexpr (F8) f[c].load(a.fc, a.fe, r, n, a.groups, col[c], rv);
      else f[c].template load<AUX>(bf, col[c] * (uint32_t)sizeof(T));
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) f[c].get4(h, v[c] + 4 * h);
  }
  const float inv_own = own ? 1.f / (float)own : 0.f;
  WaveMoments wm;
  wm.init((float)own);
  if (wpg > 1) {
    if (lane == 0) counts[wave] = wm.count;
    __syncthreads();
  }
  if (a.qc) {
    const RowBuf bq(a.qc, r * n, rv ? n : 0), be(a.qe, r * a.groups, rv ? a.groups : 0);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      uint2 codes;
      const uint32_t e = act8_encode(v[c], codes);
      __builtin_amdgcn_raw_buffer_store_b64(u32v2{codes.x, codes.y}, bq.r, col[c], 0, 0);
      // a quad's first lane stores its E; the others' stores fall past the end
      __builtin_amdgcn_raw_buffer_store_b8((uint8_t)e, be.r, (t & 3) == 0 ? col[c] >> 5 : kNoOffset, 0, 0);
    }
  }
  // mean and 1 / sqrt(variance + eps) of the row held as v; k: which norm
  auto moments = [&](int k, float& mu, float& rs) {
    // the pieces' sums as differences from the first's
    float s0 = 0.f, s = 0.f, d = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const float* p = v[c];
      const float sc = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      if (c == 0) s0 = sc;
      else s += on[c] ? sc - s0 : 0.f;
    }
    float m = fmaf(s, inv_own, 0.125f * s0);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if (on[c])
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float e = v[c][i] - m;
          d = fmaf(e, e, d);
        }
    wm.merge(m, d);
    if (wpg > 1) {
      if (lane == 0) red[k][wave] = make_float2(m, d);
      __syncthreads();
      const float m0 = red[k][q * wpg].x;
      float sum = 0.f;
      for (int w = q * wpg; w < (q + 1) * wpg; ++w) sum = fmaf(counts[w], red[k][w].x - m0, sum);
      m = m0 + sum / (float)n;
      d = 0.f;
      for (int w = q * wpg; w < (q + 1) * wpg; ++w) {
        const float2 e = red[k][w];
        d += fmaf(counts[w] * (e.x - m), e.x - m, e.y);
      }
    }
    mu = m;
    rs = rsqrtf(d / (float)n + a.eps);
  };
  float mf = 0.f, rf = 1.f, my = 0.f, ry = 0.f;
  if (post) moments(0, mf, rf);
  const RowBuf by = row(a.y, r, rv);
  const RowBuf bpg = row(a.post_g, 0, post), bpb = row(a.post_b, 0, post);
  const RowBuf bgt = row(a.gate, a.gate && rv ? (int)r / a.rpg : 0, a.gate != nullptr);
  const uint32_t gate_or = a.gate ? 0u : one_bits<T>(), post_or = post ? 0u : one_bits<T>();
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const Raw8<T> pg = vec(bpg, c, post_or), pb = vec(bpb, c, 0u), gt = vec(bgt, c, gate_or);
    Raw8<T> o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x4[4], g4[4], b4[4], t4[4];
      x[c].get4(h, x4);
      pg.get4(h, g4);
      pb.get4(h, b4);
      gt.get4(h, t4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = fmaf((v[c][4 * h + i] - mf) * rf, g4[i], b4[i]);
        v[c][4 * h + i] = fmaf(a.scale * t4[i], p, x4[i]);
      }
      o.put4(h, v[c] + 4 * h);
    }
    o.store(by, col[c] * (uint32_t)sizeof(T));
  }
  if (pre) {
    moments(1, my, ry);
    const RowBuf bh = row(a.h, r, rv), bhg = row(a.pre_g, 0, true), bhb = row(a.pre_b, 0, true);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const Raw8<T> hg = vec(bhg, c, 0u), hb = vec(bhb, c, 0u);
      Raw8<T> o;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float g4[4], b4[4];
        hg.get4(h, g4);
        hb.get4(h, b4);
#pragma unroll
        for (int i = 0; i < 4; ++i) b4[i] = fmaf((v[c][4 * h + i] - my) * ry, g4[i], b4[i]);
        o.put4(h, b4);
      }
      o.store(bh, col[c] * (uint32_t)sizeof(T));
    }
  }
  if (rv && t == 0) *reinterpret_cast<float4*>(a.stats + 4 * r) = make_float4(mf, post ? rf : 0.f, my, ry);
}

// ---- backward ---------------------------------------------------------------
// With yh = (y - my) ry, fh = (f - mf) rf and t the gradient of y:
//   t = dy + ry (dh g - mean(dh g) - yh mean(dh g yh)),   dx = t;
//   w = scale gate t;  df = rf (w pg - mean(w pg) - fh mean(w pg fh)), or w
//   without the post norm.
// Parameter gradients are sums over rows. Those of the post norm and the gate
// all follow from two column sums per gate row, S1 = sum t and S2 = sum t fh
// (t f without the post norm), as the gate is constant over them:
//   d post_b = scale sum_G gate S1, d post_g = scale sum_G gate S2,
//   d gate = scale (pg S2 + pb S1), or scale S2.
// A block takes a chunk of rpb rows of one gate row and stores a partial row
// of each of its four column sums; gnorm_final adds the partials in a fixed
// order.
struct GnBwd {
  const void *f, *y, *dh, *dy, *gate, *post_g, *pre_g;
  const uint8_t *fc, *fe;
  void *dx, *df;
  const float* stats;
  float* part;  // sum k (0: dh, 1: dh yh, 2: t, 3: t fh) of chunk c at part[(k * chunks + c) * n]
  int rows, n, groups, rpg, rpb, cpg, tpr;
  int post, pre;
  float scale;
};

// a thread's part of one row, as loaded
template <typename T, int NCH, bool F8>
struct GnRow {
  int64_t r;
  bool rv;
  float4 st;
  Raw8<T> dh[NCH], y[NCH], dy[NCH];
  std::conditional_t<F8, Raw8Q, Raw8<T>> f[NCH];
};

// A block of 512 threads (one per CU: two waves per SIMD, 256 registers each)
// whose G = blockDim / tpr groups of tpr threads take the chunk's rows in turn;
// thread t of a group owns the NCH 8-column pieces t + c tpr. Every group runs
// the same number of rows, so the barriers line up. The four column sums would
// take half of the register file at full width; the two of the pre norm live in
// LDS. That leaves room for the next row's dh and y (PF, bf16), so that loads are
// in flight all the time; its dy and f follow into the registers of the current
// row's once these are used up. With four pieces a thread that is all 256
// registers, and a few spill (5 where f comes from the store, 1 else). KEEP:
// values stay in registers from their one load; the widest float32 rows are
// loaded again where they are used instead.
template <typename T, int NCH, bool F8, bool KEEP, bool PF>
__global__ void __launch_bounds__(512) gnorm_bwd_kernel(GnBwd a) {
  using Row = GnRow<T, NCH, F8>;
  constexpr int NT = 512;
  // non-temporal loads: bf16 rows only, as a float32 piece's two 16-byte loads
  // share each cache line with those of the neighbours (2048 x 16384 bf16: 136 ->
  // 126 us, float32 1024 x 16384: 167 -> 231)
  constexpr int AUX = sizeof(T) == 2 ? 2 : 0;
  constexpr int PIECES = NT * NCH;
  // wave sums: [turn parity][norm][wave]. By parity, as with one norm alone only
  // one barrier lies between a turn's reads and the next turn's writes
  __shared__ float red[2][2][NT / 64][2];
  // column sums: half h of a thread's piece c of sum k at (2 k + h) PIECES +
  // c NT + thread, so that consecutive lanes touch consecutive 16 bytes and the
  // offsets are constants
  extern __shared__ __attribute__((aligned(16))) f32x4 sums[];
  const int tpr = a.tpr, G = (int)blockDim.x / tpr, wpg = tpr >> 6;
  // a group is whole waves: its number, and with it the row and its statistics,
  // are scalars
  const int q = __builtin_amdgcn_readfirstlane((int)threadIdx.x / tpr);
  const int t = (int)threadIdx.x - q * tpr;
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const int n = a.n, chunks = (int)gridDim.x, row_bytes = n * (int)sizeof(T);
  const int gi = (int)blockIdx.x / a.cpg, ci = (int)blockIdx.x % a.cpg;
  const int64_t r0 = (int64_t)gi * a.rpg + (int64_t)ci * a.rpb;
  const int64_t r1 = min((int64_t)(gi + 1) * a.rpg, r0 + a.rpb);
  const bool post = a.post, pre = a.pre, rf = post || a.gate;  // rf: f is read
  // an absent gain or gate is 1: its zeros or-ed with the bits of 1
  const RowBuf pre_g(a.pre_g, 0, pre ? row_bytes : 0), post_g(a.post_g, 0, post ? row_bytes : 0);
  const RowBuf gate(a.gate, a.gate ? (int64_t)gi * row_bytes : 0, a.gate ? row_bytes : 0);
  const uint32_t gate_or = a.gate ? 0u : one_bits<T>(), post_or = post ? 0u : one_bits<T>();
  uint32_t col[NCH];
  f32x4* const mine = sums + threadIdx.x;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = 8u * (uint32_t)(t + c * tpr);
#pragma unroll
    for (int k = 0; k < 4; ++k) mine[k * PIECES + c * NT] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 s2[NCH][2], s3[NCH][2];  // column sums of t and t fh
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h) s2[c][h] = s3[c][h] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float inv_n = 1.f / (float)n;
  // sums of two values over the row's threads; every thread of the block calls
  auto row_sum2 = [&](int par, int k, float& u, float& v) {
    u = wave_add(u);
    v = wave_add(v);
    if (wpg > 1) {
      if (lane == 0) {
        red[par][k][wave][0] = u;
        red[par][k][wave][1] = v;
      }
      __syncthreads();
      u = v = 0.f;
      for (int w = q * wpg; w < (q + 1) * wpg; ++w) {
        u += red[par][k][w][0];
        v += red[par][k][w][1];
      }
    }
  };
  // Lanes past the row and rows past the chunk read zeros, an absent pre norm a
  // zero dh, an absent post norm f itself (mean 0, 1 / deviation 1): the
  // arithmetic has no branches on these.
  const int steps = (a.rpb + G - 1) / G;
  auto fetch_row = [&](int it, Row& R) {
    R.r = r0 + q + (int64_t)it * G;
    R.rv = it < steps && R.r < r1;
    R.st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (R.rv) R.st = *reinterpret_cast<const float4*>(a.stats + 4 * R.r);
    if (!post) R.st.x = 0.f, R.st.y = 1.f;
    if (!pre) R.st.z = R.st.w = 0.f;
  };
  auto row = [&](const void* v, const Row& R, bool on) {
    return RowBuf(v, R.r * row_bytes, on && R.rv ? row_bytes : 0);
  };
  auto fetch_h = [&](Row& R) {  // what the pre norm needs
    const RowBuf bh = row(a.dh, R, pre), by = row(a.y, R, pre);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      R.dh[c].template load<AUX>(bh, col[c] * (uint32_t)sizeof(T));
      R.y[c].template load<AUX>(by, col[c] * (uint32_t)sizeof(T));
    }
  };
  auto fetch_d = [&](Row& R) {
    const RowBuf b = row(a.dy, R, a.dy != nullptr);
#pragma unroll
    for (int c = 0; c < NCH; ++c) R.dy[c].template load<AUX>(b, col[c] * (uint32_t)sizeof(T));
  };
  auto fetch_f = [&](Row& R) {
    if constexpr (F8) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) R.f[c].load(a.fc, a.fe, R.r, n, a.groups, col[c], rf && R.rv);
    } else {
      const RowBuf b = row(a.f, R, rf);
#pragma unroll
      for (int c = 0; c < NCH; ++c) R.f[c].template load<AUX>(b, col[c] * (uint32_t)sizeof(T));
    }
  };
  Row cur;
  fetch_row(0, cur);
  if (KEEP) {
    fetch_h(cur);
    fetch_d(cur);
    fetch_f(cur);
  }
  for (int it = 0; it < steps; ++it) {
    Row nxt;
    fetch_row(it + 1, nxt);
    if (PF) fetch_h(nxt);
    // yh = (y - my) ry, fh = (f - mf) rr: the mean is subtracted first, so that
    // rows far from zero keep their digits
    const float ry = cur.st.w, my = cur.st.z, rr = cur.st.y, mf = cur.st.x;
    float m1 = 0.f, m2 = 0.f;
    if (pre) {
      if (!KEEP) fetch_h(cur);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        Raw8<T> g;
        g.load(pre_g, col[c] * (uint32_t)sizeof(T));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float d4[4], y4[4], g4[4];
          cur.dh[c].get4(h, d4);
          cur.y[c].get4(h, y4);
          g.get4(h, g4);
          f32x4 u = mine[h * PIECES + c * NT], v = mine[(2 + h) * PIECES + c * NT];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float yh = (y4[i] - my) * ry, w = d4[i] * g4[i];
            u[i] += d4[i];
            v[i] = fmaf(d4[i], yh, v[i]);
            m1 += w;
            m2 = fmaf(w, yh, m2);
          }
          mine[h * PIECES + c * NT] = u;
          mine[(2 + h) * PIECES + c * NT] = v;
        }
        if (KEEP) {
          cur.dh[c].renew();
          cur.y[c].renew();
        }
        if (NCH > 2) __builtin_amdgcn_sched_barrier(0);  // one piece's temporaries at a time
      }
      row_sum2(it & 1, 0, m1, m2);
      m1 *= inv_n;
      m2 *= inv_n;
    }
    if (!KEEP) {
      fetch_h(cur);
      fetch_d(cur);
      fetch_f(cur);
    }
    const float m2r = m2 * ry;  // times y - my
    float w[NCH][8];
    float m3 = 0.f, m4 = 0.f;
    const RowBuf bx = row(a.dx, cur, a.dx != nullptr), bf = row(a.df, cur, a.df != nullptr);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      Raw8<T> g, gg, pg, o;
      g.load(pre_g, col[c] * (uint32_t)sizeof(T));
      gg.load(gate, col[c] * (uint32_t)sizeof(T));
      pg.load(post_g, col[c] * (uint32_t)sizeof(T));
      gg.or_bits(gate_or);
      pg.or_bits(post_or);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float t4[4], d4[4], v4[4], f4[4];
        cur.dy[c].get4(h, t4);
        cur.dh[c].get4(h, d4);
        cur.y[c].get4(h, f4);
        g.get4(h, v4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          t4[i] = fmaf(ry, fmaf(-m2r, f4[i] - my, fmaf(d4[i], v4[i], -m1)), t4[i]);
        o.put4(h, t4);
        cur.f[c].get4(h, f4);
        gg.get4(h, v4);
        pg.get4(h, d4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f4[i] = (f4[i] - mf) * rr;
          s2[c][h][i] += t4[i];
          s3[c][h][i] = fmaf(t4[i], f4[i], s3[c][h][i]);
          t4[i] *= a.scale * v4[i] * d4[i];
          m3 += t4[i];
          m4 = fmaf(t4[i], f4[i], m4);
          w[c][4 * h + i] = t4[i];
        }
      }
      o.store(bx, col[c] * (uint32_t)sizeof(T));
      if (NCH > 2) __builtin_amdgcn_sched_barrier(0);
    }
    if (KEEP && !PF) fetch_h(nxt);
    if (KEEP) fetch_d(nxt);
    if (post) {
      row_sum2(it & 1, 1, m3, m4);
      m3 *= inv_n;
      m4 *= inv_n * rr;  // times f - mf
      if (!KEEP) fetch_f(cur);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      Raw8<T> o;
      if (KEEP) cur.f[c].renew();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float t4[4], f4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t4[i] = w[c][4 * h + i];
        if (post) {
          cur.f[c].get4(h, f4);
#pragma unroll
          for (int i = 0; i < 4; ++i) t4[i] = rr * fmaf(-m4, f4[i] - mf, t4[i] - m3);
        }
        o.put4(h, t4);
      }
      o.store(bf, col[c] * (uint32_t)sizeof(T));
    }
    if (KEEP) fetch_f(nxt);
    cur = nxt;
  }
  // the groups' sums of a column, added in group order by all threads, then a
  // partial row each: the pre norm's, already in LDS, then the others
  auto put = [&](int k) {  // sums k and k + 1
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float* out = a.part + ((int64_t)(k + j) * chunks + blockIdx.x) * n;
      const f32x4* src = sums + 2 * j * PIECES;
      for (int e = (int)threadIdx.x; 4 * e < n; e += (int)blockDim.x) {
        const int p = e >> 1, h = e & 1, c = p / tpr;
        const f32x4* at = src + h * PIECES + c * NT + (p - c * tpr);
        f32x4 v = at[0];
        for (int gq = 1; gq < G; ++gq) v += at[gq * tpr];
        *reinterpret_cast<f32x4*>(out + 4 * e) = v;
      }
    }
  };
  if (pre) put(0);
  if (!rf) return;
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mine[h * PIECES + c * NT] = s2[c][h];
      mine[(2 + h) * PIECES + c * NT] = s3[c][h];
    }
  put(2);
}

struct GnFinal {
  const float* part;  // as GnBwd's
  const void *gate, *post_g, *post_b;
  float *dgate, *dpost_g, *dpost_b, *dpre_g, *dpre_b;
  int n, gates, cpg, pre, post, lanes, accumulate;
  float scale;
};

// Sums of the partial rows: 64 columns (4 per thread) x 64 chunk lanes per
// block, a lane adding every 64th chunk, the lanes' sums added in order.
// Jobs 0 and 1: the pre norm's shift and gain; 2 and 3: the post norm's, each
// chunk weighted by its gate; from 4 on the gate, `lanes` lanes to a gate row.
// With one gate row (or none) job 4 forms the post norm's sums as well, so that
// the partials of t and t fh are read once (16384 columns, 256 chunks: 100 MB
// down to 67). Bound by latency but for the widest rows: a lane's loads are
// issued four at a time.
template <typename T>
__global__ void __launch_bounds__(1024) gnorm_final_kernel(GnFinal a) {
  __shared__ f32x4 red[2][64][16];
  const int e = threadIdx.x % 16, q = threadIdx.x / 16;
  const int tiles = (a.n + 63) / 64, job = (int)blockIdx.x / tiles;
  const int c = ((int)blockIdx.x % tiles) * 64 + 4 * e;
  const bool on = c < a.n;
  const int chunks = a.gates * a.cpg;
  const T* gate = static_cast<const T*>(a.gate);
  const bool one = a.gates == 1;
  if (job < 2 ? !a.pre : job < 4 && (one || !a.post)) return;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto get = [&](const float* p) { return *reinterpret_cast<const f32x4*>(p); };
  auto vec = [&](const void* p, int64_t at) {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f(static_cast<const T*>(p)[at + i]);
    return v;
  };
  auto put = [&](float* o, f32x4 v) {
    if (a.accumulate) v += get(o);
    *reinterpret_cast<f32x4*>(o) = v;
  };
  // sum over the chunks k0, k0 + step, ... < kn of w(k) times the partial rows p
  auto sum = [&](const float* p, int k0, int kn, int step, auto&& w) {
    f32x4 s = zero;
    for (int k = k0; k < kn; k += 4 * step) {
      f32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = on && k + j * step < kn ? w(k + j * step) * get(p + (int64_t)(k + j * step) * a.n) : zero;
#pragma unroll
      for (int j = 0; j < 4; ++j) s += v[j];
    }
    return s;
  };
  auto unit = [](int) { return 1.f; };
  const bool gated = job >= 4;
  const int lanes = gated ? a.lanes : 64, ql = q % lanes;
  const int64_t g = gated ? (int64_t)(job - 4) * (64 / lanes) + q / lanes : 0;
  const bool there = on && (!gated || g < a.gates);
  f32x4 s1 = zero, s2 = zero;
  if (!gated) {
    const float* p = a.part + (int64_t)job * chunks * a.n + c;
    if (job < 2) s1 = sum(p, q, chunks, 64, unit);
    else if (on) s1 = sum(p, q, chunks, 64, [&](int k) { return vec(gate, (int64_t)(k / a.cpg) * a.n + c); });
  } else if (there) {
    const float* p2 = a.part + ((int64_t)3 * chunks + g * a.cpg) * a.n + c;
    s2 = sum(p2, ql, a.cpg, lanes, unit);
    if (a.post) s1 = sum(p2 - (int64_t)chunks * a.n, ql, a.cpg, lanes, unit);
  }
  red[0][q][e] = s1;
  red[1][q][e] = s2;
  __syncthreads();
  // eight lanes' sums at a time, then the eights
  const int span = min(8, lanes);
  if (ql % span == 0) {
    for (int k = 1; k < span; ++k) {
      s1 += red[0][q + k][e];
      s2 += red[1][q + k][e];
    }
    red[0][q][e] = s1;
    red[1][q][e] = s2;
  }
  __syncthreads();
  if (ql != 0 || !there) return;
  for (int k = 8; k < lanes; k += 8) {
    s1 += red[0][q + k][e];
    s2 += red[1][q + k][e];
  }
  if (!gated) {
    if (job >= 2) s1 *= a.scale;
    put((job == 0 ? a.dpre_b : job == 1 ? a.dpre_g : job == 2 ? a.dpost_b : a.dpost_g) + c, s1);
    return;
  }
  if (one && a.post) {
    const f32x4 w = gate ? vec(gate, c) * a.scale : f32x4{a.scale, a.scale, a.scale, a.scale};
    put(a.dpost_g + c, w * s2);
    put(a.dpost_b + c, w * s1);
  }
  if (!gate) return;
  f32x4 v = s2;
  if (a.post) v = vec(a.post_g, c) * s2 + vec(a.post_b, c) * s1;
  put(a.dgate + g * a.n + c, v * a.scale);
}

// The backward's launch shape. A thread owns one, two or four pieces (a row of up
// to 2048 columns is a wave's), three from 8193 to 12288 columns, so that all 512
// threads of a block have some; float32 stays at two up to 8192 columns, which
// its registers hold (4096 x 2048: 61 -> 55 us). A block takes as many rows at
// once as that gives. Chunks: about one per CU, in whole turns of the block's
// groups. From two pieces a thread on a kernel's 147 to 256 registers let one
// block onto a CU, so that more chunks run one after the other and add partial
// rows (bf16 8192 x 1024: 31 us, with 512 chunks 37; two blocks at a time on a CU,
// which would take 128 registers, were not tried); fewer leave CUs idle where rows
// are few (256 x 16384: 45 us, 84 with at least 8 rows a chunk).
// pieces of 8 columns per thread
int gn_pieces(int n) { return n <= 512 ? 1 : n <= 1024 ? 2 : n > 8192 && n <= 12288 ? 3 : 4; }

struct GnShape {
  int nch, tpr, G, rpg, rpb, cpg;
};
GnShape gn_shape(const GnormDims& z) {
  GnShape h{};
  h.nch = z.dt == ORBIT_F32 && z.n > 512 && z.n <= 8192 ? 2 : gn_pieces(z.n);
  h.tpr = (int)(cdiv(cdiv(z.n, 8 * h.nch), 64) * 64);
  h.G = 512 / h.tpr;
  h.rpg = z.rows / std::max(1, z.gates);
  const int turns = std::max(1, (int)(((int64_t)z.rows + 128 * h.G) / (256 * h.G)));
  h.rpb = std::min(h.rpg, turns * h.G);
  h.G = std::min(h.G, h.rpb);
  h.cpg = (int)cdiv(h.rpg, h.rpb);
  return h;
}

// A row of up to 2048 columns is a wave's (one, two or four pieces a thread);
// wider ones take up to 512 threads with four pieces, or three from 8193 to 12288
// columns (2048 x 12288: 50 us, with four pieces on 384 threads 57). Narrow
// rows share blocks of 256 threads. Non-temporal loads in bf16 from 96 MB of x,
// f, y and h on, which the caches would not hold (134 MB: 31.1 -> 29.1 us, 67
// MB: 15.2 -> 16.4).
template <typename T, bool F8>
orbit_status gnorm_fwd_t(GnFwd& a, const KernelInfo& ki, hipStream_t s) {
  const int nch = gn_pieces(a.n);
  a.tpr = (int)(cdiv(cdiv(a.n, 8 * nch), 64) * 64);
  const int G = std::min(std::max(1, 256 / a.tpr), a.rows);
  const bool stream = sizeof(T) == 2 && 8.0 * a.rows * a.n >= 96e6;
  const dim3 grid((unsigned)cdiv(a.rows, G)), block((unsigned)(G * a.tpr));
#define GNF(C)                                                                              \
  return stream ? launch(ki, gnorm_fwd_kernel<T, C, F8, sizeof(T) == 2>, grid, block, 0, s, a) \
                : launch(ki, gnorm_fwd_kernel<T, C, F8, false>, grid, block, 0, s, a)
  switch (nch) {
    case 1: GNF(1);
    case 2: GNF(2);
    case 3: GNF(3);
    default: GNF(4);
  }
#undef GNF
}

}  // namespace

orbit_status gnorm_fwd(const GnormDims& z, const GnormParams& p, const void* x, const void* f, void* store, void* y,
                       void* h, float* stats, hipStream_t s) {
  GnFwd a{};
  a.x = x; a.f = f; a.gate = z.gates ? p.gate : nullptr;
  a.post_g = p.post_g; a.post_b = p.post_b; a.pre_g = p.pre_g; a.pre_b = p.pre_b;
  a.y = y; a.h = h; a.stats = stats;
  if (store) {
    uint8_t* codes = static_cast<uint8_t*>(store);
    uint8_t* exps = codes + act8_exp_offset(z.rows, z.n);
    if (f) { a.qc = codes; a.qe = exps; }
    else { a.fc = codes; a.fe = exps; }
  }
  a.rows = z.rows; a.n = z.n; a.groups = act8_groups(z.n); a.rpg = z.rows / std::max(1, z.gates);
  a.post = z.post; a.pre = z.pre; a.scale = z.scale; a.eps = z.eps;
  const double e = z.dt == ORBIT_BF16 ? 2.0 : 4.0, q = 1.0 + 1.0 / kAct8Group;
  const double rn = (double)z.rows * z.n;
  KernelInfo ki{z.dt == ORBIT_BF16 ? "gnorm_fwd<bf16>" : "gnorm_fwd<f32>", 16.0 * rn,
                rn * (e * (2 + (f ? 1 : 0) + z.pre) + (store ? q : 0.0))};
  if (z.dt == ORBIT_BF16) return a.fc ? gnorm_fwd_t<bf16, true>(a, ki, s) : gnorm_fwd_t<bf16, false>(a, ki, s);
  return a.fc ? gnorm_fwd_t<float, true>(a, ki, s) : gnorm_fwd_t<float, false>(a, ki, s);
}

size_t gnorm_bwd_ws_bytes(const GnormDims& z) {
  return align_up((size_t)4 * std::max(1, z.gates) * gn_shape(z).cpg * (size_t)z.n * sizeof(float));
}

namespace {

template <typename T, int NCH, bool F8>
orbit_status gnorm_bwd_run(const GnBwd& a, const KernelInfo& ki, int chunks, int threads, hipStream_t s) {
  constexpr bool KEEP = sizeof(T) == 2 || NCH < 4, PF = sizeof(T) == 2;
  constexpr int LDS = 512 * NCH * 64;
  const auto kern = gnorm_bwd_kernel<T, NCH, F8, KEEP, PF>;
  static const bool once = [&] {
    // lift the default dynamic-LDS cap (a failure surfaces as a launch error)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    (void)hipGetLastError();
    return true;
  }();
  (void)once;
  return launch(ki, kern, dim3((unsigned)chunks), dim3((unsigned)threads), (size_t)LDS, s, a);
}

template <typename T, bool F8>
orbit_status gnorm_bwd_t(const GnBwd& a, const GnShape& h, const KernelInfo& ki, int chunks, hipStream_t s) {
  const int threads = h.G * h.tpr;
  switch (h.nch) {
    case 1: return gnorm_bwd_run<T, 1, F8>(a, ki, chunks, threads, s);
    case 2: return gnorm_bwd_run<T, 2, F8>(a, ki, chunks, threads, s);
    case 3: return gnorm_bwd_run<T, 3, F8>(a, ki, chunks, threads, s);
    default: return gnorm_bwd_run<T, 4, F8>(a, ki, chunks, threads, s);
  }
}

}  // namespace

orbit_status gnorm_bwd(const GnormDims& z, const GnormParams& p, const void* f, const void* store, const void* y,
                       const float* stats, const void* dh, const void* dy, void* dx, void* df, const GnormGrads& g,
                       int accumulate, void* ws, hipStream_t s) {
  const int gates = std::max(1, z.gates);
  const GnShape h = gn_shape(z);
  GnBwd a{};
  a.f = f; a.y = y; a.dh = dh; a.dy = dy; a.gate = z.gates ? p.gate : nullptr;
  a.post_g = z.post ? p.post_g : nullptr; a.pre_g = z.pre ? p.pre_g : nullptr; a.dx = dx; a.df = df; a.stats = stats;
  if (!f && store) {
    a.fc = static_cast<const uint8_t*>(store);
    a.fe = a.fc + act8_exp_offset(z.rows, z.n);
  }
  a.part = static_cast<float*>(ws);
  a.rows = z.rows; a.n = z.n; a.groups = act8_groups(z.n);
  a.rpg = h.rpg; a.rpb = h.rpb; a.cpg = h.cpg; a.tpr = h.tpr;
  a.post = z.post; a.pre = z.pre; a.scale = z.scale;
  const int chunks = gates * h.cpg;
  const bool rf = z.post || z.gates;
  const double e = z.dt == ORBIT_BF16 ? 2.0 : 4.0, rn = (double)z.rows * z.n;
  KernelInfo ki{z.dt == ORBIT_BF16 ? "gnorm_bwd<bf16>" : "gnorm_bwd<f32>", 30.0 * rn,
                rn * (e * (2 * z.pre + (df ? 1 : 0) + (dy ? 1 : 0) + (dx ? 1 : 0) + (rf && f ? 1 : 0)) +
                      (rf && !f ? 1.0 + 1.0 / kAct8Group : 0.0)) +
                    4.0 * chunks * z.n * (2 * z.pre + 2 * rf)};
  if (z.dt == ORBIT_BF16) {
    if (a.fc) ORBIT_TRY((gnorm_bwd_t<bf16, true>(a, h, ki, chunks, s)));
    else ORBIT_TRY((gnorm_bwd_t<bf16, false>(a, h, ki, chunks, s)));
  } else {
    if (a.fc) ORBIT_TRY((gnorm_bwd_t<float, true>(a, h, ki, chunks, s)));
    else ORBIT_TRY((gnorm_bwd_t<float, false>(a, h, ki, chunks, s)));
  }
  if (!z.pre && !rf) return ORBIT_OK;
  GnFinal b{};
  b.part = a.part;
  b.gate = a.gate; b.post_g = p.post_g; b.post_b = p.post_b;
  b.dgate = g.gate; b.dpost_g = g.post_g; b.dpost_b = g.post_b; b.dpre_g = g.pre_g; b.dpre_b = g.pre_b;
  b.n = z.n; b.gates = gates; b.cpg = h.cpg; b.pre = z.pre; b.post = z.post;
  b.accumulate = accumulate; b.scale = z.scale;
  b.lanes = std::min(64, pow2_ceil(h.cpg));
  KernelInfo kf{"gnorm_final", 0.0, 4.0 * chunks * z.n * (2 * z.pre + 2 * rf)};
  const int64_t jobs = rf ? 4 + cdiv(gates, 64 / b.lanes) : 2;
  const dim3 fgrid((unsigned)(cdiv(z.n, 64) * jobs));
  if (z.dt == ORBIT_BF16) return launch(kf, gnorm_final_kernel<bf16>, fgrid, dim3(1024), 0, s, b);
  return launch(kf, gnorm_final_kernel<float>, fgrid, dim3(1024), 0, s, b);
}

}  // namespace orbit
