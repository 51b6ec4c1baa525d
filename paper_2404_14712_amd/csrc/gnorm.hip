// Gated norms, forward and backward (gnorm.h). HBM-bound: a row's values stay
// in registers between the passes over it, so every tensor is read and written
// once; statistics and parameter gradients are float32.
#include <algorithm>
#include <type_traits>

#include "act8.h"
#include "gnorm.h"
#include "rowbuf.h"

namespace orbit {
namespace {

template <typename T> ORBIT_DEV void load8(const T* p, float* f);
template <> ORBIT_DEV void load8<bf16>(const bf16* p, float* f) { unpack(ld128(p), f, (bf16*)nullptr); }
template <> ORBIT_DEV void load8<float>(const float* p, float* f) {
  unpack(ld128(p), f, (float*)nullptr);
  unpack(ld128(p + 4), f + 4, (float*)nullptr);
}
template <typename T> ORBIT_DEV void store8(T* p, const float* f);
template <> ORBIT_DEV void store8<bf16>(bf16* p, const float* f) { st128(p, pack(f, (bf16*)nullptr)); }
template <> ORBIT_DEV void store8<float>(float* p, const float* f) {
  st128(p, pack(f, (float*)nullptr));
  st128(p + 4, pack(f + 4, (float*)nullptr));
}

// sum over the TPR threads of a row: a wave, or the whole 256-thread block
// (then `red` is 4 floats of LDS and the call ends with a barrier)
template <int TPR> ORBIT_DEV float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[0] + red[1]) + (red[2] + red[3]);
    __syncthreads();
  }
  return v;
}

struct GnFwd {
  const void *x, *f, *gate, *post_g, *post_b, *pre_g, *pre_b;
  void *y, *h;
  const uint8_t *fc, *fe;  // the store that f is read from (f null)
  uint8_t *qc, *qe;        // the store that receives f (may be null)
  float* stats;
  int rows, n, groups, rpg;  // rpg: rows per gate row
  int post, pre;
  float scale, eps;
};

// mean and 1 / sqrt(variance + eps) of a row held as v[NCH][8]
template <int NCH, int TPR>
ORBIT_DEV void row_stats(const float (*v)[8], const bool* on, int n, float eps, float* red, float& mu, float& r) {
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c)
    if (on[c])
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[c][i];
  mu = row_sum<TPR>(s, red) / (float)n;
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c)
    if (on[c])
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = v[c][i] - mu;
        q += t * t;
      }
  r = rsqrtf(row_sum<TPR>(q, red) / (float)n + eps);
}

// TPR threads per row, thread t of a row owning the 8-column pieces t + c TPR,
// so that a quad holds the 32 columns of a group of the store. y is written
// rounded to the storage type, h and the statistics come from its float32
// value: h then carries one rounding instead of two, and the backward's
// (rounded y - mean) differs from the exact one by y's rounding alone.
template <typename T, int NCH, int TPR>
__global__ void __launch_bounds__(256) gnorm_fwd_kernel(GnFwd a) {
  __shared__ float red[4];
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (row >= a.rows) return;  // whole waves (TPR 64); never with TPR 256
  const int64_t base = row * a.n;
  int col[NCH];
  bool on[NCH];
  float v[NCH][8], x[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = 8 * (t + c * TPR);
    on[c] = col[c] < a.n;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = x[c][i] = 0.f;
    if (on[c]) {
      if (a.f) load8(static_cast<const T*>(a.f) + base + col[c], v[c]);
      else act8_decode(*reinterpret_cast<const uint2*>(a.fc + base + col[c]),
                       a.fe[row * a.groups + (col[c] >> 5)], v[c]);
      load8(static_cast<const T*>(a.x) + base + col[c], x[c]);
    }
  }
  if (a.qc) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      uint2 q;
      const uint32_t e = act8_encode(v[c], q);
      if (on[c]) {
        *reinterpret_cast<uint2*>(a.qc + base + col[c]) = q;
        if ((t & 3) == 0) a.qe[row * a.groups + (col[c] >> 5)] = (uint8_t)e;
      }
    }
  }
  float mf = 0.f, rf = 0.f, my = 0.f, ry = 0.f;
  if (a.post) row_stats<NCH, TPR>(v, on, a.n, a.eps, red, mf, rf);
  const T* gate = static_cast<const T*>(a.gate);
  if (gate) gate += (row / a.rpg) * a.n;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if (!on[c]) continue;
    float w[8], b[8];
    if (a.post) {
      load8(static_cast<const T*>(a.post_g) + col[c], w);
      load8(static_cast<const T*>(a.post_b) + col[c], b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = (v[c][i] - mf) * rf * w[i] + b[i];
    }
    if (gate) {
      load8(gate + col[c], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = x[c][i] + a.scale * v[c][i];
    store8(static_cast<T*>(a.y) + base + col[c], v[c]);
  }
  if (a.pre) {
    row_stats<NCH, TPR>(v, on, a.n, a.eps, red, my, ry);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (!on[c]) continue;
      float w[8], b[8];
      load8(static_cast<const T*>(a.pre_g) + col[c], w);
      load8(static_cast<const T*>(a.pre_b) + col[c], b);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = (v[c][i] - my) * ry * w[i] + b[i];
      store8(static_cast<T*>(a.h) + base + col[c], w);
    }
  }
  if (t == 0) *reinterpret_cast<float4*>(a.stats + 4 * row) = make_float4(mf, rf, my, ry);
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
// of each of its four column sums; gnorm_final and ColFinal add the partials
// in a fixed order.
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

// 8 codes of a store and their group's E
struct Raw8Q {
  u32v2 q;
  uint32_t e;
  ORBIT_DEV void renew() { asm volatile("" : "+v"(q)); }
  ORBIT_DEV void get4(int h, float* f) const { act8_decode4(q[h], e, f); }
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

// A block of 512 threads (one per CU, 256 registers each) whose G = blockDim /
// tpr groups of tpr threads take the chunk's rows in turn; thread t of a group
// owns the NCH 8-column pieces t + c tpr. Every group runs the same number of
// rows, so the barriers line up. The four column sums would take half of the
// register file at full width; the two of the pre norm live in LDS. That leaves
// room for the next row's dh and y (PF, bf16), so that loads are in flight all
// the time; its dy and f follow into the registers of the current row's once
// these are used up. KEEP:
// values stay in registers from their one load; the widest float32 rows are
// loaded again where they are used instead.
template <typename T, int NCH, bool F8, bool KEEP, bool PF>
__global__ void __launch_bounds__(512) gnorm_bwd_kernel(GnBwd a) {
  using Row = GnRow<T, NCH, F8>;
  constexpr int NT = 512;
  constexpr int PIECES = NT * NCH;
  __shared__ float red[2][NT / 64][2];
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
  const int r0 = gi * a.rpg + ci * a.rpb, r1 = min((gi + 1) * a.rpg, r0 + a.rpb);
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
  auto row_sum2 = [&](int k, float& u, float& v) {
    u = wave_sum(u);
    v = wave_sum(v);
    if (wpg > 1) {
      if (lane == 0) {
        red[k][wave][0] = u;
        red[k][wave][1] = v;
      }
      __syncthreads();
      u = v = 0.f;
      for (int w = q * wpg; w < (q + 1) * wpg; ++w) {
        u += red[k][w][0];
        v += red[k][w][1];
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
      R.dh[c].load(bh, col[c] * (uint32_t)sizeof(T));
      R.y[c].load(by, col[c] * (uint32_t)sizeof(T));
    }
  };
  auto fetch_d = [&](Row& R) {
    const RowBuf b = row(a.dy, R, a.dy != nullptr);
#pragma unroll
    for (int c = 0; c < NCH; ++c) R.dy[c].load(b, col[c] * (uint32_t)sizeof(T));
  };
  auto fetch_f = [&](Row& R) {
    if constexpr (F8) {
      const bool v = rf && R.rv;
      const RowBuf bq(a.fc, R.r * n, v ? n : 0), be(a.fe, R.r * a.groups, v ? a.groups : 0);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        R.f[c].q = __builtin_amdgcn_raw_buffer_load_b64(bq.r, col[c], 0, 0);
        // where nothing is read: any E but 0, which stands for NaN
        R.f[c].e = __builtin_amdgcn_raw_buffer_load_b8(be.r, col[c] >> 5, 0, 0) | (v && col[c] < (uint32_t)n ? 0u : 7u);
      }
    } else {
      const RowBuf b = row(a.f, R, rf);
#pragma unroll
      for (int c = 0; c < NCH; ++c) R.f[c].load(b, col[c] * (uint32_t)sizeof(T));
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
    // yh = y ry - my ry, fh = f rf - mf rf
    const float ry = cur.st.w, oy = -cur.st.z * ry, rr = cur.st.y, of = -cur.st.x * rr;
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
            const float yh = fmaf(y4[i], ry, oy), w = d4[i] * g4[i];
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
        if (NCH == 4) __builtin_amdgcn_sched_barrier(0);  // one piece's temporaries at a time
      }
      row_sum2(0, m1, m2);
      m1 *= inv_n;
      m2 *= inv_n;
    }
    if (!KEEP) {
      fetch_h(cur);
      fetch_d(cur);
      fetch_f(cur);
    }
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
          t4[i] = fmaf(ry, fmaf(-m2, fmaf(f4[i], ry, oy), fmaf(d4[i], v4[i], -m1)), t4[i]);
        o.put4(h, t4);
        cur.f[c].get4(h, f4);
        gg.get4(h, v4);
        pg.get4(h, d4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f4[i] = fmaf(f4[i], rr, of);
          s2[c][h][i] += t4[i];
          s3[c][h][i] = fmaf(t4[i], f4[i], s3[c][h][i]);
          t4[i] *= a.scale * v4[i] * d4[i];
          m3 += t4[i];
          m4 = fmaf(t4[i], f4[i], m4);
          w[c][4 * h + i] = t4[i];
        }
      }
      o.store(bx, col[c] * (uint32_t)sizeof(T));
      if (NCH == 4) __builtin_amdgcn_sched_barrier(0);
    }
    if (KEEP && !PF) fetch_h(nxt);
    if (KEEP) fetch_d(nxt);
    if (post) {
      row_sum2(1, m3, m4);
      m3 *= inv_n;
      m4 *= inv_n;
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
          for (int i = 0; i < 4; ++i) t4[i] = rr * fmaf(-m4, fmaf(f4[i], rr, of), t4[i] - m3);
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
// down to 67).
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
  if (job < 4) {
    const float* p = a.part + (int64_t)job * chunks * a.n + c;
    f32x4 s = zero;
    if (on) {
      if (job < 2) {
#pragma unroll 8
        for (int k = q; k < chunks; k += 64) s += get(p + (int64_t)k * a.n);
      } else {
#pragma unroll 8
        for (int k = q; k < chunks; k += 64) s += vec(gate, (int64_t)(k / a.cpg) * a.n + c) * get(p + (int64_t)k * a.n);
      }
    }
    red[0][q][e] = s;
    __syncthreads();
    if (q != 0 || !on) return;
    s = zero;
#pragma unroll 8
    for (int k = 0; k < 64; ++k) s += red[0][k][e];
    if (job >= 2) s *= a.scale;
    put((job == 0 ? a.dpre_b : job == 1 ? a.dpre_g : job == 2 ? a.dpost_b : a.dpost_g) + c, s);
    return;
  }
  const int per = 64 / a.lanes, ql = q % a.lanes;
  const int64_t g = (int64_t)(job - 4) * per + q / a.lanes;
  f32x4 s1 = zero, s2 = zero;
  if (on && g < a.gates) {
    const float* p2 = a.part + ((int64_t)3 * chunks + g * a.cpg) * a.n + c;
    const float* p1 = p2 - (int64_t)chunks * a.n;
#pragma unroll 8
    for (int k = ql; k < a.cpg; k += a.lanes) {
      s2 += get(p2 + (int64_t)k * a.n);
      if (a.post) s1 += get(p1 + (int64_t)k * a.n);
    }
  }
  red[0][q][e] = s1;
  red[1][q][e] = s2;
  __syncthreads();
  if (ql != 0 || !on || g >= a.gates) return;
  for (int k = 1; k < a.lanes; ++k) {
    s1 += red[0][q + k][e];
    s2 += red[1][q + k][e];
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
// to 1024 columns is a wave's), a block as many rows at once as 512 threads
// hold. Chunks: about one per CU, whole turns of the block's groups.
struct GnShape {
  int nch, tpr, G, rpg, rpb, cpg;
};
GnShape gn_shape(const GnormDims& z) {
  GnShape h{};
  h.nch = z.n <= 512 ? 1 : z.n <= 1024 ? 2 : 4;
  h.tpr = (int)(cdiv(cdiv(z.n, 8 * h.nch), 64) * 64);
  h.G = 512 / h.tpr;
  h.rpg = z.rows / std::max(1, z.gates);
  const int turns = std::max<int>({1, (8 + h.G - 1) / h.G, (z.rows + 128 * h.G) / (256 * h.G)});
  h.rpb = std::min(h.rpg, turns * h.G);
  h.G = std::min(h.G, h.rpb);
  h.cpg = (int)cdiv(h.rpg, h.rpb);
  return h;
}

template <typename T>
orbit_status gnorm_fwd_t(const GnFwd& a, const KernelInfo& ki, hipStream_t s) {
  const dim3 block(256);
  if (a.n <= 2048) {
    const dim3 grid((unsigned)cdiv(a.rows, 4));
    if (a.n <= 512) return launch(ki, gnorm_fwd_kernel<T, 1, 64>, grid, block, 0, s, a);
    if (a.n <= 1024) return launch(ki, gnorm_fwd_kernel<T, 2, 64>, grid, block, 0, s, a);
    return launch(ki, gnorm_fwd_kernel<T, 4, 64>, grid, block, 0, s, a);
  }
  const dim3 grid((unsigned)a.rows);
  if (a.n <= 4096) return launch(ki, gnorm_fwd_kernel<T, 2, 256>, grid, block, 0, s, a);
  if (a.n <= 8192) return launch(ki, gnorm_fwd_kernel<T, 4, 256>, grid, block, 0, s, a);
  return launch(ki, gnorm_fwd_kernel<T, 8, 256>, grid, block, 0, s, a);
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
  if (z.dt == ORBIT_BF16) return gnorm_fwd_t<bf16>(a, ki, s);
  return gnorm_fwd_t<float>(a, ki, s);
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
  if (h.nch == 4) return gnorm_bwd_run<T, 4, F8>(a, ki, chunks, threads, s);
  if (h.nch == 2) return gnorm_bwd_run<T, 2, F8>(a, ki, chunks, threads, s);
  return gnorm_bwd_run<T, 1, F8>(a, ki, chunks, threads, s);
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
