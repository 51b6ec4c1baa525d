// Gated norms, forward and backward (gnorm.h). HBM-bound: a row's values stay
// in registers between the passes over it, so every tensor is read and written
// once; statistics and parameter gradients are float32.
#include <algorithm>

#include "act8.h"
#include "gnorm.h"

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

template <typename T, int NCH>
__global__ void __launch_bounds__(512) gnorm_bwd_kernel(GnBwd a) {
  __shared__ float red[2][8][2];
  const int tpr = a.tpr, G = (int)blockDim.x / tpr, wpg = tpr >> 6;
  const int q = (int)threadIdx.x / tpr, t = (int)threadIdx.x % tpr;
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const int n = a.n, chunks = (int)gridDim.x;
  const int gi = (int)blockIdx.x / a.cpg, ci = (int)blockIdx.x % a.cpg;
  const int r0 = gi * a.rpg + ci * a.rpb, r1 = min((gi + 1) * a.rpg, r0 + a.rpb);
  const T* gate = static_cast<const T*>(a.gate);
  if (gate) gate += (int64_t)gi * n;
  const bool rf_ = a.post || gate;  // f is read
  int col[NCH];
  bool on[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = 8 * (t + c * tpr);
    on[c] = col[c] < n;
  }
  float s[4][NCH][8];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[k][c][i] = 0.f;
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
  const int steps = (a.rpb + G - 1) / G;
  for (int it = 0; it < steps; ++it) {
    const int64_t r = r0 + q + (int64_t)it * G;
    const bool rv = r < r1;
    const int64_t base = r * n;
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (rv) st = *reinterpret_cast<const float4*>(a.stats + 4 * r);
    float tv[NCH][8], fv[NCH][8], wv[NCH][8];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) tv[c][i] = fv[c][i] = wv[c][i] = 0.f;
      if (!(rv && on[c])) continue;
      if (a.dy) load8(static_cast<const T*>(a.dy) + base + col[c], tv[c]);
      if (rf_) {
        if (a.f) load8(static_cast<const T*>(a.f) + base + col[c], fv[c]);
        else act8_decode(*reinterpret_cast<const uint2*>(a.fc + base + col[c]),
                         a.fe[r * a.groups + (col[c] >> 5)], fv[c]);
      }
      if (a.pre) {
        float yv[8], g8[8];
        load8(static_cast<const T*>(a.dh) + base + col[c], wv[c]);
        load8(static_cast<const T*>(a.y) + base + col[c], yv);
        load8(static_cast<const T*>(a.pre_g) + col[c], g8);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float yh = (yv[i] - st.z) * st.w;
          s[0][c][i] += wv[c][i];
          s[1][c][i] += wv[c][i] * yh;
          wv[c][i] *= g8[i];
          s1 += wv[c][i];
          s2 += wv[c][i] * yh;
        }
      }
    }
    if (a.pre) {
      row_sum2(0, s1, s2);
      const float m1 = s1 * inv_n, m2 = s2 * inv_n;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        if (!(rv && on[c])) continue;
        float yv[8];
        load8(static_cast<const T*>(a.y) + base + col[c], yv);
#pragma unroll
        for (int i = 0; i < 8; ++i) tv[c][i] += st.w * (wv[c][i] - m1 - (yv[i] - st.z) * st.w * m2);
      }
    }
    float s3 = 0.f, s4 = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (!(rv && on[c])) continue;
      if (a.dx) store8(static_cast<T*>(a.dx) + base + col[c], tv[c]);
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (a.post) fv[c][i] = (fv[c][i] - st.x) * st.y;
        s[2][c][i] += tv[c][i];
        s[3][c][i] += tv[c][i] * fv[c][i];
        wv[c][i] = a.scale * tv[c][i];
      }
      if (gate) {
        load8(gate + col[c], w);
#pragma unroll
        for (int i = 0; i < 8; ++i) wv[c][i] *= w[i];
      }
      if (a.post) {
        load8(static_cast<const T*>(a.post_g) + col[c], w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          wv[c][i] *= w[i];
          s3 += wv[c][i];
          s4 += wv[c][i] * fv[c][i];
        }
      }
    }
    if (a.post) {
      row_sum2(1, s3, s4);
      const float m3 = s3 * inv_n, m4 = s4 * inv_n;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) wv[c][i] = st.y * (wv[c][i] - m3 - fv[c][i] * m4);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if (a.df && rv && on[c]) store8(static_cast<T*>(a.df) + base + col[c], wv[c]);
  }
  // the groups' sums, added in group order through LDS, then a partial row each
  __shared__ float comb[NCH == 2 ? 512 * 16 : 1];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k < 2 ? !a.pre : !rf_) continue;
    if (NCH == 2 && G > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) comb[threadIdx.x * 16 + c * 8 + i] = s[k][c][i];
      __syncthreads();
      if (q == 0)
        for (int gq = 1; gq < G; ++gq)
#pragma unroll
          for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[k][c][i] += comb[(gq * tpr + t) * 16 + c * 8 + i];
    }
    if (q != 0) continue;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if (on[c]) store8(a.part + ((int64_t)k * chunks + blockIdx.x) * n + col[c], s[k][c]);
  }
}

struct GnFinal {
  const float *p1, *p2;  // partials of S1 and S2 [gates * cpg][n]
  const void *gate, *post_g, *post_b;
  float *dgate, *dpost_g, *dpost_b;
  int n, gates, cpg, post, accumulate;
  float scale;
};

// 16 columns x 16 chunk lanes per block; the lanes' sums are added in order
template <typename T>
__global__ void __launch_bounds__(256) gnorm_final_kernel(GnFinal a) {
  __shared__ float red[2][16][17];
  const int e = threadIdx.x % 16, q = threadIdx.x / 16;
  const int64_t c = (int64_t)blockIdx.x * 16 + e;
  const bool on = c < a.n;
  const float pg = on && a.post ? to_f(static_cast<const T*>(a.post_g)[c]) : 1.f;
  const float pb = on && a.post ? to_f(static_cast<const T*>(a.post_b)[c]) : 0.f;
  float dg = 0.f, db = 0.f;
  for (int g = 0; g < a.gates; ++g) {
    float s1 = 0.f, s2 = 0.f;
    if (on) {
      for (int k = q; k < a.cpg; k += 16) {
        const int64_t at = ((int64_t)g * a.cpg + k) * a.n + c;
        if (a.post) s1 += a.p1[at];
        s2 += a.p2[at];
      }
    }
    __syncthreads();
    red[0][q][e] = s1;
    red[1][q][e] = s2;
    __syncthreads();
    if (q == 0 && on) {
      s1 = s2 = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        s1 += red[0][k][e];
        s2 += red[1][k][e];
      }
      const float gt = a.gate ? to_f(static_cast<const T*>(a.gate)[(int64_t)g * a.n + c]) : 1.f;
      dg += gt * s2;
      db += gt * s1;
      if (a.gate) {
        const float v = a.scale * (pg * s2 + pb * s1);
        float* o = a.dgate + (int64_t)g * a.n + c;
        *o = a.accumulate ? *o + v : v;
      }
    }
  }
  if (q == 0 && on && a.post) {
    a.dpost_g[c] = a.accumulate ? a.dpost_g[c] + a.scale * dg : a.scale * dg;
    a.dpost_b[c] = a.accumulate ? a.dpost_b[c] + a.scale * db : a.scale * db;
  }
}

// rows per chunk of the backward: 16, or 8 where 16-row chunks leave CUs idle
int gn_rpb(const GnormDims& z) { return cdiv(z.rows, 16) >= 256 ? 16 : 8; }
int gn_rpg(const GnormDims& z) { return z.rows / std::max(1, z.gates); }
int gn_cpg(const GnormDims& z) { return (int)cdiv(gn_rpg(z), gn_rpb(z)); }

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
  a.rows = z.rows; a.n = z.n; a.groups = act8_groups(z.n); a.rpg = gn_rpg(z);
  a.post = z.post; a.pre = z.pre; a.scale = z.scale; a.eps = z.eps;
  const double e = z.dt == ORBIT_BF16 ? 2.0 : 4.0, q = 1.0 + 1.0 / kAct8Group;
  const double rn = (double)z.rows * z.n;
  KernelInfo ki{z.dt == ORBIT_BF16 ? "gnorm_fwd<bf16>" : "gnorm_fwd<f32>", 16.0 * rn,
                rn * (e * (2 + (f ? 1 : 0) + z.pre) + (store ? q : 0.0))};
  if (z.dt == ORBIT_BF16) return gnorm_fwd_t<bf16>(a, ki, s);
  return gnorm_fwd_t<float>(a, ki, s);
}

size_t gnorm_bwd_ws_bytes(const GnormDims& z) {
  return align_up((size_t)4 * std::max(1, z.gates) * gn_cpg(z) * (size_t)z.n * sizeof(float));
}

orbit_status gnorm_bwd(const GnormDims& z, const GnormParams& p, const void* f, const void* store, const void* y,
                       const float* stats, const void* dh, const void* dy, void* dx, void* df, const GnormGrads& g,
                       int accumulate, void* ws, ColFinal& fin, hipStream_t s) {
  const int gates = std::max(1, z.gates);
  GnBwd a{};
  a.f = f; a.y = y; a.dh = dh; a.dy = dy; a.gate = z.gates ? p.gate : nullptr;
  a.post_g = p.post_g; a.pre_g = p.pre_g; a.dx = dx; a.df = df; a.stats = stats;
  if (!f && store) {
    a.fc = static_cast<const uint8_t*>(store);
    a.fe = a.fc + act8_exp_offset(z.rows, z.n);
  }
  a.part = static_cast<float*>(ws);
  a.rows = z.rows; a.n = z.n; a.groups = act8_groups(z.n);
  a.rpg = gn_rpg(z); a.rpb = gn_rpb(z); a.cpg = gn_cpg(z);
  a.post = z.post; a.pre = z.pre; a.scale = z.scale;
  const int nch = z.n <= 8192 ? 2 : 4;
  a.tpr = (int)(cdiv(cdiv(z.n, 8 * nch), 64) * 64);
  const int chunks = gates * a.cpg;
  const dim3 grid((unsigned)chunks), block((unsigned)(512 / a.tpr * a.tpr));
  const bool rf = z.post || z.gates;
  const double e = z.dt == ORBIT_BF16 ? 2.0 : 4.0, rn = (double)z.rows * z.n;
  KernelInfo ki{z.dt == ORBIT_BF16 ? "gnorm_bwd<bf16>" : "gnorm_bwd<f32>", 30.0 * rn,
                rn * (e * (1 + 2 * z.pre + (dy ? 1 : 0) + (dx ? 1 : 0) + (rf && f ? 1 : 0)) +
                      (rf && !f ? 1.0 + 1.0 / kAct8Group : 0.0)) +
                    4.0 * chunks * z.n * (2 * z.pre + 2 * rf)};
  const bool wide = nch == 4;
  if (z.dt == ORBIT_BF16) {
    if (wide) ORBIT_TRY(launch(ki, gnorm_bwd_kernel<bf16, 4>, grid, block, 0, s, a));
    else ORBIT_TRY(launch(ki, gnorm_bwd_kernel<bf16, 2>, grid, block, 0, s, a));
  } else {
    if (wide) ORBIT_TRY(launch(ki, gnorm_bwd_kernel<float, 4>, grid, block, 0, s, a));
    else ORBIT_TRY(launch(ki, gnorm_bwd_kernel<float, 2>, grid, block, 0, s, a));
  }
  if (z.pre) {
    fin.add(a.part, z.n, chunks, z.n, g.pre_b);
    fin.add(a.part + (int64_t)chunks * z.n, z.n, chunks, z.n, g.pre_g);
  }
  if (!rf) return ORBIT_OK;
  GnFinal b{};
  b.p1 = a.part + (int64_t)2 * chunks * z.n;
  b.p2 = a.part + (int64_t)3 * chunks * z.n;
  b.gate = a.gate; b.post_g = p.post_g; b.post_b = p.post_b;
  b.dgate = g.gate; b.dpost_g = g.post_g; b.dpost_b = g.post_b;
  b.n = z.n; b.gates = gates; b.cpg = a.cpg; b.post = z.post; b.accumulate = accumulate; b.scale = z.scale;
  KernelInfo kf{"gnorm_final", 0.0, 8.0 * chunks * z.n};
  const dim3 fgrid((unsigned)cdiv(z.n, 16));
  if (z.dt == ORBIT_BF16) return launch(kf, gnorm_final_kernel<bf16>, fgrid, dim3(256), 0, s, b);
  return launch(kf, gnorm_final_kernel<float>, fgrid, dim3(256), 0, s, b);
}

}  // namespace orbit
