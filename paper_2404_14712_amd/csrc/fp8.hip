// The 8-bit floating-point store (fp8.h): packing a matrix in one or both
// orientations from one read, and reading a store back. HBM-bound.
#include <algorithm>

#include "fp8.h"
#include "lanes.h"
#include "rowbuf.h"

namespace orbit {
namespace {

struct PackArgs {
  const void* x;
  int64_t ldx, rows, n;
  uint8_t *codes, *exps;      // [rows, wide], [rows, groups] (null: not written)
  uint8_t *codes_t, *exps_t;  // [n, wide_t], [n, groups_t]
  int64_t wide, groups, wide_t, groups_t;
  float* part;                // [row tiles, n] column sums
  unsigned tiles_m, tiles_n;
  int stream;                 // x passes the caches (bf16)
};

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// maximum over 16 consecutive lanes
ORBIT_DEV uint32_t row16_umax(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
}
// sum over the four lanes 16 apart
ORBIT_DEV float col4_sum(float v) {
  float a, b;
  wave_pair<4>(v, a, b);
  wave_pair<5>(a + b, a, b);
  return a + b;
}

// largest magnitudes above this end at 448 2^119, or are infinite or NaN: blocks
// that hold one take the slow way through fp8_encode8
constexpr uint32_t kFp8Top = 0x7f600000u;

// A thread's 8 x 8 values of a tile, their largest magnitudes and their codes. MW
// words hold the largest of the 8 columns.
template <typename T> struct PackTile;

// bf16 stays packed: maxima are taken on pairs of 16-bit patterns, and the
// conversion takes a pair of values with the scale
template <> struct PackTile<bf16> {
  static constexpr int MW = 4;
  uint32_t w[8][4];
  ORBIT_DEV void load(int j, const bf16* p) {
    const U128 u = ld128(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[j][i] = u.w[i];
  }
  ORBIT_DEV void load_nt(int j, const bf16* p) {
    const U128 u = ld128nt(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[j][i] = u.w[i];
  }
  ORBIT_DEV void zero(int j) { w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0u; }
  ORBIT_DEV void set(int j, const float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[j][i] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)f[2 * i], (bf16)f[2 * i + 1]});
  }
  ORBIT_DEV float get(int j, int i) const {
    return __uint_as_float(i & 1 ? w[j][i >> 1] & 0xffff0000u : w[j][i >> 1] << 16);
  }
  static ORBIT_DEV uint32_t wmax(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  }
  ORBIT_DEV uint32_t mag(int j, int i) const { return w[j][i] & 0x7fff7fffu; }
  static ORBIT_DEV uint32_t top(uint32_t m) { return max(m << 16, m & 0xffff0000u); }  // of a word's two
  static ORBIT_DEV uint32_t col(const uint32_t* m, int i) { return i & 1 ? m[i >> 1] & 0xffff0000u : m[i >> 1] << 16; }
  static ORBIT_DEV uint32_t enc4(uint32_t lo, uint32_t hi, float s) {
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, lo), s, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, hi), s, true);
    return __builtin_bit_cast(uint32_t, r);
  }
  ORBIT_DEV uint2 row(int j, float s) const { return make_uint2(enc4(w[j][0], w[j][1], s), enc4(w[j][2], w[j][3], s)); }
  ORBIT_DEV uint2 column(int i, float s) const {
    uint32_t p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      p[k] = __builtin_amdgcn_perm(w[2 * k + 1][i >> 1], w[2 * k][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
    return make_uint2(enc4(p[0], p[1], s), enc4(p[2], p[3], s));
  }
};
template <> struct PackTile<float> {
  static constexpr int MW = 8;
  float f[8][8];
  ORBIT_DEV void load(int j, const float* p) { ld8(p, f[j]); }
  ORBIT_DEV void load_nt(int j, const float* p) { ld8(p, f[j]); }
  ORBIT_DEV void zero(int j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[j][i] = 0.f;
  }
  ORBIT_DEV void set(int j, const float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[j][i] = v[i];
  }
  ORBIT_DEV float get(int j, int i) const { return f[j][i]; }
  static ORBIT_DEV uint32_t wmax(uint32_t a, uint32_t b) { return max(a, b); }
  ORBIT_DEV uint32_t mag(int j, int i) const { return __float_as_uint(f[j][i]) & 0x7fffffffu; }
  static ORBIT_DEV uint32_t top(uint32_t m) { return m; }
  static ORBIT_DEV uint32_t col(const uint32_t* m, int i) { return m[i]; }
  static ORBIT_DEV uint32_t enc4(float a, float b, float c, float d, float s) {
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, s, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, s, true);
    return __builtin_bit_cast(uint32_t, r);
  }
  ORBIT_DEV uint2 row(int j, float s) const {
    return make_uint2(enc4(f[j][0], f[j][1], f[j][2], f[j][3], s), enc4(f[j][4], f[j][5], f[j][6], f[j][7], s));
  }
  ORBIT_DEV uint2 column(int i, float s) const {
    return make_uint2(enc4(f[0][i], f[1][i], f[2][i], f[3][i], s), enc4(f[4][i], f[5][i], f[6][i], f[7][i], s));
  }
};

// A block packs a tile of 128 rows x 128 columns; a thread holds 8 x 8 of it, so
// that it has 8 consecutive codes in either direction. The transposed codes pass
// through LDS, to leave as whole 128-byte runs of a column. bf16 4096 x 8192 into
// both orientations moves 135 MB in 31 us, 4.3 TB/s (a copy: 5.2); unpacked to
// floats, with clamps and tests on every value, it took 47. Tiles walked down the
// columns instead of along the rows: 38.9 against 36.5 us before the loads were
// streamed; a contiguous share of them for each XCD: 43.5.
// LATER: the transposed codes pass the caches, which leaves the room to what is read next
// (the forward of a 1B block with 8-bit products 415 -> 407 us; the weights' stores of a
// 113B block 196 -> 175); read at once they would come from memory (4096 x 8192, packed and
// read back: 63 -> 67 us).
template <typename T, bool TILED, bool ROWS, bool COLS, bool SUM, bool LATER>
__global__ void __launch_bounds__(256) fp8_pack_kernel(PackArgs a) {
  using Z = PackTile<T>;
  constexpr int P = 136;  // pitch of a column's 128 codes in LDS
  __shared__ __attribute__((aligned(16))) uint8_t tt[COLS ? 128 * P : 16];
  __shared__ uint32_t cmax[4][16 * Z::MW];  // by wave: words of the tile's columns
  __shared__ uint32_t tmax[4];
  __shared__ float csum[SUM ? 4 : 1][128];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 63, wave = tid >> 6;
  const unsigned tm = blockIdx.x / a.tiles_n, tn = blockIdx.x - tm * a.tiles_n;
  const int64_t r0 = (int64_t)tm * 128, c0 = (int64_t)tn * 128;
  const int rows = (int)std::min<int64_t>(a.rows - r0, 128), cols = (int)std::min<int64_t>(a.n - c0, 128);
  const int64_t gt = a.tiles_m, gn = a.tiles_n;

  Z z;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const T* p = static_cast<const T*>(a.x) + (r0 + ty * 8 + j) * a.ldx + c0 + tx * 8;
    if (ty * 8 + j < rows && tx * 8 + 8 <= cols) {
      if (a.stream) z.load_nt(j, p);
      else z.load(j, p);
    } else {
      z.zero(j);
    }
  }
  if ((cols & 7) && (cols >> 3) == tx) {
    // the row's last, short piece
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (ty * 8 + j >= rows) break;
      const T* p = static_cast<const T*>(a.x) + (r0 + ty * 8 + j) * a.ldx + c0 + tx * 8;
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < (cols & 7) ? to_f(p[i]) : 0.f;
      z.set(j, f);
    }
  }
  uint32_t rmax[8], kmax[Z::MW];  // float32 bits of the rows' largest; words of the columns'
#pragma unroll
  for (int i = 0; i < Z::MW; ++i) kmax[i] = 0u;
  uint32_t all = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < Z::MW; ++i) {
      const uint32_t b = z.mag(j, i);
      m = Z::wmax(m, b);
      kmax[i] = Z::wmax(kmax[i], b);
    }
    rmax[j] = Z::top(m);
    all = max(all, rmax[j]);
  }
  const bool slow = all > kFp8Top;
  if (slow) {
    // the largest finite magnitudes only
#pragma unroll
    for (int j = 0; j < 8; ++j) rmax[j] = 0u;
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = fp8_mag(z.get(j, i));
        rmax[j] = max(rmax[j], b);
        c[i] = max(c[i], b);
      }
    }
#pragma unroll
    for (int i = 0; i < Z::MW; ++i) kmax[i] = Z::MW == 8 ? c[i] : c[2 * i] >> 16 | c[2 * i + 1];
    all = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) all = max(all, rmax[j]);
  }
  if (SUM) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) t += z.get(j, i);
      t = col4_sum(t);
      if (lane < 16) csum[wave][tx * 8 + i] = t;
    }
  }
  auto lane_max = [](uint32_t v, int o) { return (uint32_t)__shfl_xor((int)v, o, 64); };
  uint32_t te = 0;
  if (TILED) {
    uint32_t t = row16_umax(all);
    t = max(t, lane_max(t, 16));
    t = max(t, lane_max(t, 32));
    if (lane == 0) tmax[wave] = t;
  } else if (COLS) {
#pragma unroll
    for (int i = 0; i < Z::MW; ++i) {
      uint32_t t = Z::wmax(kmax[i], lane_max(kmax[i], 16));
      t = Z::wmax(t, lane_max(t, 32));
      if (lane < 16) cmax[wave][tx * Z::MW + i] = t;
    }
  }
  if (TILED || COLS || SUM) __syncthreads();
  if (TILED) te = fp8_exp(max(max(tmax[0], tmax[1]), max(tmax[2], tmax[3])));
  if (SUM && tid < cols)
    a.part[(int64_t)tm * a.n + c0 + tid] = (csum[0][tid] + csum[SUM ? 1 : 0][tid]) + (csum[SUM ? 2 : 0][tid] + csum[SUM ? 3 : 0][tid]);

  if (ROWS) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t e = TILED ? te : fp8_exp(row16_umax(rmax[j]));
      const int64_t r = r0 + ty * 8 + j;
      if (ty * 8 + j < rows) {
        uint2 q;
        if (slow) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = z.get(j, i);
          q = fp8_encode8(f, e);
        } else {
          q = z.row(j, __uint_as_float(e << 23));
        }
        *reinterpret_cast<uint2*>(a.codes + r * a.wide + c0 + tx * 8) = q;
        if (tx == 0) {
          a.exps[r * a.groups + tn] = (uint8_t)e;
          if (tn + 1 == gn)
            for (int64_t g = gn; g < a.groups; ++g) a.exps[r * a.groups + g] = 0;
        }
      }
    }
  }
  if (COLS) {
    uint32_t cm[Z::MW];
    if (!TILED) {
#pragma unroll
      for (int i = 0; i < Z::MW; ++i) {
        const int k = tx * Z::MW + i;
        cm[i] = Z::wmax(Z::wmax(cmax[0][k], cmax[1][k]), Z::wmax(cmax[2][k], cmax[3][k]));
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = tx * 8 + i;
      const uint32_t e = TILED ? te : fp8_exp(Z::col(cm, i));
      uint2 q;
      if (slow) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = z.get(j, i);
        q = fp8_encode8(f, e);
      } else {
        q = z.column(i, __uint_as_float(e << 23));
      }
      *reinterpret_cast<uint2*>(tt + c * P + ty * 8) = q;
      if (ty == 0 && c < cols) {
        a.exps_t[(c0 + c) * a.groups_t + tm] = (uint8_t)e;
        if (tm + 1 == gt)
          for (int64_t g = gt; g < a.groups_t; ++g) a.exps_t[(c0 + c) * a.groups_t + g] = 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = q * 32 + (tid >> 3), k = (tid & 7) * 16;
      if (c < cols) {
        const uint2 lo = *reinterpret_cast<const uint2*>(tt + c * P + k);
        const uint2 hi = *reinterpret_cast<const uint2*>(tt + c * P + k + 8);
        u32v4* to = reinterpret_cast<u32v4*>(a.codes_t + (c0 + c) * a.wide_t + r0 + k);
        if constexpr (LATER) __builtin_nontemporal_store(u32v4{lo.x, lo.y, hi.x, hi.y}, to);
        else *to = u32v4{lo.x, lo.y, hi.x, hi.y};
      }
    }
  }
}

struct UnpackArgs {
  const uint8_t *codes, *exps;
  void* x;
  int64_t ldx, rows, n, wide, groups;
  int tx_log2;
};

// 8 values per thread; 2^tx_log2 threads of a block along a row, a wave at most: a row's
// last block is then short by less (float32 1000 x 2056 4.3 us, against 5.8 with 256 along
// the row; bf16 4096 x 8192 19.5 against 20.5)
template <typename T>
__global__ void __launch_bounds__(256) fp8_unpack_kernel(UnpackArgs a) {
  const int tx = 1 << a.tx_log2, ty = 256 >> a.tx_log2;
  const int64_t c = ((int64_t)blockIdx.x * tx + (threadIdx.x & (tx - 1))) * 8;
  if (c >= a.n) return;
  for (int64_t r = (int64_t)blockIdx.y * ty + (threadIdx.x >> a.tx_log2); r < a.rows; r += (int64_t)gridDim.y * ty) {
    const uint2 q = *reinterpret_cast<const uint2*>(a.codes + r * a.wide + c);
    float f[8];
    fp8_decode8(q, a.exps[r * a.groups + (c >> 7)], f);
    T* p = static_cast<T*>(a.x) + r * a.ldx + c;
    if (c + 8 <= a.n) {
      st8(p, f);
    } else {
      for (int i = 0; c + i < a.n; ++i) p[i] = from_f<T>(f[i]);
    }
  }
}

template <typename T, bool TILED, bool LATER>
orbit_status pack_t(const KernelInfo& ki, const PackArgs& a, dim3 grid, hipStream_t s) {
  const dim3 block(256);
  if constexpr (!LATER) {  // sums are those of output gradients, packed in rows for this pass
    if (a.part && a.codes) return launch(ki, fp8_pack_kernel<T, false, true, true, true, false>, grid, block, 0, s, a);
    if (a.part) return launch(ki, fp8_pack_kernel<T, false, false, true, true, false>, grid, block, 0, s, a);
  }
  if (a.codes && a.codes_t) return launch(ki, fp8_pack_kernel<T, TILED, true, true, false, LATER>, grid, block, 0, s, a);
  if constexpr (TILED || !LATER) {  // the forward's later store comes with the other
    if (!a.codes) return launch(ki, fp8_pack_kernel<T, TILED, false, true, false, LATER>, grid, block, 0, s, a);
  }
  return launch(ki, fp8_pack_kernel<T, TILED, true, false, false, false>, grid, block, 0, s, a);
}
template <typename T>
orbit_status pack_pick(const KernelInfo& ki, const PackArgs& a, dim3 grid, bool tiled, bool later, hipStream_t s) {
  if (tiled) return pack_t<T, true, true>(ki, a, grid, s);
  return later ? pack_t<T, false, true>(ki, a, grid, s) : pack_t<T, false, false>(ki, a, grid, s);
}

}  // namespace

orbit_status fp8_pack(orbit_dtype dt, const void* x, int64_t ldx, int64_t rows, int64_t n, bool tiled, void* store,
                      void* store_t, bool later, float* part, hipStream_t s) {
  PackArgs a{};
  a.x = x; a.ldx = ldx; a.rows = rows; a.n = n; a.part = part;
  a.wide = fp8_wide(n); a.groups = fp8_groups(n);
  a.wide_t = fp8_wide(rows); a.groups_t = fp8_groups(rows);
  a.tiles_m = (unsigned)cdiv(rows, 128); a.tiles_n = (unsigned)cdiv(n, 128);
  if (store) {
    a.codes = static_cast<uint8_t*>(store);
    a.exps = a.codes + fp8_exp_offset(rows, n);
  }
  if (store_t) {
    a.codes_t = static_cast<uint8_t*>(store_t);
    a.exps_t = a.codes_t + fp8_exp_offset(n, rows);
  }
  const double v = (double)rows * (double)n;
  KernelInfo ki{dt == ORBIT_BF16 ? "fp8_pack<bf16>" : "fp8_pack<f32>", 8.0 * v,
                v * ((dt == ORBIT_BF16 ? 2.0 : 4.0) + ((store ? 1 : 0) + (store_t ? 1 : 0)) * (1.0 + 1.0 / kFp8Block))};
  // more than the caches hold: x is streamed past them (bf16 4096 x 8192, both
  // orientations: 36.5 -> 31.0 us)
  a.stream = ki.bytes >= 96e6;
  const dim3 grid(a.tiles_m * a.tiles_n);
  return dt == ORBIT_BF16 ? pack_pick<bf16>(ki, a, grid, tiled, later, s) : pack_pick<float>(ki, a, grid, tiled, later, s);
}

orbit_status fp8_unpack(orbit_dtype dt, const void* store, int64_t rows, int64_t n, void* x, int64_t ldx,
                        hipStream_t s) {
  UnpackArgs a{};
  a.codes = static_cast<const uint8_t*>(store);
  a.exps = a.codes + fp8_exp_offset(rows, n);
  a.x = x; a.ldx = ldx; a.rows = rows; a.n = n; a.wide = fp8_wide(n); a.groups = fp8_groups(n);
  const int64_t pieces = cdiv(n, 8);
  a.tx_log2 = 2;
  while (a.tx_log2 < 6 && (1ll << a.tx_log2) < pieces) ++a.tx_log2;
  const double v = (double)rows * (double)n;
  KernelInfo ki{dt == ORBIT_BF16 ? "fp8_unpack<bf16>" : "fp8_unpack<f32>", 2.0 * v,
                v * ((dt == ORBIT_BF16 ? 2.0 : 4.0) + 1.0 + 1.0 / kFp8Block)};
  const dim3 grid((unsigned)cdiv(pieces, 1 << a.tx_log2),
                  (unsigned)std::min<int64_t>(cdiv(rows, 256 >> a.tx_log2), 65535));
  if (dt == ORBIT_BF16) return launch(ki, fp8_unpack_kernel<bf16>, grid, dim3(256), 0, s, a);
  return launch(ki, fp8_unpack_kernel<float>, grid, dim3(256), 0, s, a);
}

}  // namespace orbit
