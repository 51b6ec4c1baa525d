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
};

// maximum over 16 consecutive lanes
ORBIT_DEV uint32_t row16_umax(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
}
// maximum, sum over the four lanes 16 apart
ORBIT_DEV uint32_t col4_umax(uint32_t v) {
  v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  return max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
}
ORBIT_DEV float col4_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// A block packs a tile of 128 rows x 128 columns; a thread holds 8 x 8 of it, so
// that it has 8 consecutive codes in either direction. The transposed codes pass
// through LDS, to leave as whole 128-byte runs of a column.
template <typename T, bool TILED, bool ROWS, bool COLS>
__global__ void __launch_bounds__(256) fp8_pack_kernel(PackArgs a) {
  constexpr int P = 136;  // pitch of a column's 128 codes in LDS
  __shared__ __attribute__((aligned(16))) uint8_t tt[COLS ? 128 * P : 16];
  __shared__ uint32_t cmax[4][128];
  __shared__ float csum[4][128];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 63, wave = tid >> 6;
  const unsigned tm = blockIdx.x / a.tiles_n, tn = blockIdx.x - tm * a.tiles_n;
  const int64_t r0 = (int64_t)tm * 128, c0 = (int64_t)tn * 128;
  const int rows = (int)std::min<int64_t>(a.rows - r0, 128), cols = (int)std::min<int64_t>(a.n - c0, 128);
  const int64_t gt = a.tiles_m, gn = a.tiles_n;

  float f[8][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const T* p = static_cast<const T*>(a.x) + (r0 + ty * 8 + j) * a.ldx + c0 + tx * 8;
    const bool rv = ty * 8 + j < rows;
    if (rv && tx * 8 + 8 <= cols) {
      ld8(p, f[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[j][i] = rv && tx * 8 + i < cols ? to_f(p[i]) : 0.f;
    }
  }
  uint32_t rmax[8], kmax[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rmax[j] = kmax[j] = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = fp8_mag(f[j][i]);
      rmax[j] = max(rmax[j], b);
      kmax[i] = max(kmax[i], b);
    }
  if (a.part) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) t += f[j][i];
      t = col4_sum(t);
      if (lane < 16) csum[wave][tx * 8 + i] = t;
    }
  }
  uint32_t te = 0;
  if (TILED) {
    uint32_t t = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) t = max(t, rmax[j]);
    t = col4_umax(row16_umax(t));
    if (lane == 0) cmax[wave][0] = t;
    __syncthreads();
    te = fp8_exp(max(max(cmax[0][0], cmax[1][0]), max(cmax[2][0], cmax[3][0])));
  } else if (COLS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t t = col4_umax(kmax[i]);
      if (lane < 16) cmax[wave][tx * 8 + i] = t;
    }
    __syncthreads();
  } else if (a.part) {
    __syncthreads();
  }
  if (a.part && tid < cols) a.part[(int64_t)tm * a.n + c0 + tid] = (csum[0][tid] + csum[1][tid]) + (csum[2][tid] + csum[3][tid]);

  if (ROWS) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t e = TILED ? te : fp8_exp(row16_umax(rmax[j]));
      const int64_t r = r0 + ty * 8 + j;
      if (ty * 8 + j < rows) {
        *reinterpret_cast<uint2*>(a.codes + r * a.wide + c0 + tx * 8) = fp8_encode8(f[j], e);
        if (tx == 0) {
          a.exps[r * a.groups + tn] = (uint8_t)e;
          if (tn + 1 == gn)
            for (int64_t g = gn; g < a.groups; ++g) a.exps[r * a.groups + g] = 0;
        }
      }
    }
  }
  if (COLS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = tx * 8 + i;
      const uint32_t e = TILED ? te : fp8_exp(max(max(cmax[0][c], cmax[1][c]), max(cmax[2][c], cmax[3][c])));
      *reinterpret_cast<uint2*>(tt + c * P + ty * 8) = fp8_encode8<8>(&f[0][i], e);
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
        *reinterpret_cast<uint4*>(a.codes_t + (c0 + c) * a.wide_t + r0 + k) = make_uint4(lo.x, lo.y, hi.x, hi.y);
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

// 8 values per thread; 2^tx_log2 threads of a block along a row
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

template <typename T, bool TILED>
orbit_status pack_t(const KernelInfo& ki, const PackArgs& a, dim3 grid, hipStream_t s) {
  const dim3 block(256);
  if (a.codes && a.codes_t) return launch(ki, fp8_pack_kernel<T, TILED, true, true>, grid, block, 0, s, a);
  if (a.codes) return launch(ki, fp8_pack_kernel<T, TILED, true, false>, grid, block, 0, s, a);
  return launch(ki, fp8_pack_kernel<T, TILED, false, true>, grid, block, 0, s, a);
}

}  // namespace

orbit_status fp8_pack(orbit_dtype dt, const void* x, int64_t ldx, int64_t rows, int64_t n, bool tiled, void* store,
                      void* store_t, float* part, hipStream_t s) {
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
  const dim3 grid(a.tiles_m * a.tiles_n);
  if (dt == ORBIT_BF16) return tiled ? pack_t<bf16, true>(ki, a, grid, s) : pack_t<bf16, false>(ki, a, grid, s);
  return tiled ? pack_t<float, true>(ki, a, grid, s) : pack_t<float, false>(ki, a, grid, s);
}

orbit_status fp8_unpack(orbit_dtype dt, const void* store, int64_t rows, int64_t n, void* x, int64_t ldx,
                        hipStream_t s) {
  UnpackArgs a{};
  a.codes = static_cast<const uint8_t*>(store);
  a.exps = a.codes + fp8_exp_offset(rows, n);
  a.x = x; a.ldx = ldx; a.rows = rows; a.n = n; a.wide = fp8_wide(n); a.groups = fp8_groups(n);
  const int64_t pieces = cdiv(n, 8);
  a.tx_log2 = 2;
  while (a.tx_log2 < 8 && (1ll << a.tx_log2) < pieces) ++a.tx_log2;
  const double v = (double)rows * (double)n;
  KernelInfo ki{dt == ORBIT_BF16 ? "fp8_unpack<bf16>" : "fp8_unpack<f32>", 2.0 * v,
                v * ((dt == ORBIT_BF16 ? 2.0 : 4.0) + 1.0 + 1.0 / kFp8Block)};
  const dim3 grid((unsigned)cdiv(pieces, 1 << a.tx_log2),
                  (unsigned)std::min<int64_t>(cdiv(rows, 256 >> a.tx_log2), 65535));
  if (dt == ORBIT_BF16) return launch(ki, fp8_unpack_kernel<bf16>, grid, dim3(256), 0, s, a);
  return launch(ki, fp8_unpack_kernel<float>, grid, dim3(256), 0, s, a);
}

}  // namespace orbit
