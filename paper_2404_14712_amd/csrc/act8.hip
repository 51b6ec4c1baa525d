// The 8-bit activation store (act8.h): packing a tensor, and reading it back
// with an optional GELU. HBM-bound: 8 columns per lane, a quad per group.
#include <algorithm>

#include "act8.h"

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

// A matrix as the kernels walk it: `rows` rows of `n` columns; TX threads of a
// block along a row (8 columns each), 256 / TX rows per block. A matrix
// without gaps whose rows are whole groups is walked as one long row.
struct Act8Shape {
  int64_t rows, n, groups, tx;
  dim3 grid;
};

Act8Shape act8_shape(int64_t rows, int n, bool flat) {
  Act8Shape z{};
  z.rows = flat ? 1 : rows;
  z.n = flat ? rows * n : n;
  z.groups = cdiv(z.n, kAct8Group);
  const int64_t pieces = 4 * z.groups;
  z.tx = std::min<int64_t>(256, pow2_ceil((int)std::min<int64_t>(pieces, 256)));
  z.grid = dim3((unsigned)cdiv(pieces, z.tx), (unsigned)std::min<int64_t>(cdiv(z.rows, 256 / z.tx), 65535));
  return z;
}

template <typename T>
__global__ void __launch_bounds__(256) act8_pack_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows,
                                                        int64_t n, int64_t groups, int tx,
                                                        uint8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  const int64_t piece = (int64_t)blockIdx.x * tx + threadIdx.x % tx;
  const int64_t col = piece * 8;
  const int ty = 256 / tx;
  for (int64_t r = (int64_t)blockIdx.y * ty + threadIdx.x / tx; r < rows; r += (int64_t)gridDim.y * ty) {
    float f[8];
    if (col < n) {
      load8(x + r * ldx + col, f);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = 0.f;
    }
    uint2 q;
    const uint32_t e = act8_encode(f, q);
    if (col < n) {
      *reinterpret_cast<uint2*>(codes + r * n + col) = q;
      if (piece % 4 == 0) exps[r * groups + piece / 4] = (uint8_t)e;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) act8_unpack_kernel(const uint8_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ exps, int64_t rows, int64_t n,
                                                          int64_t groups, int tx, T* __restrict__ x, int64_t ldx,
                                                          T* __restrict__ g, int64_t ldg) {
  const int64_t piece = (int64_t)blockIdx.x * tx + threadIdx.x % tx;
  const int64_t col = piece * 8;
  const int ty = 256 / tx;
  if (col >= n) return;
  for (int64_t r = (int64_t)blockIdx.y * ty + threadIdx.x / tx; r < rows; r += (int64_t)gridDim.y * ty) {
    float f[8];
    act8_decode(*reinterpret_cast<const uint2*>(codes + r * n + col), exps[r * groups + piece / 4], f);
    if (x) store8(x + r * ldx + col, f);
    if (g) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = gelu_f(f[i]);
      store8(g + r * ldg + col, f);
    }
  }
}

}  // namespace

orbit_status act8_pack(orbit_dtype dt, const void* x, int64_t ldx, int64_t rows, int n, void* store, hipStream_t s) {
  const Act8Shape z = act8_shape(rows, n, n % kAct8Group == 0 && ldx == n);
  uint8_t* codes = static_cast<uint8_t*>(store);
  uint8_t* exps = codes + act8_exp_offset(rows, n);
  const double e = dt == ORBIT_BF16 ? 2.0 : 4.0;
  KernelInfo ki{dt == ORBIT_BF16 ? "act8_pack<bf16>" : "act8_pack<f32>", 4.0 * rows * n,
                (e + 1.0 + 1.0 / kAct8Group) * rows * n};
  if (dt == ORBIT_BF16)
    return launch(ki, act8_pack_kernel<bf16>, z.grid, dim3(256), 0, s, static_cast<const bf16*>(x), ldx, z.rows, z.n,
                  z.groups, (int)z.tx, codes, exps);
  return launch(ki, act8_pack_kernel<float>, z.grid, dim3(256), 0, s, static_cast<const float*>(x), ldx, z.rows, z.n,
                z.groups, (int)z.tx, codes, exps);
}

orbit_status act8_unpack(orbit_dtype dt, const void* store, int64_t rows, int n, void* x, int64_t ldx, void* gelu,
                         int64_t ldg, hipStream_t s) {
  const bool flat = n % kAct8Group == 0 && (!x || ldx == n) && (!gelu || ldg == n);
  const Act8Shape z = act8_shape(rows, n, flat);
  const uint8_t* codes = static_cast<const uint8_t*>(store);
  const uint8_t* exps = codes + act8_exp_offset(rows, n);
  const double e = dt == ORBIT_BF16 ? 2.0 : 4.0;
  KernelInfo ki{dt == ORBIT_BF16 ? "act8_unpack<bf16>" : "act8_unpack<f32>", 4.0 * rows * n,
                (e * ((x ? 1 : 0) + (gelu ? 1 : 0)) + 1.0 + 1.0 / kAct8Group) * rows * n};
  if (dt == ORBIT_BF16)
    return launch(ki, act8_unpack_kernel<bf16>, z.grid, dim3(256), 0, s, codes, exps, z.rows, z.n, z.groups, (int)z.tx,
                  static_cast<bf16*>(x), ldx, static_cast<bf16*>(gelu), ldg);
  return launch(ki, act8_unpack_kernel<float>, z.grid, dim3(256), 0, s, codes, exps, z.rows, z.n, z.groups, (int)z.tx,
                static_cast<float*>(x), ldx, static_cast<float*>(gelu), ldg);
}

}  // namespace orbit
