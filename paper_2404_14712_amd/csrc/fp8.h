// 8-bit floating point with a scale per block of 128: the store's layout, device
// encode and decode, host launchers of the store and of the product of two stores.
//
// X[rows, n] is kept as one e4m3 code per value and one byte E per block of 128
// consecutive columns of a row (or per tile of 128 x 128, whose rows then hold
// equal E). The block's values are code 2^(E - 127) with the smallest power of two
// that brings its largest finite |x| within the format's 448: with a that value's
// float32 bits, E = ((a + 0x1fffff) >> 23) - 8 (the addition carries into the
// exponent above 1.75 = 448 / 256). A power of two makes the scaling exact, so a
// value's only error is the code's rounding, at most 2^-4 of it (or half of the
// smallest code, 2^-10, of the scale), and it is what the matrix instruction
// applies by itself: E is its exponent operand. Within 10 .. 246 every code reads
// back as a normal float32 and bf16, exactly; only float32 values above
// 448 2^119 end there. Infinities and NaN become the NaN code, one by one, so that
// a diverged value shows where it stood.
//
// Codes lie as [rows, wide], wide = n up to a multiple of 128 with zero codes past
// n, so that a product never meets a short block; E as [rows, groups], groups = the
// blocks of a row up to a multiple of 4, so that a word holds those of 512 columns.
#pragma once
#include "common.h"
#include "gemm_args.h"

namespace orbit {

constexpr int kFp8Block = 128;
inline int64_t fp8_wide(int64_t n) { return cdiv(n, kFp8Block) * kFp8Block; }
inline int64_t fp8_groups(int64_t n) { return cdiv(n, 4 * kFp8Block) * 4; }
inline size_t fp8_exp_offset(int64_t rows, int64_t n) { return align_up((size_t)rows * (size_t)fp8_wide(n)); }
inline size_t fp8_store_bytes(int64_t rows, int64_t n) {
  return align_up(fp8_exp_offset(rows, n) + (size_t)rows * (size_t)fp8_groups(n));
}

// |x| as bits, 0 where x is not finite
ORBIT_DEV uint32_t fp8_mag(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// E of a block from its largest magnitude's bits
ORBIT_DEV uint32_t fp8_exp(uint32_t a) {
  return (uint32_t)min(246, max(10, (int)((a + 0x1fffffu) >> 23) - 8));
}
// codes of 8 values of any size with the scale 2^(E - 127)
ORBIT_DEV uint2 fp8_encode8(const float* f, uint32_t e) {
  const float up = __uint_as_float((254u - e) << 23);
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __builtin_amdgcn_fmed3f(f[4 * h + i] * up, -448.f, 448.f);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], r, true);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if ((__float_as_uint(f[i]) & 0x7fffffffu) >= 0x7f800000u)
      w[i >> 2] = (w[i >> 2] & ~(0xffu << (8 * (i & 3)))) | 0x7fu << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
// values of 8 codes
ORBIT_DEV void fp8_decode8(uint2 q, uint32_t e, float* f) {
  const float s = __uint_as_float(e << 23);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int w = (int)(h ? q.y : q.x);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    f[4 * h] = a[0] * s; f[4 * h + 1] = a[1] * s; f[4 * h + 2] = b[0] * s; f[4 * h + 3] = b[1] * s;
  }
}

// x[rows, n] -> its store and / or its transposed one ([n, rows], blocks along the
// rows; either may be null). tiled: 128 x 128 tiles share their E. part (may be
// null; not with tiles, and with store_t): float32 column sums of x, one row of n
// per 128 rows. later: store_t is for another pass (so are the stores of tiles).
orbit_status fp8_pack(orbit_dtype dt, const void* x, int64_t ldx, int64_t rows, int64_t n, bool tiled, void* store,
                      void* store_t, bool later, float* part, hipStream_t s);
orbit_status fp8_unpack(orbit_dtype dt, const void* store, int64_t rows, int64_t n, void* x, int64_t ldx,
                        hipStream_t s);

// C[M, N] = sum_k A[m, k] B[n, k] over two stores [M, K] and [N, K], with the
// epilogue of gemm_args.h (operands of type dt; C float32 where out_f32, else dt)
struct Fp8Gemm {
  const void* A = nullptr;
  const void* B = nullptr;
  void* C = nullptr;
  int64_t ldc = 0;
  int M = 0, N = 0, K = 0;
  orbit_dtype dtype = ORBIT_BF16;
  bool out_f32 = false;
  Epi epi{};
};
size_t fp8_gemm_workspace_bytes(int M, int N, int K);
orbit_status fp8_gemm(const Fp8Gemm& g, void* ws, size_t ws_bytes, hipStream_t s);

}  // namespace orbit
