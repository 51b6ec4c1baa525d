// The 8-bit activation store: layout, device encode / decode, host launchers.
//
// X[rows, n] is kept as one signed byte per value and one byte per group of 32
// consecutive columns of a row (the last group of a row may be shorter). The
// group's byte E stands for the step 2^(E - 133), the smallest power of two
// with which the group's largest value rounds to at most 127 steps: with a that
// value's float32 bits, E = (a + 0x10000) >> 23 (adding 2^16 carries into the
// exponent from 127.5 / 64 on), within 7 .. 254 so that the step and its
// reciprocal stay normal floats. A power of two makes the division, the
// rounding (to nearest, ties to even) and the read back exact in any width, so
// every value is off by at most half a step (at most 1 / 127.5 of the group's
// largest where E is not clamped) and reads back as an exact bf16. E = 0 marks a
// group that held an infinity or a NaN: it reads back as NaN throughout, so that
// a diverged value is not hidden.
#pragma once
#include "common.h"

namespace orbit {

constexpr int kAct8Group = 32;
inline int act8_groups(int n) { return (int)cdiv(n, kAct8Group); }
// the E bytes [rows, groups] follow the codes [rows, n] at this offset
inline size_t act8_exp_offset(int64_t rows, int n) { return align_up((size_t)rows * (size_t)n); }
inline size_t act8_store_bytes(int64_t rows, int n) {
  return align_up(act8_exp_offset(rows, n) + (size_t)rows * act8_groups(n));
}

// maximum over the four lanes of a quad (all four active)
ORBIT_DEV uint32_t quad_umax(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));  // lanes 1,0,3,2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));  // lanes 2,3,0,1
}

// low bytes of four words
ORBIT_DEV uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}

// Codes of a lane's 8 values, a quad holding the 32 of a group (zeros where
// the row ends); returns E. All four lanes of the quad are active.
ORBIT_DEV uint32_t act8_encode(const float* f, uint2& q) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(f[i]) & 0x7fffffffu);
  a = quad_umax(a);
  const uint32_t e = min(254u, max(7u, (a + 0x10000u) >> 23));
  const float up = __uint_as_float((260u - e) << 23);  // 2^(133 - E)
  uint32_t t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    // 1.5 2^23 + v: v rounded to an integer in the low bits, in two's complement
    t[i] = __float_as_uint(__builtin_amdgcn_fmed3f(f[i] * up, -127.f, 127.f) + 12582912.f);
  q.x = low_bytes(t[0], t[1], t[2], t[3]);
  q.y = low_bytes(t[4], t[5], t[6], t[7]);
  return a >= 0x7f800000u ? 0u : e;
}

// The values of 4 codes.
ORBIT_DEV void act8_decode4(uint32_t q, uint32_t e, float* f) {
  const float step = __uint_as_float(e == 0 ? 0x7fc00000u : (e - 6u) << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(q >> (8 * i)) * step;
}

// x[rows, n], or x - sub (sub may be null), both of leading dimension ldx -> store
orbit_status act8_pack(orbit_dtype dt, const void* x, const void* sub, int64_t ldx, int64_t rows, int n, void* store,
                       hipStream_t s);
// store -> x and / or gelu(x) (either may be null)
orbit_status act8_unpack(orbit_dtype dt, const void* store, int64_t rows, int n, void* x, int64_t ldx, void* gelu,
                         int64_t ldg, hipStream_t s);

}  // namespace orbit
