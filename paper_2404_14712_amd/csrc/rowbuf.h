// A row of a row-major tensor through the buffer unit: a wave-uniform
// descriptor of the row's bytes and one 32-bit offset per lane. Reads past the
// row give zeros and writes past it are dropped, so that kernels whose lanes
// overhang a row, whose last chunk has fewer rows, or whose tensor is absent
// (zero bytes) need no branches around their loads and stores.
#pragma once
#include "common.h"

namespace orbit {

typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32v2 __attribute__((ext_vector_type(2)));

// an offset past every descriptor: nothing is read (zeros) or written there
constexpr uint32_t kNoOffset = 0x7fffffffu;

struct RowBuf {
  __amdgpu_buffer_rsrc_t r;
  // bytes of the tensor p from byte `off` on (both wave-uniform)
  ORBIT_DEV RowBuf(const void* p, int64_t off, int bytes)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p)) + off, 0, bytes,
                                            0x00020000)) {}
};

// 8 values of T as stored (bf16 stays packed: 4 registers instead of 8); get4
// gives one half of them as floats
template <typename T>
struct Raw8 {
  static constexpr int NV = sizeof(T) / 2;
  u32v4 v[NV];
  template <int AUX = 0> ORBIT_DEV void load(const RowBuf& b, uint32_t off) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(b.r, off + 16 * i, 0, AUX);
  }
  ORBIT_DEV void store(const RowBuf& b, uint32_t off) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) __builtin_amdgcn_raw_buffer_store_b128(v[i], b.r, off + 16 * i, 0, 0);
  }
  // all bits of every word or-ed with m
  ORBIT_DEV void or_bits(uint32_t m) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] |= m;
  }
  // makes the compiler unpack again what it unpacked before, instead of
  // keeping the floats in registers
  ORBIT_DEV void renew() {
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(v[i]));
  }
  ORBIT_DEV void get4(int h, float* f) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[2 * i] = __uint_as_float(v[0][2 * h + i] << 16);
        f[2 * i + 1] = __uint_as_float(v[0][2 * h + i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[h][i]);
    }
  }
  ORBIT_DEV void put4(int h, const float* f) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x2 p = {(bf16)f[2 * i], (bf16)f[2 * i + 1]};
        v[0][2 * h + i] = __builtin_bit_cast(uint32_t, p);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[h][i] = __float_as_uint(f[i]);
    }
  }
};
// bits of 1 in T, in every place of a word
template <typename T> constexpr uint32_t one_bits() { return sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u; }

}  // namespace orbit
