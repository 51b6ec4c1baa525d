// Tiles of the kernels that copy their operands HBM -> LDS through the buffer
// unit: buffer descriptors and the wait for a ring's stage (bf16 and 8-bit products),
// and the bf16 products' K slices of 64 bytes a row, their copy plans, fragment reads
// and tile configurations.
#pragma once
#include "tile.h"

namespace orbit {

constexpr int DBK = 32;  // values of a slice's row
constexpr unsigned kOobOffset = 0x80000000u;    // beyond num_records: the copy reads zeros

#define ORBIT_LDS __attribute__((address_space(3)))

ORBIT_DEV __amdgpu_buffer_rsrc_t buffer_rsrc(const void* base, int bytes = 0x7fffffff) {
  // raw buffer over [base, base + bytes); offsets past it (kOobOffset too) read zeros
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}

// Copy plan of one operand slice (ROWS rows x 32 k) over NW waves, per lane.
//  K-major source X[row*ld + k]: LDS row r holds 64 bytes (4 chunks of 8 k);
//    logical chunk c sits at physical chunk c ^ ((r >> 2) & 3). A 1 KB copy
//    covers 16 rows.
//  M/N-major source X[k*ld + row]: LDS k-row kr holds 2 ROWS bytes (ROWS / 8
//    chunks of 8 rows); logical chunk c sits at physical chunk c ^ (4 (kr & 3)),
//    of 64 rows, two of whose k-rows span the banks, at c ^ (2 (kr & 2)).
//    A 1 KB copy covers 512 / ROWS k-rows.
template <int ROWS>
ORBIT_DEV int mn_swizzle(int kr) { return ROWS == 64 ? 2 * (kr & 2) : 4 * (kr & 3); }

template <bool KMAJ, int ROWS, int NW>
struct DmaPlan {
  static constexpr int BYTES = ROWS * DBK * 2;
  static constexpr int NL = BYTES / 1024 / NW;  // 1 KB copies per wave
  static_assert(NL >= 1 && BYTES % (1024 * NW) == 0, "copy split");
  unsigned voff[NL];
  ORBIT_DEV void init(int64_t ld, int row0, int rlim, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int blk = wave * NL + j;
      if (KMAJ) {
        const int r = blk * 16 + (lane >> 2);
        const int c = (lane & 3) ^ ((lane >> 4) & 3);
        voff[j] = (row0 + r < rlim) ? (unsigned)(r * ld * 2 + c * 16) : kOobOffset;
      } else {
        constexpr int CPR = ROWS / 8, KPB = 64 / CPR;
        const int kr = blk * KPB + lane / CPR;
        const int c = (lane % CPR) ^ mn_swizzle<ROWS>(kr);
        voff[j] = (row0 + c * 8 < rlim) ? (unsigned)(kr * ld * 2 + c * 16) : kOobOffset;
      }
    }
  }
  // RAG: K is no multiple of DBK. `left`: k of the reduction from the slice's
  // first on; a last slice short of DBK reads zeros past it (K-major: 8-k
  // pieces, else whole k-rows)
  template <bool RAG>
  ORBIT_DEV void issue(const bf16* base, int64_t ld, int left, unsigned lds, int wave, int lane) const {
    if (!RAG || left >= DBK) {
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(base);
#pragma unroll
      for (int j = 0; j < NL; ++j) dma16(r, lds + (wave * NL + j) * 1024, voff[j]);
    } else {
      const bool in = !KMAJ || (((lane & 3) ^ ((lane >> 4) & 3)) * 8 < left);
      // the address is wave-uniform, which the compiler no longer sees here
      const uint64_t p = reinterpret_cast<uint64_t>(base);
      const uint64_t u = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p) |
                         (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32;
      const __amdgpu_buffer_rsrc_t r =
          buffer_rsrc(reinterpret_cast<const void*>(u), KMAJ ? 0x7fffffff : __builtin_amdgcn_readfirstlane(left * (int)ld * 2));
#pragma unroll
      for (int j = 0; j < NL; ++j) dma16(r, lds + (wave * NL + j) * 1024, in ? voff[j] : kOobOffset);
    }
  }
};

// MFMA fragment reads from one operand slice: rows row0 + 32 i + (lane & 31),
// k-slots 8 (lane >> 5) .. +7 of the 16-deep step kk.
template <bool KMAJ, int NF, int ROWS>
struct DmaFrag {
  unsigned off[NF];
  unsigned x[2];
  ORBIT_DEV void init(int row0, int lane) {
    if (KMAJ) {
      const int f = (lane >> 2) & 3, h = lane >> 5;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) x[kk] = (unsigned)(((2 * kk + h) ^ f) << 4);
      off[0] = (unsigned)((row0 + (lane & 31)) * 64);
    } else {
      // transposing read: 16-lane group G reads k-rows 8 (G >> 1) + (q >> 2) (and
      // +4) at rows 16 (G & 1) + 4 (q & 3) .. +3; lane 16 G + i receives row
      // 16 (G & 1) + i at those k
      const int G = lane >> 4, q = lane & 15;
      const int xs = mn_swizzle<ROWS>(q >> 2);
      const int cb = 2 * (G & 1) + ((q & 3) >> 1);
#pragma unroll
      for (int i = 0; i < NF; ++i) {
        const int c = ((row0 >> 3) + i * 4 + cb) ^ xs;
        off[i] = (unsigned)((8 * (G >> 1) + (q >> 2)) * (2 * ROWS) + c * 16 + (q & 1) * 8);
      }
    }
  }
  ORBIT_DEV void read(bf16x8& f, const char* S, int i, int kk) const {
    if (KMAJ) {
      f = *reinterpret_cast<const bf16x8*>(S + off[0] + i * 2048 + x[kk]);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const char* p0 = S + off[i] + kk * 16 * (2 * ROWS);
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORBIT_LDS s16x4*)p0);
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ORBIT_LDS s16x4*)(p0 + 4 * (2 * ROWS)));
      f = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Tile configurations of the direct-to-LDS kernel. BIG: 256x256 on 8 waves
// (two per SIMD, 128x64 each), four stages, one block per CU. HALF: 256x128
// on 4 waves (128x64 each), three stages (72 KB), two independent blocks per
// CU, which fills the GPU on products with few 256x256 tiles. QUARTER: 128x128
// on 4 waves (64x64 each), four stages (64 KB), two blocks per CU, for products
// whose larger tiles leave CUs idle or need K split (eight stages, one block
// per CU: no faster, the slices' copies are not what a lone block waits for).
// THIN: 128x64, for products of 33 to 64 columns (per-head products).
template <int BM_, int BN_, int WM_, int WN_, int NS_, int OCC_, bool PP_ = false>
struct DmaCfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_, OCC = OCC_;
  static constexpr bool PP = PP_;
  static constexpr int NW = WM * WN, NT = NW * 64;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static constexpr int OPA = BM * DBK * 2, OPB = BN * DBK * 2, STB = OPA + OPB;
  static constexpr int EPB = NW * 32 * (TN * 32 + 8) * 4;   // epilogue staging
  static constexpr int LDS = NS * STB > EPB ? NS * STB : EPB;
};
using DmaBig = DmaCfg<256, 256, 2, 4, 4, 1>;
using DmaHalf = DmaCfg<256, 128, 2, 2, 3, 2>;
using DmaPP = DmaCfg<256, 256, 2, 4, 4, 1, true>;   // BIG in two wave groups
using DmaQuarter = DmaCfg<128, 128, 2, 2, 4, 2>;
using DmaThin = DmaCfg<128, 64, 4, 1, 4, 3>;

// wait until stage s has landed when copies of the next `ahead` stages
// (each NLS copies per wave) may still be in flight
template <int NLS, int NS>
ORBIT_DEV void wait_stage(int ahead) {
  if constexpr (NS > 2) {
    if (ahead >= NS - 2) wait_vmcnt<(NS - 2) * NLS>();
    else wait_stage<NLS, NS - 1>(ahead);
  } else {
    wait_vmcnt<0>();
  }
}

}  // namespace orbit
