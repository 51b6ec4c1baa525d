// The product of two 8-bit floating-point stores (fp8.h), C = A B^T with the
// epilogues of gemm_args.h, on v_mfma_scale_f32_32x32x64_f8f6f4: the instruction
// takes each operand row's E of a 32-deep piece as an exponent, so that the scales
// of the blocks cost no vector instructions and the sums stay in one float32
// accumulator.
//
// What that instruction adds exactly is the running sum: it aligns the products
// of one step to the largest of them and drops what lies more than 13 bits below
// (measured: 2^-14 of the largest is lost, where bf16 products keep 2^-23). Sums come
// out 1e-5 to 4e-5 off in the 2-norm, a hundredth of a bf16 result's own rounding, so
// bf16 results take it: at 4096 x 4096 x 8192 2.3% of them are another bf16 value than a
// float32 sum gives, and the distance to the exact sums is 1.6594e-3 against 1.6591e-3. Float32 results are formed with EXACT instead: the codes are
// turned into bf16 with their scales in the fragments, which is exact, and the bf16
// instructions keep every bit a float32 sum can, at half the rate.
//
// The other products go through LDS, whose rings are filled by copies without
// registers (dma.h). Two kernels share that work:
//   wide   256 x 256 on 4 waves, one block per CU that walks over tiles: more than 512 tiles
//          of 128 x 128;
//   tile   128 x 128, 64 x 128 or 64 x 64 on 4 waves, the smallest that leaves a block per CU,
//          K split where there are few: the rest.
//
// A few rows of A (single tokens) read B once, and what counts is the latency of that one
// read: fp8_thin_kernel spreads it over the waves of many small blocks, past 16x16x128
// instructions without LDS.
#include <algorithm>
#include <type_traits>

#include "dma.h"
#include "fp8.h"
#include "gemm.h"

namespace orbit {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Fp8Args {
  const uint8_t *A, *B, *Ae, *Be;  // codes and E bytes
  int64_t lda, ldb;                // bytes of a row of codes
  int gpa, gpb;                    // and of E
  void* C;
  int64_t ldc;
  int M, N, slices;                // 64-deep slices of K
  int splits;                      // of K, each of whole blocks of 128
  float* partial;                  // splits > 1: [splits][M][N]
  Epi epi;
};

// one wave copies 64 words from rsrc + voff (per lane) to LDS byte address lds + 4 * lane
ORBIT_DEV void dma4(__amdgpu_buffer_rsrc_t r, unsigned lds, unsigned voff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(r)
               : "memory", "m0");
}

// 2 and 8 floats as bf16, a conversion for two
ORBIT_DEV uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(bf16)a, (bf16)b}); }
ORBIT_DEV U128 pack8(const float* f) {
  return U128{{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])}};
}
// 2^(E - 127) from the low byte of an E word
ORBIT_DEV float fp8_scale(int e) { return __uint_as_float((unsigned)(e & 0xff) << 23); }
// 8 codes as bf16 values with their scale (exact)
ORBIT_DEV bf16x8 fp8_bf16x8(int lo, int hi, float s) {
  const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false);
  const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
  const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false);
  const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// The products of a slice's fragments, ea and eb holding the rows' E in their low bytes.
template <int TM, int TN, bool EXACT>
ORBIT_DEV void mma_slice(f32x16 (&c)[TM][TN], const i32x8* a, const i32x8* b, const int* ea, const int* eb) {
  if constexpr (!EXACT) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        c[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], c[i][j], 0, 0, 0, ea[i], 0, eb[j]);
  } else {
    float sa[TM], sb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = fp8_scale(ea[i]);
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = fp8_scale(eb[j]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      bf16x8 x[TM], y[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) x[i] = fp8_bf16x8(a[i][2 * k], a[i][2 * k + 1], sa[i]);
#pragma unroll
      for (int j = 0; j < TN; ++j) y[j] = fp8_bf16x8(b[j][2 * k], b[j][2 * k + 1], sb[j]);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], c[i][j], 0, 0, 0);
    }
  }
}

// The lin-th of nt tiles, as in gemm_dma_kernel: XCD-contiguous ranges of tile ids,
// walked in groups of tile rows.
template <int BM, int BN>
ORBIT_DEV void fp8_tile_of(const Fp8Args& g, int id, int& m0, int& n0) {
  const int tiles_n = (g.N + BN - 1) / BN, tiles_m = (g.M + BM - 1) / BM;
  constexpr int GR = BN == 128 ? 4 : 8;
  const int per_group = GR * tiles_n;
  const int first_m = (id / per_group) * GR;
  const int gsize = min(tiles_m - first_m, GR);
  m0 = (first_m + (id % per_group) % gsize) * BM;
  n0 = ((id % per_group) / gsize) * BN;
}
template <int BM, int BN>
ORBIT_DEV void fp8_tile(const Fp8Args& g, int lin, int nt, int& m0, int& n0) {
  const int full = nt - nt % 8;
  fp8_tile_of<BM, BN>(g, lin < full ? (lin % 8) * (full / 8) + lin / 8 : lin, m0, n0);
}
// The first block of 128 k of split s: the splits differ by one at most.
ORBIT_DEV int fp8_split_at(const Fp8Args& g, int s) { return (int)((int64_t)(g.slices >> 1) * s / g.splits); }
// A block's tile and K range: with split K an XCD takes one range.
template <int BM, int BN>
ORBIT_DEV void fp8_tile(const Fp8Args& g, int& m0, int& n0, int& split) {
  split = blockIdx.z;
  const int nt = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  if (g.splits > 1 && 8 % g.splits == 0 && (nt * g.splits) % 8 == 0) {
    const int lin = blockIdx.x + nt * (int)blockIdx.z, xcd = lin % 8;
    split = xcd % g.splits;
    fp8_tile_of<BM, BN>(g, (xcd / g.splits) * (nt * g.splits / 8) + lin / 8, m0, n0);
  } else {
    fp8_tile<BM, BN>(g, blockIdx.x, nt, m0, n0);
  }
}

// Through LDS: each wave parks 32 rows of its accumulators and reads them back as 8
// consecutive columns per lane.
template <typename T, typename OutT, typename CF>
ORBIT_DEV void fp8_epilogue(const Fp8Args& g, f32x16 (&acc)[CF::TM][CF::TN], char* smem, int wave, int lane, int m0,
                            int n0, int split) {
  constexpr int TM = CF::TM, TN = CF::TN, WTN = TN * 32, EP = WTN + 8, LPR = WTN / 8, RPI = 64 / LPR;
  const int wm = wave % CF::WM, wn = wave / CF::WM;
  float* ew = reinterpret_cast<float*>(smem) + wave * 32 * EP;
  OutT* C = static_cast<OutT*>(g.C);
  const bool raw = g.splits > 1;
  const int cl = (lane % LPR) * 8, c0 = n0 + wn * WTN + cl;
  float b8[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) b8[q] = 0.f;
  if (!raw && g.epi.bias && c0 < g.N) ld8(static_cast<const T*>(g.epi.bias) + c0, b8);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        ew[((v >> 2) * 8 + (lane >> 5) * 4 + (v & 3)) * EP + j * 32 + (lane & 31)] = acc[i][j][v];
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int it = 0; it < 32 / RPI; ++it) {
      const int rl = it * RPI + lane / LPR;
      const int r = m0 + wm * TM * 32 + i * 32 + rl;
      float v8[8];
      const f32x4 lo = *reinterpret_cast<const f32x4*>(ew + rl * EP + cl);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(ew + rl * EP + cl + 4);
#pragma unroll
      for (int q = 0; q < 4; ++q) { v8[q] = lo[q]; v8[4 + q] = hi[q]; }
      if (r < g.M && c0 < g.N) {
        if (raw) st8(g.partial + ((int64_t)split * g.M + r) * g.N + c0, v8);
        else epi_apply8<T, OutT>(g.epi, 0, r, c0, v8, C, g.ldc, b8);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Tiles of 128 x 128, 64 x 128 or 64 x 64 on 4 waves. A stage is a block of 128 k: rows of
// 128 bytes, whole cache lines, as in the wide kernel below; its halves of 64 k pass through
// two sets of registers, so that products cover the reads, and one barrier serves 128 k
// (stages of 64 k and rows of 64 bytes: 8192 x 1024 x 4096 46 us against 39, 2048 x 4096 x 2048
// 25.7 against 22.8).
//
// What a lone block per CU takes is the latency of its stages one after another, so that few
// tiles are cut small, while there are at most 256: 1024 x 1024 x 1024 on 128 x 128, 64 x 128,
// 64 x 64 9.6, 7.2, 6.3 us (float32 results 12.4, 9.9, 8.5), 1770 x 1000 x 2056 15.2, 10.9.
// Long K is shared by two groups of waves, whose sums meet in LDS at the end: bf16 results
// 1024 x 1024 x 4096 12.8 -> 11.5 us, 1024 x 4096 x 4096 25.1 -> 23.6, 512 x 512 x 2048 8.0 -> 7.8,
// but 512 x 4096 x 1536 9.2 -> 9.6 (on 128 x 128 from K = 1024: 2048 x 2048 x 1024 11.7 -> 11.2);
// float32 results, which have more to do on a stage, 1024 x 1024 x 1024 8.6 -> 8.1, 150 x 768 x
// 1000 7.0 -> 6.5, but 512 x 512 x 256 4.26 -> 4.58 and none on 128 x 128. One group has three
// stages in flight (64 x 128 on two: 2048 x 1024 x 4096 22.5 us against 17.3), except where two
// blocks share a CU (8192 x 1024 x 4096 39.2 us with two stages and two blocks, 48.9 with four
// and one).
// BM x BN by KG groups of 4 waves, each with its part of K and its own ring of NS stages
template <int BM_, int BN_, int NS, int KG>
struct TileCfg {
  static constexpr int BM = BM_, BN = BN_, WM = 2, WN = 2, TM = BM / 64, TN = BN / 64, NT = KG * 256;
  static constexpr int OPA = BM * 128, STB = OPA + BN * 128, E = NS * STB, RING = E + 2 * (BM + BN) * 4;
  static constexpr int EPB = 4 * 32 * (TN * 32 + 8) * 4;              // epilogue's rows
  static constexpr int SUM = (KG - 1) * 4 * TM * TN * 16 * 64 * 4;    // the other groups' sums, behind these
  static constexpr int LDS = KG * RING;
  static_assert(LDS >= EPB + SUM && LDS <= 160 * 1024, "LDS");
};
template <typename T, typename OutT, int BM_, int BN_, int NS, int KG>
__global__ void __launch_bounds__(KG * 256, KG == 1 && NS == 2 ? 2 : 1) gemm_fp8_tile_kernel(Fp8Args g) {
  using CF = TileCfg<BM_, BN_, NS, KG>;
  constexpr int NA = CF::BM / 32, NB = CF::BN / 32;  // copies of a wave per stage
  constexpr int BM = CF::BM, BN = CF::BN, TM = CF::TM, TN = CF::TN;
  constexpr bool EXACT = sizeof(OutT) == 4;
  extern __shared__ __attribute__((aligned(1024))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, grp = __builtin_amdgcn_readfirstlane(tid >> 8);
  char* smem = shared + grp * CF::RING;
  const int wm = wave % CF::WM, wn = wave / CF::WM;
  int m0, n0, split;
  fp8_tile<BM, BN>(g, m0, n0, split);
  m0 = __builtin_amdgcn_readfirstlane(m0);
  n0 = __builtin_amdgcn_readfirstlane(n0);
  split = __builtin_amdgcn_readfirstlane(split);
  const int beg = fp8_split_at(g, split), nb = fp8_split_at(g, split + 1) - beg;
  const int b0 = beg + nb * grp / KG, nk = beg + nb * (grp + 1) / KG - b0;  // the group's stages
  const int steps = (nb + KG - 1) / KG;                                      // the longest group's
  const int rm = min(g.M - m0, BM), rn = min(g.N - n0, BN);
  const uint8_t* Ab = g.A + (int64_t)m0 * g.lda + (int64_t)b0 * 128;
  const uint8_t* Bb = g.B + (int64_t)n0 * g.ldb + (int64_t)b0 * 128;
  const uint8_t* Aeb = g.Ae + (int64_t)m0 * g.gpa;
  const uint8_t* Beb = g.Be + (int64_t)n0 * g.gpb;

  // copy c of a wave's n: rows 8 (n wave + c) + lane / 8 of the operand; rows behind its
  // last one read zeros
  unsigned va[NA], vb[NB];
  auto offsets = [&](unsigned* v, int n, int64_t ld, int rows) {
#pragma unroll
    for (int c = 0; c < n; ++c) {
      const int r = (wave * n + c) * 8 + (lane >> 3), k = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
      v[c] = r < rows ? (unsigned)(r * (int)ld + k) : kOobOffset;
    }
  };
  offsets(va, NA, g.lda, rm);
  offsets(vb, NB, g.ldb, rn);
  // E words, of A's rows and then of B's: wave w copies 64 of them
  const bool ofa = wave < BM / 64;
  const int er = wave * 64 + lane - (ofa ? 0 : BM);
  const unsigned ve = er < (ofa ? rm : rn) ? (unsigned)(er * (ofa ? g.gpa : g.gpb)) : kOobOffset;
  const unsigned lds0 = (unsigned)(uintptr_t)(ORBIT_LDS void*)smem;
  auto issue = [&](int st) {
    const int b = b0 + st;
    if (((b & 3) == 0 || st == 0) && wave < (BM + BN) / 64)  // before the stage's codes: landed when these have
      dma4(buffer_rsrc((ofa ? Aeb : Beb) + (b >> 2) * 4), lds0 + CF::E + ((b >> 2) & 1) * ((BM + BN) * 4) + wave * 256, ve);
    const unsigned at = lds0 + (st % NS) * CF::STB;
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(Ab + (int64_t)st * 128), rb = buffer_rsrc(Bb + (int64_t)st * 128);
#pragma unroll
    for (int c = 0; c < NA; ++c) dma16(ra, at + (wave * NA + c) * 1024, va[c]);
#pragma unroll
    for (int c = 0; c < NB; ++c) dma16(rb, at + CF::OPA + (wave * NB + c) * 1024, vb[c]);
  };
  int ea[TM], eb[TN];
  auto scales = [&](int st) {
    const int b = b0 + st;
    if ((b & 3) == 0 || st == 0) {
      const int* E = reinterpret_cast<const int*>(smem + CF::E + ((b >> 2) & 1) * ((BM + BN) * 4));
      const int by = (b & 3) * 8;
#pragma unroll
      for (int i = 0; i < TM; ++i) ea[i] = (int)((unsigned)E[wm * TM * 32 + i * 32 + (lane & 31)] >> by);
#pragma unroll
      for (int j = 0; j < TN; ++j) eb[j] = (int)((unsigned)E[BM + wn * TN * 32 + j * 32 + (lane & 31)] >> by);
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) ea[i] = (int)((unsigned)ea[i] >> 8);
#pragma unroll
      for (int j = 0; j < TN; ++j) eb[j] = (int)((unsigned)eb[j] >> 8);
    }
  };
  const int lr = lane & 31;
  const unsigned oa = (unsigned)((wm * TM * 32 + lr) * 128), ob = (unsigned)(CF::OPA + (wn * TN * 32 + lr) * 128);
  unsigned x[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = (unsigned)(((2 * q + (lane >> 5)) ^ ((lr >> 1) & 7)) << 4);
  // half hf (64 k) of a stage's fragments
  auto read = [&](i32x8* fa, i32x8* fb, const char* S, int hf) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
      fa[i] = __builtin_shufflevector(*reinterpret_cast<const i32x4*>(S + oa + i * 4096 + x[2 * hf]),
                                      *reinterpret_cast<const i32x4*>(S + oa + i * 4096 + x[2 * hf + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
    for (int j = 0; j < TN; ++j)
      fb[j] = __builtin_shufflevector(*reinterpret_cast<const i32x4*>(S + ob + j * 4096 + x[2 * hf]),
                                      *reinterpret_cast<const i32x4*>(S + ob + j * 4096 + x[2 * hf + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
#pragma unroll
  for (int st = 0; st < NS; ++st)
    if (st < nk) issue(st);
  wait_stage<NA + NB, NS + 1>(max(min(nk - 1, NS - 1), 0));
  __syncthreads();
  i32x8 fa[TM], fb[TN], ga[TM], gb[TN];
  read(fa, fb, smem, 0);
  for (int kt = 0; kt < steps; ++kt) {
    const bool on = KG == 1 || kt < nk;
    const char* here = smem + (kt % NS) * CF::STB;
    if (on) {
      scales(kt);
      read(ga, gb, here, 1);
      mma_slice<TM, TN, EXACT>(acc, fa, fb, ea, eb);
    }
    // the stage is in registers everywhere and the next one has landed
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_stage<NA + NB, NS + 1>(max(min(nk - kt - 2, NS - 2), 0));
    __syncthreads();
    // past the last stage this reads a stale but in-bounds slot
    read(fa, fb, smem + ((kt + 1) % NS) * CF::STB, 0);
    if (kt + NS < nk) issue(kt + NS);
    if (on) mma_slice<TM, TN, EXACT>(acc, ga, gb, ea, eb);
  }
  wait_vmcnt<0>();
  __syncthreads();
  if constexpr (KG > 1) {
    // the groups' sums in their order
    f32x4* sums = reinterpret_cast<f32x4*>(shared + CF::EPB);
    auto at = [&](int q, int i, int j, int v) { return ((((q - 1) * 4 + wave) * TM * TN + i * TN + j) * 4 + v) * 64 + lane; };
    if (grp) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            sums[at(grp, i, j, v)] = f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
    }
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int q = 1; q < KG; ++q)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const f32x4 t = sums[at(q, i, j, v)];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][4 * v + e] += t[e];
          }
  }
  fp8_epilogue<T, OutT, CF>(g, acc, shared, wave, lane, m0, n0, split);
}

// Results of many tiles: 256 x 256 on 4 waves of 128 x 128, one per SIMD. A
// fragment is then read for four products instead of two or four (half of the LDS
// time that the MFMAs take), and a wave's own order of instructions overlaps
// everything: after an MFMA, which takes 64 cycles, come reads of the next
// fragments or a copy of the stage after the next.
//
// A stage is a block of 128 k: rows of 128 bytes, a whole cache line, since copies of
// 64-byte pieces of rows take the L2 twice the requests (measured beside the MFMAs: 77
// to 109 cycles an MFMA by the rows' distance, against 65.5). LDS holds two stages;
// chunk c of row r lies at c ^ ((r >> 1) & 7), so that fragment reads of 16
// consecutive rows meet every bank once. A stage's two halves of 64 k pass through
// two sets of registers:
//   half 0: products of X, reads of half 1 into Y; when these are done everywhere the
//           stage's slot is free and the copies of the stage after the next begin;
//   half 1: products of Y, reads of the next stage's half 0 into X, more copies.
// Blocks stay, one per CU, and walk over tiles: the stage after a tile's last is the
// next tile's first, which is in LDS when a tile's results go out through LDS of their
// own. All 256 accumulation registers hold sums, so the epilogue's 256 vector registers
// have to do without a spill: one would wait for every copy and store in flight (22
// spilled registers: 4 to 14 us a round of tiles).
//
// Measured: 8192 x 8192 x 8192 405 to 415 us by the card (2650 to 2715 TFLOP/s; two groups of 4
// waves of 128 x 64 that take turns at reading and multiplying 456), 4096 x 4096 x 8192 104 (121), 4096 x 8192 x 4096
// 109 (123), 8192 x 8192 x 1024 75 (92). A stage takes 1.49 us, 2880 TFLOP/s, near what the
// matrix cores reach on random codes at the card's power limit (3200); a round of tiles costs
// 9 to 18 us beside its stages, of which 7 are 32 MB of results at the memory's rate: there
// is no room in LDS or registers to let the next tile's sums begin before these are out.
//
// Float32 results take four bf16 instructions of 32 cycles for one of 64, and a wave has
// time to decode between them: 8192 x 8192 x 8192 748 to 775 us (1420 to 1470 TFLOP/s), 4096 x 4096 x 8192
// 200, 8192 x 8192 x 2048 227, 8192 x 4096 x 4096 202 (two groups of 4 waves, one decoding and
// multiplying while the other reads: 810, 212, 272, 229; a bf16 library product of the first
// 859), and 8192 x 8192 x 1024 142 (tiles of 128 x 128: 168).
constexpr int kWideStage = 2 * 256 * 128;
constexpr int kWideE = 2 * kWideStage, kWideBias = kWideE + 2 * 512 * 4, kWideOut = kWideBias + 2 * 1024;
constexpr int kWidePitch = 272, kWideLds = kWideOut + 4 * 16 * kWidePitch;  // 16 rows of 128 bf16 per wave
static_assert(kWideLds <= 160 * 1024, "LDS");

// what happens to a sum (with its bias) before it is stored
enum WideEpi { kWidePlain, kWideGelu, kWideGeluGrad, kWideRes, kWideF32, kWideF32Add };

template <typename T, WideEpi EPI>
__global__ void __launch_bounds__(256, 1) gemm_fp8_wide_kernel(Fp8Args g) {
  constexpr bool EXACT = EPI == kWideF32 || EPI == kWideF32Add;
  constexpr int OPA = 256 * 128;  // bytes of A in a stage
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const int nk = g.slices >> 1;  // stages of a tile, at least 2
  const int nt = ((g.M + 255) >> 8) * ((g.N + 255) >> 8);

  struct Tile {
    const uint8_t *A, *B, *Ae, *Be;
    int m0, n0, rm, rn;  // rows of A and of B, 0 past the last tile
  };
  auto tile_at = [&](int lin) {
    Tile t;
    fp8_tile<256, 256>(g, min(lin, nt - 1), nt, t.m0, t.n0);
    // (a division: left in vector registers otherwise)
    t.m0 = __builtin_amdgcn_readfirstlane(t.m0);
    t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
    t.A = g.A + (int64_t)t.m0 * g.lda;
    t.B = g.B + (int64_t)t.n0 * g.ldb;
    t.Ae = g.Ae + (int64_t)t.m0 * g.gpa;
    t.Be = g.Be + (int64_t)t.n0 * g.gpb;
    t.rm = lin < nt ? min(g.M - t.m0, 256) : 0;
    t.rn = lin < nt ? min(g.N - t.n0, 256) : 0;
    return t;
  };
  // copy c of a wave: rows 8 (8 wave + c) + lane / 8 of the operand, 16 (c / 2) rows behind
  // those of copy c & 1; the descriptor ends behind the tile's last row
  unsigned va[2], vb[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int r = (wave * 8 + c) * 8 + (lane >> 3), k = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    va[c] = (unsigned)(r * (int)g.lda + k);
    vb[c] = (unsigned)(r * (int)g.ldb + k);
  }
  // E words: wave w copies those of 64 rows of A and of B; bias: 64 words each of waves 0, 1
  const unsigned vea = (unsigned)((wave * 64 + lane) * g.gpa), veb = (unsigned)((wave * 64 + lane) * g.gpb);
  const unsigned vbias = wave < 2 ? (unsigned)((wave * 64 + lane) * 4) : kOobOffset;

  const unsigned lds0 = (unsigned)(uintptr_t)(ORBIT_LDS void*)smem;
  Tile cur = tile_at(blockIdx.x), nxt = tile_at(blockIdx.x + gridDim.x);
  int par = 0, epar = 0, bpar = 0;  // slots of the tile's first stage, first E words, bias

  // what stage st of the tile copies, st >= nk being the next tile's
  struct Src {
    __amdgpu_buffer_rsrc_t a, b;
    unsigned lds;
  };
  auto source = [&](int st) {
    const bool here = st < nk;
    const int s = here ? st : st - nk;
    const int rm = here ? cur.rm : nxt.rm, rn = here ? cur.rn : nxt.rn;
    Src x;
    x.a = buffer_rsrc((here ? cur.A : nxt.A) + s * 128, max(rm * (int)g.lda - s * 128, 0));
    x.b = buffer_rsrc((here ? cur.B : nxt.B) + s * 128, max(rn * (int)g.ldb - s * 128, 0));
    x.lds = lds0 + ((par + st) & 1) * kWideStage + wave * 8192;
    return x;
  };
  auto copy = [&](const Src& x, int c) {
    const int d = c & 7;
    if (c < 8) dma16(x.a, x.lds + c * 1024, va[d & 1] + (unsigned)((d >> 1) * 16 * (int)g.lda));
    else dma16(x.b, x.lds + OPA + d * 1024, vb[d & 1] + (unsigned)((d >> 1) * 16 * (int)g.ldb));
  };
  // the E words of stage st's 512 k, copied again with every stage of these (the same
  // words: no branch in a stage), the first time with the first one's codes
  auto copy_e = [&](int st) {
    const bool here = st < nk;
    const int s = (here ? st : st - nk) & ~3;
    const int slot = here ? epar ^ ((st >> 2) & 1) : epar ^ (((nk + 3) >> 2) & 1);
    const int rm = here ? cur.rm : nxt.rm, rn = here ? cur.rn : nxt.rn;
    const unsigned b = lds0 + kWideE + slot * 2048 + wave * 256;
    dma4(buffer_rsrc((here ? cur.Ae : nxt.Ae) + s, max(rm * g.gpa - s, 0)), b, vea);
    dma4(buffer_rsrc((here ? cur.Be : nxt.Be) + s, max(rn * g.gpb - s, 0)), b + 1024, veb);
  };
  auto copy_bias = [&](const Tile& t, int slot) {
    const int bytes = g.epi.bias ? t.rn * 2 : 0;
    dma4(buffer_rsrc(g.epi.bias ? static_cast<const char*>(g.epi.bias) + t.n0 * 2 : reinterpret_cast<const char*>(g.A), bytes),
         lds0 + kWideBias + slot * 1024 + wave * 256, vbias);
  };

  struct Set {
    i32x8 f[8];  // fragments: 4 of A, 4 of B
  };
  const int lr = lane & 31;
  const unsigned oa = (unsigned)((wm * 128 + lr) * 128), ob = (unsigned)(OPA + (wn * 128 + lr) * 128);
  unsigned x[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = (unsigned)(((2 * q + (lane >> 5)) ^ ((lr >> 1) & 7)) << 4);
  // chunk q of fragment f of half hf
  auto read = [&](Set& s, const char* S, int hf, int f, int q) {
    const i32x4 v = *reinterpret_cast<const i32x4*>(S + (f < 4 ? oa : ob) + (f & 3) * 4096 + x[2 * hf + q]);
#pragma unroll
    for (int w = 0; w < 4; ++w) s.f[f][4 * q + w] = v[w];
  };
  // E words of the fragments' rows: the stage's byte lies lowest, the next stage's above it
  int ea[4], eb[4];
  auto scales = [&](int slot) {
    const char* E = smem + kWideE + slot * 2048;
#pragma unroll
    for (int i = 0; i < 4; ++i) ea[i] = *reinterpret_cast<const int*>(E + (wm * 128 + i * 32 + lr) * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) eb[j] = *reinterpret_cast<const int*>(E + 1024 + (wn * 128 + j * 32 + lr) * 4);
  };
  // the waves meet: what each waited for holds for all
  auto meet = [&] {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };

  if constexpr (!EXACT) copy_bias(cur, 0);
  copy_e(0);
  {
    const Src s = source(0);
#pragma unroll
    for (int c = 0; c < 16; ++c) copy(s, c);
  }
  copy_e(1);
  {
    const Src s = source(1);
#pragma unroll
    for (int c = 0; c < 16; ++c) copy(s, c);
  }
  wait_vmcnt<18>();
  __syncthreads();
  for (int lin = blockIdx.x; lin < nt; lin += gridDim.x) {
    // the first half stage (read again here, so that its registers are free between
    // two tiles)
    Set X, Y;
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      read(X, smem + par * kWideStage, 0, f, 0);
      read(X, smem + par * kWideStage, 0, f, 1);
    }
    // the sums begin with the bias: lane l holds columns 8 q + 4 (l >> 5) .. +3
    f32x16 acc[4][4];
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = cur.n0 + wn * 128 + j * 32 + q * 8 + (lane >> 5) * 4;
          float b[4] = {0.f, 0.f, 0.f, 0.f};
          if (g.epi.bias && c < g.N) {
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = to_f(static_cast<const T*>(g.epi.bias)[c + e]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = b[e];
        }
    } else {
      const char* bias = smem + kWideBias + bpar * 1024 + (wn * 128 + (lane >> 5) * 4) * 2;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint2 b = *reinterpret_cast<const uint2*>(bias + (j * 32 + q * 8) * 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[i][j][4 * q] = __uint_as_float(b.x << 16);
            acc[i][j][4 * q + 1] = __uint_as_float(b.x & 0xffff0000u);
            acc[i][j][4 * q + 2] = __uint_as_float(b.y << 16);
            acc[i][j][4 * q + 3] = __uint_as_float(b.y & 0xffff0000u);
          }
        }
    }
    if constexpr (!EXACT) copy_bias(nxt, bpar ^ 1);
    // a half stage's products in 16 steps. The 8-bit instruction takes a tile's 64 k at
    // once; decoded, a step is 16 k of four tiles (row i), while the next 16 k of two
    // fragments are decoded, at the end those of the stage's other half.
    bf16x8 dec[2][8];
    float sc[8];
    auto decode = [&](const Set& s, int k, int f) {
      dec[k & 1][f] = fp8_bf16x8(s.f[f][2 * (k & 3)], s.f[f][2 * (k & 3) + 1], sc[f]);
    };
    auto product = [&](const Set& s, const Set* after, int m) {
      if constexpr (EXACT) {
        const int k = m >> 2, i = m & 3;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dec[k & 1][4 + j], dec[k & 1][i], acc[i][j], 0, 0, 0);
        if (k < 3 || after) {
          decode(k < 3 ? s : *after, k + 1, 2 * i);
          decode(k < 3 ? s : *after, k + 1, 2 * i + 1);
        }
      } else {
        const int i = m / 4, j = m % 4;
        // B's rows first: a lane then holds four consecutive columns of a row of C
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(s.f[4 + j], s.f[i], acc[i][j], 0, 0, 0, eb[j], 0, ea[i]);
      }
    };
    int t = 0;
#pragma unroll 1
    do {
      const char* here = smem + ((par + t) & 1) * kWideStage;
      const char* then = smem + ((par + t + 1) & 1) * kWideStage;
      if ((t & 3) == 0) {
        scales(epar ^ ((t >> 2) & 1));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ea[i] = (int)((unsigned)ea[i] >> 8);
          eb[i] = (int)((unsigned)eb[i] >> 8);
        }
      }
      const Src s = source(t + 2);
      if constexpr (EXACT) {
#pragma unroll
        for (int f = 0; f < 8; ++f) {
          sc[f] = fp8_scale(f < 4 ? ea[f] : eb[f - 4]);
          decode(X, 0, f);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 16; ++m) {
        if (m == 10) {
          // the whole stage is in registers
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          meet();
        }
        product(X, &Y, m);
        if (m < 8) {
          read(Y, here, 1, m, 0);
          read(Y, here, 1, m, 1);
        }
        if (m >= 10 && m != 12 && m != 15) copy(s, m < 12 ? m - 10 : m - 11);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the next stage has landed (four copies of the one after it may be in flight)
      wait_vmcnt<4>();
      meet();
      copy_e(t + 2);
#pragma unroll
      for (int m = 0; m < 16; ++m) {
        product(Y, nullptr, m);
        if (m < 8) {
          read(X, then, 0, m, 0);
          read(X, then, 0, m, 1);
        }
        if ((m & 3) != 3) copy(s, 4 + m - (m >> 2));
        __builtin_amdgcn_sched_barrier(0);
      }
    } while (++t < nk);
    // Results, 32 rows x 128 columns at a time: lane l holds row l & 31 of a product's
    // tile and of its columns 8 q + 4 (l >> 5) .. +3, q = 0 .. 3. Halves of the wave swap
    // such fours, so that a lane has 8 consecutive columns; rounded to bf16 they pass
    // through the wave's LDS, 16 rows at a time, and leave as runs of 256 bytes (runs of
    // 128 take the memory half as long again).
    //
    // Stores that nothing reads soon pass the caches, which keep the operands of tiles still
    // to come: 4096 x 4096 x 8192 113 -> 104 us, 8192 x 8192 x 1024 78 -> 75, float32 results
    // 8192 x 4096 x 4096 209 -> 202. The next kernel of a block reads what GELU' and the residual
    // leave and GELU's value (a 115M block's backward: 900 us, and 917 with all past the caches).
    constexpr int kStream = 2;
    char* out = smem + kWideOut + wave * 16 * kWidePitch;
    const int mw = cur.m0 + wm * 128, nc = cur.n0 + wn * 128;
    // rows mw + 32 i .. of a matrix from column nc: offsets behind the last row are out of
    // bounds, which reads zeros and stores nothing
    constexpr int ES = EXACT ? 4 : 2;
    auto matrix = [&](const void* D, int64_t ld, int i) {
      const int mr = mw + i * 32;
      const uint64_t p = (uint64_t)(uintptr_t)(static_cast<const char*>(D) + ((int64_t)mr * ld + nc) * ES);
      // (uniform, as the compiler does not see)
      const unsigned lo = __builtin_amdgcn_readfirstlane((int)p), hi = __builtin_amdgcn_readfirstlane((int)(p >> 32));
      return buffer_rsrc(reinterpret_cast<const void*>((uint64_t)hi << 32 | lo),
                         __builtin_amdgcn_readfirstlane(max(min(g.M - mr, 32), 0) * (int)ld * ES));
    };
    auto leave = [&](void* D, int64_t ld, int i, const U128* q, auto aux) {
      const __amdgpu_buffer_rsrc_t to = matrix(D, ld, i);
      const unsigned at = nc + (lane & 15) * 8 < g.N ? (unsigned)((lane >> 4) * (int)ld * 2 + (lane & 15) * 16) : kOobOffset;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if ((lr >> 4) == h) {
#pragma unroll
          for (int k = 0; k < 8; ++k) st128(out + (lr & 15) * kWidePitch + (k * 16 + (lane >> 5) * 8) * 2, q[k]);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(out + (it * 4 + (lane >> 4)) * kWidePitch + (lane & 15) * 16);
          __builtin_amdgcn_raw_buffer_store_b128(v, to, at + (unsigned)((h * 16 + it * 4) * 2 * (int)ld), 0,
                                                 decltype(aux)::value);
        }
        __builtin_amdgcn_wave_barrier();
      }
    };
    // the rows of the epilogue's operands, read before the rows before them leave: their
    // wait is none for those stores
    u32x4 ops[8];
    auto fetch = [&](auto at) {
      constexpr int i = decltype(at)::value;
      if constexpr (EPI == kWideGeluGrad || EPI == kWideRes) {
        const int64_t ld = EPI == kWideRes ? g.epi.ldr : g.epi.ldgi;
        const __amdgpu_buffer_rsrc_t r = matrix(EPI == kWideRes ? g.epi.res : g.epi.gelu_in, ld, i);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = k * 16 + (lane >> 5) * 8;
          ops[k] = __builtin_amdgcn_raw_buffer_load_b128(r, nc + c < g.N ? (unsigned)(lr * (int)ld * 2 + c * 2) : kOobOffset, 0, 0);
        }
      }
    };
    // (what float32 results are added to is read a row group ahead, past the caches as well:
    // 8192 x 4096 x 4096 279 us when read at each store, 240 ahead, 231 past the caches, and
    // 203 without adding; 134 MB take 26)
    // float32 results: a lane's fours as they are, 8 rows at a time, in runs of 512 bytes;
    // store n of 16 in a row group takes rows 2 n + (l >> 5)
    const unsigned col = nc + (lane & 31) * 4 < g.N ? (unsigned)((lane >> 5) * (int)g.ldc * 4 + (lane & 31) * 16) : kOobOffset;
    auto off = [&](int n) { return col + (unsigned)(n * 8 * (int)g.ldc); };
    u32x4 old[EPI == kWideF32Add ? 2 : 1][16];  // what the sums are added to, read before the rows before leave
    auto fetch_old = [&](auto at) {
      constexpr int i = decltype(at)::value;
      const __amdgpu_buffer_rsrc_t r = matrix(g.C, g.ldc, i);
#pragma unroll
      for (int n = 0; n < 16; ++n) old[i & 1][n] = __builtin_amdgcn_raw_buffer_load_b128(r, off(n), 0, kStream);
    };
    auto leave_f32 = [&](auto at) {
      constexpr int i = decltype(at)::value;
      constexpr int pitch = 528;
      static_assert(4 * 8 * pitch <= kWideLds - kWideOut, "LDS");
      const __amdgpu_buffer_rsrc_t to = matrix(g.C, g.ldc, i);
      char* o = smem + kWideOut + wave * 8 * pitch;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        if ((lr >> 3) == h) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<f32x4*>(o + (lr & 7) * pitch + (j * 32 + q * 8 + (lane >> 5) * 4) * 4) =
                  f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int n = h * 4 + it;
          f32x4 v = *reinterpret_cast<const f32x4*>(o + (it * 2 + (lane >> 5)) * pitch + (lane & 31) * 16);
          if constexpr (EPI == kWideF32Add) v += __builtin_bit_cast(f32x4, old[i & 1][n]);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), to, off(n), 0, kStream);
        }
        __builtin_amdgcn_wave_barrier();
      }
    };
    auto rows = [&](auto at) {
      constexpr int i = decltype(at)::value;
      // (from here on, not before: moved up, these rows' sums would not fit the registers)
#pragma unroll
      for (int j = 0; j < 4; ++j) asm volatile("" : "+a"(acc[i][j]));
      if constexpr (EXACT) {
        if constexpr (EPI == kWideF32Add && i < 3) fetch_old(std::integral_constant<int, i + 1>{});
        __builtin_amdgcn_sched_barrier(0);
        leave_f32(at);
        __builtin_amdgcn_sched_barrier(0);
        return;
      }
      U128 q[8];
      // the sums as they are, rounded before the halves swap: half the swaps
      auto sums = [&] {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const f32x16& c = acc[i][k >> 1];
          const int p = 8 * (k & 1);
          const auto w0 = __builtin_amdgcn_permlane32_swap(pack2(c[p], c[p + 1]), pack2(c[p + 4], c[p + 5]), false, false);
          const auto w1 = __builtin_amdgcn_permlane32_swap(pack2(c[p + 2], c[p + 3]), pack2(c[p + 6], c[p + 7]), false, false);
          q[k] = U128{{w0[0], w1[0], w0[1], w1[1]}};
        }
      };
      if constexpr (EPI == kWidePlain) {
        sums();
      } else {
        if constexpr (EPI == kWideGelu) {
          sums();
          leave(g.epi.gelu_out, g.epi.ldgo, i, q, std::integral_constant<int, kStream>{});
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          __builtin_amdgcn_sched_barrier(0);
          float v[8], t8[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int p = 8 * (k & 1) + e;
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][k >> 1][p]),
                                                            __float_as_uint(acc[i][k >> 1][p + 4]), false, false);
            v[e] = __uint_as_float(w[0]);
            v[4 + e] = __uint_as_float(w[1]);
          }
          if constexpr (EPI != kWideGelu) unpack(__builtin_bit_cast(U128, ops[k]), t8, (bf16*)nullptr);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = EPI == kWideGelu ? gelu_f(v[e]) : EPI == kWideRes ? v[e] + t8[e] : v[e] * gelu_grad_f(t8[e]);
          q[k] = pack8(v);
        }
        if constexpr (i < 3) fetch(std::integral_constant<int, i + 1>{});
        __builtin_amdgcn_sched_barrier(0);
      }
      leave(g.C, g.ldc, i, q, std::integral_constant<int, EPI == kWidePlain ? kStream : 0>{});
      __builtin_amdgcn_sched_barrier(0);
    };
    fetch(std::integral_constant<int, 0>{});
    if constexpr (EPI == kWideF32Add) fetch_old(std::integral_constant<int, 0>{});
    rows(std::integral_constant<int, 0>{});
    rows(std::integral_constant<int, 1>{});
    rows(std::integral_constant<int, 2>{});
    rows(std::integral_constant<int, 3>{});
    // the next tile
    par ^= nk & 1;
    epar ^= ((nk + 3) >> 2) & 1;
    bpar ^= 1;
    cur = nxt;
    nxt = tile_at(lin + 2 * gridDim.x);
  }
  wait_vmcnt<0>();
}

// Up to 16 MT rows of A. A block of 8 waves takes 16 columns (rows of B); its waves
// take the K blocks in turn, 128 k to an instruction, and add their sums through
// LDS. Lane l holds row l & 15 and k 32 (l >> 4) .. +31 of either operand, and of
// the result column n0 + 4 (l >> 4) + v of row l & 15 of each tile of 16.
constexpr int kThinWaves = 8;
template <typename T, typename OutT, int MT>
__global__ void __launch_bounds__(kThinWaves * 64) fp8_thin_kernel(Fp8Args g) {
  __shared__ f32x4 sum[kThinWaves][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16, lr = lane & 15, kc = (lane >> 4) * 32;
  const int split = blockIdx.z;
  const int b0 = fp8_split_at(g, split), b1 = fp8_split_at(g, split + 1);  // K blocks
  // rows past the operands read row 0 again: their results are not stored
  const int64_t br = n0 + lr < g.N ? n0 + lr : 0;
  const uint8_t *pb = g.B + br * g.ldb + kc, *pbe = g.Be + br * g.gpb;
  const uint8_t *pa[MT], *pae[MT];
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t ar = t * 16 + lr < g.M ? t * 16 + lr : 0;
    pa[t] = g.A + ar * g.lda + kc;
    pae[t] = g.Ae + ar * g.gpa;
    acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto ld32 = [](const uint8_t* p) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(p), b = *reinterpret_cast<const i32x4*>(p + 16);
    return i32x8(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // n blocks, all their loads in flight
  auto blocks = [&](int kb, auto n) {
    constexpr int NU = decltype(n)::value;
    i32x8 fb[NU], fa[NU][MT];
    int eb[NU], ea[NU][MT];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int k = kb + u * kThinWaves;
      fb[u] = ld32(pb + (int64_t)k * 128);
      eb[u] = pbe[k];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        fa[u][t] = ld32(pa[t] + (int64_t)k * 128);
        ea[u][t] = pae[t][k];
      }
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if constexpr (sizeof(OutT) == 2) {
          acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u], fa[u][t], acc[t], 0, 0, 0, eb[u], 0, ea[u][t]);
        } else {
          const float sb = fp8_scale(eb[u]), sa = fp8_scale(ea[u][t]);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_bf16x8(fb[u][2 * k], fb[u][2 * k + 1], sb),
                                                             fp8_bf16x8(fa[u][t][2 * k], fa[u][t][2 * k + 1], sa), acc[t], 0, 0, 0);
        }
      }
    }
  };
  constexpr int U = 4;  // all of a wave's up to K = 4096 (2 and their next ones: 7.7 us against 6.0 at 1 x 4096 x 4096)
  int kb = b0 + wave;
  for (; kb + (U - 1) * kThinWaves < b1; kb += U * kThinWaves) blocks(kb, std::integral_constant<int, U>{});
  for (; kb < b1; kb += kThinWaves) blocks(kb, std::integral_constant<int, 1>{});
#pragma unroll
  for (int t = 0; t < MT; ++t) sum[wave][t][lane] = acc[t];
  __syncthreads();
  // a thread per value of row i / 16, column i & 15: the waves' sums in wave order
  const float* fs = reinterpret_cast<const float*>(&sum[0][0][0]);
  for (int i = threadIdx.x; i < MT * 256; i += kThinWaves * 64) {
    const int r = i >> 4, c = i & 15;
    const int at = ((r >> 4) * 64 + (c >> 2) * 16 + (r & 15)) * 4 + (c & 3);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kThinWaves; ++w) v += fs[w * MT * 256 + at];
    if (r < g.M && n0 + c < g.N) {
      if (g.splits > 1) g.partial[((int64_t)split * g.M + r) * g.N + n0 + c] = v;
      else epi_apply<T, OutT>(g.epi, 0, r, n0 + c, v, static_cast<OutT*>(g.C), g.ldc);
    }
  }
}

enum Fp8Tile { kThin, kTile, kWide };
struct Fp8Choice { Fp8Tile tile; int splits; };

// What the wide kernel's end has: of GELU with its input kept, GELU' and the residual one,
// with bf16 results, or onto what is there with float32 ones; 32 rows within 31-bit offsets.
// The other kernels end in epi_apply, which has everything: a float32 block's layers that
// need it stay on tiles of 128 x 128 (8192 x 8192 x 1024 168 us there, 142 on the wide ones).
bool wide_has(const Fp8Gemm& f, bool out_f32) {
  const Epi& e = f.epi;
  const int fused = (e.gelu_out ? 1 : 0) + (e.gelu_in ? 1 : 0) + (e.res ? 1 : 0);
  const auto near = [](const void* p, int64_t ld) { return !p || ld < (1 << 24); };
  return (out_f32 ? fused == 0 : fused <= 1 && !e.accumulate) && e.res_row_mod == 0 && near(f.C, f.ldc) &&
         near(e.gelu_out, e.ldgo) && near(e.gelu_in, e.ldgi) && near(e.res, e.ldr);
}

Fp8Choice pick_fp8(int M, int N, int K, bool out_f32) {
  const int64_t slices = fp8_wide(K) / 64;
  // Thin, by the block's columns and what a wave has to read of A: 1 x 4096 x 1024 2.7 us against
  // 5.1 on tiles, 16 x 4096 x 1024 3.2 against 5.1, 16 x 8192 x 1024 4.7 against 5.6, 32 x 4096 x
  // 1024 3.9 against 5.3; but 8 x 16384 x 4096 21.5 against 17.7, 32 x 8192 x 1024 6.0 against 5.8,
  // 32 x 4096 x 4096 10.6 against 9.5.
  if (M <= 16 ? N <= 8192 : M <= 32 && N <= 4096 && slices <= 32) {
    // in parts of 16 blocks (K = 2048) from K = 8192 on, up to a block per CU (1 x 1024 x 8192
    // 7.1 us against 9.1 in one part, 1 x 1024 x 4096 5.7 against 5.3)
    int sp = 1;
    while (slices >= 128 && sp < 16 && cdiv(N, 16) * sp < 256 && slices / (2 * sp) >= 32) sp *= 2;
    return {kThin, sp};
  }
  // Wide, with two stages at least, where tiles of 128 x 128, two to a CU, would take a second
  // round (in us, against those: 4608 x 2048 x 4096 44.9 and 58.0, float32 results 87.2 and 89.5;
  // 5632 x 2048 x 1024 19.0 and 23.4, float32 34.5 and 34.4), but not
  // where they fit one (8192 x 1024 x 4096 47.3 and 40.2, 2048 x 3584 x 4096 45.2 and 36.4).
  if (cdiv(M, 128) * cdiv(N, 128) > 512 && slices >= 4) return {kWide, 1};
  // Split K saves slices, of 0.135 us each (float32 results: 0.233), and costs the second
  // launch, 3.5 us, and writing and reading the partial sums, 0.7 us per MB of them: 100 x 512 x
  // 8192 10.9 us in 8 parts and 20.7 in one, 512 x 1024 x 4096 14.2 in 4 and 12.2 in one. Only
  // where it leaves one block of 64 x 64 per CU.
  const int64_t t64 = cdiv(M, 64) * cdiv(N, 64);
  const double slice = out_f32 ? 0.233 : 0.135, part = 0.7e-6 * 4 * (double)M * N;
  Fp8Choice c{kTile, 1};
  double best = slice * (double)slices;
  for (int sp = 2; sp <= 8 && t64 * sp <= 256 && 2 * sp <= slices; sp *= 2) {
    const double t = slice * (double)slices / sp + 3.5 + part * sp;
    if (t < best) { best = t; c.splits = sp; }
  }
  return c;
}

template <typename T, typename OutT, int BM, int BN, int NS, int KG>
orbit_status run_tile(const Fp8Gemm& f, const Fp8Args& a, hipStream_t s) {
  KernelInfo ki{sizeof(OutT) == 2 ? "gemm_fp8_tile<bf16>" : "gemm_fp8_tile<f32>", 2.0 * f.M * f.N * (double)f.K,
                ((double)f.M + f.N) * f.K * (1.0 + 1.0 / kFp8Block) + (double)f.M * f.N * sizeof(OutT)};
  constexpr int lds = TileCfg<BM, BN, NS, KG>::LDS;
  static const bool attr = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_fp8_tile_kernel<T, OutT, BM, BN, NS, KG>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    (void)hipGetLastError();
    return true;
  }();
  (void)attr;
  const dim3 grid((unsigned)(cdiv(a.M, BM) * cdiv(a.N, BN)), 1, (unsigned)a.splits);
  return launch(ki, gemm_fp8_tile_kernel<T, OutT, BM, BN, NS, KG>, grid, dim3(KG * 256), (size_t)lds, s, a);
}

template <typename T, WideEpi EPI>
orbit_status run_wide(const Fp8Gemm& f, const Fp8Args& a, hipStream_t s) {
  KernelInfo ki{EPI >= kWideF32 ? "gemm_fp8_wide<f32>" : "gemm_fp8_wide<bf16>", 2.0 * f.M * f.N * (double)f.K,
                ((double)f.M + f.N) * f.K * (1.0 + 1.0 / kFp8Block) + (EPI == kWideF32Add ? 8.0 : EPI == kWideF32 ? 4.0 : 2.0) * f.M * f.N};
  static const bool attr = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_fp8_wide_kernel<T, EPI>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, kWideLds);
    (void)hipGetLastError();
    return true;
  }();
  (void)attr;
  const dim3 grid((unsigned)std::min<int64_t>(cdiv(a.M, 256) * cdiv(a.N, 256), 256));
  return launch(ki, gemm_fp8_wide_kernel<T, EPI>, grid, dim3(256), (size_t)kWideLds, s, a);
}

template <typename T, typename OutT>
orbit_status run_thin(const Fp8Gemm& f, const Fp8Args& a, hipStream_t s) {
  KernelInfo ki{sizeof(OutT) == 2 ? "fp8_thin<bf16>" : "fp8_thin<f32>", 2.0 * f.M * f.N * (double)f.K,
                ((double)f.M + f.N) * f.K * (1.0 + 1.0 / kFp8Block) + (double)f.M * f.N * sizeof(OutT)};
  const dim3 grid((unsigned)cdiv(a.N, 16), 1, (unsigned)a.splits), block(kThinWaves * 64);
  if (a.M <= 16) return launch(ki, fp8_thin_kernel<T, OutT, 1>, grid, block, 0, s, a);
  return launch(ki, fp8_thin_kernel<T, OutT, 2>, grid, block, 0, s, a);
}

template <typename T, typename OutT>
orbit_status run_typed8(const Fp8Gemm& f, const Fp8Args& a, Fp8Tile t, hipStream_t s) {
  switch (t) {
    case kThin: return run_thin<T, OutT>(f, a, s);
    case kTile: {
      auto tiles = [&](int bm, int bn) { return cdiv(a.M, bm) * cdiv(a.N, bn) * a.splits; };
      const bool two = a.slices / a.splits >= (sizeof(OutT) == 2 ? 32 : 8);  // groups of waves
      if (tiles(64, 64) <= 256) return two ? run_tile<T, OutT, 64, 64, 4, 2>(f, a, s) : run_tile<T, OutT, 64, 64, 4, 1>(f, a, s);
      if (tiles(64, 128) <= 256) return two ? run_tile<T, OutT, 64, 128, 3, 2>(f, a, s) : run_tile<T, OutT, 64, 128, 4, 1>(f, a, s);
      if constexpr (sizeof(OutT) == 2)
        if (a.slices >= 16 && tiles(128, 128) <= 256) return run_tile<T, OutT, 128, 128, 2, 2>(f, a, s);
      return run_tile<T, OutT, 128, 128, 2, 1>(f, a, s);
    }
    default:
      if (!wide_has(f, sizeof(OutT) == 4)) {
        set_error("fp8 product: no large tiles with this epilogue");
        return ORBIT_E_UNSUPPORTED;
      }
      if constexpr (sizeof(OutT) == 2) {
        if (f.epi.gelu_out) return run_wide<bf16, kWideGelu>(f, a, s);
        if (f.epi.gelu_in) return run_wide<bf16, kWideGeluGrad>(f, a, s);
        return f.epi.res ? run_wide<bf16, kWideRes>(f, a, s) : run_wide<bf16, kWidePlain>(f, a, s);
      } else {
        return f.epi.accumulate ? run_wide<T, kWideF32Add>(f, a, s) : run_wide<T, kWideF32>(f, a, s);
      }
  }
}

}  // namespace

size_t fp8_gemm_workspace_bytes(int M, int N, int K) {
  const int sp = std::max(pick_fp8(M, N, K, false).splits, pick_fp8(M, N, K, true).splits);
  return sp > 1 ? align_up((size_t)sp * (size_t)M * (size_t)N * sizeof(float)) : 0;
}

orbit_status fp8_gemm(const Fp8Gemm& f, void* ws, size_t ws_bytes, hipStream_t s) {
  const bool out_f32 = f.out_f32 || f.dtype == ORBIT_F32;
  Fp8Choice c = pick_fp8(f.M, f.N, f.K, out_f32);
  if (c.tile == kWide && !wide_has(f, out_f32)) c.tile = kTile;
  Fp8Args a{};
  a.A = static_cast<const uint8_t*>(f.A); a.Ae = a.A + fp8_exp_offset(f.M, f.K);
  a.B = static_cast<const uint8_t*>(f.B); a.Be = a.B + fp8_exp_offset(f.N, f.K);
  a.lda = a.ldb = fp8_wide(f.K);
  a.gpa = a.gpb = (int)fp8_groups(f.K);
  a.C = f.C; a.ldc = f.ldc;
  a.M = f.M; a.N = f.N; a.slices = (int)(a.lda / 64);
  a.epi = f.epi;
  a.epi.alpha = 1.f;
  a.splits = c.splits;
  if (c.splits > 1) {
    if (ws_bytes < fp8_gemm_workspace_bytes(f.M, f.N, f.K)) {
      set_error("fp8 product: workspace of %zu bytes is smaller than the %zu required", ws_bytes,
                fp8_gemm_workspace_bytes(f.M, f.N, f.K));
      return ORBIT_E_ARG;
    }
    a.partial = static_cast<float*>(ws);
  }
  if (f.dtype == ORBIT_F32) ORBIT_TRY((run_typed8<float, float>(f, a, c.tile, s)));
  else if (f.out_f32) ORBIT_TRY((run_typed8<bf16, float>(f, a, c.tile, s)));
  else ORBIT_TRY((run_typed8<bf16, bf16>(f, a, c.tile, s)));
  if (a.splits <= 1) return ORBIT_OK;
  GemmKArgs k{};
  k.C = f.C; k.ldc = f.ldc; k.M = f.M; k.N = f.N; k.batch = 1; k.splits = a.splits; k.vec_ok = 1;
  k.partial = a.partial; k.epi = a.epi;
  return splitk_finish(f.dtype, f.out_f32, k, s);
}

}  // namespace orbit
