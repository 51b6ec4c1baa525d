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
// bf16 results take it. Float32 results are formed with EXACT instead: the codes are
// turned into bf16 with their scales in the fragments, which is exact, and the bf16
// instructions keep every bit a float32 sum can, at half the rate.
//
// A row of a K slice is 64 bytes here as in the bf16 kernels, and an instruction
// of 64 k takes as long as two of theirs of 16: tiles, LDS ring, copies and swizzle
// are theirs (dma.h), with twice the operations per byte of LDS traffic. The E words
// of 512 k (8 slices) come by the same copies into two LDS slots of their own and
// are shifted by one block every two slices.
//
// Up to 64 rows of A (single tokens) the product is bound by reading B once:
// fp8_thin_kernel streams it past 16x16x128 instructions without LDS.
#include <algorithm>

#include "dma.h"
#include "fp8.h"
#include "gemm.h"

namespace orbit {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Fp8Args {
  const uint8_t *A, *B, *Ae, *Be;  // codes and E bytes
  int64_t lda, ldb;                // bytes of a row of codes
  int gpa, gpb;                    // and of E
  void* C;
  int64_t ldc;
  int M, N, slices;                // 64-deep slices of K
  int splits, per_split;           // slices of a split (a multiple of 8)
  float* partial;                  // splits > 1: [splits][M][N]
  Epi epi;
};

// one wave copies 64 words from rsrc + voff (per lane) to LDS byte address lds + 4 * lane
ORBIT_DEV void dma4(__amdgpu_buffer_rsrc_t r, unsigned lds, unsigned voff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(r)
               : "memory", "m0");
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

// Fragments of a slice: row row0 + 32 i + (lane & 31), chunks h and h + 2 of 16 k,
// h = lane / 32. Both operands take the same chunks, so the order of the k within
// an instruction does not matter; all of a slice's k share a block.
template <int NF>
struct Fp8Frag {
  unsigned off, x[2];
  ORBIT_DEV void init(int row0, int lane) {
    const int f = (lane >> 2) & 3, h = lane >> 5;
    x[0] = (unsigned)((h ^ f) << 4);
    x[1] = (unsigned)(((h + 2) ^ f) << 4);
    off = (unsigned)((row0 + (lane & 31)) * 64);
  }
  ORBIT_DEV void read(i32x8* f, const char* S) const {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const i32x4 a = *reinterpret_cast<const i32x4*>(S + off + i * 2048 + x[0]);
      const i32x4 b = *reinterpret_cast<const i32x4*>(S + off + i * 2048 + x[1]);
      f[i] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

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

template <typename CF> constexpr int fp8_ring() { return CF::NS * CF::STB; }
template <typename CF> constexpr int fp8_lds() {
  return std::max(fp8_ring<CF>() + 2 * (CF::BM + CF::BN) * 4, CF::EPB);
}

template <typename T, typename OutT, typename CF>
__global__ void __launch_bounds__(CF::NT, CF::OCC) gemm_fp8_kernel(Fp8Args g) {
  constexpr int BM = CF::BM, BN = CF::BN, WM = CF::WM, NS = CF::NS;
  constexpr int TM = CF::TM, TN = CF::TN, OPA = CF::OPA, STB = CF::STB;
  using PA = DmaPlan<true, BM, CF::NW>;
  using PB = DmaPlan<true, BN, CF::NW>;
  constexpr int NLS = PA::NL + PB::NL;  // copies of codes per stage per wave
  constexpr int EW = BM + BN;           // E words of 8 slices
  constexpr bool EXACT = sizeof(OutT) == 4;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  int split = blockIdx.z;

  // tile order as in gemm_dma_kernel: XCD-contiguous ranges of tile ids, walked in
  // groups of tile rows; with split K an XCD takes one K range
  const int tiles_n = (g.N + BN - 1) / BN, tiles_m = (g.M + BM - 1) / BM;
  const int nt = tiles_m * tiles_n;
  int id = blockIdx.x;
  const int full = nt - nt % 8;
  if (g.splits > 1 && 8 % g.splits == 0 && (nt * g.splits) % 8 == 0) {
    const int lin = blockIdx.x + nt * (int)blockIdx.z, xcd = lin % 8;
    split = xcd % g.splits;
    id = (xcd / g.splits) * (nt * g.splits / 8) + lin / 8;
  } else if (id < full) {
    id = (id % 8) * (full / 8) + id / 8;
  }
  constexpr int GR = BN == 128 ? 4 : 8;
  const int per_group = GR * tiles_n;
  const int first_m = (id / per_group) * GR;
  const int gsize = min(tiles_m - first_m, GR);
  const int m0 = (first_m + (id % per_group) % gsize) * BM, n0 = ((id % per_group) / gsize) * BN;
  const int sbeg = split * g.per_split;
  const int nk = min(g.slices - sbeg, g.per_split);  // even: K is padded to whole blocks

  const uint8_t* Ab = g.A + (int64_t)m0 * g.lda + (int64_t)sbeg * 64;
  const uint8_t* Bb = g.B + (int64_t)n0 * g.ldb + (int64_t)sbeg * 64;
  const uint8_t* Aeb = g.Ae + (int64_t)m0 * g.gpa + (sbeg >> 1);
  const uint8_t* Beb = g.Be + (int64_t)n0 * g.gpb + (sbeg >> 1);

  PA pa;
  PB pb;
  pa.init(g.lda >> 1, m0, g.M, wave, lane);
  pb.init(g.ldb >> 1, n0, g.N, wave, lane);
  Fp8Frag<TM> ra;
  Fp8Frag<TN> rb;
  ra.init(wm * TM * 32, lane);
  rb.init(wn * TN * 32, lane);

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  const unsigned lds0 = (unsigned)(uintptr_t)(ORBIT_LDS void*)smem;
  auto issue = [&](int st) {
    if ((st & 7) == 0) {
      // E words first: they have landed when the slice's codes have
      for (int w = wave; w < EW / 64; w += CF::NW) {
        const bool isa = w < BM / 64;
        const int r = (isa ? w : w - BM / 64) * 64 + lane;
        const unsigned vo = isa ? (m0 + r < g.M ? (unsigned)(r * g.gpa) : kOobOffset)
                                : (n0 + r < g.N ? (unsigned)(r * g.gpb) : kOobOffset);
        dma4(buffer_rsrc((isa ? Aeb : Beb) + (st >> 1)), lds0 + NS * STB + ((st >> 3) & 1) * (EW * 4) + w * 256, vo);
      }
    }
    const unsigned b = lds0 + (st % NS) * STB;
    pa.template issue<false>(reinterpret_cast<const bf16*>(Ab + st * 64), 0, DBK, b, wave, lane);
    pb.template issue<false>(reinterpret_cast<const bf16*>(Bb + st * 64), 0, DBK, b + OPA, wave, lane);
  };
  int ea[TM], eb[TN];
  auto scales = [&](int st) {
    if ((st & 7) == 0) {
      const int* E = reinterpret_cast<const int*>(smem + NS * STB + ((st >> 3) & 1) * (EW * 4));
#pragma unroll
      for (int i = 0; i < TM; ++i) ea[i] = E[wm * TM * 32 + i * 32 + (lane & 31)];
#pragma unroll
      for (int j = 0; j < TN; ++j) eb[j] = E[BM + wn * TN * 32 + j * 32 + (lane & 31)];
    } else if ((st & 1) == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) ea[i] = (int)((unsigned)ea[i] >> 8);
#pragma unroll
      for (int j = 0; j < TN; ++j) eb[j] = (int)((unsigned)eb[j] >> 8);
    }
  };
  // prologue: stages 0 .. NS-2 in flight, then wait for stage 0
#pragma unroll
  for (int st = 0; st < NS - 1; ++st)
    if (st < nk) issue(st);
  wait_stage<NLS, NS>(min(nk - 1, NS - 2));
  __syncthreads();

  i32x8 fa[TM], fb[TN];
  if constexpr (CF::PP) {
    // two wave groups half a slice apart (see gemm_dma_kernel)
    const int grp = wave >> 2;
    if (grp) __builtin_amdgcn_s_barrier();
    for (int kt = 0; kt < nk; ++kt) {
      const char* cur = smem + (kt % NS) * STB;
      ra.read(fa, cur);
      rb.read(fb, cur + OPA);
      scales(kt);
      if (kt + NS - 1 < nk) issue(kt + NS - 1);
      wait_stage<NLS, NS>(min(nk - kt - 2, NS - 2));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      mma_slice<TM, TN, EXACT>(acc, fa, fb, ea, eb);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!grp) __builtin_amdgcn_s_barrier();
  } else {
    // a slice's MFMAs run while the next slice's fragments are read
    i32x8 ga[TM], gb[TN];
    auto step = [&](int kt, const i32x8* ua, const i32x8* ub, i32x8* va, i32x8* vb) {
      if (kt + NS - 1 < nk) issue(kt + NS - 1);
      scales(kt);
      wait_stage<NLS, NS>(min(nk - kt - 2, NS - 2));
      __syncthreads();
      // past the last slice this reads a stale but in-bounds slot
      const char* nxt = smem + ((kt + 1) % NS) * STB;
      ra.read(va, nxt);
      rb.read(vb, nxt + OPA);
      mma_slice<TM, TN, EXACT>(acc, ua, ub, ea, eb);
    };
    ra.read(fa, smem);
    rb.read(fb, smem + OPA);
    for (int kt = 0; kt < nk; kt += 2) {
      step(kt, fa, fb, ga, gb);
      step(kt + 1, ga, gb, fa, fb);
    }
  }
  wait_vmcnt<0>();
  __syncthreads();

  // epilogue through LDS: each wave parks 32 rows of its accumulators and reads
  // them back as 8 consecutive columns per lane
  constexpr int WTN = TN * 32, EP = WTN + 8, LPR = WTN / 8, RPI = 64 / LPR;
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
  const int b0 = split * (g.per_split >> 1), b1 = min(g.slices >> 1, b0 + (g.per_split >> 1));  // K blocks
  // rows past the operands read row 0 again: their results are not stored
  const bool bv = n0 + lr < g.N;
  const int64_t br = bv ? n0 + lr : 0;
  const uint8_t* pb = g.B + br * g.ldb + kc;
  const uint8_t* pbe = g.Be + br * g.gpb;
  const uint8_t *pa[MT], *pae[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t ar = t * 16 + lr < g.M ? t * 16 + lr : 0;
    pa[t] = g.A + ar * g.lda + kc;
    pae[t] = g.Ae + ar * g.gpa;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto ld32 = [](const uint8_t* p) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(p), b = *reinterpret_cast<const i32x4*>(p + 16);
    return i32x8(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // U blocks at a time, the next ones' loads in flight
  constexpr int U = MT > 2 ? 1 : 2;
  i32x8 fb[U], fa[U][MT];
  int eb[U], ea[U][MT];
  auto fetch = [&](int kb, i32x8* vb, i32x8 (*va)[MT], int* web, int (*wea)[MT]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // past the range the last block again: not used
      const int k = min(kb + u * kThinWaves, b1 - 1);
      vb[u] = ld32(pb + (int64_t)k * 128);
      web[u] = pbe[k];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        va[u][t] = ld32(pa[t] + (int64_t)k * 128);
        wea[u][t] = pae[t][k];
      }
    }
  };
  if (b0 + wave < b1) fetch(b0 + wave, fb, fa, eb, ea);
  for (int kb = b0 + wave; kb < b1; kb += U * kThinWaves) {
    i32x8 nb[U], na[U][MT];
    int neb[U], nea[U][MT];
    fetch(kb + U * kThinWaves, nb, na, neb, nea);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u * kThinWaves >= b1) break;
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
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fb[u] = nb[u];
      eb[u] = neb[u];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        fa[u][t] = na[u][t];
        ea[u][t] = nea[u][t];
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) sum[wave][t][lane] = acc[t];
  __syncthreads();
  // a thread per value: row t * 16 + (l & 15), column 4 (l >> 4) + v, the waves'
  // sums in wave order
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

enum Fp8Tile { kThin, kQuarter, kHalf, kFull };
struct Fp8Choice { Fp8Tile tile; int splits; };

Fp8Choice pick_fp8(int M, int N, int K) {
  const int64_t slices = fp8_wide(K) / 64;
  if (M <= 64) {
    // a block per CU at least
    int sp = 1;
    while (sp < 16 && cdiv(N, 16) * sp < 256 && slices / (2 * sp) >= 32) sp *= 2;
    return {kThin, sp};
  }
  const int64_t t256 = cdiv(M, 256) * cdiv(N, 256), t128 = cdiv(M, 128) * cdiv(N, 128);
  if (t256 >= 192) return {kFull, 1};
  int sp = 1;
  while (sp < 8 && t128 * sp < 256 && slices / (2 * sp) >= 16) sp *= 2;
  return {kQuarter, sp};
}

// slices of a split, whole E words
int per_split_of(int64_t slices, int splits) { return (int)cdiv(cdiv(slices, splits), 8) * 8; }

template <typename T, typename OutT, typename CF>
orbit_status run_fp8(const Fp8Gemm& f, const Fp8Args& a, hipStream_t s) {
  const char* name = CF::BM == 128 ? (sizeof(OutT) == 2 ? "gemm_fp8<128x128,bf16>" : "gemm_fp8<128x128,f32>")
                     : CF::BN == 128 ? (sizeof(OutT) == 2 ? "gemm_fp8<256x128,bf16>" : "gemm_fp8<256x128,f32>")
                                     : (sizeof(OutT) == 2 ? "gemm_fp8<256x256,bf16>" : "gemm_fp8<256x256,f32>");
  KernelInfo ki{name, 2.0 * f.M * f.N * (double)f.K,
                ((double)f.M + f.N) * f.K * (1.0 + 1.0 / kFp8Block) + (double)f.M * f.N * sizeof(OutT)};
  constexpr int lds = fp8_lds<CF>();
  static const bool attr = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_fp8_kernel<T, OutT, CF>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    (void)hipGetLastError();
    return true;
  }();
  (void)attr;
  const dim3 grid((unsigned)(cdiv(a.M, CF::BM) * cdiv(a.N, CF::BN)), 1, (unsigned)a.splits);
  return launch(ki, gemm_fp8_kernel<T, OutT, CF>, grid, dim3(CF::NT), (size_t)lds, s, a);
}

template <typename T, typename OutT>
orbit_status run_thin(const Fp8Gemm& f, const Fp8Args& a, hipStream_t s) {
  KernelInfo ki{sizeof(OutT) == 2 ? "fp8_thin<bf16>" : "fp8_thin<f32>", 2.0 * f.M * f.N * (double)f.K,
                ((double)f.M + f.N) * f.K * (1.0 + 1.0 / kFp8Block) + (double)f.M * f.N * sizeof(OutT)};
  const dim3 grid((unsigned)cdiv(a.N, 16), 1, (unsigned)a.splits), block(kThinWaves * 64);
  if (a.M <= 16) return launch(ki, fp8_thin_kernel<T, OutT, 1>, grid, block, 0, s, a);
  if (a.M <= 32) return launch(ki, fp8_thin_kernel<T, OutT, 2>, grid, block, 0, s, a);
  return launch(ki, fp8_thin_kernel<T, OutT, 4>, grid, block, 0, s, a);
}

template <typename T, typename OutT>
orbit_status run_typed8(const Fp8Gemm& f, const Fp8Args& a, Fp8Tile t, hipStream_t s) {
  switch (t) {
    case kThin: return run_thin<T, OutT>(f, a, s);
    case kQuarter: return run_fp8<T, OutT, DmaQuarter>(f, a, s);
    case kHalf: return run_fp8<T, OutT, DmaHalf>(f, a, s);
    default: return run_fp8<T, OutT, DmaPP>(f, a, s);
  }
}

}  // namespace

size_t fp8_gemm_workspace_bytes(int M, int N, int K) {
  const Fp8Choice c = pick_fp8(M, N, K);
  return c.splits > 1 ? align_up((size_t)c.splits * (size_t)M * (size_t)N * sizeof(float)) : 0;
}

orbit_status fp8_gemm(const Fp8Gemm& f, void* ws, size_t ws_bytes, hipStream_t s) {
  Fp8Choice c = pick_fp8(f.M, f.N, f.K);
  Fp8Args a{};
  a.A = static_cast<const uint8_t*>(f.A); a.Ae = a.A + fp8_exp_offset(f.M, f.K);
  a.B = static_cast<const uint8_t*>(f.B); a.Be = a.B + fp8_exp_offset(f.N, f.K);
  a.lda = a.ldb = fp8_wide(f.K);
  a.gpa = a.gpb = (int)fp8_groups(f.K);
  a.C = f.C; a.ldc = f.ldc;
  a.M = f.M; a.N = f.N; a.slices = (int)(a.lda / 64);
  a.epi = f.epi;
  a.epi.alpha = 1.f;
  a.splits = 1;
  a.per_split = (int)align_up((size_t)a.slices, 8);
  if (c.splits > 1) {
    if (ws_bytes < fp8_gemm_workspace_bytes(f.M, f.N, f.K)) {
      set_error("fp8 product: workspace of %zu bytes is smaller than the %zu required", ws_bytes,
                fp8_gemm_workspace_bytes(f.M, f.N, f.K));
      return ORBIT_E_ARG;
    }
    a.per_split = per_split_of(a.slices, c.splits);
    a.splits = (int)cdiv(a.slices, a.per_split);
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
