// The 8-bit activation store (act8.h): packing a tensor, and reading it back
// with an optional GELU. HBM-bound: 8 columns per lane, a quad per group; a
// copy's rate (5.1 to 5.4 TB/s) is reached from about 50 MB on.
#include <algorithm>

#include "act8.h"
#include "rowbuf.h"

namespace orbit {
namespace {

// A matrix as the kernels walk it: `rows` rows of `n` columns; TX threads of a
// block along a row, each with U pieces of 8 columns TX pieces apart, and 256 /
// TX rows per block. A matrix without gaps whose rows are whole groups is walked
// as one long row.
struct Act8Shape {
  int64_t rows, n, groups;
  int tx_log2;
  dim3 grid;
};

// span: bytes from a row of the widest operand to the next
Act8Shape act8_shape(int64_t rows, int n, bool flat, int u, int64_t span) {
  Act8Shape z{};
  z.rows = flat ? 1 : rows;
  z.n = flat ? rows * n : n;
  z.groups = cdiv(z.n, kAct8Group);
  const int64_t pieces = cdiv(4 * z.groups, u);
  z.tx_log2 = 2;
  while (z.tx_log2 < 8 && (1ll << z.tx_log2) < pieces) ++z.tx_log2;
  // a block's rows share descriptors of 31-bit sizes: rows far apart go alone
  if (span >= (1ll << 31) >> (9 - z.tx_log2)) z.tx_log2 = 8;
  const int64_t tx = 1ll << z.tx_log2;
  z.grid = dim3((unsigned)cdiv(pieces, tx), (unsigned)std::min<int64_t>(cdiv(z.rows, 256 / tx), 65535));
  return z;
}

struct Act8Args {
  const void *x, *sub;  // sub (may be null; leading dimension ldx): x - sub is packed
  void *out, *gelu;
  const uint8_t *fc, *fe;
  uint8_t *qc, *qe;
  int64_t ldx, ldg, rows, n, groups;
  int tx_log2;
};

template <typename T, int U, int AUX>
__global__ void __launch_bounds__(256) act8_pack_kernel(Act8Args a) {
  const int tx = 1 << a.tx_log2, ty = 256 >> a.tx_log2;
  const int lx = (int)threadIdx.x & (tx - 1);
  const int64_t c0 = (int64_t)blockIdx.x * tx * U * 8;
  const int cols = (int)std::min<int64_t>(a.n - c0, tx * U * 8);
  const int64_t row0 = (int64_t)blockIdx.y * ty;
  // whole waves share a row where a row takes a wave or more; else the lanes'
  // row goes into their offsets
  const int lr = (int)threadIdx.x >> a.tx_log2;
  for (int64_t rb = row0; rb < a.rows; rb += (int64_t)gridDim.y * ty) {
    const int rows = (int)std::min<int64_t>(a.rows - rb, ty);
    const bool rv = lr < rows;
    const RowBuf bx(a.x, (rb * a.ldx + c0) * (int)sizeof(T), (int)(((rows - 1) * a.ldx + cols) * (int)sizeof(T)));
    const RowBuf bs(a.sub, (rb * a.ldx + c0) * (int)sizeof(T),
                    a.sub ? (int)(((rows - 1) * a.ldx + cols) * (int)sizeof(T)) : 0);
    const RowBuf bq(a.qc, rb * a.n + c0, (int)((rows - 1) * a.n + cols));
    const RowBuf be(a.qe, rb * a.groups + (c0 >> 5), (int)((rows - 1) * a.groups + ((cols + 31) >> 5)));
    Raw8<T> v[U], w[U];
    uint32_t col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      col[u] = (uint32_t)(u * tx + lx) * 8u;
      const bool on = rv && col[u] < (uint32_t)cols;
      const uint32_t at = on ? ((uint32_t)lr * (uint32_t)a.ldx + col[u]) * (uint32_t)sizeof(T) : kNoOffset;
      v[u].template load<AUX>(bx, at);
      if (a.sub) w[u].template load<AUX>(bs, at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = rv && col[u] < (uint32_t)cols;
      float f[8];
      v[u].get4(0, f);
      v[u].get4(1, f + 4);
      if (a.sub) {
        float g[8];
        w[u].get4(0, g);
        w[u].get4(1, g + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] -= g[i];
      }
      uint2 q;
      const uint32_t e = act8_encode(f, q);
      __builtin_amdgcn_raw_buffer_store_b64(u32v2{q.x, q.y}, bq.r, on ? (uint32_t)lr * (uint32_t)a.n + col[u] : kNoOffset, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b8(
          (uint8_t)e, be.r, on && (lx & 3) == 0 ? (uint32_t)lr * (uint32_t)a.groups + (col[u] >> 5) : kNoOffset, 0, 0);
    }
  }
}

template <typename T, int U, int AUX>
__global__ void __launch_bounds__(256) act8_unpack_kernel(Act8Args a) {
  const int tx = 1 << a.tx_log2, ty = 256 >> a.tx_log2;
  const int lx = (int)threadIdx.x & (tx - 1);
  const int64_t c0 = (int64_t)blockIdx.x * tx * U * 8;
  const int cols = (int)std::min<int64_t>(a.n - c0, tx * U * 8);
  const int64_t row0 = (int64_t)blockIdx.y * ty;
  const int lr = (int)threadIdx.x >> a.tx_log2;
  for (int64_t rb = row0; rb < a.rows; rb += (int64_t)gridDim.y * ty) {
    const int rows = (int)std::min<int64_t>(a.rows - rb, ty);
    const bool rv = lr < rows;
    const RowBuf bq(a.fc, rb * a.n + c0, (int)((rows - 1) * a.n + cols));
    const RowBuf be(a.fe, rb * a.groups + (c0 >> 5), (int)((rows - 1) * a.groups + ((cols + 31) >> 5)));
    const RowBuf bx(a.out, (rb * a.ldx + c0) * (int)sizeof(T),
                    a.out ? (int)(((rows - 1) * a.ldx + cols) * (int)sizeof(T)) : 0);
    const RowBuf bg(a.gelu, (rb * a.ldg + c0) * (int)sizeof(T),
                    a.gelu ? (int)(((rows - 1) * a.ldg + cols) * (int)sizeof(T)) : 0);
    u32v2 q[U];
    uint32_t e[U], col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      col[u] = (uint32_t)(u * tx + lx) * 8u;
      const bool on = rv && col[u] < (uint32_t)cols;
      q[u] = __builtin_amdgcn_raw_buffer_load_b64(bq.r, on ? (uint32_t)lr * (uint32_t)a.n + col[u] : kNoOffset, 0, AUX);
      e[u] = __builtin_amdgcn_raw_buffer_load_b8(be.r, on ? (uint32_t)lr * (uint32_t)a.groups + (col[u] >> 5) : kNoOffset, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = rv && col[u] < (uint32_t)cols;
      Raw8<T> o;
      float f[8];
      act8_decode4(q[u][0], e[u], f);
      act8_decode4(q[u][1], e[u], f + 4);
      if (a.out) {
        o.put4(0, f);
        o.put4(1, f + 4);
        o.store(bx, on ? ((uint32_t)lr * (uint32_t)a.ldx + col[u]) * (uint32_t)sizeof(T) : kNoOffset);
      }
      if (a.gelu) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = gelu_f(f[i]);
        o.put4(0, f);
        o.put4(1, f + 4);
        o.store(bg, on ? ((uint32_t)lr * (uint32_t)a.ldg + col[u]) * (uint32_t)sizeof(T) : kNoOffset);
      }
    }
  }
}

// Two pieces per thread keep enough loads in flight (bf16 8192 x 4096: pack 20.3
// -> 18.5 us, unpack 22.9 -> 19.5); float32 with the GELU's second output is
// better off with one where rows are whole groups (4096 x 4096: 32.5 us, two
// 39.1). From 96 MB on, more than the caches hold, bf16 loads are non-temporal
// (17.6 and 17.8 us; at 50 MB 9.1 -> 9.8; float32's two 16-byte loads a piece
// share their cache lines and lose by it, 84 MB: 13.4 -> 16.8).
template <typename T>
orbit_status act8_run(const KernelInfo& ki, Act8Args a, int64_t rows, int n, bool flat, bool pack, hipStream_t s) {
  const int u = sizeof(T) == 4 && a.gelu && flat ? 1 : 2;
  const bool stream = sizeof(T) == 2 && ki.bytes >= 96e6;
  const Act8Shape z = act8_shape(rows, n, flat, u, std::max(a.ldx, a.ldg) * (int64_t)sizeof(T));
  a.rows = z.rows; a.n = z.n; a.groups = z.groups; a.tx_log2 = z.tx_log2;
  const dim3 block(256);
  constexpr int NT = sizeof(T) == 2 ? 2 : 0;
  if (pack)
    return stream ? launch(ki, act8_pack_kernel<T, 2, NT>, z.grid, block, 0, s, a)
                  : launch(ki, act8_pack_kernel<T, 2, 0>, z.grid, block, 0, s, a);
  if (sizeof(T) == 4 && u == 1) return launch(ki, act8_unpack_kernel<T, sizeof(T) == 4 ? 1 : 2, 0>, z.grid, block, 0, s, a);
  return stream ? launch(ki, act8_unpack_kernel<T, 2, NT>, z.grid, block, 0, s, a)
                : launch(ki, act8_unpack_kernel<T, 2, 0>, z.grid, block, 0, s, a);
}

}  // namespace

orbit_status act8_pack(orbit_dtype dt, const void* x, const void* sub, int64_t ldx, int64_t rows, int n, void* store,
                       hipStream_t s) {
  Act8Args a{};
  a.x = x; a.sub = sub; a.ldx = ldx;
  a.qc = static_cast<uint8_t*>(store);
  a.qe = a.qc + act8_exp_offset(rows, n);
  const double e = dt == ORBIT_BF16 ? 2.0 : 4.0;
  KernelInfo ki{dt == ORBIT_BF16 ? "act8_pack<bf16>" : "act8_pack<f32>", 4.0 * rows * n,
                ((sub ? 2.0 : 1.0) * e + 1.0 + 1.0 / kAct8Group) * rows * n};
  const bool flat = n % kAct8Group == 0 && ldx == n;
  if (dt == ORBIT_BF16) return act8_run<bf16>(ki, a, rows, n, flat, true, s);
  return act8_run<float>(ki, a, rows, n, flat, true, s);
}

orbit_status act8_unpack(orbit_dtype dt, const void* store, int64_t rows, int n, void* x, int64_t ldx, void* gelu,
                         int64_t ldg, hipStream_t s) {
  Act8Args a{};
  a.out = x; a.ldx = x ? ldx : 0;
  a.gelu = gelu; a.ldg = gelu ? ldg : 0;
  a.fc = static_cast<const uint8_t*>(store);
  a.fe = a.fc + act8_exp_offset(rows, n);
  const double e = dt == ORBIT_BF16 ? 2.0 : 4.0;
  KernelInfo ki{dt == ORBIT_BF16 ? "act8_unpack<bf16>" : "act8_unpack<f32>", 4.0 * rows * n,
                (e * ((x ? 1 : 0) + (gelu ? 1 : 0)) + 1.0 + 1.0 / kAct8Group) * rows * n};
  const bool flat = n % kAct8Group == 0 && (!x || ldx == n) && (!gelu || ldg == n);
  if (dt == ORBIT_BF16) return act8_run<bf16>(ki, a, rows, n, flat, false, s);
  return act8_run<float>(ki, a, rows, n, flat, false, s);
}

}  // namespace orbit
