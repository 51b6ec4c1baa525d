// C ABI entry points of the 8-bit floating-point stores, their product and the
// linear layer on it, and of the rotary positions: argument validation, carving of
// the caller's buffers, kernel sequences.
#include <algorithm>

#include "abi_check.h"
#include "fp8.h"
#include "kernels.h"
#include "rope.h"

using namespace orbit;

namespace {

constexpr int64_t kFp8Codes = 1ll << 34;  // a store's codes stay below
constexpr int64_t kFp8Tiles = 1ll << 24;  // and its tiles: blocks of 256 threads in a launch of fewer than 2^32
constexpr int64_t kFp8Side = 1ll << 22;   // K: 256 rows of codes within 31-bit offsets

bool fp8_codes_fit(int64_t rows, int64_t n) {
  return rows < kFp8Codes && n < kFp8Codes && rows <= (kFp8Codes - 1) / fp8_wide(n);
}
bool fp8_tiles_fit(int64_t rows, int64_t n) {  // of sizes whose codes fit
  return cdiv(rows, 128) * cdiv(n, 128) < kFp8Tiles;
}

orbit_status fp8_store_check(const char* fn, const char* name, int64_t rows, int64_t n, const void* store, size_t bytes) {
  REQ(rows > 0 && n > 0, ORBIT_E_ARG, "%s: bad sizes %lld x %lld of %s", fn, (long long)rows, (long long)n, name);
  REQ(fp8_codes_fit(rows, n), ORBIT_E_UNSUPPORTED, "%s: %s of %lld x %lld values reaches 2^34 codes", fn, name,
      (long long)rows, (long long)n);
  REQ(fp8_tiles_fit(rows, n), ORBIT_E_UNSUPPORTED, "%s: %s of %lld x %lld values reaches 2^24 tiles", fn, name,
      (long long)rows, (long long)n);
  PTR(store, name);
  REQ(bytes >= fp8_store_bytes(rows, n), ORBIT_E_ARG, "%s: %s of %zu bytes is smaller than the %zu required", fn, name,
      bytes, fp8_store_bytes(rows, n));
  return ORBIT_OK;
}

orbit_status fp8_gemm_sizes(const char* fn, int64_t M, int64_t N, int64_t K) {
  REQ(M > 0 && N > 0 && K > 0 && N % 8 == 0, ORBIT_E_ARG,
      "%s: bad sizes M=%lld N=%lld K=%lld (N must be a multiple of 8)", fn, (long long)M, (long long)N, (long long)K);
  REQ(K < kFp8Side, ORBIT_E_UNSUPPORTED, "%s: K=%lld reaches 2^22", fn, (long long)K);
  // tiles of 128 x 128, or of 16 columns by 512 threads, in K ranges of at most 16
  REQ(N < (1ll << 26) && cdiv(M, 128) * cdiv(N, 128) < kFp8Tiles / 2, ORBIT_E_UNSUPPORTED, "%s: M=%lld N=%lld: too many tiles",
      fn, (long long)M, (long long)N);
  return ORBIT_OK;
}

orbit_status linear_check(const char* fn, const orbit_fp8_linear_desc* d) {
  REQ(d != nullptr, ORBIT_E_ARG, "%s: desc is NULL", fn);
  ORBIT_TRY(check_dtype(fn, d->dtype));
  REQ(d->rows > 0 && d->in > 0 && d->out > 0 && d->in % 8 == 0 && d->out % 8 == 0, ORBIT_E_ARG,
      "%s: bad sizes rows=%d in=%d out=%d (in and out must be multiples of 8)", fn, d->rows, d->in, d->out);
  ORBIT_TRY(fp8_gemm_sizes(fn, d->rows, d->out, d->in));
  ORBIT_TRY(fp8_gemm_sizes(fn, d->rows, d->in, d->out));
  ORBIT_TRY(fp8_gemm_sizes(fn, d->in, d->out, d->rows));
  return ORBIT_OK;
}

struct LinearWs {
  void *q, *qt;  // stores of x, or of dy and its transpose
  float* part;   // column sums of dy
  void* gws;
  size_t gws_bytes;
};

size_t linear_ws(const orbit_fp8_linear_desc& d, void* base, LinearWs* w) {
  Carver c(base);
  LinearWs t{};
  t.q = c.take<char>(fp8_store_bytes(d.rows, std::max(d.in, d.out)));
  t.qt = c.take<char>(fp8_store_bytes(d.out, d.rows));
  t.part = c.take<float>((size_t)cdiv(d.rows, 128) * d.out);
  t.gws_bytes = std::max({fp8_gemm_workspace_bytes(d.rows, d.out, d.in), fp8_gemm_workspace_bytes(d.rows, d.in, d.out),
                          fp8_gemm_workspace_bytes(d.in, d.out, d.rows)});
  t.gws = c.take<char>(t.gws_bytes);
  if (w) *w = t;
  return c.used();
}

}  // namespace

extern "C" {

size_t orbit_fp8_bytes(int64_t rows, int64_t n) {
  if (!(rows > 0 && n > 0 && fp8_codes_fit(rows, n) && fp8_tiles_fit(rows, n))) {
    set_error("orbit_fp8_bytes: bad sizes rows=%lld n=%lld", (long long)rows, (long long)n);
    return 0;
  }
  return fp8_store_bytes(rows, n);
}

orbit_status orbit_fp8_pack(int32_t dtype, int64_t rows, int64_t n, int32_t tile_rows, const void* x, int64_t ldx,
                            void* store, size_t store_bytes, void* store_t, size_t store_t_bytes, void* stream) {
  const char* fn = "orbit_fp8_pack";
  clear_error();
  ORBIT_TRY(check_dtype(fn, dtype));
  REQ(rows > 0 && n > 0, ORBIT_E_ARG, "%s: bad sizes rows=%lld n=%lld", fn, (long long)rows, (long long)n);
  REQ(tile_rows == 1 || tile_rows == 128, ORBIT_E_ARG, "%s: tile_rows must be 1 or 128", fn);
  REQ(store || store_t, ORBIT_E_ARG, "%s: both stores are NULL", fn);
  if (store) ORBIT_TRY(fp8_store_check(fn, "store", rows, n, store, store_bytes));
  if (store_t) ORBIT_TRY(fp8_store_check(fn, "store_t", n, rows, store_t, store_t_bytes));
  PTR(x, "x");
  REQ(ldx >= n && ldx % 8 == 0, ORBIT_E_ARG, "%s: ldx must be >= n and a multiple of 8", fn);
  REQ(store != store_t && x != store && x != store_t, ORBIT_E_ARG, "%s: x and the stores must not alias", fn);
  return fp8_pack((orbit_dtype)dtype, x, ldx, rows, n, tile_rows == 128, store, store_t, false, nullptr, S(stream));
}

orbit_status orbit_fp8_unpack(int32_t dtype, int64_t rows, int64_t n, const void* store, size_t store_bytes, void* x,
                              int64_t ldx, void* stream) {
  const char* fn = "orbit_fp8_unpack";
  clear_error();
  ORBIT_TRY(check_dtype(fn, dtype));
  ORBIT_TRY(fp8_store_check(fn, "store", rows, n, store, store_bytes));
  PTR(x, "x");
  REQ(ldx >= n && ldx % 8 == 0, ORBIT_E_ARG, "%s: ldx must be >= n and a multiple of 8", fn);
  REQ(x != store, ORBIT_E_ARG, "%s: x must not alias the store", fn);
  return fp8_unpack((orbit_dtype)dtype, store, rows, n, x, ldx, S(stream));
}

size_t orbit_fp8_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K) {
  if (fp8_gemm_sizes("orbit_fp8_gemm_workspace_bytes", M, N, K) != ORBIT_OK) return 0;
  return fp8_gemm_workspace_bytes(M, N, K);
}

orbit_status orbit_fp8_gemm(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* A, size_t a_bytes,
                            const void* B, size_t b_bytes, void* C, int64_t ldc, int32_t c_f32, const void* bias,
                            int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "orbit_fp8_gemm";
  clear_error();
  ORBIT_TRY(check_dtype(fn, dtype));
  ORBIT_TRY(fp8_gemm_sizes(fn, M, N, K));
  ORBIT_TRY(fp8_store_check(fn, "A", M, K, A, a_bytes));
  ORBIT_TRY(fp8_store_check(fn, "B", N, K, B, b_bytes));
  PTR(C, "C"); OPT_PTR(bias, "bias"); OPT_PTR(ws, "ws");
  REQ(ldc >= N && ldc % 8 == 0, ORBIT_E_ARG, "%s: ldc must be >= N and a multiple of 8", fn);
  REQ((c_f32 == 0 || c_f32 == 1) && (accumulate == 0 || accumulate == 1), ORBIT_E_ARG,
      "%s: c_f32 and accumulate must be 0 or 1", fn);
  REQ(!accumulate || c_f32 || dtype == ORBIT_F32, ORBIT_E_ARG, "%s: accumulate needs a float32 C", fn);
  REQ(C != A && C != B && (!ws || (ws != C && ws != A && ws != B)), ORBIT_E_ARG, "%s: C and ws must not alias an operand", fn);
  const size_t need = fp8_gemm_workspace_bytes(M, N, K);
  REQ(need == 0 || (ws && ws_bytes >= need), ORBIT_E_ARG, "%s: workspace of %zu bytes is smaller than the %zu required", fn,
      ws ? ws_bytes : 0, need);
  Fp8Gemm g;
  g.dtype = (orbit_dtype)dtype;
  g.A = A; g.B = B; g.C = C; g.ldc = ldc; g.M = M; g.N = N; g.K = K; g.out_f32 = c_f32 != 0;
  g.epi.bias = bias; g.epi.accumulate = accumulate;
  return fp8_gemm(g, ws, ws_bytes, S(stream));
}

size_t orbit_fp8_linear_saved_bytes(const orbit_fp8_linear_desc* desc) {
  if (linear_check("orbit_fp8_linear_saved_bytes", desc) != ORBIT_OK) return 0;
  return fp8_store_bytes(desc->in, desc->rows);
}

size_t orbit_fp8_linear_workspace_bytes(const orbit_fp8_linear_desc* desc) {
  if (linear_check("orbit_fp8_linear_workspace_bytes", desc) != ORBIT_OK) return 0;
  return linear_ws(*desc, nullptr, nullptr);
}

orbit_status orbit_fp8_linear_fwd(const orbit_fp8_linear_desc* desc, const void* x, int64_t ldx, const void* w_t,
                                  size_t w_t_bytes, const void* bias, void* y, int64_t ldy, void* saved, void* ws,
                                  size_t ws_bytes, void* stream) {
  const char* fn = "orbit_fp8_linear_fwd";
  clear_error();
  ORBIT_TRY(linear_check(fn, desc));
  const orbit_fp8_linear_desc& d = *desc;
  PTR(x, "x"); OPT_PTR(bias, "bias"); PTR(y, "y"); OPT_PTR(saved, "saved"); PTR(ws, "ws");
  REQ(ldx >= d.in && ldx % 8 == 0, ORBIT_E_ARG, "%s: ldx must be >= in and a multiple of 8", fn);
  REQ(ldy >= d.out && ldy % 8 == 0, ORBIT_E_ARG, "%s: ldy must be >= out and a multiple of 8", fn);
  REQ(y != x, ORBIT_E_ARG, "%s: y must not alias x", fn);
  ORBIT_TRY(fp8_store_check(fn, "w_t", d.out, d.in, w_t, w_t_bytes));
  LinearWs w;
  const size_t need = linear_ws(d, ws, &w);
  REQ(ws_bytes >= need, ORBIT_E_ARG, "%s: workspace of %zu bytes is smaller than the %zu required", fn, ws_bytes, need);
  hipStream_t s = S(stream);
  const orbit_dtype dt = (orbit_dtype)d.dtype;
  ORBIT_TRY(fp8_pack(dt, x, ldx, d.rows, d.in, false, w.q, saved, true, nullptr, s));
  Fp8Gemm g;
  g.dtype = dt;
  g.A = w.q; g.B = w_t; g.C = y; g.ldc = ldy; g.M = d.rows; g.N = d.out; g.K = d.in; g.epi.bias = bias;
  return fp8_gemm(g, w.gws, w.gws_bytes, s);
}

orbit_status orbit_fp8_linear_bwd(const orbit_fp8_linear_desc* desc, const void* saved, const void* w, size_t w_bytes,
                                  const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dw, float* db,
                                  int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "orbit_fp8_linear_bwd";
  clear_error();
  ORBIT_TRY(linear_check(fn, desc));
  const orbit_fp8_linear_desc& d = *desc;
  PTR(saved, "saved"); PTR(dy, "dy"); OPT_PTR(dx, "dx"); PTR(dw, "dw"); OPT_PTR(db, "db"); PTR(ws, "ws");
  if (dx) ORBIT_TRY(fp8_store_check(fn, "w", d.in, d.out, w, w_bytes));
  REQ(lddy >= d.out && lddy % 8 == 0, ORBIT_E_ARG, "%s: lddy must be >= out and a multiple of 8", fn);
  REQ(!dx || (lddx >= d.in && lddx % 8 == 0), ORBIT_E_ARG, "%s: lddx must be >= in and a multiple of 8", fn);
  REQ(dx != dy, ORBIT_E_ARG, "%s: dx must not alias dy", fn);
  REQ(accumulate == 0 || accumulate == 1, ORBIT_E_ARG, "%s: accumulate must be 0 or 1", fn);
  LinearWs t;
  const size_t need = linear_ws(d, ws, &t);
  REQ(ws_bytes >= need, ORBIT_E_ARG, "%s: workspace of %zu bytes is smaller than the %zu required", fn, ws_bytes, need);
  hipStream_t s = S(stream);
  const orbit_dtype dt = (orbit_dtype)d.dtype;
  ORBIT_TRY(fp8_pack(dt, dy, lddy, d.rows, d.out, false, dx ? t.q : nullptr, t.qt, false, db ? t.part : nullptr, s));
  if (dx) {
    Fp8Gemm g;
    g.dtype = dt;
    g.A = t.q; g.B = w; g.C = dx; g.ldc = lddx; g.M = d.rows; g.N = d.in; g.K = d.out;
    ORBIT_TRY(fp8_gemm(g, t.gws, t.gws_bytes, s));
  }
  Fp8Gemm g;
  g.dtype = dt;
  g.A = saved; g.B = t.qt; g.C = dw; g.ldc = d.out; g.M = d.in; g.N = d.out; g.K = d.rows;
  g.out_f32 = true; g.epi.accumulate = accumulate;
  ORBIT_TRY(fp8_gemm(g, t.gws, t.gws_bytes, s));
  if (!db) return ORBIT_OK;
  ColFinal fin;
  fin.add(t.part, d.out, (int)cdiv(d.rows, 128), d.out, db);
  return fin.run(accumulate, s);
}

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------
static orbit_status rope_check(const char* fn, const orbit_qk_rope_desc* desc, RopeDims* o) {
  REQ(desc != nullptr, ORBIT_E_ARG, "%s: desc is NULL", fn);
  const orbit_qk_rope_desc& d = *desc;
  ORBIT_TRY(check_dtype(fn, d.dtype));
  REQ(d.tokens > 0 && d.q_heads > 0 && d.k_heads > 0, ORBIT_E_ARG, "%s: sizes must be positive (tokens=%d q_heads=%d k_heads=%d)",
      fn, d.tokens, d.q_heads, d.k_heads);
  REQ(d.head_dim == 32 || d.head_dim == 64 || d.head_dim == 128 || d.head_dim == 192 || d.head_dim == 256,
      ORBIT_E_UNSUPPORTED, "%s: head_dim %d unsupported (32, 64, 128, 192, 256)", fn, d.head_dim);
  REQ((d.norm == 0 || d.norm == 1) && (d.near == 0 || d.near == 1), ORBIT_E_ARG, "%s: norm and near must be 0 or 1", fn);
  REQ(!d.norm || d.eps > 0.f, ORBIT_E_ARG, "%s: eps must be positive", fn);
  REQ(d.tokens < (1 << 24) && (int64_t)d.tokens * ((int64_t)d.q_heads + d.k_heads) < (1ll << 31) &&
      ((int64_t)d.q_heads + d.k_heads) * d.head_dim < (1ll << 31), ORBIT_E_UNSUPPORTED,
      "%s: %d tokens of %d + %d heads are too many", fn, d.tokens, d.q_heads, d.k_heads);
  RopeDims z{};
  z.T = d.tokens; z.qh = d.q_heads; z.kh = d.k_heads; z.dh = d.head_dim;
  z.norm = d.norm != 0; z.eps = d.eps; z.dt = (orbit_dtype)d.dtype;
  ORBIT_TRY(rope_axes(fn, d.axes, d.pos_rows, d.near, d.axis, &z));
  *o = z;
  return ORBIT_OK;
}

static orbit_status rope_ptrs(const char* fn, const RopeDims& z, const orbit_qk_rope_params* p, const float* pos,
                              const float* freq, bool shifts, RopeParams* o) {
  *o = RopeParams{};
  PTR(pos, "pos"); PTR(freq, "freq");
  if (!z.norm) return ORBIT_OK;
  REQ(p != nullptr, ORBIT_E_ARG, "%s: params is NULL", fn);
  PTR(p->qn_g, "qn_g"); PTR(p->kn_g, "kn_g");
  if (shifts) { PTR(p->qn_b, "qn_b"); PTR(p->kn_b, "kn_b"); }
  *o = RopeParams{p->qn_g, p->qn_b, p->kn_g, p->kn_b};
  return ORBIT_OK;
}

orbit_status orbit_qk_rope_fwd(const orbit_qk_rope_desc* desc, const orbit_qk_rope_params* p, const float* pos,
                               const float* freq, const void* src, int64_t lds, void* dst, int64_t ldd, float* mean,
                               float* rstd, void* stream) {
  const char* fn = "orbit_qk_rope_fwd";
  clear_error();
  RopeDims z;
  RopeParams rp;
  ORBIT_TRY(rope_check(fn, desc, &z));
  ORBIT_TRY(rope_ptrs(fn, z, p, pos, freq, true, &rp));
  PTR(src, "src"); PTR(dst, "dst"); OPT_PTR(mean, "mean"); OPT_PTR(rstd, "rstd");
  const int64_t n = (int64_t)(z.qh + z.kh) * z.dh;
  REQ(lds >= n && lds % 8 == 0 && ldd >= n && ldd % 8 == 0, ORBIT_E_ARG,
      "%s: leading dimensions must be >= %lld and multiples of 8", fn, (long long)n);
  REQ(dst != src || ldd == lds, ORBIT_E_ARG, "%s: dst may be src with the same leading dimension only", fn);
  REQ((mean == nullptr) == (rstd == nullptr), ORBIT_E_ARG, "%s: mean and rstd go together", fn);
  return rope_fwd(z, rp, pos, freq, src, lds, dst, ldd, mean, rstd, S(stream));
}

size_t orbit_qk_rope_bwd_workspace_bytes(const orbit_qk_rope_desc* desc) {
  RopeDims z;
  if (rope_check("orbit_qk_rope_bwd_workspace_bytes", desc, &z) != ORBIT_OK) return 0;
  return rope_bwd_ws_bytes(z);
}

orbit_status orbit_qk_rope_bwd(const orbit_qk_rope_desc* desc, const orbit_qk_rope_params* p, const float* pos,
                               const float* freq, const void* src, int64_t lds, const float* mean, const float* rstd,
                               const void* dy, int64_t lddy, void* dx, int64_t lddx, const orbit_qk_rope_grads* g,
                               int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "orbit_qk_rope_bwd";
  clear_error();
  RopeDims z;
  RopeParams rp;
  ORBIT_TRY(rope_check(fn, desc, &z));
  ORBIT_TRY(rope_ptrs(fn, z, p, pos, freq, false, &rp));
  PTR(dy, "dy"); PTR(dx, "dx");
  const int64_t n = (int64_t)(z.qh + z.kh) * z.dh;
  REQ(lddy >= n && lddy % 8 == 0 && lddx >= n && lddx % 8 == 0, ORBIT_E_ARG,
      "%s: leading dimensions must be >= %lld and multiples of 8", fn, (long long)n);
  REQ(dx != dy || lddx == lddy, ORBIT_E_ARG, "%s: dx may be dy with the same leading dimension only", fn);
  REQ(accumulate == 0 || accumulate == 1, ORBIT_E_ARG, "%s: accumulate must be 0 or 1", fn);
  RopeGrads gg{};
  if (z.norm) {
    PTR(src, "src"); PTR(mean, "mean"); PTR(rstd, "rstd"); PTR(ws, "ws");
    REQ(lds >= n && lds % 8 == 0, ORBIT_E_ARG, "%s: leading dimensions must be >= %lld and multiples of 8", fn, (long long)n);
    REQ(dx != src, ORBIT_E_ARG, "%s: dx must not alias src", fn);
    REQ(g != nullptr, ORBIT_E_ARG, "%s: grads is NULL", fn);
    PTR(g->qn_g, "grads.qn_g"); PTR(g->qn_b, "grads.qn_b"); PTR(g->kn_g, "grads.kn_g"); PTR(g->kn_b, "grads.kn_b");
    const size_t need = rope_bwd_ws_bytes(z);
    REQ(ws_bytes >= need, ORBIT_E_ARG, "%s: workspace of %zu bytes is smaller than the %zu required", fn, ws_bytes, need);
    gg = RopeGrads{g->qn_g, g->qn_b, g->kn_g, g->kn_b};
  }
  return rope_bwd(z, rp, pos, freq, src, lds, mean, rstd, dy, lddy, dx, lddx, gg, accumulate, ws, nullptr, S(stream));
}

}  // extern "C"

namespace orbit {
// the axes and positions of z.T tokens, of the call and of the block
orbit_status rope_axes(const char* fn, int32_t axes, int32_t pos_rows, int32_t near, const uint8_t* axis, RopeDims* z) {
  REQ(axes >= 1 && axes <= 4, ORBIT_E_ARG, "%s: axes=%d must be 1 to 4", fn, axes);
  REQ(pos_rows > 0 && z->T % pos_rows == 0, ORBIT_E_ARG, "%s: pos_rows=%d must divide the %d tokens", fn, pos_rows, z->T);
  REQ(near == 0 || near == 1, ORBIT_E_ARG, "%s: near must be 0 or 1", fn);
  z->axes = axes; z->pos_rows = pos_rows; z->near = near != 0;
  for (int i = 0; i < z->dh / 2; ++i) {
    REQ(axis[i] < axes, ORBIT_E_ARG, "%s: axis[%d]=%d is not below axes=%d", fn, i, axis[i], axes);
    z->ax.axis[i] = axis[i];
  }
  return ORBIT_OK;
}
}  // namespace orbit
