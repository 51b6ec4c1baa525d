// Gated norms (gnorm.hip): the norm, gate and residual scale of a sub-layer's
// output f on the residual stream x, and the norm that the next product reads:
//   p = LN(f; post) or f;  y = x + scale gate p;  h = LN(y; pre).
#pragma once
#include "kernels.h"

namespace orbit {

struct GnormDims {
  int rows, n, gates;  // gates: rows of the gate (0: none), each for rows / gates consecutive rows
  bool post, pre;
  float scale, eps;
  orbit_dtype dt;
};

struct GnormParams {
  const void *gate, *post_g, *post_b, *pre_g, *pre_b;
};

// f == nullptr: f is read from the 8-bit store; else the store (may be null)
// receives f. stats [rows, 4]: mean and 1 / sqrt(variance + eps) of f (zeros
// without the post norm) and of y (zeros without the pre norm). h is unused
// without the pre norm.
orbit_status gnorm_fwd(const GnormDims& z, const GnormParams& p, const void* x, const void* f, void* store, void* y,
                       void* h, float* stats, hipStream_t s);

// dh (null without the pre norm) and dy (null: zero) -> dx (may be null; the
// gradient of x and of y's other readers together) and df (may be null without
// the post norm and a gate), and the float32 parameter gradients. f == nullptr:
// from the store; neither is read without the post norm and a gate. ws:
// gnorm_bwd_ws_bytes.
size_t gnorm_bwd_ws_bytes(const GnormDims& z);
struct GnormGrads {
  float *gate, *post_g, *post_b, *pre_g, *pre_b;
};
orbit_status gnorm_bwd(const GnormDims& z, const GnormParams& p, const void* f, const void* store, const void* y,
                       const float* stats, const void* dh, const void* dy, void* dx, void* df, const GnormGrads& g,
                       int accumulate, void* ws, hipStream_t s);

}  // namespace orbit
