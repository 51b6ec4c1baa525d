// Rotary positions with several axes on the heads of q and k, with the
// LayerNorm over a head that may stand before them: host launchers.
#pragma once
#include "common.h"
#include "kernels.h"

namespace orbit {

constexpr int kRopePairs = 128;  // of the widest head

struct RopeAxes {
  uint8_t axis[kRopePairs];  // of each pair
};

// Pair i of a head (columns i and dh / 2 + i, or 2 i and 2 i + 1 where near) turns
// by pos[t % pos_rows][axis[i]] freq[i].
struct RopeDims {
  int T, qh, kh, dh;  // tokens, heads of q and of k (columns: q heads, then k heads)
  bool norm, near;
  int axes, pos_rows;
  float eps;
  orbit_dtype dt;
  RopeAxes ax;
};
struct RopeParams { const void *qn_g, *qn_b, *kn_g, *kn_b; };
struct RopeGrads { float *qn_g, *qn_b, *kn_g, *kn_b; };

// src -> dst (may be src); mean, rstd [T, qh + kh] (may be null)
orbit_status rope_fwd(const RopeDims& z, const RopeParams& p, const float* pos, const float* freq, const void* src,
                      int64_t lds, void* dst, int64_t ldd, float* mean, float* rstd, hipStream_t s);
size_t rope_bwd_ws_bytes(const RopeDims& z);
// gradient dy of dst -> dx of src (may be dy); parameter gradients into fin where
// it is given, else finished here
orbit_status rope_bwd(const RopeDims& z, const RopeParams& p, const float* pos, const float* freq, const void* src,
                      int64_t lds, const float* mean, const float* rstd, const void* dy, int64_t lddy, void* dx,
                      int64_t lddx, const RopeGrads& g, int accumulate, void* ws, ColFinal* fin, hipStream_t s);

// fills z's axes and positions from a caller's, checked (abi_fp8.cpp)
orbit_status rope_axes(const char* fn, int32_t axes, int32_t pos_rows, int32_t near, const uint8_t* axis, RopeDims* z);

}  // namespace orbit
