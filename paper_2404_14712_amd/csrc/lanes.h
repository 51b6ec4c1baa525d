// Reductions over a wave without LDS traffic: DPP moves within rows of 16
// lanes, lane swaps between rows. After step k every lane holds the result of
// its group of 2^(k+1) lanes; a step's partner lanes are the neighbour, the
// other pair, the other quad (mirrored within 8), the other half row (mirrored
// within 16), the other row of a pair and the other half of the wave.
#pragma once
#include "common.h"

namespace orbit {

template <int STEP> ORBIT_DEV void wave_pair(float v, float& a, float& b) {
  if constexpr (STEP < 4) {
    constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
    a = v;
    b = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xF, 0xF, true));
  } else {
    const uint32_t u = __float_as_uint(v);
    if constexpr (STEP == 4) {
      const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
      a = __uint_as_float(r[0]);
      b = __uint_as_float(r[1]);
    } else {
      const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
      a = __uint_as_float(r[0]);
      b = __uint_as_float(r[1]);
    }
  }
}

template <int STEP = 0> ORBIT_DEV float wave_add(float v) {
  float a, b;
  wave_pair<STEP>(v, a, b);
  if constexpr (STEP == 5) return a + b;
  else return wave_add<STEP + 1>(a + b);
}

// Mean and sum of squared deviations (q) of the values that a wave's lanes
// hold, from each lane's own (exact pairwise merging: no difference of large
// sums). The lanes' counts are fixed, so the merge weights are set once.
struct WaveMoments {
  float w[6], wn[6];  // step k: n_b / (n_a + n_b), n_a n_b / (n_a + n_b)
  float count;        // of the wave
  template <int STEP = 0> ORBIT_DEV void init(float n) {
    float a, b;
    wave_pair<STEP>(n, a, b);
    const float s = a + b, inv = s > 0.f ? 1.f / s : 0.f;
    w[STEP] = b * inv;
    wn[STEP] = a * b * inv;
    if constexpr (STEP == 5) count = s;
    else init<STEP + 1>(s);
  }
  template <int STEP = 0> ORBIT_DEV void merge(float& m, float& q) const {
    float ma, mb, qa, qb;
    wave_pair<STEP>(m, ma, mb);
    wave_pair<STEP>(q, qa, qb);
    const float d = mb - ma;
    m = fmaf(d, w[STEP], ma);
    q = fmaf(d * d, wn[STEP], qa + qb);
    if constexpr (STEP < 5) merge<STEP + 1>(m, q);
  }
};

}  // namespace orbit
