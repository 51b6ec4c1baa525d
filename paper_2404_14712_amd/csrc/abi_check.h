// Argument checks shared by the C ABI entry points: a failed check leaves its
// text for orbit_last_error and returns its status. `fn` names the entry point.
#pragma once
#include "common.h"

namespace orbit {

inline size_t esz(int dt) { return dt == ORBIT_BF16 ? 2 : 4; }
inline hipStream_t S(void* st) { return static_cast<hipStream_t>(st); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define REQ(cond, code, ...)        \
  do {                              \
    if (!(cond)) {                  \
      set_error(__VA_ARGS__);       \
      return code;                  \
    }                               \
  } while (0)

#define PTR(p, name)                                                        \
  do {                                                                      \
    REQ((p) != nullptr, ORBIT_E_ARG, "%s: %s is NULL", fn, name);           \
    REQ(aligned16(p), ORBIT_E_ARG, "%s: %s is not 16-byte aligned", fn, name); \
  } while (0)

#define OPT_PTR(p, name)                                                    \
  do {                                                                      \
    if (p) REQ(aligned16(p), ORBIT_E_ARG, "%s: %s is not 16-byte aligned", fn, name); \
  } while (0)

inline orbit_status check_dtype(const char* fn, int dt) {
  REQ(dt == ORBIT_F32 || dt == ORBIT_BF16, ORBIT_E_ARG, "%s: dtype %d is not ORBIT_F32 or ORBIT_BF16", fn, dt);
  return ORBIT_OK;
}

}  // namespace orbit
