// The C ABI's argument checks: a failed one records its message for wam_last_error() and
// returns its status from the entry point, before anything is launched.
#pragma once
#include <stdint.h>

#include "../../include/wamdit.h"

namespace wam {

// records the message (thread-local) and returns st
wam_status fail(wam_status st, const char* fmt, ...);

#define CHECK(cond, st, ...) \
  do {                       \
    if (!(cond)) return fail(st, __VA_ARGS__); \
  } while (0)

#define HIPCHECK(expr)                                                              \
  do {                                                                              \
    hipError_t e_ = (expr);                                                         \
    if (e_ != hipSuccess) return fail(WAM_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define TRY(expr)                      \
  do {                                 \
    wam_status s_ = (expr);            \
    if (s_ != WAM_OK) return s_;       \
  } while (0)

inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

inline wam_status need_ptr(const void* p, const char* name) {
  if (!p) return fail(WAM_EINVAL, "%s is NULL", name);
  if (!al16(p)) return fail(WAM_EINVAL, "%s is not 16-byte aligned", name);
  return WAM_OK;
}
inline wam_status opt_ptr(const void* p, const char* name) {
  if (p && !al16(p)) return fail(WAM_EINVAL, "%s is not 16-byte aligned", name);
  return WAM_OK;
}

}  // namespace wam
