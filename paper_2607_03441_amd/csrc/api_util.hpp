// What the files of the C ABI layer share: the status and message of a failing call, and argument checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "attt.h"

namespace attt {

// Sets the calling thread's message and returns `code`.
attt_status fail(attt_status code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

inline attt_status hip_fail(hipError_t e, const char* where) {
  return fail(ATTT_EHIP, "%s: %s", where, hipGetErrorString(e));
}

#define HIP_TRY(expr, where)                  \
  do {                                        \
    hipError_t e_ = (expr);                   \
    if (e_ != hipSuccess) return hip_fail(e_, where); \
  } while (0)

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

// Offsets [E+1] that start at 0 and do not decrease, with at most `limit` entries an episode.
inline attt_status check_offsets(const char* what, const int64_t* off, int32_t E, int64_t limit) {
  if (!off) return fail(ATTT_EINVAL, "%s: offsets pointer is null", what);
  if (off[0] != 0) return fail(ATTT_EINVAL, "%s: offsets[0] must be 0", what);
  for (int32_t e = 0; e < E; ++e) {
    if (off[e + 1] < off[e]) return fail(ATTT_EINVAL, "%s: offsets decrease at episode %d", what, e);
    if (off[e + 1] - off[e] > limit)
      return fail(ATTT_EUNSUPPORTED, "%s: episode %d holds %lld entries (limit %lld)", what, e,
                  (long long)(off[e + 1] - off[e]), (long long)limit);
  }
  return ATTT_OK;
}

}  // namespace attt
