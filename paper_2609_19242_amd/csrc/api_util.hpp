// What the C entry points share: error messages, kernel timing, argument checks.
#pragma once

#include "bdlm_attn.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bdlm {

// The calling thread's message (bdlm_last_error); returns `st`.
bdlm_status fail(bdlm_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
bdlm_status hip_fail(hipError_t e, const char* what);

// Kernels by id (bdlm_kernel_name).
enum KernelId {
  kKFwdBf16 = 0, kKFwdF32, kKMerge, kKBwdDqF32, kKBwdBf16, kKBwdDq, kKBwdF32,
  kKPackedFwd, kKPackedDq, kKPackedDkDv, kKPrefixAttn, kKPrefixMerge, kKCachePages, kKCacheWrite, kKCount
};

// Per-thread kernel timing (bdlm_timing_enable): events around a launch.
bool timing_on();
hipError_t timing_begin(int id, hipStream_t s);
hipError_t timing_end(hipStream_t s);

// Launch through f(), bracketed by events when timing is on.
template <class F>
hipError_t timed(int id, hipStream_t s, F&& f) {
  if (!timing_on()) return f();
  hipError_t e = timing_begin(id, s);
  if (e != hipSuccess) return e;
  e = f();
  return e != hipSuccess ? e : timing_end(s);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int64_t kMaxPos = (int64_t)1 << 30;

}  // namespace bdlm
