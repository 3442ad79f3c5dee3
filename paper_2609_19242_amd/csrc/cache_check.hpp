// Checks and records of a paged cache that its C entry points share (cache_api.cpp).
#pragma once

#include "api_util.hpp"
#include "cache.hpp"

namespace bdlm {

constexpr int64_t kMaxSeqs = (int64_t)1 << 19;  // a bit each in the bookkeeping's LDS
constexpr int64_t kMaxPages = ((int64_t)1 << 30) - 1;
constexpr int64_t kMaxRows = (int64_t)1 << 25;  // query rows x heads of one attention call (a grid dimension of the merge)
constexpr int64_t kMaxWgs = (int64_t)1 << 22;

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bdlm_status check_cache(const bdlm_cache* c);
CacheArg cache_arg(const bdlm_cache* c);

}  // namespace bdlm
