// The chunks' partial outputs of attention over a paged cache (cache.hpp)
// joined (partials.hpp), gfx950.
// Bound by reading the partials (16,384 rows of 128, 4 chunks: 8.1 us, 4.6 TB/s;
// 2,048 rows, up to 10 chunks: 5.0 us).
#include "cache.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

static_assert(kShortJoin == kFewParts, "the plan's number is the kernel's");

template <int D, bool BF16, bool FEW>
__global__ __launch_bounds__(256) void prefix_merge_kernel(const PrefixArgs a) {
  constexpr int LPR = JoinedRow<D>::LPR, RPW = FEW ? 64 / LPR : 1;  // rows per wave
  const int64_t total = (int64_t)a.requests * a.rows * a.heads;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = FEW ? threadIdx.x % LPR : threadIdx.x & 63;
  const int64_t row = ((int64_t)blockIdx.x * 4 + w) * RPW + (FEW ? (threadIdx.x & 63) / LPR : 0);
  if (row >= total) return;
  const int parts = a.prefix_chunks + a.own_chunks;
  auto at = [&](int j) { return j * total + row; };
  using Z = PartLse<BF16>;
  const Z* const z = (const Z*)a.part_lse;
  const JoinedRow<D, Z> r = FEW ? join_few<D>(a.part_o, z, at, parts, lane) : join_partials<D>(a.part_o, z, at, parts, lane);
  if (lane >= LPR) return;
  if constexpr (BF16) {
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to_bf16(r.x[e]);
    *(bf16x4*)((bf16*)a.o + row * D + lane * 4) = y;
  } else {
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)r.x[e];
    *(f32x4*)((float*)a.o + row * D + lane * 4) = y;
  }
  if (lane == 0) {
    PrefixRow pr;
    pr.token = (int)(row / a.heads);
    pr.head = (int)(row - (int64_t)pr.token * a.heads);
    pr.end = 0;
    a.lse[prefix_lse_at(a, pr)] = r.lse;
  }
}

template <int D, bool BF16>
void launch(const PrefixArgs& a, int64_t rows, hipStream_t s) {
  const bool few = a.prefix_chunks + a.own_chunks <= kFewParts;
  const int per = few ? 4 * (64 / JoinedRow<D>::LPR) : 4;  // rows of a workgroup
  const dim3 grid((unsigned)((rows + per - 1) / per)), threads(256);
  if (few) hipLaunchKernelGGL((prefix_merge_kernel<D, BF16, true>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((prefix_merge_kernel<D, BF16, false>), grid, threads, 0, s, a);
}

}  // namespace

hipError_t launch_prefix_merge(const PrefixArgs& a, int head_dim, int is_bf16, hipStream_t s) {
  const int64_t rows = (int64_t)a.requests * a.rows * a.heads;
  if (rows == 0) return hipSuccess;
  if (head_dim == 128) is_bf16 ? launch<128, true>(a, rows, s) : launch<128, false>(a, rows, s);
  else is_bf16 ? launch<64, true>(a, rows, s) : launch<64, false>(a, rows, s);
  return hipGetLastError();
}

}  // namespace bdlm
