// The chunks' partial outputs of attention over a paged cache (cache.hpp)
// joined (partials.hpp), gfx950.
// Bound by reading the partials (16,384 rows of 128, 4 chunks: 10.7 us, 3.9 TB/s;
// 2,048 rows, up to 10 chunks: 4.8 us).
#include "cache.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

template <int D, bool BF16>
__global__ __launch_bounds__(256) void prefix_merge_kernel(const PrefixArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t total = (int64_t)a.requests * a.rows * a.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= total) return;
  const JoinedRow<D> r = join_partials<D>(a.part_o, a.part_lse, [&](int j) { return j * total + row; },
                                          a.prefix_chunks + a.own_chunks, lane);
  if (lane >= JoinedRow<D>::LPR) return;
  if constexpr (BF16) {
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to_bf16(r.x[e]);
    *(bf16x4*)((bf16*)a.o + row * D + lane * 4) = y;
  } else {
    *(f32x4*)((float*)a.o + row * D + lane * 4) = r.x;
  }
  if (lane == 0) {
    PrefixRow pr;
    pr.token = (int)(row / a.heads);
    pr.head = (int)(row - (int64_t)pr.token * a.heads);
    pr.end = 0;
    a.lse[prefix_lse_at(a, pr)] = r.lse;
  }
}

}  // namespace

hipError_t launch_prefix_merge(const PrefixArgs& a, int head_dim, int is_bf16, hipStream_t s) {
  const int64_t rows = (int64_t)a.requests * a.rows * a.heads;
  const dim3 grid((unsigned)((rows + 3) / 4)), threads(256);
  if (rows == 0) return hipSuccess;
  if (head_dim == 128) {
    if (is_bf16) hipLaunchKernelGGL((prefix_merge_kernel<128, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((prefix_merge_kernel<128, false>), grid, threads, 0, s, a);
  } else {
    if (is_bf16) hipLaunchKernelGGL((prefix_merge_kernel<64, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((prefix_merge_kernel<64, false>), grid, threads, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace bdlm
