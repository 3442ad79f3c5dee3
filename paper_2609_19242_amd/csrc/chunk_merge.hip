// The chunks' partial outputs of tiles whose keys were cut (chunk_plan.hip),
// joined (partials.hpp), gfx950.  How many tiles that is only the device knows: a
// grid of at most kMergeWgs workgroups takes groups of rows of (tile, KV head) in turn.
// Bound by the launch and by reading.
#include "chunk.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

constexpr int kMergeWgs = 2048;

template <int D, bool BF16>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkArgs a) {
  using Z = PartLse<BF16>;
  constexpr int LPR = JoinedRow<D>::LPR, ROWS = 256 / LPR, GROUPS = (BF16 ? kPrefixSharedRows : kPrefixRowsF32) / ROWS;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int joins = imin(a.plan[kPlanJoins], a.max_joins);
  const int64_t units = (int64_t)joins * a.kv_heads * GROUPS;
  const Z* const z = (const Z*)a.part_lse;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int grp = (int)(u % GROUPS), kvh = (int)(u / GROUPS % a.kv_heads);
    const ChunkJoin& t = a.joins[u / GROUPS / a.kv_heads];
    if (grp * ROWS >= t.nrows) continue;
    const int64_t first = kvh * a.part_rows + t.part;
    auto write = [&](int row, int col, const JoinedRow<D, Z>& r) __attribute__((always_inline)) {
      const int n = t.row0 + row, i = n / a.group, h = kvh * a.group + (n - i * a.group);
      const int64_t token = t.token0 + i, at = token * a.os + (int64_t)h * D + col * 4;
      if constexpr (BF16) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = to_bf16(r.x[e]);
        *(bf16x4*)((bf16*)a.o + at) = y;
      } else {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (float)r.x[e];
        *(f32x4*)((float*)a.o + at) = y;
      }
      if (col == 0) a.lse[h * a.pitch + token] = r.lse;
    };
    if (t.n <= kFewParts) {  // a row per LPR lanes
      const int row = grp * ROWS + threadIdx.x / LPR, col = threadIdx.x % LPR;
      if (row < t.nrows) {
        auto at = [&](int j) { return first + (int64_t)j * t.nrows + row; };
        write(row, col, join_few<D>(a.part_o, z, at, t.n, col));
      }
    } else {  // a wave per row
      for (int row = grp * ROWS + w; row < imin(t.nrows, (grp + 1) * ROWS); row += 4) {
        auto at = [&](int j) { return first + (int64_t)j * t.nrows + row; };
        const JoinedRow<D, Z> r = join_partials<D>(a.part_o, z, at, t.n, lane);
        if (lane < LPR) write(row, lane, r);
      }
    }
  }
}

}  // namespace

hipError_t launch_chunk_merge(const ChunkArgs& a, int head_dim, int is_bf16, hipStream_t s) {
  const int64_t rows = (int64_t)a.max_joins * a.kv_heads * (is_bf16 ? kPrefixSharedRows : kPrefixRowsF32);
  const int n = (int)(rows / 4 < kMergeWgs ? rows / 4 : kMergeWgs);
  if (n == 0) return hipSuccess;
  const dim3 grid(n), threads(256);
  if (head_dim == 128) {
    if (is_bf16) hipLaunchKernelGGL((chunk_merge_kernel<128, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((chunk_merge_kernel<128, false>), grid, threads, 0, s, a);
  } else {
    if (is_bf16) hipLaunchKernelGGL((chunk_merge_kernel<64, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((chunk_merge_kernel<64, false>), grid, threads, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace bdlm
