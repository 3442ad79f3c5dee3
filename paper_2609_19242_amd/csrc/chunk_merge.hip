// The chunks' partial outputs of tiles whose keys were cut (chunk_plan.hip),
// joined (partials.hpp), gfx950.  How many there are only the device knows: a grid of
// at most kMergeWgs workgroups takes the plan's units for each KV head in turn.
// Few parts: a row per D / 4 lanes.  Many (a long walk of one request): a workgroup
// per row, whose waves take parts in turn and add up through LDS.
// Bound by the launch (4 to 5 us) and by reading: two parts each of 2,048 rows, 32 heads, d 128,
// 16.6 us (5.1 TB/s); a row per workgroup for few parts too took 17 us where nothing was cut.
#include "chunk.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

constexpr int kMergeWgs = 2048;
static_assert(kShortJoin == kFewParts, "the plan's number is the kernel's");

// The four waves' sums over their parts of a row, with maximum m of all, in wave 0's lanes < D / 4.
template <int D, class Z>
struct ManyParts {
  static constexpr int LPR = JoinedRow<D>::LPR, PP = 64 / LPR;  // lanes per part, parts of a wave at a time
  Joined4<Z> x[4][LPR];
  Z sum[4];
  __device__ __forceinline__ JoinedRow<D, Z> join(const float* o, const Z* z, int64_t first, int step, int parts, int w, int lane) {
    const int part = lane / LPR, col = lane % LPR;
    Z m = -INFINITY;
    for (int j = lane; j < parts; j += 64) m = max_of(m, z[first + (int64_t)j * step]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) m = max_of(m, xor_of(m, s));
    const Z ref = m == -INFINITY ? Z(0) : m;
    Z all = 0;
    Joined4<Z> y = {0, 0, 0, 0};
    for (int base = w * PP; base < parts; base += 16 * PP) {
      Z zz[4];
      f32x4 p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t row = first + (int64_t)imin(base + 4 * k * PP + part, parts - 1) * step;
        zz[k] = z[row];
        p[k] = *(const f32x4*)(o + row * D + col * 4);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool seen = base + 4 * k * PP + part < parts && zz[k] > -INFINITY;
        const Z f = seen ? pow2(zz[k] - ref) : Z(0);
        all += f;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = seen ? fma_of(f, Z(p[k][e]), y[e]) : y[e];
      }
    }
#pragma unroll
    for (int s = LPR; s < 64; s <<= 1) {
      all += xor_of(all, s);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += xor_of(y[e], s);
    }
    __syncthreads();  // (the sums of a row before are read)
    if (lane < LPR) x[w][lane] = y;
    if (lane == 0) sum[w] = all;
    __syncthreads();
    y = x[0][col] + x[1][col] + x[2][col] + x[3][col];
    return joined<D, Z>(y, m, sum[0] + sum[1] + sum[2] + sum[3]);
  }
};

template <int D, bool BF16>
__global__ __launch_bounds__(256) void chunk_merge_kernel(const ChunkArgs a) {
  using Z = PartLse<BF16>;
  constexpr int LPR = JoinedRow<D>::LPR;
  static_assert(256 / LPR == join_rows(D), "a unit's rows");
  __shared__ ManyParts<D, Z> many;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)plan_joins(a) * a.kv_heads;
  const Z* const z = (const Z*)a.part_lse;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int n = (int)(u / a.kv_heads), kvh = (int)(u - (int64_t)n * a.kv_heads);
    const ChunkJoin t = a.joins[n];
    const int64_t first = kvh * a.part_rows + t.part;
    auto write = [&](int row, int col, const JoinedRow<D, Z>& r) __attribute__((always_inline)) {
      const int q = t.row0 + row, i = q / a.group, h = kvh * a.group + (q - i * a.group);
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
    if (t.n <= kFewParts) {
      const int row = threadIdx.x / LPR, col = threadIdx.x % LPR;
      if (row < t.nrows) {
        auto at = [&](int j) { return first + (int64_t)j * t.step + row; };
        write(row, col, join_few<D>(a.part_o, z, at, t.n, col));
      }
    } else {
      for (int row = 0; row < t.nrows; ++row) {
        const JoinedRow<D, Z> r = many.join(a.part_o, z, first + row, t.step, t.n, w, lane);
        if (w == 0 && lane < LPR) write(row, lane, r);
      }
    }
  }
}

}  // namespace

hipError_t launch_chunk_merge(const ChunkArgs& a, int head_dim, int is_bf16, hipStream_t s) {
  const int64_t units = (int64_t)a.max_joins * a.kv_heads;
  const int n = (int)(units < kMergeWgs ? units : kMergeWgs);
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
