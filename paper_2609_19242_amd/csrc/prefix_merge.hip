// The chunks' partial outputs of attention over a paged cache (cache.hpp)
// added up, gfx950: with z_j the log2-sum-exp of chunk j of a row,
//   m = max z_j,  w_j = 2^(z_j - m),  O = sum w_j O_j / sum w_j,
//   LSE = ln 2 (m + log2 sum w_j)
// in fp32, chunk by chunk in order: the same sums on every run.  Chunks that a
// row does not see (z_j = -inf) are not read.  A wave per row, a lane per D / 64
// elements.  Bound by reading the partials (mostly from L2).
#include "cache.hpp"
#include "device.hpp"

namespace bdlm {

namespace {

constexpr float kLn2 = 0.69314718055994530942f;

template <int D, bool BF16>
__global__ __launch_bounds__(256) void prefix_merge_kernel(const PrefixArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t total = (int64_t)a.requests * a.rows * a.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= total) return;
  const int parts = a.prefix_chunks + a.own_chunks;
  float m = -INFINITY;
  for (int j = lane; j < parts; j += 64) m = fmaxf(m, a.part_lse[j * total + row]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
  float sum = 0.f, x[E] = {};
  if (m > -INFINITY) {
    for (int j = 0; j < parts; ++j) {
      const float z = a.part_lse[j * total + row];
      if (z == -INFINITY) continue;
      const float w = exp2f_fast(z - m);
      sum += w;
      const float* p = a.part_o + (j * total + row) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(w, p[e], x[e]);
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (BF16) ((bf16*)a.o)[row * D + lane * E + e] = to_bf16(x[e] * inv);
    else ((float*)a.o)[row * D + lane * E + e] = x[e] * inv;
  }
  if (lane == 0) {
    PrefixRow pr;
    pr.token = (int)(row / a.heads);
    pr.head = (int)(row - (int64_t)pr.token * a.heads);
    pr.end = 0;
    a.lse[prefix_lse_at(a, pr)] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
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
