// Partial outputs of attention over disjoint sets of keys, joined: with z_j the
// log2-sum-exp of part j of a row and O_j its normalised output,
//   m = max z_j,  w_j = 2^(z_j - m),  O = sum w_j O_j / sum w_j,
//   LSE = ln 2 (m + log2 sum w_j)
// in fp32, in an order that depends on the number of parts only.  Parts that a
// row does not see (z_j = -inf) have left no output; what lies there takes no part.
// D / 4 lanes hold 16 bytes each of a part's output, four parts' loads in flight.
// Many parts: a wave per row takes 256 / D at a time.  Few (kFewParts on the
// average): a row per D / 4 lanes, which need no exchange (16,384 rows of 4 parts,
// d 128: 10.7 -> 8.1 us; 3,000 rows of 4/2 heads in 4 parts 7.4 -> 5.5).
#pragma once

#include "common.hpp"
#include "device.hpp"

namespace bdlm {

constexpr int kFewParts = 16;

template <int D>
struct JoinedRow {
  static constexpr int LPR = D / 4;  // lanes per part
  f32x4 x;   // this lane's columns 4 (lane % LPR) .. + 3, in the lanes < LPR
  float lse;
};
template <int D>
__device__ __forceinline__ JoinedRow<D> joined(f32x4 x, float m, float sum) {
  JoinedRow<D> r;
  r.x = x * (sum > 0.f ? 1.f / sum : 0.f);
  r.lse = sum > 0.f ? (m + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
  return r;
}

// A row per LPR lanes; every lane has the LSE.
template <int D, class At>
__device__ __forceinline__ JoinedRow<D> join_few(const float* o, const float* z, At at, int parts, int lane) {
  const int col = lane % JoinedRow<D>::LPR;
  float m = -INFINITY, sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < parts; j0 += 4) {
    float zz[4];
    f32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t row = at(imin(j0 + k, parts - 1));
      zz[k] = j0 + k < parts ? z[row] : -INFINITY;
      p[k] = *(const f32x4*)(o + row * D + col * 4);
    }
    const float mn = fmaxf(fmaxf(fmaxf(zz[0], zz[1]), fmaxf(zz[2], zz[3])), m), ref = mn == -INFINITY ? 0.f : mn;
    const float al = exp2f_fast(m - ref);  // (0 before the first part seen)
    sum *= al;
    x *= al;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool seen = zz[k] > -INFINITY;
      const float w = seen ? exp2f_fast(zz[k] - ref) : 0.f;
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = seen ? fmaf(w, p[k][e], x[e]) : x[e];
    }
    m = mn;
  }
  return joined<D>(x, m, sum);
}

// A wave per row.  at(j): row of part j in `o` ([row][D]) and `z`.
template <int D, class At>
__device__ __forceinline__ JoinedRow<D> join_partials(const float* o, const float* z, At at, int parts, int lane) {
  constexpr int LPR = JoinedRow<D>::LPR, PP = 64 / LPR;  // lanes per part, parts at a time
  const int part = lane / LPR, col = lane % LPR;
  float m = -INFINITY;
  for (int j = lane; j < parts; j += 64) m = fmaxf(m, z[at(j)]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float ref = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < parts; base += 4 * PP) {
    float zz[4];
    f32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (base + k * PP >= parts) break;
      const int64_t row = at(imin(base + k * PP + part, parts - 1));
      zz[k] = z[row];
      p[k] = *(const f32x4*)(o + row * D + col * 4);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (base + k * PP >= parts) break;
      const bool seen = base + k * PP + part < parts && zz[k] > -INFINITY;
      const float w = seen ? exp2f_fast(zz[k] - ref) : 0.f;
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = seen ? fmaf(w, p[k][e], x[e]) : x[e];
    }
  }
#pragma unroll
  for (int s = LPR; s < 64; s <<= 1) {
    sum += __shfl_xor(sum, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], s);
  }
  return joined<D>(x, m, sum);
}

}  // namespace bdlm
