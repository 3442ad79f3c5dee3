// Partial outputs of attention over disjoint sets of keys, joined: with z_j the
// log2-sum-exp of part j of a row and O_j its normalised output,
//   m = max z_j,  w_j = 2^(z_j - m),  O = sum w_j O_j / sum w_j,
//   LSE = ln 2 (m + log2 sum w_j)
// in an order that depends on the number of parts only.  Sums, weights and z_j are
// fp32 (Z = float) for bf16 outputs.  For fp32 ones they are fp64: a z rounded to fp32
// is off by 2^-24 |z|, and so is the weight, relatively (z = 720, scores around 500:
// O off by 2e-5, 8 to 11 times its bound); the O_j, off by 2^-24 |O_j| at most once,
// stay fp32, half the bytes.  Parts that a
// row does not see (z_j = -inf) have left no output; what lies there takes no part.
// D / 4 lanes hold 16 bytes each of a part's output, four parts' loads in flight.
// Many parts: a wave per row takes 256 / D at a time.  Few (kFewParts on the
// average): a row per D / 4 lanes, which need no exchange (16,384 rows of 4 parts,
// d 128: 10.7 -> 8.1 us; 3,000 rows of 4/2 heads in 4 parts 7.4 -> 5.5).
#pragma once

#include "common.hpp"
#include "device.hpp"
#include "f64tile.hpp"

namespace bdlm {

constexpr int kFewParts = 16;

template <class Z>
using Joined4 = Z __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float pow2(float x) { return exp2f_fast(x); }
__device__ __forceinline__ double pow2(double x) { return exp2_f64(x); }
__device__ __forceinline__ float lse_of(float m, float sum) { return (m + log2f(sum)) * 0.69314718055994530942f; }
__device__ __forceinline__ float lse_of(double m, double sum) { return (float)((m + log2(sum)) * kLn2D); }
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double max_of(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float fma_of(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double fma_of(double a, double b, double c) { return __builtin_fma(a, b, c); }
__device__ __forceinline__ float xor_of(float x, int m) { return __shfl_xor(x, m); }
__device__ __forceinline__ double xor_of(double x, int m) { return shfl_xor_d(x, m); }

template <int D, class Z = float>
struct JoinedRow {
  static constexpr int LPR = D / 4;  // lanes per part
  Joined4<Z> x;   // this lane's columns 4 (lane % LPR) .. + 3, in the lanes < LPR
  float lse;
};
template <int D, class Z>
__device__ __forceinline__ JoinedRow<D, Z> joined(Joined4<Z> x, Z m, Z sum) {
  JoinedRow<D, Z> r;
  r.x = x * (sum > Z(0) ? Z(1) / sum : Z(0));
  r.lse = sum > Z(0) ? lse_of(m, sum) : -INFINITY;
  return r;
}

// A row per LPR lanes; every lane has the LSE.
template <int D, class Z, class At>
__device__ __forceinline__ JoinedRow<D, Z> join_few(const float* o, const Z* z, At at, int parts, int lane) {
  const int col = lane % JoinedRow<D>::LPR;
  Z m = -INFINITY, sum = 0;
  Joined4<Z> x = {0, 0, 0, 0};
  for (int j0 = 0; j0 < parts; j0 += 4) {
    Z zz[4];
    f32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t row = at(imin(j0 + k, parts - 1));
      zz[k] = j0 + k < parts ? z[row] : Z(-INFINITY);
      p[k] = *(const f32x4*)(o + row * D + col * 4);
    }
    const Z mn = max_of(max_of(max_of(zz[0], zz[1]), max_of(zz[2], zz[3])), m), ref = mn == -INFINITY ? Z(0) : mn;
    const Z al = pow2(m - ref);  // (0 before the first part seen)
    sum *= al;
    x *= al;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool seen = zz[k] > -INFINITY;
      const Z w = seen ? pow2(zz[k] - ref) : Z(0);
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = seen ? fma_of(w, Z(p[k][e]), x[e]) : x[e];
    }
    m = mn;
  }
  return joined<D, Z>(x, m, sum);
}

// A wave per row.  at(j): row of part j in `o` ([row][D]) and `z`.
template <int D, class Z, class At>
__device__ __forceinline__ JoinedRow<D, Z> join_partials(const float* o, const Z* z, At at, int parts, int lane) {
  constexpr int LPR = JoinedRow<D>::LPR, PP = 64 / LPR;  // lanes per part, parts at a time
  const int part = lane / LPR, col = lane % LPR;
  Z m = -INFINITY;
  for (int j = lane; j < parts; j += 64) m = max_of(m, z[at(j)]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) m = max_of(m, xor_of(m, s));
  const Z ref = m == -INFINITY ? Z(0) : m;
  Z sum = 0;
  Joined4<Z> x = {0, 0, 0, 0};
  for (int base = 0; base < parts; base += 4 * PP) {
    Z zz[4];
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
      const Z w = seen ? pow2(zz[k] - ref) : Z(0);
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = seen ? fma_of(w, Z(p[k][e]), x[e]) : x[e];
    }
  }
#pragma unroll
  for (int s = LPR; s < 64; s <<= 1) {
    sum += xor_of(sum, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += xor_of(x[e], s);
  }
  return joined<D, Z>(x, m, sum);
}

}  // namespace bdlm
