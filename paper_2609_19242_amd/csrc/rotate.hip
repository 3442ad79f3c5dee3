// Norms of queries and keys for each head with the position rotation in the
// same pass, forward and backward, bf16 and fp32, gfx950.
//
// For a head's row x of D elements with weight w, at positions p_a, with pair i
// of the first `dim` elements on axis a(i) turning by t_i = p_a(i) f_i:
//   r = 1 / sqrt(mean x^2 + eps),  n = x r w  (no norm: n = x),
//   y = n, its pairs (n1, n2) turned to (n1 cos t - n2 sin t, n2 cos t + n1 sin t).
// Backward, with g = dy turned by -t and h = g w:
//   dw = sum over rows and heads of g x r,  dx = r (h - x r mean(h x r)).
// r is formed again from x, which backward reads in any case: nothing is saved.
//
// Bound by memory.  D / 16 lanes hold a head's row, 16 elements each in two runs
// of 8 (16 bytes in bf16): pair partners lie in the same lane (halves D / 2
// apart, or neighbours), so that the rotation needs no exchange, and a pass of a
// wave reads whole 128-byte lines.  A lane forms its 8 cosines and sines once per
// row and keeps them for all passes over the row's heads.
//
// Rounding.  An angle is position times frequency in 64 bits, in quarter turns,
// reduced there to half a quarter; sine and cosine of the rest in fp32 by their
// Taylor series to x^9 and x^10 (|x| <= pi / 4: the rest of the series is below
// 2^-28).  bf16: the sum of squares and all products are fp32 (so squares must stay
// below 2^127: |x| < 2^60), the outputs are rounded once.  fp32: the sums over a row
// are fp64.  dw: fp32 sums of a lane's rows, a wave's and a workgroup's lanes in a
// fixed order, the workgroups' in fp64; it is returned in fp32.
#include "device.hpp"
#include "rotate.hpp"

namespace bdlm {

namespace {

constexpr int kWaves = 4;

// 8 consecutive elements.
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_bf16(x[e]);
  *(bf16x8*)p = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// The type of sums over a head's row.
template <class T> struct SumOf { typedef float type; };
template <> struct SumOf<float> { typedef double type; };

__device__ __forceinline__ float shfl_x(float x, int m) { return __shfl_xor(x, m); }
__device__ __forceinline__ double shfl_x(double x, int m) { return __shfl_xor(x, m); }
template <int LPR, class S>
__device__ __forceinline__ S row_sum(S x) {
#pragma unroll
  for (int m = 1; m < LPR; m <<= 1) x += shfl_x(x, m);
  return x;
}

__device__ __forceinline__ float inverse_root(float x) { return __builtin_amdgcn_rsqf(x); }
__device__ __forceinline__ float inverse_root(double x) { return (float)(1.0 / sqrt(x)); }

// Cosine and sine of `u` quarter turns.
__device__ __forceinline__ void turn_of(double u, float& c, float& s) {
  const double n = __builtin_rint(u);
  const float x = (float)(u - n) * 1.57079632679489661923f, x2 = x * x;
  const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;
  c = (q + 1) & 2 ? -a : a;
  s = q & 2 ? -b : b;
}

// Where a lane's two runs of 8 elements lie in a head's row.
template <bool IL>
__device__ __forceinline__ void runs_of(int l, int dim, int& a, int& b) {
  const bool halves = !IL && 16 * l < dim;
  a = halves ? 8 * l : 16 * l;
  b = halves ? dim / 2 + 8 * l : 16 * l + 8;
}

// The lane's pairs turned (by -t: `back`).
template <bool IL>
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8], bool back) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& x = IL ? (j < 4 ? a[2 * j] : b[2 * j - 8]) : a[j];
    float& y = IL ? (j < 4 ? a[2 * j + 1] : b[2 * j - 7]) : b[j];
    const float sn = back ? -s[j] : s[j], u = x, v = y;
    x = fmaf(u, c[j], -(v * sn));
    y = fmaf(v, c[j], u * sn);
  }
}

// What a lane knows of the wave's rows: its row's cosines and sines.
template <int D, bool IL>
struct Lane {
  static constexpr int LPR = D / 16, HPG = 64 / LPR;
  int l, ra, rb, sub, head, heads;  // lane of its head's row; runs; row of the wave's; first head, heads side by side
  int64_t row;
  bool ok;
  float c[8], s[8];
  __device__ __forceinline__ Lane(const RotateArgs& a, int lane) {
    l = lane % LPR;
    runs_of<IL>(l, a.dim, ra, rb);
    heads = HPG / a.rows_per;
    sub = lane / LPR / heads;
    head = lane / LPR % heads;
  }
  __device__ __forceinline__ void seek(const RotateArgs& a, int64_t set) {
    row = set * a.rows_per + sub;
    ok = row < a.rows;
    if (!ok) row = a.rows - 1;
    if (16 * l < a.dim) {
      if (a.axes == 1) {
        const double p = (double)a.pos[row];
#pragma unroll
        for (int j = 0; j < 8; ++j) turn_of(p * a.quarters[8 * l + j], c[j], s[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          turn_of((double)a.pos[a.axis[8 * l + j] * a.rows + row] * a.quarters[8 * l + j], c[j], s[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 1.f, s[j] = 0.f;
    }
  }
};

template <class T>
__device__ __forceinline__ void load_weight(const RotateTensor& t, int ra, int rb, float (&wa)[8], float (&wb)[8]) {
  if (t.w) {
    load8((const T*)t.w + ra, wa);
    load8((const T*)t.w + rb, wb);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) wa[e] = wb[e] = 1.f;
  }
}

template <class T, int D, bool IL, bool NORM>
__global__ __launch_bounds__(kWaves * 64) void rotate_fwd_kernel(const RotateArgs a) {
  using S = typename SumOf<T>::type;
  const int lane = threadIdx.x & 63;
  Lane<D, IL> me(a, lane);
  const int64_t sets = (a.rows + a.rows_per - 1) / a.rows_per;
  const int64_t first = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t n = first; n < sets * a.split; n += (int64_t)gridDim.x * kWaves) {
    const int64_t set = n / a.split;
    const int part = (int)(n - set * a.split);
    me.seek(a, set);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const RotateTensor& t = a.t[i];
      float wa[8], wb[8];
      if constexpr (NORM) load_weight<T>(t, me.ra, me.rb, wa, wb);
      // (the keys' passes follow the queries' in the deal)
      for (int p = i == 0 ? part : (part - a.t[0].passes % a.split + a.split) % a.split; p < t.passes; p += a.split) {
        const int h = p * me.heads + me.head;
        const bool mine = me.ok && h < t.heads;
        const int64_t at = me.row * t.xs + (int64_t)(mine ? h : 0) * D;
        float x[8], y[8];
        load8((const T*)t.x + at + me.ra, x);
        load8((const T*)t.x + at + me.rb, y);
        if constexpr (NORM) {
          S ss = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += (S)x[e] * (S)x[e] + (S)y[e] * (S)y[e];
          ss = row_sum<D / 16>(ss);
          const float r = inverse_root(ss * (S)(1.0 / D) + (S)a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = x[e] * r * wa[e];
            y[e] = y[e] * r * wb[e];
          }
        }
        turn<IL>(x, y, me.c, me.s, false);
        if (mine) {
          T* o = (T*)t.out + me.row * t.outs + (int64_t)h * D;
          store8(o + me.ra, x);
          store8(o + me.rb, y);
        }
      }
    }
  }
}

template <class T, int D, bool IL, bool NORM>
__global__ __launch_bounds__(kWaves * 64) void rotate_bwd_kernel(const RotateArgs a) {
  using S = typename SumOf<T>::type;
  constexpr int LPR = D / 16;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Lane<D, IL> me(a, lane);
  const int64_t sets = (a.rows + a.rows_per - 1) / a.rows_per;
  float dw[2][16];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f;
  for (int64_t n = (int64_t)blockIdx.x * kWaves + w; n < sets * a.split; n += (int64_t)gridDim.x * kWaves) {
    const int64_t set = n / a.split;
    const int part = (int)(n - set * a.split);
    me.seek(a, set);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const RotateTensor& t = a.t[i];
      float wa[8], wb[8];
      if constexpr (NORM) load_weight<T>(t, me.ra, me.rb, wa, wb);
      for (int p = i == 0 ? part : (part - a.t[0].passes % a.split + a.split) % a.split; p < t.passes; p += a.split) {
        const int h = p * me.heads + me.head;
        const bool mine = me.ok && h < t.heads;
        const int64_t head = (int64_t)(mine ? h : 0) * D;
        float g[8], k[8], x[8], y[8];
        if constexpr (NORM) {
          load8((const T*)t.x + me.row * t.xs + head + me.ra, x);
          load8((const T*)t.x + me.row * t.xs + head + me.rb, y);
        }
        load8((const T*)t.dy + me.row * t.dys + head + me.ra, g);
        load8((const T*)t.dy + me.row * t.dys + head + me.rb, k);
        turn<IL>(g, k, me.c, me.s, true);
        if constexpr (NORM) {
          S ss = 0, hx = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss += (S)x[e] * (S)x[e] + (S)y[e] * (S)y[e];
            hx += (S)(g[e] * wa[e]) * (S)x[e] + (S)(k[e] * wb[e]) * (S)y[e];
          }
          ss = row_sum<LPR>(ss);
          hx = row_sum<LPR>(hx);
          const float r = inverse_root(ss * (S)(1.0 / D) + (S)a.eps);
          const float m = (float)(hx * (S)(1.0 / D) * (S)r);  // mean(h x r)
          if (mine) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              dw[i][e] = fmaf(g[e], x[e] * r, dw[i][e]);
              dw[i][8 + e] = fmaf(k[e], y[e] * r, dw[i][8 + e]);
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            g[e] = r * fmaf(-(x[e] * r), m, g[e] * wa[e]);
            k[e] = r * fmaf(-(y[e] * r), m, k[e] * wb[e]);
          }
        }
        if (mine) {
          T* o = (T*)t.out + me.row * t.outs + head;
          store8(o + me.ra, g);
          store8(o + me.rb, k);
        }
      }
    }
  }
  if constexpr (NORM) {
    if (!a.partials) return;
    // the lanes that hold the same elements, then the waves, in a fixed order
    __shared__ float sums[kWaves][2][D];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
#pragma unroll
        for (int m = LPR; m < 64; m <<= 1) dw[i][e] += __shfl_xor(dw[i][e], m);
        if (lane < LPR) sums[w][i][(e < 8 ? me.ra : me.rb) + (e & 7)] = dw[i][e];
      }
    __syncthreads();
    for (int n = threadIdx.x; n < 2 * D; n += kWaves * 64) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) x += sums[k][n / D][n % D];
      a.partials[(int64_t)blockIdx.x * 2 * D + n] = x;
    }
  }
}

// The workgroups' sums added up: 16 columns a workgroup, 64 rows of partials at a time.
template <int D>
__global__ __launch_bounds__(1024) void rotate_dw_kernel(const RotateArgs a) {
  __shared__ double sums[64][16];
  const int col = threadIdx.x & 15, at = threadIdx.x >> 4, n = blockIdx.x * 16 + col;
  double x = 0.0;
  for (int r = at; r < a.wgs; r += 64) x += (double)a.partials[(int64_t)r * 2 * D + n];
  sums[at][col] = x;
  __syncthreads();
  if (at == 0) {
    for (int k = 1; k < 64; ++k) x += sums[k][col];
    float* const dw = a.dw[n / D];
    if (dw) dw[n % D] = (float)x;
  }
}

template <class T, int D, bool IL>
void launch(const RotateArgs& a, bool bwd, hipStream_t s) {
  const dim3 grid(a.wgs), threads(kWaves * 64);
  const bool norm = a.eps > 0;
  if (!bwd) {
    if (norm) hipLaunchKernelGGL((rotate_fwd_kernel<T, D, IL, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((rotate_fwd_kernel<T, D, IL, false>), grid, threads, 0, s, a);
    return;
  }
  if (a.wgs == 0) {  // (no rows: zeros)
  } else if (norm) hipLaunchKernelGGL((rotate_bwd_kernel<T, D, IL, true>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((rotate_bwd_kernel<T, D, IL, false>), grid, threads, 0, s, a);
  if (a.partials) hipLaunchKernelGGL((rotate_dw_kernel<D>), dim3(2 * D / 16), dim3(1024), 0, s, a);
}
template <class T, int D>
void launch(const RotateArgs& a, int il, bool bwd, hipStream_t s) {
  il ? launch<T, D, true>(a, bwd, s) : launch<T, D, false>(a, bwd, s);
}
hipError_t launch(const RotateArgs& a, int head_dim, int is_bf16, int il, bool bwd, hipStream_t s) {
  if (is_bf16) head_dim == 128 ? launch<bf16, 128>(a, il, bwd, s) : launch<bf16, 64>(a, il, bwd, s);
  else head_dim == 128 ? launch<float, 128>(a, il, bwd, s) : launch<float, 64>(a, il, bwd, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate_fwd(const RotateArgs& a, int head_dim, int is_bf16, int interleaved, hipStream_t s) {
  return launch(a, head_dim, is_bf16, interleaved, false, s);
}
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, int is_bf16, int interleaved, hipStream_t s) {
  return launch(a, head_dim, is_bf16, interleaved, true, s);
}

}  // namespace bdlm
