// The work of a step of attention over a paged cache (chunk.hpp), laid out on the
// device from the sequences' lengths and the numbers of new tokens, gfx950.
//
// One workgroup: a scan of the requests' rows and tiles, the walks' total and
// longest, then the items.  Walks longer than a share of all of them (the walks of
// all KV heads by the workgroups to fill) are cut into equal chunks; the longer half
// of the items comes first.  The numbers do not depend on timing.
//
// Room.  With unit >= total / share, chunks beyond the first of each tile are at most
// sum floor((n - 1) / unit) < share, or, where the chunk limit is what cuts, tiles times
// what a table holds by the limit: the host makes that much room; a plan writes no more.
#include "chunk.hpp"

namespace bdlm {

namespace {

constexpr int kT = 1024;
constexpr int kLdsTiles = 8192;  // first tiles of that many requests are searched in LDS

template <class T>
__device__ __forceinline__ T block_scan(T x, T& total, T* wsum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  T v = x;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const T y = __shfl_up(v, s);
    if (lane >= s) v += y;
  }
  __syncthreads();  // (the sums of a scan before are read)
  if (lane == 63) wsum[w] = v;
  __syncthreads();
  T base = 0, t = 0;
#pragma unroll
  for (int k = 0; k < kT / 64; ++k) {
    const T y = wsum[k];
    if (k < w) base += y;
    t += y;
  }
  total = t;
  return base + v - x;
}

__device__ __forceinline__ int tile_rows(const ChunkPlanArgs& a, int64_t per) {
  return a.f32 ? kPrefixRowsF32 : per > 2 * kPrefixWaveRows ? kPrefixSharedRows : kPrefixWaveRows;
}

// A request: its first row, rows in the call, position of the first, tokens.
struct Request {
  int seq, token0, rows, pos0, len;
};
__device__ __forceinline__ Request request_of(const ChunkPlanArgs& a, int r, int start) {
  Request q;
  q.seq = a.seqs[r];
  if ((unsigned)q.seq >= (unsigned)a.seqs_in_cache) q.seq = -1;
  const int n = q.seq < 0 ? 0 : a.lens[q.seq], count = imax(a.counts[r], 0);
  q.len = n < 0 ? 0 : (int64_t)n > a.top ? (int)a.top : n;
  q.token0 = start;
  q.rows = imin(count, a.rows - start);
  q.pos0 = (int)((int64_t)q.len - count < -kBig ? -kBig : (int64_t)q.len - count);  // (then no row of the call sees anything)
  return q;
}

// A tile's walk.
struct Walk {
  int row0, nrows, n, gap_at, gap, w0;
};
__device__ __forceinline__ Walk walk_of(const ChunkPlanArgs& a, const Request& q, int tile) {
  const int64_t per = (int64_t)q.rows * a.group;
  const int tr = tile_rows(a, per);
  Walk w;
  w.row0 = tile * tr;
  w.nrows = imin(tr, (int)(per - w.row0));
  w.n = 0;
  w.gap_at = kBig;
  w.gap = w.w0 = 0;
  const int x0 = q.pos0 + w.row0 / a.group, x1 = q.pos0 + (w.row0 + w.nrows - 1) / a.group;
  if (x1 < 0) return w;
  const int end = imin(a.M * (x1 / a.M + 1), q.len);
  const int w0 = a.window > 0 ? imax(a.M * (imax(x0, 0) / a.M + 1) - a.window, 0) : 0;
  const int sinks = (imin(a.sinks, end) + 15) & ~15, first = w0 & ~15;
  w.n = end;
  w.w0 = w0;
  if (first > sinks) {
    w.gap_at = sinks;
    w.gap = first - sinks;
    w.w0 = w0 - w.gap;
    w.n = end > first ? sinks + end - first : imin(sinks, end);  // (blocks past the window's start: no key of it may be there)
  }
  return w;
}

__global__ __launch_bounds__(kT) void chunk_plan_kernel(const ChunkPlanArgs a) {
  __shared__ int tile0_lds[kLdsTiles];
  __shared__ int64_t wsum[kT / 64];
  __shared__ int longest_lds;
  const int tid = threadIdx.x;
  int32_t* const starts = a.plan + kChunkHead;
  int32_t* const tile0 = starts + a.requests;
  ChunkItemRec* const items = (ChunkItemRec*)(tile0 + a.requests + 1);
  ChunkJoin* const joins = (ChunkJoin*)(items + a.max_items);
  if (tid == 0) longest_lds = 0;

  // rows and tiles of the requests
  int64_t rows = 0, tiles = 0;
  for (int r0 = 0; r0 < a.requests; r0 += kT) {
    const int r = r0 + tid;
    const int64_t count = r < a.requests ? imax(a.counts[r], 0) : 0;
    int64_t all;
    const int64_t start = rows + block_scan(count, all, wsum);
    rows += all;
    const int first = start < a.rows ? (int)start : a.rows;
    const int64_t used = count < a.rows - first ? count : a.rows - first, per = used * a.group;
    const int tr = tile_rows(a, per);
    const int64_t at = tiles + block_scan((per + tr - 1) / tr, all, wsum);
    tiles += all;
    if (r < a.requests) {
      starts[r] = first;
      tile0[r] = (int)at;
      if (r < kLdsTiles) tile0_lds[r] = (int)at;
    }
  }
  if (tid == 0) tile0[a.requests] = (int)tiles;
  __syncthreads();
  const int T = (int)tiles;
  const bool in_lds = a.requests <= kLdsTiles;
  // The request of tile g: the last one whose first tile is not behind it.
  auto walk_at = [&](int g, Request& q) __attribute__((always_inline)) -> Walk {
    int lo = 0, hi = a.requests;  // tile0[lo] <= g < tile0[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((in_lds ? tile0_lds[mid] : tile0[mid]) <= g) lo = mid;
      else hi = mid;
    }
    q = request_of(a, lo, starts[lo]);
    return walk_of(a, q, g - (in_lds ? tile0_lds[lo] : tile0[lo]));
  };

  // what all walks come to, and the share of a workgroup
  int64_t mine = 0;
  int longest = 0;
  for (int g = tid; g < T; g += kT) {
    Request q;
    const int n = walk_at(g, q).n;
    mine += n;
    longest = imax(longest, n);
  }
  int64_t total;
  block_scan(mine, total, wsum);
  atomicMax(&longest_lds, longest);
  __syncthreads();
  longest = longest_lds;
  const int64_t share = (total * a.kv_heads + a.slots - 1) / a.slots;
  const int unit = (int)(share < a.least ? a.least : share > a.limit - 64 ? a.limit - 64 : share);
  const int half = imin(longest, unit) / 2;

  // the items, those longer than half of the longest first
  int64_t placed = 0, part_rows = 0;  // (items << 32 | cut tiles)
  for (int pass = 0; pass < 2; ++pass)
    for (int g0 = 0; g0 < T; g0 += kT) {
      const int g = g0 + tid;
      Request q;
      Walk w{};
      int n = 0, size = 0;
      if (g < T) {
        w = walk_at(g, q);
        const int cut = imax((w.n + unit - 1) / unit, 1);
        size = imax(((w.n + cut - 1) / cut + 63) & ~63, 64);
        n = imax((w.n + size - 1) / size, 1);
        if ((imin(size, w.n) > half) != (pass == 0)) n = 0;
      }
      int64_t all;
      const int64_t at = placed + block_scan((int64_t)n << 32 | (n > 1), all, wsum);
      placed += all;
      int64_t part = part_rows + block_scan((int64_t)(n > 1 ? n * w.nrows : 0), all, wsum);
      part_rows += all;
      if (n == 0) continue;
      const int i0 = (int)(at >> 32), j = (int)(at & 0xffffffff);
      const bool shared = !a.f32 && w.row0 + w.nrows > 0 && tile_rows(a, (int64_t)q.rows * a.group) == kPrefixSharedRows;
      if (i0 + (int64_t)n > a.max_items || (n > 1 && (j >= a.max_joins || part + (int64_t)n * w.nrows > a.max_part_rows)))
        continue;  // (never: the host made room)
      for (int c = 0; c < n; ++c) {
        ChunkItemRec x;
        x.seq = q.seq;
        x.token0 = q.token0;
        x.pos0 = q.pos0;
        x.len = q.len;
        x.row0 = w.row0;
        x.nrows = w.nrows;
        x.k0 = c * size;
        x.k1 = imin((c + 1) * size, w.n);
        x.gap_at = w.gap_at;
        x.gap = w.gap;
        x.w0 = w.w0;
        x.part = n > 1 ? (int)part + c * w.nrows | (shared ? kSharedTile : 0) : ~(shared ? kSharedTile : 0);
        items[i0 + c] = x;
      }
      if (n > 1) joins[j] = ChunkJoin{q.token0, w.row0, w.nrows, (int)part, n, 0, 0, 0};
    }
  if (tid == 0) {
    a.plan[kPlanItems] = (int)(placed >> 32);
    a.plan[kPlanJoins] = (int)(placed & 0xffffffff);
    a.plan[kPlanRows] = (int)(rows < a.rows ? rows : a.rows);
  }
}

}  // namespace

hipError_t launch_chunk_plan(const ChunkPlanArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kT), 0, s, a);
  return hipGetLastError();
}

}  // namespace bdlm
