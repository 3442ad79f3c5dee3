// The work of a step of attention over a paged cache (chunk.hpp), laid out on the
// device from the sequences' lengths and the numbers of new tokens, gfx950.
//
// One workgroup: a scan of the requests' rows and tiles, the walks' lengths, the
// unit, then the items.  Walks longer than the unit are cut into equal chunks; the
// longer half of the items comes first, and each half from behind, since a prompt's later
// tiles have longer walks (a prompt of 8,000 tokens, 32/8 heads: 547 -> 514 us, 48 decoding
// requests with 3 pieces of prompts 186 -> 156).  The numbers do not depend on timing.
// Bound by latency: the chain count, sequence, length, then three passes over the tiles,
// 7 us for 5 requests, 9 for 200.
//
// The unit.  Half of a workgroup's share of all walks to twice as much, in 32 steps:
// the one with the least cost in keys, which is the longer of (rounds of longer items
// times their size) and the share, and a start-up per item and what the partial sums
// cost (4 x D bytes written and read per row, at 4.5 TB/s against 40 ns per key).  Rounds are
// what matters: 4 requests of 64 rows behind 16,000 tokens, cut by the share alone,
// came to 544 items for 512 places.
//
// Room.  With unit >= total / (2 slots / KV heads), chunks beyond the first of each tile
// are at most sum floor((n - 1) / unit) <= 2 slots / KV heads, or, where the chunk limit is
// what cuts, tiles times what a table holds by the limit, and never more than tiles times a
// walk's keys by the least unit: the host makes that much room, and launches no merge where
// no walk can be that long.
#include "chunk.hpp"
#include "device.hpp"

namespace bdlm {

namespace {

constexpr int kT = 512;
constexpr int kLdsRequests = 2048;  // requests that are kept in LDS (more are read again)
constexpr int kLdsTiles = 2048;     // tiles for which the unit is looked for (with more, the share)
constexpr int kUnits = 32;
constexpr float kStartKeys = 64.f;  // a workgroup's start-up
constexpr float kPartRows = 176.f;  // partial rows that take as long as a key of a slot

// A value from a lane before this one, 0 where there is none (row_shr by 1 to 8 within
// 16 lanes; the last lane of a row of 16, of 32, to those behind): no way through LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ int before(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t before(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)before<CTRL, ROWS>((int)(x >> 32)) << 32 | (uint32_t)before<CTRL, ROWS>((int)x));
}
// x of this lane and those before it, joined (0 is neutral); lane 63 has the wave's.
template <class T, class F>
__device__ __forceinline__ T wave_scan(T x, F&& join) {
  x = join(x, before<0x111, 0xf>(x));
  x = join(x, before<0x112, 0xf>(x));
  x = join(x, before<0x114, 0xf>(x));
  x = join(x, before<0x118, 0xf>(x));
  x = join(x, before<0x142, 0xa>(x));
  return join(x, before<0x143, 0xc>(x));
}
template <class T>
__device__ __forceinline__ T add(T a, T b) { return a + b; }
// Exclusive prefix sums over the workgroup's threads, and the total.  (Between two with the same wsum lies a barrier.)
template <class T>
__device__ __forceinline__ T block_scan(T x, T& all, int64_t* wsum) {
  const int w = threadIdx.x >> 6;
  const T up_to = wave_scan(x, add<T>);
  if ((threadIdx.x & 63) == 63) wsum[w] = up_to;
  __syncthreads();
  T first = 0;
  all = 0;
#pragma unroll
  for (int k = 0; k < kT / 64; ++k) {
    const T a = (T)wsum[k];
    if (k < w) first += a;
    all += a;
  }
  return first + up_to - x;
}

__device__ __forceinline__ int tile_rows(const ChunkPlanArgs& a, int per) {
  return a.f32 ? kPrefixRowsF32 : per > 2 * kPrefixWaveRows ? kPrefixSharedRows : kPrefixWaveRows;
}
// x / n for the uniform n of a call, mostly 1 or a power of two (x >= 0).
__device__ __forceinline__ int over(int x, int n) { return (n & (n - 1)) == 0 ? x >> __builtin_ctz(n) : x / n; }

// A request: its first tile, its first row and rows in the call, the position of the first, tokens.
struct Request {
  int tile0, token0, rows, pos0, len, seq;
};
// The sequence of request r, its tokens and new ones.
__device__ __forceinline__ void load_request(const ChunkPlanArgs& a, int r, Request& q, int& count) {
  count = imax(a.counts[r], 0);
  q.seq = a.seqs[r];
  if ((unsigned)q.seq >= (unsigned)a.seqs_in_cache) q.seq = -1;
  const int n = q.seq < 0 ? 0 : a.lens[q.seq];
  q.len = n < 0 ? 0 : (int64_t)n > a.top ? (int)a.top : n;
  const int64_t pos0 = (int64_t)q.len - count;
  q.pos0 = pos0 < -kBig ? -kBig : (int)pos0;  // (then no row of the call sees anything)
}
__device__ __forceinline__ void place_request(const ChunkPlanArgs& a, int64_t start, int count, Request& q) {
  q.token0 = start < a.rows ? (int)start : a.rows;
  q.rows = imin(count, a.rows - q.token0);
}

// A tile's walk.
struct Walk {
  int row0, nrows, n, gap_at, gap, w0;
  bool shared;
};
__device__ __forceinline__ Walk walk_of(const ChunkPlanArgs& a, const Request& q, int tile) {
  const int per = q.rows * a.group, tr = tile_rows(a, per);
  Walk w;
  w.shared = tr == kPrefixSharedRows;
  w.row0 = tile * tr;
  w.nrows = imin(tr, per - w.row0);
  w.n = 0;
  w.gap_at = kBig;
  w.gap = w.w0 = 0;
  const int x0 = q.pos0 + over(w.row0, a.group), x1 = q.pos0 + over(w.row0 + w.nrows - 1, a.group);
  if (x1 < 0) return w;
  const int end = imin(a.M * (over(x1, a.M) + 1), q.len);
  const int w0 = a.window > 0 ? imax(a.M * (over(imax(x0, 0), a.M) + 1) - a.window, 0) : 0;
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
  __shared__ int req[6][kLdsRequests];
  __shared__ int64_t wsum[2][kT / 64];
  __shared__ int tile_n[kLdsTiles], tile_nrows[kLdsTiles];
  __shared__ unsigned long long total_lds;
  __shared__ int longest_lds, short_lds;  // (short: whether the room does not hold all)
  __shared__ f32x4 sums[kT / kUnits][kUnits];
  __shared__ int best_lds;
  const int tid = threadIdx.x;
  int32_t* const starts = a.plan + kChunkHead;
  int32_t* const tile0 = starts + a.requests;
  ChunkItemRec* const items = (ChunkItemRec*)(tile0 + a.requests + 1);
  ChunkJoin* const joins = (ChunkJoin*)(items + a.max_items);
  if (tid == 0) longest_lds = 0, short_lds = 0, total_lds = 0;

  // the requests' rows and tiles
  int64_t rows = 0;
  int tiles = 0;
#pragma unroll 1
  for (int r0 = 0; r0 < a.requests; r0 += kT) {
    const int r = r0 + tid;
    Request q;
    int count = 0;
    if (r < a.requests) load_request(a, r, q, count);
    int64_t all;
    const int64_t start = block_scan((int64_t)count, all, wsum[0]);
    place_request(a, rows + start, count, q);
    rows += all;
    const int per = q.rows * a.group, tr = tile_rows(a, per);
    int all_tiles;
    q.tile0 = tiles + block_scan(over(per + tr - 1, tr), all_tiles, wsum[1]);
    tiles += all_tiles;
    if (r < a.requests) {
      starts[r] = q.token0;
      tile0[r] = q.tile0;
      if (r < kLdsRequests) {
        req[0][r] = q.tile0;
        req[1][r] = q.token0;
        req[2][r] = q.rows;
        req[3][r] = q.pos0;
        req[4][r] = q.len;
        req[5][r] = q.seq;
      }
    }
  }
  if (tid == 0) tile0[a.requests] = tiles;
  __syncthreads();
  const int T = tiles;
  const bool in_lds = a.requests <= kLdsRequests;
  // Tile g of all: its request is the last one whose first tile is not behind it.
  auto walk_at = [&](int g, Request& q) __attribute__((always_inline)) -> Walk {
    int lo = 0, hi = a.requests;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((in_lds ? req[0][mid] : tile0[mid]) <= g) lo = mid;
      else hi = mid;
    }
    if (in_lds) {
      q = Request{req[0][lo], req[1][lo], req[2][lo], req[3][lo], req[4][lo], req[5][lo]};
    } else {
      int count;
      load_request(a, lo, q, count);
      place_request(a, starts[lo], count, q);
      q.tile0 = tile0[lo];
    }
    return walk_of(a, q, g - q.tile0);
  };

  // 0: what all walks come to, and the longest; 1 (more tiles than threads): items, and those
  // of the longer half of the walks; 2: the items, those first.
  int unit = 0, half = 0;
  int64_t total = 0;
  int longest = 0;
  int64_t all_items = 0, placed = 0, parts = 0;  // (longer items << 32 | others; cut tiles << 32 | their partial rows)
  Request q{};
  Walk w{};
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    if (pass == 1 && T <= kT) continue;
#pragma unroll 1
    for (int g0 = 0; g0 < T; g0 += kT) {
      const int g = g0 + tid;
      if (g < T && (pass == 0 || T > kT)) w = walk_at(g, q);
      if (pass == 0) {
        if (g < T) {
          total += w.n;
          longest = imax(longest, w.n);
          if (T <= kLdsTiles) tile_n[g] = w.n, tile_nrows[g] = w.nrows;
        }
        continue;
      }
      int n = 0, size = 0;
      if (g < T) {
        const int cut = imax(over(w.n + unit - 1, unit), 1);
        size = imax((over(w.n + cut - 1, cut) + 63) & ~63, 64);
        n = imax(over(w.n + size - 1, size), 1);
      }
      const bool is_longer = imin(size, w.n) > half;
      // units of the merge: a row each where there are many parts
      const int join = n > kShortJoin ? 1 : a.join_rows, units = n > 1 ? (w.nrows + join - 1) / join : 0;
      int64_t all_x, all_y;
      if (T > kT) __syncthreads();
      int64_t x = block_scan(is_longer ? (int64_t)n << 32 : n, all_x, wsum[0]);
      if (pass == 1) {
        all_items += all_x;
        continue;
      }
      if (T <= kT) all_items = all_x;
      const int64_t y = parts + block_scan(n > 1 ? (int64_t)units << 32 | n * w.nrows : (int64_t)0, all_y, wsum[1]);
      x += placed;
      placed += all_x;
      parts += all_y;
      // (from behind: a prompt's later tiles are longer)
      const int longer = (int)(all_items >> 32), others = (int)(all_items & 0xffffffff), j = (int)(y >> 32);
      const int i0 = (is_longer ? longer - (int)(x >> 32) : longer + others - (int)(x & 0xffffffff)) - n;
      const int64_t part = y & 0xffffffff;
      // (never: the host made room; else there is no plan, below)
      if (i0 < 0 || i0 + (int64_t)n > a.max_items || (n > 1 && (j + units > a.max_joins || part + (int64_t)n * w.nrows > a.max_part_rows))) {
        short_lds = 1;
        continue;
      }
      ChunkItemRec rec{q.seq, q.token0, q.pos0, q.len, w.row0, w.nrows, 0, 0, w.gap_at, w.gap, w.w0, 0};
      const int flag = w.shared ? kSharedTile : 0;
#pragma unroll 1
      for (int c = 0; c < n; ++c) {
        rec.k0 = c * size;
        rec.k1 = imin((c + 1) * size, w.n);
        rec.part = n > 1 ? (int)part + c * w.nrows | flag : ~flag;
        items[i0 + c] = rec;
      }
#pragma unroll 1
      for (int u = 0; u < units; ++u)
        joins[j + u] = ChunkJoin{q.token0, w.row0 + u * join, imin(join, w.nrows - u * join), (int)part + u * join, n, w.nrows, 0, 0};
    }
    if (pass == 0) {
      const int64_t wave_total = wave_scan(total, add<int64_t>);
      const int wave_longest = wave_scan(longest, [](int x, int y) { return imax(x, y); });
      if ((tid & 63) == 63) {
        atomicAdd(&total_lds, (unsigned long long)wave_total);
        atomicMax(&longest_lds, wave_longest);
      }
      __syncthreads();
      const int64_t all = (int64_t)total_lds * a.kv_heads, over_two = (all + 2 * a.slots - 1) >> __builtin_ctz(2 * a.slots);
      const int least = imax(a.least, over_two < kBig ? (int)over_two : kBig), most = a.limit - 64;
      const float per_slot = 1.f / (float)a.slots, share = (float)all * per_slot;
      auto unit_of = [&](int k) __attribute__((always_inline)) {
        return imin(imax((int)fminf(0.5f * share * exp2f_fast((float)k * (2.f / (kUnits - 1))), 1e9f), least), most);
      };
      if (T > kLdsTiles) {
        unit = unit_of(kUnits / 2);
      } else {  // a unit per lane, tiles dealt to groups of kUnits lanes
        const int k = tid % kUnits, grp = tid / kUnits;
        const float u = (float)unit_of(k), inv = __builtin_amdgcn_rcpf(u);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};  // longer items, their keys, items, partial rows
#pragma unroll 2
        for (int g = grp; g < T; g += kT / kUnits) {
          const float n = (float)tile_n[g], cut = fmaxf(ceilf(fmaf(n, inv, -1e-4f)), 1.f);
          const bool is_longer = 2.f * n > u * cut;
          x += f32x4{is_longer ? cut : 0.f, is_longer ? n : 0.f, cut, cut > 1.f ? cut * (float)tile_nrows[g] : 0.f};
        }
        sums[grp][k] = x;
        __syncthreads();
        if (tid < kUnits) {
#pragma unroll
          for (int j = 1; j < kT / kUnits; ++j) x += sums[j][k];
          const float kvh = (float)a.kv_heads, kvh_slot = kvh * per_slot;
          const float rounds = x[0] > 0.f ? ceilf(x[0] * kvh_slot) * x[1] * __builtin_amdgcn_rcpf(x[0]) : 0.f;
          float cost = fmaxf(rounds, share) + x[2] * kvh_slot * kStartKeys + x[3] * kvh * (1.f / kPartRows);
          int best = k;
#pragma unroll
          for (int m = kUnits / 2; m > 0; m >>= 1) {  // the longest of the best
            const float c = __shfl_xor(cost, m);
            const int j = __shfl_xor(best, m);
            if (c < cost || (c == cost && j > best)) cost = c, best = j;
          }
          if (tid == 0) best_lds = best;
        }
        __syncthreads();
        unit = unit_of(best_lds);
      }
      half = imin(longest_lds, unit) / 2;
    }
  }
  // (a barrier for LDS alone: one that waits for the items' stores too takes 0.5 us)
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (tid == 0) put_chunk_head(a, placed, parts, rows, short_lds == 0);
}

}  // namespace

hipError_t launch_chunk_plan(const ChunkPlanArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kT), 0, s, a);
  return hipGetLastError();
}

}  // namespace bdlm
