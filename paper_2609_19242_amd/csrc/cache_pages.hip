// Operations on the pages of a cache, gfx950: grow, fork, free, compact, and
// writing new rows.  All bookkeeping is on the device (tables, lengths and
// reference counts), so a decoding loop needs no host round trip and can be
// captured; the results do not depend on timing: free pages are given out in
// ascending order to the listed sequences in their order, and counts change by
// integer atomics.
//
// Bookkeeping runs in one workgroup (a few microseconds: the work is a scan of
// the reference counts up to the pages needed and of the list); it checks the
// list first and changes nothing but the status if it does not hold.  It is bound
// by the scan's steps, each a round of loads and two barriers, so a step takes 16
// pages per thread (of 100,000 pages the last ones free: grow 22 us, with one page
// per thread 69; compact with nothing to move 45 us, 199).  Page data is moved by a
// second kernel, 16 bytes per lane, at the speed of a copy (compact: 1.5 GB in 289
// us, 5.1 TB/s; fork of 96 sequences over 32 layers 32 us).  A write of 96 x 8 rows
// of 2 KB takes 5 us, three loads in a row and the launch.
#include "cache.hpp"
#include "device.hpp"

namespace bdlm {

namespace {

constexpr int kT = 1024;         // threads of the bookkeeping workgroup
constexpr int kWordsLds = 16384; // a bit per sequence: 2^19 sequences

// Outcomes (bdlm_cache_status).
enum : int { kOk = 0, kBadList = 1, kNoPages = 2 };

constexpr int kPer = 16;         // pages per thread of a scan's step, their counts in flight together

// Exclusive prefix sum over the workgroup's threads; total of all.
template <class T>
__device__ __forceinline__ T block_scan(T x, T& total, int64_t* wsum) {
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
  for (int k = 0; k < kT / 64; ++k) {
    const T y = (T)wsum[k];
    if (k < w) base += y;
    t += y;
  }
  total = t;
  return base + v - x;
}

// Reference counts of the kPer pages from p on, 0 past the last (out: pages there are).
__device__ __forceinline__ int load_refs(const CacheArg& c, int64_t p, int (&refs)[kPer]) {
  typedef int32_t quad __attribute__((ext_vector_type(4), aligned(4)));
  const int64_t left = c.pages - p;
  if (left >= kPer) {
#pragma unroll
    for (int k = 0; k < kPer / 4; ++k) {
      const quad x = *(const quad*)(c.refs + p + 4 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) refs[4 * k + e] = x[e];
    }
    return kPer;
  }
  for (int k = 0; k < kPer; ++k) refs[k] = k < left ? c.refs[p + k] : 0;
  return left < 0 ? 0 : (int)left;
}

__device__ __forceinline__ int clamped_len(const CacheArg& c, int seq) {
  const int64_t top = (int64_t)c.max_pages * c.page_size;
  const int n = c.lens[seq];
  return n < 0 ? 0 : (int64_t)n > top ? (int)top : n;
}
__device__ __forceinline__ int pages_of(const CacheArg& c, int64_t tokens) {
  return (int)((tokens + c.page_size - 1) / c.page_size);
}

// The first `need` free pages in ascending order into list[0 .. need); false:
// fewer are free (found: how many).
__device__ bool take_free(const CacheArg& c, int64_t need, int32_t* list, int64_t* wsum, int& found) {
  found = 0;
  for (int64_t p0 = 0; p0 < c.pages && found < need; p0 += kT * kPer) {
    const int64_t p = p0 + threadIdx.x * kPer;
    int refs[kPer], mine = 0, total;
    const int n = load_refs(c, p, refs);
#pragma unroll
    for (int k = 0; k < kPer; ++k) mine += k < n && refs[k] == 0;
    int at = found + block_scan(mine, total, wsum);
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (k < n && refs[k] == 0) {
        if (at < need) list[at] = (int32_t)(p + k);
        ++at;
      }
    found += total;
  }
  __syncthreads();  // the list is read by other threads
  return found >= need;
}

// One bit per sequence: false if a listed number is out of range or listed twice.
__device__ bool mark(const CacheArg& c, const int32_t* list, int n, unsigned* bits, int* bad) {
  for (int i = threadIdx.x; i < (c.seqs + 31) / 32; i += kT) bits[i] = 0;
  if (threadIdx.x == 0) *bad = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kT) {
    const int s = list[i];
    if ((unsigned)s >= (unsigned)c.seqs) *bad = 1;
    else if (atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31) & 1) *bad = 1;
  }
  __syncthreads();
  const bool ok = *bad == 0;
  __syncthreads();  // (read by all before the caller's own checks write it)
  return ok;
}

// work: [0] 1 if the operation goes ahead, [1] moves; then a list of pages.
__global__ __launch_bounds__(kT) void cache_grow_kernel(const CacheArg c, const CacheList l, int32_t* work) {
  __shared__ __attribute__((aligned(16))) unsigned bits[kWordsLds];
  __shared__ int64_t wsum[kT / 64];
  __shared__ int bad;
  int32_t* const list = work + kCacheHead;
  bool ok = mark(c, l.a, l.n, bits, &bad);
  if (ok) {
    for (int i = threadIdx.x; i < l.n; i += kT) {
      const int s = l.a[i], add = l.b[i];
      if (add < 0 || (int64_t)clamped_len(c, s) + add > (int64_t)c.max_pages * c.page_size) bad = 1;
    }
    __syncthreads();
    ok = bad == 0;
  }
  int64_t need = 0;
  int found = 0;
  bool enough = true;
  if (ok) {
    for (int i0 = 0; i0 < l.n; i0 += kT) {
      const int i = i0 + threadIdx.x;
      int64_t pages = 0, total;  // (the pages asked for may pass 32 bits)
      if (i < l.n) {
        const int n = clamped_len(c, l.a[i]);
        pages = pages_of(c, (int64_t)n + l.b[i]) - pages_of(c, n);
      }
      block_scan(pages, total, wsum);
      need += total;
    }
    enough = take_free(c, need, list, wsum, found);
  }
  if (threadIdx.x == 0) {
    c.status[0] = !ok ? kBadList : enough ? kOk : kNoPages;
    c.status[1] = ok && !enough ? (int32_t)(need - found < 0x7fffffff ? need - found : 0x7fffffff) : 0;
  }
  if (!ok || !enough) return;
  // Sequence i of a round gets the pages list[given + first[i] ..]: thread by
  // thread for every page, so that a long prompt's pages take no longer than a
  // batch's (one sequence, 2,048 pages: 257 us by one thread, 10 by all).
  int* const first = (int*)bits;                      // [kT]
  int64_t* const entry = (int64_t*)(bits + kT);       // [kT]: where its first new page stands in the table, less first[i]
  int64_t given = 0;
  for (int i0 = 0; i0 < l.n; i0 += kT) {
    const int i = i0 + threadIdx.x;
    int n = 0, add = 0, held = 0, pages = 0, s = 0, total;
    if (i < l.n) {
      s = l.a[i];
      n = clamped_len(c, s);
      add = l.b[i];
      held = pages_of(c, n);
      pages = pages_of(c, (int64_t)n + add) - held;
    }
    const int at = block_scan(pages, total, wsum);
    first[threadIdx.x] = at;
    entry[threadIdx.x] = (int64_t)s * c.max_pages + held - at;
    __syncthreads();
    for (int k = threadIdx.x; k < total; k += kT) {
      int lo = 0;  // the last with first[lo] <= k
#pragma unroll
      for (int step = kT / 2; step > 0; step >>= 1)
        if (first[lo + step] <= k) lo += step;
      const int32_t p = list[given + k];
      c.table[entry[lo] + k] = p;
      c.refs[p] = 1;
    }
    given += total;
    if (i < l.n) c.lens[s] = n + add;
  }
}

// Pages for the children's partial last pages: list[i] = child i's page or -1.
__global__ __launch_bounds__(kT) void cache_fork_plan_kernel(const CacheArg c, const CacheList l, int32_t* work) {
  __shared__ __attribute__((aligned(16))) unsigned bits[kWordsLds];
  __shared__ int64_t wsum[kT / 64];
  __shared__ int bad;
  int32_t* const of_child = work + kCacheHead;
  int32_t* const list = of_child + l.n;
  bool ok = mark(c, l.b, l.n, bits, &bad);
  if (ok) {
    for (int i = threadIdx.x; i < l.n; i += kT) {
      const int p = l.a[i];
      // parents in range and no children themselves; children empty
      if ((unsigned)p >= (unsigned)c.seqs || (bits[p >> 5] >> (p & 31) & 1) || c.lens[l.b[i]] != 0) bad = 1;
    }
    __syncthreads();
    ok = bad == 0;
  }
  int64_t need = 0;
  int found = 0;
  bool enough = true;
  if (ok) {
    for (int i0 = 0; i0 < l.n; i0 += kT) {
      const int i = i0 + threadIdx.x;
      const int part = i < l.n && clamped_len(c, l.a[i]) % c.page_size != 0;
      int total;
      const int at = block_scan(part, total, wsum);
      if (i < l.n) of_child[i] = part ? (int32_t)(need + at) : -1;
      need += total;
    }
    enough = take_free(c, need, list, wsum, found);
  }
  if (threadIdx.x == 0) {
    c.status[0] = !ok ? kBadList : enough ? kOk : kNoPages;
    c.status[1] = ok && !enough ? (int32_t)(need - found < 0x7fffffff ? need - found : 0x7fffffff) : 0;
    work[0] = ok && enough;
  }
  if (!ok || !enough) return;
  for (int i = threadIdx.x; i < l.n; i += kT) {
    const int at = of_child[i];
    if (at >= 0) of_child[i] = list[at];
  }
}

// 16-byte copies of n bytes by the workgroup's threads.
__device__ __forceinline__ void copy_bytes(char* dst, const char* src, int64_t n) {
  const int64_t step = (int64_t)blockDim.x * 16;
  int64_t b = (int64_t)threadIdx.x * 16;
  for (; b + 3 * step < n; b += 4 * step) {
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = *(const u32x4*)(src + b + k * step);
#pragma unroll
    for (int k = 0; k < 4; ++k) *(u32x4*)(dst + b + k * step) = x[k];
  }
  for (; b < n; b += step) *(u32x4*)(dst + b) = *(const u32x4*)(src + b);
}

// Workgroup (i, y): the rows of child i's partial page in K (V) of layer y / 2; y = 0 also writes its table row.
__global__ __launch_bounds__(256) void cache_fork_kernel(const CacheArg c, const CacheList l, const int32_t* work) {
  if (work[0] == 0) return;
  const int i = blockIdx.x, parent = l.a[i], child = l.b[i];
  const int n = clamped_len(c, parent), full = n / c.page_size, part = n - full * c.page_size;
  const int page = work[kCacheHead + i];
  const int32_t* const from = c.table + (int64_t)parent * c.max_pages;
  for (int y = blockIdx.y; y < 2 * c.layers; y += gridDim.y) {
    if (part > 0) {
      const int old = from[full];
      if ((unsigned)old < (unsigned)c.pages) {
        char* const base = ((y & 1) ? c.v : c.k) + (y >> 1) * c.layer_bytes;
        copy_bytes(base + page * c.page_bytes, base + old * c.page_bytes, (int64_t)part * c.row_bytes);
      }
    }
  }
  if (blockIdx.y != 0) return;
  int32_t* const to = c.table + (int64_t)child * c.max_pages;
  for (int k = threadIdx.x; k < c.max_pages; k += 256) {
    int p = -1;
    if (k < full) {
      p = from[k];
      if ((unsigned)p < (unsigned)c.pages) atomicAdd(&c.refs[p], 1);
    } else if (k == full && part > 0) {
      p = page;
      c.refs[p] = 1;
    }
    to[k] = p;
  }
  if (threadIdx.x == 0) c.lens[child] = n;
}

// A sequence listed twice is freed once: whoever takes its length frees it.
// The first workgroup also writes the status.
__global__ __launch_bounds__(256) void cache_free_kernel(const CacheArg c, const CacheList l) {
  __shared__ int len, bad;
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < l.n; i += 256)
      if ((unsigned)l.a[i] >= (unsigned)c.seqs) bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) {
      c.status[0] = bad ? kBadList : kOk;
      c.status[1] = 0;
    }
    if (l.n == 0) return;
  }
  const int s = l.a[blockIdx.x];
  if ((unsigned)s >= (unsigned)c.seqs) return;
  if (threadIdx.x == 0) len = atomicExch(&c.lens[s], 0);
  __syncthreads();
  if (len <= 0) return;
  const int64_t top = (int64_t)c.max_pages * c.page_size;
  const int held = pages_of(c, len < top ? len : top);
  int32_t* const row = c.table + (int64_t)s * c.max_pages;
  for (int k = threadIdx.x; k < held; k += 256) {
    const int p = row[k];
    row[k] = -1;
    if ((unsigned)p >= (unsigned)c.pages) continue;
    int old = c.refs[p];
    while (old > 0) {  // (a count never falls below none)
      const int seen = atomicCAS(&c.refs[p], old, old - 1);
      if (seen == old) break;
      old = seen;
    }
  }
}

// Moves: the i-th free page below the live count takes the i-th live page at
// or above it.  list[0 .. n): free pages, list[pages .. pages + n): live ones;
// list[2 pages + p]: where page p >= live goes, -1 for a page that no table
// should hold.  The references move here, before the data.
__global__ __launch_bounds__(kT) void cache_compact_plan_kernel(const CacheArg c, int32_t* work) {
  __shared__ int64_t wsum[kT / 64];
  int32_t* const dst = work + kCacheHead;
  int32_t* const src = dst + c.pages;
  int64_t live = 0;
  for (int64_t p = threadIdx.x * kPer; p < c.pages; p += kT * kPer) {
    int refs[kPer];
    load_refs(c, p, refs);
#pragma unroll
    for (int k = 0; k < kPer; ++k) live += refs[k] > 0;
  }
  int64_t all;
  block_scan(live, all, wsum);
  live = all;
  int64_t holes = 0, moves = 0;
  for (int64_t p0 = 0; p0 < c.pages; p0 += kT * kPer) {
    const int64_t p = p0 + threadIdx.x * kPer;
    int refs[kPer];
    const int n = load_refs(c, p, refs);
    int64_t mine = 0, total;  // holes, and from bit 32 on moves
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (k < n && refs[k] <= 0 && p + k < live) mine += 1;
      if (k < n && refs[k] > 0 && p + k >= live) mine += (int64_t)1 << 32;
    }
    const int64_t at = block_scan(mine, total, wsum);
    int64_t ah = holes + (int32_t)at, am = moves + (at >> 32);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (k >= n) break;
      const bool move = refs[k] > 0 && p + k >= live;
      if (refs[k] <= 0 && p + k < live) dst[ah++] = (int32_t)(p + k);
      if (p + k >= live) src[c.pages + p + k] = move ? (int32_t)am : -1;
      if (move) src[am++] = (int32_t)(p + k);
    }
    holes += (int32_t)total;
    moves += total >> 32;
  }
  if (threadIdx.x == 0) {
    work[0] = (int32_t)live;
    work[1] = (int32_t)moves;
    c.status[0] = kOk;
    c.status[1] = 0;
  }
  __syncthreads();  // the lists are read by other threads
  for (int64_t m = threadIdx.x; m < moves; m += kT) {
    const int from = src[m], to = dst[m];
    src[c.pages + from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
}

__global__ __launch_bounds__(256) void cache_compact_kernel(const CacheArg c, const int32_t* work) {
  const int32_t* const dst = work + kCacheHead;
  const int32_t* const src = dst + c.pages;
  const int live = work[0], moves = work[1];
  const int64_t units = (int64_t)moves * 2 * c.layers;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int y = (int)(u / moves), m = (int)(u - (int64_t)y * moves);
    char* const base = ((y & 1) ? c.v : c.k) + (y >> 1) * c.layer_bytes;
    copy_bytes(base + dst[m] * c.page_bytes, base + src[m] * c.page_bytes, c.page_bytes);
  }
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t e = at; e < (int64_t)c.seqs * c.max_pages; e += step) {
    const int p = c.table[e];
    if (p < live || p >= c.pages) continue;
    const int to = src[c.pages + p];
    if (to >= 0) c.table[e] = to;
  }
}

// Rows of new tokens: sequence i's counts[i] rows go to its last positions.  Workgroup (i, y): every gridDim.y-th row.
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArg c, const CacheRows r) {
  const int i = blockIdx.x, s = r.seqs[i];
  if ((unsigned)s >= (unsigned)c.seqs) return;
  const int per = r.rows / r.n;
  const int64_t first = r.starts ? r.starts[i] : (int64_t)i * per;
  const int count = r.counts[i];
  const int64_t limit = r.starts ? r.rows : first + per;  // rows of this sequence in the new tensors end here
  // 16-byte pieces of several rows at a time
  const int pieces = c.row_bytes / 16;
  const int64_t j0 = first < 0 ? -first : 0, j1 = first + count < limit ? count : limit - first;
  for (int64_t x = j0 * pieces + (int64_t)blockIdx.y * 256 + threadIdx.x; x < j1 * pieces; x += (int64_t)gridDim.y * 256) {
    const int64_t j = x / pieces, row = first + j;
    const int b = (int)(x - j * pieces) * 16;
    // (loaded before the sequence's length and page are known: those take two loads in a row)
    const u32x4 xk = *(const u32x4*)(r.k + row * r.k_stride + b), xv = *(const u32x4*)(r.v + row * r.v_stride + b);
    const int64_t at_token = (int64_t)clamped_len(c, s) - count + j;
    if (at_token < 0) continue;
    const int pos = (int)at_token, e = pos / c.page_size;
    const int page = c.table[(int64_t)s * c.max_pages + e];
    if ((unsigned)page >= (unsigned)c.pages) continue;
    const int64_t at = r.layer * c.layer_bytes + page * c.page_bytes + (int64_t)(pos - e * c.page_size) * c.row_bytes + b;
    *(u32x4*)(c.k + at) = xk;
    *(u32x4*)(c.v + at) = xv;
  }
}

}  // namespace

hipError_t launch_cache_grow(const CacheArg& c, const CacheList& l, int32_t* work, hipStream_t s) {
  hipLaunchKernelGGL(cache_grow_kernel, dim3(1), dim3(kT), 0, s, c, l, work);
  return hipGetLastError();
}

hipError_t launch_cache_fork(const CacheArg& c, const CacheList& l, int32_t* work, hipStream_t s) {
  hipLaunchKernelGGL(cache_fork_plan_kernel, dim3(1), dim3(kT), 0, s, c, l, work);
  if (l.n > 0) {
    const int y = 2 * c.layers;
    hipLaunchKernelGGL(cache_fork_kernel, dim3(l.n, y < 4096 ? y : 4096), dim3(256), 0, s, c, l, work);
  }
  return hipGetLastError();
}

hipError_t launch_cache_free(const CacheArg& c, const CacheList& l, hipStream_t s) {
  hipLaunchKernelGGL(cache_free_kernel, dim3(l.n > 0 ? l.n : 1), dim3(256), 0, s, c, l);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheArg& c, int32_t* work, hipStream_t s) {
  hipLaunchKernelGGL(cache_compact_plan_kernel, dim3(1), dim3(kT), 0, s, c, work);
  hipLaunchKernelGGL(cache_compact_kernel, dim3(2048), dim3(256), 0, s, c, work);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheArg& c, const CacheRows& r, hipStream_t s) {
  if (r.n == 0 || r.rows == 0) return hipSuccess;
  const int64_t per = ((r.starts ? r.rows : r.rows / r.n) * (int64_t)(c.row_bytes / 16) + 255) / 256;
  const int y = (int)(per < 1 ? 1 : per > 64 ? 64 : per);
  hipLaunchKernelGGL(cache_write_kernel, dim3(r.n, y), dim3(256), 0, s, c, r);
  return hipGetLastError();
}

}  // namespace bdlm
