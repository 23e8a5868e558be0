// Pages of a paged cache: forked, reserved, compacted and copied.
//
// The page table says everything: which pages are named (in use), and which more
// than once (shared), is read off it into two bitmaps, a bit a page, by atomic ORs
// (their order does not matter: of two entries that name a page one finds its bit
// set).  Needs and free pages are then numbered by prefix sums in ascending order,
// so results do not depend on thread timing.
//
// What bounds them is latency: a launch (2.2 us each), the round trips start -> table
// entry -> bitmap -> page, and a barrier or two a prefix sum.  64 requests of 4096
// positions in pages of 64: fork 2.3 us, reserve 8.4 (as three launches 14.4).  A compact
// of a table of 8320 entries and as many pages 11 (as four launches 18).
#include <algorithm>

#include "internal.hpp"
#include "pages.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWide = 1024;   // threads of the single block that numbers needs and pages

// Workspace: the bitmaps, a word per 32 pages, then per request the needs of the
// requests up to it, and the free pages in ascending order (compact: per word the
// moved pages before it).
struct Space {
  uint32_t* named;
  uint32_t* shared;
  int32_t* upto;
  int32_t* list;
};
__host__ __device__ inline int words_of(int num_pages) { return int((int64_t(num_pages) + 31) / 32); }
__host__ __device__ inline int64_t padded(int64_t n) { return (n + 63) & ~int64_t(63); }
__device__ __forceinline__ Space space_of(const PagesArgs& a) {
  const int64_t words = padded(words_of(a.num_pages));
  uint32_t* w = static_cast<uint32_t*>(a.ws);
  int32_t* upto = reinterpret_cast<int32_t*>(w + 2 * words);
  return Space{w, w + words, upto, upto + padded(a.batch)};
}

// A small pool and table: one block does it all in one launch, bitmaps in LDS.  One
// launch / clear, scan and the rest (us in a graph, entries of the table, pages):
// reserve 4160, 4500 7.7 / 12.3; 16384, 18000 9.2 / 13.7; 32768, 35000 12.5 / 16.3;
// 65536, 65000 17.5 / 17.7; 131072 25.6 / 18.3; compact 7.4 / 13.5; 12.8 / 17.2; 23.2 /
// 23.6; 37.4 / 29.4.
constexpr int kSmallPages = 65536, kSmallEntries = 32768;
struct Bitmaps {
  uint32_t named[kSmallPages / 32], shared[kSmallPages / 32];
  int32_t before[kSmallPages / 32];   // compact's list
};

__device__ __forceinline__ bool is_page(int e, int num_pages) { return uint32_t(e) < uint32_t(num_pages); }

__global__ __launch_bounds__(kThreads) void pages_fork(PagesArgs a) {
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= int64_t(a.batch) * a.max_pages) return;
  const int q = int(i / a.max_pages), c = int(i - int64_t(q) * a.max_pages);
  const int from = a.source ? a.source[q] : q;
  const bool kept = uint32_t(from) < uint32_t(a.batch) && (!a.keep || (int64_t(c) << a.page_log2) < a.keep[q]);
  a.out[i] = kept ? a.table[int64_t(from) * a.max_pages + c] : -1;
}

__global__ __launch_bounds__(kThreads) void pages_clear(PagesArgs a) {
  const int64_t n = 2 * padded(words_of(a.num_pages));
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads)
    static_cast<uint32_t*>(a.ws)[i] = 0;
}

constexpr int kEach = 8;   // table entries of a thread that are loaded together

// Named and shared pages of the table, which is copied to `out` where that is
// another: thread t of n.
__device__ __forceinline__ void scan(const PagesArgs& a, const Space& s, int64_t t, int64_t n) {
  const int64_t items = int64_t(a.batch) * a.max_pages;
  for (int64_t i0 = t; i0 < items; i0 += kEach * n) {
    int e[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) e[k] = i0 + k * n < items ? a.table[i0 + k * n] : -1;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (a.out != a.table && i0 + k * n < items) a.out[i0 + k * n] = e[k];
      if (!is_page(e[k], a.num_pages)) continue;
      const uint32_t bit = 1u << (e[k] & 31);
      if (atomicOr(s.named + (e[k] >> 5), bit) & bit) atomicOr(s.shared + (e[k] >> 5), bit);
    }
  }
}
__global__ __launch_bounds__(kThreads) void pages_scan(PagesArgs a) {
  scan(a, space_of(a), int64_t(blockIdx.x) * kThreads + threadIdx.x, int64_t(gridDim.x) * kThreads);
}
// The same by one block of a small table, into its LDS.
__device__ __forceinline__ Space scan_small(const PagesArgs& a, Bitmaps* maps) {
  Space s = space_of(a);
  s.named = maps->named;
  s.shared = maps->shared;
  for (int w = threadIdx.x; w < words_of(a.num_pages); w += kWide) s.named[w] = s.shared[w] = 0;
  __syncthreads();
  scan(a, s, threadIdx.x, kWide);
  __syncthreads();
  return s;
}

// Exclusive prefix sums of x over the block's threads in order; total: of all.
__device__ __forceinline__ int block_prefix(int x, int* total) {
  __shared__ int sums[kWide / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  __syncthreads();   // sums are free
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWide / 64; ++w) {
    const int v = sums[w];
    if (w < wave) before += v;
    all += v;
  }
  *total = all;
  return before + incl - x;
}

// What column `first + j` of request q needs.
struct Need {
  int64_t at;        // of the table's entry
  int entry;
  bool page, copy;   // a free page; its contents copied from `entry`
};
__device__ __forceinline__ Need need_of(const PagesArgs& a, const uint32_t* shared, int q, int j) {
  Need r{0, -1, false, false};
  const int64_t limit = int64_t(a.max_pages) << a.page_log2;
  const int64_t s = a.start ? a.start[q] : 0;
  const int n = a.counts ? min(a.counts[q], a.rows) : a.rows;
  const int64_t lo = s > 0 ? s : 0, hi = s + n < limit ? s + n : limit;   // positions
  if (lo >= hi) return r;
  const int64_t c = (lo >> a.page_log2) + j;
  if ((c << a.page_log2) >= hi) return r;
  r.at = int64_t(q) * a.max_pages + c;
  r.entry = a.table[r.at];
  if (!is_page(r.entry, a.num_pages)) {
    r.page = true;
  } else if ((shared[r.entry >> 5] >> (r.entry & 31)) & 1u) {
    r.page = true;
    r.copy = lo > (c << a.page_log2) || hi < ((c + 1) << a.page_log2);
  }
  return r;
}

// One block: the needs in order, the free pages in order, one to the other.  Up to
// kWide items keep what they need in registers from the first pass to the last.
template <bool SMALL>
__global__ __launch_bounds__(kWide) void pages_reserve(PagesArgs a) {
  Space s;
  if constexpr (SMALL) {
    __shared__ Bitmaps maps;
    s = scan_small(a, &maps);
  } else {
    s = space_of(a);
  }
  const Need none{0, -1, false, false};
  const int64_t items = int64_t(a.batch) * a.columns;
  const bool once = items <= kWide;
  Need need = none;
  int wanted = 0, rank = 0, total;
  for (int64_t i0 = 0; i0 < items; i0 += kWide) {
    const int64_t i = i0 + threadIdx.x;
    const int q = int(i / a.columns), j = int(i - int64_t(q) * a.columns);
    need = i < items ? need_of(a, s.shared, q, j) : none;
    rank = wanted + block_prefix(need.page, &total);
    if (i < items && j == a.columns - 1) s.upto[q] = rank + need.page;
    wanted += total;
  }
  const int words = words_of(a.num_pages);
  int free = 0;
  for (int w0 = 0; w0 < words; w0 += kWide) {
    const int w = w0 + threadIdx.x;
    uint32_t bits = w < words ? ~s.named[w] : 0u;
    if (w == words - 1 && (a.num_pages & 31)) bits &= (1u << (a.num_pages & 31)) - 1u;
    int at = free + block_prefix(__popc(bits), &total);
    for (; bits && at < wanted; bits &= bits - 1, ++at) s.list[at] = 32 * w + __builtin_ctz(bits);
    free += total;
  }
  __syncthreads();   // upto and list are written
  int pages = 0, copies = 0, taken = 0;
  for (int64_t i0 = 0; i0 < items; i0 += kWide) {
    const int64_t i = i0 + threadIdx.x;
    const int q = int(i / a.columns), j = int(i - int64_t(q) * a.columns);
    if (!once) {
      need = i < items ? need_of(a, s.shared, q, j) : none;
      rank = pages + block_prefix(need.page, &total);
      pages += total;
    }
    const int upto = i < items ? s.upto[q] : 0;
    const bool granted = i < items && (upto <= free || upto == (q > 0 ? s.upto[q - 1] : 0));
    const bool copy = granted && need.copy;
    const int place = copies + block_prefix(copy, &total);
    copies += total;
    if (granted && need.page) {
      const int to = s.list[rank];
      ++taken;
      a.out[need.at] = to;
      if (copy) {
        a.pairs[2 * int64_t(place)] = need.entry;
        a.pairs[2 * int64_t(place) + 1] = to;
      }
    }
    if (i < items && j == 0) a.granted[q] = granted;
  }
  block_prefix(taken, &total);
  if (threadIdx.x == 0) {
    a.totals[0] = copies;
    a.totals[1] = free - total;
  }
}

// Table entries from `live` on become the pages that took theirs: thread t of n.
__device__ __forceinline__ void remap(const PagesArgs& a, const Space& s, int live, int64_t t, int64_t n) {
  const int64_t items = int64_t(a.batch) * a.max_pages;
  for (int64_t i0 = t; i0 < items; i0 += kEach * n) {
    int e[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) e[k] = i0 + k * n < items ? a.table[i0 + k * n] : -1;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (!is_page(e[k], a.num_pages)) {
        e[k] = -1;
      } else if (e[k] >= live) {
        const int w = e[k] >> 5, first = max(live - 32 * w, 0);   // the word's pages below live stay
        const uint32_t before = s.named[w] & ((1u << (e[k] & 31)) - 1u) & ~((1u << first) - 1u);
        e[k] = a.pairs[2 * int64_t(s.list[w] + __popc(before)) + 1];
      }
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (i0 + k * n < items) a.out[i0 + k * n] = e[k];
  }
}
__global__ __launch_bounds__(kThreads) void pages_remap(PagesArgs a) {
  remap(a, space_of(a), a.totals[1], int64_t(blockIdx.x) * kThreads + threadIdx.x, int64_t(gridDim.x) * kThreads);
}

// One block: pages in use from `live` on to the free ones below it.
template <bool SMALL>
__global__ __launch_bounds__(kWide) void pages_compact(PagesArgs a) {
  Space s;
  if constexpr (SMALL) {
    __shared__ Bitmaps maps;
    s = scan_small(a, &maps);
    s.list = maps.before;
  } else {
    s = space_of(a);
  }
  const int words = words_of(a.num_pages);
  int live = 0, total;
  for (int w0 = 0; w0 < words; w0 += kWide) {
    const int w = w0 + threadIdx.x;
    block_prefix(w < words ? __popc(s.named[w]) : 0, &total);
    live += total;
  }
  int from = 0, to = 0;
  for (int w0 = 0; w0 < words; w0 += kWide) {
    const int w = w0 + threadIdx.x;
    const uint32_t named = w < words ? s.named[w] : 0u;
    const int below = min(max(live - 32 * w, 0), 32);   // pages of this word that lie below live
    const uint32_t mask = below == 32 ? ~0u : (1u << below) - 1u;
    uint32_t away = named & ~mask, holes = w < words ? ~named & mask : 0u;
    int rank = from + block_prefix(__popc(away), &total);
    if (w < words) s.list[w] = rank;
    from += total;
    for (; away; away &= away - 1, ++rank) a.pairs[2 * int64_t(rank)] = 32 * w + __builtin_ctz(away);
    rank = to + block_prefix(__popc(holes), &total);
    to += total;
    for (; holes; holes &= holes - 1, ++rank) a.pairs[2 * int64_t(rank) + 1] = 32 * w + __builtin_ctz(holes);
  }
  if (threadIdx.x == 0) {
    a.totals[0] = from;
    a.totals[1] = live;
  }
  if constexpr (SMALL) {
    __syncthreads();   // pairs and list are written
    remap(a, s, live, threadIdx.x, kWide);
  }
}

bool is_small(const PagesArgs& a) { return a.num_pages <= kSmallPages && int64_t(a.batch) * a.max_pages <= kSmallEntries; }

unsigned blocks_for(int64_t items) { return unsigned(std::min<int64_t>(2048, (items + kThreads - 1) / kThreads)); }

hipError_t launch_scan(const PagesArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(pages_clear, dim3(blocks_for(2 * words_of(a.num_pages))), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(pages_scan, dim3(blocks_for(int64_t(a.batch) * a.max_pages)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// A unit of the copy: 16 KB of a page's keys or values, or a page's exponents; a
// thread has four loads of 16 bytes in flight.  Bound by memory: 512 MB read and
// written (compact, e4m3) in 92 us, 5.6 TB/s; 975 MB of e2m1 pages in 188, 5.2; 134 MB in
// 13.8, 71 in e2m1 in 11.8, as far as the caches hold them.
constexpr int kUnit = 16384;
__global__ __launch_bounds__(kThreads) void cache_copy(PageCopyArgs a) {
  const int pairs = min(a.count[0], a.max_pairs);
  const int rows = int((a.row_bytes + kUnit - 1) / kUnit), exps = int((a.exp_bytes + kUnit - 1) / kUnit);
  const int per = 2 * (rows + exps);
  const int64_t units = int64_t(pairs) * per;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = int(u / per);
    int part = int(u - int64_t(pair) * per);
    const int from = a.pairs[2 * int64_t(pair)], to = a.pairs[2 * int64_t(pair) + 1];
    if (!is_page(from, a.num_pages) || !is_page(to, a.num_pages) || from == to) continue;
    const bool is_exp = part >= 2 * rows;
    if (is_exp) part -= 2 * rows;
    const int64_t bytes = is_exp ? a.exp_bytes : a.row_bytes;
    const int each = is_exp ? exps : rows;
    const bool is_v = part >= each;
    if (is_v) part -= each;
    char* base = static_cast<char*>(is_exp ? static_cast<void*>(is_v ? a.v_exp : a.k_exp) : is_v ? a.v : a.k);
    const u32x4* src = reinterpret_cast<const u32x4*>(base + from * bytes + int64_t(part) * kUnit);
    u32x4* dst = reinterpret_cast<u32x4*>(base + to * bytes + int64_t(part) * kUnit);
    const int n = int(min(int64_t(kUnit), bytes - int64_t(part) * kUnit) / 16);
    constexpr int kEach = kUnit / 16 / kThreads;
    u32x4 x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (int(threadIdx.x) + i * kThreads < n) x[i] = src[threadIdx.x + i * kThreads];
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (int(threadIdx.x) + i * kThreads < n) dst[threadIdx.x + i * kThreads] = x[i];
  }
}

}  // namespace

size_t pages_workspace(int batch, int num_pages) {
  return size_t(2 * padded(words_of(num_pages)) + padded(batch) + padded(num_pages)) * sizeof(uint32_t);
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s) {
  const int64_t n = int64_t(a.batch) * a.max_pages;
  hipLaunchKernelGGL(pages_fork, dim3(unsigned((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t s) {
  if (is_small(a)) {
    hipLaunchKernelGGL(pages_reserve<true>, dim3(1), dim3(kWide), 0, s, a);
    return hipGetLastError();
  }
  const hipError_t e = launch_scan(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_reserve<false>, dim3(1), dim3(kWide), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  if (is_small(a)) {
    hipLaunchKernelGGL(pages_compact<true>, dim3(1), dim3(kWide), 0, s, a);
    return hipGetLastError();
  }
  const hipError_t e = launch_scan(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_compact<false>, dim3(1), dim3(kWide), 0, s, a);
  hipLaunchKernelGGL(pages_remap, dim3(blocks_for(int64_t(a.batch) * a.max_pages)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_copy(const PageCopyArgs& a, hipStream_t s) {
  const int64_t rows = (a.row_bytes + kUnit - 1) / kUnit, exps = (a.exp_bytes + kUnit - 1) / kUnit;
  const int64_t units = int64_t(a.max_pairs) * 2 * (rows + exps);
  hipLaunchKernelGGL(cache_copy, dim3(unsigned(std::min<int64_t>(2048, units))), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace dartree
