// Pages of a paged cache: forked, reserved, compacted and copied.
//
// The page table says everything: which pages are named (in use), and which more
// than once (shared), is read off it into two bitmaps, a bit a page, by atomic ORs
// (their order does not matter: of two entries that name a page one finds its bit
// set).  Needs and free pages are then numbered by prefix sums in ascending order,
// so results do not depend on thread timing.
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
__host__ __device__ inline int words_of(int num_pages) { return (num_pages + 31) / 32; }
__host__ __device__ inline int64_t padded(int64_t n) { return (n + 63) & ~int64_t(63); }
__device__ __forceinline__ Space space_of(const PagesArgs& a) {
  const int64_t words = padded(words_of(a.num_pages));
  uint32_t* w = static_cast<uint32_t*>(a.ws);
  int32_t* upto = reinterpret_cast<int32_t*>(w + 2 * words);
  return Space{w, w + words, upto, upto + padded(a.batch)};
}

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

// Named and shared pages of the table, which is copied to `out` where that is another.
__global__ __launch_bounds__(kThreads) void pages_scan(PagesArgs a) {
  const Space s = space_of(a);
  const int64_t n = int64_t(a.batch) * a.max_pages;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    const int e = a.table[i];
    if (a.out != a.table) a.out[i] = e;
    if (!is_page(e, a.num_pages)) continue;
    const uint32_t bit = 1u << (e & 31);
    if (atomicOr(s.named + (e >> 5), bit) & bit) atomicOr(s.shared + (e >> 5), bit);
  }
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

// One block: the needs in order, the free pages in order, one to the other.
__global__ __launch_bounds__(kWide) void pages_reserve(PagesArgs a) {
  const Space s = space_of(a);
  const int64_t items = int64_t(a.batch) * a.columns;
  int wanted = 0, total;
  for (int64_t i0 = 0; i0 < items; i0 += kWide) {
    const int64_t i = i0 + threadIdx.x;
    const int q = int(i / a.columns), j = int(i - int64_t(q) * a.columns);
    const Need n = i < items ? need_of(a, s.shared, q, j) : Need{0, -1, false, false};
    const int before = block_prefix(n.page, &total);
    if (i < items && j == a.columns - 1) s.upto[q] = wanted + before + n.page;
    wanted += total;
  }
  const int words = words_of(a.num_pages);
  int free = 0;
  for (int w0 = 0; w0 < words; w0 += kWide) {
    const int w = w0 + threadIdx.x;
    uint32_t bits = w < words ? ~s.named[w] : 0u;
    if (w == words - 1 && (a.num_pages & 31)) bits &= (1u << (a.num_pages & 31)) - 1u;
    int rank = free + block_prefix(__popc(bits), &total);
    for (; bits && rank < wanted; bits &= bits - 1, ++rank) s.list[rank] = 32 * w + __builtin_ctz(bits);
    free += total;
  }
  __syncthreads();   // upto and list are written
  int pages = 0, copies = 0, taken = 0;
  for (int64_t i0 = 0; i0 < items; i0 += kWide) {
    const int64_t i = i0 + threadIdx.x;
    const int q = int(i / a.columns), j = int(i - int64_t(q) * a.columns);
    Need n = i < items ? need_of(a, s.shared, q, j) : Need{0, -1, false, false};
    const int upto = i < items ? s.upto[q] : 0;
    const bool granted = i < items && (upto <= free || upto == (q > 0 ? s.upto[q - 1] : 0));
    const int rank = pages + block_prefix(n.page, &total);
    pages += total;
    if (!granted) n.page = n.copy = false;
    const int place = copies + block_prefix(n.copy, &total);
    copies += total;
    block_prefix(n.page, &total);
    taken += total;
    if (n.page) {
      const int to = s.list[rank];
      a.out[n.at] = to;
      if (n.copy) {
        a.pairs[2 * int64_t(place)] = n.entry;
        a.pairs[2 * int64_t(place) + 1] = to;
      }
    }
    if (i < items && j == 0) a.granted[q] = granted;
  }
  if (threadIdx.x == 0) {
    a.totals[0] = copies;
    a.totals[1] = free - taken;
  }
}

// One block: pages in use from `live` on to the free ones below it.
__global__ __launch_bounds__(kWide) void pages_compact(PagesArgs a) {
  const Space s = space_of(a);
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
}

__global__ __launch_bounds__(kThreads) void pages_remap(PagesArgs a) {
  const Space s = space_of(a);
  const int live = a.totals[1];
  const int64_t n = int64_t(a.batch) * a.max_pages;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    int e = a.table[i];
    if (!is_page(e, a.num_pages)) {
      e = -1;
    } else if (e >= live) {
      const int w = e >> 5, first = max(live - 32 * w, 0);   // the word's pages below live stay
      const uint32_t before = s.named[w] & ((1u << (e & 31)) - 1u) & ~((1u << first) - 1u);
      e = a.pairs[2 * int64_t(s.list[w] + __popc(before)) + 1];
    }
    a.out[i] = e;
  }
}

unsigned blocks_for(int64_t items) { return unsigned(std::min<int64_t>(2048, (items + kThreads - 1) / kThreads)); }

hipError_t launch_scan(const PagesArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(pages_clear, dim3(blocks_for(2 * words_of(a.num_pages))), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(pages_scan, dim3(blocks_for(int64_t(a.batch) * a.max_pages)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// A unit of the copy: 16 KB of a page's keys or values, or a page's exponents.
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
  const hipError_t e = launch_scan(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_reserve, dim3(1), dim3(kWide), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const hipError_t e = launch_scan(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pages_compact, dim3(1), dim3(kWide), 0, s, a);
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
