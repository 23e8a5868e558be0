// Declarations of the page kernels and their part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "dartree/pages.h"

namespace dartree {

struct PagesArgs {
  int batch, page_log2, num_pages, max_pages;
  const int32_t* table;
  int32_t* out;
  const int32_t* source;   // fork
  const int32_t* keep;
  int rows, columns;       // reserve: columns that `rows` positions can touch
  const int32_t* start;
  const int32_t* counts;
  int32_t* pairs;
  int32_t* totals;
  int32_t* granted;
  void* ws;
};
size_t pages_workspace(int batch, int num_pages);
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s);

struct PageCopyArgs {
  int num_pages;
  int64_t row_bytes, exp_bytes;   // of a page's keys and of its exponents (0: none), multiples of 16
  void* k;
  void* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  const int32_t* pairs;
  int max_pairs;
  const int32_t* count;
};
hipError_t launch_cache_copy(const PageCopyArgs& a, hipStream_t s);

}  // namespace dartree
