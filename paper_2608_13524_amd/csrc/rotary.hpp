// Declarations of the rotary kernels and their part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "dartree/rotary.h"

namespace dartree {

struct RotaryArgs {
  int batch, rows, heads_q, heads_kv, head_dim, rotary_dim, layout, bf16, inverse, first;
  float amplitude;
  const uint64_t* turns;
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  const int32_t* positions;
  const int32_t* start;
  const int32_t* counts;
  int block_rows, turned, head_items;   // set by the launcher
  uint32_t head_magic;
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s);

}  // namespace dartree
