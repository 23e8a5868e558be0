// Declarations shared by the serving kernels (paged cache, attention over it,
// verification) and their part of the C ABI.
#pragma once

#include "dartree/serve.h"
#include "internal.hpp"

namespace dartree {

constexpr int kHead = 128;   // elements of a head
constexpr int kExpLow = -100;   // least exponent of an e4m3 row, of an e2m1 block
constexpr int kBlock = 32;      // elements of an e2m1 block, which has an exponent of its own

// Exponent bytes from here on can stand for 2^128, which no bf16 or fp32 number
// is: the e4m3 numbers nearest to 248 .. 255 times 2^120, bf16's largest, are 256
// times that.  Rows with such a byte are converted with the largest bf16 number in
// the place of an infinity (a NaN stays one).
constexpr uint32_t kTopByte = 127 + 120;
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {   // two bf16
  if ((w & 0x7FFFu) == 0x7F80u) w -= 1;
  if ((w & 0x7FFF0000u) == 0x7F800000u) w -= 0x10000u;
  return w;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight e2m1 elements times a power of two in bf16, exact.  The conversion takes the
// power from the exponent bits of `scale`; all of them set makes NaN of every element.
__device__ __forceinline__ u32x4 expand8(uint32_t x, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3))};
}

// A cache as the kernels see it.
struct CacheView {
  int batch, heads_kv, page_log2, num_pages, max_pages;
  void* k;
  void* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  const int32_t* table;
};

struct CacheMoveArgs {
  CacheView c;
  int bits;               // an element's: 16 (bf16), 8 (e4m3) or 4 (e2m1)
  int source_rows, rows;
  const uint16_t* k_in;   // write: source
  const uint16_t* v_in;
  int64_t row_stride;
  uint16_t* k_out;        // read: destination
  uint16_t* v_out;
  const int32_t* index;
  const int32_t* counts;
  const int32_t* start;
};
hipError_t launch_cache_write(const CacheMoveArgs& a, hipStream_t s);
hipError_t launch_cache_read(const CacheMoveArgs& a, hipStream_t s);

struct PagedArgs {
  CacheView c;
  int bits;
  int batch, budget, max_ctx, heads_q, heads_kv, group;
  float scale_log2;       // softmax scale * log2(e)
  const uint16_t* q;
  const uint16_t* k_tree;
  const uint16_t* v_tree;
  int64_t q_stride, kv_stride;
  const uint64_t* mask;
  const int32_t* num_nodes;
  const int32_t* ctx_len;
  uint16_t* out;
  void* ws;
};
size_t paged_attention_workspace(int batch, int budget, int max_ctx, int heads_q, int heads_kv, int bits);
hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t s);

struct VerifyArgs {
  int batch, budget, max_len, vocab, bf16;   // chain: budget = depth
  const int32_t* tokens;
  const int32_t* parents;     // NULL: a chain
  const int32_t* num_nodes;
  const void* target;
  const void* draft;
  int64_t row_stride;
  double inv_t;               // 1 / T, 0 at T = 0
  const float* uniforms;
  int32_t* accepted;
  int32_t* num_accepted;
  int32_t* bonus;
  void* ws;
};
size_t verify_tree_workspace(int batch, int budget, int max_len, int vocab);
size_t verify_chain_workspace(int batch, int depth, int vocab);
hipError_t launch_verify_tree(const VerifyArgs& a, hipStream_t s);
hipError_t launch_verify_chain(const VerifyArgs& a, hipStream_t s);

}  // namespace dartree
