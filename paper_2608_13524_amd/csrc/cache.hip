// The paged key/value cache: rows of 128 bf16 elements written to pages, as
// they are or in e4m3 with one power of two per row, and read back.
//
// A row is 16 lanes of 8 elements (16 bytes of bf16, 8 of e4m3); a lane moves
// its eighth of the key and of the value row of one (request, position, head),
// heads fastest, so that a wave reads 1 KB of consecutive source bytes and
// writes whole 128- or 256-byte rows.  A power of two as scale costs nothing:
// e4m3 is a floating type, its rounding is relative, and scaling by a power of
// two is exact, so the bytes are the nearest ones to x 2^-e whatever the order
// of operations.
#include "reduce.hpp"
#include "serve.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Slot of position `pos` of request q: its index among all (page, slot) pairs
// of head 0, or -1 where there is none.
__device__ __forceinline__ int64_t slot_of(const CacheView& c, int q, int64_t pos) {
  if (pos < 0 || (pos >> c.page_log2) >= c.max_pages) return -1;
  const int page = c.table[int64_t(q) * c.max_pages + (pos >> c.page_log2)];
  if (page < 0 || page >= c.num_pages) return -1;
  return ((int64_t(page) * c.heads_kv) << c.page_log2) + (pos & ((1 << c.page_log2) - 1));
}

// Least e >= kExpLow with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return min(max(e, kExpLow), 120);
}

__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight elements of a row (16 lanes hold it) to e4m3; the row's exponent in e.
__device__ __forceinline__ u32x2 quantise(u32x4 x, int& e) {
  float f[8], m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = low(x[i]);
    f[2 * i + 1] = high(x[i]);
    m = fmaxf(m, fmaxf(fabsf(f[2 * i]), fabsf(f[2 * i + 1])));
  }
  m = row16_max(m);
  e = row_exponent(m);
  // 2^-e; with an infinity in the row 0, which makes that a NaN and the other values 0
  const float s = m == INFINITY ? 0.f : __uint_as_float(uint32_t(127 - e) << 23);
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * s, f[4 * i + 1] * s, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * s, f[4 * i + 3] * s, w, true);
    out[i] = uint32_t(w);
  }
  return out;
}

template <bool E8>
__global__ __launch_bounds__(256) void cache_write(CacheMoveArgs a) {
  const unsigned r = blockIdx.x * 16 + (threadIdx.x >> 4);   // below 2^31
  const int lane = threadIdx.x & 15;
  const int head = int(r % unsigned(a.c.heads_kv));
  const unsigned qi = r / unsigned(a.c.heads_kv);
  const int q = int(qi / unsigned(a.rows)), i = int(qi % unsigned(a.rows));
  if (q >= a.c.batch) return;
  const int n = a.counts ? a.counts[q] : a.rows;
  const int src = a.index ? a.index[qi] : i;
  const int64_t slot = slot_of(a.c, q, int64_t(a.start ? a.start[q] : 0) + i);
  if (i >= n || src < 0 || src >= a.source_rows || slot < 0) return;   // the same for a row's 16 lanes
  const int64_t at = (int64_t(q) * a.source_rows + src) * a.row_stride + head * kHead + lane * 8;
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.k_in + at);
  const u32x4 v = *reinterpret_cast<const u32x4*>(a.v_in + at);
  const int64_t row = slot + (int64_t(head) << a.c.page_log2);
  const int64_t to = row * kHead + lane * 8;
  if (E8) {
    int ek, ev;
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.k) + to) = quantise(k, ek);
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.v) + to) = quantise(v, ev);
    if (lane == 0) {
      a.c.k_exp[row] = uint8_t(ek + 127);
      a.c.v_exp[row] = uint8_t(ev + 127);
    }
  } else {
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.c.k) + to) = k;
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.c.v) + to) = v;
  }
}

// Eight e4m3 elements times the power of two of exponent byte e, in bf16.
__device__ __forceinline__ u32x4 expand(u32x2 x, uint32_t e) {
  const float s = __uint_as_float(e << 23);
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    out[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, false));
    out[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, true));
  }
  return out;
}

template <bool E8>
__global__ __launch_bounds__(256) void cache_read(CacheMoveArgs a) {
  const unsigned r = blockIdx.x * 16 + (threadIdx.x >> 4);   // below 2^31
  const int lane = threadIdx.x & 15;
  const int head = int(r % unsigned(a.c.heads_kv));
  const unsigned qi = r / unsigned(a.c.heads_kv);
  const int q = int(qi / unsigned(a.rows)), i = int(qi % unsigned(a.rows));
  if (q >= a.c.batch) return;
  if (a.counts && i >= a.counts[q]) return;
  const int64_t slot = slot_of(a.c, q, int64_t(a.start ? a.start[q] : 0) + i);
  u32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
  if (slot >= 0) {
    const int64_t row = slot + (int64_t(head) << a.c.page_log2);
    const int64_t from = row * kHead + lane * 8;
    if (E8) {
      const u32x2 xk = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.c.k) + from);
      const u32x2 xv = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.c.v) + from);
      const uint32_t ek = a.c.k_exp[row], ev = a.c.v_exp[row];
      k = expand(xk, ek);
      v = expand(xv, ev);
      if (max(ek, ev) >= kTopByte) {   // once, behind all loads
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          k[i] = finite_pair(k[i]);
          v[i] = finite_pair(v[i]);
        }
      }
    } else {
      k = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.c.k) + from);
      v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.c.v) + from);
    }
  }
  const int64_t to = int64_t(r) * kHead + lane * 8;   // [q][i][head]
  *reinterpret_cast<u32x4*>(a.k_out + to) = k;
  *reinterpret_cast<u32x4*>(a.v_out + to) = v;
}

unsigned blocks_of(const CacheMoveArgs& a) {
  return unsigned((int64_t(a.c.batch) * a.rows * a.c.heads_kv + 15) / 16);
}

}  // namespace

hipError_t launch_cache_write(const CacheMoveArgs& a, hipStream_t s) {
  if (a.eight) hipLaunchKernelGGL(cache_write<true>, dim3(blocks_of(a)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cache_write<false>, dim3(blocks_of(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheMoveArgs& a, hipStream_t s) {
  if (a.eight) hipLaunchKernelGGL(cache_read<true>, dim3(blocks_of(a)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(cache_read<false>, dim3(blocks_of(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dartree
