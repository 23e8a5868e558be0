// The paged key/value cache: rows of 128 bf16 elements written to pages, as
// they are, in e4m3 with one power of two per row or in e2m1 with one per 32
// elements, and read back.
//
// A row is 16 lanes of 8 elements (16 bytes of bf16, 8 of e4m3, 4 of e2m1); a lane moves
// its eighth of the key and of the value row of one (request, position, head),
// heads fastest (but see Move), so that a wave reads 1 KB of consecutive source bytes and
// writes whole rows of 256, 128 or 64 bytes.  A power of two as scale costs nothing:
// e4m3 is a floating type, its rounding is relative, and scaling by a power of
// two is exact, so the bytes are the nearest ones to x 2^-e whatever the order
// of operations.
//
// e2m1 has one bit of mantissa and two of exponent, so a power of two serves 32 elements,
// four lanes.  Bound by memory: a ragged batch of 8 x 2048 positions of 8 heads is written
// and read in 28 us (127 MB, 4.5 TB/s); 16 x 16 in 3.2 and 3.1, the launch.  Two rows a
// thread, their loads in flight together, take as long.
#include "reduce.hpp"
#include "serve.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Slot of position `pos` of request q: its index among all (page, slot) pairs
// of head 0, or -1 where there is none.
__device__ __forceinline__ int64_t slot_of(const CacheView& c, int q, int64_t pos) {
  if (pos < 0 || (pos >> c.page_log2) >= c.max_pages) return -1;
  const int page = c.table[int64_t(q) * c.max_pages + (pos >> c.page_log2)];
  if (page < 0 || page >= c.num_pages) return -1;
  return ((int64_t(page) * c.heads_kv) << c.page_log2) + (pos & ((1 << c.page_log2) - 1));
}

// What 16 lanes move: head `head` of row i of request q; r: its place in [q][i][head].
// A block's 16 are consecutive heads and rows, but in e2m1, where a row of the cache is half
// a line of 128 bytes, 16 positions of one head, so that no line is written or read by
// blocks of two XCDs (us, write / read of 8 x 2048 positions of 8 heads 17.0 / 15.9 -> 16.1 /
// 14.9, 8 x 8192 68 / 67 -> 64 / 61; e4m3 18 / 17 either way, bf16 99 / 93 -> 105 / 102).
struct Move {
  int q, i, head;
  unsigned r;   // below 2^31
};
template <int BITS>
__host__ __device__ __forceinline__ bool by_positions(const CacheMoveArgs& a) {
  return BITS == 4 && a.rows >= 16;
}
template <int BITS>
__device__ __forceinline__ bool move_of(const CacheMoveArgs& a, Move* m) {
  const unsigned heads = unsigned(a.c.heads_kv), rows = unsigned(a.rows), part = threadIdx.x >> 4;
  if (by_positions<BITS>(a)) {
    const unsigned tiles = (rows + 15) / 16, tile = blockIdx.x / heads, q = tile / tiles, i = (tile - q * tiles) * 16 + part;
    const unsigned head = blockIdx.x - tile * heads;
    *m = Move{int(q), int(i), int(head), (q * rows + i) * heads + head};
    return i < rows;
  }
  const unsigned r = blockIdx.x * 16 + part, qi = r / heads, q = qi / rows;
  *m = Move{int(q), int(qi - q * rows), int(r - qi * heads), r};
  return int(q) < a.c.batch;
}

__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Least e >= kExpLow with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return min(max(e, kExpLow), 120);
}

// Least e >= kExpLow with amax <= 6 * 2^e = 1.5 * 2^(e + 2).  At most 125: 6 * 2^126
// is no bf16 number, so the numbers above 6 * 2^125 are held as that.
__device__ __forceinline__ int block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 2 + ((u & 0x7FFFFFu) > 0x400000u);
  return min(max(e, kExpLow), 125);
}

// Eight elements of a row to e2m1, the first in the lowest bits, and the exponent
// byte of their block, which four lanes hold.  The conversion divides by its scale,
// rounds to the nearest, ties to the even code, and takes what is above 6 as 6.  A
// NaN or an infinity has no e2m1 code: the whole block counts as NaN (byte 255).
__device__ __forceinline__ uint32_t quantise4(u32x4 x, uint32_t& byte) {
  float f[8], m = 0.f;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = low(x[i]);
    f[2 * i + 1] = high(x[i]);
    m = fmaxf(m, fmaxf(fabsf(f[2 * i]), fabsf(f[2 * i + 1])));
    odd |= (x[i] & 0x7F80u) == 0x7F80u || (x[i] & 0x7F800000u) == 0x7F800000u;
  }
  if (odd) m = INFINITY;
  m = fmaxf(m, __shfl_xor(m, 1));
  m = fmaxf(m, __shfl_xor(m, 2));
  const int e = block_exponent(m);
  const float s = __uint_as_float(uint32_t(127 + e) << 23);
  uint32_t out = 0;
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[0], f[1], s, 0);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[2], f[3], s, 1);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[4], f[5], s, 2);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, f[6], f[7], s, 3);
  byte = m == INFINITY ? 255u : uint32_t(e + 127);
  return m == INFINITY ? 0u : out;
}

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

template <int BITS>
__global__ __launch_bounds__(256) void cache_write(CacheMoveArgs a) {
  const int lane = threadIdx.x & 15;
  Move m;
  if (!move_of<BITS>(a, &m)) return;
  const int q = m.q, i = m.i, head = m.head;
  const int n = a.counts ? a.counts[q] : a.rows;
  const int src = a.index ? a.index[int64_t(q) * a.rows + i] : i;
  const int64_t slot = slot_of(a.c, q, int64_t(a.start ? a.start[q] : 0) + i);
  if (i >= n || src < 0 || src >= a.source_rows || slot < 0) return;   // the same for a row's 16 lanes
  const int64_t at = (int64_t(q) * a.source_rows + src) * a.row_stride + head * kHead + lane * 8;
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.k_in + at);
  const u32x4 v = *reinterpret_cast<const u32x4*>(a.v_in + at);
  const int64_t row = slot + (int64_t(head) << a.c.page_log2);
  const int64_t to = row * kHead + lane * 8;
  if constexpr (BITS == 8) {
    int ek, ev;
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.k) + to) = quantise(k, ek);
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.v) + to) = quantise(v, ev);
    if (lane == 0) {
      a.c.k_exp[row] = uint8_t(ek + 127);
      a.c.v_exp[row] = uint8_t(ev + 127);
    }
  } else if constexpr (BITS == 4) {
    uint32_t ek, ev;
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.c.k) + to / 2) = quantise4(k, ek);
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.c.v) + to / 2) = quantise4(v, ev);
    if ((lane & 3) == 0) {
      a.c.k_exp[row * (kHead / kBlock) + (lane >> 2)] = uint8_t(ek);
      a.c.v_exp[row * (kHead / kBlock) + (lane >> 2)] = uint8_t(ev);
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

template <int BITS>
__global__ __launch_bounds__(256) void cache_read(CacheMoveArgs a) {
  const int lane = threadIdx.x & 15;
  Move m;
  if (!move_of<BITS>(a, &m)) return;
  const int q = m.q, i = m.i, head = m.head;
  if (a.counts && i >= a.counts[q]) return;
  const int64_t slot = slot_of(a.c, q, int64_t(a.start ? a.start[q] : 0) + i);
  u32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
  if (slot >= 0) {
    const int64_t row = slot + (int64_t(head) << a.c.page_log2);
    const int64_t from = row * kHead + lane * 8;
    if constexpr (BITS == 8) {
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
    } else if constexpr (BITS == 4) {
      const uint32_t xk = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.c.k) + from / 2);
      const uint32_t xv = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.c.v) + from / 2);
      const int64_t block = row * (kHead / kBlock) + (lane >> 2);
      k = expand8(xk, __uint_as_float(uint32_t(a.c.k_exp[block]) << 23));
      v = expand8(xv, __uint_as_float(uint32_t(a.c.v_exp[block]) << 23));
    } else {
      k = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.c.k) + from);
      v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.c.v) + from);
    }
  }
  const int64_t to = int64_t(m.r) * kHead + lane * 8;   // [q][i][head]
  *reinterpret_cast<u32x4*>(a.k_out + to) = k;
  *reinterpret_cast<u32x4*>(a.v_out + to) = v;
}

template <int BITS>
unsigned blocks_of(const CacheMoveArgs& a) {
  if (by_positions<BITS>(a)) return unsigned(int64_t(a.c.batch) * ((a.rows + 15) / 16) * a.c.heads_kv);
  return unsigned((int64_t(a.c.batch) * a.rows * a.c.heads_kv + 15) / 16);
}

template <int BITS>
hipError_t launch_write(const CacheMoveArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(cache_write<BITS>, dim3(blocks_of<BITS>(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int BITS>
hipError_t launch_read(const CacheMoveArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(cache_read<BITS>, dim3(blocks_of<BITS>(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheMoveArgs& a, hipStream_t s) {
  return a.bits == 4 ? launch_write<4>(a, s) : a.bits == 8 ? launch_write<8>(a, s) : launch_write<16>(a, s);
}

hipError_t launch_cache_read(const CacheMoveArgs& a, hipStream_t s) {
  return a.bits == 4 ? launch_read<4>(a, s) : a.bits == 8 ? launch_read<8>(a, s) : launch_read<16>(a, s);
}

}  // namespace dartree
