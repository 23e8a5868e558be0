// Rotary positions: pairs of elements of queries and keys turned by the angles of
// their row's position.
//
// A row's angles are the same for all of its heads, so a block forms them once per
// row, a pair a lane, and keeps their cosines and sines in LDS.  An angle is
// position * frequency modulo one turn: the frequency is a 64-bit fraction of a turn,
// the product wraps by itself, and its top two bits (after rounding) say the quarter.
// What is left, within an eighth of a turn of it, goes through the Taylor series of
// sine and cosine (11th and 12th order left out: 2e-9 and 2e-10), so positions of any
// size are as exact as the first ones.
//
// Bound by HBM from about a thousand rows on (8 x 2048 rows of 32 + 8 heads in bf16: 252 MB of
// a ragged batch in 45 us, 5.6 TB/s), by the launch below that (64 rows 3.9 us).  An item
// is read, turned and written before the next: four of a thread in flight took 61 us
// there, 86 for 62 with interleaved pairs.  Lengths off the vector width (V 1) go
// element by element, the copied part too: 16384 rows of 40 heads of 128, halves, in bf16 61
// us (5.5 TB/s) whole, 159 for 126 turned, 200 for 36 and 24, 213 for 2; in fp32 117, 190,
// 245 (24: 127, vectors) and 265.
#include "internal.hpp"
#include "rotary.hpp"

namespace dartree {
namespace {

constexpr int kThreads = 256;

// Sine and cosine of `turn` / 2^64 turns.
__device__ __forceinline__ void sine_cosine(uint64_t turn, float& s, float& c) {
  const uint64_t y = turn + (uint64_t(1) << 61);
  const int quarter = int(y >> 62);
  const int64_t rest = int64_t(y & ((uint64_t(1) << 62) - 1)) - (int64_t(1) << 61);
  const float a = float(double(rest) * (6.283185307179586476925 / 18446744073709551616.0));
  const float q = a * a;
  const float sn = fmaf(a * q, fmaf(q, fmaf(q, fmaf(q, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), a);
  const float cs = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float ss = quarter & 1 ? cs : sn, cc = quarter & 1 ? sn : cs;
  s = quarter & 2 ? -ss : ss;
  c = (quarter + 1) & 2 ? -cc : cc;
}

template <typename T>
__device__ __forceinline__ float value(T x) {
  return float(x);
}

// V elements of a head are V * sizeof(T) bytes, read and written at once.
template <typename T, int V>
struct alignas(V * sizeof(T)) Piece {
  T x[V];
};

// Item c < turned of a head: HALF, V elements of the first half and the same of the
// second; interleaved, V elements that are V / 2 pairs (V 1: one pair).  The items
// behind them: V elements that are copied (V 1: one).
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_rows(RotaryArgs a) {
  extern __shared__ float angles[];   // [rows of the block][cos, sin][pairs]
  const int pairs = a.rotary_dim / 2;
  const int64_t row0 = int64_t(blockIdx.x) * a.block_rows;
  const int64_t all = int64_t(a.batch) * a.rows;
  for (int i = threadIdx.x; i < a.block_rows * pairs; i += kThreads) {
    const int r = i / pairs, pair = i - r * pairs;
    const int64_t row = row0 + r;
    if (row >= all) break;
    const int q = int(row / a.rows), n = int(row - int64_t(q) * a.rows);
    const int64_t pos = int64_t(a.first) + (a.start ? a.start[q] : 0) + (a.positions ? a.positions[row] : n);
    float s, c;
    sine_cosine(uint64_t(pos) * a.turns[pair], s, c);
    angles[(2 * r) * pairs + pair] = c * a.amplitude;
    angles[(2 * r + 1) * pairs + pair] = (a.inverse ? -s : s) * a.amplitude;
  }
  __syncthreads();
  const int lanes = kThreads / a.block_rows, r = threadIdx.x / lanes;
  const int64_t row = row0 + r;
  if (row >= all) return;
  const int q = int(row / a.rows);
  if (a.counts && int(row - int64_t(q) * a.rows) >= a.counts[q]) return;
  const float* cs = angles + (2 * r) * pairs;
  const float* sn = cs + pairs;
  const int items = (a.heads_q + a.heads_kv) * a.head_items;
  for (int i = threadIdx.x - r * lanes; i < items; i += lanes) {
    const int head = a.head_items == 1 ? i : int(__umulhi(unsigned(i), a.head_magic));   // i / head_items
    const int c = i - head * a.head_items;
    const bool is_q = head < a.heads_q;
    const int h = is_q ? head : head - a.heads_q;
    const T* from = static_cast<const T*>(is_q ? a.q : a.k) + row * (is_q ? a.q_stride : a.k_stride) + h * a.head_dim;
    T* to = static_cast<T*>(is_q ? a.q_out : a.k_out) + row * (is_q ? a.q_out_stride : a.k_out_stride) + h * a.head_dim;
    typedef Piece<T, V> P;
    if (c >= a.turned) {
      const int d = a.rotary_dim + (c - a.turned) * V;
      if (from != to) *reinterpret_cast<P*>(to + d) = *reinterpret_cast<const P*>(from + d);
    } else if constexpr (HALF || V == 1) {
      const int d0 = HALF ? c * V : 2 * c, d1 = HALF ? d0 + pairs : d0 + 1;
      const P x = *reinterpret_cast<const P*>(from + d0), y = *reinterpret_cast<const P*>(from + d1);
      P u, v;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float co = cs[c * V + j], si = sn[c * V + j], xf = value(x.x[j]), yf = value(y.x[j]);
        u.x[j] = T(fmaf(xf, co, -(yf * si)));
        v.x[j] = T(fmaf(yf, co, xf * si));
      }
      *reinterpret_cast<P*>(to + d0) = u;
      *reinterpret_cast<P*>(to + d1) = v;
    } else {
      const P x = *reinterpret_cast<const P*>(from + c * V);
      P u;
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        const float co = cs[c * (V / 2) + j], si = sn[c * (V / 2) + j], xf = value(x.x[2 * j]), yf = value(x.x[2 * j + 1]);
        u.x[2 * j] = T(fmaf(xf, co, -(yf * si)));
        u.x[2 * j + 1] = T(fmaf(yf, co, xf * si));
      }
      *reinterpret_cast<P*>(to + c * V) = u;
    }
  }
}

template <typename T, int V>
hipError_t launch(RotaryArgs a, hipStream_t s) {
  const bool half = a.layout == DARTREE_ROTARY_HALF;
  const int pairs = a.rotary_dim / 2;
  a.turned = half ? pairs / V : V == 1 ? pairs : a.rotary_dim / V;
  a.head_items = a.turned + (a.head_dim - a.rotary_dim) / V;
  a.head_magic = uint32_t((uint64_t(1) << 32) / unsigned(a.head_items) + 1);   // items < 2^21, head_items <= 512
  const int64_t rows = int64_t(a.batch) * a.rows;
  // Rows of a block until its threads have two items each, four at most; one where rows are few.
  // One / two / four rows (us, bf16, halves, heads): 16384 rows of 40 60 / 61 / 64, of 5 18.2 / 13.6 /
  // 11.3, 1024 of 40 5.3 / 5.4 / 5.9, of 5 3.3 / 3.4 / 3.3; 2331 rows of 16 interleaved in fp32
  // one 9.8, four 11.5.
  const int row_items = (a.heads_q + a.heads_kv) * a.head_items;
  a.block_rows = 1;
  while (rows >= 2048 && a.block_rows < 4 && a.block_rows * row_items < 2 * kThreads) a.block_rows *= 2;
  const dim3 grid(unsigned((rows + a.block_rows - 1) / a.block_rows));
  auto* kernel = half ? rotary_rows<T, V, true> : rotary_rows<T, V, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), size_t(a.block_rows) * a.rotary_dim * sizeof(float), s, a);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_type(const RotaryArgs& a, hipStream_t s) {
  const int unit = a.layout == DARTREE_ROTARY_HALF ? 2 * V : V;
  return a.rotary_dim % unit == 0 ? launch<T, V>(a, s) : launch<T, 1>(a, s);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s) {
  return a.bf16 ? launch_type<__bf16, 8>(a, s) : launch_type<float, 4>(a, s);
}

}  // namespace dartree
