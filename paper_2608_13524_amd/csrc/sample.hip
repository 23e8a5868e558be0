// Verification of drafted tokens against the target's probabilities from given
// random numbers: trees of chosen tokens, and chains drawn from the drafter.
//
// A row of logits is cut into segments of 4096 elements (counted from the 16
// bytes its start lies in, so that every load is aligned).  A segment's record
// is its maximum, the maximum's first index and the sum of exp((z - max) / T).
// Sums are taken in 64 bits and exponentials to 3e-12: the final token is where the
// cumulated mass passes u of the whole, and with 32 bits (1e-7) one draw in
// sixty of a flat 151936-token row would land on a neighbour.  The vector units
// do 64-bit fused multiply-adds at the 32-bit rate, and ExpTable needs eleven of
// them an element, so a pass stays near the time its bytes take.
//
// Trees: with few rows the records of every row are taken at once (one pass
// over the logits, all compute units) and a block per request then walks the
// tree in LDS.  With many, only rows along the likeliest paths are read (below).
// Chains: the records of every row, then one pass over the final row.
#include <algorithm>

#include "reduce.hpp"
#include "serve.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kSeg = 4096;
constexpr int kMaxSeg = (DARTREE_MAX_VOCAB + 7 + kSeg - 1) / kSeg;
int segments(int vocab) { return (vocab + 7 + kSeg - 1) / kSeg; }

struct Record {
  float m;      // maximum (-inf: no mass)
  int32_t arg;  // its first index
  double s;     // sum of exp((z - m) / T)
};

// What blocks of one launch hand to the request's last block goes past the
// caches of a compute unit and an XCD (relaxed atomics of the device's scope), and
// a block arrives once its words are there.  A release and an acquire instead
// write back and drop a whole L2: 24.2 us for the final tokens of eight chains
// against 21.7.
__device__ __forceinline__ void hand_over(uint64_t* p, uint64_t x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t taken_over(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool arrive_last(int32_t* arrived, int blocks) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  return __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
}

// exp(x) for x <= 0 (or -inf): 2^n 2^f with |f| <= 1/2, the Taylor series of
// 2^f to degree 12 (the next term is below 2e-16).  x is given times log2(e).
__device__ __forceinline__ double exp64(double t) {
  t = fmax(t, -1200.0);   // 2^-1200 is 0 in 64 bits
  const double n = __builtin_rint(t), f = t - n;
  double p = 2.5678435993488206e-11;              // ln(2)^12 / 12!
  p = fma(p, f, 4.4455382718708115e-10);
  p = fma(p, f, 7.0549116208011233e-09);
  p = fma(p, f, 1.0178086009239699e-07);
  p = fma(p, f, 1.3215486790144307e-06);
  p = fma(p, f, 1.5252733804059841e-05);
  p = fma(p, f, 1.5403530393381608e-04);
  p = fma(p, f, 1.3333558146428443e-03);
  p = fma(p, f, 9.6181291076284772e-03);
  p = fma(p, f, 5.5504108664821580e-02);
  p = fma(p, f, 2.4022650695910071e-01);
  p = fma(p, f, 6.9314718055994531e-01);
  p = fma(p, f, 1.0);
  return __builtin_ldexp(p, int(n));
}

// 2^(i / 32)
__constant__ double kExp32[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002,
};

// The same for the many elements of a pass: exp((z - m) / T) = 2^(n / 32) 2^(f / 32),
// |f| <= 1/2, from a table in LDS (32 entries take 64 banks: no conflicts) and a
// series to degree 4 (the next term is below 2e-12).  z is at most m.
struct ExpTable {
  const double* table;   // LDS
  double c32, m;         // 32 log2(e) / T
  __device__ ExpTable(const double* t, double c, float mm) : table(t), c32(32.0 * c), m(mm) {}
  // 2^(f / 32) from t = n + f
  __device__ static double series(double t, int& n) {
    constexpr double kRound = 6755399441055744.0;   // 1.5 * 2^52: adding it leaves the nearest whole number in the low bits
    const double r = t + kRound, f = t - (r - kRound);
    n = int(uint32_t(__builtin_bit_cast(uint64_t, r)));
    double p = 9.172562701824643e-09;
    p = fma(p, f, 1.6938509724371819e-06);
    p = fma(p, f, 0.00023459619820224677);
    p = fma(p, f, 0.02166084939249829);
    return fma(p, f, 1.0);
  }
  __device__ double scaled(float z) const { return (double(z) - m) * c32; }   // the difference is exact
  // The same with one operation less, m c32 rounded first: good to 2^-34 where that
  // is below 2^20.  Takes NaN, not +inf.
  __device__ bool near() const { return m < 3.40282347e+38 && fabs(m * c32) < 1048576.0; }
  __device__ double scaled_near(float z) const { return fma(double(z), c32, -(m * c32)); }
  // Added to a sum that is at least 1: NaN and -inf give 2^-1000, nothing beside it.
  __device__ void add(double t, double& sum) const {
    int n;
    const double p = series(fmax(t, -32000.0), n);
    const uint64_t e = __builtin_bit_cast(uint64_t, table[n & 31]) + (uint64_t(uint32_t(n & ~31) << 15) << 32);
    sum = fma(__builtin_bit_cast(double, e), p, sum);
  }
  // by itself: 2^-1200 is 0 in 64 bits
  __device__ double of(float z) const {
    int n;
    const double p = series(fmax(scaled(z), -38400.0), n);
    return __builtin_ldexp(table[n & 31] * p, n >> 5);
  }
};

__device__ __forceinline__ float sane(float z) { return z != z ? -INFINITY : fminf(z, 3.40282347e+38f); }

// Row of logits as 16-byte chunks counted from the aligned address at or below
// its start: chunk c holds elements c * N - shift .. of the row.
template <bool BF>
struct RowView {
  static constexpr int N = BF ? 8 : 4;
  const char* base;   // of element 0
  int shift, vocab;
  __device__ RowView(const void* z, int64_t row, int64_t stride, int v)
      : base(static_cast<const char*>(z) + row * stride * (BF ? 2 : 4)), vocab(v) {
    shift = int((reinterpret_cast<uintptr_t>(base) & 15u) / (BF ? 2 : 4));
  }
  __device__ float at(int i) const {
    return sane(BF ? bf16_to_f32(reinterpret_cast<const uint16_t*>(base)[i]) : reinterpret_cast<const float*>(base)[i]);
  }
  // elements of chunk c (first: the index of its first); -inf where there is
  // none.  RAW: NaN and +inf as they are
  template <bool RAW = false>
  __device__ void load(int c, float (&x)[N], int& first) const {
    first = c * N - shift;
    if (first >= 0 && first + N <= vocab) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + int64_t(first) * (BF ? 2 : 4));
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = BF ? __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16) : __uint_as_float(w[BF ? 0 : i]);
        if (!RAW) x[i] = sane(x[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = first + i >= 0 && first + i < vocab ? at(first + i) : -INFINITY;
    }
  }
};

__device__ __forceinline__ double wave_sum64(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}
__device__ __forceinline__ int wave_min_int(int x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off));
  return x;
}

// A block's share of a segment in registers, and the segment's record from it
// (table: kExp32 in LDS).
template <bool BF, int NT>
struct Segment {
  static constexpr int N = RowView<BF>::N, L = kSeg / N / NT;
  float x[L][N];
  int first[L];
  __device__ void load(const RowView<BF>& z, int seg) {
#pragma unroll
    for (int l = 0; l < L; ++l) z.template load<true>(seg * (kSeg / N) + l * NT + threadIdx.x, x[l], first[l]);
  }
};
template <bool BF, int NT>
__device__ __forceinline__ void segment_record(const Segment<BF, NT>& in, const double* table, double c, Record* out) {
  constexpr int N = RowView<BF>::N, L = kSeg / N / NT, W = NT / 64;
  __shared__ float sm[W];
  __shared__ int sa[W];
  __shared__ double ss[W];
  const auto& x = in.x;
  const auto& first = in.first;
  float m = -INFINITY;
#pragma unroll
  for (int l = 0; l < L; ++l)
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[l][i]);   // passes over NaN
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  m = wave_max(m);
  if (lane == 0) sm[wave] = m;
  __syncthreads();
  m = sm[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, sm[w]);
  m = fminf(m, 3.40282347e+38f);
  int arg = INT32_MAX;
  double s = 0.0;
  if (m != -INFINITY) {
    if (c == 0.0) {
#pragma unroll
      for (int l = 0; l < L; ++l)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[l][i] >= m) arg = min(arg, first[l] + i);
    } else {
      const ExpTable e(table, c, m);
      if (e.near()) {
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
          for (int i = 0; i < N; ++i) e.add(e.scaled_near(x[l][i]), s);
      } else {   // +inf counts as the largest number
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
          for (int i = 0; i < N; ++i) e.add(e.scaled(sane(x[l][i])), s);
      }
    }
  }
  if (c == 0.0) {
    arg = wave_min_int(arg);
    if (lane == 0) sa[wave] = arg;
  } else {
    s = wave_sum64(s);
    if (lane == 0) ss[wave] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Record r;
    r.m = m;
    r.arg = c == 0.0 ? sa[0] : 0;
    r.s = c == 0.0 ? 0.0 : ss[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      if (c == 0.0) r.arg = min(r.arg, sa[w]);
      else r.s += ss[w];
    }
    *out = r;
  }
}

// A row's records joined by 8 lanes (kJoin); the same in each.
constexpr int kJoin = 8;
__device__ __forceinline__ Record join_records(const Record* rec, int nseg, double c) {
  constexpr int H = 5;   // records at a time: 8 x 5 are those of 163840 tokens
  const int l = threadIdx.x & (kJoin - 1);
  Record r{-INFINITY, INT32_MAX, 0.0};
  for (int i0 = l; i0 < nseg; i0 += kJoin * H) {
    Record o[H];
    float m = r.m;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      o[h] = rec[min(i0 + kJoin * h, nseg - 1)];
      if (i0 + kJoin * h >= nseg) o[h].m = -INFINITY;
      m = fmaxf(m, o[h].m);
    }
    if (m == -INFINITY) continue;
    if (m > r.m) {
      r.s = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - double(m)) * c);
      r.arg = INT32_MAX;
      r.m = m;
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (o[h].m != -INFINITY) {
        if (o[h].m == m) r.arg = min(r.arg, o[h].arg);
        r.s += o[h].s * exp64((double(o[h].m) - double(m)) * c);
      }
  }
  float m = r.m;
#pragma unroll
  for (int off = 1; off < kJoin; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));
  if (m == -INFINITY) return r;
  if (r.m != m) r.arg = INT32_MAX;
  r.s = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - double(m)) * c);
  r.m = m;
#pragma unroll
  for (int off = 1; off < kJoin; off <<= 1) {   // a sum of the same two numbers on both sides
    r.arg = min(r.arg, __shfl_xor(r.arg, off));
    r.s += __shfl_xor(r.s, off);
  }
  return r;
}

// The distribution of a row: weight of a logit, its share of the whole.
struct Law {
  double m, s, c;   // c: log2(e) / T, 0 at T = 0
  int arg;
  __device__ Law(const Record& r, double cc) : m(r.m), s(r.s), c(cc), arg(r.arg) {}
  __device__ bool empty() const { return m == -INFINITY; }
  __device__ double weight(float z, int i) const {   // unnormalised, at most 1
    return c == 0.0 ? (i == arg ? 1.0 : 0.0) : exp64((double(z) - m) * c);
  }
  __device__ double share(float z, int i) const { return empty() ? 0.0 : c == 0.0 ? weight(z, i) : weight(z, i) / s; }
};

// The first token whose cumulated weight passes `target` in segment `seg`,
// by a block of NT threads; `weight(c, w)` gives the weights of chunk c (w[i] of
// element first + i, 0 where there is none) and returns first.  -1 if none does
// and, in *last, the segment's last token of positive weight (-1: none).
template <int NT, int N, typename F>
__device__ __forceinline__ int pick_in_segment(int seg, double target, F&& weight, int* last) {
  constexpr int kChunks = kSeg / N, kEach = kChunks > NT ? kChunks / NT : 1;   // consecutive chunks per thread
  __shared__ double wsum[NT / 64];
  __shared__ int got[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) {
    got[0] = INT32_MAX;
    got[1] = -1;
  }
  double w[kEach][N], sum = 0.0;
  int first[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int c = int(threadIdx.x) * kEach + k;
    first[k] = 0;
    if (c < kChunks) {
      first[k] = weight(seg * kChunks + c, w[k]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) w[k][i] = 0.0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum += w[k][i];
  }
  double incl = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  double cum = incl - sum;
#pragma unroll
  for (int x = 0; x < NT / 64; ++x) {   // all read at once
    const double o = wsum[x];
    cum += x < wave ? o : 0.0;
  }
  int found = INT32_MAX, pos = -1;
#pragma unroll
  for (int k = 0; k < kEach; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      cum += w[k][i];
      if (w[k][i] > 0.0) {
        pos = first[k] + i;
        if (found == INT32_MAX && cum > target) found = pos;
      }
    }
  // a wave's tokens rise with its lanes; whole numbers: the order of waves does not matter
  const uint64_t hit = __ballot(found != INT32_MAX), some = __ballot(pos >= 0);
  if (hit && lane == __builtin_ctzll(hit)) atomicMin(&got[0], found);
  if (some && lane == 63 - __builtin_clzll(some)) atomicMax(&got[1], pos);
  __syncthreads();
  const int r = got[0];
  *last = got[1];
  __syncthreads();
  return r == INT32_MAX ? -1 : r;
}

// The weight of a segment, in every thread of the block.
template <int NT, int N, typename F>
__device__ __forceinline__ double segment_weight(int seg, F&& weight) {
  __shared__ double wsum[NT / 64];
  double sum = 0.0;
  for (int c = threadIdx.x; c < kSeg / N; c += NT) {
    double w[N];
    weight(seg * (kSeg / N) + c, w);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += w[i];
  }
  sum = wave_sum64(sum);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) wsum[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < NT / 64; ++w) sum += wsum[w];
  return sum;
}

// The first token whose cumulated weight passes u of the whole, given the
// segments' weights in LDS (block-uniform result; -1: no weight at all).
template <int NT, int N, typename F>
__device__ __forceinline__ int pick(const double* seg_weight, int nseg, float u, F&& weight) {
  __shared__ double target;
  __shared__ int chosen;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x, each = (nseg + 63) / 64;
    double sum = 0.0;
    for (int k = 0; k < each; ++k) {
      const int s = lane * each + k;
      if (s < nseg) sum += seg_weight[s];
    }
    double incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const double o = __shfl_up(incl, off);
      if (lane >= off) incl += o;
    }
    const double t = double(u) * __shfl(incl, 63);
    const uint64_t past = __ballot(incl > t);
    if (lane == 0) chosen = -1;
    if (past && lane == __builtin_ctzll(past)) {
      double cum = incl - sum;
      for (int k = 0; k < each; ++k) {
        const int s = lane * each + k;
        if (s >= nseg || !(seg_weight[s] > 0.0)) continue;
        chosen = s;   // the last of positive weight if the sums round differently
        target = t - cum;
        cum += seg_weight[s];
        if (cum > t) break;
      }
    }
  }
  __syncthreads();
  const int sg = chosen;
  int last = -1;
  if (sg >= 0) {
    const int got = pick_in_segment<NT, N>(sg, target, weight, &last);
    if (got >= 0) return got;
    if (last >= 0) return last;   // a sum rounded differently: the segment's last token
  }
  // u at or past 1 (or not a number): the row's last token of positive weight
  for (int s = nseg - 1; s >= 0 && last < 0; --s) {
    const int got = pick_in_segment<NT, N>(s, INFINITY, weight, &last);
    if (got >= 0) return got;
  }
  return last;
}

// ---------------------------------------------------------------------------
// Records
// ---------------------------------------------------------------------------

// Every row of z, then those of y: block (row, segment).
template <bool BF>
__global__ __launch_bounds__(256) void row_records(const void* z, int64_t zrows, const void* y, int64_t stride, int vocab, int nseg,
                                                   double c, Record* rec, int32_t* counters, int ncounters) {
  if (blockIdx.x == 0)   // for the next launch
    for (int i = threadIdx.x; i < ncounters; i += 256) counters[i] = 0;
  const int row = blockIdx.x / nseg, seg = blockIdx.x - row * nseg;
  const RowView<BF> v(row < zrows ? z : y, row < zrows ? row : row - zrows, stride, vocab);
  __shared__ double table[32];
  Segment<BF, 256> s;
  s.load(v, seg);
  if (threadIdx.x < 32) table[threadIdx.x] = kExp32[threadIdx.x];   // read after a barrier
  segment_record<BF, 256>(s, table, c, rec + blockIdx.x);
}

// ---------------------------------------------------------------------------
// Trees
// ---------------------------------------------------------------------------

// The final token of row `row` without the tokens of `gone` (LDS; the shares of the
// first kShares in `share`), by a block of NT threads.
constexpr int kShares = 64;
template <bool BF, int NT>
__device__ int final_token(const VerifyArgs& a, int64_t row, const Record* rec, int nseg, const Law& law, const int32_t* gone,
                           const double* share, int ngone, float u, double* segw, const double* table) {
  constexpr int N = RowView<BF>::N;
  const RowView<BF> z(a.target, row, a.row_stride, a.vocab);
  if (law.empty()) return -1;
  if (law.c == 0.0) return law.arg;   // all of the mass on one token: it remains, or nothing does and p decides
  const ExpTable e(table, law.c, float(law.m));
  for (int pass = 0; pass < 2; ++pass) {   // second: nothing was left of p
    const int n = pass == 0 ? ngone : 0;
    bool again = false;
    for (int s = threadIdx.x; s < nseg; s += NT) {
      const Record r = rec[s];
      const double all = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - law.m) * law.c);
      double w = all;
      bool many = false;
      for (int i = 0; i < n; ++i) {
        if ((gone[i] + z.shift) / kSeg != s) continue;
        if (i < kShares) w -= share[i] * law.s;
        else many = true;
      }
      // little is left of a sum, or its tokens' shares are not at hand: add it up again
      const bool redo = many || (w != all && w <= 1e-4 * all);
      segw[s] = redo ? -1.0 : w;
      again |= redo;
    }
    auto weight = [&](int chunk, double (&w)[N]) {
      float x[N];
      int first;
      z.load(chunk, x, first);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = x[i] == -INFINITY ? 0.0 : e.of(x[i]);
      for (int k = 0; k < n; ++k) {
        const int d = gone[k] - first;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (d == i) w[i] = 0.0;
      }
      return first;
    };
    if (__syncthreads_or(again))
      for (int s = 0; s < nseg; ++s)
        if (segw[s] < 0.0) {   // the same for all threads
          const double w = segment_weight<NT, N>(s, weight);
          if (threadIdx.x == 0) segw[s] = w;
        }
    const int t = pick<NT, N>(segw, nseg, u, weight);
    if (t >= 0) return t;
    __syncthreads();
  }
  return -1;
}

constexpr int kWalkNodes = 1024;   // nodes of a tree walked in LDS, and threads of its block

// All rows' records at hand: a block per request.
template <bool BF>
__global__ __launch_bounds__(kWalkNodes) void tree_walk(VerifyArgs a, int nseg, double c, const Record* rec) {
  __shared__ int32_t tok[kWalkNodes], par[kWalkNodes];
  __shared__ float us[kWalkNodes];
  __shared__ double share[kWalkNodes];
  __shared__ float rm[kWalkNodes + 1];
  __shared__ int32_t rarg[kWalkNodes + 1];
  __shared__ double rs[kWalkNodes + 1];
  __shared__ double segw[kMaxSeg], table[32];
  __shared__ int at_s, tested_s;
  const int q = blockIdx.x, B = a.budget;
  const int n = min(max(a.num_nodes[q], 0), B);
  const int lane = threadIdx.x & 63;
  const Record* qrec = rec + int64_t(q) * (B + 1) * nseg;
  if (threadIdx.x < 32) table[threadIdx.x] = kExp32[threadIdx.x];
  // the drafted tokens' logits, then the rows' laws, then the tokens' shares
  const int j = threadIdx.x;
  float zj = -INFINITY;
  if (j < n) {
    const int t = a.tokens[int64_t(q) * B + j], p = a.parents[int64_t(q) * B + j];
    tok[j] = t;
    par[j] = p;
    us[j] = a.uniforms[int64_t(q) * (B + 1) + j + 1];
    if (p >= -1 && p < n && t >= 0 && t < a.vocab)
      zj = RowView<BF>(a.target, int64_t(q) * (B + 1) + p + 1, a.row_stride, a.vocab).at(t);
  }
  for (int row = threadIdx.x / kJoin; row <= n; row += kWalkNodes / kJoin) {
    const Record r = join_records(qrec + int64_t(row) * nseg, nseg, c);
    if (threadIdx.x % kJoin == 0) {
      rm[row] = r.m;
      rarg[row] = r.arg;
      rs[row] = r.s;
    }
  }
  __syncthreads();
  if (j < n) {
    const int p = par[j], t = tok[j];
    share[j] = p >= -1 && p < n && t >= 0 && t < a.vocab ? Law(Record{rm[p + 1], rarg[p + 1], rs[p + 1]}, c).share(zj, t) : 0.0;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    int at = -1, count = 0;
    bool tested = false;
    const int steps = min(a.max_len, n);
    while (count < steps) {
      double taken = 0.0;
      int next = -1;
      tested = true;
      for (int j0 = 0; j0 < n && next < 0; j0 += 64) {
        uint64_t kids = __ballot(j0 + lane < n && par[j0 + lane] == at);
        while (kids) {
          const int j = j0 + __builtin_ctzll(kids);
          kids &= kids - 1;
          if (double(us[j]) * (1.0 - taken) < share[j]) {
            next = j;
            break;
          }
          taken += share[j];
        }
      }
      if (next < 0) break;
      if (lane == 0) a.accepted[int64_t(q) * a.max_len + count] = next;
      at = next;
      ++count;
      tested = false;
    }
    for (int j = count + lane; j < a.max_len; j += 64) a.accepted[int64_t(q) * a.max_len + j] = -1;
    if (lane == 0) {
      at_s = at;
      tested_s = tested;
      a.num_accepted[q] = count;
    }
    // the tested children's tokens and shares, gathered where the tree's were
    int m = 0;
    for (int j0 = 0; j0 < n && tested; j0 += 64) {
      const bool kid = j0 + lane < n && par[j0 + lane] == at && tok[j0 + lane] >= 0 && tok[j0 + lane] < a.vocab;
      const int t = kid ? tok[j0 + lane] : 0;
      const double s = kid ? share[j0 + lane] : 0.0;
      const uint64_t b = __ballot(kid);
      if (kid) {
        tok[m + __popcll(b & ((1ull << lane) - 1))] = t;
        share[m + __popcll(b & ((1ull << lane) - 1))] = s;
      }
      m += __popcll(b);
    }
    if (lane == 0) tested_s = m;
  }
  __syncthreads();
  const int at = at_s;
  const Law law(Record{rm[at + 1], rarg[at + 1], rs[at + 1]}, c);
  const int t = final_token<BF, kWalkNodes>(a, int64_t(q) * (B + 1) + at + 1, qrec + int64_t(at + 1) * nseg, nseg, law, tok, share, tested_s,
                                a.uniforms[int64_t(q) * (B + 1)], segw, table);
  if (threadIdx.x == 0) a.bonus[q] = t;
}

// Many rows: only those on the likeliest path are read.  Per request, the drafted
// tokens' logits give every node its best child without any row's law; the rows
// along the best children from the current node are read in one launch, and a
// walk goes on until it leaves them.  kRounds of that, the first with the few rows
// that most trees end in, and the last walk reads the rows it still lacks by
// itself (a block per request, 45 us a row of 151936): a target that agrees with the
// drafter leaves the best children seldom (by_path has both kinds).  16 trees of 512 nodes of depth 16, vocab
// 151936 fp32: 2 rounds of 17 rows 83.9 us, of 8 and 17 88.2, a third round 78.4,
// a fourth 82.9.  One node a launch, its last block walking on, took 194.
constexpr int kFirstRows = 8;   // rows of the first round
constexpr int kPathRows = 32;   // and of the others
constexpr int kRounds = 3;
constexpr int kPathThreads = 1024;

struct Walk {
  int32_t at, count, done, len;   // current node, accepted nodes, rows of the path to read
  int32_t path[kPathRows];
};

// The rows from the current node along the best children (child[row]: best child
// of the node of that row, -1: none), at most as many as can still be accepted.
__device__ __forceinline__ void plan_path(Walk* w, int at, int count, int rows, int max_len, const int32_t* child) {
  int len = 0, row = at + 1;
  while (true) {
    w->path[len++] = row;
    if (len == rows || count + len > max_len) break;
    const int c = child[row];
    if (c < 0) break;
    row = c + 1;
  }
  w->at = at;
  w->count = count;
  w->done = 0;
  w->len = len;
}

// Block per request: the drafted tokens' logits zd [b][B], every row's best child
// [b][B+1] (the largest logit, the lowest index among equals), the first path.
template <bool BF>
__global__ __launch_bounds__(kPathThreads) void path_begin(VerifyArgs a, Walk* walk, float* zd, int32_t* child) {
  __shared__ unsigned long long best[DARTREE_MAX_SORT + 1];
  __shared__ int32_t kid[DARTREE_MAX_SORT + 1];
  const int q = blockIdx.x, B = a.budget, n = min(max(a.num_nodes[q], 0), B);
  for (int r = threadIdx.x; r <= n; r += kPathThreads) best[r] = 0;
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += kPathThreads) {
    const int t = a.tokens[int64_t(q) * B + j], p = a.parents[int64_t(q) * B + j];
    float z = -INFINITY;
    if (p >= -1 && p < n && t >= 0 && t < a.vocab) {
      z = RowView<BF>(a.target, int64_t(q) * (B + 1) + p + 1, a.row_stride, a.vocab).at(t);
      // a key is never 0, and a maximum does not depend on the order
      atomicMax(&best[p + 1], (unsigned long long)rank_key(z, j));
    }
    zd[int64_t(q) * B + j] = z;
  }
  __syncthreads();
  for (int r = threadIdx.x; r <= n; r += kPathThreads) {
    const int c = best[r] ? key_id(best[r]) : -1;
    kid[r] = c == r - 1 ? -1 : c;   // not itself
    child[int64_t(q) * (B + 1) + r] = kid[r];
  }
  __syncthreads();
  if (threadIdx.x == 0) plan_path(walk + q, -1, 0, kFirstRows, min(a.max_len, n), kid);
}

// The records of the paths' rows: block (request, row of its path, segment).
template <bool BF>
__global__ __launch_bounds__(256) void path_records(VerifyArgs a, int nseg, int rows, int nrows, double c, const Walk* walk, Record* rec) {
  __shared__ double table[32];
  const int seg = blockIdx.x % nseg, i = blockIdx.x / nseg % rows, q = blockIdx.x / nseg / rows;
  if (walk[q].done || i >= walk[q].len) return;
  if (threadIdx.x < 32) table[threadIdx.x] = kExp32[threadIdx.x];   // read after a barrier
  const RowView<BF> z(a.target, int64_t(q) * (a.budget + 1) + walk[q].path[i], a.row_stride, a.vocab);
  Segment<BF, 256> s;
  s.load(z, seg);
  segment_record<BF, 256>(s, table, c, rec + (int64_t(q) * nrows + i) * nseg + seg);
}

// A segment's record by one wave, in one pass: every lane keeps the maximum of its
// elements and the sum beside it.
template <bool BF>
__device__ __forceinline__ void wave_record(const RowView<BF>& z, int seg, const double* table, double c, Record* out) {
  constexpr int N = RowView<BF>::N, L = kSeg / N / 64, H = 16 / N;
  float m = -INFINITY;
  int arg = INT32_MAX;
  double s = 0.0;
#pragma unroll 1
  for (int l = 0; l < L; l += H) {
    float x[H][N], top = m;
    int first[H];
#pragma unroll
    for (int h = 0; h < H; ++h) z.load(seg * (kSeg / N) + (l + h) * 64 + (threadIdx.x & 63), x[h], first[h]);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, x[h][i]);
    if (top == -INFINITY) continue;
    if (top > m) {
      s = m == -INFINITY ? 0.0 : s * exp64((double(m) - double(top)) * c);
      arg = INT32_MAX;
      m = top;
    }
    const ExpTable e(table, c, m);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (c == 0.0) arg = x[h][i] == m ? min(arg, first[h] + i) : arg;
        else e.add(e.scaled(x[h][i]), s);
      }
  }
  const float whole = wave_max(m);
  if (m != whole) {
    s = m == -INFINITY ? 0.0 : s * exp64((double(m) - double(whole)) * c);
    arg = INT32_MAX;
  }
  if (c == 0.0) arg = wave_min_int(arg);
  else s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) *out = Record{whole, c == 0.0 ? arg : 0, s};
}

// The first child of `at` whose token is taken, -1: none (one wave).  FILL: the
// children's tokens and shares are gathered, m of them.
template <bool FILL>
__device__ __forceinline__ int test_children(const Law& law, int at, int n, int vocab, const int32_t* tok, const int32_t* par,
                                             const float* us, const float* zs, int32_t* gone, double* share, int& m) {
  const int lane = threadIdx.x & 63;
  double taken = 0.0;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const bool is = j < n && par[j] == at;
    uint64_t kids = __ballot(is);
    if (!kids) continue;
    const int t = is ? tok[j] : -1;
    const bool in = t >= 0 && t < vocab;
    const double s = in ? law.share(zs[j], t) : 0.0;
    if (FILL) {
      const uint64_t b = __ballot(in);
      const int to = m + __popcll(b & ((1ull << lane) - 1));
      if (in) gone[to] = t;
      if (in && to < kShares) share[to] = s;
      m += __popcll(b);
      continue;
    }
    const float u = is ? us[j] : 0.f;
    while (kids) {
      const int l = __builtin_ctzll(kids);
      kids &= kids - 1;
      const double sl = __shfl(s, l);
      if (double(__shfl(u, l)) * (1.0 - taken) < sl) return j0 + l;
      taken += sl;
    }
  }
  return -1;
}

// Block per request: walk as far as the path's rows reach, LAST: to the end.  The
// children of all rows on the path are tested at once, a wave per row; the walk is
// then a few steps in LDS (16 trees of 512 nodes: 15 us; one wave that goes from
// node to node takes 26).
template <bool BF, bool LAST>
__global__ __launch_bounds__(kPathThreads) void path_walk(VerifyArgs a, int nseg, int nrows, double c, Walk* walk, Record* rec,
                                                          const float* zd, const int32_t* child) {
  __shared__ int32_t tok[DARTREE_MAX_SORT], par[DARTREE_MAX_SORT], kid[DARTREE_MAX_SORT + 1], gone[DARTREE_MAX_SORT];
  __shared__ float us[DARTREE_MAX_SORT], zs[DARTREE_MAX_SORT];
  __shared__ float rm[kPathRows];
  __shared__ int32_t rarg[kPathRows], path[kPathRows], next[kPathRows];
  __shared__ double rs[kPathRows], share[kShares], table[32], segw[kMaxSeg];
  __shared__ int ngone;
  const int q = blockIdx.x, B = a.budget, wave = threadIdx.x >> 6;
  Walk& w = walk[q];
  if (w.done) return;
  const int n = min(max(a.num_nodes[q], 0), B);
  Record* qrec = rec + int64_t(q) * nrows * nseg;
  int len = w.len, at = w.at, count = w.count;
  for (int i = threadIdx.x; i < len; i += kPathThreads) path[i] = w.path[i];
  for (int j = threadIdx.x; j < n; j += kPathThreads) {
    tok[j] = a.tokens[int64_t(q) * B + j];
    par[j] = a.parents[int64_t(q) * B + j];
    us[j] = a.uniforms[int64_t(q) * (B + 1) + j + 1];
    zs[j] = zd[int64_t(q) * B + j];
  }
  if (!LAST)
    for (int r = threadIdx.x; r <= n; r += kPathThreads) kid[r] = child[int64_t(q) * (B + 1) + r];
  if (threadIdx.x < 32) table[threadIdx.x] = kExp32[threadIdx.x];
  const int steps = min(a.max_len, n);
  int slot, m = 0;
  while (true) {   // once, and again for each row that LAST reads; a turn accepts a node or ends
    for (int i = threadIdx.x / kJoin; i < len; i += kPathThreads / kJoin) {
      const Record r = join_records(qrec + int64_t(i) * nseg, nseg, c);
      if (threadIdx.x % kJoin == 0) {
        rm[i] = r.m;
        rarg[i] = r.arg;
        rs[i] = r.s;
      }
    }
    __syncthreads();
    for (int i = wave; i < len; i += kPathThreads / 64) {
      int none = 0;
      const int j = count + i < steps
                        ? test_children<false>(Law(Record{rm[i], rarg[i], rs[i]}, c), path[i] - 1, n, a.vocab, tok, par, us, zs, gone, share, none)
                        : -1;
      if ((threadIdx.x & 63) == 0) next[i] = j;
    }
    __syncthreads();
    // the same by every thread
    for (slot = 0;;) {
      const int j = next[slot];
      if (j < 0) break;
      if (threadIdx.x == 0) a.accepted[int64_t(q) * a.max_len + count] = j;
      at = j;
      ++count;
      if (slot + 1 == len || path[slot + 1] != at + 1) {
        slot = -1;   // off the path
        break;
      }
      ++slot;
    }
    if (slot >= 0) break;
    if (!LAST) {
      if (threadIdx.x == 0) plan_path(&w, at, count, kPathRows, steps, kid);
      return;
    }
    const RowView<BF> z(a.target, int64_t(q) * (B + 1) + at + 1, a.row_stride, a.vocab);
    for (int s = wave; s < nseg; s += kPathThreads / 64) wave_record<BF>(z, s, table, c, qrec + s);
    __syncthreads();
    if (threadIdx.x == 0) path[0] = at + 1;
    len = 1;
  }
  const Law law(Record{rm[slot], rarg[slot], rs[slot]}, c);
  if (wave == 0) {
    if (count < steps) test_children<true>(law, at, n, a.vocab, tok, par, us, zs, gone, share, m);
    if (threadIdx.x == 0) ngone = m;
  }
  for (int j = count + threadIdx.x; j < a.max_len; j += kPathThreads) a.accepted[int64_t(q) * a.max_len + j] = -1;
  __syncthreads();
  const int t = final_token<BF, kPathThreads>(a, int64_t(q) * (B + 1) + at + 1, qrec + int64_t(slot) * nseg, nseg, law, gone, share,
                                              ngone, a.uniforms[int64_t(q) * (B + 1)], segw, table);
  if (threadIdx.x == 0) {
    a.num_accepted[q] = count;
    a.bonus[q] = t;
    w.done = 1;
  }
}

// ---------------------------------------------------------------------------
// Chains
// ---------------------------------------------------------------------------

constexpr int kPick = 512;   // threads of the blocks below

// Laws of the rows of a request's chain in LDS, and how many tokens pass.
struct ChainRows {
  float m[2 * DARTREE_MAX_DEPTH + 1];
  int32_t arg[2 * DARTREE_MAX_DEPTH + 1];
  double s[2 * DARTREE_MAX_DEPTH + 1];
  int count;
};
template <bool BF>
__device__ __forceinline__ int chain_walk(const VerifyArgs& a, int nseg, double c, const Record* trec, const Record* drec,
                                          ChainRows& rows) {
  const int q = blockIdx.y, D = a.budget;
  const int n = a.num_nodes ? min(max(a.num_nodes[q], 0), D) : D;
  // thread i: token i's logits and random number, while the rows' records arrive
  const int i = threadIdx.x;
  int tok = -1;
  float zt = -INFINITY, yt = -INFINITY, u = 0.f;
  if (i < n) {
    tok = a.tokens[int64_t(q) * D + i];
    if (tok >= 0 && tok < a.vocab) {
      zt = RowView<BF>(a.target, int64_t(q) * (D + 1) + i, a.row_stride, a.vocab).at(tok);
      if (c != 0.0) yt = RowView<BF>(a.draft, int64_t(q) * D + i, a.row_stride, a.vocab).at(tok);
    }
    u = a.uniforms[int64_t(q) * (D + 1) + i + 1];
  }
  const int nrow = c == 0.0 ? n + 1 : 2 * n + 1;   // target rows 0 .. n, then the draft's 0 .. n - 1
  for (int row = threadIdx.x / kJoin; row < nrow; row += kPick / kJoin) {
    const Record* at = row <= n ? trec + (int64_t(q) * (D + 1) + row) * nseg : drec + (int64_t(q) * D + row - n - 1) * nseg;
    const Record r = join_records(at, nseg, c);
    if (threadIdx.x % kJoin == 0) {
      rows.m[row] = r.m;
      rows.arg[row] = r.arg;
      rows.s[row] = r.s;
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    bool pass = false;
    if (i < n && tok >= 0 && tok < a.vocab) {
      const double px = Law(Record{rows.m[i], rows.arg[i], rows.s[i]}, c).share(zt, tok);
      const int d = n + 1 + i;
      pass = c == 0.0 ? px > 0.0 : double(u) * Law(Record{rows.m[d], rows.arg[d], rows.s[d]}, c).share(yt, tok) < px;
    }
    const uint64_t stop = __ballot(!pass);   // bits at and past n are set, unless n = 64
    if (i == 0) rows.count = stop ? min(__builtin_ctzll(stop), n) : n;
  }
  __syncthreads();
  return n;
}

// Weight of the final token's law: [p - q]_+ after a rejection, p after the last token.
template <bool BF>
struct Residual {
  static constexpr int N = RowView<BF>::N;
  RowView<BF> z, y;
  Law p, q;
  ExpTable ep, eq;
  double pn, qn;   // 1 / their wholes
  bool reject;
  __device__ int operator()(int chunk, double (&w)[N]) const {
    float x[N];
    int first;
    z.load(chunk, x, first);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i] == -INFINITY ? 0.0 : ep.of(x[i]);
    if (reject) {
      float v[N];
      if (y.shift == z.shift) {
        int f;
        y.load(chunk, v, f);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = first + i >= 0 && first + i < y.vocab ? y.at(first + i) : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < N; ++i)
        w[i] = fmax(w[i] * pn - (q.empty() || v[i] == -INFINITY ? 0.0 : eq.of(v[i]) * qn), 0.0);
    }
    return first;
  }
};
template <bool BF>
__device__ __forceinline__ Residual<BF> residual_of(const VerifyArgs& a, double c, const ChainRows& rows, int n, const double* table) {
  const int q = blockIdx.y, D = a.budget, k = rows.count;
  const bool reject = k < n && c != 0.0;
  const int d = reject ? n + 1 + k : 0;
  return Residual<BF>{RowView<BF>(a.target, int64_t(q) * (D + 1) + k, a.row_stride, a.vocab),
                      RowView<BF>(a.draft, reject ? int64_t(q) * D + k : 0, a.row_stride, a.vocab),
                      Law(Record{rows.m[k], rows.arg[k], rows.s[k]}, c), Law(Record{rows.m[d], rows.arg[d], rows.s[d]}, c),
                      ExpTable(table, c, rows.m[k]), ExpTable(table, c, rows.m[d]), 1.0 / rows.s[k], 1.0 / rows.s[d], reject};
}

// The final token: block (segment, request).  After a rejection every block
// takes its segment's weight of [p - q]_+ and a request's last block to arrive
// draws; otherwise the first block draws from p by its records.
template <bool BF>
__global__ __launch_bounds__(kPick) void chain_final(VerifyArgs a, int nseg, double c, const Record* trec, const Record* drec,
                                                     uint64_t* segw, int32_t* arrived) {
  constexpr int N = RowView<BF>::N;
  __shared__ ChainRows rows;
  __shared__ double sw[kMaxSeg], table[32];
  __shared__ int last_s;
  const int q = blockIdx.y, D = a.budget;
  if (threadIdx.x < 32) table[threadIdx.x] = kExp32[threadIdx.x];
  const int n = chain_walk<BF>(a, nseg, c, trec, drec, rows);
  Residual<BF> f = residual_of<BF>(a, c, rows, n, table);
  int t = -1;
  if (f.reject && !f.p.empty()) {
    const double sum = segment_weight<kPick, N>(blockIdx.x, f);
    if (threadIdx.x == 0) {
      hand_over(segw + int64_t(q) * nseg + blockIdx.x, __builtin_bit_cast(uint64_t, sum));
      last_s = arrive_last(arrived + q, nseg);
    }
    __syncthreads();
    if (!last_s) return;
    for (int s = threadIdx.x; s < nseg; s += kPick) sw[s] = __builtin_bit_cast(double, taken_over(segw + int64_t(q) * nseg + s));
    t = pick<kPick, N>(sw, nseg, a.uniforms[int64_t(q) * (D + 1)], f);
  } else if (blockIdx.x > 0) {
    return;
  }
  if (t < 0 && !f.p.empty()) {   // after the last token, or nothing left of p
    if (c == 0.0) {
      t = f.p.arg;
    } else {
      f.reject = false;
      const Record* rec = trec + (int64_t(q) * (D + 1) + rows.count) * nseg;
      __syncthreads();
      for (int s = threadIdx.x; s < nseg; s += kPick) {
        const Record r = rec[s];
        sw[s] = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - f.p.m) * c);
      }
      t = pick<kPick, N>(sw, nseg, a.uniforms[int64_t(q) * (D + 1)], f);
    }
  }
  if (threadIdx.x == 0) {
    a.num_accepted[q] = rows.count;
    a.bonus[q] = t;
  }
}

constexpr size_t kAlign = 256;
size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// Rows of a request's path in a round, and whether to go by paths.  The rows along
// the best children are read together, but after kRounds departures from them a
// block reads each further row by itself, 45 us at a vocabulary of 151936.  So the
// gain depends on the target: every row / by paths (us, path_rows 17, fp32), where it
// follows the best child 85 % of the time, and where every node has two children
// that hold 95 % in equal parts (full trees):
//   batch x nodes x vocab, unread            best child    equal children
//   1 x 64 x 151936, 29 MB                    25 / 28         24 / 53
//   16 x 64 x 32000, 98 MB                    43 / 44         43 / 93
//   4 x 64 x 151936, 117 MB                   52 / 45         51 / 101
//   6 x 64 x 151936, 175 MB                   75 / 44         65 / 129
//   8 x 64 x 151936, 233 MB                   87 / 51         87 / 146
//   1 x 512 x 151936, 301 MB                  94 / 26         95 / 155
//   16 x 64 x 151936, 466 MB                 164 / 60        160 / 178
//   4 x 512 x 151936, 1.2 GB                 294 / 52        293 / 263
//   16 x 512 x 151936, 4.8 GB               1200 / 77       1200 / 344
// Past the border, 150 MB, the one gains about the factor that the other loses (as fp32:
// the workspace is sized without the type).  The worst walk, 16 accepted nodes that
// are none of them their parent's best child, takes 630 to 700 us at this vocabulary and
// 240 to 270 at 32000.
int path_rows(int budget, int max_len) { return std::min({kPathRows, max_len + 1, budget + 1}); }
bool by_path(int batch, int budget, int max_len, int vocab) {
  return budget > kWalkNodes || 4.0 * vocab * batch * (budget + 1 - path_rows(budget, max_len)) > 150e6;
}
struct PathLayout {
  size_t walk, zd, child, rec, total;
};
PathLayout path_layout(int batch, int budget, int max_len, int vocab) {
  const size_t b = batch, B = budget;
  PathLayout l{};
  l.zd = up(b * sizeof(Walk));
  l.child = l.zd + up(b * B * sizeof(float));
  l.rec = l.child + up(b * (B + 1) * sizeof(int32_t));
  l.total = l.rec + up(b * path_rows(budget, max_len) * segments(vocab) * sizeof(Record));
  return l;
}

template <bool BF>
hipError_t tree(const VerifyArgs& a, hipStream_t s) {
  const int nseg = segments(a.vocab);
  const double c = a.inv_t * 1.4426950408889634;
  hipError_t e;
  if (!by_path(a.batch, a.budget, a.max_len, a.vocab)) {
    Record* rec = static_cast<Record*>(a.ws);
    const int64_t rows = int64_t(a.batch) * (a.budget + 1);
    hipLaunchKernelGGL(row_records<BF>, dim3(unsigned(rows * nseg)), dim3(256), 0, s, a.target, rows, nullptr, a.row_stride,
                       a.vocab, nseg, c, rec, nullptr, 0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(tree_walk<BF>, dim3(a.batch), dim3(kWalkNodes), 0, s, a, nseg, c, rec);
    return hipGetLastError();
  }
  const PathLayout l = path_layout(a.batch, a.budget, a.max_len, a.vocab);
  const int nrows = path_rows(a.budget, a.max_len);
  char* ws = static_cast<char*>(a.ws);
  Walk* walk = reinterpret_cast<Walk*>(ws);
  float* zd = reinterpret_cast<float*>(ws + l.zd);
  int32_t* child = reinterpret_cast<int32_t*>(ws + l.child);
  Record* rec = reinterpret_cast<Record*>(ws + l.rec);
  hipLaunchKernelGGL(path_begin<BF>, dim3(a.batch), dim3(kPathThreads), 0, s, a, walk, zd, child);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  for (int round = 0; round < kRounds; ++round) {
    const int rows = round ? nrows : std::min(nrows, kFirstRows);
    hipLaunchKernelGGL(path_records<BF>, dim3(unsigned(a.batch * rows * nseg)), dim3(256), 0, s, a, nseg, rows, nrows, c, walk, rec);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (round + 1 < kRounds)
      hipLaunchKernelGGL((path_walk<BF, false>), dim3(a.batch), dim3(kPathThreads), 0, s, a, nseg, nrows, c, walk, rec, zd, child);
    else
      hipLaunchKernelGGL((path_walk<BF, true>), dim3(a.batch), dim3(kPathThreads), 0, s, a, nseg, nrows, c, walk, rec, zd, child);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

template <bool BF>
hipError_t chain(const VerifyArgs& a, hipStream_t s) {
  const int nseg = segments(a.vocab);
  const double c = a.inv_t * 1.4426950408889634;
  Record* trec = static_cast<Record*>(a.ws);
  Record* drec = trec + int64_t(a.batch) * (a.budget + 1) * nseg;
  uint64_t* segw = reinterpret_cast<uint64_t*>(drec + int64_t(a.batch) * a.budget * nseg);
  int32_t* arrived = reinterpret_cast<int32_t*>(segw + int64_t(a.batch) * nseg);
  const int64_t trows = int64_t(a.batch) * (a.budget + 1), drows = c != 0.0 ? int64_t(a.batch) * a.budget : 0;
  hipLaunchKernelGGL(row_records<BF>, dim3(unsigned((trows + drows) * nseg)), dim3(256), 0, s, a.target, trows, a.draft, a.row_stride,
                     a.vocab, nseg, c, trec, arrived, a.batch);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(chain_final<BF>, dim3(c != 0.0 ? nseg : 1, a.batch), dim3(kPick), 0, s, a, nseg, c, trec, drec, segw, arrived);
  return hipGetLastError();
}

}  // namespace

size_t verify_tree_workspace(int batch, int budget, int max_len, int vocab) {
  const size_t nseg = segments(vocab);
  if (by_path(batch, budget, max_len, vocab)) return path_layout(batch, budget, max_len, vocab).total;
  return up(size_t(batch) * (budget + 1) * nseg * sizeof(Record));
}

size_t verify_chain_workspace(int batch, int depth, int vocab) {
  const size_t nseg = segments(vocab), b = batch;
  return up(b * (2 * size_t(depth) + 1) * nseg * sizeof(Record) + b * nseg * sizeof(double) + b * sizeof(int32_t));
}

hipError_t launch_verify_tree(const VerifyArgs& a, hipStream_t s) { return a.bf16 ? tree<true>(a, s) : tree<false>(a, s); }
hipError_t launch_verify_chain(const VerifyArgs& a, hipStream_t s) { return a.bf16 ? chain<true>(a, s) : chain<false>(a, s); }

}  // namespace dartree
