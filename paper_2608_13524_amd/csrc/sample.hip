// Verification of drafted tokens against the target's probabilities from given
// random numbers: trees of chosen tokens, and chains drawn from the drafter.
//
// A row of logits is cut into segments of 4096 elements (counted from the 16
// bytes its start lies in, so that every load is aligned).  A segment's record
// is its maximum, the maximum's first index and the sum of exp((z - max) / T).
// Exponentials and sums are taken in 64 bits: the final token is where the
// cumulated mass passes u of the whole, and with 32 bits (1e-7) one draw in
// sixty of a flat 151936-token row would land on a neighbour.  The vector units
// do 64-bit fused multiply-adds at the 32-bit rate, so exp64's 20 operations an
// element stay under the time its bytes take.
//
// Trees: with few rows the records of every row are taken at once (one pass
// over the logits, all compute units) and a block per request then walks the
// tree in LDS.  With many, only the rows on the path are read, one level per
// launch.  Chains: the records of every row, then one pass over the final row.
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
  // elements of chunk c (first: the index of its first); -inf where there is none
  __device__ void load(int c, float (&x)[N], int& first) const {
    first = c * N - shift;
    if (first >= 0 && first + N <= vocab) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + int64_t(first) * (BF ? 2 : 4));
#pragma unroll
      for (int i = 0; i < N; ++i)
        x[i] = sane(BF ? __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16) : __uint_as_float(w[BF ? 0 : i]));
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
__device__ __forceinline__ int wave_max_int(int x) { return -wave_min_int(-x); }

// Record of segment `seg` of a row, by a block of 256 threads.
template <bool BF>
__device__ __forceinline__ void segment_record(const RowView<BF>& z, int seg, double c, Record* out) {
  constexpr int N = RowView<BF>::N, L = kSeg / N / 256;
  __shared__ float sm[4];
  __shared__ int sa[4];
  __shared__ double ss[4];
  float x[L][N];
  int first[L];
  float m = -INFINITY;
#pragma unroll
  for (int l = 0; l < L; ++l) z.load(seg * (kSeg / N) + l * 256 + threadIdx.x, x[l], first[l]);
#pragma unroll
  for (int l = 0; l < L; ++l)
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, x[l][i]);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  m = wave_max(m);
  if (lane == 0) sm[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  int arg = INT32_MAX;
  double s = 0.0;
  if (m != -INFINITY) {
    if (c == 0.0) {
#pragma unroll
      for (int l = 0; l < L; ++l)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[l][i] == m) arg = min(arg, first[l] + i);
    } else {
      const double md = m;
#pragma unroll
      for (int l = 0; l < L; ++l)
#pragma unroll
        for (int i = 0; i < N; ++i) s += exp64((double(x[l][i]) - md) * c);
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
    r.arg = c == 0.0 ? min(min(sa[0], sa[1]), min(sa[2], sa[3])) : 0;
    r.s = c == 0.0 ? 0.0 : (ss[0] + ss[1]) + (ss[2] + ss[3]);
    *out = r;
  }
}

// A row's records joined by 16 lanes (all 64 of a wave must call); the same in each.
__device__ __forceinline__ Record join_records(const Record* rec, int nseg, double c) {
  const int l16 = threadIdx.x & 15;
  Record r{-INFINITY, INT32_MAX, 0.0};
  for (int i = l16; i < nseg; i += 16) {   // indices grow, so an equal maximum keeps the first
    const Record o = rec[i];
    if (o.m == -INFINITY) continue;
    if (o.m > r.m) {
      r.s = r.m == -INFINITY ? o.s : r.s * exp64((double(r.m) - double(o.m)) * c) + o.s;
      r.m = o.m;
      r.arg = o.arg;
    } else {
      r.s += o.s * exp64((double(o.m) - double(r.m)) * c);
    }
  }
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) {
    const float m = __shfl_xor(r.m, off);
    const int arg = __shfl_xor(r.arg, off);
    const double s = __shfl_xor(r.s, off);
    const float top = fmaxf(r.m, m);
    // the same expression on both sides, so that all lanes agree to the bit
    const double mine = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - double(top)) * c);
    const double theirs = m == -INFINITY ? 0.0 : s * exp64((double(m) - double(top)) * c);
    r.arg = r.m == m ? min(r.arg, arg) : r.m > m ? r.arg : arg;
    r.s = mine + theirs;
    r.m = top;
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

// Threads of a block (blockDim.x a multiple of 64, at most 1024) that agree on
// the first token whose cumulated weight passes `target` in segment `seg`, where
// `weight(c, w)` gives the weights of chunk c (w[i] of element first + i, 0
// where there is none) and returns first.  -1 if none does and, in *last, the
// last token of positive weight (-1: none).
template <int N, typename F>
__device__ __forceinline__ int pick_in_segment(int seg, double target, F&& weight, int* last) {
  __shared__ double wsum[16];
  __shared__ int got[2];
  const int nt = blockDim.x, waves = nt >> 6, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunks = kSeg / N, each = (chunks + nt - 1) / nt;   // consecutive chunks per thread
  if (threadIdx.x == 0) {
    got[0] = INT32_MAX;
    got[1] = -1;
  }
  double sum = 0.0;
  for (int k = 0; k < each; ++k) {
    const int c = int(threadIdx.x) * each + k;
    if (c >= chunks) break;
    double w[N];
    weight(seg * chunks + c, w);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += w[i];
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
  for (int w = 0; w < wave && w < waves; ++w) cum += wsum[w];
  int found = INT32_MAX, pos = -1;
  if (sum > 0.0)
    for (int k = 0; k < each; ++k) {
      const int c = int(threadIdx.x) * each + k;
      if (c >= chunks) break;
      double w[N];
      const int first = weight(seg * chunks + c, w);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        cum += w[i];
        if (w[i] > 0.0) {
          pos = first + i;
          if (found == INT32_MAX && cum > target) found = first + i;
        }
      }
    }
  found = wave_min_int(found);
  pos = wave_max_int(pos);
  if (lane == 0) {
    atomicMin(&got[0], found);   // whole numbers: the order does not matter
    atomicMax(&got[1], pos);
  }
  __syncthreads();
  const int r = got[0];
  *last = got[1];
  __syncthreads();
  return r == INT32_MAX ? -1 : r;
}

// The weight of a segment, in every thread of the block.
template <int N, typename F>
__device__ __forceinline__ double segment_weight(int seg, F&& weight) {
  __shared__ double wsum[16];
  double sum = 0.0;
  for (int c = threadIdx.x; c < kSeg / N; c += blockDim.x) {
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
  for (int w = 0; w < int(blockDim.x >> 6); ++w) sum += wsum[w];
  return sum;
}

// The first token whose cumulated weight passes u of the whole, given the
// segments' weights in LDS (block-uniform result; -1: no weight at all).
template <int N, typename F>
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
    const int got = pick_in_segment<N>(sg, target, weight, &last);
    if (got >= 0) return got;
    if (last >= 0) return last;   // a sum rounded differently: the segment's last token
  }
  // u at or past 1 (or not a number): the row's last token of positive weight
  for (int s = nseg - 1; s >= 0 && last < 0; --s) {
    const int got = pick_in_segment<N>(s, INFINITY, weight, &last);
    if (got >= 0) return got;
  }
  return last;
}

// ---------------------------------------------------------------------------
// Records
// ---------------------------------------------------------------------------

// Every row: block (row, segment).
template <bool BF>
__global__ __launch_bounds__(256) void row_records(const void* z, int64_t stride, int vocab, int nseg, double c, Record* rec) {
  const int row = blockIdx.x / nseg, seg = blockIdx.x - row * nseg;
  const RowView<BF> v(z, row, stride, vocab);
  segment_record<BF>(v, seg, c, rec + blockIdx.x);
}

// State of a request's walk (level by level).
struct Walk {
  int32_t at, count, done, pad;
};

// The current row of every request: block (request, segment).
template <bool BF>
__global__ __launch_bounds__(256) void level_records(VerifyArgs a, int nseg, double c, Walk* walk, Record* rec, int level) {
  const int q = blockIdx.x / nseg, seg = blockIdx.x - q * nseg;
  Walk w{-1, 0, 0, 0};
  if (level > 0) w = walk[q];
  if (w.done) return;
  const RowView<BF> v(a.target, int64_t(q) * (a.budget + 1) + w.at + 1, a.row_stride, a.vocab);
  segment_record<BF>(v, seg, c, rec + blockIdx.x);
}

// ---------------------------------------------------------------------------
// Trees
// ---------------------------------------------------------------------------

// The final token of row `row` without the tokens of `gone` (LDS), by a block.
template <bool BF>
__device__ int final_token(const VerifyArgs& a, int64_t row, const Record* rec, int nseg, const Law& law, const int32_t* gone,
                           int ngone, float u, double* segw) {
  constexpr int N = RowView<BF>::N;
  const RowView<BF> z(a.target, row, a.row_stride, a.vocab);
  if (law.empty()) return -1;
  if (law.c == 0.0) return law.arg;   // all of the mass on one token: it remains, or nothing does and p decides
  for (int pass = 0; pass < 2; ++pass) {   // second: nothing was left of p
    const int n = pass == 0 ? ngone : 0;
    __syncthreads();
    for (int s = threadIdx.x; s < nseg; s += blockDim.x) {
      const Record r = rec[s];
      const double all = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - law.m) * law.c);
      double w = all;
      for (int i = 0; i < n; ++i) {
        const int t = gone[i];
        if ((t + z.shift) / kSeg == s) w -= law.weight(z.at(t), t);
      }
      segw[s] = w == all || w > 1e-4 * all ? w : -1.0;   // -1: little is left of the sum, add it up again
    }
    auto weight = [&](int chunk, double (&w)[N]) {
      float x[N];
      int first;
      z.load(chunk, x, first);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = x[i] == -INFINITY ? 0.0 : law.weight(x[i], first + i);
      for (int k = 0; k < n; ++k) {
        const int d = gone[k] - first;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (d == i) w[i] = 0.0;
      }
      return first;
    };
    __syncthreads();
    for (int s = 0; s < nseg && n > 0; ++s)
      if (segw[s] < 0.0) {   // the same for all threads
        const double w = segment_weight<N>(s, weight);
        if (threadIdx.x == 0) segw[s] = w;
      }
    const int t = pick<N>(segw, nseg, u, weight);
    if (t >= 0) return t;
  }
  return -1;
}

constexpr int kWalkNodes = 1024;   // nodes of a tree walked in LDS

// All rows' records at hand: a block per request.
template <bool BF>
__global__ __launch_bounds__(512) void tree_walk(VerifyArgs a, int nseg, double c, const Record* rec) {
  __shared__ int32_t tok[kWalkNodes], par[kWalkNodes];
  __shared__ float us[kWalkNodes];
  __shared__ double share[kWalkNodes];
  __shared__ float rm[kWalkNodes + 1];
  __shared__ int32_t rarg[kWalkNodes + 1];
  __shared__ double rs[kWalkNodes + 1];
  __shared__ double segw[kMaxSeg];
  __shared__ int at_s, tested_s;
  const int q = blockIdx.x, B = a.budget;
  const int n = min(max(a.num_nodes[q], 0), B);
  const int lane = threadIdx.x & 63;
  const Record* qrec = rec + int64_t(q) * (B + 1) * nseg;
  for (int row = threadIdx.x >> 4; row < ((n + 4) & ~3); row += blockDim.x >> 4) {   // whole waves
    const Record r = join_records(qrec + int64_t(min(row, n)) * nseg, nseg, c);
    if ((threadIdx.x & 15) == 0 && row <= n) {
      rm[row] = r.m;
      rarg[row] = r.arg;
      rs[row] = r.s;
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const int t = a.tokens[int64_t(q) * B + j], p = a.parents[int64_t(q) * B + j];
    tok[j] = t;
    par[j] = p;
    us[j] = a.uniforms[int64_t(q) * (B + 1) + j + 1];
    double s = 0.0;
    if (p >= -1 && p < n && t >= 0 && t < a.vocab) {
      const RowView<BF> z(a.target, int64_t(q) * (B + 1) + p + 1, a.row_stride, a.vocab);
      s = Law(Record{rm[p + 1], rarg[p + 1], rs[p + 1]}, c).share(z.at(t), t);
    }
    share[j] = s;
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
    // the tested children's tokens, gathered where the tree's tokens were
    int m = 0;
    for (int j0 = 0; j0 < n && tested; j0 += 64) {
      const bool kid = j0 + lane < n && par[j0 + lane] == at && tok[j0 + lane] >= 0 && tok[j0 + lane] < a.vocab;
      const int t = kid ? tok[j0 + lane] : 0;
      const uint64_t b = __ballot(kid);
      if (kid) tok[m + __popcll(b & ((1ull << lane) - 1))] = t;
      m += __popcll(b);
    }
    if (lane == 0) tested_s = m;
  }
  __syncthreads();
  const int at = at_s;
  const Law law(Record{rm[at + 1], rarg[at + 1], rs[at + 1]}, c);
  const int t = final_token<BF>(a, int64_t(q) * (B + 1) + at + 1, qrec + int64_t(at + 1) * nseg, nseg, law, tok, tested_s,
                                a.uniforms[int64_t(q) * (B + 1)], segw);
  if (threadIdx.x == 0) a.bonus[q] = t;
}

// One level: the records of the current row at hand, a block per request.
template <bool BF>
__global__ __launch_bounds__(256) void level_step(VerifyArgs a, int nseg, double c, Walk* walk, const Record* rec, int level) {
  __shared__ int32_t kid[DARTREE_MAX_SORT], gone[DARTREE_MAX_SORT];
  __shared__ int wcount[4], next_s, ngone_s;
  __shared__ double segw[kMaxSeg];
  const int q = blockIdx.x, B = a.budget, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Walk w{-1, 0, 0, 0};
  if (level > 0) w = walk[q];
  if (w.done) return;
  const int n = min(max(a.num_nodes[q], 0), B);
  const int64_t row = int64_t(q) * (B + 1) + w.at + 1;
  const Record r = join_records(rec + int64_t(q) * nseg, nseg, c);
  const Law law(r, c);
  const RowView<BF> z(a.target, row, a.row_stride, a.vocab);
  int nkid = 0;
  if (w.count < min(a.max_len, n))
    for (int j0 = 0; j0 < n; j0 += 256) {   // the children in index order
      const int j = j0 + threadIdx.x;
      const bool is = j < n && a.parents[int64_t(q) * B + j] == w.at;
      const uint64_t b = __ballot(is);
      __syncthreads();
      if (lane == 0) wcount[wave] = __popcll(b);
      __syncthreads();
      int at = nkid + __popcll(b & ((1ull << lane) - 1));
      for (int x = 0; x < wave; ++x) at += wcount[x];
      if (is) kid[at] = j;
      nkid += wcount[0] + wcount[1] + wcount[2] + wcount[3];
    }
  __syncthreads();
  if (wave == 0) {
    double taken = 0.0;
    int next = -1, m = 0;
    for (int i0 = 0; i0 < nkid && next < 0; i0 += 64) {
      const int j = i0 + lane < nkid ? kid[i0 + lane] : -1;
      const int t = j >= 0 ? a.tokens[int64_t(q) * B + j] : -1;
      const bool in = t >= 0 && t < a.vocab;
      const double s = in ? law.share(z.at(t), t) : 0.0;
      const float u = j >= 0 ? a.uniforms[int64_t(q) * (B + 1) + j + 1] : 0.f;
      const uint64_t b = __ballot(in);
      if (in) gone[m + __popcll(b & ((1ull << lane) - 1))] = t;
      m += __popcll(b);
      for (int i = 0; i < min(64, nkid - i0); ++i) {
        const double si = __shfl(s, i);
        if (double(__shfl(u, i)) * (1.0 - taken) < si) {
          next = __shfl(j, i);
          break;
        }
        taken += si;
      }
    }
    if (lane == 0) {
      next_s = next;
      ngone_s = m;
    }
  }
  __syncthreads();
  const int next = next_s;
  if (next >= 0) {
    if (threadIdx.x == 0) {
      a.accepted[int64_t(q) * a.max_len + w.count] = next;
      walk[q] = Walk{next, w.count + 1, 0, 0};
    }
    return;
  }
  for (int j = w.count + threadIdx.x; j < a.max_len; j += 256) a.accepted[int64_t(q) * a.max_len + j] = -1;
  const int t = final_token<BF>(a, row, rec + int64_t(q) * nseg, nseg, law, gone, ngone_s, a.uniforms[int64_t(q) * (B + 1)], segw);
  if (threadIdx.x == 0) {
    a.num_accepted[q] = w.count;
    a.bonus[q] = t;
    walk[q] = Walk{w.at, w.count, 1, 0};
  }
}

// ---------------------------------------------------------------------------
// Chains
// ---------------------------------------------------------------------------

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
  const int nrow = c == 0.0 ? n + 1 : 2 * n + 1;   // target rows 0 .. n, then the draft's 0 .. n - 1
  for (int row = threadIdx.x >> 4; row < ((nrow + 3) & ~3); row += blockDim.x >> 4) {   // whole waves
    const int x = min(row, nrow - 1);
    const Record* at = x <= n ? trec + (int64_t(q) * (D + 1) + x) * nseg : drec + (int64_t(q) * D + x - n - 1) * nseg;
    const Record r = join_records(at, nseg, c);
    if ((threadIdx.x & 15) == 0 && row < nrow) {
      rows.m[row] = r.m;
      rows.arg[row] = r.arg;
      rows.s[row] = r.s;
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int i = threadIdx.x;
    bool pass = false;
    if (i < n) {
      const int t = a.tokens[int64_t(q) * D + i];
      if (t >= 0 && t < a.vocab) {
        const Law p(Record{rows.m[i], rows.arg[i], rows.s[i]}, c);
        const RowView<BF> z(a.target, int64_t(q) * (D + 1) + i, a.row_stride, a.vocab);
        const double px = p.share(z.at(t), t);
        if (c == 0.0) {
          pass = px > 0.0;
        } else {
          const int d = n + 1 + i;
          const Law ql(Record{rows.m[d], rows.arg[d], rows.s[d]}, c);
          const RowView<BF> y(a.draft, int64_t(q) * D + i, a.row_stride, a.vocab);
          pass = double(a.uniforms[int64_t(q) * (D + 1) + i + 1]) * ql.share(y.at(t), t) < px;
        }
      }
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
  double pn, qn;   // 1 / their wholes
  bool reject;
  __device__ int operator()(int chunk, double (&w)[N]) const {
    float x[N];
    int first;
    z.load(chunk, x, first);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i] == -INFINITY ? 0.0 : p.weight(x[i], first + i);
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
        w[i] = fmax(w[i] * pn - (q.empty() || v[i] == -INFINITY ? 0.0 : q.weight(v[i], first + i) * qn), 0.0);
    }
    return first;
  }
};
template <bool BF>
__device__ __forceinline__ Residual<BF> residual_of(const VerifyArgs& a, double c, const ChainRows& rows, int n) {
  const int q = blockIdx.y, D = a.budget, k = rows.count;
  const bool reject = k < n && c != 0.0;
  const int d = reject ? n + 1 + k : 0;
  return Residual<BF>{RowView<BF>(a.target, int64_t(q) * (D + 1) + k, a.row_stride, a.vocab),
                      RowView<BF>(a.draft, reject ? int64_t(q) * D + k : 0, a.row_stride, a.vocab),
                      Law(Record{rows.m[k], rows.arg[k], rows.s[k]}, c), Law(Record{rows.m[d], rows.arg[d], rows.s[d]}, c),
                      1.0 / rows.s[k], 1.0 / rows.s[d], reject};
}

// The residual's weight by segments: block (segment, request).
template <bool BF>
__global__ __launch_bounds__(256) void chain_residual(VerifyArgs a, int nseg, double c, const Record* trec, const Record* drec,
                                                      double* segw) {
  constexpr int N = RowView<BF>::N;
  __shared__ ChainRows rows;
  __shared__ double ss[4];
  const int n = chain_walk<BF>(a, nseg, c, trec, drec, rows);
  const Residual<BF> f = residual_of<BF>(a, c, rows, n);
  if (!f.reject || f.p.empty()) return;
  double sum = 0.0;
  for (int l = 0; l < kSeg / N / 256; ++l) {
    double w[N];
    f(blockIdx.x * (kSeg / N) + l * 256 + threadIdx.x, w);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += w[i];
  }
  sum = wave_sum64(sum);
  if ((threadIdx.x & 63) == 0) ss[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) segw[int64_t(blockIdx.y) * nseg + blockIdx.x] = (ss[0] + ss[1]) + (ss[2] + ss[3]);
}

// The final token: a block per request.
template <bool BF>
__global__ __launch_bounds__(256) void chain_final(VerifyArgs a, int nseg, double c, const Record* trec, const Record* drec,
                                                   const double* segw) {
  constexpr int N = RowView<BF>::N;
  __shared__ ChainRows rows;
  __shared__ double sw[kMaxSeg];
  const int q = blockIdx.y, D = a.budget;
  const int n = chain_walk<BF>(a, nseg, c, trec, drec, rows);
  const float u = a.uniforms[int64_t(q) * (D + 1)];
  Residual<BF> f = residual_of<BF>(a, c, rows, n);
  int t = -1;
  if (f.p.empty()) {
  } else if (c == 0.0) {
    t = f.p.arg;
  } else {
    if (f.reject) {
      for (int s = threadIdx.x; s < nseg; s += 256) sw[s] = segw[int64_t(q) * nseg + s];
      t = pick<N>(sw, nseg, u, f);
    }
    if (t < 0) {   // after the last token, or nothing left of p
      f.reject = false;
      const Record* rec = trec + (int64_t(q) * (D + 1) + rows.count) * nseg;
      __syncthreads();
      for (int s = threadIdx.x; s < nseg; s += 256) {
        const Record r = rec[s];
        sw[s] = r.m == -INFINITY ? 0.0 : r.s * exp64((double(r.m) - f.p.m) * c);
      }
      t = pick<N>(sw, nseg, u, f);
    }
  }
  if (threadIdx.x == 0) {
    a.num_accepted[q] = rows.count;
    a.bonus[q] = t;
  }
}

constexpr size_t kAlign = 256;
size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool by_level(int, int budget, int, int) { return budget > kWalkNodes; }

template <bool BF>
hipError_t tree(const VerifyArgs& a, hipStream_t s) {
  const int nseg = segments(a.vocab);
  const double c = a.inv_t * 1.4426950408889634;
  if (!by_level(a.batch, a.budget, a.max_len, a.vocab)) {
    Record* rec = static_cast<Record*>(a.ws);
    const int64_t rows = int64_t(a.batch) * (a.budget + 1);
    hipLaunchKernelGGL(row_records<BF>, dim3(unsigned(rows * nseg)), dim3(256), 0, s, a.target, a.row_stride, a.vocab, nseg, c, rec);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(tree_walk<BF>, dim3(a.batch), dim3(512), 0, s, a, nseg, c, rec);
    return hipGetLastError();
  }
  Walk* walk = static_cast<Walk*>(a.ws);
  Record* rec = reinterpret_cast<Record*>(static_cast<char*>(a.ws) + up(a.batch * sizeof(Walk)));
  for (int level = 0; level <= std::min(a.max_len, a.budget); ++level) {
    hipLaunchKernelGGL(level_records<BF>, dim3(unsigned(a.batch * nseg)), dim3(256), 0, s, a, nseg, c, walk, rec, level);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(level_step<BF>, dim3(a.batch), dim3(256), 0, s, a, nseg, c, walk, rec, level);
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
  double* segw = reinterpret_cast<double*>(drec + int64_t(a.batch) * a.budget * nseg);
  hipLaunchKernelGGL(row_records<BF>, dim3(unsigned(a.batch * (a.budget + 1) * nseg)), dim3(256), 0, s, a.target, a.row_stride,
                     a.vocab, nseg, c, trec);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (c != 0.0) {
    hipLaunchKernelGGL(row_records<BF>, dim3(unsigned(a.batch * a.budget * nseg)), dim3(256), 0, s, a.draft, a.row_stride, a.vocab,
                       nseg, c, drec);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(chain_residual<BF>, dim3(nseg, a.batch), dim3(256), 0, s, a, nseg, c, trec, drec, segw);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(chain_final<BF>, dim3(1, a.batch), dim3(256), 0, s, a, nseg, c, trec, drec, segw);
  return hipGetLastError();
}

}  // namespace

size_t verify_tree_workspace(int batch, int budget, int max_len, int vocab) {
  const size_t nseg = segments(vocab);
  if (by_level(batch, budget, max_len, vocab)) return up(batch * sizeof(Walk)) + up(batch * nseg * sizeof(Record));
  return up(size_t(batch) * (budget + 1) * nseg * sizeof(Record));
}

size_t verify_chain_workspace(int batch, int depth, int vocab) {
  const size_t nseg = segments(vocab), b = batch;
  return up(b * (2 * size_t(depth) + 1) * nseg * sizeof(Record) + b * nseg * sizeof(double));
}

hipError_t launch_verify_tree(const VerifyArgs& a, hipStream_t s) { return a.bf16 ? tree<true>(a, s) : tree<false>(a, s); }
hipError_t launch_verify_chain(const VerifyArgs& a, hipStream_t s) { return a.bf16 ? chain<true>(a, s) : chain<false>(a, s); }

}  // namespace dartree
