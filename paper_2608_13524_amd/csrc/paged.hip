// Attention of drafted trees, chains and single tokens over a paged cache.
//
// One pass over the keys with a running maximum and sum per query row.  Work
// is counted in steps of keys: those of a request's context, then those of its
// tree, for every (key/value head, tile of query rows).  The steps of all requests
// lie on one line that the blocks share equally (or every block takes one whole
// item, where there are many), so ragged contexts cost no idle compute units; an
// item cut by a block's end leaves partial results, which a second launch joins
// in block order.
//
// Up to 16 query rows of a key/value head, or few items (paged_attention): a step
// is a chunk of 32 keys for each of the block's four or eight waves, and a wave
// works from registers alone.  S^T = K Q^T leaves lane (c = lane % 16, g = lane / 16) with
// query c's weights of keys 4 g .. 4 g + 3 of both 16-key tiles, the B operand of
// O^T = V^T P^T with the keys taken in that order.  For V a lane reads eight dims,
// 8 c .. 8 c + 7, of those same keys and transposes them in registers; column tile
// t of the product is then dims 8 c + t, and a lane ends with dims 32 g .. 32 g + 31
// of its query.  A tile lies in one page, so every load has a scalar base and an
// offset that is the lane's own.  Keys in e4m3 become bf16 on the way with their
// power of two applied by the conversion (exact).  A head's keys and values are read
// once for 16 query rows (again for the next 16, from a cache where it holds them)
// and never pass through LDS.
//
// More rows (paged_tiles): below.
#include <algorithm>

#include "reduce.hpp"
#include "serve.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kChunk = 32;            // keys of a wave's share of a step

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// sum += eight bf16 weights, in 32 bits, two a lane and instruction.  Weights are
// rounded to bf16 because the matrix instructions multiply pairs of one 16-bit type
// (in two parts they would take twice the products and their operands); the rounded
// ones are summed, as they multiply the values, so that a common rounding cancels.
// At most 2^-8 of a weight, so 2^-8 of the largest value in a result, whose own
// rounding to bf16 is up to 2^-8 of it; the dense layer rounds its weights alike.
__device__ __forceinline__ void add_weights(u32x4 w, float& sum) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, uint32_t(w[i])), ones, sum, false);
}

// A tree's values that are no numbers must not reach rows that do not see them
// (their weight there is 0, and 0 times a NaN is a NaN): they are multiplied as
// zeros and added to the rows that do see them after the tree's last step.
// odd_bits: bits 15 and 31 of the result are set where a half of w is an infinity
// or a NaN.
constexpr uint32_t kOdd = 0x80008000u;
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
__device__ __forceinline__ uint32_t without_odd(uint32_t w) {
  const uint32_t b = odd_bits(w);
  return w & ~((b & 0x8000u ? 0xFFFFu : 0u) | (b & 0x80000000u ? 0xFFFF0000u : 0u));
}
__device__ __forceinline__ float odd_part(uint16_t v) {
  return (v & 0x7F80u) == 0x7F80u ? __uint_as_float(uint32_t(v) << 16) : 0.f;
}

template <bool HI>
__device__ __forceinline__ uint32_t expand2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

__device__ __forceinline__ u32x4 finite_pairs(u32x4 w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = finite_pair(w[i]);
  return w;
}

// Small arrays that a launch only reads, at addresses that are the same for all
// lanes: scalar loads, which do not queue behind the vector loads in flight.
typedef const __attribute__((address_space(4))) int32_t* Uniform;
__device__ __forceinline__ Uniform uniform_array(const int32_t* p) { return (Uniform)p; }

template <int STEP>
struct Extent {   // a request's keys, in steps of STEP
  int ctx, nodes;
  __device__ int ctx_steps() const { return (ctx + STEP - 1) / STEP; }
  __device__ int steps() const { return max(1, ctx_steps() + (nodes + STEP - 1) / STEP); }
};
template <int STEP>
__device__ __forceinline__ Extent<STEP> extent_of(const PagedArgs& a, int q) {
  return Extent<STEP>{a.ctx_len ? min(max(a.ctx_len[q], 0), a.max_ctx) : a.max_ctx,
                a.num_nodes ? min(max(a.num_nodes[q], 0), a.budget) : a.budget};
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x))))) | (int64_t(uniform(int(x >> 32))) << 32);
}

// The same of a request that is the same for all lanes.
template <int STEP>
__device__ __forceinline__ Extent<STEP> extent_at(const PagedArgs& a, int q) {
  return Extent<STEP>{a.ctx_len ? min(max(uniform_array(a.ctx_len)[q], 0), a.max_ctx) : a.max_ctx,
                      a.num_nodes ? min(max(uniform_array(a.num_nodes)[q], 0), a.budget) : a.budget};
}

// Sum over the requests of their steps.
template <int STEP>
__device__ __forceinline__ int64_t all_steps(const PagedArgs& a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) total += wave_sum_int(q0 + lane < a.batch ? extent_of<STEP>(a, q0 + lane).steps() : 0);
  return total;
}

// The request that step `at` of the line lies in (`per` steps of the line per
// step of a request) and the steps before that request.
template <int STEP>
__device__ __forceinline__ int find_request(const PagedArgs& a, int64_t at, int per, int64_t* before) {
  const int lane = threadIdx.x & 63;
  int64_t sum = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) {
    const int mine = q0 + lane < a.batch ? extent_of<STEP>(a, q0 + lane).steps() : 0;
    int incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(incl, off);
      if (lane >= off) incl += o;
    }
    const uint64_t past = __ballot((sum + incl) * per > at);
    if (past) {
      const int l = __builtin_ctzll(past);
      *before = (sum + uniform(__shfl(incl - mine, l))) * per;
      return uniform(q0 + l);
    }
    sum += uniform(__shfl(incl, 63));
  }
  *before = sum * per;
  return a.batch;   // not reached for steps of the line
}

// Where a block begins on the line (or its item, where every block has a whole one).
struct Place {
  int q, item, step, left;   // request, item of it, step of that, steps the block has
};
template <int STEP>
__device__ __forceinline__ bool place_of(const PagedArgs& a, int whole, int per, int blk, int blocks, Place* p) {
  if (whole) {
    p->q = blk / per;
    p->item = blk - p->q * per;
    p->step = 0;
    p->left = extent_at<STEP>(a, p->q).steps();
    return true;
  }
  const int64_t total = uniform64(all_steps<STEP>(a) * per);
  const int64_t s0 = total * blk / blocks, s1 = total * (blk + 1) / blocks;
  p->left = uniform(int(s1 - s0));
  if (p->left <= 0) return false;
  int64_t before;
  p->q = find_request<STEP>(a, s0, per, &before);
  const int steps = extent_at<STEP>(a, p->q).steps();
  const int64_t in = s0 - before;
  p->item = uniform(int(in / steps));
  p->step = uniform(int(in - int64_t(p->item) * steps));
  return true;
}

struct Rows {   // a wave's running result for its query rows
  f32x4 o[8];   // o[t][i]: dim 32 g + 8 i + t
  float m, l;   // l: this lane's keys only
};
__device__ __forceinline__ void clear(Rows& r) {
  r.m = -INFINITY;
  r.l = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) r.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int N>
struct Index {
  static constexpr int value = N;
};

template <bool E8>
struct Chunk {   // 32 keys and values as read
  u32x4 k[2][E8 ? 2 : 4];
  u32x2 v8[E8 ? 8 : 1];
  u32x4 v16[E8 ? 1 : 8];
  uint32_t ke[2];
  u32x2 ve;
};

// Scores of a chunk.  TOP: keys' exponents may be kTopByte and more.
template <bool E8, bool TOP>
__device__ __forceinline__ void chunk_scores(const Chunk<E8>& c, const u32x4 (&qf)[4], f32x4 (&s)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x4 kf;
      if constexpr (E8) {
        const float sc = __uint_as_float(uint32_t(c.ke[t]) << 23);
        const uint32_t w0 = c.k[t][ks >> 1][2 * (ks & 1)], w1 = c.k[t][ks >> 1][2 * (ks & 1) + 1];
        kf = u32x4{expand2<false>(w0, sc), expand2<true>(w0, sc), expand2<false>(w1, sc), expand2<true>(w1, sc)};
        if constexpr (TOP) kf = finite_pairs(kf);
      } else {
        kf = c.k[t][ks];
      }
      s[t] = mfma16(kf, qf[ks], s[t]);
    }
  }
}

// Weights of a chunk from its scores.  vis: bit k set where the lane's query sees
// key k (masked: some bit is clear).
__device__ __forceinline__ void chunk_weights(f32x4 (&s)[2], const bool masked, const uint32_t vis, const float c2,
                                              Rows& st, u32x4& p) {
  const int g = (threadIdx.x & 63) >> 4;
  if (masked) {
    const uint32_t b = vis >> (4 * g);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!((b >> (16 * t + i)) & 1u)) s[t][i] = -INFINITY;
  }
  // The reference m of a row moves only when a key exceeds it by more than 2^8,
  // so most chunks need no exchange between lanes and no rescaling; weights
  // stay below 2^8 and a row that has seen no key keeps m = -inf, l = 0, O = 0.
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
  if (__any(top * c2 > st.m * c2 + 8.f)) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m = top * c2 > st.m * c2 + 8.f ? top : st.m;
    const float f = __builtin_amdgcn_exp2f((st.m - (m == -INFINITY ? 0.f : m)) * c2);
    st.l *= f;
#pragma unroll
    for (int t = 0; t < 8; ++t) st.o[t] *= f;
    st.m = m;
  }
  const float ref = -(st.m == -INFINITY ? 0.f : st.m) * c2;
  bf16x8 w;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[4 * t + i] = __bf16(__builtin_amdgcn_exp2f(fmaf(s[t][i], c2, ref)));
  p = __builtin_bit_cast(u32x4, w);
  add_weights(p, st.l);
}

// O of a chunk.  V: dims 8 c + 2 j, 8 c + 2 j + 1 of eight keys, transposed.  A key
// that is not there has zeros instead of what its memory holds: 0 * NaN is NaN.
template <bool E8, bool TOP>
__device__ __forceinline__ void chunk_values(const Chunk<E8>& c, const uint32_t there, const u32x4& p, Rows& st) {
  const int g = (threadIdx.x & 63) >> 4;
  const uint32_t here = there >> (4 * g);
  const bool whole = there == ~0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (E8) {
        const uint32_t byte = (c.ve[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        const float sc = __uint_as_float(byte << 23);
        w[e] = (j & 1) ? expand2<true>(c.v8[e][j >> 1], sc) : expand2<false>(c.v8[e][j >> 1], sc);
        if constexpr (TOP) w[e] = finite_pair(w[e]);
      } else {
        w[e] = c.v16[e][j];
      }
      if (!whole) w[e] = (here >> (16 * (e >> 2) + (e & 3))) & 1u ? w[e] : 0u;
    }
    u32x4 lo, hi;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      lo[x] = __builtin_amdgcn_perm(w[2 * x + 1], w[2 * x], 0x05040100u);
      hi[x] = __builtin_amdgcn_perm(w[2 * x + 1], w[2 * x], 0x07060302u);
    }
    st.o[2 * j] = mfma16(lo, p, st.o[2 * j]);
    st.o[2 * j + 1] = mfma16(hi, p, st.o[2 * j + 1]);
  }
}

// Partial results: slot s of part_o holds the unnormalised rows [ROWS][128] of
// one cut item, part_ml their {m, l}.  Block i's first item, if cut at its
// beginning, is slot 2 i, its last, if it begins there and is cut at its end,
// slot 2 i + 1.
struct Parts {
  float* o;
  float* ml;
};
template <int ROWS>
__device__ __forceinline__ Parts parts_of(const PagedArgs& a, int blocks) {
  float* o = static_cast<float*>(a.ws);
  return Parts{o, o + int64_t(blocks) * 2 * ROWS * kHead};
}

template <bool E8, int W>
__global__ __launch_bounds__(64 * W, 8 / W) void paged_attention(PagedArgs a, int whole) {
  constexpr int kWaves = W, kStep = kChunk * W;
  __shared__ __attribute__((aligned(16))) float red[kWaves * 8 * 64 * 4];
  __shared__ float ml[kWaves][16][2];
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int rows = a.budget * a.group, ntile = (rows + 15) / 16;
  const int per = a.heads_kv * ntile;   // items of a request
  const int blocks = gridDim.x, blk = xcd_order(blockIdx.x, blocks);
  const Parts parts = parts_of<16>(a, blocks);
  const int words = 2 * ((a.budget + 63) / 64);
  const int page_size = 1 << a.c.page_log2;

  Place at;
  if (!place_of<kStep>(a, whole, per, blk, blocks, &at)) return;
  int q = uniform(at.q), item = uniform(at.item), step = uniform(at.step), left = uniform(at.left);
  while (left > 0) {
    const Extent<kStep> ex = extent_at<kStep>(a, q);
    const int steps = ex.steps(), nctx = ex.ctx_steps();
    const int n = min(left, steps - step);
    const int kvh = item / ntile, rt = item - kvh * ntile;

    u32x4 qf[4];
    Rows st;
    const int row = min(rt * 16 + c16, rows - 1);   // past the end: the last row, never stored
    const int node = row / a.group;
    const int64_t from = (int64_t(q) * a.budget + node) * a.q_stride + (kvh * a.group + row - node * a.group) * kHead;
    // operand ks: dims 64 (ks / 2) + 16 g + 8 (ks % 2) .. + 7, for keys alike
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      qf[ks] = *reinterpret_cast<const u32x4*>(a.q + from + 64 * (ks >> 1) + 16 * g + 8 * (ks & 1));
    const uint32_t* mrow = a.mask ? reinterpret_cast<const uint32_t*>(a.mask) + (int64_t(q) * a.budget + node) * words : nullptr;
    clear(st);

    // The context: chunks of keys kb .. kb + 31, a step apart.  The next chunk's keys
    // are fetched once this one's scores are formed, its values once this one's
    // are added, so a chunk's bytes are in flight all the time.
    const Uniform table = uniform_array(a.c.table) + int64_t(q) * a.c.max_pages;
    const int kb0 = step * kStep + wave * kChunk;
    const int chunks = kb0 < ex.ctx ? min(min(step + n, nctx) - step, (ex.ctx - kb0 + kStep - 1) / kStep) : 0;
    if (chunks > 0) {
      Chunk<E8> ch;
      f32x4 sc[2];
      u32x4 p;
      int p0, p1;   // pages of the halves of the chunk to fetch next
      auto look_up = [&](int kb) __attribute__((always_inline)) {
        p0 = table[kb >> a.c.page_log2];
        p1 = table[min(kb + 16, ex.ctx - 1) >> a.c.page_log2];
      };
      int64_t row0[2] = {0, 0};   // the tiles' first rows
      uint32_t next = 0;          // which keys of the fetched chunk are there
      const int koff = E8 ? c16 * kHead + 16 * g : c16 * 2 * kHead + 32 * g, voff = E8 ? 4 * g * kHead + 8 * c16 : 4 * g * 2 * kHead + 16 * c16;
      auto fetch_keys = [&](int kb) __attribute__((always_inline)) {
        const int valid = min(kChunk, ex.ctx - kb);
        next = valid == 32 ? ~0u : (1u << valid) - 1u;
        const bool in0 = uint32_t(p0) < uint32_t(a.c.num_pages), in1 = uint32_t(p1) < uint32_t(a.c.num_pages);
        if (!in0) next &= 0xFFFF0000u;
        if (!in1) next &= 0x0000FFFFu;
        const int64_t h0 = in0 ? p0 : 0, h1 = in1 ? p1 : 0;   // any page: what is read is not used
        row0[0] = ((h0 * a.heads_kv + kvh) << a.c.page_log2) + (kb & (page_size - 1));
        row0[1] = ((h1 * a.heads_kv + kvh) << a.c.page_log2) + ((kb + 16) & (page_size - 1));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const char* kp = static_cast<const char*>(a.c.k) + row0[t] * (E8 ? kHead : 2 * kHead);
          if constexpr (E8) {
            ch.k[t][0] = *reinterpret_cast<const u32x4*>(kp + koff);
            ch.k[t][1] = *reinterpret_cast<const u32x4*>(kp + koff + 64);
            ch.ke[t] = (a.c.k_exp + row0[t])[c16];
          } else {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              ch.k[t][ks] = *reinterpret_cast<const u32x4*>(kp + koff + 128 * (ks >> 1) + 16 * (ks & 1));
          }
        }
      };
      auto fetch_values = [&] __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const char* vp = static_cast<const char*>(a.c.v) + row0[e >> 2] * (E8 ? kHead : 2 * kHead);
          if constexpr (E8) ch.v8[e] = *reinterpret_cast<const u32x2*>(vp + voff + (e & 3) * kHead);
          else ch.v16[e] = *reinterpret_cast<const u32x4*>(vp + voff + (e & 3) * 2 * kHead);
        }
        if constexpr (E8) {
#pragma unroll
          for (int t = 0; t < 2; ++t) ch.ve[t] = *reinterpret_cast<const uint32_t*>(a.c.v_exp + row0[t] + 4 * g);
        }
      };
      uint32_t most = 0;   // of the exponents of keys that are there
      auto walk = [&](auto TOP) __attribute__((always_inline)) {
        look_up(kb0);
        fetch_keys(kb0);
        fetch_values();
#pragma unroll 1
        for (int i = 0; i < chunks; ++i) {
          const uint32_t there = next;
          const int kb = kb0 + (i + 1) * kStep;
          const bool more = i + 1 < chunks;
          if (more) look_up(kb);
          chunk_scores<E8, TOP.value>(ch, qf, sc);
          uint32_t e0 = E8 ? ch.ke[0] : 0, e1 = E8 ? ch.ke[1] : 0;
          if (more) fetch_keys(kb);
          if constexpr (E8 && !TOP.value) {
            if (there != ~0u) {
              if (!((there >> c16) & 1u)) e0 = 0;
              if (!((there >> (16 + c16)) & 1u)) e1 = 0;
            }
            most = max(most, max(e0, e1));
          }
          chunk_weights(sc, there != ~0u, there, a.scale_log2, st, p);
          chunk_values<E8, TOP.value>(ch, there, p, st);
          if (more) fetch_values();
        }
      };
      walk(Index<false>());
      if constexpr (E8) {
        // Rows with a key of kTopByte and more, and values that gave something else than
        // a finite sum (as the infinities of such exponents do): once more, converted
        // with care.  Tests in the loop cost 5 % (1 x 64 nodes x 2048 positions:
        // 19.1 us, without any 18.2, this way 18.4).
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum = fmaf(st.o[t][i], 0.f, sum);
        if (__any(most >= kTopByte || sum != 0.f)) {
          clear(st);
          walk(Index<true>());
        }
      }
    }
    // the tree's own keys
    auto sees = [&](int kb) {   // of kb .. kb + 31
      return mrow ? mrow[kb >> 5] : node < kb ? 0u : node - kb >= 31 ? ~0u : (2u << (node - kb)) - 1u;
    };
    bool odd = false;   // the same for the wave
    for (int s = max(step, nctx); s < step + n; ++s) {
      const int kb = (s - nctx) * kStep + wave * kChunk;
      if (kb >= ex.nodes) break;
      const int valid = min(kChunk, ex.nodes - kb);
      const uint32_t there = valid == 32 ? ~0u : (1u << valid) - 1u;
      auto at = [&](int key) {
        return (int64_t(q) * a.budget + min(kb + key, ex.nodes - 1)) * a.kv_stride + kvh * kHead;
      };
      Chunk<false> ch;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint16_t* kp = a.k_tree + at(16 * t + c16) + 16 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          ch.k[t][ks] = *reinterpret_cast<const u32x4*>(kp + 64 * (ks >> 1) + 8 * (ks & 1));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        ch.v16[e] = *reinterpret_cast<const u32x4*>(a.v_tree + at(16 * (e >> 2) + 4 * g + (e & 3)) + 8 * c16);
      const uint32_t seen = sees(kb);
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) bits |= odd_bits(ch.v16[e][j]);
      if (__any(bits & kOdd)) {
        odd = true;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) ch.v16[e][j] = without_odd(ch.v16[e][j]);
      }
      f32x4 sc[2];
      u32x4 p;
      chunk_scores<false, false>(ch, qf, sc);
      chunk_weights(sc, true, seen & there, a.scale_log2, st, p);
      chunk_values<false, false>(ch, there, p, st);
    }
    if (odd)
      for (int s = max(step, nctx); s < step + n; ++s) {
        const int kb = (s - nctx) * kStep + wave * kChunk;
        if (kb >= ex.nodes) break;
        const uint32_t seen = sees(kb);
        for (int key = 0; key < min(kChunk, ex.nodes - kb); ++key) {
          if (!((seen >> key) & 1u)) continue;
          const uint16_t* vp = a.v_tree + (int64_t(q) * a.budget + kb + key) * a.kv_stride + kvh * kHead + 32 * g;
#pragma unroll
          for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[t][i] += odd_part(vp[8 * i + t]);
        }
      }

    // join the waves: their rows scaled to the block's maximum, added in wave order
    float l = st.l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      ml[wave][c16][0] = st.m;
      ml[wave][c16][1] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<f32x4*>(&red[((wave * 8 + 2 * i + h) * 64 + lane) * 4]) =
            f32x4{st.o[4 * h][i], st.o[4 * h + 1][i], st.o[4 * h + 2][i], st.o[4 * h + 3][i]};
    __syncthreads();
    const bool direct = n == steps;
    const int slot = 2 * blk + (step > 0 ? 0 : 1);
    if (wave < 4) {   // a wave: dims 32 g + 8 wave .. + 7
      float M = ml[0][c16][0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, ml[w][c16][0]);
      float L = 0.f;
      f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = ml[w][c16][0];
        const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - M) * a.scale_log2);
        L += f * ml[w][c16][1];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          v[h] += f * *reinterpret_cast<const f32x4*>(&red[((w * 8 + 2 * wave + h) * 64 + lane) * 4]);
      }
      if (rt * 16 + c16 < rows) {
        if (direct) {
          const float inv = L > 0.f ? 1.f / L : 0.f;   // a row that sees nothing is zero
          bf16x8 o;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = __bf16(v[i >> 2][i & 3] * inv);
          const int64_t head = (int64_t(q) * a.budget + node) * a.heads_q + kvh * a.group + row - node * a.group;
          *reinterpret_cast<bf16x8*>(a.out + head * kHead + 32 * g + 8 * wave) = o;
        } else {
          float* po = parts.o + (int64_t(slot) * 16 + c16) * kHead + 32 * g + 8 * wave;
          *reinterpret_cast<f32x4*>(po) = v[0];
          *reinterpret_cast<f32x4*>(po + 4) = v[1];
          if (wave == 0 && g == 0) {
            parts.ml[(int64_t(slot) * 16 + c16) * 2] = M;
            parts.ml[(int64_t(slot) * 16 + c16) * 2 + 1] = L;
          }
        }
      }
    }
    __syncthreads();   // red and ml are free again

    left -= n;
    step = 0;
    if (++item == per) {
      item = 0;
      ++q;
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows: a block's W waves hold 16 RG query rows each and share tiles of 64
// keys through LDS, in bf16 (e4m3 is converted once, as it is stored).  Tile
// s + 1 travels in registers while tile s is multiplied, in two buffers.  A row
// of 256 bytes keeps its 16-byte chunk c at c ^ k_place or c ^ v_place of the
// row: K is read a row per lane, V transposed (ds_read_b64_tr_b16: lane l gets dim
// l % 16 of keys 4 (l / 16) .. + 3).  Here the rows of S^T are the keys in order,
// so lane group g holds the weights of keys 4 g .. + 3 of every 16, and V's
// operand is read in that order.
// ---------------------------------------------------------------------------
constexpr int kTile = 64;
constexpr int kRowBytes = 2 * kHead, kTileBytes = kTile * kRowBytes;
#define LDS_AS __attribute__((address_space(3)))
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// XOR of the places of a row's 16-byte chunks.  K: 16 rows' reads of one chunk
// take 16 places.  V: a transposed read takes two places of eight consecutive
// rows, a write all places of one parity of two rows.
__device__ __forceinline__ int k_place(int key) { return key & 15; }
__device__ __forceinline__ int v_place(int key) { return ((key & 7) << 1) | (key & 1); }

// The thread's number, computed anew where this stands: keeps what is derived
// from it for a later part of a kernel out of the registers of the loop before.
__device__ __forceinline__ int thread_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

template <int RG, bool E8, int W>
__global__ __launch_bounds__(64 * W, 8 / W) void paged_tiles(PagedArgs a, int whole) {
  __shared__ __attribute__((aligned(16))) char smem[4 * kTileBytes];   // [buffer][K, V]
  __shared__ int odd;   // the last of the block's items (counted from 1) whose tree holds values that are no numbers
  LDS_AS char* const lds = (LDS_AS char*)smem;
  constexpr int kRows = 16 * W * RG;
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int rows = a.budget * a.group, ntile = (rows + kRows - 1) / kRows;
  const int per = a.heads_kv * ntile;
  const int blocks = gridDim.x, blk = xcd_order(blockIdx.x, blocks);
  const int page_mask = (1 << a.c.page_log2) - 1;
  const float c2 = a.scale_log2;

  Place at;
  if (!place_of<kTile>(a, whole, per, blk, blocks, &at)) return;
  int q = uniform(at.q), item = uniform(at.item), step = uniform(at.step), left = uniform(at.left);
  if (threadIdx.x == 0) odd = 0;
  __syncthreads();

  for (int turn = 1; left > 0; ++turn) {
    const Extent<kTile> ex = extent_at<kTile>(a, q);
    const int steps = ex.steps(), nctx = ex.ctx_steps();
    const int n = min(left, steps - step), last = step + n;
    const int kvh = item / ntile, rt = item - kvh * ntile;

    u32x4 qf[RG][4];
    float m[RG], l[RG], bar[RG], ref[RG];   // bar: a score above it moves the reference m; ref = -m c2
    f32x4 o[RG][8];
    {
      const int tid = thread_again();
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        const int row = min(rt * kRows + (tid >> 6) * (16 * RG) + r * 16 + (tid & 15), rows - 1);   // past the end: the last row, never stored
        const int node = row / a.group;
        const uint16_t* qp = a.q + (int64_t(q) * a.budget + node) * a.q_stride + (kvh * a.group + row - node * a.group) * kHead;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qf[r][ks] = *reinterpret_cast<const u32x4*>(qp + 32 * ks + 8 * ((tid & 63) >> 4));
        m[r] = bar[r] = -INFINITY;
        l[r] = ref[r] = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) o[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }

    // operand addresses within a buffer, the same for all tiles
    int ka[4], va[8];
    const int vr = 4 * g + (r16 >> 2);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) ka[ks] = r16 * kRowBytes + ((4 * ks + g) ^ k_place(r16)) * 16;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      va[t] = kTileBytes + vr * kRowBytes + ((2 * t + ((r16 & 3) >> 1)) ^ v_place(vr)) * 16 + (r16 & 1) * 8;

    // scores of 32 keys, half c of the tile in buffer B
    auto scores = [&](auto B, auto C, f32x4 (&sc)[RG][2]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < RG; ++r) sc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const u32x4 kf = *reinterpret_cast<const LDS_AS u32x4*>(
              lds + ka[ks] + (B.value * 2 * kTileBytes + (C.value * 32 + t * 16) * kRowBytes));
#pragma unroll
          for (int r = 0; r < RG; ++r) sc[r][t] = mfma16(kf, qf[r][ks], sc[r][t]);
        }
      }
    };
    // unseen keys out; the reference of a row moves as in chunk_weights, one test for all rows
    auto settle = [&](bool masked, const uint32_t (&vis)[RG], f32x4 (&sc)[RG][2]) __attribute__((always_inline)) {
      if (masked) {
#pragma unroll
        for (int r = 0; r < RG; ++r) {
          const uint32_t bits = vis[r] >> (4 * g);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!((bits >> (16 * t + i)) & 1u)) sc[r][t][i] = -INFINITY;
        }
      }
      float top[RG];
      bool grow = false;
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        top[r] = sc[r][0][0];
#pragma unroll
        for (int x = 1; x < 8; ++x) top[r] = fmaxf(top[r], sc[r][x >> 2][x & 3]);
        grow |= top[r] > bar[r];
      }
      if (__any(grow)) {
#pragma unroll
        for (int r = 0; r < RG; ++r) {
          float x = fmaxf(top[r], __shfl_xor(top[r], 16));
          x = fmaxf(x, __shfl_xor(x, 32));
          if (x <= bar[r]) x = m[r];
          const float f = __builtin_amdgcn_exp2f((m[r] - (x == -INFINITY ? 0.f : x)) * c2);
          l[r] *= f;
#pragma unroll
          for (int t = 0; t < 8; ++t) o[r][t] *= f;
          m[r] = x;
          bar[r] = x + 8.f / c2;
          ref[r] = x == -INFINITY ? 0.f : -x * c2;
        }
      }
    };
    auto weights = [&](const f32x4 (&sc)[RG][2], u32x4 (&p)[RG]) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        bf16x8 w;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[4 * t + i] = __bf16(__builtin_amdgcn_exp2f(fmaf(sc[r][t][i], c2, ref[r])));
        p[r] = __builtin_bit_cast(u32x4, w);
        add_weights(p[r], l[r]);
      }
    };
    auto values = [&](auto B, auto C, const u32x4 (&p)[RG]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const LDS_AS char* at = lds + va[t] + (B.value * 2 * kTileBytes + C.value * 32 * kRowBytes);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at + 16 * kRowBytes));
        const u32x4 vf = __builtin_bit_cast(u32x4, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
        for (int r = 0; r < RG; ++r) o[r][t] = mfma16(vf, p[r], o[r][t]);
      }
    };

    // Tiles first .. end - 1 of one source.  fetch(s): a thread's share of tile s
    // into registers; store(B): the fetched tile to buffer B, returning which of
    // its keys are there (one that is not has zeros for values: 0 * NaN is NaN);
    // sees(s, r, there): what row group r sees of the keys that are.
    auto sweep = [&](const int first, const int end, auto&& fetch, auto&& store, auto&& sees, const bool tree) __attribute__((always_inline)) {
      if (first >= end) return;
      fetch(first);
      uint64_t there = store(Index<0>());
      if (first + 1 < end) fetch(first + 1);
      __syncthreads();
      f32x4 sa[RG][2], sb[RG][2];
      u32x4 p[RG];
      uint32_t seen[2][RG];
      scores(Index<0>(), Index<0>(), sa);
      auto tile = [&](auto B, int s) __attribute__((always_inline)) {
        const Index<1 - B.value> other;
        const bool masked = tree || there != ~0ull;
        if (masked) {
#pragma unroll
          for (int r = 0; r < RG; ++r) {
            const uint64_t vis = sees(s, r, there);
            seen[0][r] = uint32_t(vis);
            seen[1][r] = uint32_t(vis >> 32);
          }
        }
        // the products of the next 32 keys' scores run beside the exponentials of these
        settle(masked, seen[0], sa);
        scores(B, Index<1>(), sb);
        weights(sa, p);
        values(B, Index<0>(), p);
        settle(masked, seen[1], sb);
        if (s + 1 < end) {
          there = store(other);
          if (s + 2 < end) fetch(s + 2);
        }
        __syncthreads();
        scores(other, Index<0>(), sa);   // after the last tile: not used
        weights(sb, p);
        values(B, Index<1>(), p);
        __syncthreads();   // both buffers are free again
      };
#pragma unroll 1
      for (int s = first; s < end; s += 2) {
        tile(Index<0>(), s);
        if (s + 1 < end) tile(Index<1>(), s + 1);
      }
    };

    {   // the context
      const int32_t* table = a.c.table + int64_t(q) * a.c.max_pages;
      constexpr int kRowsWave = E8 ? 8 : 4, kShares = kTile / (kRowsWave * W);
      u32x4 kx[kShares], vx[kShares];
      uint32_t ke[kShares], ve[kShares];
      uint64_t in_flight = 0;
      int page;   // lane i % 4: the page of the i-th 16 keys of the tile to fetch next
      auto look_up = [&](int s) __attribute__((always_inline)) {
        page = table[min(s * kTile + 16 * (thread_again() & 3), ex.ctx - 1) >> a.c.page_log2];
      };
      // a wave's keys of a share lie in one group of 16, so in one page: eight rows
      // of 128 bytes in e4m3, four of 256 in bf16, from key first_key(i)
      auto first_key = [&](int i) { return kRowsWave * (W * i + wave); };
      auto fetch = [&](int s) __attribute__((always_inline)) {
        const int kb = s * kTile, valid = min(kTile, ex.ctx - kb);
        in_flight = valid == 64 ? ~0ull : (1ull << valid) - 1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (uint32_t(__builtin_amdgcn_readlane(page, i)) >= uint32_t(a.c.num_pages)) in_flight &= ~(0xFFFFull << (16 * i));
#pragma unroll
        for (int i = 0; i < kShares; ++i) {
          const int of = __builtin_amdgcn_readlane(page, first_key(i) >> 4);
          const int64_t in = uint32_t(of) < uint32_t(a.c.num_pages) ? of : 0;   // any page: what is read is not used
          const int64_t row0 = ((in * a.heads_kv + kvh) << a.c.page_log2) + ((kb + first_key(i)) & page_mask);
          const int64_t byte0 = row0 * (E8 ? kHead : 2 * kHead);
          kx[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.c.k) + byte0 + 16 * lane);
          vx[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.c.v) + byte0 + 16 * lane);
          if constexpr (E8) {
            ke[i] = a.c.k_exp[row0 + (lane >> 3)];
            ve[i] = a.c.v_exp[row0 + (lane >> 3)];
          }
        }
        look_up(s + 1);
      };
      auto store = [&](auto B) __attribute__((always_inline)) -> uint64_t {
        const uint64_t there = in_flight;
        const u32x4 zero{0, 0, 0, 0};
        LDS_AS char* const kt = lds + B.value * 2 * kTileBytes;
#pragma unroll
        for (int i = 0; i < kShares; ++i) {
          const int key = first_key(i) + (E8 ? lane >> 3 : g);
          const bool gone = there != ~0ull && !((there >> key) & 1);
          if (gone) vx[i] = zero;
          if constexpr (E8) {
            const float sk = __uint_as_float(ke[i] << 23), sv = gone ? 1.f : __uint_as_float(ve[i] << 23);
            u32x4 k[2], v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              k[h] = u32x4{expand2<false>(kx[i][2 * h], sk), expand2<true>(kx[i][2 * h], sk), expand2<false>(kx[i][2 * h + 1], sk),
                           expand2<true>(kx[i][2 * h + 1], sk)};
              v[h] = u32x4{expand2<false>(vx[i][2 * h], sv), expand2<true>(vx[i][2 * h], sv), expand2<false>(vx[i][2 * h + 1], sv),
                           expand2<true>(vx[i][2 * h + 1], sv)};
            }
            if (__builtin_expect(__any(max(ke[i], ve[i]) >= kTopByte), 0)) {   // 2 % of 16 x 512 nodes x 2048 positions
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                k[h] = finite_pairs(k[h]);
                v[h] = finite_pairs(v[h]);
              }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = 2 * (lane & 7) + h;
              *reinterpret_cast<LDS_AS u32x4*>(kt + key * kRowBytes + (c ^ k_place(key)) * 16) = k[h];
              *reinterpret_cast<LDS_AS u32x4*>(kt + kTileBytes + key * kRowBytes + (c ^ v_place(key)) * 16) = v[h];
            }
          } else {
            *reinterpret_cast<LDS_AS u32x4*>(kt + key * kRowBytes + (r16 ^ k_place(key)) * 16) = kx[i];
            *reinterpret_cast<LDS_AS u32x4*>(kt + kTileBytes + key * kRowBytes + (r16 ^ v_place(key)) * 16) = vx[i];
          }
        }
        return there;
      };
      if (step < min(last, nctx)) look_up(step);
      sweep(step, min(last, nctx), fetch, store, [&](int, int, uint64_t there) { return there; }, false);
    }
    const int tid = thread_again();
    int node[RG], row[RG];
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      row[r] = rt * kRows + (tid >> 6) * (16 * RG) + r * 16 + (tid & 15);
      node[r] = min(row[r], rows - 1) / a.group;
    }
    {   // the tree's own keys
      const int words = (a.budget + 63) / 64;
      constexpr int kShares = kTile / (4 * W);
      const int key0 = tid >> 4, c = tid & 15;
      u32x4 kx[kShares], vx[kShares];
      uint64_t in_flight = 0, next_seen[RG], seen[RG];   // mask words of the tile in flight, of the stored one
      auto fetch = [&](int s) __attribute__((always_inline)) {
        const int kb = (s - nctx) * kTile, valid = min(kTile, ex.nodes - kb);   // 0 where a request has no keys at all
        in_flight = valid >= 64 ? ~0ull : (1ull << max(valid, 0)) - 1;
        if (a.mask) {
#pragma unroll
          for (int r = 0; r < RG; ++r)
            next_seen[r] = a.mask[(int64_t(q) * a.budget + node[r]) * words + min(s - nctx, words - 1)];
        }
#pragma unroll
        for (int i = 0; i < kShares; ++i) {
          const int key = min(kb + 4 * W * i + key0, a.budget - 1);
          const int64_t off = (int64_t(q) * a.budget + key) * a.kv_stride + kvh * kHead + 8 * c;
          kx[i] = *reinterpret_cast<const u32x4*>(a.k_tree + off);
          vx[i] = *reinterpret_cast<const u32x4*>(a.v_tree + off);
        }
      };
      auto store = [&](auto B) __attribute__((always_inline)) -> uint64_t {
        const u32x4 zero{0, 0, 0, 0};
        LDS_AS char* const kt = lds + B.value * 2 * kTileBytes;
#pragma unroll
        for (int i = 0; i < kShares; ++i) {
          const int key = 4 * W * i + key0;
          if (!((in_flight >> key) & 1)) vx[i] = zero;
          if ((odd_bits(vx[i][0]) | odd_bits(vx[i][1]) | odd_bits(vx[i][2]) | odd_bits(vx[i][3])) & kOdd) {
            odd = turn;
#pragma unroll
            for (int x = 0; x < 4; ++x) vx[i][x] = without_odd(vx[i][x]);
          }
          *reinterpret_cast<LDS_AS u32x4*>(kt + key * kRowBytes + (c ^ k_place(key)) * 16) = kx[i];
          *reinterpret_cast<LDS_AS u32x4*>(kt + kTileBytes + key * kRowBytes + (c ^ v_place(key)) * 16) = vx[i];
        }
#pragma unroll
        for (int r = 0; r < RG; ++r) seen[r] = next_seen[r];
        return in_flight;
      };
      auto sees = [&](int s, int r, uint64_t there) __attribute__((always_inline)) -> uint64_t {
        if (a.mask) return there & seen[r];
        const int d = node[r] - (s - nctx) * kTile;   // a chain's node sees keys up to its own
        return there & (d < 0 ? 0ull : d >= 63 ? ~0ull : (2ull << d) - 1);
      };
      sweep(max(step, nctx), last, fetch, store, sees, true);
      // a wave that is ahead may have raised it for its next item: then nothing is found here
      if (odd >= turn) {
        for (int s = max(step, nctx); s < last; ++s) {
          const int kb = (s - nctx) * kTile, valid = min(kTile, ex.nodes - kb);
          if (valid <= 0) break;
          const uint64_t there = valid == kTile ? ~0ull : (1ull << valid) - 1;
#pragma unroll
          for (int r = 0; r < RG; ++r) {
            const int d = node[r] - kb;
            const uint64_t sees = there & (a.mask ? a.mask[(int64_t(q) * a.budget + node[r]) * words + (s - nctx)]
                                                  : d < 0 ? 0ull : d >= 63 ? ~0ull : (2ull << d) - 1);
            for (int key = 0; key < valid; ++key) {
              if (!((sees >> key) & 1)) continue;
              const uint16_t* vp = a.v_tree + (int64_t(q) * a.budget + kb + key) * a.kv_stride + kvh * kHead + 4 * ((tid & 63) >> 4);
#pragma unroll
              for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[r][t][i] += odd_part(vp[16 * t + i]);
            }
          }
        }
      }
    }

    const bool direct = n == steps;
    const int slot = 2 * blk + (step > 0 ? 0 : 1);
    const int ge = (tid & 63) >> 4;
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      float total = l[r];
      total += __shfl_xor(total, 16);
      total += __shfl_xor(total, 32);
      if (row[r] >= rows) continue;
      if (direct) {
        const float inv = total > 0.f ? 1.f / total : 0.f;   // a row that sees nothing is zero
        uint16_t* op = a.out + ((int64_t(q) * a.budget + node[r]) * a.heads_q + kvh * a.group + row[r] - node[r] * a.group) * kHead;
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int t = 0; t < 8; ++t)
          *reinterpret_cast<bf16x4*>(op + 16 * t + 4 * ge) =
              bf16x4{__bf16(o[r][t][0] * inv), __bf16(o[r][t][1] * inv), __bf16(o[r][t][2] * inv), __bf16(o[r][t][3] * inv)};
      } else {
        const Parts parts = parts_of<kRows>(a, blocks);
        const int64_t lr = int64_t(slot) * kRows + row[r] - rt * kRows;
#pragma unroll
        for (int t = 0; t < 8; ++t) *reinterpret_cast<f32x4*>(parts.o + lr * kHead + 16 * t + 4 * ge) = o[r][t];
        if (ge == 0) {
          parts.ml[lr * 2] = m[r];
          parts.ml[lr * 2 + 1] = total;
        }
      }
    }

    left -= n;
    step = 0;
    if (++item == per) {
      item = 0;
      ++q;
    }
  }
}

// A row's partial result while parts are folded into it in order.  A part without
// a seen key has a sum of 0 (of NaN where its only keys are).
struct Folded {
  float m, l;
  f32x4 o;
};
template <int N>
__device__ __forceinline__ void fold(Folded& r, const bool (&use)[N], const float (&m)[N], const float (&l)[N], const f32x4 (&o)[N],
                                     float c2) {
  float top = r.m;
  bool any = false;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (use[i] && l[i] != 0.f) {
      any = true;
      top = fmaxf(top, m[i]);
    }
  if (!any) return;
  const float f = __builtin_amdgcn_exp2f((r.m - top) * c2);
  r.l = r.l == 0.f ? 0.f : r.l * f;
  r.o *= r.l == 0.f ? 0.f : f;
  r.m = top;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (use[i] && l[i] != 0.f) {
      const float w = __builtin_amdgcn_exp2f((m[i] - top) * c2);
      r.l += w * l[i];
      r.o += o[i] * w;
    }
}

// Join the partial results of the items that were cut: block (item, 8 / G of its
// rows), 32 lanes for each G-th of a row's parts.  B parts are loaded together
// and folded in block order, then the G results.
template <int ROWS, int STEP, int G>
__global__ __launch_bounds__(256) void paged_join(PagedArgs a, int blocks) {
  constexpr int R = 8 / G, B = G == 1 ? 8 : 4;
  const int rows = a.budget * a.group, ntile = (rows + ROWS - 1) / ROWS, per = a.heads_kv * ntile;
  const int part = blockIdx.x % (ROWS / R);
  const int it = blockIdx.x / (ROWS / R);
  const int q = it / per, item = it - q * per;
  const int lane = threadIdx.x & 63;
  int64_t total = 0, before = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) {
    const int mine = q0 + lane < a.batch ? extent_of<STEP>(a, q0 + lane).steps() : 0;
    total += wave_sum_int(mine);
    before += wave_sum_int(q0 + lane < q ? mine : 0);
  }
  const int steps = extent_at<STEP>(a, q).steps();
  total = uniform64(total * per);
  const int64_t first = uniform64(before * per + int64_t(item) * steps);
  const int b0 = int(((first + 1) * blocks - 1) / total), b1 = int(((first + steps) * blocks - 1) / total);
  if (b0 == b1) return;
  const int kvh = item / ntile, rt = item - kvh * ntile;
  const int group = threadIdx.x >> 5;
  const int lr = part * R + group % R, row = rt * ROWS + lr, d = 4 * (threadIdx.x & 31);
  if (row >= rows) return;   // G > 1: the whole block
  const Parts parts = parts_of<ROWS>(a, blocks);
  const int each = (b1 - b0 + G) / G, c1 = G == 1 ? b1 : min(b0 + (group + 1) * each - 1, b1);
  Folded r{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const bool sparse = total < blocks;   // fewer steps than blocks: some have none
  for (int c0 = G == 1 ? b0 : b0 + group * each; c0 <= c1; c0 += B) {
    float m[B], l[B];
    f32x4 o[B];
    bool use[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int b = min(c0 + i, c1);
      const int64_t p = int64_t(2 * b + (b == b0 ? 1 : 0)) * ROWS + lr;
      const f32x2 ml = *reinterpret_cast<const f32x2*>(parts.ml + 2 * p);
      o[i] = *reinterpret_cast<const f32x4*>(parts.o + p * kHead + d);
      m[i] = ml[0];
      l[i] = ml[1];
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int b = c0 + i;
      use[i] = b <= c1 && !(sparse && total * b / blocks == total * (b + 1) / blocks);
    }
    fold(r, use, m, l, o, a.scale_log2);
  }
  if constexpr (G > 1) {
    __shared__ f32x4 go[G][32];
    __shared__ float gm[G], gl[G];
    go[group][threadIdx.x & 31] = r.o;
    if ((threadIdx.x & 31) == 0) {
      gm[group] = r.m;
      gl[group] = r.l;
    }
    __syncthreads();
    if (group > 0) return;
    float m[G], l[G];
    f32x4 o[G];
    bool use[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      m[i] = gm[i];
      l[i] = gl[i];
      o[i] = go[i][threadIdx.x];
      use[i] = true;
    }
    r = Folded{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
    fold(r, use, m, l, o, a.scale_log2);
  }
  const float inv = r.l > 0.f ? 1.f / r.l : r.l;   // a row that sees nothing is zero
  const int node = row / a.group;
  uint16_t* out = a.out + ((int64_t(q) * a.budget + node) * a.heads_q + kvh * a.group + row - node * a.group) * kHead + d;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(out) = bf16x4{__bf16(r.o[0] * inv), __bf16(r.o[1] * inv), __bf16(r.o[2] * inv), __bf16(r.o[3] * inv)};
}

// Which kernel, its tile's query rows and the blocks of a launch: as many as the
// chip holds, sharing the line of steps, or one per item.
enum Kernel { kFew, kFewWhole, kTiles64, kTiles128, kTiles256 };
struct Plan {
  Kernel kernel;
  int rows, blocks, whole;
  int64_t items;
};
Plan plan_of(int batch, int budget, int max_ctx, int heads_q, int heads_kv, int eight) {
  constexpr int kResident = 512;   // two blocks of four waves a compute unit
  const int rows = budget * (heads_q / heads_kv);
  const int64_t heads = int64_t(batch) * heads_kv;
  auto tiles_of = [&](int n) { return heads * ((rows + n - 1) / n); };
  Plan p{};
  // Few 16-row items with few keys: a block of eight waves takes each, with no
  // partial results and no second launch.  A compute unit draws about 47 GB/s,
  // 1.4 us per 256 keys of e4m3.  Whole / shared (us, 32 / 8 heads, e4m3 unless
  // said): 1 request x 64 nodes, 512 positions 10 / 18, 1024 13 / 21, 2048 18.4 /
  // 21.4, 2450 21.1 / 21.5, 2700 22.7 / 21.6, 3300 25 / 23.5, 4096 32 / 26 (bf16 1100
  // 16 / 20, 1500 19.2 / 19.9, 2048 24 / 22); 40 nodes 2048 17.8 / 20.7, 2450 20.5 /
  // 20.6; 2 x 64 x 2048 20 / 25; 4 x 64 x 700 21.5 / 21.8, 960 24.5 / 23.4, 1500 31 /
  // 29, 8 x 64 x 1024 48 / 36; 4 x 16 x 2048 20 / 23; single tokens: 1 x 512 8 / 10,
  // 1 x 2048 18 / 10, 8 x 800 10.8 / 11.6, 8 x 2048 18 / 16, 16 x 2048 18.5 / 20.6,
  // 32 x 800 14 / 18, 2048 25 / 31.
  const int64_t turns = ((int64_t(max_ctx) + budget + 255) / 256) * (eight ? 1 : 2), few = tiles_of(16);
  // At most 64 items of 16 rows over middle contexts: shared out as for few rows
  // (us, 1 request, 32 / 8 heads, whole or tiles of 64 rows / this way): 8 nodes,
  // 1280 positions 12.8 / 10.7, 2048 16.9 / 12.1, 16000 22.1 / 18.9, 32768 in bf16
  // 41 / 47; 16 x 4096 20.5 / 16.3, 16000 25.2 / 25.3; 32 x 1280 13.2 / 15.2, 2048 17.5 / 15.9, 4096
  // 21.4 / 19.5, 8192 26.0 / 25.8.
  const bool middle = rows > 16 && few <= 64 && turns > (few <= 32 ? 4 : 8) && turns <= (few <= 32 ? 64 : 32);
  if (!middle && few <= 512 && (turns <= 3 || (turns <= 4 && rows > 16) || (turns <= 9 && few <= 256 && (rows > 16 || few >= 128)))) {
    p.kernel = kFewWhole;
    p.rows = 16;
    p.items = p.blocks = int(few);
    p.whole = 1;
    return p;
  }
  const int step = rows <= 16 || middle ? 128 : kTile;
  const int64_t steps = (int64_t(max_ctx) + step - 1) / step + (budget + step - 1) / step;
  // 128 rows a tile (two groups a wave) double a tile's products per byte from LDS,
  // and a cut item's partial results; worth it where blocks take eight steps and
  // more.  256 rows (eight waves, an item a block) halve the work of storing tiles;
  // worth it from three quarters of an item a compute unit on, where few of their
  // rows are idle.  128 rows / 256 rows (us, 512 nodes over 2048 positions, 32 / 8
  // heads, e4m3, 64 items of 256 rows a request; whole and ragged contexts):
  // 2 requests 89 / 101, 3 127 / 107 and 116 / 101, 4 137 / 115 and 140 / 100, 5 191 /
  // 197, 8 255 / 215 and 244 / 191, 12 367 / 313 and 365 / 290, 16 435 / 397 and 405 /
  // 375, 17 468 / 480, 32 ragged 741 / 707; 4 over 500 positions 69 / 53, over 16000
  // 632 / 575; bf16 alike.
  const bool wide = tiles_of(256) >= 192 && 10 * 256 * tiles_of(256) <= 11 * 128 * tiles_of(128);
  p.kernel = rows <= 16 || middle ? kFew : rows <= 64 || tiles_of(128) * steps < 8 * kResident ? kTiles64 : wide ? kTiles256 : kTiles128;
  p.rows = p.kernel == kFew ? 16 : p.kernel == kTiles64 ? 64 : p.kernel == kTiles128 ? 128 : 256;
  p.items = tiles_of(p.rows);
  p.whole = p.kernel == kTiles256 || p.items >= 4 * kResident;
  p.blocks = int(p.whole ? p.items : std::min<int64_t>(kResident, p.items * steps));
  return p;
}

template <typename K>
hipError_t launch_whole(K* kernel, int threads, const PagedArgs& a, const Plan& p, hipStream_t s) {
  hipLaunchKernelGGL(kernel, dim3(p.blocks), dim3(threads), 0, s, a, 1);
  return hipGetLastError();
}
template <int ROWS, int STEP, typename K>
hipError_t launch(K* kernel, const PagedArgs& a, const Plan& p, hipStream_t s) {
  if (p.whole) return launch_whole(kernel, 256, a, p, s);
  hipLaunchKernelGGL(kernel, dim3(p.blocks), dim3(256), 0, s, a, 0);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Many parts an item are shared out over eight groups of lanes, which takes eight
  // times the blocks (us, with one group / eight, 32 / 8 heads: 16 rows, 64 parts,
  // one token over 8192 positions 19.3 / 14.1; 16 parts, 4 tokens over 16384 36.9 /
  // 35.7; 64 rows, 32 parts, 2 x 16 nodes over 65536 116.5 / 116.1; 16 parts, 64
  // nodes over 8192 32.0 / 32.9).
  if (p.blocks > std::max(8, ROWS / 4) * p.items)
    hipLaunchKernelGGL((paged_join<ROWS, STEP, 8>), dim3(unsigned(p.items * ROWS)), dim3(256), 0, s, a, p.blocks);
  else
    hipLaunchKernelGGL((paged_join<ROWS, STEP, 1>), dim3(unsigned(p.items * (ROWS / 8))), dim3(256), 0, s, a, p.blocks);
  return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace(int batch, int budget, int max_ctx, int heads_q, int heads_kv, int eight) {
  const Plan p = plan_of(batch, budget, max_ctx, heads_q, heads_kv, eight);
  return p.whole ? 0 : size_t(p.blocks) * 2 * p.rows * (kHead + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t s) {
  const Plan p = plan_of(a.batch, a.budget, a.max_ctx, a.heads_q, a.heads_kv, a.eight);
  switch (p.kernel) {
    case kFew:
      return a.eight ? launch<16, 128>(paged_attention<true, 4>, a, p, s) : launch<16, 128>(paged_attention<false, 4>, a, p, s);
    case kFewWhole:
      return a.eight ? launch_whole(paged_attention<true, 8>, 512, a, p, s) : launch_whole(paged_attention<false, 8>, 512, a, p, s);
    case kTiles64:
      return a.eight ? launch<64, kTile>(paged_tiles<1, true, 4>, a, p, s) : launch<64, kTile>(paged_tiles<1, false, 4>, a, p, s);
    case kTiles128:
      return a.eight ? launch<128, kTile>(paged_tiles<2, true, 4>, a, p, s) : launch<128, kTile>(paged_tiles<2, false, 4>, a, p, s);
    default:
      return a.eight ? launch_whole(paged_tiles<2, true, 8>, 512, a, p, s) : launch_whole(paged_tiles<2, false, 8>, 512, a, p, s);
  }
}

}  // namespace dartree
