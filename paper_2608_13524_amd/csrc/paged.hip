// Attention of drafted trees, chains and single tokens over a paged cache.
//
// One pass over the keys with a running maximum and sum per query row.  Work
// is counted in steps of 128 keys: those of a request's context, then those of
// its tree, for every (key/value head, tile of 16 RG query rows).  The steps of
// all requests lie on one line that the blocks share equally (or every block
// takes one whole item, where there are many), so ragged contexts cost no idle
// compute units; an item cut by a block's end leaves partial results, which a
// second launch joins in block order.
//
// A step's four chunks of 32 keys go to the block's four waves, and a wave works
// from registers alone.  S^T = K Q^T: row r of the two 16-key tiles is key
// 8 (r / 4) + 4 t + r % 4, which leaves lane (c = lane % 16, g = lane / 16) with
// query c's weights of keys 8 g .. 8 g + 7 in order, the B operand of O^T = V^T P^T.
// For V a lane reads eight dims, 8 c .. 8 c + 7, of those same keys and
// transposes them in registers; column tile t of the product is then dims 8 c + t,
// and a lane ends with dims 32 g .. 32 g + 31 of its query.  Keys in e4m3 become
// bf16 on the way with their power of two applied by the conversion (exact).
// Every key and value byte is read once per tile and never passes through LDS.
#include <algorithm>

#include "reduce.hpp"
#include "serve.hpp"

namespace dartree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kChunk = 32;            // keys of a wave's share of a step
constexpr int kWaves = 4;
constexpr int kStep = kChunk * kWaves;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool HI>
__device__ __forceinline__ uint32_t expand2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

struct Extent {   // a request's keys
  int ctx, nodes;
  __device__ int ctx_steps() const { return (ctx + kStep - 1) / kStep; }
  __device__ int steps() const { return max(1, ctx_steps() + (nodes + kStep - 1) / kStep); }
};
__device__ __forceinline__ Extent extent_of(const PagedArgs& a, int q) {
  return Extent{a.ctx_len ? min(max(a.ctx_len[q], 0), a.max_ctx) : a.max_ctx,
                a.num_nodes ? min(max(a.num_nodes[q], 0), a.budget) : a.budget};
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x))))) | (int64_t(uniform(int(x >> 32))) << 32);
}

// Sum over the requests of their steps.
__device__ __forceinline__ int64_t all_steps(const PagedArgs& a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) total += wave_sum_int(q0 + lane < a.batch ? extent_of(a, q0 + lane).steps() : 0);
  return total;
}

// The request that step `at` of the line lies in (`per` steps of the line per
// step of a request) and the steps before that request.
__device__ __forceinline__ int find_request(const PagedArgs& a, int64_t at, int per, int64_t* before) {
  const int lane = threadIdx.x & 63;
  int64_t sum = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) {
    const int mine = q0 + lane < a.batch ? extent_of(a, q0 + lane).steps() : 0;
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

template <int RG>
struct Rows {   // a wave's running result for its query rows
  f32x4 o[RG][8];   // o[.][t][i]: dim 32 g + 8 i + t
  float m[RG], l[RG];   // l: this lane's keys only
};

template <int RG, bool E8>
struct Chunk {   // 32 keys and values as read
  u32x4 k[2][E8 ? 2 : 4];
  u32x2 v8[E8 ? 8 : 1];
  u32x4 v16[E8 ? 1 : 8];
  uint8_t ke[2];
  u32x2 ve;
};

// S, softmax and O of one chunk.  vis: bit 8 g + i set where lane group g's key i
// is seen by row group r's query (masked: some bit is clear).
template <int RG, bool E8>
__device__ __forceinline__ void chunk_step(const Chunk<RG, E8>& c, const u32x4 (&qf)[RG][4], const bool masked,
                                           const uint32_t (&vis)[RG], const uint32_t there, const float c2, Rows<RG>& st) {
  const int g = (threadIdx.x & 63) >> 4;
  f32x4 s[RG][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int r = 0; r < RG; ++r) s[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x4 kf;
      if constexpr (E8) {
        const float sc = __uint_as_float(uint32_t(c.ke[t]) << 23);
        const uint32_t w0 = c.k[t][ks >> 1][2 * (ks & 1)], w1 = c.k[t][ks >> 1][2 * (ks & 1) + 1];
        kf = u32x4{expand2<false>(w0, sc), expand2<true>(w0, sc), expand2<false>(w1, sc), expand2<true>(w1, sc)};
      } else {
        kf = c.k[t][ks];
      }
#pragma unroll
      for (int r = 0; r < RG; ++r) s[r][t] = mfma16(kf, qf[r][ks], s[r][t]);
    }
  }
  if (masked) {
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      const uint32_t b = vis[r] >> (8 * g);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!((b >> (4 * t + i)) & 1u)) s[r][t][i] = -INFINITY;
    }
  }
  // The reference m of a row moves only when a key exceeds it by more than 2^8,
  // so most chunks need no exchange between lanes and no rescaling; weights
  // stay below 2^8 and a row that has seen no key keeps m = -inf, l = 0, O = 0.
  u32x4 p[RG];
#pragma unroll
  for (int r = 0; r < RG; ++r) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][t][i]);
    if (__any(top * c2 > st.m[r] * c2 + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m = top * c2 > st.m[r] * c2 + 8.f ? top : st.m[r];
      const float f = __builtin_amdgcn_exp2f((st.m[r] - (m == -INFINITY ? 0.f : m)) * c2);
      st.l[r] *= f;
#pragma unroll
      for (int t = 0; t < 8; ++t) st.o[r][t] *= f;
      st.m[r] = m;
    }
    const float ref = -(st.m[r] == -INFINITY ? 0.f : st.m[r]) * c2;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[r][t][i] = __builtin_amdgcn_exp2f(fmaf(s[r][t][i], c2, ref));
        st.l[r] += s[r][t][i];
      }
    bf16x8 w;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * t + i] = __bf16(s[r][t][i]);
    p[r] = __builtin_bit_cast(u32x4, w);
  }
  // V: dims 8 c + 2 j, 8 c + 2 j + 1 of eight keys, transposed.  A key that is
  // not there has zeros instead of what its memory holds: 0 * NaN is NaN.
  const uint32_t here = there >> (8 * g);
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
      } else {
        w[e] = c.v16[e][j];
      }
      if (!whole) w[e] = (here >> e) & 1u ? w[e] : 0u;
    }
    u32x4 lo, hi;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      lo[x] = __builtin_amdgcn_perm(w[2 * x + 1], w[2 * x], 0x05040100u);
      hi[x] = __builtin_amdgcn_perm(w[2 * x + 1], w[2 * x], 0x07060302u);
    }
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      st.o[r][2 * j] = mfma16(lo, p[r], st.o[r][2 * j]);
      st.o[r][2 * j + 1] = mfma16(hi, p[r], st.o[r][2 * j + 1]);
    }
  }
}

// Partial results: slot s of part_o holds the unnormalised rows [16 RG][128] of
// one cut item, part_ml their {m, l}.  Block i's first item, if cut at its
// beginning, is slot 2 i, its last, if it begins there and is cut at its end,
// slot 2 i + 1.
struct Parts {
  float* o;
  float* ml;
};
template <int RG>
__device__ __forceinline__ Parts parts_of(const PagedArgs& a, int blocks) {
  float* o = static_cast<float*>(a.ws);
  return Parts{o, o + int64_t(blocks) * 2 * 16 * RG * kHead};
}

template <int RG, bool E8>
__global__ __launch_bounds__(256, RG == 1 ? 2 : 1) void paged_attention(PagedArgs a, int whole) {
  __shared__ __attribute__((aligned(16))) float red[kWaves * RG * 8 * 64 * 4];
  __shared__ float ml[kWaves][16 * RG][2];
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int rows = a.budget * a.group, ntile = (rows + 16 * RG - 1) / (16 * RG);
  const int per = a.heads_kv * ntile;   // items of a request
  const int blocks = gridDim.x, blk = xcd_order(blockIdx.x, blocks);
  const Parts parts = parts_of<RG>(a, blocks);
  const int words = 2 * ((a.budget + 63) / 64);
  const int page_size = 1 << a.c.page_log2;

  int q, item, step, left;   // request, item of it, step of that, steps the block still has
  if (whole) {
    q = blk / per;
    item = blk - q * per;
    step = 0;
    left = uniform(extent_of(a, q).steps());
  } else {
    const int64_t total = uniform64(all_steps(a) * per);
    const int64_t s0 = total * blk / blocks, s1 = total * (blk + 1) / blocks;
    left = uniform(int(s1 - s0));
    if (left <= 0) return;
    int64_t before;
    q = find_request(a, s0, per, &before);
    const int steps = uniform(extent_of(a, q).steps());
    const int64_t in = s0 - before;
    item = uniform(int(in / steps));
    step = uniform(int(in - int64_t(item) * steps));
  }

  while (left > 0) {
    Extent ex = extent_of(a, q);
    ex.ctx = uniform(ex.ctx);
    ex.nodes = uniform(ex.nodes);
    const int steps = ex.steps(), nctx = ex.ctx_steps();
    const int n = min(left, steps - step);
    const int kvh = item / ntile, rt = item - kvh * ntile;

    u32x4 qf[RG][4];
    Rows<RG> st;
    const uint32_t* mrow[RG];
    int node[RG];
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      const int row = min(rt * 16 * RG + r * 16 + c16, rows - 1);   // past the end: the last row, never stored
      node[r] = row / a.group;
      const int64_t at = (int64_t(q) * a.budget + node[r]) * a.q_stride + (kvh * a.group + row - node[r] * a.group) * kHead;
      // operand ks: dims 64 (ks / 2) + 16 g + 8 (ks % 2) .. + 7, for keys alike
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        qf[r][ks] = *reinterpret_cast<const u32x4*>(a.q + at + 64 * (ks >> 1) + 16 * g + 8 * (ks & 1));
      mrow[r] = a.mask ? reinterpret_cast<const uint32_t*>(a.mask) + (int64_t(q) * a.budget + node[r]) * words : nullptr;
      st.m[r] = -INFINITY;
      st.l[r] = 0.f;
#pragma unroll
      for (int t = 0; t < 8; ++t) st.o[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // context: chunk of keys kb .. kb + 31
    const int32_t* table = a.c.table + int64_t(q) * a.c.max_pages;
    auto pages_of = [&](int kb, int& p0, int& p1) {   // pages of the chunk's halves; -1: none
      p0 = table[kb >> a.c.page_log2];
      p0 = p0 < a.c.num_pages ? p0 : -1;
      const int k1 = kb + 16;
      p1 = k1 < ex.ctx ? table[k1 >> a.c.page_log2] : -1;
      p1 = p1 < a.c.num_pages ? p1 : -1;
    };
    const int end = min(step + n, nctx);
    for (int s = step; s < end; ++s) {
      const int kb = s * kStep + wave * kChunk;
      if (kb >= ex.ctx) break;
      int p0, p1;
      pages_of(kb, p0, p1);
      p0 = uniform(p0);
      p1 = uniform(p1);
      if (p0 < 0 && p1 < 0) continue;
      const int valid = min(kChunk, ex.ctx - kb);
      uint32_t there = valid == 32 ? ~0u : (1u << valid) - 1u;
      if (p0 < 0) there &= 0xFFFF0000u;
      if (p1 < 0) there &= 0x0000FFFFu;
      const int h0 = p0 < 0 ? p1 : p0, h1 = p1 < 0 ? p0 : p1;   // a page to read from in any case
      auto row_of = [&](int key) {
        const int64_t page = key < 16 ? h0 : h1;
        return ((page * a.heads_kv + kvh) << a.c.page_log2) + ((kb + key) & (page_size - 1));
      };
      Chunk<RG, E8> ch;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t row = row_of(8 * (c16 >> 2) + 4 * t + (c16 & 3));
        if constexpr (E8) {
          const uint8_t* kp = static_cast<const uint8_t*>(a.c.k) + row * kHead + 16 * g;
          ch.k[t][0] = *reinterpret_cast<const u32x4*>(kp);
          ch.k[t][1] = *reinterpret_cast<const u32x4*>(kp + 64);
          ch.ke[t] = a.c.k_exp[row];
        } else {
          const uint16_t* kp = static_cast<const uint16_t*>(a.c.k) + row * kHead + 16 * g;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            ch.k[t][ks] = *reinterpret_cast<const u32x4*>(kp + 64 * (ks >> 1) + 8 * (ks & 1));
        }
      }
      const int64_t vrow = row_of(8 * g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (E8)
          ch.v8[e] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.c.v) + (vrow + e) * kHead + 8 * c16);
        else
          ch.v16[e] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.c.v) + (vrow + e) * kHead + 8 * c16);
      }
      if constexpr (E8) ch.ve = *reinterpret_cast<const u32x2*>(a.c.v_exp + vrow);
      uint32_t vis[RG];
#pragma unroll
      for (int r = 0; r < RG; ++r) vis[r] = there;
      chunk_step<RG, E8>(ch, qf, there != ~0u, vis, there, a.scale_log2, st);
    }
    // the tree's own keys
    for (int s = max(step, nctx); s < step + n; ++s) {
      const int kb = (s - nctx) * kStep + wave * kChunk;
      if (kb >= ex.nodes) break;
      const int valid = min(kChunk, ex.nodes - kb);
      const uint32_t there = valid == 32 ? ~0u : (1u << valid) - 1u;
      auto at = [&](int key) {
        return (int64_t(q) * a.budget + min(kb + key, ex.nodes - 1)) * a.kv_stride + kvh * kHead;
      };
      Chunk<RG, false> ch;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint16_t* kp = a.k_tree + at(8 * (c16 >> 2) + 4 * t + (c16 & 3)) + 16 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          ch.k[t][ks] = *reinterpret_cast<const u32x4*>(kp + 64 * (ks >> 1) + 8 * (ks & 1));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        ch.v16[e] = *reinterpret_cast<const u32x4*>(a.v_tree + at(8 * g + e) + 8 * c16);
      uint32_t vis[RG];
#pragma unroll
      for (int r = 0; r < RG; ++r) {
        if (mrow[r]) vis[r] = mrow[r][kb >> 5] & there;
        else vis[r] = node[r] < kb ? 0u : (node[r] - kb >= 31 ? ~0u : (2u << (node[r] - kb)) - 1u) & there;
      }
      chunk_step<RG, false>(ch, qf, true, vis, there, a.scale_log2, st);
    }

    // join the four waves: their rows scaled to the block's maximum, added in wave order
#pragma unroll
    for (int r = 0; r < RG; ++r) {
      float l = st.l[r];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (g == 0) {
        ml[wave][r * 16 + c16][0] = st.m[r];
        ml[wave][r * 16 + c16][1] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<f32x4*>(&red[(((wave * RG + r) * 8 + 2 * i + h) * 64 + lane) * 4]) =
              f32x4{st.o[r][4 * h][i], st.o[r][4 * h + 1][i], st.o[r][4 * h + 2][i], st.o[r][4 * h + 3][i]};
    }
    __syncthreads();
    const bool direct = n == steps;
    const int slot = 2 * blk + (step > 0 ? 0 : 1);
#pragma unroll
    for (int r = 0; r < RG; ++r) {   // this wave: dims 32 g + 8 wave .. + 7 of every row
      const int lr = r * 16 + c16, row = rt * 16 * RG + lr;
      float M = ml[0][lr][0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, ml[w][lr][0]);
      float L = 0.f;
      f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = ml[w][lr][0];
        const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - M) * a.scale_log2);
        L += f * ml[w][lr][1];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          v[h] += f * *reinterpret_cast<const f32x4*>(&red[(((w * RG + r) * 8 + 2 * wave + h) * 64 + lane) * 4]);
      }
      if (row < rows) {
        if (direct) {
          const float inv = L > 0.f ? 1.f / L : 0.f;   // a row that sees nothing is zero
          bf16x8 o;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = __bf16(v[i >> 2][i & 3] * inv);
          const int nd = row / a.group;
          const int64_t head = (int64_t(q) * a.budget + nd) * a.heads_q + kvh * a.group + row - nd * a.group;
          *reinterpret_cast<bf16x8*>(a.out + head * kHead + 32 * g + 8 * wave) = o;
        } else {
          float* po = parts.o + (int64_t(slot) * 16 * RG + lr) * kHead + 32 * g + 8 * wave;
          *reinterpret_cast<f32x4*>(po) = v[0];
          *reinterpret_cast<f32x4*>(po + 4) = v[1];
          if (wave == 0 && g == 0) {
            parts.ml[(int64_t(slot) * 16 * RG + lr) * 2] = M;
            parts.ml[(int64_t(slot) * 16 * RG + lr) * 2 + 1] = L;
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

// Join the partial results of the items that were cut: block (item, eight of its
// rows), 32 lanes per row.
template <int RG>
__global__ __launch_bounds__(256) void paged_attention_join(PagedArgs a, int blocks) {
  const int rows = a.budget * a.group, ntile = (rows + 16 * RG - 1) / (16 * RG), per = a.heads_kv * ntile;
  const int part = blockIdx.x % (2 * RG);
  const int it = blockIdx.x / (2 * RG);
  const int q = it / per, item = it - q * per;
  const int lane = threadIdx.x & 63;
  int64_t total = 0, before = 0;
  for (int q0 = 0; q0 < a.batch; q0 += 64) {
    const int mine = q0 + lane < a.batch ? extent_of(a, q0 + lane).steps() : 0;
    total += wave_sum_int(mine);
    before += wave_sum_int(q0 + lane < q ? mine : 0);
  }
  const int steps = uniform(extent_of(a, q).steps());
  total = uniform64(total * per);
  const int64_t first = uniform64(before * per + int64_t(item) * steps);
  const int b0 = int(((first + 1) * blocks - 1) / total), b1 = int(((first + steps) * blocks - 1) / total);
  if (b0 == b1) return;
  const int kvh = item / ntile, rt = item - kvh * ntile;
  const int lr = part * 8 + (threadIdx.x >> 5), row = rt * 16 * RG + lr, d = 4 * (threadIdx.x & 31);
  if (row >= rows) return;
  const Parts parts = parts_of<RG>(a, blocks);
  float M = -INFINITY, L = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  for (int b = b0; b <= b1; ++b) {
    if (total * b / blocks == total * (b + 1) / blocks) continue;   // fewer steps than blocks: one without any
    const int64_t p = int64_t(2 * b + (b == b0 ? 1 : 0)) * 16 * RG + lr;
    const float m = parts.ml[2 * p], l = parts.ml[2 * p + 1];
    const f32x4 o = *reinterpret_cast<const f32x4*>(parts.o + p * kHead + d);
    if (m == -INFINITY) continue;
    const float top = fmaxf(M, m);
    const float f = __builtin_amdgcn_exp2f((M - top) * a.scale_log2), w = __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
    L = L * f + l * w;
    acc = acc * f + o * w;
    M = top;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  const int node = row / a.group;
  uint16_t* out = a.out + ((int64_t(q) * a.budget + node) * a.heads_q + kvh * a.group + row - node * a.group) * kHead + d;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(out) = bf16x4{__bf16(acc[0] * inv), __bf16(acc[1] * inv), __bf16(acc[2] * inv), __bf16(acc[3] * inv)};
}

// Row groups of 16 per tile, and the blocks of a launch.
struct Plan {
  int rg, blocks, whole;
  int64_t items;
};
Plan plan_of(int batch, int budget, int max_ctx, int heads_q, int heads_kv) {
  const int rows = budget * (heads_q / heads_kv);
  Plan p{};
  p.rg = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.items = int64_t(batch) * heads_kv * ((rows + 16 * p.rg - 1) / (16 * p.rg));
  const int resident = p.rg == 1 ? 512 : 256;
  p.whole = p.items >= 4 * resident;
  const int64_t steps = std::max(1, (max_ctx + kStep - 1) / kStep + (budget + kStep - 1) / kStep);
  p.blocks = int(p.whole ? p.items : std::min<int64_t>(resident, p.items * steps));
  return p;
}

template <int RG>
hipError_t launch(const PagedArgs& a, const Plan& p, hipStream_t s) {
  if (a.eight) hipLaunchKernelGGL((paged_attention<RG, true>), dim3(p.blocks), dim3(256), 0, s, a, p.whole);
  else hipLaunchKernelGGL((paged_attention<RG, false>), dim3(p.blocks), dim3(256), 0, s, a, p.whole);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.whole) return e;
  hipLaunchKernelGGL(paged_attention_join<RG>, dim3(unsigned(p.items * 2 * RG)), dim3(256), 0, s, a, p.blocks);
  return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace(int batch, int budget, int max_ctx, int heads_q, int heads_kv, int) {
  const Plan p = plan_of(batch, budget, max_ctx, heads_q, heads_kv);
  return p.whole ? 0 : size_t(p.blocks) * 2 * 16 * p.rg * (kHead + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedArgs& a, hipStream_t s) {
  const Plan p = plan_of(a.batch, a.budget, a.max_ctx, a.heads_q, a.heads_kv);
  return p.rg == 1 ? launch<1>(a, p, s) : p.rg == 2 ? launch<2>(a, p, s) : launch<4>(a, p, s);
}

}  // namespace dartree
