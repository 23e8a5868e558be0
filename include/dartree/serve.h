/*
 * libdartree, the serving side of a verification step: a paged key/value cache
 * that accepted tokens are written to and read back from, the attention of a
 * tree of drafted tokens over it, and the verification of drafted tokens from
 * given random numbers.  Conventions (stream, errors, alignment, validation
 * before anything is enqueued) are those of dartree.h; the calls here
 * allocate nothing and can be captured into a graph.  Sizes that would need a
 * launch of 2^32 threads are DARTREE_ERR_UNSUPPORTED.
 *
 * A verification step of a serving loop:
 *   dartree_build_tree            the draft
 *   dartree_tree_attention_paged  per layer of the target, over cache and tree
 *   dartree_verify_tree           accepted nodes and the next token
 *   dartree_cache_write           per layer, the accepted nodes' keys and values
 */
#ifndef DARTREE_SERVE_H
#define DARTREE_SERVE_H

#include "dartree.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- paged key/value cache ----------------------------------------------- */

typedef enum dartree_cache_type {
  DARTREE_CACHE_BF16 = 0, /* keys and values as given */
  DARTREE_CACHE_E4M3 = 1  /* 8 bits (OCP e4m3: 4 exponent bits, 3 of mantissa, largest 448) and one power of
                             two per position, head and side */
} dartree_cache_type;

/* Shape of a cache (host struct). */
typedef struct dartree_cache_params {
  int32_t batch;     /* b >= 1 requests: rows of the page table */
  int32_t heads_kv;  /* key/value heads, >= 1 */
  int32_t head_dim;  /* 128 */
  int32_t page;      /* positions of a page: 16, 32, 64, 128 or 256 */
  int32_t num_pages; /* pages in the pool, >= 1 */
  int32_t max_pages; /* columns of the page table, >= 1; max_pages * page <= 2^30 */
  int32_t type;      /* dartree_cache_type */
} dartree_cache_params;

/* Device memory of a cache.  Position t of request q lies in slot t % page of
 * page table[q][t / page].  An entry outside [0, num_pages) stands for no
 * page: its positions are dropped by a write, read as zeros and are not seen
 * by attention. */
typedef struct dartree_cache {
  void* k;              /* [num_pages][heads_kv][page][128], bf16 or e4m3 */
  void* v;
  uint8_t* k_exp;       /* E4M3: [num_pages][heads_kv][page], a row stands for its values * 2^(exp - 127); */
  uint8_t* v_exp;       /* BF16: not used, may be NULL */
  const int32_t* table; /* [b][max_pages] */
} dartree_cache;

/* Host-only check of `p` (no HIP call). */
dartree_status dartree_cache_validate(const dartree_cache_params* p);

/* Write keys and values into the cache: for request q and i < counts[q]
 * (counts NULL: rows; values above rows count as rows, negative ones as 0),
 * position start[q] + i (start NULL: 0) takes source row index[q][i] (index
 * NULL: row i, and source_rows >= rows).  A source row outside [0,
 * source_rows), a negative position and one past the page table are skipped,
 * so an acceptance walk's indices (-1 after the last) can be passed as they
 * are.  k, v: bf16, row j of request q at (q * source_rows + j) * row_stride
 * elements, heads_kv * 128 elements each; row_stride >= heads_kv * 128, a
 * multiple of 8 (rows of a fused projection need no copy).  index: [b][rows].
 *
 * E4M3: a row of 128 is held as e4m3(x * 2^-e), nearest even, with the least
 * e >= -100 for which the row's largest magnitude is at most 448 * 2^e (e =
 * -100 for a row of zeros); exp = e + 127.  Above e = -100 only values below
 * 2^-13.8 of the row's largest fall into e4m3's subnormals (a row's largest is
 * held above 224, the least normal number is 2^-6).
 * A NaN stays one; an infinity becomes one, and the other values of its row 0.
 *
 * Within a call, no two (request, position) pairs may share a slot.  Slots
 * that are not written keep their contents. */
dartree_status dartree_cache_write(const dartree_cache_params* p, const dartree_cache* cache, int32_t source_rows,
                                   int32_t rows, const void* k, const void* v, int64_t row_stride,
                                   const int32_t* index, const int32_t* counts, const int32_t* start,
                                   hipStream_t stream);

/* Read positions back as dense bf16: k, v [b][rows][heads_kv][128], row i of
 * request q is position start[q] + i for i < counts[q] (NULL as above), the
 * layout dartree_tree_attention takes its context in.  Exact: e4m3 times a
 * power of two fits bf16, but for +-2^128: the numbers from 248 * 2^120 (3.30e38)
 * on are held as that, and are read as bf16's largest, 255 * 2^120.  Positions
 * without a page are zeros; rows at and past counts[q] are left as they were. */
dartree_status dartree_cache_read(const dartree_cache_params* p, const dartree_cache* cache, int32_t rows, void* k,
                                  void* v, const int32_t* counts, const int32_t* start, hipStream_t stream);

/* ---- attention over the cache ---------------------------------------------- */

/* Bytes of device workspace for dartree_tree_attention_paged (host only):
 * partial results where keys are shared out over blocks, at most 65 MiB.  The size
 * belongs to these parameters: fewer requests, nodes or positions can need more
 * (0 where every block takes whole items).  A loop over several sizes keeps the
 * largest of their answers. */
dartree_status dartree_tree_attention_paged_workspace_size(const dartree_attn_params* a, const dartree_cache_params* p,
                                                           size_t* bytes);

/* dartree_tree_attention with the context in a paged cache.  The query of
 * node i of request q attends to the first ctx_len[q] positions (NULL: all
 * max_ctx; values are taken into 0 .. max_ctx) and to the nodes j < num_nodes[q]
 * (NULL: budget) whose bit is set in mask row i; mask NULL: j <= i, a chain
 * (budget 1: a single token).  Positions without a page and nodes at and past
 * num_nodes[q] are not seen; what the memory of a key holds that a row does not
 * see does not matter to that row, NaN and infinities included.
 * Every row i < budget is computed; one that sees nothing is 0.
 * a: as in dartree_tree_attention, with max_ctx <= max_pages * page, batch,
 * heads_kv and head_dim as in p; max_ctx is not limited otherwise.
 * q: bf16, node i of request r at (r * budget + i) * q_stride elements,
 * heads_q * 128 each; k_tree, v_tree: likewise with kv_stride and heads_kv;
 * strides are multiples of 8.  out: bf16 [b][budget][heads_q][128].
 * Products of bf16 values (e4m3 keys and values as dartree_cache_read gives
 * them) with fp32 accumulation, fp32 softmax; the weights are rounded to bf16 for
 * the weighted sum of values, the output to bf16.  Weights are at most 2^8 before
 * they are divided by their sum: values below 2^89 cannot overflow it.  The order
 * of sums is fixed by the arguments: equal calls give equal bits. */
dartree_status dartree_tree_attention_paged(const dartree_attn_params* a, const dartree_cache_params* p,
                                            const dartree_cache* cache, const void* q, int64_t q_stride,
                                            const void* k_tree, const void* v_tree, int64_t kv_stride,
                                            const uint64_t* mask, const int32_t* num_nodes, const int32_t* ctx_len,
                                            void* out, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- verification from given random numbers ---------------------------------- */

/* The target's distribution p of a row of logits is softmax(z / T) at T > 0
 * and all mass on the first largest logit at T = 0.  A NaN logit counts as
 * -inf, +inf as the largest finite number; a row without any mass (all -inf)
 * accepts nothing and its token is -1.  logits_type: DARTREE_FP32 or
 * DARTREE_BF16.  Sums, quotients and comparisons are taken in 64 bits, the
 * exponentials are good to 3e-12: a result can differ from the definition's only
 * where it hangs on less than 3e-11 of a row's mass. */

/* Bytes of device workspace for dartree_verify_tree / dartree_verify_chain
 * (host only).  That of trees, too, belongs to these sizes: smaller ones can need
 * more (all rows' records instead of those of some paths). */
dartree_status dartree_verify_tree_workspace_size(int32_t batch, int32_t budget, int32_t max_len, int32_t vocab,
                                                  size_t* bytes);
dartree_status dartree_verify_chain_workspace_size(int32_t batch, int32_t depth, int32_t vocab, size_t* bytes);

/* Verify trees whose tokens were chosen, not drawn (those of this library):
 * lossless sampling from the target.  Tree arrays as in dartree_accept_walk;
 * target_logits [b][B+1] rows of `vocab`, row_stride elements apart (>= vocab):
 * index 0 after the verified context, index i + 1 after node i.  uniforms
 * [b][B+1] in [0, 1): index 0 for the final token, index j + 1 for the test of
 * node j.  From the root, with p of the current row: the children are tested
 * in index order, child j with token x_j accepted iff
 *   u_{j+1} * (1 - sum of p over the children tested before) < p(x_j);
 * an accepted child becomes current.  If none is (or there is none), the final
 * token is drawn from p without the tested children's tokens: the lowest token
 * whose cumulated mass exceeds u_0 times the whole (where nothing is left, from
 * p).  After max_len accepted nodes no child is tested and the token is drawn
 * from p.  A token outside [0, vocab) has no mass.  Writes accepted
 * [b][max_len] (-1 after the last), num_accepted [b] and bonus [b] as
 * dartree_accept_walk does.  Children of one node must hold distinct tokens
 * (the builds' do; otherwise the final token is some token of the row).
 * 1 <= budget <= DARTREE_MAX_SORT, 1 <= max_len <= 2^20.  ws: device, 256-byte
 * aligned. */
dartree_status dartree_verify_tree(int32_t batch, int32_t budget, int32_t max_len, int32_t vocab, int32_t logits_type,
                                   const int32_t* tokens, const int32_t* parents, const int32_t* num_nodes,
                                   const void* target_logits, int64_t row_stride, float temperature,
                                   const float* uniforms, int32_t* accepted, int32_t* num_accepted, int32_t* bonus,
                                   void* ws, size_t ws_bytes, hipStream_t stream);

/* Verify chains drawn from the drafter, eq. (1) and (2): tokens [b][depth],
 * of which the first num_tokens[q] count (NULL: depth), token i drawn from the
 * distribution q_i of draft_logits row i (at the same T); target_logits
 * [b][depth + 1] rows: row i before token i.  uniforms [b][depth + 1]: index 0
 * for the final token, i + 1 for the test of token i, accepted iff
 *   u_{i+1} * q_i(x_i) < p_i(x_i)   (T = 0: iff x_i is the target's token).
 * At the first rejected i the final token is drawn from [p_i - q_i]_+ (from
 * p_i where that holds nothing), after the last accepted one from the
 * following row's p, as above.  Rows are row_stride elements apart in both.
 * Writes num_accepted [b] and bonus [b].  At T = 0 draft_logits is not read
 * and may be NULL.  1 <= depth <= DARTREE_MAX_DEPTH. */
dartree_status dartree_verify_chain(int32_t batch, int32_t depth, int32_t vocab, int32_t logits_type,
                                    const int32_t* tokens, const int32_t* num_tokens, const void* target_logits,
                                    const void* draft_logits, int64_t row_stride, float temperature,
                                    const float* uniforms, int32_t* num_accepted, int32_t* bonus, void* ws,
                                    size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DARTREE_SERVE_H */
