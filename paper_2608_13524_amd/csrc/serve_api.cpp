// C ABI of the serving operators (dartree/serve.h): argument checks, then one
// launcher each.  Nothing here touches the device before every check passed.
#include <math.h>

#include "serve.hpp"

using namespace dartree;

namespace {

bool given(const void* p) { return p && aligned16(p); }
bool optional(const void* p) { return !p || aligned16(p); }

dartree_status check_cache(const dartree_cache_params* p) {
  if (!p) return DARTREE_ERR_INVALID_ARG;
  if (p->batch < 1 || p->heads_kv < 1 || p->head_dim < 1 || p->page < 1 || p->num_pages < 1 || p->max_pages < 1)
    return DARTREE_ERR_INVALID_ARG;
  if (p->type != DARTREE_CACHE_BF16 && p->type != DARTREE_CACHE_E4M3) return DARTREE_ERR_INVALID_ARG;
  if (p->head_dim != kHead || p->heads_kv > 4096) return DARTREE_ERR_UNSUPPORTED;
  if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1)) != 0) return DARTREE_ERR_UNSUPPORTED;
  if (int64_t(p->max_pages) * p->page > (int64_t(1) << 30)) return DARTREE_ERR_UNSUPPORTED;
  return DARTREE_OK;
}

dartree_status check_memory(const dartree_cache_params& p, const dartree_cache* c) {
  if (!c || !given(c->k) || !given(c->v) || !given(c->table)) return DARTREE_ERR_INVALID_ARG;
  if (p.type == DARTREE_CACHE_E4M3 && (!given(c->k_exp) || !given(c->v_exp))) return DARTREE_ERR_INVALID_ARG;
  return DARTREE_OK;
}

CacheView view_of(const dartree_cache_params& p, const dartree_cache& c) {
  int log2 = 0;
  while ((1 << log2) < p.page) ++log2;
  return CacheView{p.batch, p.heads_kv, log2, p.num_pages, p.max_pages, c.k, c.v, c.k_exp, c.v_exp, c.table};
}

// A launch holds fewer than 2^32 threads: rows of 16 lanes here.
dartree_status check_rows(const dartree_cache_params& p, int32_t rows) {
  if (rows < 1) return DARTREE_ERR_INVALID_ARG;
  if (double(p.batch) * rows * p.heads_kv > double(1 << 27)) return DARTREE_ERR_UNSUPPORTED;
  return DARTREE_OK;
}

bool stride_ok(int64_t stride, int64_t least) { return stride >= least && stride % 8 == 0 && stride <= (int64_t(1) << 40); }

dartree_status check_paged(const dartree_attn_params* a, const dartree_cache_params* p) {
  dartree_status v = check_cache(p);
  if (v != DARTREE_OK) return v;
  if (!a) return DARTREE_ERR_INVALID_ARG;
  if (a->batch < 1 || a->budget < 1 || a->max_ctx < 0 || a->heads_q < 1 || a->heads_kv < 1 || a->head_dim < 1)
    return DARTREE_ERR_INVALID_ARG;
  if (a->batch != p->batch || a->heads_kv != p->heads_kv || a->head_dim != p->head_dim) return DARTREE_ERR_INVALID_ARG;
  if (a->heads_q % a->heads_kv != 0 || !(a->scale > 0.f) || !isnormal(a->scale * 1.4426950408889634f))
    return DARTREE_ERR_INVALID_ARG;
  if (a->max_ctx > int64_t(p->max_pages) * p->page) return DARTREE_ERR_INVALID_ARG;
  if (a->budget > DARTREE_MAX_SORT) return DARTREE_ERR_UNSUPPORTED;
  // items and steps are counted in 31 bits: query rows, and key steps of 128 over all requests
  if (int64_t(a->batch) * a->budget * a->heads_q > (int64_t(1) << 30)) return DARTREE_ERR_UNSUPPORTED;
  // and a launch holds fewer than 2^32 threads: at most 512 for 16 query rows
  if (double(a->batch) * a->heads_kv * ((int64_t(a->budget) * (a->heads_q / a->heads_kv) + 15) / 16) > double(1 << 22))
    return DARTREE_ERR_UNSUPPORTED;
  if (int64_t(a->batch) * (a->max_ctx / 128 + a->budget / 128 + 2) > (int64_t(1) << 30)) return DARTREE_ERR_UNSUPPORTED;
  return DARTREE_OK;
}

dartree_status check_verify(int32_t batch, int32_t budget, int32_t rows, int32_t vocab, int32_t type, float t) {
  if (batch < 1 || budget < 1 || vocab < 1) return DARTREE_ERR_INVALID_ARG;
  if (type != DARTREE_FP32 && type != DARTREE_BF16) return DARTREE_ERR_INVALID_ARG;
  if (!isfinite(t) || t < 0.f) return DARTREE_ERR_INVALID_ARG;
  if (vocab > DARTREE_MAX_VOCAB) return DARTREE_ERR_UNSUPPORTED;
  // a launch holds fewer than 2^32 threads: 256 for every segment of a request's rows
  if (double(batch) * rows * (vocab / 4096 + 2) > double((1 << 24) - 1) || batch > 65535) return DARTREE_ERR_UNSUPPORTED;
  return DARTREE_OK;
}
dartree_status check_tree(int32_t batch, int32_t budget, int32_t max_len, int32_t vocab, int32_t type, float t) {
  if (max_len < 1) return DARTREE_ERR_INVALID_ARG;
  if (budget > DARTREE_MAX_SORT || max_len > (1 << 20)) return DARTREE_ERR_UNSUPPORTED;
  return check_verify(batch, budget, budget + 1, vocab, type, t);
}
dartree_status check_chain(int32_t batch, int32_t depth, int32_t vocab, int32_t type, float t) {
  if (depth > DARTREE_MAX_DEPTH) return DARTREE_ERR_UNSUPPORTED;
  return check_verify(batch, depth, 2 * depth + 1, vocab, type, t);
}

}  // namespace

extern "C" {

dartree_status dartree_cache_validate(const dartree_cache_params* p) { return check_cache(p); }

dartree_status dartree_cache_write(const dartree_cache_params* p, const dartree_cache* cache, int32_t source_rows,
                                   int32_t rows, const void* k, const void* v, int64_t row_stride,
                                   const int32_t* index, const int32_t* counts, const int32_t* start,
                                   hipStream_t stream) {
  dartree_status s = check_cache(p);
  if (s != DARTREE_OK) return s;
  if ((s = check_memory(*p, cache)) != DARTREE_OK) return s;
  if ((s = check_rows(*p, rows)) != DARTREE_OK) return s;
  if (source_rows < 1 || (!index && source_rows < rows)) return DARTREE_ERR_INVALID_ARG;
  if (!given(k) || !given(v) || !optional(index) || !optional(counts) || !optional(start)) return DARTREE_ERR_INVALID_ARG;
  if (!stride_ok(row_stride, int64_t(p->heads_kv) * kHead)) return DARTREE_ERR_INVALID_ARG;
  CacheMoveArgs a{};
  a.c = view_of(*p, *cache);
  a.eight = p->type == DARTREE_CACHE_E4M3;
  a.source_rows = source_rows;
  a.rows = rows;
  a.k_in = static_cast<const uint16_t*>(k);
  a.v_in = static_cast<const uint16_t*>(v);
  a.row_stride = row_stride;
  a.index = index;
  a.counts = counts;
  a.start = start;
  return hip_status(launch_cache_write(a, stream));
}

dartree_status dartree_cache_read(const dartree_cache_params* p, const dartree_cache* cache, int32_t rows, void* k,
                                  void* v, const int32_t* counts, const int32_t* start, hipStream_t stream) {
  dartree_status s = check_cache(p);
  if (s != DARTREE_OK) return s;
  if ((s = check_memory(*p, cache)) != DARTREE_OK) return s;
  if ((s = check_rows(*p, rows)) != DARTREE_OK) return s;
  if (!given(k) || !given(v) || !optional(counts) || !optional(start)) return DARTREE_ERR_INVALID_ARG;
  CacheMoveArgs a{};
  a.c = view_of(*p, *cache);
  a.eight = p->type == DARTREE_CACHE_E4M3;
  a.rows = rows;
  a.k_out = static_cast<uint16_t*>(k);
  a.v_out = static_cast<uint16_t*>(v);
  a.counts = counts;
  a.start = start;
  return hip_status(launch_cache_read(a, stream));
}

dartree_status dartree_tree_attention_paged_workspace_size(const dartree_attn_params* a, const dartree_cache_params* p,
                                                           size_t* bytes) {
  if (!bytes) return DARTREE_ERR_INVALID_ARG;
  const dartree_status s = check_paged(a, p);
  if (s != DARTREE_OK) return s;
  *bytes = paged_attention_workspace(a->batch, a->budget, a->max_ctx, a->heads_q, a->heads_kv, p->type == DARTREE_CACHE_E4M3);
  return DARTREE_OK;
}

dartree_status dartree_tree_attention_paged(const dartree_attn_params* a, const dartree_cache_params* p,
                                            const dartree_cache* cache, const void* q, int64_t q_stride,
                                            const void* k_tree, const void* v_tree, int64_t kv_stride,
                                            const uint64_t* mask, const int32_t* num_nodes, const int32_t* ctx_len,
                                            void* out, void* ws, size_t ws_bytes, hipStream_t stream) {
  dartree_status s = check_paged(a, p);
  if (s != DARTREE_OK) return s;
  if ((s = check_memory(*p, cache)) != DARTREE_OK) return s;
  if (!given(q) || !given(k_tree) || !given(v_tree) || !given(out) || !optional(mask) || !optional(num_nodes) ||
      !optional(ctx_len))
    return DARTREE_ERR_INVALID_ARG;
  if (!stride_ok(q_stride, int64_t(a->heads_q) * kHead) || !stride_ok(kv_stride, int64_t(a->heads_kv) * kHead))
    return DARTREE_ERR_INVALID_ARG;
  const int eight = p->type == DARTREE_CACHE_E4M3;
  if (!workspace_fits(ws, ws_bytes,
                      paged_attention_workspace(a->batch, a->budget, a->max_ctx, a->heads_q, a->heads_kv, eight)))
    return DARTREE_ERR_WORKSPACE;
  PagedArgs g{};
  g.c = view_of(*p, *cache);
  g.eight = eight;
  g.batch = a->batch;
  g.budget = a->budget;
  g.max_ctx = a->max_ctx;
  g.heads_q = a->heads_q;
  g.heads_kv = a->heads_kv;
  g.group = a->heads_q / a->heads_kv;
  g.scale_log2 = a->scale * 1.4426950408889634f;
  g.q = static_cast<const uint16_t*>(q);
  g.k_tree = static_cast<const uint16_t*>(k_tree);
  g.v_tree = static_cast<const uint16_t*>(v_tree);
  g.q_stride = q_stride;
  g.kv_stride = kv_stride;
  g.mask = mask;
  g.num_nodes = num_nodes;
  g.ctx_len = ctx_len;
  g.out = static_cast<uint16_t*>(out);
  g.ws = ws;
  return hip_status(launch_paged_attention(g, stream));
}

dartree_status dartree_verify_tree_workspace_size(int32_t batch, int32_t budget, int32_t max_len, int32_t vocab,
                                                  size_t* bytes) {
  if (!bytes) return DARTREE_ERR_INVALID_ARG;
  const dartree_status s = check_tree(batch, budget, max_len, vocab, DARTREE_FP32, 1.f);
  if (s != DARTREE_OK) return s;
  *bytes = verify_tree_workspace(batch, budget, max_len, vocab);
  return DARTREE_OK;
}

dartree_status dartree_verify_chain_workspace_size(int32_t batch, int32_t depth, int32_t vocab, size_t* bytes) {
  if (!bytes) return DARTREE_ERR_INVALID_ARG;
  const dartree_status s = check_chain(batch, depth, vocab, DARTREE_FP32, 1.f);
  if (s != DARTREE_OK) return s;
  *bytes = verify_chain_workspace(batch, depth, vocab);
  return DARTREE_OK;
}

dartree_status dartree_verify_tree(int32_t batch, int32_t budget, int32_t max_len, int32_t vocab, int32_t logits_type,
                                   const int32_t* tokens, const int32_t* parents, const int32_t* num_nodes,
                                   const void* target_logits, int64_t row_stride, float temperature,
                                   const float* uniforms, int32_t* accepted, int32_t* num_accepted, int32_t* bonus,
                                   void* ws, size_t ws_bytes, hipStream_t stream) {
  dartree_status s = check_tree(batch, budget, max_len, vocab, logits_type, temperature);
  if (s != DARTREE_OK) return s;
  if (!given(tokens) || !given(parents) || !given(num_nodes) || !given(target_logits) || !given(uniforms) ||
      !given(accepted) || !given(num_accepted) || !given(bonus))
    return DARTREE_ERR_INVALID_ARG;
  if (row_stride < vocab || row_stride > (int64_t(1) << 40)) return DARTREE_ERR_INVALID_ARG;
  if (!workspace_fits(ws, ws_bytes, verify_tree_workspace(batch, budget, max_len, vocab))) return DARTREE_ERR_WORKSPACE;
  VerifyArgs a{};
  a.batch = batch;
  a.budget = budget;
  a.max_len = max_len;
  a.vocab = vocab;
  a.bf16 = logits_type == DARTREE_BF16;
  a.tokens = tokens;
  a.parents = parents;
  a.num_nodes = num_nodes;
  a.target = target_logits;
  a.row_stride = row_stride;
  a.inv_t = temperature > 0.f ? 1.0 / double(temperature) : 0.0;
  a.uniforms = uniforms;
  a.accepted = accepted;
  a.num_accepted = num_accepted;
  a.bonus = bonus;
  a.ws = ws;
  return hip_status(launch_verify_tree(a, stream));
}

dartree_status dartree_verify_chain(int32_t batch, int32_t depth, int32_t vocab, int32_t logits_type,
                                    const int32_t* tokens, const int32_t* num_tokens, const void* target_logits,
                                    const void* draft_logits, int64_t row_stride, float temperature,
                                    const float* uniforms, int32_t* num_accepted, int32_t* bonus, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
  dartree_status s = check_chain(batch, depth, vocab, logits_type, temperature);
  if (s != DARTREE_OK) return s;
  if (!given(tokens) || !optional(num_tokens) || !given(target_logits) || !given(uniforms) || !given(num_accepted) ||
      !given(bonus) || !(temperature > 0.f ? given(draft_logits) : optional(draft_logits)))
    return DARTREE_ERR_INVALID_ARG;
  if (row_stride < vocab || row_stride > (int64_t(1) << 40)) return DARTREE_ERR_INVALID_ARG;
  if (!workspace_fits(ws, ws_bytes, verify_chain_workspace(batch, depth, vocab))) return DARTREE_ERR_WORKSPACE;
  VerifyArgs a{};
  a.batch = batch;
  a.budget = depth;
  a.vocab = vocab;
  a.bf16 = logits_type == DARTREE_BF16;
  a.tokens = tokens;
  a.num_nodes = num_tokens;
  a.target = target_logits;
  a.draft = draft_logits;
  a.row_stride = row_stride;
  a.inv_t = temperature > 0.f ? 1.0 / double(temperature) : 0.0;
  a.uniforms = uniforms;
  a.num_accepted = num_accepted;
  a.bonus = bonus;
  a.ws = ws;
  return hip_status(launch_verify_chain(a, stream));
}

}  // extern "C"
