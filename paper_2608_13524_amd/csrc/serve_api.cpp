// C ABI of the serving operators (dartree/serve.h, pages.h, rotary.h): argument
// checks, then one launcher each.  Nothing here touches the device before every check passed.
#include <math.h>

#include "pages.hpp"
#include "rotary.hpp"
#include "serve.hpp"

using namespace dartree;

namespace {

bool given(const void* p) { return p && aligned16(p); }
bool optional(const void* p) { return !p || aligned16(p); }

dartree_status check_cache(const dartree_cache_params* p) {
  if (!p) return DARTREE_ERR_INVALID_ARG;
  if (p->batch < 1 || p->heads_kv < 1 || p->head_dim < 1 || p->page < 1 || p->num_pages < 1 || p->max_pages < 1)
    return DARTREE_ERR_INVALID_ARG;
  if (p->type != DARTREE_CACHE_BF16 && p->type != DARTREE_CACHE_E4M3 && p->type != DARTREE_CACHE_E2M1)
    return DARTREE_ERR_INVALID_ARG;
  if (p->head_dim != kHead || p->heads_kv > 4096) return DARTREE_ERR_UNSUPPORTED;
  if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1)) != 0) return DARTREE_ERR_UNSUPPORTED;
  if (int64_t(p->max_pages) * p->page > (int64_t(1) << 30)) return DARTREE_ERR_UNSUPPORTED;
  return DARTREE_OK;
}

dartree_status check_memory(const dartree_cache_params& p, const dartree_cache* c) {
  if (!c || !given(c->k) || !given(c->v) || !given(c->table)) return DARTREE_ERR_INVALID_ARG;
  if (p.type != DARTREE_CACHE_BF16 && (!given(c->k_exp) || !given(c->v_exp))) return DARTREE_ERR_INVALID_ARG;
  return DARTREE_OK;
}

int bits_of(const dartree_cache_params& p) {
  return p.type == DARTREE_CACHE_BF16 ? 16 : p.type == DARTREE_CACHE_E4M3 ? 8 : 4;
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

dartree_status check_table(const dartree_cache_params* p) {
  const dartree_status s = check_cache(p);
  if (s != DARTREE_OK) return s;
  return int64_t(p->batch) * p->max_pages > (int64_t(1) << 30) ? DARTREE_ERR_UNSUPPORTED : DARTREE_OK;
}

bool apart(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x + a_bytes <= y || y + b_bytes <= x;
}

// A table and what becomes of it: the same memory (where that may be) or none in common.
bool tables_ok(const dartree_cache_params& p, const int32_t* table, const int32_t* out, bool same) {
  const int64_t bytes = int64_t(p.batch) * p.max_pages * 4;
  return given(table) && given(out) && ((same && table == out) || apart(table, bytes, out, bytes));
}

PagesArgs pages_of(const dartree_cache_params& p, const int32_t* table, int32_t* out) {
  PagesArgs a{};
  a.batch = p.batch;
  while ((1 << a.page_log2) < p.page) ++a.page_log2;
  a.num_pages = p.num_pages;
  a.max_pages = p.max_pages;
  a.table = table;
  a.out = out;
  return a;
}

dartree_status check_rotary(const dartree_rotary_params* p) {
  if (!p) return DARTREE_ERR_INVALID_ARG;
  if (p->batch < 1 || p->rows < 1 || p->heads_q < 0 || p->heads_kv < 0 || p->heads_q + int64_t(p->heads_kv) < 1)
    return DARTREE_ERR_INVALID_ARG;
  if (p->head_dim < 1 || p->rotary_dim < 2 || p->rotary_dim % 2 != 0 || p->rotary_dim > p->head_dim)
    return DARTREE_ERR_INVALID_ARG;
  if (p->layout != DARTREE_ROTARY_HALF && p->layout != DARTREE_ROTARY_INTERLEAVED) return DARTREE_ERR_INVALID_ARG;
  if (p->type != DARTREE_FP32 && p->type != DARTREE_BF16) return DARTREE_ERR_INVALID_ARG;
  if (p->inverse != 0 && p->inverse != 1) return DARTREE_ERR_INVALID_ARG;
  if (!isfinite(p->amplitude)) return DARTREE_ERR_INVALID_ARG;
  if (p->head_dim % 8 != 0 || p->head_dim > 512 || p->heads_q > 2048 || p->heads_kv > 2048) return DARTREE_ERR_UNSUPPORTED;
  // a launch holds fewer than 2^32 threads: 256 for a row
  return double(p->batch) * p->rows > double(1 << 24) - 1 ? DARTREE_ERR_UNSUPPORTED : DARTREE_OK;
}

// Rows of one of rotary's tensors and of its output.
bool rotary_rows_ok(const dartree_rotary_params& p, int heads, const void* x, int64_t stride, const void* out,
                    int64_t out_stride) {
  if (heads == 0) return true;
  const int64_t row = int64_t(heads) * p.head_dim;
  return given(x) && given(out) && stride_ok(stride, row) && stride_ok(out_stride, row) && (x != out || stride == out_stride);
}

// `count` rows of `bytes`, `step` bytes apart.
struct RowSet {
  uintptr_t at;
  int64_t bytes, step, count;
};
// No byte in common: the sets follow each other, or each lies beside the other's rows, as parts of the
// rows of one tensor do (exact for one step; for two, of all rows that lie so).
bool rows_apart(const RowSet& x, const RowSet& y) {
  const auto end = [](const RowSet& r) { return __int128(r.at) + __int128(r.count - 1) * r.step + r.bytes; };
  if (end(x) <= __int128(y.at) || end(y) <= __int128(x.at)) return true;
  if (x.count == 1) return false;
  int64_t gap = x.step, r = y.step;   // their greatest common divisor
  while (r != 0) {
    const int64_t t = gap % r;
    gap = r;
    r = t;
  }
  const int64_t d = int64_t((__int128(y.at) - __int128(x.at)) % gap), beside = d < 0 ? d + gap : d;
  return beside >= x.bytes && beside + y.bytes <= gap;
}

// The outputs are their inputs, or apart from both inputs, and from each other.
bool rotary_apart(const dartree_rotary_params& p, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                  const void* q_out, int64_t q_out_stride, const void* k_out, int64_t k_out_stride) {
  const int64_t size = p.type == DARTREE_BF16 ? 2 : 4, count = int64_t(p.batch) * p.rows;
  const auto rows = [&](const void* at, int heads, int64_t stride) {
    return RowSet{reinterpret_cast<uintptr_t>(at), heads * int64_t(p.head_dim) * size, stride * size, count};
  };
  const RowSet qi = rows(q, p.heads_q, q_stride), qo = rows(q_out, p.heads_q, q_out_stride);
  const RowSet ki = rows(k, p.heads_kv, k_stride), ko = rows(k_out, p.heads_kv, k_out_stride);
  if (p.heads_q > 0 && q != q_out && !rows_apart(qi, qo)) return false;
  if (p.heads_kv > 0 && k != k_out && !rows_apart(ki, ko)) return false;
  return p.heads_q == 0 || p.heads_kv == 0 || (rows_apart(qo, ki) && rows_apart(qo, ko) && rows_apart(qi, ko));
}

// The fraction of a turn in `radians`, in units of 2^-64.  1 / (2 pi) in two numbers of 64 bits of
// mantissa (x87), so that the whole turns of fast pairs take no bits from it: within a unit up to 2^60.
uint64_t turn_of(long double radians) {
  const long double high = 0.159154943091895335769L, low = -2.03622285290738401775e-22L;
  const long double p = radians * high, rest = fmal(radians, high, -p) + radians * low;
  long double t = fmodl(fmodl(p, 1.0L) + rest, 1.0L);
  if (t < 0) t += 1.0L;
  const long double u = rintl(t * 18446744073709551616.0L);
  return u >= 18446744073709551616.0L ? 0 : uint64_t(u);
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
  a.bits = bits_of(*p);
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
  a.bits = bits_of(*p);
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
  *bytes = paged_attention_workspace(a->batch, a->budget, a->max_ctx, a->heads_q, a->heads_kv, bits_of(*p));
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
  const int bits = bits_of(*p);
  if (!workspace_fits(ws, ws_bytes,
                      paged_attention_workspace(a->batch, a->budget, a->max_ctx, a->heads_q, a->heads_kv, bits)))
    return DARTREE_ERR_WORKSPACE;
  PagedArgs g{};
  g.c = view_of(*p, *cache);
  g.bits = bits;
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

dartree_status dartree_pages_workspace_size(const dartree_cache_params* p, size_t* bytes) {
  if (!bytes) return DARTREE_ERR_INVALID_ARG;
  const dartree_status s = check_table(p);
  if (s != DARTREE_OK) return s;
  *bytes = pages_workspace(p->batch, p->num_pages);
  return DARTREE_OK;
}

dartree_status dartree_pages_fork(const dartree_cache_params* p, const int32_t* table, int32_t* out,
                                  const int32_t* source, const int32_t* keep, hipStream_t stream) {
  const dartree_status s = check_table(p);
  if (s != DARTREE_OK) return s;
  if (!tables_ok(*p, table, out, !source) || !optional(source) || !optional(keep)) return DARTREE_ERR_INVALID_ARG;
  PagesArgs a = pages_of(*p, table, out);
  a.source = source;
  a.keep = keep;
  return hip_status(launch_pages_fork(a, stream));
}

dartree_status dartree_pages_reserve(const dartree_cache_params* p, const int32_t* table, int32_t* out, int32_t rows,
                                     const int32_t* start, const int32_t* counts, int32_t* pairs, int32_t max_pairs,
                                     int32_t* totals, int32_t* granted, void* ws, size_t ws_bytes, hipStream_t stream) {
  const dartree_status s = check_table(p);
  if (s != DARTREE_OK) return s;
  if (rows < 1) return DARTREE_ERR_INVALID_ARG;
  if (!tables_ok(*p, table, out, true) || !optional(start) || !optional(counts) || !given(pairs) || !given(totals) ||
      !given(granted))
    return DARTREE_ERR_INVALID_ARG;
  const int64_t columns = (int64_t(rows) + p->page - 2) / p->page + 1;
  PagesArgs a = pages_of(*p, table, out);
  a.columns = int(columns < p->max_pages ? columns : p->max_pages);
  if (max_pairs < int64_t(p->batch) * a.columns) return DARTREE_ERR_INVALID_ARG;
  if (!workspace_fits(ws, ws_bytes, pages_workspace(p->batch, p->num_pages))) return DARTREE_ERR_WORKSPACE;
  a.rows = rows;
  a.start = start;
  a.counts = counts;
  a.pairs = pairs;
  a.totals = totals;
  a.granted = granted;
  a.ws = ws;
  return hip_status(launch_pages_reserve(a, stream));
}

dartree_status dartree_pages_compact(const dartree_cache_params* p, const int32_t* table, int32_t* out, int32_t* pairs,
                                     int32_t max_pairs, int32_t* totals, void* ws, size_t ws_bytes, hipStream_t stream) {
  const dartree_status s = check_table(p);
  if (s != DARTREE_OK) return s;
  if (!tables_ok(*p, table, out, true) || !optional(pairs) || (!pairs && p->num_pages > 1) || !given(totals) ||
      max_pairs < p->num_pages / 2)
    return DARTREE_ERR_INVALID_ARG;
  if (!workspace_fits(ws, ws_bytes, pages_workspace(p->batch, p->num_pages))) return DARTREE_ERR_WORKSPACE;
  PagesArgs a = pages_of(*p, table, out);
  a.pairs = pairs;
  a.totals = totals;
  a.ws = ws;
  return hip_status(launch_pages_compact(a, stream));
}

dartree_status dartree_cache_copy(const dartree_cache_params* p, const dartree_cache* cache, const int32_t* pairs,
                                  int32_t max_pairs, const int32_t* count, hipStream_t stream) {
  const dartree_status s = check_cache(p);
  if (s != DARTREE_OK) return s;
  if (!cache || !given(cache->k) || !given(cache->v) || !given(pairs) || !given(count) || max_pairs < 1)
    return DARTREE_ERR_INVALID_ARG;
  const int bits = bits_of(*p);
  if (bits != 16 && (!given(cache->k_exp) || !given(cache->v_exp))) return DARTREE_ERR_INVALID_ARG;
  const int64_t rows = int64_t(p->heads_kv) * p->page;
  PageCopyArgs a{};
  a.num_pages = p->num_pages;
  a.row_bytes = rows * kHead * bits / 8;
  a.exp_bytes = bits == 16 ? 0 : bits == 8 ? rows : rows * (kHead / kBlock);
  a.k = cache->k;
  a.v = cache->v;
  a.k_exp = cache->k_exp;
  a.v_exp = cache->v_exp;
  a.pairs = pairs;
  a.max_pairs = max_pairs;
  a.count = count;
  return hip_status(launch_cache_copy(a, stream));
}

dartree_status dartree_rotary_turns(int32_t rotary_dim, double base, const dartree_rotary_scaling* scaling,
                                    uint64_t* turns) {
  if (!turns || rotary_dim < 2 || rotary_dim % 2 != 0 || !isfinite(base) || !(base > 0)) return DARTREE_ERR_INVALID_ARG;
  if (rotary_dim > 512) return DARTREE_ERR_UNSUPPORTED;
  const int rule = scaling ? scaling->rule : DARTREE_ROTARY_PLAIN;
  if (rule < DARTREE_ROTARY_PLAIN || rule > DARTREE_ROTARY_TURNS) return DARTREE_ERR_INVALID_ARG;
  const long double factor = rule == DARTREE_ROTARY_PLAIN ? 1.0L : (long double)scaling->factor;
  if (rule != DARTREE_ROTARY_PLAIN && (!isfinite(scaling->factor) || !(scaling->factor > 0))) return DARTREE_ERR_INVALID_ARG;
  if (rule == DARTREE_ROTARY_TURNS && (!isfinite(scaling->low) || !isfinite(scaling->high) || !(scaling->low < scaling->high) ||
                                       scaling->length < 1))
    return DARTREE_ERR_INVALID_ARG;
  const long double r = rotary_dim, pi = 3.14159265358979323846264338327950288L;
  long double b = base;
  if (rule == DARTREE_ROTARY_BASE && rotary_dim > 2) b *= powl(factor, r / (r - 2));
  for (int i = 0; i < rotary_dim / 2; ++i) {
    long double f = powl(b, -2 * i / r);
    if (rule == DARTREE_ROTARY_LINEAR) f /= factor;
    if (rule == DARTREE_ROTARY_TURNS) {
      long double s = (scaling->length * f / (2 * pi) - scaling->low) / ((long double)scaling->high - scaling->low);
      s = s < 0 ? 0 : s > 1 ? 1 : s;
      f *= s + (1 - s) / factor;
    }
    turns[i] = turn_of(f);
  }
  return DARTREE_OK;
}

dartree_status dartree_rotary_turns_of(int32_t pairs, const double* radians, uint64_t* turns) {
  if (pairs < 1 || !radians || !turns) return DARTREE_ERR_INVALID_ARG;
  for (int i = 0; i < pairs; ++i)
    if (!isfinite(radians[i])) return DARTREE_ERR_INVALID_ARG;
  for (int i = 0; i < pairs; ++i) turns[i] = turn_of(radians[i]);
  return DARTREE_OK;
}

dartree_status dartree_rotary(const dartree_rotary_params* p, const uint64_t* turns, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out,
                              int64_t k_out_stride, const int32_t* positions, const int32_t* start,
                              const int32_t* counts, hipStream_t stream) {
  const dartree_status s = check_rotary(p);
  if (s != DARTREE_OK) return s;
  if (!given(turns) || !optional(positions) || !optional(start) || !optional(counts)) return DARTREE_ERR_INVALID_ARG;
  if (!rotary_rows_ok(*p, p->heads_q, q, q_stride, q_out, q_out_stride) ||
      !rotary_rows_ok(*p, p->heads_kv, k, k_stride, k_out, k_out_stride))
    return DARTREE_ERR_INVALID_ARG;
  if (!rotary_apart(*p, q, q_stride, k, k_stride, q_out, q_out_stride, k_out, k_out_stride)) return DARTREE_ERR_INVALID_ARG;
  RotaryArgs a{};
  a.batch = p->batch;
  a.rows = p->rows;
  a.heads_q = p->heads_q;
  a.heads_kv = p->heads_kv;
  a.head_dim = p->head_dim;
  a.rotary_dim = p->rotary_dim;
  a.layout = p->layout;
  a.bf16 = p->type == DARTREE_BF16;
  a.inverse = p->inverse;
  a.first = p->first;
  a.amplitude = p->amplitude;
  a.turns = turns;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.positions = positions;
  a.start = start;
  a.counts = counts;
  return hip_status(launch_rotary(a, stream));
}

}  // extern "C"
