/*
 * libdartree, the pages of a paged cache (dartree/serve.h): taken for positions to
 * come, shared between requests, copied where a shared one is written, moved
 * together and given back, on the device.  Conventions (stream, errors, alignment,
 * validation before anything is enqueued) are those of dartree.h; the calls
 * allocate nothing and can be captured into a graph.
 *
 * The page table is the whole state: a page is in use while an entry of the table
 * names it, shared while more than one does, and free otherwise.  Nothing counts
 * references beside it, so nothing can disagree with it; a prefix that is to
 * outlive its requests is kept by a row of the table of its own.  One table can
 * serve the caches of all layers: the calls on it are made once, dartree_cache_copy
 * once for each layer.
 *
 * A step of a serving loop:
 *   dartree_pages_fork     ended requests give their pages back, others are continued
 *                          several times over, or dropped tokens' pages go
 *   dartree_pages_reserve  the next positions get pages of their own
 *   dartree_cache_copy     per layer: what they shared, copied
 *   dartree_cache_write    per layer
 *
 * Only batch, page, num_pages and max_pages of the cache's parameters matter to
 * the calls on the table; batch * max_pages <= 2^30.
 */
#ifndef DARTREE_PAGES_H
#define DARTREE_PAGES_H

#include "dartree/serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device workspace (256-byte aligned) for dartree_pages_reserve and
 * dartree_pages_compact (host only). */
dartree_status dartree_pages_workspace_size(const dartree_cache_params* p, size_t* bytes);

/* Row q of `out` ([b][max_pages]) becomes the entries of row source[q] of `table`
 * that hold its first keep[q] positions, -1 in the other columns.  source NULL: q
 * itself; a source outside [0, b): no entry.  keep NULL: all; negative: none.
 * Forks (source), trims and frees (keep).  out may be table where source is NULL;
 * otherwise the two do not overlap. */
dartree_status dartree_pages_fork(const dartree_cache_params* p, const int32_t* table, int32_t* out,
                                  const int32_t* source, const int32_t* keep, hipStream_t stream);

/* Pages for positions start[q] .. start[q] + counts[q] - 1 of every request (start
 * NULL: 0; counts NULL: rows, values above rows count as rows, negative ones as 0;
 * positions outside 0 .. max_pages * page - 1 are left out), so that they can be
 * written without another request seeing it.  `out` is `table` but for the columns
 * of these positions: an entry that names no page gets a free one, and so does one
 * whose page another entry names too; others stay.  Free pages are taken in
 * ascending order, by requests and columns in ascending order.  pairs
 * [max_pairs][2] lists, in that order, {page, the one in its place} of the shared
 * ones, but for those whose every position is to be written: what
 * dartree_cache_copy copies.  Entries of pairs past the last are left as they were.
 * granted[q] is 1 where request q has what it needs: it needs nothing, or the
 * needs of requests 0 .. q together do not exceed the free pages; else it is 0 and
 * the request's row stays as it is in `table`.
 * totals[0] = pairs listed, totals[1] = free pages left (pages that `table` does not
 * name, less those taken).
 * out may be table, or overlaps it nowhere.  1 <= rows; max_pairs at least
 * b * min(max_pages, (rows + page - 2) / page + 1). */
dartree_status dartree_pages_reserve(const dartree_cache_params* p, const int32_t* table, int32_t* out, int32_t rows,
                                     const int32_t* start, const int32_t* counts, int32_t* pairs, int32_t max_pairs,
                                     int32_t* totals, int32_t* granted, void* ws, size_t ws_bytes, hipStream_t stream);

/* The n pages in use move to pages 0 .. n - 1: those from n on, in ascending order,
 * to the free ones below n, in ascending order.  `out` is `table` with their new
 * places (an entry that names no page becomes -1), pairs lists {page, its new
 * place}, totals[0] = pairs listed, totals[1] = n.  Entries of pairs past the last
 * are left as they were.  out may be table, or overlaps it nowhere.  max_pairs at
 * least num_pages / 2. */
dartree_status dartree_pages_compact(const dartree_cache_params* p, const int32_t* table, int32_t* out, int32_t* pairs,
                                     int32_t max_pairs, int32_t* totals, void* ws, size_t ws_bytes, hipStream_t stream);

/* Copy pages (keys, values and exponents) of a cache: pairs[i][0] to pairs[i][1] for
 * i < count[0] (device memory, such as `totals`; at most max_pairs >= 1 are copied).
 * A pair with a page outside the pool is left out.  No page is copied to twice, nor
 * both from and to (lists of the calls above are like that).  cache->table is not
 * read and may be NULL. */
dartree_status dartree_cache_copy(const dartree_cache_params* p, const dartree_cache* cache, const int32_t* pairs,
                                  int32_t max_pairs, const int32_t* count, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DARTREE_PAGES_H */
