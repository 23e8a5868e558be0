/*
 * libdartree, rotary positions of queries and keys: pairs of elements turned by an
 * angle that grows with the position, so that a product of a query and a key
 * depends on their distance.  Conventions (stream, errors, alignment, validation
 * before anything is enqueued) are those of dartree.h; the device call allocates
 * nothing and can be captured into a graph.
 *
 * In a step of a serving loop (dartree/serve.h) it stands between the target's
 * projections and the attention: the rows of a prompt before dartree_cache_write,
 * those of a drafted tree, at their depths, before dartree_tree_attention_paged
 * (the accepted nodes' keys are written to the cache as they are then).
 */
#ifndef DARTREE_ROTARY_H
#define DARTREE_ROTARY_H

#include "dartree.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dartree_rotary_layout {
  DARTREE_ROTARY_HALF = 0,       /* pair i: elements i and i + rotary_dim / 2 */
  DARTREE_ROTARY_INTERLEAVED = 1 /* pair i: elements 2 i and 2 i + 1 */
} dartree_rotary_layout;

/* How the frequencies f_i = base^(-2 i / rotary_dim), in radians a position, are
 * changed for contexts longer than the trained ones. */
typedef enum dartree_rotary_rule {
  DARTREE_ROTARY_PLAIN = 0,  /* not at all */
  DARTREE_ROTARY_LINEAR = 1, /* f_i / factor: positions are compressed */
  DARTREE_ROTARY_BASE = 2,   /* base becomes base * factor^(r / (r - 2)), r = rotary_dim: the slowest pair is compressed
                                by factor, the fastest not at all (r = 2: as PLAIN) */
  DARTREE_ROTARY_TURNS = 3   /* by the turns n_i = length f_i / (2 pi) of a pair over the trained length: pairs with n_i
                                >= high stay, those with n_i <= low are compressed by factor, between them
                                f_i (s + (1 - s) / factor), s = (n_i - low) / (high - low) */
} dartree_rotary_rule;

/* Host struct; members that a rule does not name are not read. */
typedef struct dartree_rotary_scaling {
  int32_t rule;     /* dartree_rotary_rule */
  double factor;    /* > 0 */
  double low, high; /* low < high */
  int32_t length;   /* >= 1 */
} dartree_rotary_scaling;

/* The table of frequencies that dartree_rotary reads, for rotary_dim / 2 pairs
 * (host only, `turns` is host memory): turns[i] is the fraction of a turn that
 * pair i makes from one position to the next, in units of 2^-64.  A position's
 * angle is their product modulo one turn, exact in 64-bit integers.  A pair of f
 * radians a position is within two units where f <= 1, so that its angle at position
 * 2^20 is good to 2^-43 of a turn, and within about 2 f units where it is faster
 * (frequencies are formed in 64 bits of mantissa).  scaling NULL: PLAIN.
 * rotary_dim: even, 2 .. 512; base > 0, finite. */
dartree_status dartree_rotary_turns(int32_t rotary_dim, double base, const dartree_rotary_scaling* scaling,
                                    uint64_t* turns);

/* The same table of any `pairs` finite frequencies, in radians a position (host only),
 * within one unit each (up to 2^60 radians).  For rules that are not among those above,
 * such as a ramp over the pairs' numbers i between two bounds in the place of TURNS'
 * over their turns n_i, which gives other angles: a model's own rule decides. */
dartree_status dartree_rotary_turns_of(int32_t pairs, const double* radians, uint64_t* turns);

typedef struct dartree_rotary_params {
  int32_t batch, rows;       /* b requests of `rows` rows, >= 1 */
  int32_t heads_q, heads_kv; /* heads of a row of q and of k; one of them may be 0 (then its pointers are not used) */
  int32_t head_dim;          /* a multiple of 8, 8 .. 512 */
  int32_t rotary_dim;        /* even, 2 .. head_dim: the first elements of a head; the others are copied */
  int32_t layout;            /* dartree_rotary_layout */
  int32_t type;              /* DARTREE_BF16 or DARTREE_FP32 */
  int32_t inverse;           /* 1: turned back.  The gradient of a call with 0 (and of its inverse with 1, both times
                                amplitude), and a key's move from one position to another */
  int32_t first;             /* added to every position */
  float amplitude;           /* of the turned elements, finite (1, or what a rule for long contexts asks for) */
} dartree_rotary_params;

/* Row i < counts[r] (NULL: rows; values above rows count as rows) of request r is
 * turned by the angles of position first + start[r] (NULL: 0) + positions[r][i]
 * (NULL: i): (x, y) of a pair becomes amplitude (x cos - y sin, y cos + x sin).
 * A drafted tree's rows take its depths (1 ..) as positions, the context's length
 * as start and first = -1.  turns: device, from the calls above.  Rows at and past
 * counts[r] are left as they were in the outputs.
 * q: row i of request r at (r * rows + i) * q_stride elements, heads_q * head_dim
 * elements each; k, q_out and k_out likewise with strides of their own, multiples of
 * 8.  q_out may be q with the same stride (elements past rotary_dim are not touched
 * then), k_out likewise k; otherwise an output's rows overlap neither q's nor k's rows
 * nor the other output's, which is checked (rows side by side in one tensor do not
 * overlap), nor anything else that the call reads.
 * Angles in 64-bit integers, sines and cosines to 2^-23, products in fp32; bf16
 * outputs are rounded once.  batch * rows < 2^24. */
dartree_status dartree_rotary(const dartree_rotary_params* p, const uint64_t* turns, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out,
                              int64_t k_out_stride, const int32_t* positions, const int32_t* start,
                              const int32_t* counts, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DARTREE_ROTARY_H */
