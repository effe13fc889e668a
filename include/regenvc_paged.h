/*
 * regenvc_paged.h -- C ABI of the gfx950 kernels of a bf16 key/value cache in
 * pages, for a process that streams many sequences: the append that norms and
 * rotates on the way, attention of new tokens to the places of their sequence,
 * and attention to only those pages that a cheap score selects.
 *
 * A pool of pages holds a fixed number of tokens each.  A sequence has places
 * 0, 1, ... (its tokens' positions); row b of a table names the pages of
 * sequence b in order.  The new tokens of all sequences stand packed in tensors
 * [T, heads, D]: those of sequence b in rows first[b] .. first[b + 1] - 1.
 * They are the last ones of its lens[b] places: with n of them, row first[b] + i
 * is the token of place lens[b] - n + i.
 *
 * Conventions are those of regenvc_attn.h (status codes, regenvc_last_error,
 * device pointers owned by the caller, validation before any launch, work
 * enqueued on `stream`, gfx950 only, bit-identical results run to run).  None
 * of these calls allocates; none writes anything but its outputs and workspace.
 */
#ifndef REGENVC_PAGED_H
#define REGENVC_PAGED_H

#include <stdint.h>

#include "regenvc_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A pool of `pages` pages of `page` places for `heads` key heads, in caller
   memory, contiguous, 16-byte aligned.  D in {64, 128}; page a power of two, 16
   to 1024; pages below 2^30; heads at most 65535; k and v of at most 2^47 bytes each. */
typedef struct {
    void *k, *v;  /* bf16 [pages, heads, page, D] */
    void *means;  /* bf16 [pages, heads, D]: each page's mean key; or NULL */
    int32_t pages, page, heads, D;
} regenvc_page_pool;

/* The sequences of a call; all three arrays int32 in device memory, 4-byte
   aligned.  B at most 2^20, T below 2^26, columns * page below 2^30.
     table: [B, columns], row stride table_stride elements.  Sequences may share
            pages that no call writes.  An entry outside [0, pages) is a page
            without places: nothing is read or written there.
     first: [B + 1], ascending, in [0, T].  Rows before first[0] and from first[B]
            on belong to no sequence: their outputs are left as they were.
     lens:  [B]; below 0 counts as 0.  Attention and selection hold it to columns *
            page; an append beyond that stores what the table has room for */
typedef struct {
    const int32_t *table, *first, *lens;
    int64_t table_stride;
    int32_t B, columns, T;
} regenvc_page_batch;

/* A rotation of the first 2 * pairs channels of a head, a multiple of 16, at
   most D.  Pair i of the token at place p is turned by p * turns[i] full turns
   (taken in 64 bits) and multiplied by `amplitude`:
     (a, b) -> amplitude (a cos - b sin, a sin + b cos)
   interleaved != 0: pair i is channels 2 i and 2 i + 1; else i and pairs + i.
     turns: double [pairs] in device memory, 8-byte aligned */
typedef struct {
    const double *turns;
    int32_t pairs, interleaved;
    float amplitude;
} regenvc_rotary;

/* New tokens to the cache.  For every token and head of q and k:
     y = x * w / sqrt(mean over D of x^2 + eps)   (w bf16 [D]; NULL: y = x)
     z = y rotated at the token's place           (rotary NULL: z = y)
   in fp32, rounded to bf16 once.  q's z goes to q_out, k's and the unchanged v to
   the token's place; a token whose place is negative, past the table or on a
   page outside the pool is not stored.  With pool->means, the mean key of every
   page that the new tokens touch is taken anew over its first places up to
   lens[b]: their sum in 64 bits over their number, rounded to bf16 as the keys are.
     q:     bf16 [T, H, D], or NULL with H = 0 (then q_out and w_q are NULL)
     k, v:  bf16 [T, heads, D];  q_out: bf16 [T, H, D], may be q itself
            (stride_b of these tensors is not looked at)
     w_q, w_k: bf16 [D], 16-byte aligned, or NULL
   The pages written must be neither shared by sequences of the call nor named twice
   by one. */
regenvc_status regenvc_paged_append(const regenvc_page_pool *pool, const regenvc_page_batch *batch,
                                    const regenvc_tensor *q, const regenvc_tensor *k, const regenvc_tensor *v,
                                    const void *w_q, const void *w_k, float eps, const regenvc_rotary *rotary,
                                    const regenvc_tensor *q_out, int32_t H, void *stream);

/* Attention of q (bf16 [T, H, D], H a multiple of the pool's heads; query head h
   reads key head h / (H / heads)) to the places of its sequence: causal != 0: to
   those up to the token's own; else to all lens[b].  Scores and sums are fp32; a
   softmax weight is rounded to bf16 before it multiplies a value, whatever
   o_dtype is; O is normalized by the sum of the rounded weights, LSE takes them
   unrounded.  What lies in places that a query does not see is of no account to
   it, infinities and NaN included (in the values of a causal call's own tokens they
   cost time: up to 256 queries before such a token are done again, key by key, 100
   times as long as the call or more).  A query that sees no place gives O = 0, LSE =
   -inf.
     o:   [T, H, D] in o_dtype; lse: f32 [H, T] or NULL
     selected: NULL, or int32 [T / q_block + B, heads, count] as from
          regenvc_paged_select: queries first[b] + i q_block .. + q_block - 1 of
          sequence b (block first[b] / q_block + b + i) see only the places of the
          pages that their block and key head names (indices into the
          sequence's row of the table; -1, and any other outside it: none).  A
          page named twice counts twice.
     max_rows, max_len: the most new tokens and places of a sequence that the
          work is planned for, 0 <= max_rows <= T, 0 <= max_len <= columns * page;
          longer ones are computed right, only less evenly
   H T is at most 2^29, q_block in [1, 2^20], count in [1, 16384].  A call of more
   workgroups (tiles, times key ranges) than one launch can have is refused: 2^23 -
   1 of tiles of 16 or 256 rows, 2^24 - 1 of 32 or 64.
   workspace: 256-byte aligned, at least regenvc_paged_attn_workspace bytes (NULL
   if that is 0). */
regenvc_status regenvc_paged_attn_fwd(const regenvc_tensor *q, const regenvc_page_pool *pool,
                                      const regenvc_page_batch *batch, const int32_t *selected, int32_t q_block,
                                      int32_t count, int32_t causal, int32_t max_rows, int32_t max_len,
                                      const regenvc_tensor *o, regenvc_dtype o_dtype, float *lse, int32_t H,
                                      float softmax_scale, void *workspace, int64_t workspace_bytes, void *stream);

/* The shape of such a call, for its plan.  selected: count, or 0 without; causal
   as in the call. */
typedef struct {
    int32_t B, T, H, heads, D, page, q_block, count, max_rows, max_len, causal;
} regenvc_paged_attn_shape;

/* Workspace bytes of such a call on n_cu compute units.  Host-only. */
regenvc_status regenvc_paged_attn_workspace(const regenvc_paged_attn_shape *shape, int32_t n_cu, int64_t *bytes);

/* Its decomposition: rows of a workgroup's tile (queries times the H / heads
   heads that share a key head), workgroups launched, and whether keys may be cut
   into ranges (the device decides by the sequences' lengths). */
typedef struct {
    int32_t tile_rows, workgroups, split;
} regenvc_paged_attn_plan;
regenvc_status regenvc_paged_attn_plan_query(const regenvc_paged_attn_shape *shape, int32_t n_cu,
                                             regenvc_paged_attn_plan *plan);

/* The pages that each block of q_block queries of a sequence reads, for every
   key head.  Candidates are the pages with a place that the block's last query
   sees (causal != 0: up to its own; else lens[b]).  The first keep_first of them
   and the last keep_last are taken; of the others those of the highest score
     sum over the block's queries and the key head's query heads of q, dot the
     page's mean key (pool->means)
   (64-bit sums; NaN counts as -inf; ties go to the lower page), until `count` are
   taken.  The last pages are counted from the block's last query: so that in a
   causal call every query keeps the page that it stands in, keep_last has to be
   (q_block - 1 + page - 1) / page + 1 (1 for single queries, 2 for blocks of up to
   page + 1).  With less, the earlier queries of a block see their own page only if its
   score wins (one that sees none of the block's pages gives O = 0), by a mean that
   holds keys of later tokens.
     selected: int32 [T / q_block + B, heads, count]; block i of sequence b is
          first[b] / q_block + b + i; pages ascending, then -1; every entry is
          written, blocks without queries (with H = 0: all) with -1
   keep_first, keep_last >= 0, their sum at most count; count in [1, 16384],
   columns at most 16384, q_block in [1, 2^20], T / q_block + B below 2^24, H T at
   most 2^29. */
regenvc_status regenvc_paged_select(const regenvc_tensor *q, const regenvc_page_pool *pool,
                                    const regenvc_page_batch *batch, int32_t H, int32_t q_block, int32_t count,
                                    int32_t keep_first, int32_t keep_last, int32_t causal, int32_t *selected,
                                    void *stream);

#ifdef __cplusplus
}
#endif

#endif /* REGENVC_PAGED_H */
