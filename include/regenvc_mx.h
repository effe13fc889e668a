/*
 * regenvc_mx.h -- C ABI of the gfx950 kernels that work in MXFP4: blocks of 32
 * values of four bits (E2M1: a sign and the magnitudes 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6) under one power-of-two scale byte (E8M0: 2^(byte - 127); 255: NaN).
 * Linear layers with weights and activations in that form, for a decoder that
 * runs in real time on fewer bits than the paper's bf16 (Sec. 5.1), and
 * attention over a key/value cache held in it: the conditioning tokens that
 * Sec. 3.9 streams to the GPU, or earlier windows' tokens, at a quarter of
 * bf16's bytes.
 *
 * Bringing a block to MXFP4:
 *     scale = 2^max(-127, floor(log2 max|x|) - 2)
 *     code  = x / scale to the nearest magnitude, ties to the even code, 6 at most
 * A block of zeros has scale byte 0; one that holds an infinity or NaN has
 * scale byte 255 and stands for NaN.
 *
 * Conventions are those of regenvc_attn.h (status codes, regenvc_last_error,
 * device pointers owned by the caller, validation before any launch, work
 * enqueued on `stream`, gfx950 only, bit-identical results run to run).  None
 * of these calls allocates; none writes anything but its outputs and workspace.
 */
#ifndef REGENVC_MX_H
#define REGENVC_MX_H

#include <stdint.h>

#include "regenvc_attn.h"
#include "regenvc_dit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the codes and of the scales of a matrix [rows, K], rows below 2^26.
   K is taken in steps of 256 columns, the last one filled up with zeros.
     codes:  row-major, 128 bytes a step; column 2 i of a row in the low half
             of its byte i
     scales: for every 16 rows (the last ones filled up) and every step a line
             of 128 bytes: row x of the 16 and columns 64 g .. 64 g + 63 of the
             step have bytes 2 (16 g + x) and 2 (16 g + x) + 1
   Host-only. */
regenvc_status regenvc_mx_bytes(int32_t rows, int32_t K, int64_t *code_bytes, int64_t *scale_bytes);

/* A matrix to MXFP4: x bf16 or f32 [rows, K], row stride ldx elements.  K and
   ldx multiples of 8 (K <= 2^20), x and codes 16-byte aligned, scales 2-byte,
   else REGENVC_ERR_UNSUPPORTED. */
regenvc_status regenvc_mx_quantize(const void *x, regenvc_dtype x_dtype, int64_t ldx, void *codes, void *scales,
                                   int32_t rows, int32_t K, void *stream);

/* The values of a matrix in MXFP4: out bf16 (rounded to nearest even, which
   only values below 2^-126 and above the bf16 range need) or f32 [rows, K],
   row stride ldo, a multiple of 8; rows at most 2^26 - 4. */
regenvc_status regenvc_mx_dequantize(const void *codes, const void *scales, void *out, regenvc_dtype out_dtype,
                                     int64_t ldo, int32_t rows, int32_t K, void *stream);

/* A linear layer y = a W^T with the epilogues of regenvc_linear_fwd, both
   operands in MXFP4, fp32 accumulation:
     a:          bf16 [M, K] (row stride lda, a multiple of 8), brought to
                 MXFP4 by the call; or NULL with a_codes, a_scales: [M, K] in MXFP4
     w_codes, w_scales: [N, K] in MXFP4
     bias, gate, out, ldo, epilogue: as regenvc_linear_fwd
   M, N, K >= 0; K a multiple of 8, at most 2^20; N a multiple of 16, below
   2^20; M below 2^26, M N at most 2^42; pointers 16-byte aligned.  workspace:
   256-byte aligned, at least
   regenvc_mx_linear_workspace bytes (a's codes and scales; NULL if that is 0).
   The kernel, chosen by size, sets the order of the fp32 sum: a row may come
   out a rounding apart in calls of different numbers of rows. */
regenvc_status regenvc_mx_linear_fwd(const void *a, int64_t lda, const void *a_codes, const void *a_scales,
                                     const void *w_codes, const void *w_scales, const void *bias, const float *gate,
                                     void *out, int64_t ldo, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                                     void *workspace, int64_t workspace_bytes, void *stream);

/* Workspace bytes of such a call; `quantized`: a is in MXFP4 already.  Host-only. */
regenvc_status regenvc_mx_linear_workspace(int32_t M, int32_t N, int32_t K, int32_t quantized, int64_t *bytes);

/* The decomposition of such a call (k_ranges is 1).  Host-only. */
regenvc_status regenvc_mx_linear_plan_query(int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t n_cu,
                                            regenvc_tile_plan *plan);

/* A key/value cache of B sequences of `heads` key heads and `capacity` places,
   in caller memory: codes [B, heads, capacity, D / 2] (channel 2 i of a place
   in the low half of its byte i) and scales [B, heads, capacity, D / 32],
   contiguous, codes 16-byte aligned.  D in {64, 128}, capacity at most 2^30.  A place is a token's
   keys and values; their order has no meaning (attention is unmasked; position
   is in the rotated keys), so a cache may be rolled over. */
typedef struct {
    void *k_codes, *k_scales, *v_codes, *v_scales;
    int32_t B, capacity, heads, D;
} regenvc_mx_cache;

/* New tokens to the cache: k, v bf16 [B, S, heads, D].  Token i of sequence b,
   i < count[b], goes to place (start[b] + i) mod capacity; of more than
   `capacity` tokens only the last ones are kept.  start, count: int32 [B] in
   device memory, or NULL (0 and S); counts are held to [0, S], a sequence with
   a negative start is left as it is.  No place but those is written.  B is at
   most 65535, S heads D / 8 below 2^31. */
regenvc_status regenvc_mx_cache_append(const regenvc_mx_cache *cache, const regenvc_tensor *k, const regenvc_tensor *v,
                                       int32_t S, const int32_t *start, const int32_t *count, void *stream);

/* The cache's values: k, v bf16 or f32 [B, capacity, heads, D] contiguous.  B is
   at most 65535, capacity heads D / 8 below 2^31. */
regenvc_status regenvc_mx_cache_values(const regenvc_mx_cache *cache, void *k, void *v, regenvc_dtype dtype,
                                       void *stream);

/* Attention of q (bf16 [B, Sq, H, D], H a multiple of the cache's heads; query
   head h reads key head h / (H / heads)) over all of the first lens[b] places of
   each sequence.  Scores and sums are fp32; a softmax weight is rounded to bf16
   before it multiplies a value, whatever o_dtype is.  O, normalized by the sum of
   the rounded weights, is within 2^-8 (sum of weight |v| + |O|) of the softmax's,
   besides fp32 roundings; LSE takes the weights unrounded.
     o:    [B, Sq, H, D] in o_dtype; lse: f32 [B, H, Sq] or NULL
     lens: int32 [B] in device memory, held to [0, capacity], or NULL: max_len
           for all.  A sequence without a place gives O = 0, LSE = -inf.
     max_len: what the work is planned for, 0 <= max_len <= capacity; lens
           beyond it are computed right, only less evenly
   What lies behind lens[b] is not read.  B Sq H is at most 2^29, B times the
   cache's heads below 2^22.  workspace: 256-byte aligned, at least
   regenvc_mx_attn_cache_workspace bytes (NULL if that is 0). */
regenvc_status regenvc_mx_attn_cache_fwd(const regenvc_tensor *q, const regenvc_mx_cache *cache, const int32_t *lens,
                                         int32_t max_len, const regenvc_tensor *o, regenvc_dtype o_dtype, float *lse,
                                         int32_t B, int32_t H, int32_t Sq, float softmax_scale, void *workspace,
                                         int64_t workspace_bytes, void *stream);

/* Workspace bytes of such a call on n_cu compute units.  Host-only. */
regenvc_status regenvc_mx_attn_cache_workspace(int32_t B, int32_t H, int32_t heads, int32_t Sq, int32_t max_len,
                                               int32_t D, int32_t n_cu, int64_t *bytes);

/* The decomposition of such a call: rows of a workgroup's tile (of the Sq * H /
   heads rows that share a key head) and the ranges that the keys are cut into. */
typedef struct {
    int32_t tile_rows, row_tiles, key_ranges;
} regenvc_mx_attn_plan;
regenvc_status regenvc_mx_attn_cache_plan_query(int32_t B, int32_t H, int32_t heads, int32_t Sq, int32_t max_len,
                                                int32_t D, int32_t n_cu, regenvc_mx_attn_plan *plan);

#ifdef __cplusplus
}
#endif

#endif /* REGENVC_MX_H */
