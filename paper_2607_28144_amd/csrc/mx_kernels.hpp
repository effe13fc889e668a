// Internal launch interface of the MXFP4 kernels: quantisation, linear layers
// and attention over a key/value cache in four bits.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tile_plan.hpp"

namespace regenvc {
namespace mx {

// A matrix [rows, K] in MXFP4.  K is taken in steps of 256 columns, the last
// one filled up with zeros.  Codes: row-major, 128 bytes a step, column 2 i of
// a row in the low half of its byte i.  Scales: for each 16 rows and each step
// one line of 128 bytes, in the order in which the lanes of the matrix
// instructions take them: row x of the 16 and columns 64 g .. 64 g + 63 of the
// step have the bytes 2 (16 g + x) and 2 (16 g + x) + 1.
constexpr int kStepK = 256;
constexpr int kStepBytes = 128;
inline __host__ __device__ int steps_of(int K)
{
    return (K + kStepK - 1) / kStepK;
}
inline int64_t code_bytes(int64_t rows, int K)
{
    return rows * steps_of(K) * kStepBytes;
}
inline int64_t scale_bytes(int64_t rows, int K)
{
    return (rows + 15) / 16 * steps_of(K) * 128;
}

// x: bf16 or f32 [rows, K], row stride ldx elements (a multiple of 8, as K).
struct QuantizeArgs {
    const void *x;
    int64_t ldx;
    uint8_t *codes, *scales;
    int32_t rows, K;
    bool f32;
};
hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream);

// out: bf16 or f32 [rows, K], row stride ldo.
struct DequantizeArgs {
    const uint8_t *codes, *scales;
    void *out;
    int64_t ldo;
    int32_t rows, K;
    bool f32;
};
hipError_t launch_dequantize(const DequantizeArgs &a, hipStream_t stream);

// y = a W^T with the epilogues of LinearEpi: a in MXFP4, or (codes null) bf16
// rows that the call brings to MXFP4 itself.
struct LinearArgs {
    const void *a;
    int64_t lda;
    const uint8_t *a_codes, *a_scales;
    const uint8_t *w_codes, *w_scales;
    const void *bias;
    const float *gate;
    void *out;
    int64_t ldo;
    int32_t M, N, K;
    int32_t epi;
    void *ws;  // a's codes and scales: linear_workspace bytes
};
int64_t linear_workspace(int M, int N, int K, bool quantized);
// The plan: rows x columns of a tile and its waves (K is not split).
TilePlan linear_plan(int M, int N, int K, int epi, int n_cu);
hipError_t launch_linear(const LinearArgs &a, hipStream_t stream);

// A key/value cache: codes [B, heads, capacity, D / 2] and scales [B, heads,
// capacity, D / 32] of each, contiguous.
struct Cache {
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int32_t B, capacity, heads, D;
};
// k, v: bf16 [B, S, heads, D] with strides.  Token i < count[b] (null: S) goes
// to place (start[b] + i) mod capacity, of more than `capacity` tokens the last ones.
struct AppendArgs {
    Cache c;
    const void *k, *v;
    int64_t k_sb, k_ss, k_sh, v_sb, v_ss, v_sh;
    const int32_t *start, *count;
    int32_t S;
};
hipError_t launch_append(const AppendArgs &a, hipStream_t stream);

// k, v: bf16 or f32 [B, capacity, heads, D] contiguous.
struct ValuesArgs {
    Cache c;
    void *k, *v;
    bool f32;
};
hipError_t launch_values(const ValuesArgs &a, hipStream_t stream);

// q: bf16 [B, Sq, H, D] with strides, H a multiple of the cache's heads;
// lens[b] places of sequence b (null: max_len; held to [0, capacity]); o: bf16 or f32; lse: f32
// [B, H, Sq] or null.
struct AttnCacheArgs {
    Cache c;
    const void *q;
    void *o;
    int64_t q_sb, q_ss, q_sh, o_sb, o_ss, o_sh;
    float *lse;
    const int32_t *lens;
    int32_t B, H, Sq, max_len;
    float scale;
    bool f32;
    char *ws;
};
// The decomposition: rows of a workgroup (of the Sq * H / heads that share a
// key head), their tiles, and the ranges that each sequence's keys are cut into.
struct AttnCachePlan {
    int32_t tile_rows, row_tiles, key_ranges;
    int64_t ws_bytes;
};
AttnCachePlan attn_cache_plan(int B, int H, int heads, int Sq, int max_len, int D, int n_cu);
hipError_t launch_attn_cache(const AttnCacheArgs &a, int n_cu, hipStream_t stream);

}  // namespace mx
}  // namespace regenvc
