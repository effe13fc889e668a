// Device helpers of attention on v_mfma_f32_16x16x32_bf16 with transposed scores
// (a lane holds keys of one query row), shared by the kernels that read a cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace regenvc {
namespace cache_attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -3.0e38f;  // a running maximum before any key: below every score, and finite

// x combined over the lanes l, l^16, l^32, l^48 (each gets the result).
__device__ __forceinline__ float quad_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float t = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
    return fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
}
__device__ __forceinline__ float quad_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float t = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
    return __uint_as_float(u[0]) + __uint_as_float(u[1]);
}

// 16-byte chunk of a V row in LDS (2 D bytes a row) where chunk c of key row r
// is kept: pairs of chunks change places with the row, so that the transposing
// reads (32 bytes of each of 8 rows at a time) do not meet in a bank.
template <int D>
__device__ __forceinline__ int v_slot(int r, int c)
{
    return c ^ ((D == 128 ? r & 7 : r >> 1 & 3) << 1);
}

// The same for K rows.  A fragment read takes chunk D / 32 g + ks of 16 rows,
// served for rows 0-3, 12-15 of one g with rows 4-11 of the next (or the other
// way round): their chunks, a block or half a block apart, are kept apart by
// rows 4-11 counting in that bit too (1560 queries x 32760 places x 12 heads, 303
// us: 301 so, with a third of the conflict cycles).
template <int D>
__device__ __forceinline__ int k_slot(int r, int c)
{
    return c ^ (D == 128 ? (r & 15) ^ ((r + 4 & 8) >> 1) : (r >> 1 & 1) | (r & 4 ? 6 : 0));
}

// log2(e) times the softmax scale.  Never 0, so that -inf, the score of a
// place past the end, stays -inf; a scale of 0 still gives equal weights.
__device__ __forceinline__ float log2_scale(float scale)
{
    return fmaxf(scale * kLog2e, 1.2e-38f);
}

// Weights are formed against a reference m that is raised only where a lane's
// sum of 8 or 16 weights passes this (or is not finite: the first tile): a
// weight is then at most as much above 1, which fp32 sums and bf16 operands
// hold as well, and the common path needs no maximum.
constexpr float kSpecLimit = 256.0f;

// Two weights, rounded to bf16, into a P operand, and their sum (as rounded) to rs.
__device__ __forceinline__ void put_pair(bf16x8 &dst, int j, float x0, float x1, float &rs)
{
    const bf16x2 pk = {(__bf16)x0, (__bf16)x1}, one = {(__bf16)1.0f, (__bf16)1.0f};
    dst[j] = pk[0];
    dst[j + 1] = pk[1];
    rs = __builtin_amdgcn_fdot2_f32_bf16(pk, one, rs, false);
}

// Weights of 32 keys (8 of them this lane's) for one row against m: in bf16, their sum, their sum as rounded.
__device__ __forceinline__ void weights32(const f32x4 (&s)[2], float c, float m, float &lsum, float &rsum, bf16x8 &p)
{
    lsum = 0.f, rsum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c, -m));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][(i & 3) + 1], c, -m));
        put_pair(p, i, e0, e1, rsum);
        lsum += e0 + e1;
    }
}

}  // namespace cache_attn
}  // namespace regenvc
