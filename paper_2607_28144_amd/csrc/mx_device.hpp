// Device helpers of the MXFP4 format: blocks of 32 values of 4 bits (E2M1:
// sign, magnitudes 0 0.5 1 1.5 2 3 4 6) under one power-of-two scale byte
// (E8M0: 2^(byte - 127); 255: every value of the block is NaN).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace regenvc {
namespace mx {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 32;
constexpr uint32_t kNanScale = 255;

// The scale byte of a block whose largest magnitude has these bits (as an
// f32 without its sign): two to the (its exponent - 2), so that it lies in [4,
// 8) and 6 or less after rounding; not below 2^-127; 255 if it is not finite.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits)
{
    const int e = (int)(amax_bits >> 23);
    return e == 255 ? kNanScale : (uint32_t)max(e - 2, 0);
}

// 1 / scale as an f32: exact, a block's values times it are too (or round to
// 0 either way); 0 for a block of NaN, whose codes do not matter.
__device__ __forceinline__ float scale_inverse(uint32_t byte)
{
    return __uint_as_float(byte == kNanScale ? 0u : (254u - byte) << 23);
}

// The scale as an f32.
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == kNanScale ? 0x7fc00000u : byte << 23);
}

// Eight values, already divided by the scale, as eight codes (value i in bits
// 4 i): to nearest, ties to even, held at 6.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8])
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], 1.0f, 3);
    return r;
}

// Eight codes as bf16 values times a scale given as f32 (a power of two: exact).
__device__ __forceinline__ bf16x8 decode8(uint32_t code, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The larger of a block's magnitudes over four neighbouring lanes.
__device__ __forceinline__ uint32_t quad_lane_max(uint32_t v)
{
    v = max(v, (uint32_t)__shfl_xor((int)v, 1, 64));
    return max(v, (uint32_t)__shfl_xor((int)v, 2, 64));
}

// Eight values of a block held by four neighbouring lanes (eight each): the
// block's scale byte, and this lane's codes.
__device__ __forceinline__ uint32_t quantize_quad(const float (&x)[8], uint32_t &code)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    const uint32_t byte = scale_byte(quad_lane_max(m));
    const float inv = scale_inverse(byte);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i] * inv;
    code = byte == kNanScale ? 0u : encode8(v);
    return byte;
}

}  // namespace mx
}  // namespace regenvc
