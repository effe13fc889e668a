// C ABI of the MXFP4 kernels (include/regenvc_mx.h): synchronous argument
// validation before any launch, then the kernels on the caller's stream.
#include "regenvc_mx.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "abi_util.hpp"
#include "attn_kernels.hpp"
#include "mx_kernels.hpp"

using regenvc::abi::aligned;
using regenvc::abi::failf;
using regenvc::abi::overlaps;
using regenvc::abi::Range;
using regenvc::abi::range_of;
namespace mx = regenvc::mx;

namespace {

constexpr int32_t kMaxK = 1 << 20;
constexpr int32_t kMaxN = 65535 * 16;               // 16 channels per workgroup, in the grid's second dimension
constexpr int64_t kMaxOut = (int64_t)1 << 42;        // 2^30 tiles of 64 x 64
constexpr int32_t kMaxRows = 1 << 26;                // codes and scales of 2^20 columns stay far within int64
constexpr int32_t kMaxDequantize = kMaxRows - 4;     // workgroups of 256 for four rows each: less than 2^32 threads
constexpr int32_t kMaxPlaces = 1 << 30;              // a tile past the last place stays within int32

regenvc_status done()
{
    regenvc::abi::clear_error();
    return REGENVC_OK;
}

regenvc_status check_matrix(const char *fn, int32_t rows, int32_t K)
{
    if (rows < 0 || K < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (rows=%d K=%d)", fn, rows, K);
    if (K % 8 != 0 || K > kMaxK)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: K=%d is not a multiple of 8, at most %d", fn, K, kMaxK);
    if (rows >= kMaxRows) return failf(REGENVC_ERR_UNSUPPORTED, "%s: %d rows, must be below %d", fn, rows, kMaxRows);
    return REGENVC_OK;
}

regenvc_status check_dtype(const char *fn, regenvc_dtype t)
{
    if (t != REGENVC_BF16 && t != REGENVC_F32) return failf(REGENVC_ERR_INVALID_ARG, "%s: dtype %d", fn, t);
    return REGENVC_OK;
}

int64_t span(int64_t rows, int64_t ld, int64_t C, int64_t elem)
{
    return ((rows - 1) * ld + C) * elem;
}

regenvc_status check_linear_shape(const char *fn, int32_t M, int32_t N, int32_t K, int32_t epi)
{
    if (M < 0 || N < 0 || K < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (M=%d N=%d K=%d)", fn, M, N, K);
    if (epi != REGENVC_EPI_BIAS && epi != REGENVC_EPI_BIAS_GELU && epi != REGENVC_EPI_GATED_RESIDUAL)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: unknown epilogue %d", fn, epi);
    if (N % 16 != 0) return failf(REGENVC_ERR_UNSUPPORTED, "%s: N=%d is not a multiple of 16", fn, N);
    if (N > kMaxN || (int64_t)M * N > kMaxOut)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: an output of %d x %d (N at most %d, M N at most 2^42)", fn, M, N, kMaxN);
    return check_matrix(fn, M, K);
}

regenvc_status check_cache(const char *fn, const regenvc_mx_cache *c, Range (&r)[4])
{
    if (c == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: cache is NULL", fn);
    if (c->B < 0 || c->capacity < 0 || c->heads < 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: negative cache size (B=%d capacity=%d heads=%d)", fn, c->B, c->capacity,
                     c->heads);
    if (c->D != 64 && c->D != 128) return failf(REGENVC_ERR_UNSUPPORTED, "%s: head dim D=%d (only 64 and 128)", fn, c->D);
    if (c->capacity > kMaxPlaces)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: a capacity of %d, at most %d", fn, c->capacity, kMaxPlaces);
    int64_t n = 0;
    if (__builtin_mul_overflow((int64_t)c->B * c->heads, (int64_t)c->capacity, &n) || n > INT64_MAX / 512)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: the cache's offsets overflow int64", fn);
    const void *p[4] = {c->k_codes, c->v_codes, c->k_scales, c->v_scales};
    for (int i = 0; i < 4; ++i) {
        if (n > 0 && p[i] == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL cache pointer", fn);
        if (i < 2 && !aligned(p[i], 16))
            return failf(REGENVC_ERR_UNSUPPORTED, "%s: the cache's codes are not 16-byte aligned", fn);
        r[i] = range_of(p[i], n * c->D / (i < 2 ? 2 : 32));
    }
    return REGENVC_OK;
}

mx::Cache cache_of(const regenvc_mx_cache &c)
{
    auto u8 = [](void *p) { return static_cast<uint8_t *>(p); };
    return mx::Cache{u8(c.k_codes), u8(c.k_scales), u8(c.v_codes), u8(c.v_scales), c.B, c.capacity, c.heads, c.D};
}

// The four parts of a cache overlap neither each other nor r.
bool meets(const Range (&c)[4], const Range &r)
{
    return std::any_of(c, c + 4, [&](const Range &x) { return overlaps(x, r); });
}
bool meets_itself(const Range (&c)[4])
{
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (overlaps(c[i], c[j])) return true;
    return false;
}

regenvc_status check_attn_shape(const char *fn, int32_t B, int32_t H, int32_t heads, int32_t Sq, int32_t max_len,
                                int32_t D)
{
    if (B < 0 || H < 0 || Sq < 0 || heads < 0 || max_len < 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (B=%d H=%d heads=%d Sq=%d max_len=%d)", fn, B, H, heads, Sq,
                     max_len);
    if (D != 64 && D != 128) return failf(REGENVC_ERR_UNSUPPORTED, "%s: head dim D=%d (only 64 and 128)", fn, D);
    if (H > 0 && (heads == 0 || H % heads != 0))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: H=%d is not a multiple of the cache's %d heads", fn, H, heads);
    if (max_len > kMaxPlaces)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: max_len=%d, at most %d", fn, max_len, kMaxPlaces);
    // a launch has less than 2^32 threads: 256 per 16 or 32 rows that share a key head, 512 per 256 of more than 128
    int64_t rows = 0;
    if (__builtin_mul_overflow((int64_t)Sq * H, (int64_t)std::max(B, 1), &rows) || rows > (int64_t)1 << 29 ||
        (int64_t)B * heads >= (int64_t)1 << 22)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: B * Sq * H is more than 2^29, or B * heads 2^22 or more", fn);
    return REGENVC_OK;
}

}  // namespace

extern "C" {

regenvc_status regenvc_mx_bytes(int32_t rows, int32_t K, int64_t *code_bytes, int64_t *scale_bytes)
{
    const char *fn = "regenvc_mx_bytes";
    if (code_bytes == nullptr || scale_bytes == nullptr)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: code_bytes or scale_bytes is NULL", fn);
    const regenvc_status st = check_matrix(fn, rows, K);
    if (st != REGENVC_OK) return st;
    *code_bytes = mx::code_bytes(rows, K);
    *scale_bytes = mx::scale_bytes(rows, K);
    return done();
}

regenvc_status regenvc_mx_quantize(const void *x, regenvc_dtype x_dtype, int64_t ldx, void *codes, void *scales,
                                   int32_t rows, int32_t K, void *stream)
{
    const char *fn = "regenvc_mx_quantize";
    regenvc_status st = check_matrix(fn, rows, K);
    if (st == REGENVC_OK) st = check_dtype(fn, x_dtype);
    if (st != REGENVC_OK) return st;
    if (rows == 0 || K == 0) return done();
    if (ldx < K || ldx % 8 != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: row stride ldx=%lld (a multiple of 8, >= K)", fn, (long long)ldx);
    if (!x || !codes || !scales) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    if (!aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 2))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: x and codes must be 16-byte, scales 2-byte aligned", fn);
    const Range rx = range_of(x, span(rows, ldx, K, x_dtype == REGENVC_F32 ? 4 : 2));
    const Range rc = range_of(codes, mx::code_bytes(rows, K)), rs = range_of(scales, mx::scale_bytes(rows, K));
    if (overlaps(rx, rc) || overlaps(rx, rs) || overlaps(rc, rs))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: x, codes and scales overlap", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const mx::QuantizeArgs a{x, ldx, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), rows, K,
                             x_dtype == REGENVC_F32};
    return regenvc::abi::launch_status(mx::launch_quantize(a, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_mx_dequantize(const void *codes, const void *scales, void *out, regenvc_dtype out_dtype,
                                     int64_t ldo, int32_t rows, int32_t K, void *stream)
{
    const char *fn = "regenvc_mx_dequantize";
    regenvc_status st = check_matrix(fn, rows, K);
    if (st == REGENVC_OK) st = check_dtype(fn, out_dtype);
    if (st != REGENVC_OK) return st;
    if (rows > kMaxDequantize)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: %d rows, at most %d", fn, rows, kMaxDequantize);
    if (rows == 0 || K == 0) return done();
    if (ldo < K || ldo % 8 != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: row stride ldo=%lld (a multiple of 8, >= K)", fn, (long long)ldo);
    if (!out || !codes || !scales) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    if (!aligned(out, 16) || !aligned(codes, 16))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: out and codes must be 16-byte aligned", fn);
    const Range ro = range_of(out, span(rows, ldo, K, out_dtype == REGENVC_F32 ? 4 : 2));
    if (overlaps(ro, range_of(codes, mx::code_bytes(rows, K))) || overlaps(ro, range_of(scales, mx::scale_bytes(rows, K))))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const mx::DequantizeArgs a{static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), out, ldo, rows, K,
                               out_dtype == REGENVC_F32};
    return regenvc::abi::launch_status(mx::launch_dequantize(a, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_mx_linear_workspace(int32_t M, int32_t N, int32_t K, int32_t quantized, int64_t *bytes)
{
    const char *fn = "regenvc_mx_linear_workspace";
    if (bytes == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    const regenvc_status st = check_linear_shape(fn, M, N, K, REGENVC_EPI_BIAS);
    if (st != REGENVC_OK) return st;
    *bytes = mx::linear_workspace(M, N, K, quantized != 0);
    return done();
}

regenvc_status regenvc_mx_linear_plan_query(int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t n_cu,
                                            regenvc_tile_plan *plan)
{
    const char *fn = "regenvc_mx_linear_plan_query";
    if (plan == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: plan is NULL", fn);
    if (n_cu < 1) return failf(REGENVC_ERR_INVALID_ARG, "%s: n_cu=%d < 1", fn, n_cu);
    const regenvc_status st = check_linear_shape(fn, M, N, K, epilogue);
    if (st != REGENVC_OK) return st;
    const regenvc::TilePlan p = mx::linear_plan(M, N, K, epilogue, n_cu);
    *plan = regenvc_tile_plan{p.bm, p.bn, p.waves, p.splits};
    return done();
}

regenvc_status regenvc_mx_linear_fwd(const void *a, int64_t lda, const void *a_codes, const void *a_scales,
                                     const void *w_codes, const void *w_scales, const void *bias, const float *gate,
                                     void *out, int64_t ldo, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                                     void *workspace, int64_t workspace_bytes, void *stream)
{
    const char *fn = "regenvc_mx_linear_fwd";
    regenvc_status st = check_linear_shape(fn, M, N, K, epilogue);
    if (st != REGENVC_OK) return st;
    if (gate != nullptr && epilogue != REGENVC_EPI_GATED_RESIDUAL)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: a gate needs the gated-residual epilogue", fn);
    if (workspace_bytes < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
    const bool quantized = a == nullptr && K > 0;
    if (a != nullptr && (a_codes != nullptr || a_scales != nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: give a, or a_codes and a_scales", fn);
    if (M == 0 || N == 0) return done();
    if (ldo < N || ldo % 8 != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: row stride ldo=%lld (a multiple of 8, >= N)", fn, (long long)ldo);
    if (a != nullptr && K > 0 && (lda < K || lda % 8 != 0))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: row stride lda=%lld (a multiple of 8, >= K)", fn, (long long)lda);
    if (out == nullptr || (K > 0 && (w_codes == nullptr || w_scales == nullptr)) ||
        (quantized && (a_codes == nullptr || a_scales == nullptr)))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    for (const void *p : {a, a_codes, a_scales, w_codes, w_scales, bias, static_cast<const void *>(gate),
                          static_cast<const void *>(out)})
        if (!aligned(p, 16)) return failf(REGENVC_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);
    if (workspace != nullptr && !aligned(workspace, 256))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: workspace must be 256-byte aligned", fn);
    const int64_t ws_bytes = workspace != nullptr ? workspace_bytes : 0;
    const Range ro = range_of(out, span(M, ldo, N, epilogue == REGENVC_EPI_GATED_RESIDUAL ? 4 : 2));
    const Range rw = range_of(workspace, ws_bytes);
    const Range in[] = {range_of(a, a != nullptr ? span(M, lda, K, 2) : 0),
                        range_of(a_codes, a_codes != nullptr ? mx::code_bytes(M, K) : 0),
                        range_of(a_scales, a_scales != nullptr ? mx::scale_bytes(M, K) : 0),
                        range_of(w_codes, w_codes != nullptr ? mx::code_bytes(N, K) : 0),
                        range_of(w_scales, w_scales != nullptr ? mx::scale_bytes(N, K) : 0),
                        range_of(bias, bias != nullptr ? (int64_t)N * 2 : 0),
                        range_of(gate, gate != nullptr ? (int64_t)N * 4 : 0)};
    for (const Range &r : in) {
        if (overlaps(r, ro)) return failf(REGENVC_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
        if (overlaps(r, rw)) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace overlaps another argument", fn);
    }
    if (overlaps(ro, rw)) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace overlaps another argument", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const int64_t need = mx::linear_workspace(M, N, K, quantized);
    if (ws_bytes < need)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace of %lld bytes, this call needs %lld", fn, (long long)ws_bytes,
                     (long long)need);
    auto u8 = [](const void *p) { return static_cast<const uint8_t *>(p); };
    const mx::LinearArgs la{a,   lda, u8(a_codes), u8(a_scales), u8(w_codes), u8(w_scales), bias, gate, out, ldo, M,
                            N,   K,   epilogue,    workspace};
    return regenvc::abi::launch_status(mx::launch_linear(la, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_mx_cache_append(const regenvc_mx_cache *cache, const regenvc_tensor *k, const regenvc_tensor *v,
                                       int32_t S, const int32_t *start, const int32_t *count, void *stream)
{
    const char *fn = "regenvc_mx_cache_append";
    Range rc[4];
    regenvc_status st = check_cache(fn, cache, rc);
    if (st != REGENVC_OK) return st;
    if (S < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: S=%d < 0", fn, S);
    if (cache->B == 0 || cache->heads == 0 || cache->capacity == 0 || S == 0) return done();
    Range rk, rv;
    if ((st = regenvc::abi::view_range("k", k, cache->B, S, cache->heads, cache->D, 2, &rk)) != REGENVC_OK) return st;
    if ((st = regenvc::abi::view_range("v", v, cache->B, S, cache->heads, cache->D, 2, &rv)) != REGENVC_OK) return st;
    if (!aligned(start, 4) || !aligned(count, 4))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: start and count must be 4-byte aligned", fn);
    const int64_t nb = (int64_t)cache->B * 4;
    if (meets_itself(rc) || meets(rc, rk) || meets(rc, rv) || (start && meets(rc, range_of(start, nb))) ||
        (count && meets(rc, range_of(count, nb))))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: the cache overlaps itself or an input", fn);
    if (cache->B > 65535 || (int64_t)S > INT32_MAX / ((int64_t)cache->heads * (cache->D / 8)))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: too many sequences or tokens for one call", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const mx::AppendArgs a{cache_of(*cache), k->ptr,      v->ptr,      k->stride_b, k->stride_s, k->stride_h, v->stride_b,
                           v->stride_s,      v->stride_h, start,       count,       S};
    return regenvc::abi::launch_status(mx::launch_append(a, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_mx_cache_values(const regenvc_mx_cache *cache, void *k, void *v, regenvc_dtype dtype,
                                       void *stream)
{
    const char *fn = "regenvc_mx_cache_values";
    Range rc[4];
    regenvc_status st = check_cache(fn, cache, rc);
    if (st == REGENVC_OK) st = check_dtype(fn, dtype);
    if (st != REGENVC_OK) return st;
    const int64_t n = (int64_t)cache->B * cache->heads * cache->capacity * cache->D;
    if (n == 0) return done();
    if (!k || !v) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    if (!aligned(k, 16) || !aligned(v, 16)) return failf(REGENVC_ERR_UNSUPPORTED, "%s: k and v must be 16-byte aligned", fn);
    const Range rk = range_of(k, n * (dtype == REGENVC_F32 ? 4 : 2)), rv = range_of(v, n * (dtype == REGENVC_F32 ? 4 : 2));
    if (overlaps(rk, rv) || meets(rc, rk) || meets(rc, rv))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: k, v and the cache overlap", fn);
    if (cache->B > 65535 || (int64_t)cache->capacity > INT32_MAX / ((int64_t)cache->heads * (cache->D / 8)))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: too many sequences or places for one call", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const mx::ValuesArgs a{cache_of(*cache), k, v, dtype == REGENVC_F32};
    return regenvc::abi::launch_status(mx::launch_values(a, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_mx_attn_cache_workspace(int32_t B, int32_t H, int32_t heads, int32_t Sq, int32_t max_len,
                                               int32_t D, int32_t n_cu, int64_t *bytes)
{
    const char *fn = "regenvc_mx_attn_cache_workspace";
    if (bytes == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    if (n_cu < 1) return failf(REGENVC_ERR_INVALID_ARG, "%s: n_cu=%d < 1", fn, n_cu);
    const regenvc_status st = check_attn_shape(fn, B, H, heads, Sq, max_len, D);
    if (st != REGENVC_OK) return st;
    *bytes = (int64_t)B * H * Sq > 0 ? mx::attn_cache_plan(B, H, heads, Sq, max_len, D, n_cu).ws_bytes : 0;
    return done();
}

regenvc_status regenvc_mx_attn_cache_plan_query(int32_t B, int32_t H, int32_t heads, int32_t Sq, int32_t max_len,
                                                int32_t D, int32_t n_cu, regenvc_mx_attn_plan *plan)
{
    const char *fn = "regenvc_mx_attn_cache_plan_query";
    if (plan == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: plan is NULL", fn);
    if (n_cu < 1) return failf(REGENVC_ERR_INVALID_ARG, "%s: n_cu=%d < 1", fn, n_cu);
    const regenvc_status st = check_attn_shape(fn, B, H, heads, Sq, max_len, D);
    if (st != REGENVC_OK) return st;
    *plan = regenvc_mx_attn_plan{};
    if ((int64_t)B * H * Sq > 0) {
        const mx::AttnCachePlan p = mx::attn_cache_plan(B, H, heads, Sq, max_len, D, n_cu);
        *plan = regenvc_mx_attn_plan{p.tile_rows, p.row_tiles, p.key_ranges};
    }
    return done();
}

regenvc_status regenvc_mx_attn_cache_fwd(const regenvc_tensor *q, const regenvc_mx_cache *cache, const int32_t *lens,
                                         int32_t max_len, const regenvc_tensor *o, regenvc_dtype o_dtype, float *lse,
                                         int32_t B, int32_t H, int32_t Sq, float softmax_scale, void *workspace,
                                         int64_t workspace_bytes, void *stream)
{
    const char *fn = "regenvc_mx_attn_cache_fwd";
    Range rc[4];
    regenvc_status st = check_cache(fn, cache, rc);
    if (st == REGENVC_OK) st = check_attn_shape(fn, B, H, cache->heads, Sq, max_len, cache->D);
    if (st == REGENVC_OK) st = check_dtype(fn, o_dtype);
    if (st == REGENVC_OK) st = regenvc::abi::softmax_scale_ok(softmax_scale);
    if (st != REGENVC_OK) return st;
    if (B != cache->B) return failf(REGENVC_ERR_INVALID_ARG, "%s: B=%d, the cache holds %d sequences", fn, B, cache->B);
    if (max_len > cache->capacity)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: max_len=%d, the cache holds %d places", fn, max_len, cache->capacity);
    if (workspace_bytes < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
    if (B == 0 || H == 0 || Sq == 0) return done();
    const int D = cache->D, elem = o_dtype == REGENVC_F32 ? 4 : 2;
    Range rq, ro;
    if ((st = regenvc::abi::view_range("q", q, B, Sq, H, D, 2, &rq)) != REGENVC_OK) return st;
    if ((st = regenvc::abi::view_range("o", o, B, Sq, H, D, elem, &ro)) != REGENVC_OK) return st;
    if (!regenvc::abi::view_injective(o, B, Sq, H, D))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: elements of o share an address", fn);
    if (!aligned(lse, 4) || !aligned(lens, 4))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: lse and lens must be 4-byte aligned", fn);
    if (workspace != nullptr && !aligned(workspace, 256))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: workspace must be 256-byte aligned", fn);
    const Range rl = range_of(lse, lse != nullptr ? (int64_t)B * H * Sq * 4 : 0);
    const Range rn = range_of(lens, lens != nullptr ? (int64_t)B * 4 : 0);
    const Range rw = range_of(workspace, workspace != nullptr ? workspace_bytes : 0);
    for (const Range &r : {ro, rl, rw})
        if (overlaps(r, rq) || overlaps(r, rn) || meets(rc, r))
            return failf(REGENVC_ERR_INVALID_ARG, "%s: an output or the workspace overlaps an input", fn);
    if (overlaps(ro, rl) || overlaps(ro, rw) || overlaps(rl, rw))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: o, lse and the workspace overlap", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const int n_cu = regenvc::device_cu_count();
    const int64_t need = mx::attn_cache_plan(B, H, cache->heads, Sq, max_len, D, n_cu).ws_bytes;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace of %lld bytes, this call needs %lld", fn,
                     (long long)(workspace != nullptr ? workspace_bytes : 0), (long long)need);
    const mx::AttnCacheArgs a{cache_of(*cache), q->ptr,      o->ptr, q->stride_b, q->stride_s, q->stride_h,
                              o->stride_b,      o->stride_s, o->stride_h, lse,    lens,        B,
                              H,                Sq,          max_len,     softmax_scale, o_dtype == REGENVC_F32,
                              static_cast<char *>(workspace)};
    return regenvc::abi::launch_status(mx::launch_attn_cache(a, n_cu, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
