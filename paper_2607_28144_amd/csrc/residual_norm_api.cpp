// C ABI of the seam between two branches (regenvc_residual_norm_*,
// include/regenvc_dit.h): synchronous argument validation before any launch.
#include "regenvc_dit.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "abi_util.hpp"
#include "attn_kernels.hpp"
#include "residual_norm.hpp"

using regenvc::abi::aligned;
using regenvc::abi::failf;
using regenvc::abi::overlaps;
using regenvc::abi::Range;
using regenvc::abi::range_of;

namespace {

// A named argument in device memory: its bytes, and whether it is written.
struct Buffer {
    const char *name;
    const void *ptr;
    int64_t bytes;
    bool out;
};

regenvc_status check_norm(const char *fn, const char *name, const regenvc_norm *n, bool may_be_none)
{
    if (n == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: %s is NULL", fn, name);
    if (n->kind != REGENVC_NORM_LAYER && n->kind != REGENVC_NORM_RMS && !(may_be_none && n->kind == REGENVC_NORM_NONE))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: %s kind %d", fn, name, n->kind);
    if (n->kind == REGENVC_NORM_NONE && (n->w != nullptr || n->b != nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: %s has weights but no norm", fn, name);
    if (n->kind == REGENVC_NORM_RMS && n->b != nullptr)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: %s: an RMS norm has no bias", fn, name);
    if (!std::isfinite(n->eps) || n->eps < 0.f)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: %s eps must be finite, >= 0", fn, name);
    return REGENVC_OK;
}

// Rows and channels of a call, and of the query of its workspace.
regenvc_status check_size(const char *fn, int32_t rows, int32_t C)
{
    if (rows < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: rows=%d < 0", fn, rows);
    // a launch has less than 2^32 threads: workgroups of 256 for four rows each, or for one
    if (rows > (C <= 2048 ? (1 << 26) - 4 : (1 << 24) - 1))
        return failf(REGENVC_ERR_UNSUPPORTED,
                     "%s: %d rows, must be below 2^26 - 3 (2^24 with more than 2048 channels)", fn, rows);
    if (C < 8 || C % 8 != 0 || C > 8192)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: C=%d is not a multiple of 8 in [8, 8192]", fn, C);
    return REGENVC_OK;
}

regenvc_status check_common(const char *fn, regenvc_dtype dtype, const regenvc_norm *post, const regenvc_norm *pre,
                            const regenvc_row_vectors *v, float alpha, int32_t rows, int32_t C, bool backward)
{
    regenvc_status st = check_size(fn, rows, C);
    if (st != REGENVC_OK) return st;
    if (dtype != REGENVC_BF16 && dtype != REGENVC_F32) return failf(REGENVC_ERR_INVALID_ARG, "%s: dtype %d", fn, dtype);
    st = check_norm(fn, "post", post, true);
    if (st == REGENVC_OK) st = check_norm(fn, "pre", pre, false);
    if (st != REGENVC_OK) return st;
    if (!std::isfinite(alpha)) return failf(REGENVC_ERR_INVALID_ARG, "%s: alpha is not finite", fn);
    if (v == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: vectors is NULL", fn);
    if (v->group_rows < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: group_rows=%d < 0", fn, v->group_rows);
    if (backward ? v->scale == nullptr && v->shift != nullptr : (v->scale == nullptr) != (v->shift == nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: give scale and shift together", fn);
    if ((v->scale != nullptr || v->shift != nullptr) && (pre->w != nullptr || pre->b != nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: give scale and shift, or the weights of pre", fn);
    const bool grouped = v->group_rows > 0 && v->group_rows < rows;
    if (grouped && (v->gate || v->scale || v->shift) && (v->ld < C || v->ld % 4 != 0))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: vectors are ld=%lld elements apart (a multiple of 4, >= C)", fn,
                     (long long)v->ld);
    return REGENVC_OK;
}

regenvc_status check_ld(const char *fn, const char *name, int64_t ld, int32_t C)
{
    if (ld < C || ld % 8 != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: row stride %s=%lld (a multiple of 8, >= C)", fn, name, (long long)ld);
    return REGENVC_OK;
}

// Alignment of every buffer that is there, and no output over another one, but
// for the first over the second where the call is in place: these two by their
// places in the list, for another buffer at the same address is refused.
template <size_t N>
regenvc_status check_buffers(const char *fn, const Buffer (&b)[N], bool in_place)
{
    for (const Buffer &x : b)
        if (x.ptr != nullptr && !aligned(x.ptr, 16))
            return failf(REGENVC_ERR_UNSUPPORTED, "%s: %s is not 16-byte aligned", fn, x.name);
    for (size_t i = 0; i < N; ++i) {
        if (!b[i].out || b[i].ptr == nullptr) continue;
        for (size_t j = 0; j < N; ++j) {
            if (i == j || b[j].ptr == nullptr || (b[j].out && j < i)) continue;
            if (i == 0 && j == 1 && in_place) continue;
            if (overlaps(range_of(b[i].ptr, b[i].bytes), range_of(b[j].ptr, b[j].bytes)))
                return failf(REGENVC_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, b[i].name, b[j].name);
        }
    }
    return REGENVC_OK;
}

int64_t span(int64_t rows, int64_t ld, int64_t C, int64_t elem)
{
    return ((rows - 1) * ld + C) * elem;
}

regenvc::NormSpec spec(const regenvc_norm &n)
{
    return regenvc::NormSpec{n.kind, n.eps, static_cast<const uint16_t *>(n.w), static_cast<const uint16_t *>(n.b)};
}

regenvc::ResidualNormArgs common_args(const void *y, int64_t ldy, regenvc_dtype dtype, const regenvc_norm *post,
                                      const regenvc_norm *pre, const regenvc_row_vectors *v, float alpha, int32_t rows,
                                      int32_t C)
{
    regenvc::ResidualNormArgs a{};
    a.y = y, a.ldy = ldy;
    a.post = spec(*post), a.pre = spec(*pre);
    a.gate = v->gate, a.scale = v->scale, a.shift = v->shift, a.ldv = v->ld;
    a.alpha = alpha;
    a.rows = rows, a.C = C, a.group_rows = v->group_rows > 0 && v->group_rows < rows ? v->group_rows : rows;
    a.f32 = dtype == REGENVC_F32;
    return a;
}

}  // namespace

extern "C" {

regenvc_status regenvc_residual_norm_fwd(const float *x, int64_t ldx, const void *y, int64_t ldy, regenvc_dtype dtype,
                                         const regenvc_norm *post, const regenvc_norm *pre,
                                         const regenvc_row_vectors *vectors, float alpha, float *x_out, int64_t ldxo,
                                         void *h, int64_t ldh, int32_t rows, int32_t C, void *stream)
{
    const char *fn = "regenvc_residual_norm_fwd";
    regenvc_status st = check_common(fn, dtype, post, pre, vectors, alpha, rows, C, false);
    if (st == REGENVC_OK) st = check_ld(fn, "ldx", ldx, C);
    if (st == REGENVC_OK) st = check_ld(fn, "ldy", ldy, C);
    if (st == REGENVC_OK) st = check_ld(fn, "ldxo", ldxo, C);
    if (st == REGENVC_OK) st = check_ld(fn, "ldh", ldh, C);
    if (st != REGENVC_OK) return st;
    if (rows == 0) {
        regenvc::abi::clear_error();
        return REGENVC_OK;
    }
    if (!x || !y || !x_out || !h) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    regenvc::ResidualNormArgs a = common_args(y, ldy, dtype, post, pre, vectors, alpha, rows, C);
    const int64_t e = a.f32 ? 4 : 2, groups = (rows + a.group_rows - 1) / a.group_rows;
    const int64_t vec = span(groups, a.ldv, C, 4);
    const Buffer bufs[] = {{"x_out", x_out, span(rows, ldxo, C, 4), true},
                           {"x", x, span(rows, ldx, C, 4), false},
                           {"h", h, span(rows, ldh, C, e), true},
                           {"y", y, span(rows, ldy, C, e), false},
                           {"gate", a.gate, vec, false},
                           {"scale", a.scale, vec, false},
                           {"shift", a.shift, vec, false},
                           {"pre w", pre->w, (int64_t)C * 2, false},
                           {"pre b", pre->b, (int64_t)C * 2, false},
                           {"post w", post->w, (int64_t)C * 2, false},
                           {"post b", post->b, (int64_t)C * 2, false}};
    if ((st = check_buffers(fn, bufs, x_out == x && ldxo == ldx)) != REGENVC_OK) return st;
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    a.x = x, a.ldx = ldx;
    a.x_out = x_out, a.ldxo = ldxo, a.h = h, a.ldh = ldh;
    return regenvc::abi::launch_status(regenvc::launch_residual_norm_fwd(a, static_cast<hipStream_t>(stream)), fn);
}

regenvc_status regenvc_residual_norm_bwd_workspace(int32_t rows, int32_t C, int32_t group_rows, int32_t group_sums,
                                                   int32_t row_sums, int32_t n_cu, int64_t *bytes)
{
    const char *fn = "regenvc_residual_norm_bwd_workspace";
    if (bytes == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    if (rows < 0 || group_rows < 0 || n_cu < 1 || group_sums < 0 || group_sums > 3 || row_sums < 0 || row_sums > 4)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: bad size (rows=%d group_rows=%d sums=%d, %d n_cu=%d)", fn, rows,
                     group_rows, group_sums, row_sums, n_cu);
    const regenvc_status st = check_size(fn, rows, C);
    if (st != REGENVC_OK) return st;
    *bytes = 0;
    if (rows > 0)
        *bytes = regenvc::residual_norm_workspace(
            regenvc::residual_norm_plan(rows, C, group_rows > 0 && group_rows < rows ? group_rows : rows, n_cu), C,
            group_sums, row_sums);
    regenvc::abi::clear_error();
    return REGENVC_OK;
}

regenvc_status regenvc_residual_norm_bwd(const float *x_out, int64_t ldx, const void *y, int64_t ldy,
                                         regenvc_dtype dtype, const regenvc_norm *post, const regenvc_norm *pre,
                                         const regenvc_row_vectors *vectors, float alpha, const void *gh, int64_t ldgh,
                                         const float *gx, int64_t ldgx, float *dx, int64_t lddx, void *dy, int64_t lddy,
                                         const regenvc_norm_grads *grads, int32_t rows, int32_t C, void *workspace,
                                         int64_t workspace_bytes, void *stream)
{
    const char *fn = "regenvc_residual_norm_bwd";
    regenvc_status st = check_common(fn, dtype, post, pre, vectors, alpha, rows, C, true);
    if (st == REGENVC_OK) st = check_ld(fn, "ldx", ldx, C);
    if (st == REGENVC_OK) st = check_ld(fn, "ldy", ldy, C);
    if (st == REGENVC_OK) st = check_ld(fn, "ldgh", ldgh, C);
    if (st == REGENVC_OK && gx != nullptr) st = check_ld(fn, "ldgx", ldgx, C);
    if (st == REGENVC_OK) st = check_ld(fn, "lddx", lddx, C);
    if (st == REGENVC_OK) st = check_ld(fn, "lddy", lddy, C);
    if (st != REGENVC_OK) return st;
    if (grads == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: grads is NULL", fn);
    if (workspace_bytes < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
    if ((grads->dgate && !vectors->gate) || ((grads->dscale || grads->dshift) && !vectors->scale) ||
        (grads->dw && !pre->w) || (grads->db && !pre->b) || (grads->dpost_w && !post->w) || (grads->dpost_b && !post->b))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: a gradient of a vector that is not there", fn);
    if (rows == 0) {  // no rows: nothing to write but sums over none of them
        for (float *g : {grads->dw, grads->db, grads->dpost_w, grads->dpost_b})
            if (g != nullptr)
                return failf(REGENVC_ERR_INVALID_ARG, "%s: gradients of weights need at least one row", fn);
        regenvc::abi::clear_error();
        return REGENVC_OK;
    }
    if (!x_out || !y || !gh || !dx || !dy) return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL data pointer", fn);
    regenvc::ResidualNormArgs a = common_args(y, ldy, dtype, post, pre, vectors, alpha, rows, C);
    const int64_t e = a.f32 ? 4 : 2, groups = (rows + a.group_rows - 1) / a.group_rows;
    const int64_t vec = span(groups, a.ldv, C, 4), gvec = groups * C * 4, cvec = (int64_t)C * 4;
    const int group_sums = (grads->dgate != nullptr) + (grads->dscale != nullptr) + (grads->dshift != nullptr);
    const int row_sums = (grads->dw != nullptr) + (grads->db != nullptr) + (grads->dpost_w != nullptr) +
                         (grads->dpost_b != nullptr);
    const Buffer bufs[] = {{"dx", dx, span(rows, lddx, C, 4), true},
                           {"gx", gx, span(rows, ldgx, C, 4), false},
                           {"dy", dy, span(rows, lddy, C, e), true},
                           {"dgate", grads->dgate, gvec, true},
                           {"dscale", grads->dscale, gvec, true},
                           {"dshift", grads->dshift, gvec, true},
                           {"dw", grads->dw, cvec, true},
                           {"db", grads->db, cvec, true},
                           {"dpost_w", grads->dpost_w, cvec, true},
                           {"dpost_b", grads->dpost_b, cvec, true},
                           {"workspace", workspace_bytes > 0 ? workspace : nullptr, workspace_bytes, true},
                           {"x_out", x_out, span(rows, ldx, C, 4), false},
                           {"y", y, span(rows, ldy, C, e), false},
                           {"gh", gh, span(rows, ldgh, C, e), false},
                           {"gate", a.gate, vec, false},
                           {"scale", a.scale, vec, false},
                           {"pre w", pre->w, (int64_t)C * 2, false},
                           {"pre b", pre->b, (int64_t)C * 2, false},
                           {"post w", post->w, (int64_t)C * 2, false},
                           {"post b", post->b, (int64_t)C * 2, false}};
    if ((st = check_buffers(fn, bufs, dx == gx && lddx == ldgx)) != REGENVC_OK) return st;
    if (workspace != nullptr && !aligned(workspace, 256))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: workspace must be 256-byte aligned", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    const int n_cu = regenvc::device_cu_count();
    const int64_t need = regenvc::residual_norm_workspace(regenvc::residual_norm_plan(rows, C, a.group_rows, n_cu), C,
                                                          group_sums, row_sums);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace of %lld bytes, this call needs %lld", fn,
                     (long long)(workspace != nullptr ? workspace_bytes : 0), (long long)need);
    a.x = x_out, a.ldx = ldx;
    a.gh = gh, a.ldgh = ldgh, a.gx = gx, a.ldgx = ldgx;
    a.dx = dx, a.lddx = lddx, a.dy = dy, a.lddy = lddy;
    a.dgate = grads->dgate, a.dscale = grads->dscale, a.dshift = grads->dshift;
    a.dw = grads->dw, a.db = grads->db, a.dpost_w = grads->dpost_w, a.dpost_b = grads->dpost_b;
    a.ws = static_cast<float *>(workspace);
    return regenvc::abi::launch_status(regenvc::launch_residual_norm_bwd(a, n_cu, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
