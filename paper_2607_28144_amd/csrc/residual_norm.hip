// gfx950 kernels of the seam between two branches of a diffusion-transformer
// block: what a branch gave is normalized, gated and added to the residual
// stream, and the stream is normalized for the next branch, in one pass over
// the rows; and the gradients of that step.  With N(t) = (t - mean) / sigma or
// t / rms over a row's C channels:
//     u  = N_post(y) w_post + b_post        (or u = y)
//     x' = alpha x + gate u
//     h  = N_pre(x') (1 + scale) + shift    (or N_pre(x') w + b)
//
// HBM-bound: forward reads x and y and writes x' and h (12 bytes a value with
// bf16 branches), backward reads x', y, gh and gx and writes dx and dy (18).  A
// row stays in registers from its loads to its stores, so that statistics,
// also the backward's own, cost no second read: one wave per row up to 2048
// channels, four waves per row up to 8192, eight channels (16 or 32 bytes) per
// lane and access.  Mean and variance are two passes over the registers.
#include "residual_norm.hpp"

#include <algorithm>

namespace regenvc {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct F8 {
    float v[8];
};

// eight values of a row as they are held between load and use
template <bool F32>
struct Raw;
template <>
struct Raw<true> {
    f32x4 a, b;
    __device__ float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
template <>
struct Raw<false> {
    bf16x8 a;
    __device__ float operator[](int i) const { return (float)a[i]; }
};

template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const void *p, int64_t at)
{
    Raw<F32> r;
    if constexpr (F32) {
        const float *q = static_cast<const float *>(p) + at;
        r.a = *reinterpret_cast<const f32x4 *>(q);
        r.b = *reinterpret_cast<const f32x4 *>(q + 4);
    } else {
        r.a = *reinterpret_cast<const bf16x8 *>(static_cast<const uint16_t *>(p) + at);
    }
    return r;
}

template <bool F32>
__device__ __forceinline__ void store8(void *p, int64_t at, const F8 &x)
{
    if constexpr (F32) {
        float *q = static_cast<float *>(p) + at;
        *reinterpret_cast<f32x4 *>(q) = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
        *reinterpret_cast<f32x4 *>(q + 4) = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
    } else {
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)x.v[i];
        *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(p) + at) = o;
    }
}

// eight values of an f32 or bf16 vector, or of a missing one
__device__ __forceinline__ F8 vec_f32(const float *p, int64_t at, float missing)
{
    F8 r;
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = missing;
        return r;
    }
    const Raw<true> q = load_raw<true>(p, at);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = q[i];
    return r;
}
__device__ __forceinline__ F8 vec_bf16(const uint16_t *p, int at, float missing)
{
    F8 r;
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = missing;
        return r;
    }
    const Raw<false> q = load_raw<false>(p, at);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = q[i];
    return r;
}

// what the pre-norm's values are multiplied by, and what is added
__device__ __forceinline__ F8 pre_mul(const ResidualNormArgs &a, int64_t gv, int c)
{
    if (a.scale == nullptr) return vec_bf16(a.pre.w, c, 1.f);
    F8 m = vec_f32(a.scale, gv + c, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) m.v[i] += 1.f;
    return m;
}
__device__ __forceinline__ F8 pre_add(const ResidualNormArgs &a, int64_t gv, int c)
{
    return a.shift != nullptr ? vec_f32(a.shift, gv + c, 0.f) : vec_bf16(a.pre.b, c, 0.f);
}

// Sums of N values over the lanes of a row: its wave, or its workgroup's four
// waves (through LDS; `turn` names the half that this sum uses, so that one
// barrier a sum suffices).
template <int WPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float (*lds)[2 * kWaves], int &turn)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += __shfl_xor(s[k], m, 64);
    if constexpr (WPR > 1) {
        float *slot = lds[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) slot[k * kWaves + (threadIdx.x >> 6)] = s[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = (slot[k * kWaves] + slot[k * kWaves + 1]) + (slot[k * kWaves + 2] + slot[k * kWaves + 3]);
    }
}

// Mean (0 for RMS) and 1/sigma of the row whose values val(v, i) this lane
// holds for v < NV with on[v].
template <int WPR, int NV, class Val>
__device__ __forceinline__ void row_stats(const Val &val, const bool (&on)[NV], int kind, float inv_c, float eps,
                                          float (*lds)[2 * kWaves], int &turn, float &mu, float &rstd)
{
    mu = 0.f;
    if (kind == kNormLayer) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += val(v, i);
        row_sum<WPR>(s, lds, turn);
        mu = s[0] * inv_c;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (on[v]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = val(v, i) - mu;
                q[0] = fmaf(d, d, q[0]);
            }
        }
    row_sum<WPR>(q, lds, turn);
    rstd = rsqrtf(q[0] * inv_c + eps);
}

// Forward: WPR waves per row, NV eight-channel chunks per lane.
template <int NV, int WPR, bool F32>
__global__ __launch_bounds__(kThreads) void residual_norm_fwd_kernel(ResidualNormArgs a)
{
    constexpr int TPR = 64 * WPR;  // lanes of a row
    __shared__ float lds[2][2 * kWaves];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const int64_t row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * (kThreads / TPR) + (int)threadIdx.x / TPR);
    if (row >= a.rows) return;  // with WPR > 1 the whole workgroup
    const int64_t gv = (int64_t)((int)row / a.group_rows) * a.ldv;
    const float inv_c = 1.0f / (float)a.C;

    bool on[NV];
    Raw<F32> y[NV];
    F8 r[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        on[v] = c < a.C;
        y[v] = Raw<F32>{};
        if (on[v]) y[v] = load_raw<F32>(a.y, row * a.ldy + c);
        r[v] = on[v] ? vec_f32(a.x, row * a.ldx + c, 0.f) : F8{};
    }
    float mu = 0.f, rstd = 1.f;
    const bool post = a.post.kind != kNormNone;
    if (post)
        row_stats<WPR, NV>([&](int v, int i) { return y[v][i]; }, on, a.post.kind, inv_c, a.post.eps, lds, turn, mu, rstd);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (!on[v]) continue;
        const F8 g = vec_f32(a.gate, gv + c, 1.f);
        F8 u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.v[i] = (y[v][i] - mu) * rstd;
        if (post) {
            const F8 w = vec_bf16(a.post.w, c, 1.f), b = vec_bf16(a.post.b, c, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) u.v[i] = fmaf(u.v[i], w.v[i], b.v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) r[v].v[i] = fmaf(g.v[i], u.v[i], a.alpha * r[v].v[i]);
        store8<true>(a.x_out, row * a.ldxo + c, r[v]);
    }
    row_stats<WPR, NV>([&](int v, int i) { return r[v].v[i]; }, on, a.pre.kind, inv_c, a.pre.eps, lds, turn, mu, rstd);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (!on[v]) continue;
        const F8 mul = pre_mul(a, gv, c), add = pre_add(a, gv, c);
        F8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h.v[i] = fmaf((r[v].v[i] - mu) * rstd, mul.v[i], add.v[i]);
        store8<F32>(a.h, row * a.ldh + c, h);
    }
}

// Sums over rows that the backward pass keeps per lane, one F8 per chunk.
enum Sum { kSumGate, kSumMul, kSumAdd, kSumPostW, kSumPostB };

// Backward of one row, in the order of the chain rule (m = mean over the C
// channels, n = N_pre(x'), p = N_post(y)):
//     g  = gh (1 + scale)          dr = gx + (g - m(g) - n m(g n)) / sigma
//     dx = alpha dr                du = gate dr         dgate = sum dr u
//     q  = du w_post               dy = (q - m(q) - p m(q p)) / sigma_y
//     dscale, dw = sum gh n        dshift, db = sum gh
//     dpost_w = sum du p           dpost_b = sum du
// (without m(g), m(q) for RMS norms; dy = du without a post-norm).  A
// workgroup walks the rows of its segments, keeps the sums over them in
// registers and adds its waves' through LDS at the end of a segment, in a
// fixed order: no atomics.  NS: sums held (3, 4 with a post-norm, 5 with its bias).
template <int NV, int WPR, bool F32, int NS>
__global__ __launch_bounds__(kThreads) void residual_norm_bwd_kernel(ResidualNormArgs a, ResidualNormPlan p,
                                                                     float *group_ws, float *row_ws)
{
    constexpr int TPR = 64 * WPR, RPB = kThreads / TPR;  // lanes of a row, rows at a time
    constexpr bool POST = NS > 3;
    __shared__ float lds[2][2 * kWaves];
    __shared__ __attribute__((aligned(16))) float stage[RPB > 1 ? RPB * NV * TPR * 8 : 4];
    int turn = 0;
    const int t = threadIdx.x % TPR, lane_row = threadIdx.x / TPR;
    const float inv_c = 1.0f / (float)a.C;
    const bool modulated = a.scale != nullptr;
    bool on[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) on[v] = (v * TPR + t) * 8 < a.C;

    F8 sum[NS][NV];
    auto clear = [&](int s) {
#pragma unroll
        for (int v = 0; v < NV; ++v) sum[s][v] = F8{};
    };
    // the workgroup's sum s to out [C] (null: dropped)
    auto flush = [&](int s, float *out) {
        if (out == nullptr) return;
        if constexpr (RPB > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v) store8<true>(stage, (lane_row * NV + v) * TPR * 8 + t * 8, sum[s][v]);
            __syncthreads();
            for (int c = threadIdx.x; c < a.C; c += kThreads) {
                float z = stage[c];
#pragma unroll
                for (int k = 1; k < RPB; ++k) z += stage[k * NV * TPR * 8 + c];
                out[c] = z;
            }
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (on[v]) store8<true>(out, (v * TPR + t) * 8, sum[s][v]);
        }
    };
#pragma unroll
    for (int s = 0; s < NS; ++s) clear(s);

    for (int64_t seg = blockIdx.x; seg < p.segments(); seg += gridDim.x) {
        const int group = (int)(seg / p.per_group), part = (int)(seg % p.per_group);
        const int64_t gr0 = (int64_t)group * a.group_rows;
        const int64_t n = min((int64_t)a.group_rows, a.rows - gr0);
        const int64_t r0 = gr0 + n * part / p.per_group, r1 = gr0 + n * (part + 1) / p.per_group;
        const int64_t gv = (int64_t)group * a.ldv;
        for (int64_t rr = r0; rr < r1; rr += RPB) {
            const int64_t row = __builtin_amdgcn_readfirstlane((int)rr + lane_row);
            if (row >= r1) break;  // with WPR > 1 never within a row
            Raw<F32> y[NV], gh[NV];
            Raw<true> x[NV], gx[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * TPR + t) * 8;
                y[v] = gh[v] = Raw<F32>{};
                x[v] = gx[v] = Raw<true>{};
                if (on[v]) {
                    x[v] = load_raw<true>(a.x, row * a.ldx + c);
                    gh[v] = load_raw<F32>(a.gh, row * a.ldgh + c);
                    y[v] = load_raw<F32>(a.y, row * a.ldy + c);
                    if (a.gx != nullptr) gx[v] = load_raw<true>(a.gx, row * a.ldgx + c);
                }
            }
            float mu, rstd;
            row_stats<WPR, NV>([&](int v, int i) { return x[v][i]; }, on, a.pre.kind, inv_c, a.pre.eps, lds, turn, mu,
                               rstd);
            float m[2] = {0.f, 0.f};
            F8 g[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!on[v]) continue;
                const F8 mul = pre_mul(a, gv, (v * TPR + t) * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float nn = (x[v][i] - mu) * rstd;
                    g[v].v[i] = gh[v][i] * mul.v[i];
                    m[0] += g[v].v[i];
                    m[1] = fmaf(g[v].v[i], nn, m[1]);
                    sum[kSumMul][v].v[i] = fmaf(gh[v][i], nn, sum[kSumMul][v].v[i]);
                    sum[kSumAdd][v].v[i] += gh[v][i];
                }
            }
            row_sum<WPR>(m, lds, turn);
            const float mg = a.pre.kind == kNormLayer ? m[0] * inv_c : 0.f, mgn = m[1] * inv_c;
            float mu_y = 0.f, rstd_y = 1.f;
            if constexpr (POST)
                row_stats<WPR, NV>([&](int v, int i) { return y[v][i]; }, on, a.post.kind, inv_c, a.post.eps, lds, turn,
                                   mu_y, rstd_y);
            m[0] = m[1] = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!on[v]) continue;
                const int c = (v * TPR + t) * 8;
                const F8 gate = vec_f32(a.gate, gv + c, 1.f);
                F8 w, b, dx;
                if constexpr (POST) w = vec_bf16(a.post.w, c, 1.f), b = vec_bf16(a.post.b, c, 0.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float nn = (x[v][i] - mu) * rstd;
                    const float dr = gx[v][i] + rstd * (g[v].v[i] - mg - nn * mgn);
                    dx.v[i] = a.alpha * dr;
                    const float du = gate.v[i] * dr;
                    float u = y[v][i];
                    g[v].v[i] = du;
                    if constexpr (POST) {
                        const float pn = (u - mu_y) * rstd_y;
                        u = fmaf(pn, w.v[i], b.v[i]);
                        sum[kSumPostW][v].v[i] = fmaf(du, pn, sum[kSumPostW][v].v[i]);
                        if constexpr (NS > 4) sum[kSumPostB][v].v[i] += du;
                        const float q = du * w.v[i];
                        g[v].v[i] = q;
                        m[0] += q;
                        m[1] = fmaf(q, pn, m[1]);
                    }
                    sum[kSumGate][v].v[i] = fmaf(dr, u, sum[kSumGate][v].v[i]);
                }
                store8<true>(a.dx, row * a.lddx + c, dx);
            }
            float mq = 0.f, mqp = 0.f;
            if constexpr (POST) {
                row_sum<WPR>(m, lds, turn);
                mq = a.post.kind == kNormLayer ? m[0] * inv_c : 0.f, mqp = m[1] * inv_c;
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!on[v]) continue;
                F8 dy;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    dy.v[i] = POST ? rstd_y * (g[v].v[i] - mq - (y[v][i] - mu_y) * rstd_y * mqp) : g[v].v[i];
                store8<F32>(a.dy, row * a.lddy + (v * TPR + t) * 8, dy);
            }
        }
        // the sums over a group's rows: whole, or this segment's share
        const bool whole = p.per_group == 1;
        int k = 0;  // the segment's share: one row of C per sum asked for
        auto to = [&](float *out) -> float * {
            if (out == nullptr) return nullptr;
            return whole ? out + (int64_t)group * a.C : group_ws + ((int64_t)k++ * p.segments() + seg) * a.C;
        };
        flush(kSumGate, to(a.dgate));
        clear(kSumGate);
        if (modulated) {
            flush(kSumMul, to(a.dscale));
            flush(kSumAdd, to(a.dshift));
            clear(kSumMul);
            clear(kSumAdd);
        }
    }
    int k = 0;
    auto to = [&](float *out) -> float * {
        return out == nullptr ? nullptr : row_ws + ((int64_t)k++ * gridDim.x + blockIdx.x) * a.C;
    };
    if (!modulated) {
        flush(kSumMul, to(a.dw));
        flush(kSumAdd, to(a.db));
    }
    if constexpr (POST) flush(kSumPostW, to(a.dpost_w));
    if constexpr (NS > 4) flush(kSumPostB, to(a.dpost_b));
}

// out[j][g][c] = sum over k < n of part[j][g n + k][c], for the outputs asked
// for: workgroup (c / 64, g, j), 64 columns by 16 slices of k.
struct ReduceArgs {
    const float *part;
    float *out[4];
    int32_t n, C;
};
__global__ __launch_bounds__(1024) void residual_norm_reduce_kernel(ReduceArgs a)
{
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    const int64_t g = blockIdx.y, groups = gridDim.y;
    const float *p = a.part + ((int64_t)blockIdx.z * groups + g) * a.n * a.C;
    float s = 0.f;
    if (c < a.C) {
#pragma unroll 8
        for (int k = slice; k < a.n; k += 16) s += p[(int64_t)k * a.C + c];
    }
    lds[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice != 0 || c >= a.C) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x & 63];
    a.out[blockIdx.z][g * a.C + c] = s;
}

template <int NV, int WPR, bool F32>
hipError_t fwd_t(const ResidualNormArgs &a, hipStream_t stream)
{
    const unsigned per = kThreads / (64 * WPR);
    hipLaunchKernelGGL((residual_norm_fwd_kernel<NV, WPR, F32>), dim3((a.rows + per - 1) / per), dim3(kThreads), 0, stream,
                       a);
    return hipGetLastError();
}

template <int NV, int WPR, bool F32>
hipError_t bwd_t(const ResidualNormArgs &a, const ResidualNormPlan &p, float *gws, float *rws, hipStream_t stream)
{
    const dim3 grid((unsigned)p.blocks), block(kThreads);
    if (a.post.kind == kNormNone)
        hipLaunchKernelGGL((residual_norm_bwd_kernel<NV, WPR, F32, 3>), grid, block, 0, stream, a, p, gws, rws);
    else if (a.dpost_b == nullptr)
        hipLaunchKernelGGL((residual_norm_bwd_kernel<NV, WPR, F32, 4>), grid, block, 0, stream, a, p, gws, rws);
    else
        hipLaunchKernelGGL((residual_norm_bwd_kernel<NV, WPR, F32, 5>), grid, block, 0, stream, a, p, gws, rws);
    return hipGetLastError();
}

// f.template operator()<NV, WPR>() for a row of C channels: one wave per row
// up to 2048, four beyond.
template <class F>
hipError_t by_width(int C, const F &f)
{
    if (C <= 512) return f.template operator()<1, 1>();
    if (C <= 1024) return f.template operator()<2, 1>();
    if (C <= 1536) return f.template operator()<3, 1>();
    if (C <= 2048) return f.template operator()<4, 1>();
    if (C <= 4096) return f.template operator()<2, 4>();
    if (C <= 6144) return f.template operator()<3, 4>();
    return f.template operator()<4, 4>();
}

struct Fwd {
    const ResidualNormArgs &a;
    hipStream_t s;
    template <int NV, int WPR>
    hipError_t operator()() const
    {
        return a.f32 ? fwd_t<NV, WPR, true>(a, s) : fwd_t<NV, WPR, false>(a, s);
    }
};
struct Bwd {
    const ResidualNormArgs &a;
    const ResidualNormPlan &p;
    float *gws, *rws;
    hipStream_t s;
    template <int NV, int WPR>
    hipError_t operator()() const
    {
        return a.f32 ? bwd_t<NV, WPR, true>(a, p, gws, rws, s) : bwd_t<NV, WPR, false>(a, p, gws, rws, s);
    }
};

}  // namespace

hipError_t launch_residual_norm_fwd(const ResidualNormArgs &a, hipStream_t stream)
{
    return by_width(a.C, Fwd{a, stream});
}

ResidualNormPlan residual_norm_plan(int rows, int C, int group_rows, int n_cu)
{
    ResidualNormPlan p{};
    p.groups = (rows + group_rows - 1) / group_rows;
    const int at_once = C <= 2048 ? kWaves : 1;  // rows that a workgroup works on at a time
    const int want = 2 * n_cu;
    p.per_group = std::max(1, std::min((want + p.groups - 1) / p.groups, group_rows / (2 * at_once)));
    p.blocks = (int)std::min<int64_t>(p.segments(), want);
    return p;
}

int64_t residual_norm_workspace(const ResidualNormPlan &p, int C, int group_sums, int row_sums)
{
    return ((p.per_group > 1 ? group_sums * p.segments() : 0) + (int64_t)row_sums * p.blocks) * C * (int64_t)sizeof(float);
}

hipError_t launch_residual_norm_bwd(const ResidualNormArgs &a, int n_cu, hipStream_t stream)
{
    const ResidualNormPlan p = residual_norm_plan(a.rows, a.C, a.group_rows, n_cu);
    ReduceArgs group{}, all{};
    int ng = 0, na = 0;
    const bool modulated = a.scale != nullptr;
    // in the kernel's order
    if (p.per_group > 1)
        for (float *o : {a.dgate, modulated ? a.dscale : nullptr, modulated ? a.dshift : nullptr})
            if (o != nullptr) group.out[ng++] = o;
    for (float *o : {modulated ? nullptr : a.dw, modulated ? nullptr : a.db, a.dpost_w, a.dpost_b})
        if (o != nullptr) all.out[na++] = o;
    float *row_ws = a.ws + (int64_t)ng * p.segments() * a.C;
    hipError_t e = by_width(a.C, Bwd{a, p, a.ws, row_ws, stream});
    auto reduce = [&](ReduceArgs &r, const float *part, int n, int groups, int outs) {
        if (e != hipSuccess || outs == 0) return;
        r.part = part, r.n = n, r.C = a.C;
        hipLaunchKernelGGL(residual_norm_reduce_kernel, dim3((unsigned)((a.C + 63) / 64), (unsigned)groups, (unsigned)outs),
                           dim3(1024), 0, stream, r);
        e = hipGetLastError();
    };
    reduce(group, a.ws, p.per_group, p.groups, ng);
    reduce(all, row_ws, p.blocks, 1, na);
    return e;
}

}  // namespace regenvc
