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

// NT: past the caches, as an output that fills them would otherwise be written
// when the kernel ends.  Measured at 10920 x 1536: forward 41.1 us without, 35.4
// with x_out stored so, 37.4 with h, 37.0 with both; backward 68.4 without, 65.8
// with dy stored so, 67.8 with dx, 71.8 with both.
template <bool F32, bool NT = false>
__device__ __forceinline__ void store8(void *p, int64_t at, const F8 &x)
{
    auto put = [](auto *q, auto v) {
        if constexpr (NT)
            __builtin_nontemporal_store(v, q);
        else
            *q = v;
    };
    if constexpr (F32) {
        f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(p) + at);
        put(q, f32x4{x.v[0], x.v[1], x.v[2], x.v[3]});
        put(q + 1, f32x4{x.v[4], x.v[5], x.v[6], x.v[7]});
    } else {
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)x.v[i];
        put(reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(p) + at), o);
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
__device__ __forceinline__ Raw<false> raw_bf16(const uint16_t *p, int at, float missing)
{
    if (p != nullptr) return load_raw<false>(p, at);
    Raw<false> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.a[i] = (__bf16)missing;
    return r;
}
__device__ __forceinline__ F8 vec_bf16(const uint16_t *p, int at, float missing)
{
    const Raw<false> q = raw_bf16(p, at, missing);
    F8 r;
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

// x summed over the wave: four steps within rows of 16 lanes by DPP, two
// exchanges of rows; no LDS.  Every lane gets the sum.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x)
{
    x = dpp_add<0xb1>(x);   // lane ^ 1
    x = dpp_add<0x4e>(x);   // lane ^ 2
    x = dpp_add<0x141>(x);  // 7 - lane, of 8
    x = dpp_add<0x140>(x);  // 15 - lane, of 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(u[0]) + __uint_as_float(u[1]);
}

// Sum over the lanes of a row: its wave, or its workgroup's four waves
// (through LDS; `turn` names the half that this sum uses, so that one barrier
// a sum suffices).
template <int WPR>
__device__ __forceinline__ float row_sum(float s, float (*lds)[kWaves], int &turn)
{
    s = wave_sum(s);
    if constexpr (WPR > 1) {
        float *slot = lds[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = s;
        __syncthreads();
        s = (slot[0] + slot[1]) + (slot[2] + slot[3]);
    }
    return s;
}

// Mean (0 for RMS) and 1/sigma of the row whose values val(v, i) this lane
// holds for v < NV with on[v].
template <int WPR, int NV, class Val>
__device__ __forceinline__ void row_stats(const Val &val, const bool (&on)[NV], int kind, float inv_c, float eps,
                                          float (*lds)[kWaves], int &turn, float &mu, float &rstd)
{
    mu = 0.f;
    if (kind == kNormLayer) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += val(v, i);
        mu = row_sum<WPR>(s, lds, turn) * inv_c;
    }
    float q = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (on[v]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = val(v, i) - mu;
                q = fmaf(d, d, q);
            }
        }
    rstd = rsqrtf(row_sum<WPR>(q, lds, turn) * inv_c + eps);
}

// Forward: WPR waves per row, NV eight-channel chunks per lane.  10920 x 1536,
// norms on both sides, a modulation per 1560 rows, 201 MB: 35 us where two sets of
// rows take turns, 41 with three (5.7 and 4.9 TB/s; a 2 GiB copy: 4.9, so that two
// sets are partly read from the last-level cache); in f32 with three, 268 MB: 60 us
// in a graph of such calls, where bf16 takes 45; one row: 3.6 us.
template <int NV, int WPR, bool F32>
__global__ __launch_bounds__(kThreads) void residual_norm_fwd_kernel(ResidualNormArgs a)
{
    constexpr int TPR = 64 * WPR;  // lanes of a row
    __shared__ float lds[2][kWaves];
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
        store8<true, true>(a.x_out, row * a.ldxo + c, r[v]);
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

// Sums over rows that the backward pass keeps per lane.
enum Sum { kSumGate, kSumMul, kSumAdd, kSumPostW, kSumPostB };

// A row's values of one lane, as loaded.
template <bool F32>
struct RowIn {
    Raw<true> x, gx;
    Raw<F32> y, gh;
};

// What a row's waves tell each other: count, mean and sum of squared
// deviations of their columns (a mean of 0 for RMS norms), or plain sums.
struct Share {
    float v[4];
};

// Mean and 1/sigma of a row from its waves' shares (Chan's combination, exact
// in the mean's square); wave w holds min(512, C - 512 w) columns.
__device__ __forceinline__ void join_stats(const Share *sh, int waves, int C, int at, bool layer, float inv_c, float eps,
                                           float &mu, float &rstd)
{
    float s = 0.f, q = 0.f;
    mu = 0.f;
    if (layer) {
        for (int w = 0; w < waves; ++w) s = fmaf((float)min(512, C - 512 * w), sh[w].v[at], s);
        mu = s * inv_c;
    }
    for (int w = 0; w < waves; ++w) {
        const float d = sh[w].v[at] - mu;
        q += layer ? fmaf((float)min(512, C - 512 * w) * d, d, sh[w].v[at + 1]) : sh[w].v[at + 1];
    }
    rstd = rsqrtf(q * inv_c + eps);
}

// Backward of one row, in the order of the chain rule (m = mean over the C
// channels, n = N_pre(x'), p = N_post(y)):
//     g  = gh (1 + scale)          dr = gx + (g - m(g) - n m(g n)) / sigma
//     dx = alpha dr                du = gate dr         dgate = sum dr u
//     q  = du w_post               dy = (q - m(q) - p m(q p)) / sigma_y
//     dscale, dw = sum gh n        dshift, db = sum gh
//     dpost_w = sum du p           dpost_b = sum du
// (without m(g), m(q) for RMS norms; dy = du without a post-norm).
//
// A row is worked on by W = ceil(C / 512) waves, eight channels per lane, which
// hold the sums over rows, a row's values and the next row's, already requested,
// in 130 to 185 registers a lane: three waves per SIMD with 3 sums or, in bf16,
// 4, otherwise two; a workgroup works on R rows at a time.  The waves
// of a row exchange their shares of its statistics through LDS: of both norms
// in one step, then m(g), m(g n), then m(q), m(q p).  The sums over rows stay
// in registers until a segment ends and are then added over the R rows through
// LDS, in a fixed order: no atomics.  NS: sums held (3, 4 with a post-norm, 5
// with its bias).
// WIDE: more than eight waves, so at most 128 registers a lane.  In bf16 3 sums
// need two more; the others spill, 24 of them (3 sums in f32) to 110 (5), which
// goes through memory beside the rows: 2000 x 8192 with 3, 4 and 5 sums 86, 136
// and 182 us in bf16 (295 MB of rows), 114, 179 and 200 in f32 (393 MB).
// 10920 x 1536 without a post-norm: 59 us, 302 MB, 5.1 TB/s; 1560 x 2048 with
// one: 18.4 us, 57 MB, 3.1: 512 workgroups of three rows, whose sums (12.6 MB)
// come on top.  With the joining launch, three sets of tensors in turn, 10920 x
// 1536 with 3, 4 and 5 sums: 72, 80 and 100 us in bf16, 97, 111 and 114 in f32;
// with a modulation for every row, each of which is then a segment of its own
// with nothing requested ahead of it, 123 and 146 with 3 sums.
template <bool F32, int NS, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 512) __attribute__((amdgpu_waves_per_eu(WIDE ? 4 : NS == 3 ? 3 : 2)))
void residual_norm_bwd_kernel(ResidualNormArgs a, ResidualNormPlan p, float *group_ws,
                                                                 float *row_ws)
{
    constexpr bool POST = NS > 3;
    __shared__ Share share[3][16];
    __shared__ __attribute__((aligned(16))) float stage[8 * 512];
    const int W = p.row_waves, R = p.rows_at_once;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slot = wave / W, rw = wave - slot * W;  // which of the R rows, which wave of it
    const int c = rw * 512 + lane * 8;
    const bool on = c < a.C;
    const float inv_c = 1.0f / (float)a.C, inv_n = 1.0f / (float)min(512, a.C - 512 * rw);
    const bool modulated = a.scale != nullptr, pre_layer = a.pre.kind == kNormLayer, post_layer = a.post.kind == kNormLayer;

    F8 sum[NS] = {};
    // the workgroup's sum s to out [C] (null: dropped)
    auto flush = [&](int s, float *out) {
        if (out == nullptr) return;
        if (R > 1) {
            __syncthreads();
            store8<true>(stage, (slot * W + rw) * 512 + lane * 8, sum[s]);
            __syncthreads();
            for (int k = threadIdx.x; k < a.C; k += blockDim.x) {
                float z = stage[k];
                for (int j = 1; j < R; ++j) z += stage[j * W * 512 + k];
                out[k] = z;
            }
        } else if (on) {
            store8<true>(out, c, sum[s]);
        }
    };
    auto load = [&](RowIn<F32> &in, int64_t row, bool valid) {
        in = RowIn<F32>{};
        if (!valid || !on) return;
        in.x = load_raw<true>(a.x, row * a.ldx + c);
        in.gh = load_raw<F32>(a.gh, row * a.ldgh + c);
        in.y = load_raw<F32>(a.y, row * a.ldy + c);
        if (a.gx != nullptr) in.gx = load_raw<true>(a.gx, row * a.ldgx + c);
    };
    // this wave's count-free share of a row's statistics
    auto wave_stats = [&](const auto &v, bool layer, float &mean, float &dev) {
        mean = 0.f;
        if (layer) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
            mean = wave_sum(s) * inv_n;
        }
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = v[i] - mean;
            q = fmaf(d, d, q);
        }
        dev = wave_sum(on ? q : 0.f);
    };

    for (int64_t seg = blockIdx.x; seg < p.segments(); seg += gridDim.x) {
        const int group = (int)(seg / p.per_group), part = (int)(seg % p.per_group);
        const int64_t gr0 = (int64_t)group * a.group_rows;
        const int64_t n = min((int64_t)a.group_rows, a.rows - gr0);
        const int64_t r0 = gr0 + n * part / p.per_group, r1 = gr0 + n * (part + 1) / p.per_group;
        const int64_t gv = (int64_t)group * a.ldv;
        RowIn<F32> next;
        load(next, r0 + slot, r0 + slot < r1);
        // the vectors stay in registers too: a load of them within a row would wait, as loads return in order, for the
        // next row's
        F8 mul{}, gate{};
        Raw<false> pw{}, pb{};
        if (on) {
            mul = pre_mul(a, gv, c);
            gate = vec_f32(a.gate, gv + c, 1.f);
            if constexpr (POST) pw = raw_bf16(a.post.w, c, 1.f), pb = raw_bf16(a.post.b, c, 0.f);
        }
        for (int64_t rr = r0; rr < r1; rr += R) {  // the same number of rounds, and of barriers, for all R rows
            const int64_t row = rr + slot;
            const bool valid = row < r1;
            const RowIn<F32> in = next;
            load(next, row + R, row + R < r1);
            // statistics of both norms
            Share mine{};
            wave_stats(in.x, pre_layer, mine.v[0], mine.v[1]);
            if constexpr (POST) wave_stats(in.y, post_layer, mine.v[2], mine.v[3]);
            float mu, rstd, mu_y = 0.f, rstd_y = 1.f;
            if (W > 1) {
                if (lane == 0) share[0][wave] = mine;
                __syncthreads();
            }
            if (W > 1) {
                join_stats(share[0] + slot * W, W, a.C, 0, pre_layer, inv_c, a.pre.eps, mu, rstd);
                if constexpr (POST) join_stats(share[0] + slot * W, W, a.C, 2, post_layer, inv_c, a.post.eps, mu_y, rstd_y);
            } else {
                mu = mine.v[0], rstd = rsqrtf(mine.v[1] * inv_c + a.pre.eps);
                if constexpr (POST) mu_y = mine.v[2], rstd_y = rsqrtf(mine.v[3] * inv_c + a.post.eps);
            }
            // m(g), m(g n)
            F8 g{};
            float m0 = 0.f, m1 = 0.f;
            if (on && valid) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float nn = (in.x[i] - mu) * rstd;
                    g.v[i] = in.gh[i] * mul.v[i];
                    m0 += g.v[i];
                    m1 = fmaf(g.v[i], nn, m1);
                    sum[kSumMul].v[i] = fmaf(in.gh[i], nn, sum[kSumMul].v[i]);
                    sum[kSumAdd].v[i] += in.gh[i];
                }
            }
            auto row_means = [&](int buf) {  // m0, m1 summed over the row, times 1 / C
                m0 = wave_sum(m0), m1 = wave_sum(m1);
                if (W > 1) {
                    if (lane == 0) share[buf][wave].v[0] = m0, share[buf][wave].v[1] = m1;
                    __syncthreads();
                    m0 = m1 = 0.f;
                    for (int w = 0; w < W; ++w) m0 += share[buf][slot * W + w].v[0], m1 += share[buf][slot * W + w].v[1];
                }
                m0 *= inv_c, m1 *= inv_c;
            };
            row_means(1);
            const float mg = pre_layer ? m0 : 0.f, mgn = m1;
            m0 = m1 = 0.f;
            if (on && valid) {
                F8 dx;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float nn = (in.x[i] - mu) * rstd;
                    const float dr = in.gx[i] + rstd * (g.v[i] - mg - nn * mgn);
                    dx.v[i] = a.alpha * dr;
                    const float du = gate.v[i] * dr;
                    float u = in.y[i];
                    g.v[i] = du;
                    if constexpr (POST) {
                        const float pn = (u - mu_y) * rstd_y;
                        u = fmaf(pn, pw[i], pb[i]);
                        sum[kSumPostW].v[i] = fmaf(du, pn, sum[kSumPostW].v[i]);
                        if constexpr (NS > 4) sum[kSumPostB].v[i] += du;
                        g.v[i] = du * pw[i];
                        m0 += g.v[i];
                        m1 = fmaf(g.v[i], pn, m1);
                    }
                    sum[kSumGate].v[i] = fmaf(dr, u, sum[kSumGate].v[i]);
                }
                store8<true>(a.dx, row * a.lddx + c, dx);
            }
            float mq = 0.f, mqp = 0.f;
            if constexpr (POST) {
                row_means(2);
                mq = post_layer ? m0 : 0.f, mqp = m1;
            }
            if (on && valid) {
                F8 dy;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    dy.v[i] = POST ? rstd_y * (g.v[i] - mq - (in.y[i] - mu_y) * rstd_y * mqp) : g.v[i];
                store8<F32, true>(a.dy, row * a.lddy + c, dy);
            }
            // without a post-norm the first exchange of the next row lies one barrier behind the last read of this
            // one's share[0], as with one
        }
        // the sums over a group's rows: whole, or this segment's share
        const bool whole = p.per_group == 1;
        int k = 0;  // the segment's share: one row of C per sum asked for
        auto to = [&](float *out) -> float * {
            if (out == nullptr) return nullptr;
            return whole ? out + (int64_t)group * a.C : group_ws + ((int64_t)k++ * p.segments() + seg) * a.C;
        };
        flush(kSumGate, to(a.dgate));
        sum[kSumGate] = F8{};
        if (modulated) {
            flush(kSumMul, to(a.dscale));
            flush(kSumAdd, to(a.dshift));
            sum[kSumMul] = sum[kSumAdd] = F8{};
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

// The sums of segments and workgroups joined, in order: workgroup (c / 64, y)
// adds, for job y, n rows of C that lie behind one another; 64 columns by 16
// slices of the rows.  Jobs: for each sum over a group's rows and each group,
// then for each sum over all rows.  4 to 5 us, most of it a launch.
struct ReduceArgs {
    const float *group_part, *row_part;
    float *group_out[3], *row_out[4];
    int32_t groups, group_jobs, group_n, row_n, C;
};
__global__ __launch_bounds__(1024) void residual_norm_reduce_kernel(ReduceArgs a)
{
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    const int job = blockIdx.y, rj = job - a.group_jobs;
    const bool grouped = rj < 0;
    const int n = grouped ? a.group_n : a.row_n;
    const float *p = grouped ? a.group_part + (int64_t)job * n * a.C : a.row_part + (int64_t)rj * n * a.C;
    float *out = grouped ? a.group_out[job / a.groups] + (int64_t)(job % a.groups) * a.C : a.row_out[rj];
    float s = 0.f;
    if (c < a.C) {
#pragma unroll 8
        for (int k = slice; k < n; k += 16) s += p[(int64_t)k * a.C + c];
    }
    lds[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice != 0 || c >= a.C) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x & 63];
    out[c] = s;
}

template <int NV, int WPR, bool F32>
hipError_t fwd_t(const ResidualNormArgs &a, hipStream_t stream)
{
    const unsigned per = kThreads / (64 * WPR);
    hipLaunchKernelGGL((residual_norm_fwd_kernel<NV, WPR, F32>), dim3((a.rows + per - 1) / per), dim3(kThreads), 0, stream,
                       a);
    return hipGetLastError();
}

template <bool F32, bool WIDE>
hipError_t bwd_t(const ResidualNormArgs &a, const ResidualNormPlan &p, float *gws, float *rws, hipStream_t stream)
{
    const dim3 grid((unsigned)p.blocks), block(64 * p.row_waves * p.rows_at_once);
    if (a.post.kind == kNormNone)
        hipLaunchKernelGGL((residual_norm_bwd_kernel<F32, 3, WIDE>), grid, block, 0, stream, a, p, gws, rws);
    else if (a.dpost_b == nullptr)
        hipLaunchKernelGGL((residual_norm_bwd_kernel<F32, 4, WIDE>), grid, block, 0, stream, a, p, gws, rws);
    else
        hipLaunchKernelGGL((residual_norm_bwd_kernel<F32, 5, WIDE>), grid, block, 0, stream, a, p, gws, rws);
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
}  // namespace

hipError_t launch_residual_norm_fwd(const ResidualNormArgs &a, hipStream_t stream)
{
    return by_width(a.C, Fwd{a, stream});
}

ResidualNormPlan residual_norm_plan(int rows, int C, int group_rows, int n_cu)
{
    ResidualNormPlan p{};
    p.groups = (int)(((int64_t)rows + group_rows - 1) / group_rows);
    p.row_waves = (C + 511) / 512;
    p.rows_at_once = std::max(1, 4 / p.row_waves);
    // Workgroups per compute unit: as many as its registers hold, for the more rows are under way the better memory
    // latency passes, but each costs a row per sum in the workspace: a third one pays from 8 rows per workgroup on
    // (10920 rows of 1536 channels: 106, 65 and 63 us with one, two and three; 1560 of 2048: 23, 18 and 20).  Measured
    // with 3 sums in bf16; the forms with 5 sums, and those in f32 with a post-norm, have registers for two, and the
    // third's rows come in a second round (the times at the kernel), for what a plan goes by is rows and channels only.
    const int64_t per_cu = p.row_waves > 4 ? 1 : p.row_waves <= 3 && rows >= 24 * (int64_t)n_cu ? 3 : 2;
    const int64_t want = per_cu * n_cu;
    p.per_group = (int)std::max<int64_t>(1, std::min<int64_t>(want / p.groups, group_rows / p.rows_at_once));
    p.blocks = (int)std::min(p.segments(), want);
    return p;
}

int64_t residual_norm_workspace(const ResidualNormPlan &p, int C, int group_sums, int row_sums)
{
    return ((p.per_group > 1 ? group_sums * p.segments() : 0) + (int64_t)row_sums * p.blocks) * C * (int64_t)sizeof(float);
}

hipError_t launch_residual_norm_bwd(const ResidualNormArgs &a, int n_cu, hipStream_t stream)
{
    const ResidualNormPlan p = residual_norm_plan(a.rows, a.C, a.group_rows, n_cu);
    ReduceArgs r{};
    int ng = 0, na = 0;
    const bool modulated = a.scale != nullptr;
    // in the kernel's order
    if (p.per_group > 1)
        for (float *o : {a.dgate, modulated ? a.dscale : nullptr, modulated ? a.dshift : nullptr})
            if (o != nullptr) r.group_out[ng++] = o;
    for (float *o : {modulated ? nullptr : a.dw, modulated ? nullptr : a.db, a.dpost_w, a.dpost_b})
        if (o != nullptr) r.row_out[na++] = o;
    float *row_ws = a.ws + (int64_t)ng * p.segments() * a.C;
    const bool wide = p.row_waves > 8;
    const hipError_t e = a.f32 ? (wide ? bwd_t<true, true>(a, p, a.ws, row_ws, stream) : bwd_t<true, false>(a, p, a.ws, row_ws, stream))
                               : (wide ? bwd_t<false, true>(a, p, a.ws, row_ws, stream) : bwd_t<false, false>(a, p, a.ws, row_ws, stream));
    if (e != hipSuccess || ng + na == 0) return e;
    r.group_part = a.ws, r.row_part = row_ws;
    r.groups = p.groups, r.group_jobs = ng * p.groups, r.group_n = p.per_group, r.row_n = p.blocks, r.C = a.C;
    hipLaunchKernelGGL(residual_norm_reduce_kernel, dim3((unsigned)((a.C + 63) / 64), (unsigned)(r.group_jobs + na)),
                       dim3(1024), 0, stream, r);
    return hipGetLastError();
}

}  // namespace regenvc
