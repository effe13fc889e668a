// gfx950 kernels around a bf16 key/value cache in pages: the append that norms
// and rotates, the mean keys of pages, and the choice of pages by their score.
#include <algorithm>

#include "paged_device.hpp"

namespace regenvc {
namespace paged {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));  // eight bf16, the first of a pair in the low half
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
// Rounded once: through an f32 in between, a number next to the middle of two bf16 could go the wrong way.
__device__ __forceinline__ uint16_t bf16_of(double x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ u32x4 load16(const uint16_t *p)
{
    return *reinterpret_cast<const u32x4 *>(p);
}

// ---------------------------------------------------------------- append
// x summed over the D / 8 lanes that hold a head (each gets the result).
template <int LPH>
__device__ __forceinline__ float head_sum(float x)
{
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kXor1, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kXor2, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kMirror8, 0xf, 0xf, true));
    if (LPH == 16) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kRotate8, 0xf, 0xf, true));
    return x;
}

// HBM-bound: every channel is read once and written once.  A workgroup takes the
// new tokens of one stretch of up to 64 places within a page; pairs of its waves take the
// heads of q, k and v, which follow one another, 64 / (D / 8) of them at a time (16
// bytes a lane), through all of its tokens, four in flight.  Sines and cosines of
// the stretch are formed once, in LDS; the angles in 64 bits before the whole turns
// are taken off: at place 2^20 an f32 product would be off by 0.06 rad.  The halves
// layout pairs a lane with one rot / 16 lanes on, whose channels come by lane
// exchange.
//
// Mean keys: where a page is no longer than a stretch, the waves that have a key head
// have all that the page's mean takes; the tokens that were there before they read
// back.  Sums of bf16 values in 64 bits are exact for all but absurd spreads, so
// the mean does not depend on how the tokens came.  It is rounded to bf16, as the
// keys that it stands for: a score then reads 1 / (2 page) of the places' bytes.
//
// Stretches of sequence b are numbered from first[b] / 64 + 2 b: n tokens touch at
// most n / 64 + 2.  Tokens before place 0 are in stretches below 0: only q is written.
//
// 10920 tokens of 36 heads of 128, normed, rotated and with means (201 MB): 48 us, 4.2
// TB/s (a copy: 5.1); without means and rotation 44.  A token with 39 older keys in
// its page: 7.5 us.  One wave to a group of heads instead of two: 57 us, 129 registers
// instead of 128: 56.
constexpr int kStretch = 6, kInFlight = 4;

// Rows r, r + step, ... below `rows` of a page's head added to sum.
__device__ __forceinline__ void add_rows(double (&sum)[8], const uint16_t *k, int D, int r, int step, int rows)
{
    for (; r < rows; r += 8 * step) {
        u32x4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = load16(k + min(r + j * step, rows - 1) * D);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (r + j * step >= rows) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[2 * e] += (double)lo(x[j][e]), sum[2 * e + 1] += (double)hi(x[j][e]);
        }
    }
}

template <int D>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) void append_kernel(AppendArgs a)
{
    constexpr int LPH = D / 8, HPW = 64 / LPH, S = 1 << kStretch;
    // A token's cosines, then its sines of both signs, times the amplitude.  The two sines are read together, by the two
    // halves of a head: four banks apart.
    constexpr int NEG = D / 2, POS = D + 4, ROW = 3 * D / 2 + 8;
    __shared__ f32x4 turn[S][ROW / 4];
    __shared__ double part[4][64][8];  // sums of keys, of the second wave of each pair
    const int tid = threadIdx.x, lane = tid & 63, sub = lane / LPH, d0 = lane % LPH * 8;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), s = min(a.c.shift, kStretch);
    const int b = last_from(a.n.B, blockIdx.x, [&](int i) { return (int64_t)(first_of(a.n, i) >> s) + 2 * i; });
    if (b < 0) return;
    const int f0 = first_of(a.n, b), rows = first_of(a.n, b + 1) - f0, len = max(0, a.n.lens[b]), start = len - rows;
    const int64_t at = ((int64_t)(start >> s) + (int64_t)blockIdx.x - (f0 >> s) - 2 * b) << s;  // the stretch's first place
    const int begin = (int)max((int64_t)start, at), count = (int)(min((int64_t)len, at + (1 << s)) - begin);
    if (count <= 0) return;
    const int row0 = f0 + (begin - start);
    const int64_t col = at >> a.c.shift;
    int page = -1;
    if (at >= 0 && col < a.n.columns) page = a.n.table[b * a.n.table_stride + col];
    const bool stored = page >= 0 && page < a.c.pages;
    const int in_page = begin & ((1 << a.c.shift) - 1);
    const bool mean = a.c.means != nullptr && a.c.shift <= kStretch && stored;
    const int total = a.H + 2 * a.c.heads, keys0 = a.H, keys1 = a.H + a.c.heads;
    const int64_t page0 = (int64_t)max(page, 0) * a.c.heads;
    const int pairs = a.pairs, rot = 2 * pairs;
    for (int i = tid; i < count * pairs; i += 512) {
        const int t = i / pairs, p = i - t * pairs;
        const float x = (float)__builtin_amdgcn_fract((double)(begin + t) * a.turns[p]);
        const float sine = a.amplitude * __builtin_amdgcn_sinf(x);
        float *row = reinterpret_cast<float *>(turn[t]);
        row[p] = a.amplitude * __builtin_amdgcn_cosf(x);
        row[NEG + p] = -sine;
        row[POS + p] = sine;
    }
    __syncthreads();

    const bool turned = d0 < rot;
    const int partner = a.interleaved ? lane : d0 < pairs ? lane + pairs / 8 : lane - pairs / 8;  // in the same head
    const int p0 = !turned ? 0 : a.interleaved ? d0 / 2 : d0 < pairs ? d0 : d0 - pairs;  // the first of this lane's pairs
    const int sine0 = (d0 < pairs ? NEG : POS) + p0;  // in the halves layout
    const bool whole = LPH == 16 && rot == D;         // then a lane's partner is 8 lanes on
    // a pair of waves to a group of heads, for every other batch of tokens
    const int pair = wave >> 1, second = wave & 1;
    for (int g0 = 4 * blockIdx.y; g0 * HPW < total; g0 += 4 * gridDim.y) {
        const int g = g0 + pair;
        const int h = min(g * HPW + sub, total - 1);
        const bool live = g * HPW + sub < total;
        const bool is_q = h < keys0, is_k = !is_q && h < keys1;
        const int hk = is_k ? h - keys0 : h - keys1;  // of k and v
        const uint16_t *src = d0 + (is_q ? a.q + h * a.q_sh : is_k ? a.k + hk * a.k_sh : a.v + hk * a.v_sh);
        const int64_t ss = is_q ? a.q_ss : is_k ? a.k_ss : a.v_ss;
        const int64_t cell = (page0 + hk) << a.c.shift;
        uint16_t *dst = d0 + (is_q ? a.q_out + row0 * a.o_ss + h * a.o_sh : (is_k ? a.c.k : a.c.v) + (cell + in_page) * D);
        const int64_t ds = is_q ? a.o_ss : D;
        const bool store = live && (is_q || stored), only_v = g * HPW >= keys1;
        const uint16_t *weight = is_q ? a.w_q : is_k ? a.w_k : nullptr;
        const bool norm = weight != nullptr, turns = turned && (is_q || is_k), sums = mean && is_k;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.f;
        if (norm) {
            const u32x4 x = load16(weight + d0);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[2 * e] = lo(x[e]), w[2 * e + 1] = hi(x[e]);
        }
        double sum[8] = {};
        if (sums && live) add_rows(sum, a.c.k + cell * D + d0, D, second, 2, in_page);
        u32x4 next[kInFlight];
        auto load = [&](int t0) {  // past the last token that again
#pragma unroll
            for (int j = 0; j < kInFlight; ++j) next[j] = load16(src + (row0 + min(t0 + j, count - 1)) * ss);
        };
        const int end = g * HPW < total ? count : 0;
        if (second * kInFlight < end) load(second * kInFlight);
        for (int t0 = second * kInFlight; t0 < end; t0 += 2 * kInFlight) {
            u32x4 x[kInFlight];
#pragma unroll
            for (int j = 0; j < kInFlight; ++j) x[j] = next[j];
            load(t0 + 2 * kInFlight);
#pragma unroll
            for (int j = 0; j < kInFlight; ++j) {
                const int t = t0 + j;
                if (t >= count) break;
                u32x4 o = x[j];
                if (!only_v) {
                    float q = 0.f, y[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[2 * e] = lo(x[j][e]), y[2 * e + 1] = hi(x[j][e]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) q = fmaf(y[e], y[e], q);
                    // the mean by a product: D is a power of two
                    const float r = __builtin_amdgcn_rsqf(fmaf(head_sum<LPH>(q), 1.0f / D, a.eps));
                    if (norm) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = y[e] * r * w[e];
                    }
                    if (rot > 0) {
                        float f[8];
                        if (a.interleaved) {
                            const f32x4 c = turn[t][p0 / 4], neg = turn[t][(NEG + p0) / 4], pos = turn[t][(POS + p0) / 4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                f[2 * e] = fmaf(y[2 * e + 1], neg[e], y[2 * e] * c[e]);
                                f[2 * e + 1] = fmaf(y[2 * e], pos[e], y[2 * e + 1] * c[e]);
                            }
                        } else {
                            float z[8];
                            if (whole) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) z[e] = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(y[e]), kRotate8, 0xf, 0xf, true));
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], partner, 64);
                            }
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const f32x4 c = turn[t][p0 / 4 + i], v = turn[t][sine0 / 4 + i];
#pragma unroll
                                for (int e = 0; e < 4; ++e) f[4 * i + e] = fmaf(z[4 * i + e], v[e], y[4 * i + e] * c[e]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = turns ? f[e] : y[e];
                    }
                    if (is_q || is_k) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = pack(y[2 * e], y[2 * e + 1]);
                    }
                    if (sums) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[2 * e] += (double)lo(o[e]), sum[2 * e + 1] += (double)hi(o[e]);
                    }
                }
                if (store) *reinterpret_cast<u32x4 *>(dst + t * ds) = o;
            }
        }
        if (!mean) continue;  // the same for all waves
        if (second) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[pair][lane][e] = sum[e];
        }
        __syncthreads();
        if (sums && live && !second) {
            const double n = in_page + count;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += part[pair][lane][e];
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = bf16_of(sum[2 * e] / n) | (uint32_t)bf16_of(sum[2 * e + 1] / n) << 16;
            *reinterpret_cast<u32x4 *>(a.c.means + (page0 + hk) * D + d0) = o;
        }
        __syncthreads();
    }
}

// Mean keys of longer pages, from the pages as the append left them: a workgroup
// per page that the call's new tokens touch and head.  Pages of sequence b are
// numbered as the stretches are.
template <int D>
__global__ __launch_bounds__(256) void means_kernel(AppendArgs a)
{
    constexpr int LPR = D / 8, RPP = 256 / LPR;
    __shared__ double part[RPP][D];
    const int hk = blockIdx.y, page_size = 1 << a.c.shift;
    const int b = last_from(a.n.B, blockIdx.x, [&](int i) { return (int64_t)(first_of(a.n, i) >> a.c.shift) + 2 * i; });
    if (b < 0) return;
    const int f0 = first_of(a.n, b), f1 = first_of(a.n, b + 1), len = max(0, a.n.lens[b]);
    if (f1 <= f0) return;
    const int start = len - (f1 - f0);  // may be negative: tokens before place 0 are not stored
    const int64_t col = (max(start, 0) >> a.c.shift) + (int64_t)blockIdx.x - (f0 >> a.c.shift) - 2 * b;
    if (col >= a.n.columns || col << a.c.shift >= len) return;
    const int page = a.n.table[b * a.n.table_stride + col];
    if (page < 0 || page >= a.c.pages) return;
    const int rows = min(page_size, len - (int)(col << a.c.shift));
    const int d0 = threadIdx.x % LPR * 8, r0 = threadIdx.x / LPR;
    const uint16_t *k = a.c.k + ((int64_t)page * a.c.heads + hk) * (D << a.c.shift) + d0;
    double s[8] = {};
    for (int r = r0; r < rows; r += RPP) {
        const u32x4 x = load16(k + r * D);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[2 * e] += (double)lo(x[e]), s[2 * e + 1] += (double)hi(x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[r0][d0 + e] = s[e];
    __syncthreads();
    if (threadIdx.x >= D) return;
    double sum = 0;
#pragma unroll
    for (int r = 0; r < RPP; ++r) sum += part[r][threadIdx.x];
    a.c.means[((int64_t)page * a.c.heads + hk) * D + threadIdx.x] = bf16_of(sum / rows);
}

// ---------------------------------------------------------------- selection
// A score as a number whose unsigned order is the scores'.
__device__ __forceinline__ uint64_t order_of(double s)
{
    if (s != s) s = -__builtin_inf();
    s = fmin(s, 1.7976931348623157e308) + 0.0;  // -0 as 0; +inf stays below the pages that are always taken
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}
constexpr uint64_t kTaken = ~(uint64_t)0;

template <int CTRL>
__device__ __forceinline__ double from_lane(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t l = __builtin_amdgcn_mov_dpp((int)u, CTRL, 0xf, 0xf, true);
    const uint32_t h = __builtin_amdgcn_mov_dpp((int)(u >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)h << 32 | l);
}
// x summed over the four rows of 16 lanes.
__device__ __forceinline__ double rows_sum(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const auto l = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
    const auto h = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    const double y = __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
    const uint64_t v = __builtin_bit_cast(uint64_t, y);
    const auto m = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto n = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    return __builtin_bit_cast(double, (uint64_t)n[0] << 32 | m[0]) + __builtin_bit_cast(double, (uint64_t)n[1] << 32 | m[1]);
}
// Of 2 n sums spread over pairs of lanes, those that this lane keeps (`upper`: the last n), with its partner's part.
template <int CTRL, int N>
__device__ __forceinline__ void keep_half(double (&x)[N], int n, bool upper)
{
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        if (j >= n) break;
        const double mine = upper ? x[j + n] : x[j], other = upper ? x[j] : x[j + n];
        x[j] = mine + from_lane<CTRL>(other);
    }
}
// Eight sums spread over the D / 8 lanes that hold a row: each lane gets one of them, that of number `which`.
template <int LPR>
__device__ __forceinline__ double share_out(double (&x)[8], int &which)
{
    const int l = threadIdx.x;
    if constexpr (LPR == 16) {
        keep_half<kRotate8>(x, 4, l & 8);
        keep_half<kMirror8>(x, 2, l & 4);
        keep_half<kXor2>(x, 1, l & 2);
        which = (l & 8 ? 4 : 0) + (l & 4 ? 2 : 0) + (l & 2 ? 1 : 0);
        return x[0] + from_lane<kXor1>(x[0]);
    } else {
        keep_half<kMirror8>(x, 4, l & 4);
        keep_half<kXor2>(x, 2, l & 2);
        keep_half<kXor1>(x, 1, l & 1);
        which = (l & 4 ? 4 : 0) + (l & 2 ? 2 : 0) + (l & 1 ? 1 : 0);
        return x[0];
    }
}

// A workgroup per block of queries and key head.  The sum of the block's
// queries and the scores are taken in 64 bits, so that the choice is that of
// the exact scores: in 32, two pages whose scores lie within 2^-22 of one another
// would go by the order of summation.  D / 8 lanes share a page's mean, kAtOnce
// of them in flight.  The count-th largest score is found digit by digit from the
// highest in which any differ, eight bits a pass over the scores in LDS, until a
// digit splits none that are left.  One query, 16 of 512 pages for each of 12 heads:
// 10.9 us, of 25000 cycles 2000 for the sequence, 5500 for pages, queries and means,
// 8000 for the products (64-bit operations take eight cycles), 4000 for the digits.
constexpr int kAtOnce = 8;

template <int D, int THREADS>
__global__ __launch_bounds__(THREADS) void select_kernel(SelectArgs a)
{
    constexpr int LPR = D / 8, RPP = THREADS / LPR;
    constexpr int WAVES = THREADS / 64;
    extern __shared__ uint64_t key[];
    __shared__ double part[WAVES][D], qsum[D];
    __shared__ uint32_t hist[256];
    __shared__ uint64_t prefix_s;
    __shared__ uint32_t bound[WAVES][2];
    __shared__ int taken_s[WAVES][2];
    __shared__ int left_s, done_s;
    static_assert(sizeof(part) + sizeof(qsum) + sizeof(hist) + sizeof(bound) + sizeof(taken_s) + 64 + kMaxSelectColumns * sizeof(uint64_t) <= 160 * 1024,
                  "the scores of the largest call and the rest fit the LDS");
    const int hk = blockIdx.y, tid = threadIdx.x, G = a.H / a.c.heads;
    int32_t *out = a.selected + ((int64_t)blockIdx.x * a.c.heads + hk) * a.count;
    const Block k = block_of(a.n, a.c.shift, a.q_block, blockIdx.x);
    const int end = k.rows == 0 ? 0 : a.causal ? max(0, k.pos + k.rows) : k.len;
    const int seen = (end + (1 << a.c.shift) - 1) >> a.c.shift;  // candidates; at most the columns
    if (seen <= a.count) {
        for (int i = tid; i < a.count; i += THREADS) out[i] = i < seen ? i : -1;
        return;
    }
    const int d0 = tid % LPR * 8, r0 = tid / LPR;
    const int32_t *pages = a.n.table + k.b * a.n.table_stride;
    auto lookup = [&](int p0, int (&at)[kAtOnce]) {  // the pool's pages of this lane's candidates from p0 on, -1 for none
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int p = p0 + j * RPP + r0;
            at[j] = pages[min(p, seen - 1)];
            if (p >= seen || at[j] >= a.c.pages) at[j] = -1;
        }
    };
    int at[kAtOnce];
    u32x4 x[kAtOnce];
    bool there[kAtOnce];
    auto load = [&](const int (&at)[kAtOnce]) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            there[j] = at[j] >= 0;
            x[j] = u32x4{0, 0, 0, 0};
            if (there[j]) x[j] = load16(a.c.means + ((int64_t)at[j] * a.c.heads + hk) * D + d0);
        }
    };
    lookup(0, at);
    {
        double s[8] = {};
        const int rows = k.rows * G;  // at most H T, which is at most 2^29
        for (int r = r0; r < rows; r += 4 * RPP) {
            u32x4 y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // past the last row that again, with no part in the sum
                const int i = min(r + j * RPP, rows - 1), query = i / G;
                y[j] = load16(a.q + (int64_t)(k.row + query) * a.q_ss + (int64_t)(hk * G + i - query * G) * a.q_sh + d0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (r + j * RPP >= rows) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[2 * e] += (double)lo(y[j][e]), s[2 * e + 1] += (double)hi(y[j][e]);
            }
        }
        load(at);  // in flight until the queries' sum is there
        // over the rows that a wave has at once, then over the waves
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (LPR == 8) s[e] += from_lane<kRotate8>(s[e]);
            s[e] = rows_sum(s[e]);
            if ((tid & 63) < LPR) part[tid >> 6][d0 + e] = s[e];
        }
    }
    __syncthreads();
    if (tid < D) {
        double sum = 0;
#pragma unroll
        for (int r = 0; r < WAVES; ++r) sum += part[r][tid];
        qsum[tid] = sum;
    }
    __syncthreads();
    double qs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) qs[e] = qsum[d0 + e];
    uint32_t low = 0, high = 0;
    for (int p0 = 0; p0 < seen; p0 += RPP * kAtOnce) {
        double sum[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            sum[j] = there[j] ? 0.0 : -__builtin_inf();
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[j] = fma(qs[2 * e], (double)lo(x[j][e]), fma(qs[2 * e + 1], (double)hi(x[j][e]), sum[j]));
        }
        if (p0 + RPP * kAtOnce < seen) {
            lookup(p0 + RPP * kAtOnce, at);
            load(at);
        }
        int j;
        const double score = share_out<LPR>(sum, j);
        const int p = p0 + j * RPP + r0;
        if (p < seen) {
            const uint64_t v = p < a.keep_first || p >= seen - a.keep_last ? kTaken : order_of(score);
            key[p] = v;
            // of their upper halves, the least and the most: of the pages always taken, neither
            if (v != kTaken) low = max(low, ~(uint32_t)(v >> 32)), high = max(high, (uint32_t)(v >> 32));
        }
    }
    // Digits from the highest bit in which the scores' upper halves differ: those with key >> shift above `prefix` are
    // taken, `left` of those equal to it.
    low = wave_max(low), high = wave_max(high);
    if ((tid & 63) == 0) bound[tid >> 6][0] = low, bound[tid >> 6][1] = high;
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) low = max(low, bound[i][0]), high = max(high, bound[i][1]);
    low = ~low;
    const int kept = a.keep_first + a.keep_last;  // at most count, and fewer than the candidates
    int left = a.count - kept;
    int shift = low == high ? 32 : 64 - __builtin_clz(low ^ high);
    uint64_t prefix = shift >= 64 ? 0 : (uint64_t)high >> (shift - 32);
    bool done = left == 0;  // the pages always taken are all
    if (done) shift = 0, prefix = kTaken - 1;
    while (!done && shift > 0) {
        const int bits = min(shift, 8);
        shift -= bits;
        for (int p = tid; p < seen; p += THREADS) {
            const uint64_t v = key[p];
            if (v != kTaken && (shift + bits >= 64 || v >> (shift + bits) == prefix))
                atomicAdd(&hist[(v >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        if (tid < 64) {  // lane i has the digits 255 - 4 i .. 252 - 4 i
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = hist[255 - 4 * tid - i], hist[255 - 4 * tid - i] = 0, sum += c[i];
            const uint32_t upto = wave_upto(sum);
            uint32_t above = upto - sum;
            if (above < (uint32_t)left && upto >= (uint32_t)left) {  // one lane: the digit of the last one taken is here
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (above < (uint32_t)left && above + c[i] >= (uint32_t)left) {
                        prefix_s = prefix << bits | (uint64_t)(255 - 4 * tid - i);
                        left_s = left - (int)above;
                        done_s = (int)c[i] == left - (int)above;
                        break;
                    }
                    above += c[i];
                }
            }
        }
        __syncthreads();
        prefix = prefix_s, left = left_s, done = done_s != 0;
    }
    // In order of the pages; of equal scores the first `left`.  Every wave counts those of its stretch of pages, then puts
    // them where those before it end.
    const int wave = tid >> 6, lane = tid & 63, stretch = ((seen + WAVES - 1) / WAVES + 63) & ~63;
    const int first = min(seen, wave * stretch), last = min(seen, first + stretch);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    auto look = [&](int p, bool &above, bool &equal) {
        const uint64_t full = p < last ? key[p] : 0;
        above = p < last && (full == kTaken || full >> shift > prefix);
        equal = p < last && !above && full >> shift == prefix;
    };
    int n_above = 0, n_equal = 0;
    for (int p = first; p < last; p += 64) {
        bool above, equal;
        look(p + lane, above, equal);
        n_above += __popcll(__builtin_amdgcn_ballot_w64(above));
        n_equal += __popcll(__builtin_amdgcn_ballot_w64(equal));
    }
    if (lane == 0) taken_s[wave][0] = n_above, taken_s[wave][1] = n_equal;
    __syncthreads();
    int n = 0;
    for (int i = 0; i < wave; ++i) {
        const int e = min(taken_s[i][1], left);
        n += taken_s[i][0] + e;
        left -= e;
    }
    for (int p = first; p < last; p += 64) {
        bool above, equal;
        look(p + lane, above, equal);
        const uint64_t eq = __builtin_amdgcn_ballot_w64(equal);
        const bool take = above || (equal && __popcll(eq & below) < left);
        const uint64_t taken = __builtin_amdgcn_ballot_w64(take);
        if (take) out[n + __popcll(taken & below)] = p + lane;
        n += __popcll(taken);
        left -= min(left, __popcll(eq));
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int n_cu, hipStream_t stream)
{
    const int hpw = 512 / a.c.D, groups = (a.H + 2 * a.c.heads + hpw - 1) / hpw, s = std::min(a.c.shift, kStretch);
    const int64_t stretches = ((int64_t)a.n.T >> s) + 2 * (int64_t)a.n.B;
    // the heads of a stretch over several workgroups, as far as 32 waves to a compute unit take
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>((groups + 3) / 4, 4 * n_cu / std::max<int64_t>(1, stretches - a.n.B)));
    const dim3 grid((unsigned)stretches, (unsigned)splits);
    if (a.c.D == 128)
        hipLaunchKernelGGL(append_kernel<128>, grid, dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL(append_kernel<64>, grid, dim3(512), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.c.means == nullptr || a.c.heads == 0 || a.c.shift <= kStretch) return e;
    const dim3 pages((unsigned)((a.n.T >> a.c.shift) + 2 * a.n.B), (unsigned)a.c.heads);
    if (a.c.D == 128)
        hipLaunchKernelGGL(means_kernel<128>, pages, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(means_kernel<64>, pages, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_select(const SelectArgs &a, int64_t blocks, int n_cu, hipStream_t stream)
{
    const dim3 grid((unsigned)blocks, (unsigned)a.c.heads);
    const size_t lds = a.n.columns <= a.count ? 0 : (size_t)a.n.columns * 8;
    // few workgroups: as many waves to each as there can be, whose latencies and 64-bit products are what it takes
    const bool few = (int64_t)grid.x * grid.y <= n_cu;
    if (a.c.D == 128 && few)
        hipLaunchKernelGGL((select_kernel<128, 1024>), grid, dim3(1024), lds, stream, a);
    else if (a.c.D == 128)
        hipLaunchKernelGGL((select_kernel<128, 256>), grid, dim3(256), lds, stream, a);
    else if (few)
        hipLaunchKernelGGL((select_kernel<64, 1024>), grid, dim3(1024), lds, stream, a);
    else
        hipLaunchKernelGGL((select_kernel<64, 256>), grid, dim3(256), lds, stream, a);
    return hipGetLastError();
}

}  // namespace paged
}  // namespace regenvc
