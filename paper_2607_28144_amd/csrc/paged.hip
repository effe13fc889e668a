// gfx950 kernels around a bf16 key/value cache in pages: the append that norms
// and rotates, the mean keys of pages, and the choice of pages by their score.
#include <algorithm>

#include "paged_device.hpp"

namespace regenvc {
namespace paged {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));  // eight bf16, the first of a pair in the low half
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ u32x4 load16(const uint16_t *p)
{
    return *reinterpret_cast<const u32x4 *>(p);
}

// ---------------------------------------------------------------- append
// HBM-bound: every channel is read once and written once.  D / 8 lanes hold a
// head, 16 bytes each, so a wave works on 8 (D = 64) or 4 heads at once; the
// heads of q, k and v follow one another.  The angles are a lane's own (8
// channels of every head that it meets) and formed once per token, in 64 bits
// before the whole turns are taken off: at place 2^20 an f32 product would be
// off by 0.06 rad.  The halves layout pairs a lane with one rot / 16 lanes on,
// whose raw channels come by lane exchange and are normed here again.
constexpr int kBatchLoads = 4;  // groups of heads in flight

template <int D>
__global__ __launch_bounds__(64) void append_kernel(AppendArgs a)
{
    constexpr int LPH = D / 8, HPW = 64 / LPH;
    const int lane = threadIdx.x, sub = lane / LPH, d0 = lane % LPH * 8;
    const int t = blockIdx.x, splits = gridDim.y;
    // the sequence and place of this token
    const int b = last_from(a.n.B, t, [&](int i) { return (int64_t)first_of(a.n, i); });
    if (b < 0 || t >= first_of(a.n, b + 1)) return;
    const int pos = max(0, a.n.lens[b]) - (first_of(a.n, b + 1) - t);
    const int col = pos >> a.c.shift;
    int page = -1;
    if (pos >= 0 && col < a.n.columns) page = a.n.table[b * a.n.table_stride + col];
    const bool stored = page >= 0 && page < a.c.pages;
    const int64_t cell = (int64_t)page * a.c.heads * (D << a.c.shift) + (int64_t)(pos & ((1 << a.c.shift) - 1)) * D;

    const int rot = 2 * a.pairs;
    const bool turned = d0 < rot;
    float cs[8], sn[8];  // of each channel's pair; the sine with the sign that its partner enters with
    if (turned) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = d0 + e, i = a.interleaved ? d >> 1 : d < a.pairs ? d : d - a.pairs;
            const float x = (float)__builtin_amdgcn_fract((double)pos * a.turns[i]);
            const bool second = a.interleaved ? d & 1 : d >= a.pairs;
            cs[e] = a.amplitude * __builtin_amdgcn_cosf(x);
            sn[e] = a.amplitude * __builtin_amdgcn_sinf(x) * (second ? 1.f : -1.f);
        }
    }
    const int partner = a.interleaved ? lane : d0 < a.pairs ? lane + a.pairs / 8 : lane - a.pairs / 8;  // in the same head
    const int pd0 = partner % LPH * 8;
    const int total = a.H + 2 * a.c.heads, groups = (total + HPW - 1) / HPW;
    u32x4 wq = {}, wk = {}, wqp = {}, wkp = {};
    if (a.w_q != nullptr) wq = load16(a.w_q + d0), wqp = load16(a.w_q + (turned ? pd0 : d0));
    if (a.w_k != nullptr) wk = load16(a.w_k + d0), wkp = load16(a.w_k + (turned ? pd0 : d0));

    for (int g0 = blockIdx.y; g0 < groups; g0 += splits * kBatchLoads) {
        u32x4 x[kBatchLoads];
#pragma unroll
        for (int j = 0; j < kBatchLoads; ++j) {
            const int h = (g0 + j * splits) * HPW + sub;
            x[j] = u32x4{0, 0, 0, 0};
            if (h < a.H)
                x[j] = load16(a.q + t * a.q_ss + h * a.q_sh + d0);
            else if (h < a.H + a.c.heads)
                x[j] = load16(a.k + t * a.k_ss + (h - a.H) * a.k_sh + d0);
            else if (h < total)
                x[j] = load16(a.v + t * a.v_ss + (h - a.H - a.c.heads) * a.v_sh + d0);
        }
#pragma unroll
        for (int j = 0; j < kBatchLoads; ++j) {
            if (g0 + j * splits >= groups) break;
            const int h = (g0 + j * splits) * HPW + sub;
            const bool is_q = h < a.H, is_k = !is_q && h < a.H + a.c.heads;
            const bool norm = is_q ? a.w_q != nullptr : is_k && a.w_k != nullptr;
            float r = 1.f;
            {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fmaf(hi(x[j][e]), hi(x[j][e]), fmaf(lo(x[j][e]), lo(x[j][e]), s));
#pragma unroll
                for (int m = LPH / 2; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
                if (norm) r = 1.0f / sqrtf(s / (float)D + a.eps);
            }
            u32x4 p;  // the partner's raw channels
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = (uint32_t)__shfl((int)x[j][e], partner, 64);
            if (h >= total) continue;
            float y[8], z[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = is_q ? wq[e] : wk[e], wp = is_q ? wqp[e] : wkp[e];
                y[2 * e] = norm ? lo(x[j][e]) * r * lo(w) : lo(x[j][e]);
                y[2 * e + 1] = norm ? hi(x[j][e]) * r * hi(w) : hi(x[j][e]);
                z[2 * e] = norm ? lo(p[e]) * r * lo(wp) : lo(p[e]);
                z[2 * e + 1] = norm ? hi(p[e]) * r * hi(wp) : hi(p[e]);
            }
            if (turned && (is_q || is_k)) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = y[e] * cs[e] + (a.interleaved ? y[e ^ 1] : z[e]) * sn[e];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = f[e];
            }
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = is_q || is_k ? pack(y[2 * e], y[2 * e + 1]) : x[j][e];
            uint16_t *dst;
            if (is_q)
                dst = a.q_out + t * a.o_ss + h * a.o_sh;
            else if (stored)
                dst = (is_k ? a.c.k : a.c.v) + cell + (int64_t)(is_k ? h - a.H : h - a.H - a.c.heads) * (D << a.c.shift);
            else
                continue;
            *reinterpret_cast<u32x4 *>(dst + d0) = o;
        }
    }
}

// Mean keys of the pages that a call's new tokens touch, from the pages as the
// append left them.  A workgroup per page and head; sums of bf16 values in 64
// bits are exact for all but absurd spreads, so the mean does not depend on how
// the tokens came.  Rounded to bf16, as the keys that it stands for: a score
// then reads 1 / (2 page) of the places' bytes.  Pages of sequence b are numbered from
// first[b] / page + 2 b: n tokens touch at most n / page + 2.
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
    const __bf16 m = (__bf16)(float)(sum / rows);
    a.c.means[((int64_t)page * a.c.heads + hk) * D + threadIdx.x] = __builtin_bit_cast(uint16_t, m);
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
// of them in flight: their latencies are what bounds it.  The count-th largest
// score is found digit by digit from the top, eight bits a pass over the scores in
// LDS, until a digit splits none that are left.
constexpr int kSelectThreads = 512, kAtOnce = 8;

template <int D>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(SelectArgs a)
{
    constexpr int LPR = D / 8, RPP = kSelectThreads / LPR;
    constexpr int WAVES = kSelectThreads / 64;
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
        for (int i = tid; i < a.count; i += kSelectThreads) out[i] = i < seen ? i : -1;
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
    lookup(0, at);
    {
        double s[8] = {};
        const int rows = k.rows * G;  // at most H T
        for (int r = r0; r < rows; r += 4 * RPP) {
            u32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // past the last row that again, with no part in the sum
                const int at = min(r + j * RPP, rows - 1), query = at / G;
                x[j] = load16(a.q + (int64_t)(k.row + query) * a.q_ss + (int64_t)(hk * G + at - query * G) * a.q_sh + d0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (r + j * RPP >= rows) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[2 * e] += (double)lo(x[j][e]), s[2 * e + 1] += (double)hi(x[j][e]);
            }
        }
        // over the rows that a wave has at once, then over the waves
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int m = LPR; m < 64; m <<= 1) s[e] += __shfl_xor(s[e], m, 64);
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
        u32x4 x[kAtOnce];
        bool there[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            there[j] = at[j] >= 0;
            x[j] = u32x4{0, 0, 0, 0};
            if (there[j]) x[j] = load16(a.c.means + ((int64_t)at[j] * a.c.heads + hk) * D + d0);
        }
        if (p0 + RPP * kAtOnce < seen) lookup(p0 + RPP * kAtOnce, at);
        double sum[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            sum[j] = there[j] ? 0.0 : -__builtin_inf();
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[j] = fma(qs[2 * e], (double)lo(x[j][e]), fma(qs[2 * e + 1], (double)hi(x[j][e]), sum[j]));
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
        for (int p = tid; p < seen; p += kSelectThreads) {
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
    const int hpw = 512 / a.c.D, groups = (a.H + 2 * a.c.heads + hpw - 1) / hpw;
    // few tokens: a token's heads over several waves
    const int splits = std::max(1, std::min(groups, 8 * n_cu / a.n.T));
    const dim3 grid((unsigned)a.n.T, (unsigned)splits);
    if (a.c.D == 128)
        hipLaunchKernelGGL(append_kernel<128>, grid, dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(append_kernel<64>, grid, dim3(64), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.c.means == nullptr) return e;
    const dim3 pages((unsigned)((a.n.T >> a.c.shift) + 2 * a.n.B), (unsigned)a.c.heads);
    if (a.c.D == 128)
        hipLaunchKernelGGL(means_kernel<128>, pages, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(means_kernel<64>, pages, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_select(const SelectArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.n.T / a.q_block + a.n.B), (unsigned)a.c.heads);
    const size_t lds = a.n.columns <= a.count ? 0 : (size_t)a.n.columns * 8;
    if (a.c.D == 128)
        hipLaunchKernelGGL(select_kernel<128>, grid, dim3(kSelectThreads), lds, stream, a);
    else
        hipLaunchKernelGGL(select_kernel<64>, grid, dim3(kSelectThreads), lds, stream, a);
    return hipGetLastError();
}

}  // namespace paged
}  // namespace regenvc
