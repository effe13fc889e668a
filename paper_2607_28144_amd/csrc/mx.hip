// gfx950 kernels of MXFP4: bringing rows to four bits and back, and linear
// layers whose operands are both in that form, on the scaled matrix
// instruction v_mfma_scale_f32_16x16x128_f8f6f4 with fp32 accumulation.
//
// A row's codes lie 128 bytes a step of 256 columns, which is the row of the
// bf16 tile kernels (64 columns a step) in bytes: copies, LDS image and
// fragment reads are theirs.  A lane's fragment is one block of 32 codes (16
// bytes) and that block's scale byte.  Half ks of a step (128 deep) takes from
// lane group g = lane / 16 the block 2 g + ks of the step's eight -- the sum
// over K may be taken in any order, and so a lane's two scale bytes of a step
// are neighbours: one 16-bit load serves both halves, the matrix instruction
// picking byte ks of it.
#include "mx_kernels.hpp"

#include <algorithm>

#include "attn_kernels.hpp"
#include "dit_kernels.hpp"
#include "gemm_tile.hpp"
#include "mx_device.hpp"

namespace regenvc {
namespace mx {
namespace {

// ---------------------------------------------------------------- to MXFP4 and back
template <bool F32>
__device__ __forceinline__ void load8(const void *p, int64_t at, float (&x)[8])
{
    if constexpr (F32) {
        const float *q = static_cast<const float *>(p) + at;
        const f32x4 a = *reinterpret_cast<const f32x4 *>(q), b = *reinterpret_cast<const f32x4 *>(q + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
        const bf16x8 a = *reinterpret_cast<const bf16x8 *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
}

// HBM-bound: 2 (or 4) bytes read and 0.53 written per value.  A workgroup
// takes 16 rows and two steps (512 columns): a wave's 64 lanes a row at a
// time, eight columns each, four lanes sharing a block; the scale bytes are
// gathered in LDS and leave as whole lines.
template <bool F32>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a, int nk)
{
    __shared__ uint8_t sc[16][16];  // [row][block of the two steps]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r0 = (int64_t)blockIdx.y * 16;
    const int c = blockIdx.x * 512 + lane * 8;
    float x[4][8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t row = r0 + 4 * p + wave;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[p][i] = 0.f;
        if (row < a.rows && c < a.K) load8<F32>(a.x, row * a.ldx + c, x[p]);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t row = r0 + 4 * p + wave;
        uint32_t code;
        const uint32_t byte = quantize_quad(x[p], code);
        if ((lane & 3) == 0) sc[4 * p + wave][lane >> 2] = (uint8_t)byte;
        if (row < a.rows && c < nk * kStepK) *reinterpret_cast<uint32_t *>(a.codes + (row * nk) * kStepBytes + c / 2) = code;
    }
    __syncthreads();
    const int t = threadIdx.x, step = t >> 6;  // of the two
    if (t >= 128 || blockIdx.x * 2 + step >= nk) return;
    const int r = lane & 15, b = step * 8 + 2 * (lane >> 4);
    *reinterpret_cast<uint16_t *>(a.scales + ((int64_t)blockIdx.y * nk + blockIdx.x * 2 + step) * 128 + lane * 2) =
        (uint16_t)(sc[r][b] | sc[r][b + 1] << 8);
}

template <bool F32>
__global__ __launch_bounds__(256) void dequantize_kernel(DequantizeArgs a, int nk)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6);
    const int c = blockIdx.x * 512 + lane * 8;
    if (row >= a.rows || c >= a.K) return;
    const uint32_t code = *reinterpret_cast<const uint32_t *>(a.codes + row * nk * kStepBytes + c / 2);
    const int kt = c / kStepK, blk = c % kStepK / kBlock;
    const float s = scale_value(
        a.scales[((row >> 4) * nk + kt) * 128 + ((blk >> 1) * 16 + (int)(row & 15)) * 2 + (blk & 1)]);
    const bf16x8 v = decode8(code, 1.0f);
    if constexpr (F32) {
        float *o = static_cast<float *>(a.out) + row * a.ldo + c;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<f32x4 *>(o + 4 * h) = f32x4{(float)v[4 * h] * s, (float)v[4 * h + 1] * s,
                                                          (float)v[4 * h + 2] * s, (float)v[4 * h + 3] * s};
    } else {
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)((float)v[i] * s);
        *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(a.out) + row * a.ldo + c) = o;
    }
}

// ---------------------------------------------------------------- few rows
__device__ __forceinline__ f32x4 mfma(u32x4 w, u32x4 a, f32x4 c, int ks, uint32_t ws, uint32_t as)
{
    const i32x8 wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8 av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return ks == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, c, 4, 4, 0, (int)ws, 0, (int)as)
                   : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, c, 4, 4, 1, (int)ws, 1, (int)as);
}

// One block of 32 columns of a bf16 row, brought to MXFP4 by one lane: its
// codes, and its scale byte.  Columns from K on are zeros.
__device__ __forceinline__ uint32_t quantize_block(const uint16_t *row, int c, int K, u32x4 &codes)
{
    bf16x8 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = bf16x8{};
        if (c + 8 * j < K) v[j] = *reinterpret_cast<const bf16x8 *>(row + c + 8 * j);
    }
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint((float)v[j][i]) & 0x7fffffffu);
    const uint32_t byte = scale_byte(m);
    const float inv = scale_inverse(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[j][i] * inv;
        codes[j] = byte == kNanScale ? 0u : encode8(x);
    }
    return byte;
}

// Up to 16 MB rows: the weights are read once and bound the time, and there
// is little of everything, so a workgroup takes 16 output channels and all
// rows, its W waves taking the steps of K in turn; their sums meet in LDS.
// QUANT: a is bf16 and each workgroup brings its rows to MXFP4 itself (in
// registers), which saves a launch.
template <int MB, int W, int EPI, bool QUANT>
__global__ __launch_bounds__(64 * W) void linear_rows_kernel(LinearArgs a, int nk)
{
    __shared__ f32x4 red[W][MB * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, x = lane & 15;
    const int n0 = blockIdx.x * 16;
    const uint8_t *wc = a.w_codes + (int64_t)(n0 + x) * nk * kStepBytes + g * 32;
    const uint8_t *wsc = a.w_scales + (int64_t)blockIdx.x * nk * 128 + lane * 2;
    f32x4 acc[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[mb] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kt = wave; kt < nk; kt += W) {
        u32x4 w[2];
        w[0] = *reinterpret_cast<const u32x4 *>(wc + (int64_t)kt * kStepBytes);
        w[1] = *reinterpret_cast<const u32x4 *>(wc + (int64_t)kt * kStepBytes + 16);
        const uint32_t ws = *reinterpret_cast<const uint16_t *>(wsc + (int64_t)kt * 128);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int64_t row = min(mb * 16 + x, a.M - 1);
            u32x4 f[2];
            uint32_t as;
            if constexpr (QUANT) {
                const uint16_t *p = static_cast<const uint16_t *>(a.a) + row * a.lda;
                as = quantize_block(p, kt * kStepK + 64 * g, a.K, f[0]);
                as |= quantize_block(p, kt * kStepK + 64 * g + 32, a.K, f[1]) << 8;
            } else {
                const uint8_t *p = a.a_codes + (row * nk + kt) * kStepBytes + g * 32;
                f[0] = *reinterpret_cast<const u32x4 *>(p);
                f[1] = *reinterpret_cast<const u32x4 *>(p + 16);
                as = *reinterpret_cast<const uint16_t *>(a.a_scales + ((int64_t)min(mb, (a.M - 1) >> 4) * nk + kt) * 128 +
                                                         lane * 2);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) acc[mb] = mfma(w[ks], f[ks], acc[mb], ks, ws, as);
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) red[wave][mb * 64 + lane] = acc[mb];
    __syncthreads();
    for (int t = threadIdx.x; t < MB * 64; t += 64 * W) {
        f32x4 y = red[0][t];
#pragma unroll
        for (int k = 1; k < W; ++k) y += red[k][t];
        const int m = (t >> 6) * 16 + (t & 15), n = n0 + 4 * ((t & 63) >> 4);
        if (m >= a.M) continue;
        y += tile::load_bias4(static_cast<const uint16_t *>(a.bias), n);
        if constexpr (EPI == kEpiGatedRes) {
            f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + m * a.ldo + n);
            const f32x4 gv =
                a.gate != nullptr ? *reinterpret_cast<const f32x4 *>(a.gate + n) : f32x4{1.f, 1.f, 1.f, 1.f};
            *q = *q + gv * y;
        } else {
            bf16x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = (__bf16)tile::activate<EPI>(y[i]);
            *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + m * a.ldo + n) = o;
        }
    }
}

// ---------------------------------------------------------------- tiles
// Four waves per tile of (32 MB) rows x (32 NB) channels, WPE workgroups per
// compute unit, two LDS stages of codes and of scale lines.
template <int MB_, int NB_, int WPE_>
struct Shape {
    static constexpr int MB = MB_, NB = NB_, WPE = WPE_;
    static constexpr int BM = 32 * MB, BN = 32 * NB;
    static constexpr int A_BYTES = BM * kStepBytes, W_BYTES = BN * kStepBytes;
    static constexpr int S_CHUNKS = 8 * 2 * (MB + NB);  // 16-byte chunks of a step's scale lines, A's first
    static constexpr int S_COPIES = (S_CHUNKS + 63) / 64;
    static constexpr int S_BYTES = S_COPIES * 1024;
    static constexpr int RINGS = 2 * (A_BYTES + W_BYTES + S_BYTES);
    static constexpr int LDS = RINGS > BM * BN * 2 ? RINGS : BM * BN * 2;  // the output is staged there too
    static_assert(LDS * WPE <= 160 * 1024 && S_COPIES <= 4, "tile shape");
};

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

// The K loop over steps [k0, k1): acc[nb][mb][i] as in tile::mma4.  A step's
// second half (ks = 1) is read beside the MFMAs of its first, the next step's
// first half beside those of its second; copies run two steps ahead.
template <class S>
__device__ __forceinline__ void mma_mx(const tile::Dense<false> &as, const tile::Dense<false> &ws, const uint8_t *a_sc,
                                       const uint8_t *w_sc, int nk, int k0, int k1, char *smem,
                                       f32x4 (&acc)[S::NB][S::MB])
{
    constexpr int MB = S::MB, NB = S::NB, NM = MB * NB, NF = MB + NB;
    constexpr int AP = S::A_BYTES / 4096, WP = S::W_BYTES / 4096;  // copies per wave and step, and one of scales
    constexpr uint32_t W0 = 2 * S::A_BYTES, S0 = W0 + 2 * S::W_BYTES;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, g = lane >> 4, x = lane & 15;

    tile::Dense<false>::Row arow[AP], wrow[WP];
#pragma unroll
    for (int i = 0; i < AP; ++i) {
        const int r = (wave * AP + i) * 8 + (lane >> 3);
        arow[i] = as.row(r, tile::swz(r, lane & 7));
    }
#pragma unroll
    for (int i = 0; i < WP; ++i) {
        const int r = (wave * WP + i) * 8 + (lane >> 3);
        wrow[i] = ws.row(r, tile::swz(r, lane & 7));
    }
    // this wave's copy of scale lines (waves past the number of copies repeat one)
    const int scopy = wave % S::S_COPIES, chunk = min(scopy * 64 + lane, S::S_CHUNKS - 1), line = chunk >> 3;
    const int64_t rb = line < 2 * MB ? min((as.r0 >> 4) + line, (as.rows - 1) >> 4)
                                     : min((ws.r0 >> 4) + line - 2 * MB, (ws.rows - 1) >> 4);
    const uint8_t *ssrc = (line < 2 * MB ? a_sc : w_sc) + rb * nk * 128 + (chunk & 7) * 16;

    const uint32_t lds0 = (uint32_t)(uintptr_t)(tile::lds_char *)smem;
    const uint32_t la0 = __builtin_amdgcn_readfirstlane(lds0 + wave * AP * 1024);
    const uint32_t lw0 = __builtin_amdgcn_readfirstlane(lds0 + W0 + wave * WP * 1024);
    const uint32_t ls0 = __builtin_amdgcn_readfirstlane(lds0 + S0 + scopy * 1024);
    const int kl = k1 - 1;
    // copy l of step kt (A's, W's, the scales') into stage st
    auto copy = [&](int l, int kt, int st) {
        if (l < AP) {
            const auto s = as.at(kt);
            as.copy(as.addr(arow[l], s), la0 + st * S::A_BYTES + l * 1024);
        } else if (l < AP + WP) {
            const auto s = ws.at(kt);
            ws.copy(ws.addr(wrow[l - AP], s), lw0 + st * S::W_BYTES + (l - AP) * 1024);
        } else {
            tile::lds_copy16_v(ssrc + (int64_t)kt * 128, ls0 + st * S::S_BYTES);
        }
    };
    constexpr int NC = AP + WP + 1;

#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};

    u32x4 fa[2][MB], fw[2][NB];
    uint32_t sa[MB], sw[NB], sa1[MB], sw1[NB];
    const int ra = wm * 16 * MB + x, rw = wn * 16 * NB + x;
    const tile::lds_char *s = (const tile::lds_char *)smem;
    // fragment f (W's first) of half ks from stage st
    auto rd = [&](int st, int ks, int f) {
        if (f < NB)
            fw[ks][f] = *(const lds_u32x4 *)(s + W0 + st * S::W_BYTES + (rw + f * 16) * kStepBytes +
                                             tile::swz(rw, 2 * g + ks) * 16);
        else
            fa[ks][f - NB] = *(const lds_u32x4 *)(s + st * S::A_BYTES + (ra + (f - NB) * 16) * kStepBytes +
                                                  tile::swz(ra, 2 * g + ks) * 16);
    };
    auto rd_scale = [&](int st, int f) {
        const tile::lds_char *p = s + S0 + st * S::S_BYTES + lane * 2;
        if (f < NB)
            sw1[f] = *(const lds_u16 *)(p + (2 * MB + wn * NB + f) * 128);
        else
            sa1[f - NB] = *(const lds_u16 *)(p + (wm * MB + f - NB) * 128);
    };
    auto next_scales = [&] {
#pragma unroll
        for (int i = 0; i < MB; ++i) sa[i] = sa1[i];
#pragma unroll
        for (int i = 0; i < NB; ++i) sw[i] = sw1[i];
    };
    auto mfma2 = [&](int ks, int i) {
#pragma unroll
        for (int j = i; j < i + 2; ++j)
            acc[j % NB][j / NB] = mfma(fw[ks][j % NB], fa[ks][j / NB], acc[j % NB][j / NB], ks, sw[j % NB], sa[j / NB]);
    };

#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int l = 0; l < NC; ++l) copy(l, min(k0 + st, kl), st);
    __asm__ volatile("s_waitcnt vmcnt(%0)" : : "n"(NC) : "memory");
    __builtin_amdgcn_s_barrier();
    __asm__ volatile("" : : : "memory");
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        rd(0, 0, f);
        rd_scale(0, f);
    }
    next_scales();

    constexpr int RD = NM * 3 / 4;  // a half's reads and copies are spread over this many MFMAs
    int st = 0;
    for (int kt = k0; kt < k1; ++kt) {
#pragma unroll
        for (int i = 0; i < NM; i += 2) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
                if (f * RD / NF / 2 * 2 == i) rd(st, 1, f);
            mfma2(0, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        // step kt + 1 has landed, and every wave has read all of step kt
        __asm__ volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" : : : "memory");
        const int k2 = min(kt + 2, kl);
#pragma unroll
        for (int i = 0; i < NM; i += 2) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
                if (f * RD / NF / 2 * 2 == i) {
                    rd(st ^ 1, 0, f);
                    rd_scale(st ^ 1, f);
                }
#pragma unroll
            for (int l = 0; l < NC; ++l)
                if (l * RD / NC / 2 * 2 == i) copy(l, k2, st);
            mfma2(1, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        next_scales();
        st ^= 1;
    }
    if constexpr (S::WPE == 1) {  // wait states before acc_value's reads of the last results
        __asm__ volatile("s_nop 15\n\ts_nop 15" : : : "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    tile::wait_all_copies();
}

// One tile per workgroup; EPI == kPartial: K range blockIdx.x / n_tiles of `splits`.
template <class S, int EPI>
__global__ __launch_bounds__(tile::kThreads4) __attribute__((amdgpu_waves_per_eu(S::WPE, S::WPE)))
void linear_tile_kernel(LinearArgs a, float *part, int nk, int tiles_n, int n_tiles, int splits)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    constexpr bool PART = EPI == tile::kPartial;
    const int sp = PART ? (int)blockIdx.x / n_tiles : 0;
    int tm, tn;
    tile::tile_of((int)blockIdx.x - sp * n_tiles, tiles_n, n_tiles, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN;
    const int k0 = PART ? (int)((int64_t)sp * nk / splits) : 0;
    const int k1 = PART ? (int)((int64_t)(sp + 1) * nk / splits) : nk;
    const tile::Dense<false> as{reinterpret_cast<const uint16_t *>(a.a_codes), (int64_t)nk * (kStepBytes / 2), a.M, m0};
    const tile::Dense<false> ws{reinterpret_cast<const uint16_t *>(a.w_codes), (int64_t)nk * (kStepBytes / 2), a.N, n0};
    f32x4 acc[S::NB][S::MB];
    if (k1 > k0) {
        mma_mx<S>(as, ws, a.a_scales, a.w_scales, nk, k0, k1, smem, acc);
    } else {
#pragma unroll
        for (int nb = 0; nb < S::NB; ++nb)
#pragma unroll
            for (int mb = 0; mb < S::MB; ++mb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const tile::Out o{static_cast<const uint16_t *>(a.bias), a.gate, PART ? part : a.out, PART ? (int64_t)a.N : a.ldo,
                      a.M, a.N};
    tile::store4<S, EPI>(o, m0, n0, sp, smem, acc);
}

typedef Shape<8, 8, 1> Tile256x256;
typedef Shape<4, 4, 2> Tile128x128;
typedef Shape<2, 4, 3> Tile64x128;
enum TileId : int32_t { kRows, kTile256x256, kTile128x128, kTile64x128 };

// Rows up to which the few-row kernel runs, and up to which it brings bf16
// rows to MXFP4 itself.
constexpr int kFewRows = 64, kQuantRows = 16;

template <int MB, int W, bool QUANT>
hipError_t launch_rows_t(const LinearArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.N / 16)), block(64 * W);
    const int nk = steps_of(a.K);
    switch (a.epi) {
    case kEpiBias: hipLaunchKernelGGL((linear_rows_kernel<MB, W, kEpiBias, QUANT>), grid, block, 0, stream, a, nk); break;
    case kEpiBiasGelu: hipLaunchKernelGGL((linear_rows_kernel<MB, W, kEpiBiasGelu, QUANT>), grid, block, 0, stream, a, nk); break;
    case kEpiGatedRes: hipLaunchKernelGGL((linear_rows_kernel<MB, W, kEpiGatedRes, QUANT>), grid, block, 0, stream, a, nk); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <int W>
hipError_t launch_rows(const LinearArgs &a, hipStream_t stream)
{
    if (a.M <= 16 && a.a_codes == nullptr) return launch_rows_t<1, W, true>(a, stream);
    if (a.M <= 16) return launch_rows_t<1, W, false>(a, stream);
    if (a.M <= 32) return launch_rows_t<2, W, false>(a, stream);
    return launch_rows_t<4, W, false>(a, stream);
}

template <class S, int EPI>
hipError_t launch_tile_t(const LinearArgs &a, float *part, int splits, hipStream_t stream)
{
    const int tiles_n = tile::tiles_along(a.N, S::BN), n_tiles = tile::tiles_along(a.M, S::BM) * tiles_n;
    hipLaunchKernelGGL((linear_tile_kernel<S, EPI>), dim3((unsigned)n_tiles * (unsigned)splits), dim3(tile::kThreads4), 0,
                       stream, a, part, steps_of(a.K), tiles_n, n_tiles, splits);
    return hipGetLastError();
}

template <class S>
hipError_t launch_tile(const LinearArgs &a, float *part, int splits, hipStream_t stream)
{
    if (splits > 1) {
        const hipError_t e = launch_tile_t<S, tile::kPartial>(a, part, splits, stream);
        if (e != hipSuccess) return e;
        return launch_linear_reduce(regenvc::LinearArgs{nullptr, nullptr, a.bias, a.gate, a.out, 0, a.ldo, a.M, a.N, a.K,
                                                        a.epi, part, 0},
                                    splits, stream);
    }
    switch (a.epi) {
    case kEpiBias: return launch_tile_t<S, kEpiBias>(a, nullptr, 1, stream);
    case kEpiBiasGelu: return launch_tile_t<S, kEpiBiasGelu>(a, nullptr, 1, stream);
    case kEpiGatedRes: return launch_tile_t<S, kEpiGatedRes>(a, nullptr, 1, stream);
    }
    return hipErrorInvalidValue;
}

int64_t align256(int64_t b)
{
    return (b + 255) / 256 * 256;
}

}  // namespace

TilePlan linear_plan(int M, int N, int K, int epi, int n_cu, int64_t ws_bytes)
{
    if (M <= kFewRows) return TilePlan{kRows, 1, M <= 16 ? 16 : M <= 32 ? 32 : 64, 16, steps_of(K) > 8 ? 16 : 4};
    const TileCost costs[] = {
        {kTile256x256, 256, 256, 4, epi == kEpiBias ? 7.7 : 10.9, 7.7, 1.0, 1.2, true},
        {kTile128x128, 128, 128, 4, 2.0, 2.0, 0.424, 0.988, true},
        {kTile64x128, 64, 128, 4, 1.5, 1.5, 0.396, 0.951, true},
    };
    return plan_tiles(costs, SplitCost{5.1, 8.1e6, epi == kEpiGatedRes ? 8 : 2}, M, N, steps_of(K), n_cu, ws_bytes);
}

LinearNeed linear_need(int M, int N, int K, int epi, bool quantized, int n_cu)
{
    LinearNeed need{};
    if (M == 0 || N == 0) return need;
    if (!quantized && M > kQuantRows && K > 0) need.least = align256(code_bytes(M, K)) + align256(scale_bytes(M, K));
    const TilePlan p = linear_plan(M, N, K, epi, n_cu, INT64_MAX);
    need.total = need.least + (p.splits > 1 ? (int64_t)p.splits * M * N * (int64_t)sizeof(float) : 0);
    return need;
}

hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream)
{
    const int nk = steps_of(a.K);
    const dim3 grid((unsigned)((nk + 1) / 2), (unsigned)((a.rows + 15) / 16)), block(256);
    if (a.f32)
        hipLaunchKernelGGL(quantize_kernel<true>, grid, block, 0, stream, a, nk);
    else
        hipLaunchKernelGGL(quantize_kernel<false>, grid, block, 0, stream, a, nk);
    return hipGetLastError();
}

hipError_t launch_dequantize(const DequantizeArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.K + 511) / 512), (unsigned)((a.rows + 3) / 4)), block(256);
    if (a.f32)
        hipLaunchKernelGGL(dequantize_kernel<true>, grid, block, 0, stream, a, steps_of(a.K));
    else
        hipLaunchKernelGGL(dequantize_kernel<false>, grid, block, 0, stream, a, steps_of(a.K));
    return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &args, hipStream_t stream)
{
    LinearArgs a = args;
    char *part = a.ws;
    int64_t left = a.ws_bytes;
    if (a.a_codes == nullptr && a.M > kQuantRows && a.K > 0) {
        const int64_t codes = align256(code_bytes(a.M, a.K)), least = codes + align256(scale_bytes(a.M, a.K));
        uint8_t *q = reinterpret_cast<uint8_t *>(a.ws);
        const hipError_t e = launch_quantize(QuantizeArgs{a.a, a.lda, q, q + codes, a.M, a.K, false}, stream);
        if (e != hipSuccess) return e;
        a.a_codes = q, a.a_scales = q + codes;
        part += least, left -= least;
    }
    const TilePlan p = linear_plan(a.M, a.N, a.K, a.epi, device_cu_count(), left);
    float *sums = reinterpret_cast<float *>(part);
    switch (p.tile) {
    case kRows: return p.waves == 16 ? launch_rows<16>(a, stream) : launch_rows<4>(a, stream);
    case kTile256x256: return launch_tile<Tile256x256>(a, sums, p.splits, stream);
    case kTile128x128: return launch_tile<Tile128x128>(a, sums, p.splits, stream);
    case kTile64x128: return launch_tile<Tile64x128>(a, sums, p.splits, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace mx
}  // namespace regenvc
