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
// eight values of a row as they are held between load and use
template <bool F32>
struct Raw8 {
    f32x4 a, b;
    __device__ float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
template <>
struct Raw8<false> {
    bf16x8 a;
    __device__ float operator[](int i) const { return (float)a[i]; }
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> load8(const void *p, int64_t at)
{
    if constexpr (F32) {
        const f32x4 *q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at);
        return Raw8<F32>{q[0], q[1]};
    } else {
        return Raw8<F32>{*reinterpret_cast<const bf16x8 *>(static_cast<const uint16_t *>(p) + at)};
    }
}

// HBM-bound: 2 (or 4) bytes read and 0.53 written per value.  A workgroup
// takes 16 rows and two steps (512 columns): a wave's 64 lanes a row at a
// time, eight columns each, four lanes sharing a block; the scale bytes are
// gathered in LDS and leave as whole lines.  10920 x 1536: 8.7-10.3 us, 4.1-4.9
// TB/s; 1365 x 8960: 7.5 us, 4.2; 21 x 1536: 3.5 us, a launch.  From f32 13.1 us
// (76 MB, 5.8 TB/s) and 10.5 (5.3).
template <bool F32>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a, int nk)
{
    __shared__ uint8_t sc[16][16];  // [row][block of the two steps]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * 16;
    const int c = blockIdx.y * 512 + lane * 8;
    // All loads before the first use, and without branches where there are 16 rows (10920 x 1536: 9.9 us with branches,
    // 9.1 so); past the last column they repeat columns, which become zeros.
    Raw8<F32> v[4] = {};
    auto load = [&](int p) { v[p] = load8<F32>(a.x, (r0 + 4 * p + wave) * a.ldx + min(c, a.K - 8)); };
    if (r0 + 16 <= a.rows) {
#pragma unroll
        for (int p = 0; p < 4; ++p) load(p);
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p)
            if (r0 + 4 * p + wave < a.rows) load(p);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t row = r0 + 4 * p + wave;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c < a.K ? v[p][i] : 0.f;
        uint32_t code;
        const uint32_t byte = quantize_quad(x, code);
        if ((lane & 3) == 0) sc[4 * p + wave][lane >> 2] = (uint8_t)byte;
        if (row < a.rows && c < nk * kStepK) *reinterpret_cast<uint32_t *>(a.codes + (row * nk) * kStepBytes + c / 2) = code;
    }
    __syncthreads();
    const int t = threadIdx.x, step = t >> 6;  // of the two
    if (t >= 128 || (int)blockIdx.y * 2 + step >= nk) return;
    const int r = lane & 15, b = step * 8 + 2 * (lane >> 4);
    *reinterpret_cast<uint16_t *>(a.scales + ((int64_t)blockIdx.x * nk + blockIdx.y * 2 + step) * 128 + lane * 2) =
        (uint16_t)(sc[r][b] | sc[r][b + 1] << 8);
}

// HBM-bound the other way round: a wave per row and 512 columns, eight of them a
// lane.  10920 x 1536 to bf16 8.5 us (42 MB, 5.0 TB/s), to f32 14.8 (5.1); 1365 x
// 8960 7.0 (4.4) and 11.9 (4.6).
template <bool F32>
__global__ __launch_bounds__(256) void dequantize_kernel(DequantizeArgs a, int nk)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int c = blockIdx.y * 512 + lane * 8;
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

// 32 columns of a bf16 row, from c on, as loaded by one lane (past the end the
// last ones again), and brought to MXFP4: codes and scale byte.  Columns from K on
// are zeros.
struct Block32 {
    bf16x8 v[4];
};
__device__ __forceinline__ Block32 load_block(const uint16_t *row, int c, int K)
{
    Block32 b;
#pragma unroll
    for (int j = 0; j < 4; ++j) b.v[j] = *reinterpret_cast<const bf16x8 *>(row + min(c + 8 * j, K - 8));
    return b;
}
__device__ __forceinline__ uint32_t quantize_block(const Block32 &b, int c, int K, u32x4 &codes)
{
    float x[4][8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[j][i] = c + 8 * j < K ? (float)b.v[j][i] : 0.f;
            m = max(m, __float_as_uint(x[j][i]) & 0x7fffffffu);
        }
    const uint32_t byte = scale_byte(m);
    const float inv = scale_inverse(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] *= inv;
        codes[j] = byte == kNanScale ? 0u : encode8(x[j]);
    }
    return byte;
}

// Up to 16 MB rows: the weights are read once and bound the time, and there
// is little of everything, so a workgroup takes 16 output channels and all
// rows, its W waves taking the steps of K in turn; their sums meet in LDS.
// QUANT: a is bf16 and each workgroup brings its rows to MXFP4 itself, in
// registers.  blockIdx.x: tile of 16 MB rows.  1 x 1536 x 1536: 3.8 us in a graph of
// such calls, of which an empty kernel has about 2.5 and the weights' bytes 0.3;
// what is left is latency, so that loads do not wait for one another (4.5 with
// branches around them and the epilogue's loads at the end).  The next step's loads
// ahead of a step's products gained nothing.
template <int MB, int W, int EPI, bool QUANT>
__global__ __launch_bounds__(64 * W) void linear_rows_kernel(LinearArgs a, int nk)
{
    static_assert(W >= MB, "a thread joins the sums of four channels of a row at most");
    __shared__ f32x4 red[W][MB * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, x = lane & 15;
    const int n0 = blockIdx.y * 16, m0 = blockIdx.x * 16 * MB;
    // what this thread's share of the epilogue reads
    const int64_t m = m0 + wave * 16 + x;
    const int n = n0 + 4 * g;
    u32x2 bias = {0, 0};
    f32x4 gate = {1.f, 1.f, 1.f, 1.f};
    if (a.bias != nullptr) bias = *reinterpret_cast<const u32x2 *>(static_cast<const uint16_t *>(a.bias) + n);
    if (EPI == kEpiGatedRes && a.gate != nullptr) gate = *reinterpret_cast<const f32x4 *>(a.gate + n);
    const uint8_t *wc = a.w_codes + (int64_t)(n0 + x) * nk * kStepBytes + g * 32;
    const uint8_t *wsc = a.w_scales + (int64_t)blockIdx.y * nk * 128 + lane * 2;
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
            const int64_t row = min(m0 + mb * 16 + x, a.M - 1);
            u32x4 f[2];
            uint32_t as;
            if constexpr (QUANT) {
                const uint16_t *p = static_cast<const uint16_t *>(a.a) + row * a.lda;
                const int c = kt * kStepK + 64 * g;
                const Block32 b0 = load_block(p, c, a.K), b1 = load_block(p, c + 32, a.K);
                __builtin_amdgcn_sched_barrier(0);
                as = quantize_block(b0, c, a.K, f[0]);
                as |= quantize_block(b1, c + 32, a.K, f[1]) << 8;
            } else {
                const uint8_t *p = a.a_codes + (row * nk + kt) * kStepBytes + g * 32;
                f[0] = *reinterpret_cast<const u32x4 *>(p);
                f[1] = *reinterpret_cast<const u32x4 *>(p + 16);
                as = *reinterpret_cast<const uint16_t *>(a.a_scales + ((int64_t)min((m0 >> 4) + mb, (a.M - 1) >> 4) * nk + kt) * 128 +
                                                         lane * 2);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) acc[mb] = mfma(w[ks], f[ks], acc[mb], ks, ws, as);
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) red[wave][mb * 64 + lane] = acc[mb];
    __syncthreads();
    if (wave >= MB || m >= a.M) return;
    f32x4 part[W];
#pragma unroll
    for (int k = 0; k < W; ++k) part[k] = red[k][threadIdx.x];
    __builtin_amdgcn_sched_barrier(0);
    f32x4 y = part[0];
#pragma unroll
    for (int k = 1; k < W; ++k) y += part[k];
    y += f32x4{__uint_as_float(bias[0] << 16), __uint_as_float(bias[0] & 0xffff0000u), __uint_as_float(bias[1] << 16),
               __uint_as_float(bias[1] & 0xffff0000u)};
    if constexpr (EPI == kEpiGatedRes) {
        f32x4 *q = reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + m * a.ldo + n);
        *q = *q + gate * y;
    } else {
        bf16x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (__bf16)tile::activate<EPI>(y[i]);
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + m * a.ldo + n) = o;
    }
}

// ---------------------------------------------------------------- tiles
// Four waves per tile of (32 MB) rows x (32 NB) channels, each with a quarter
// of it, WPE workgroups per compute unit.  A workgroup walks tiles blockIdx.x,
// blockIdx.x + gridDim.x, ...: the steps of all of them form one stream
// through an LDS ring of ST stages of codes and scale lines, so that the next
// tile's first steps land while this one's last are multiplied and its output
// is stored (10920 x 8960 x 1536: 133 us with a workgroup per tile, 101 so).
// What a tile needs besides its steps is kept short: its place without
// divisions, its biases from one wait (a branch and a wait for each of them cost
// 2800 cycles a tile: 103 us, 97 without).
//
// What bounds it: per 128 x 128 tile and step, 512 cycles of matrix
// instructions per SIMD and 1024 of LDS (34 KB of copies at 64 bytes a cycle,
// 64 KB of fragment reads at 128); two workgroups per compute unit take about
// 1000.  8192 x 8192 x 8192: 273-292 us, 3.8-4.0 PFLOP/s, with the matrix units
// busy for 52 % of the cycles and the clock down to 1.79 GHz: the power limit.
// 10920 x 8960 x 1536: 94 us, with GELU 108 (2.8 PFLOP/s), of which the epilogue
// (196 MB of output; an exponential and a reciprocal for each of 98 million
// values) takes 14 and 28: without it 80.  1365 x 1536 x 8960: 17.4 us (2.2
// PFLOP/s).
// Larger tiles do less LDS work per MFMA, but 256 x 256 leaves a wave alone on
// its SIMD with 256 accumulators: 310-338 us for the same product, and no
// second workgroup beside its epilogue.  Where there are few tiles, their
// steps wait for memory, all workgroups being at the same place in K: four
// stages then pay (1365 x 1536 x 8960, 132 tiles: 29.8 us with two stages, 22.7
// with four; 240 tiles of 96 x 96: 17.4, with five or six 17.8).  All of a step's
// fragments read a step ahead, into a second set of registers: 18.6.  K is not
// split: over 216 shapes the best split of each was 0.07 % faster than the best
// whole one.
template <int MB_, int NB_, int WPE_, int ST_>
struct Shape {
    static constexpr int MB = MB_, NB = NB_, WPE = WPE_, ST = ST_;
    static constexpr int BM = 32 * MB, BN = 32 * NB;
    static constexpr int A_BYTES = BM * kStepBytes, W_BYTES = BN * kStepBytes;
    static constexpr int S_CHUNKS = 8 * 2 * (MB + NB);  // 16-byte chunks of a step's scale lines, A's first
    static constexpr int S_COPIES = (S_CHUNKS + 63) / 64;
    static constexpr int S_BYTES = S_COPIES * 1024;
    static constexpr int OUT = ST * (A_BYTES + W_BYTES + S_BYTES);  // where 16 rows of each wave's output are staged
    static constexpr int OUT_ROW = 16 * NB * 2;
    static constexpr bool STAGED = NB == 4 && (OUT + 4 * 16 * OUT_ROW) * WPE <= 160 * 1024;
    static constexpr int LDS = OUT + (STAGED ? 4 * 16 * OUT_ROW : 0);
    static_assert(LDS * WPE <= 160 * 1024 && S_COPIES <= 4 && (!STAGED || NB == 4), "tile shape");
};

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) uint16_t lds_u16;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

// Where a row's eight chunks lie in its 128 bytes of a stage.  A fragment read
// takes chunk 2 g + ks of 16 rows, for g = 0 .. 3; 16 of its lanes are served
// at a time, of two neighbouring g, eight rows each: their chunks have to lie
// an odd number of places apart, or they share banks with rows of the same
// parity (a read of 12 cycles instead of 8).
__device__ __forceinline__ int place_of(int row, int g, int ks)
{
    return (g + 4 * ks) ^ (row & 7);
}
__device__ __forceinline__ int chunk_at(int row, int place)
{
    const int p = place ^ (row & 7);
    return (p & 3) * 2 + (p >> 2);
}

// A pointer that is the same in every lane, in scalar registers.
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const uint8_t *>((uint64_t)hi << 32 | lo);
}

// The tiles of a launch: tiles_m x tiles_n of them in groups of kGroupM row
// blocks, in the order of tile::tile_of.  inv_group, inv_last: 2^32 / d rounded
// down, for the sizes of a group and the row blocks of the last one; a division
// by them is a high product and one correction, where the compiler's own (four
// for an item, twice per tile) would take longer than a step.
struct Tiles {
    int nk, tiles_n, n_tiles, groups;
    uint32_t group, inv_group, last, inv_last;
};
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t d, uint32_t inv)  // n < 2^31
{
    const uint32_t q = __umulhi(n, inv);  // right, or one too small
    return n - q * d >= d ? q + 1 : q;
}
struct Item {
    int m0, n0;
};
template <class S>
__device__ __forceinline__ Item item_of(const Tiles &t, int id)
{
    const int xcd = id & 7;
    const uint32_t tile = (uint32_t)(xcd * (t.n_tiles >> 3) + min(xcd, t.n_tiles & 7) + (id >> 3));
    const uint32_t group = quotient(tile, t.group, t.inv_group), in = tile - group * t.group;
    const bool whole = (int)group + 1 < t.groups;
    const uint32_t gm = whole ? (uint32_t)tile::kGroupM : t.last;
    const uint32_t tn = whole ? in / (uint32_t)tile::kGroupM : quotient(in, t.last, t.inv_last);
    return Item{(int)(group * tile::kGroupM + in - tn * gm) * S::BM, (int)tn * S::BN};
}

// A lane's biases of a wave's channels n0 .. n0 + 16 NB - 1 (4 g .. 4 g + 3 of
// each 16; those past the last channel, which are not stored, repeat others).
template <int NB>
__device__ __forceinline__ void load_bias(const LinearArgs &a, int n0, int g, u32x2 (&raw)[NB])
{
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) raw[nb] = u32x2{0, 0};
    if (a.bias == nullptr) return;
    const uint16_t *p = static_cast<const uint16_t *>(a.bias) + 4 * g;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) raw[nb] = *reinterpret_cast<const u32x2 *>(p + min(n0 + nb * 16, a.N - 16));
}

// A wave's quarter of a tile from its accumulators: row x of 16, channels 4 g ..
// 4 g + 3 of 16 in a lane.  f32 outputs go straight from there, 64 bytes of a row
// per 16 channels; what they are added to is read a block of channels ahead
// (10920 x 4608 x 1536: 112 us with each read waited for, 97 so).  bf16: 64 channels go 16 rows at a time through LDS of the
// wave's own, so that a store writes 128 bytes of each of 8 rows, past the caches
// (the next reader is another launch; left in L2 they are written when the kernel
// ends: 10920 x 1536 x 1536 23.1 us, past it 20.8).  Fewer channels: lanes of
// neighbouring g exchange halves of two blocks of 16, so that each has eight
// channels of one; such stores, of 64 bytes or 32 of a row, are slower past the
// caches (1365 x 1536 x 8960: 18.4 and 19.7).  WHOLE: no row or channel of the
// tile lies past the last one.
template <class S, int EPI, bool WHOLE>
__device__ __forceinline__ void store_tile(const LinearArgs &a, int m0, int n0, char *smem, f32x4 (&acc)[S::NB][S::MB])
{
    constexpr int MB = S::MB, NB = S::NB;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, x = lane & 15;
    auto round4 = [&](int nb, int mb) {
        bf16x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (__bf16)tile::activate<EPI>(acc[nb][mb][i]);
        return w;
    };
    if constexpr (EPI == kEpiGatedRes) {
        // a block of 16 channels' values are read while the one before is added and stored
        float *p = static_cast<float *>(a.out) + (int64_t)(m0 + x) * a.ldo + n0 + 4 * g;
        const int64_t rows16 = 16 * a.ldo;
        auto live = [&](int nb, int mb) { return WHOLE || (m0 + mb * 16 + x < a.M && n0 + nb * 16 < a.N); };
        f32x4 old[2][MB], gv[2];
        auto fetch = [&](int nb) {
            gv[nb & 1] = f32x4{1.f, 1.f, 1.f, 1.f};
            if (a.gate != nullptr && (WHOLE || n0 + nb * 16 < a.N))
                gv[nb & 1] = *reinterpret_cast<const f32x4 *>(a.gate + n0 + nb * 16 + 4 * g);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                if (live(nb, mb)) old[nb & 1][mb] = *reinterpret_cast<const f32x4 *>(p + mb * rows16 + nb * 16);
        };
        fetch(0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (nb + 1 < NB) fetch(nb + 1);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                if (live(nb, mb))
                    *reinterpret_cast<f32x4 *>(p + mb * rows16 + nb * 16) =
                        old[nb & 1][mb] + gv[nb & 1] * acc[nb][mb];
        }
    } else if constexpr (S::STAGED) {
        tile::lds_char *stg = (tile::lds_char *)smem + S::OUT + wave * 16 * S::OUT_ROW;
        const int r0 = lane >> 3, c = lane & 7;
        uint16_t *p = static_cast<uint16_t *>(a.out) + (int64_t)(m0 + r0) * a.ldo + n0 + c * 8;
        const int64_t rows8 = 8 * a.ldo;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                *(lds_bf16x4 *)(stg + x * S::OUT_ROW + ((nb * 2 + g / 2) ^ (x & 7)) * 16 + (g & 1) * 8) = round4(nb, mb);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 v = *(const lds_u32x4 *)(stg + (j * 8 + r0) * S::OUT_ROW + (c ^ r0) * 16);
                if (WHOLE || (m0 + mb * 16 + j * 8 + r0 < a.M && n0 + c * 8 < a.N))
                    __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
                p += rows8;
            }
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(a.out) + (int64_t)(m0 + x) * a.ldo;
        const int64_t rows16 = 16 * a.ldo;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const bool row = WHOLE || m0 + mb * 16 + x < a.M;
            u32x2 w[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) w[nb] = __builtin_bit_cast(u32x2, round4(nb, mb));
#pragma unroll
            for (int nb = 0; nb + 1 < NB; nb += 2) {
                const auto lo = __builtin_amdgcn_permlane16_swap(w[nb][0], w[nb + 1][0], false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(w[nb][1], w[nb + 1][1], false, false);
                const int n = n0 + (nb + (g & 1)) * 16 + (g >> 1) * 8;
                if (row && (WHOLE || n < a.N)) *reinterpret_cast<u32x4 *>(p + n) = u32x4{lo[0], hi[0], lo[1], hi[1]};
            }
            if constexpr (NB % 2 != 0) {
                const int n = n0 + (NB - 1) * 16 + 4 * g;
                if (row && (WHOLE || n < a.N)) *reinterpret_cast<u32x2 *>(p + n) = w[NB - 1];
            }
            p += rows16;
        }
    }
}

template <class S, int EPI>
__global__ __launch_bounds__(tile::kThreads4) __attribute__((amdgpu_waves_per_eu(S::WPE, S::WPE)))
void linear_tile_kernel(LinearArgs a, Tiles t)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    constexpr int MB = S::MB, NB = S::NB, NM = MB * NB, NF = MB + NB, ST = S::ST;
    constexpr int AP = S::A_BYTES / 4096, WP = S::W_BYTES / 4096, NC = AP + WP + 1;  // copies per wave and step
    constexpr uint32_t W0 = ST * S::A_BYTES, S0 = W0 + ST * S::W_BYTES;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, g = lane >> 4, x = lane & 15;
    const int ld = t.nk * kStepBytes;  // bytes of a row of codes
    int stride = gridDim.x;
    __asm__ volatile("" : "+s"(stride));  // read once: a scalar load in the loop would make every wait for LDS a full one

    // The copies: where the next step's come from (row offsets of the item's
    // tile, clamped to the last row; those rows are never stored).
    const uint32_t lds0 = (uint32_t)(uintptr_t)(tile::lds_char *)smem;
    const uint32_t la0 = __builtin_amdgcn_readfirstlane(lds0 + wave * AP * 1024);
    const uint32_t lw0 = __builtin_amdgcn_readfirstlane(lds0 + W0 + wave * WP * 1024);
    const int scopy = wave % S::S_COPIES;  // waves past the number of scale copies repeat one
    const uint32_t ls0 = __builtin_amdgcn_readfirstlane(lds0 + S0 + scopy * 1024);
    const int chunk = min(scopy * 64 + lane, S::S_CHUNKS - 1), line = chunk >> 3;
    const uint8_t *abase, *wbase, *ssrc, *a_scales = a.a_scales, *w_scales = a.w_scales;
    __asm__ volatile("" : "+s"(a_scales), "+s"(w_scales));
    uint32_t aoff[AP], woff[WP];
    int c_item = blockIdx.x, c_kt;
    auto aim = [&] {  // at item c_item
        const Item it = item_of<S>(t, c_item);
        abase = a.a_codes + (int64_t)it.m0 * ld;
        wbase = a.w_codes + (int64_t)it.n0 * ld;
#pragma unroll
        for (int i = 0; i < AP; ++i) {
            const int r = (wave * AP + i) * 8 + (lane >> 3);
            aoff[i] = (uint32_t)min(r, a.M - 1 - it.m0) * (uint32_t)ld + chunk_at(r, lane & 7) * 16;
        }
#pragma unroll
        for (int i = 0; i < WP; ++i) {
            const int r = (wave * WP + i) * 8 + (lane >> 3);
            woff[i] = (uint32_t)min(r, a.N - 1 - it.n0) * (uint32_t)ld + chunk_at(r, lane & 7) * 16;
        }
        const int64_t rb = line < 2 * MB ? min((it.m0 >> 4) + line, (a.M - 1) >> 4)
                                         : min((it.n0 >> 4) + line - 2 * MB, (a.N - 1) >> 4);
        ssrc = (line < 2 * MB ? a_scales : w_scales) + rb * t.nk * 128 + (chunk & 7) * 16;
        c_kt = 0;
    };
    auto copy = [&](int l, int st) {  // copy l of the step aimed at, into stage st
        const int64_t k = (int64_t)c_kt * kStepBytes;
        if (l < AP)
            tile::lds_copy16_s(uniform(abase + k), aoff[l], __builtin_amdgcn_readfirstlane(la0 + st * S::A_BYTES + l * 1024));
        else if (l < AP + WP)
            tile::lds_copy16_s(uniform(wbase + k), woff[l - AP],
                               __builtin_amdgcn_readfirstlane(lw0 + st * S::W_BYTES + (l - AP) * 1024));
        else
            tile::lds_copy16_v(ssrc + k, __builtin_amdgcn_readfirstlane(ls0 + st * S::S_BYTES));
    };
    auto advance = [&] {  // to the next step; past the last one, that again (into stages that nobody reads)
        if (++c_kt < t.nk) return;
        if (c_item + stride < t.n_tiles) {
            c_item += stride;
            aim();
        } else {
            --c_kt;
        }
    };

    u32x4 fa[2][MB], fw[2][NB];
    uint32_t sa[MB], sw[NB], sa1[MB], sw1[NB];
    const int ra = wm * 16 * MB + x, rw = wn * 16 * NB + x;
    const tile::lds_char *s = (const tile::lds_char *)smem;
    // fragment f (W's first) of half ks from stage st
    auto rd = [&](int st, int ks, int f) {
        if (f < NB)
            fw[ks][f] = *(const lds_u32x4 *)(s + W0 + st * S::W_BYTES + (rw + f * 16) * kStepBytes +
                                             place_of(rw, g, ks) * 16);
        else
            fa[ks][f - NB] = *(const lds_u32x4 *)(s + st * S::A_BYTES + (ra + (f - NB) * 16) * kStepBytes +
                                                  place_of(ra, g, ks) * 16);
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
    f32x4 acc[NB][MB];
    auto mfma2 = [&](int ks, int i) {
#pragma unroll
        for (int j = i; j < i + 2 && j < NM; ++j)
            acc[j % NB][j / NB] = mfma(fw[ks][j % NB], fa[ks][j / NB], acc[j % NB][j / NB], ks, sw[j % NB], sa[j / NB]);
    };

    // The compiler would sink a half's MFMAs across the barrier and the branch of advance() to their last use (10920 x
    // 8960 x 1536: 111 us, pinned 101).
    auto pin = [&] {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) __asm__ volatile("" : "+v"(acc[nb][mb]));
    };

    aim();
#pragma unroll
    for (int st = 0; st < ST; ++st) {
#pragma unroll
        for (int l = 0; l < NC; ++l) copy(l, st);
        advance();
    }
    __asm__ volatile("s_waitcnt vmcnt(%0)" : : "n"((ST - 1) * NC) : "memory");
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
    u32x2 raw[NB];
    load_bias<NB>(a, item_of<S>(t, blockIdx.x).n0 + wn * 16 * NB, g, raw);
    for (int item = blockIdx.x; item < t.n_tiles; item += stride) {
        const Item it = item_of<S>(t, item);
        const int m0 = it.m0 + wm * 16 * MB, n0 = it.n0 + wn * 16 * NB;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                acc[nb][mb] = f32x4{__uint_as_float(raw[nb][0] << 16), __uint_as_float(raw[nb][0] & 0xffff0000u),
                                    __uint_as_float(raw[nb][1] << 16), __uint_as_float(raw[nb][1] & 0xffff0000u)};
        if (item + stride < t.n_tiles) load_bias<NB>(a, item_of<S>(t, item + stride).n0 + wn * 16 * NB, g, raw);
        __builtin_amdgcn_s_setprio(1);  // before the other workgroup's epilogue (10920 x 8960 x 1536: 97.4 us, 95.4 so)
        for (int kt = 0; kt < t.nk; ++kt) {
            const int st1 = st + 1 == ST ? 0 : st + 1;
            // first half; the second half's fragments are read beside it
#pragma unroll
            for (int i = 0; i < NM; i += 2) {
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    if (f * RD / NF / 2 * 2 == i) rd(st, 1, f);
                mfma2(0, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            pin();
            // the next step has landed (an output's stores, counted too, only make this wait longer), and every
            // wave has read all of this one
            __asm__ volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((ST - 2) * NC) : "memory");
            __builtin_amdgcn_s_barrier();
            __asm__ volatile("" : : : "memory");
            if (ST == 2 && kt == 0) {
                // the next tile's biases have landed too: known here, the compiler does not wait for later copies where
                // they are used
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) __asm__ volatile("" : "+v"(raw[nb]));
            }
            // second half; beside it the next step's first fragments, and copies into this step's stage
#pragma unroll
            for (int i = 0; i < NM; i += 2) {
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    if (f * RD / NF / 2 * 2 == i) {
                        rd(st1, 0, f);
                        rd_scale(st1, f);
                    }
#pragma unroll
                for (int l = 0; l < NC; ++l)
                    if (l * RD / NC / 2 * 2 == i) copy(l, st);
                mfma2(1, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            pin();
            advance();
            next_scales();
            st = st1;
        }
        __builtin_amdgcn_s_setprio(0);
        if (m0 + 16 * MB <= a.M && n0 + 16 * NB <= a.N)
            store_tile<S, EPI, true>(a, m0, n0, smem, acc);
        else
            store_tile<S, EPI, false>(a, m0, n0, smem, acc);
    }
    tile::wait_all_copies();
}

typedef Shape<4, 4, 2, 2> Tile128x128;
typedef Shape<4, 4, 1, 4> Tile128x128Deep;  // four stages: for few tiles, one workgroup per compute unit
typedef Shape<3, 3, 1, 4> Tile96x96;
typedef Shape<2, 4, 2, 3> Tile64x128;
typedef Shape<2, 2, 2, 4> Tile64x64;
enum TileId : int32_t { kRows, kTile128x128, kTile128x128Deep, kTile96x96, kTile64x128, kTile64x64 };

template <int MB, int W, bool QUANT>
hipError_t launch_rows_t(const LinearArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.M + 16 * MB - 1) / (16 * MB)), (unsigned)(a.N / 16)), block(64 * W);
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
hipError_t launch_tile_t(const LinearArgs &a, hipStream_t stream)
{
    const int tiles_n = tile::tiles_along(a.N, S::BN);
    const int tiles_m = tile::tiles_along(a.M, S::BM), groups = tile::tiles_along(tiles_m, tile::kGroupM);
    const uint32_t group = (uint32_t)(tile::kGroupM * tiles_n), last = (uint32_t)(tiles_m - (groups - 1) * tile::kGroupM);
    const Tiles t{steps_of(a.K), tiles_n, tiles_m * tiles_n, groups, group, (uint32_t)(((uint64_t)1 << 32) / group),
                  last, (uint32_t)((((uint64_t)1 << 32) - 1) / last)};
    const int grid = std::min(t.n_tiles, device_cu_count() * S::WPE);
    hipLaunchKernelGGL((linear_tile_kernel<S, EPI>), dim3((unsigned)grid), dim3(tile::kThreads4), 0, stream, a, t);
    return hipGetLastError();
}

template <class S>
hipError_t launch_tile(const LinearArgs &a, hipStream_t stream)
{
    switch (a.epi) {
    case kEpiBias: return launch_tile_t<S, kEpiBias>(a, stream);
    case kEpiBiasGelu: return launch_tile_t<S, kEpiBiasGelu>(a, stream);
    case kEpiGatedRes: return launch_tile_t<S, kEpiGatedRes>(a, stream);
    }
    return hipErrorInvalidValue;
}

int64_t align256(int64_t b)
{
    return (b + 255) / 256 * 256;
}

}  // namespace

// Few rows: where the weights' bytes and latency count, not reuse of a tile.
// Measured (quantisation included), few-row kernel against the best tile: 1536
// x 1536 5.4 and 7.4 us with one row, 7.6 and 8.6 with 64; 8960 x 1536 7.9 and
// 8.1 with 17 rows, 8.8 and 8.3 with 32; 1536 x 8960 15.8 and 15.0 with 64.
static bool few_rows(int M, int N)
{
    return M <= 16 || (M <= 32 && N <= 4096) || (M <= 64 && N <= 1536);
}

// Whether the few-row kernel brings bf16 rows to MXFP4 itself: each workgroup
// does it again, which up to 16 rows of 2048 costs less than a launch
// (1536 x 1536 and one row 4.6 us against 5.4, 512 x 512 3.1 against 4.8; K =
// 8960 8.6 against 7.4).
static bool quantizes_itself(int M, int K)
{
    return M <= 16 && K <= 2048;
}

TilePlan linear_plan(int M, int N, int K, int epi, int n_cu)
{
    const int nk = steps_of(K);
    // waves along K: one step for each, but four where there are workgroups for all compute units without that
    if (few_rows(M, N) || K == 0)
        return TilePlan{kRows, 1, M <= 16 ? 16 : M <= 32 ? 32 : 64, 16, nk > 8 ? 16 : nk > 4 && N / 16 <= n_cu ? 8 : 4};
    // Fitted to the times of 3240 launches (12 pairs of N and K from 256 to 8960, 18 row counts from 65 to 10920, three
    // epilogues, every tile): the choice is on average 0.1 % slower than the best, at most 8 %; fitted to half of the
    // row counts, 0.3 to 0.7 % on the others.
    struct Cost {
        int32_t tile, bm, bn;
        double fixed[3], step, load, once;  // us per tile (by epilogue), per step, factor on whole rounds, per launch
    };
    static const Cost costs[] = {
        {kTile128x128, 128, 128, {0.446, 1.130, 3.261}, 0.398, 1.247, 0.58},
        {kTile128x128Deep, 128, 128, {1.016, 1.677, 3.688}, 0.379, 1.292, 0.00},
        {kTile96x96, 96, 96, {1.218, 1.352, 1.774}, 0.324, 1.314, 0.06},
        {kTile64x128, 64, 128, {0.472, 0.928, 1.582}, 0.293, 1.089, 0.52},
        {kTile64x64, 64, 64, {0.426, 0.399, 0.792}, 0.188, 1.095, 0.34},
    };
    const Cost *best = nullptr;
    double best_t = INFINITY;
    for (const Cost &c : costs) {
        const int64_t tiles = (int64_t)((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
        const double one = c.fixed[epi] + nk * c.step;
        double t = c.once + (double)(tiles / n_cu) * one * c.load;
        if (tiles % n_cu > 0) t += one * (1.0 + (c.load - 1.0) * (double)(tiles % n_cu) / n_cu);
        if (t < best_t) best_t = t, best = &c;
    }
    return TilePlan{best->tile, 1, best->bm, best->bn, 4};
}

int64_t linear_workspace(int M, int N, int K, bool quantized)
{
    if (M == 0 || N == 0 || K == 0 || quantized || quantizes_itself(M, K)) return 0;
    return align256(code_bytes(M, K)) + align256(scale_bytes(M, K));
}

hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream)
{
    const int nk = steps_of(a.K);
    const dim3 grid((unsigned)((a.rows + 15) / 16), (unsigned)((nk + 1) / 2)), block(256);
    if (a.f32)
        hipLaunchKernelGGL(quantize_kernel<true>, grid, block, 0, stream, a, nk);
    else
        hipLaunchKernelGGL(quantize_kernel<false>, grid, block, 0, stream, a, nk);
    return hipGetLastError();
}

hipError_t launch_dequantize(const DequantizeArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.rows + 3) / 4), (unsigned)((a.K + 511) / 512)), block(256);
    if (a.f32)
        hipLaunchKernelGGL(dequantize_kernel<true>, grid, block, 0, stream, a, steps_of(a.K));
    else
        hipLaunchKernelGGL(dequantize_kernel<false>, grid, block, 0, stream, a, steps_of(a.K));
    return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &args, hipStream_t stream)
{
    LinearArgs a = args;
    if (linear_workspace(a.M, a.N, a.K, a.a_codes != nullptr) > 0) {
        uint8_t *codes = reinterpret_cast<uint8_t *>(a.ws), *scales = codes + align256(code_bytes(a.M, a.K));
        const hipError_t e = launch_quantize(QuantizeArgs{a.a, a.lda, codes, scales, a.M, a.K, false}, stream);
        if (e != hipSuccess) return e;
        a.a_codes = codes, a.a_scales = scales;
    }
    const TilePlan p = linear_plan(a.M, a.N, a.K, a.epi, device_cu_count());
    switch (p.tile) {
    case kRows:  // (K = 0: no steps, any M)
        return p.waves == 16 ? launch_rows<16>(a, stream) : p.waves == 8 ? launch_rows<8>(a, stream) : launch_rows<4>(a, stream);
    case kTile128x128: return launch_tile<Tile128x128>(a, stream);
    case kTile128x128Deep: return launch_tile<Tile128x128Deep>(a, stream);
    case kTile96x96: return launch_tile<Tile96x96>(a, stream);
    case kTile64x128: return launch_tile<Tile64x128>(a, stream);
    case kTile64x64: return launch_tile<Tile64x64>(a, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace mx
}  // namespace regenvc
