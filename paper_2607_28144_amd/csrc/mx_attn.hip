// gfx950 kernels of a key/value cache held in MXFP4: the append that fills it
// and exact attention over it.
//
// Codes and scales lie head-major, [B, heads, capacity, ...]: what a head's
// queries read of consecutive tokens is contiguous (64 + 4 bytes a token at D
// = 128), whichever XCD reads it.  Blocks of 32 run along D, so that a token
// is brought to four bits by itself, when it arrives.
//
// Attention.  Scores are computed transposed, S^T = K Q^T, on
// v_mfma_f32_16x16x32_bf16: K as it stands in four bits, turned to bf16 in
// registers (exact: a code is a small integer over two, a scale a power of
// two), Q in bf16.  A lane's accumulator then holds, for one query row, keys
// 4 g .. 4 g + 3 of 16 (g = lane / 16): rounded to bf16, two of them are the B
// operand of O^T = V^T P^T in the key order {4 g + i, 16 + 4 g + i}, which
// the transposing LDS reads of V follow.  The sum over d of K Q^T may be taken
// in any order too: lane group g takes the D / 4 channels from D / 4 g on, one
// piece of the cache's row per lane.
//
// Query heads that share a key head are rows of one tile: row r is query r / G
// of head G hk + r % G.  Two running sums per row, as in the bf16 attention:
// O is divided by the sum of the weights as rounded to bf16, LSE takes that of
// the unrounded ones.
#include "mx_kernels.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mx_device.hpp"

namespace regenvc {
namespace mx {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;

// ---------------------------------------------------------------- append, read back
// HBM-bound.  One lane per eight channels of a token's head, keys and values
// both; blockIdx.y: the sequence.  32760 tokens x 12 x 128: 51 us, 254 MB, 5.0
// TB/s; read back (values_kernel), 2 x 3120 tokens: 9 us, 48 MB, 5.3.
template <int D>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    constexpr uint32_t per = D / 8;  // lanes of a head's row
    const uint32_t id = blockIdx.x * 256u + threadIdx.x, n = (uint32_t)a.S * a.c.heads * per;
    const int64_t b = blockIdx.y;
    const int count = a.count != nullptr ? min(a.count[b], a.S) : a.S;
    const int start = a.start != nullptr ? a.start[b] : 0;
    const uint32_t at = min(id, n - 1);
    const uint32_t chunk = at % per, th = at / per, i = th / (uint32_t)a.c.heads, h = th - i * a.c.heads;
    // of more tokens than the cache holds, only the last ones: no two tokens share a place
    const bool live = id < n && (int)i < count && (int64_t)i + a.c.capacity >= count && start >= 0;
    bf16x8 q[2] = {};
    if (live) {
        q[0] = *reinterpret_cast<const bf16x8 *>(static_cast<const uint16_t *>(a.k) + b * a.k_sb + i * a.k_ss + h * a.k_sh +
                                                 chunk * 8);
        q[1] = *reinterpret_cast<const bf16x8 *>(static_cast<const uint16_t *>(a.v) + b * a.v_sb + i * a.v_ss + h * a.v_sh +
                                                 chunk * 8);
    }
    const uint32_t cap = (uint32_t)a.c.capacity, place = ((uint32_t)max(start, 0) % cap + i) % cap;
    const int64_t token = (b * a.c.heads + h) * a.c.capacity + place;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (float)q[v][k];
        uint32_t code;
        const uint32_t byte = quantize_quad(x, code);
        if (!live) continue;
        *reinterpret_cast<uint32_t *>((v ? a.c.v_codes : a.c.k_codes) + token * (D / 2) + chunk * 4) = code;
        if ((chunk & 3) == 0) (v ? a.c.v_scales : a.c.k_scales)[token * (D / 32) + chunk / 4] = (uint8_t)byte;
    }
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void values_kernel(ValuesArgs a)
{
    constexpr uint32_t per = D / 8;
    const uint32_t id = blockIdx.x * 256u + threadIdx.x, n = (uint32_t)a.c.capacity * a.c.heads * per;
    if (id >= n) return;
    const int64_t b = blockIdx.y;
    const uint32_t chunk = id % per, th = id / per, place = th / (uint32_t)a.c.heads, h = th - place * a.c.heads;
    const int64_t token = (b * a.c.heads + h) * a.c.capacity + place;
    uint32_t code[2], byte[2];  // both before the first store, which the compiler would not move a load across
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        code[v] = *reinterpret_cast<const uint32_t *>((v ? a.c.v_codes : a.c.k_codes) + token * (D / 2) + chunk * 4);
        byte[v] = (v ? a.c.v_scales : a.c.k_scales)[token * (D / 32) + chunk / 4];
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const float s = scale_value(byte[v]);
        const bf16x8 x = decode8(code[v], 1.0f);
        const int64_t at = (b * n + id) * 8;
        if constexpr (F32) {
            float *o = static_cast<float *>(v ? a.v : a.k) + at;
#pragma unroll
            for (int h4 = 0; h4 < 2; ++h4)
                *reinterpret_cast<f32x4 *>(o + 4 * h4) = f32x4{(float)x[4 * h4] * s, (float)x[4 * h4 + 1] * s,
                                                               (float)x[4 * h4 + 2] * s, (float)x[4 * h4 + 3] * s};
        } else {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (__bf16)((float)x[i] * s);
            *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(v ? a.v : a.k) + at) = o;
        }
    }
}

// ---------------------------------------------------------------- attention
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

// A scale byte as the f32 that the conversion takes: it reads the exponent.
__device__ __forceinline__ float scale_bits(uint32_t byte)
{
    return __uint_as_float(byte << 23);
}

// What a workgroup works on.
struct Place {
    int b, hk, tile, range;  // sequence, key head, tile of its rows, range of its keys
    int len, k0, k1;         // the sequence's places, this range of them
};
constexpr int kKeyAlign = 64;  // ranges of keys begin at multiples of it

__device__ __forceinline__ Place place_of(const AttnCacheArgs &a, const AttnCachePlan &p)
{
    Place w;
    uint32_t id = blockIdx.x;  // 32-bit unsigned throughout: the divisions are on the way to the first load
    const uint32_t ranges = p.key_ranges, tiles = p.row_tiles, heads = a.c.heads;
    const uint32_t q = id / ranges;
    w.range = (int)(id - q * ranges);
    const uint32_t q2 = q / tiles;
    w.tile = (int)(q - q2 * tiles);
    w.b = (int)(q2 / heads);
    w.hk = (int)(q2 - w.b * heads);
    const int len = a.lens != nullptr ? a.lens[w.b] : a.max_len;
    w.len = max(0, min(len, a.c.capacity));
    const uint32_t units = ((uint32_t)w.len + kKeyAlign - 1) / kKeyAlign;  // < 2^25, ranges <= 64
    w.k0 = (int)(units * w.range / ranges) * kKeyAlign;
    w.k1 = min(w.len, (int)(units * (w.range + 1) / ranges) * kKeyAlign);
    return w;
}

// Partial results of the key ranges in the workspace: O (f32, normalized over
// the range) [range][b][query][head][D], then LSE in log2 units
// [range][b][query][head] (-inf: no key).
__device__ __forceinline__ float *part_o(const AttnCacheArgs &a, int64_t range, int64_t b, int64_t s, int64_t h)
{
    return reinterpret_cast<float *>(a.ws) + (((range * a.B + b) * a.Sq + s) * a.H + h) * a.c.D;
}
__device__ __forceinline__ float *part_lse(const AttnCacheArgs &a, int ranges, int64_t range, int64_t b, int64_t s,
                                           int64_t h)
{
    return reinterpret_cast<float *>(a.ws) + (int64_t)ranges * a.B * a.Sq * a.H * a.c.D + ((range * a.B + b) * a.Sq + s) * a.H +
           h;
}

__device__ __forceinline__ void store_out4(const AttnCacheArgs &a, int64_t b, int64_t s, int64_t h, int d, f32x4 v)
{
    const int64_t at = b * a.o_sb + s * a.o_ss + h * a.o_sh + d;
    if (a.f32) {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.o) + at) = v;
    } else {
        const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.o) + at) = o;
    }
}

// Q rows of a lane: row r of the (query, head) rows that share the key head,
// the channels D / 4 g + 8 s + 0..7 of it for s < D / 32.
template <int D>
__device__ __forceinline__ void load_q(const AttnCacheArgs &a, const Place &w, int row, int G, bf16x8 (&q)[D / 32])
{
    const int g = (threadIdx.x & 63) >> 4;
    const int rows = a.Sq * G;
    const int r = min(row, rows - 1);
    const uint16_t *p = static_cast<const uint16_t *>(a.q) + (int64_t)w.b * a.q_sb + (int64_t)(r / G) * a.q_ss +
                        (int64_t)(w.hk * G + r % G) * a.q_sh + D / 4 * g;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 8 * s);
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

// Few rows (tiles of 16 MB for a key head): memory-bound.  Every wave walks key
// tiles of its own, 32 keys at a time, with nothing shared: K's codes go from
// memory to registers and the matrix unit; V's through 2 D x 32 bytes of
// wave-private LDS, for the transposition.  The waves' results meet in LDS.
// With its join, in a graph of such calls: one query against 10920 places, 12 heads
// of 128 (17.8 MB), 11.7 us; 12 rows each of 16 sequences x 4 key heads of 64 (18.8
// MB, 69050 places in all) 13.6; a query of each of 8 sequences of 10920 places x 12
// heads (143 MB) 32, 4.5 TB/s; of 64 (1.14 GB) 193, 5.9 TB/s.  For few bytes the
// time is a chain of latencies (lengths, queries, first codes, join).
constexpr int kFewWaves = 4;

template <int D, int MB>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(MB == 1 ? 3 : 2)))
void attn_few_kernel(AttnCacheArgs a, AttnCachePlan p)
{
    constexpr int KS = D / 32, DB = D / 16, NBLK = D / 32;
    constexpr int V_BYTES = 32 * D * 2;
    constexpr int RED = kFewWaves * 16 * MB * D * 4;
    constexpr int LDS = kFewWaves * V_BYTES > RED ? kFewWaves * V_BYTES : RED;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    __shared__ float stat[kFewWaves][3][16 * MB];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, x = lane & 15;
    const Place w = place_of(a, p);
    const int G = a.H / a.c.heads, rows = a.Sq * G;
    const float c = log2_scale(a.scale);

    bf16x8 q[MB][KS];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) load_q<D>(a, w, w.tile * 16 * MB + mb * 16 + x, G, q[mb]);
    f32x4 o[MB][DB];
    float m[MB], l[MB], r[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        m[mb] = kNone, l[mb] = r[mb] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[mb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int64_t head = ((int64_t)w.b * a.c.heads + w.hk) * a.c.capacity;
    const uint8_t *kc = a.c.k_codes + head * (D / 2), *vc = a.c.v_codes + head * (D / 2);
    const uint8_t *ks = a.c.k_scales + head * NBLK, *vs = a.c.v_scales + head * NBLK;

    // this lane's pieces of a tile: of K, rows x and 16 + x, D / 8 bytes from D / 8 g on;
    // of V, one block (16 bytes) of keys lane / NBLK + 64 / NBLK j.  Past the end the last
    // key again, with no weight: loads without branches are counted, and those of the next
    // tile not waited for (8 sequences of 10920 places, a query each: 40.5 us, 36.1 so; two
    // tiles ahead 35.8, but one query against 32760 17.9 instead of 17.1).
    constexpr int VK = 64 / NBLK, NVJ = 32 / VK;
    struct Piece {
        u32x4 kcode[2], vcode[NVJ];
        uint32_t kscale[2], vscale[NVJ];
    };
    auto load = [&](Piece &t, int key0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t key = min(key0 + 16 * j + x, w.k1 - 1);
            if constexpr (D == 128) {
                t.kcode[j] = *reinterpret_cast<const u32x4 *>(kc + key * 64 + g * 16);
            } else {
                const u32x2 c2 = *reinterpret_cast<const u32x2 *>(kc + key * 32 + g * 8);
                t.kcode[j] = u32x4{c2[0], c2[1], 0, 0};
            }
            t.kscale[j] = ks[key * NBLK + g * NBLK / 4];
        }
#pragma unroll
        for (int j = 0; j < NVJ; ++j) {
            const int64_t key = min(key0 + lane / NBLK + VK * j, w.k1 - 1);
            t.vcode[j] = *reinterpret_cast<const u32x4 *>(vc + key * (D / 2) + lane % NBLK * 16);
            t.vscale[j] = vs[key * NBLK + lane % NBLK];
        }
    };
    lds_char *vl = (lds_char *)smem + wave * V_BYTES;
    const int step = 32 * kFewWaves;
    int key0 = w.k0 + 32 * wave;
    Piece cur, nxt;
    if (key0 < w.k1) load(cur, key0);
    for (; key0 < w.k1; key0 += step) {
        load(nxt, key0 + step);  // in flight beside this tile
        // V to LDS as bf16
#pragma unroll
        for (int j = 0; j < NVJ; ++j) {
            const int row = lane / NBLK + VK * j, blk = lane % NBLK;
            const float sc = scale_bits(cur.vscale[j]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                *(lds_bf16x8 *)(vl + row * D * 2 + v_slot<D>(row, blk * 4 + t) * 16) = decode8(cur.vcode[j][t], sc);
        }
        f32x4 s[MB][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            bf16x8 kf[KS];
            const float sc = scale_bits(cur.kscale[j]);
#pragma unroll
            for (int t = 0; t < KS; ++t) kf[t] = decode8(cur.kcode[j][t], sc);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                s[mb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    s[mb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], q[mb][t], s[mb][j], 0, 0, 0);
            }
        }
        if (key0 + 32 > w.k1) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (key0 + 16 * (i >> 2) + 4 * g + (i & 3) >= w.k1) s[mb][i >> 2][i & 3] = -INFINITY;
        }
        bf16x8 pw[MB];
        float le[MB], re[MB];
        bool over = false;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            weights32(s[mb], c, m[mb], le[mb], re[mb], pw[mb]);
            over |= !(le[mb] <= kSpecLimit);
        }
        if (__builtin_amdgcn_ballot_w64(over) != 0) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                float t = s[mb][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) t = fmaxf(t, s[mb][i >> 2][i & 3]);
                const float mn = fmaxf(m[mb], quad_max(t) * c);
                const float alpha = __builtin_amdgcn_exp2f(m[mb] - mn);
                m[mb] = mn;
                l[mb] *= alpha, r[mb] *= alpha;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[mb][d] *= alpha;
                weights32(s[mb], c, mn, le[mb], re[mb], pw[mb]);
            }
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) l[mb] += le[mb], r[mb] += re[mb];
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const int row = 4 * g + (x >> 2), col = d * 16 + 4 * (x & 3);
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (lds_bf16x4 *)(vl + row * D * 2 + v_slot<D>(row, col >> 3) * 16 + (col & 7) * 2));
            const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (lds_bf16x4 *)(vl + (row + 16) * D * 2 + v_slot<D>(row + 16, col >> 3) * 16 + (col & 7) * 2));
            const bf16x8 vf = {lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pw[mb], o[mb][d], 0, 0, 0);
        }
        cur = nxt;
    }
    // the four waves' results, in a fixed order
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        l[mb] = quad_sum(l[mb]);
        r[mb] = quad_sum(r[mb]);
        if (g == 0) stat[wave][0][mb * 16 + x] = m[mb], stat[wave][1][mb * 16 + x] = l[mb], stat[wave][2][mb * 16 + x] = r[mb];
    }
    __syncthreads();  // also: no wave reads V from LDS any more
    float *sum = reinterpret_cast<float *>(smem) + wave * 16 * MB * D;  // [wave][row][D]
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = mb * 16 + x;
        float mm = stat[0][0][row];
#pragma unroll
        for (int t = 1; t < kFewWaves; ++t) mm = fmaxf(mm, stat[t][0][row]);
        const float f = __builtin_amdgcn_exp2f(m[mb] - mm);
#pragma unroll
        for (int d = 0; d < DB; ++d)
            *reinterpret_cast<f32x4 *>(sum + row * D + (((d * 4 + g) ^ (x & 7)) * 4)) = o[mb][d] * f;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < 16 * MB * (D / 4); t += 64 * kFewWaves) {
        const int row = t / (D / 4), d4 = t % (D / 4);
        const int gr = w.tile * 16 * MB + row;
        if (gr >= rows) continue;
        float mm = stat[0][0][row];
#pragma unroll
        for (int k = 1; k < kFewWaves; ++k) mm = fmaxf(mm, stat[k][0][row]);
        float ll = 0.f, rr = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) {
            const float f = __builtin_amdgcn_exp2f(stat[k][0][row] - mm);
            ll = fmaf(stat[k][1][row], f, ll);
            rr = fmaf(stat[k][2][row], f, rr);
        }
        const bool none = ll == 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k)
            v += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(smem) + (k * 16 * MB + row) * D +
                                                  ((d4 ^ (row & 7)) * 4));
        v = none ? f32x4{0.f, 0.f, 0.f, 0.f} : v * (1.0f / rr);
        const float lse2 = none ? -INFINITY : mm + __builtin_amdgcn_logf(ll);
        const int64_t s = gr / G, h = w.hk * G + gr % G;
        if (p.key_ranges == 1) {
            store_out4(a, w.b, s, h, d4 * 4, v);
            if (d4 == 0 && a.lse != nullptr) a.lse[((int64_t)w.b * a.H + h) * a.Sq + s] = lse2 * kLn2;
        } else {
            *reinterpret_cast<f32x4 *>(part_o(a, w.range, w.b, s, h) + d4 * 4) = v;
            if (d4 == 0) *part_lse(a, p.key_ranges, w.range, w.b, s, h) = lse2;
        }
    }
}

// Many rows: matrix- and vector-bound, on the schedule of the bf16 attention's
// ping-pong kernel.  Eight waves of 32 rows, two per SIMD: waves 0-3 and 4-7
// alternate, in opposite phases, between
//   M(u): matrix instructions only: O^T += V^T P^T of tile u - 1, then S^T = K
//         Q^T of tile u (64 keys), fragments read kAhead of them ahead;
//   V(u): vector instructions only: the weights of tile u, and this wave's part
//         of bringing tile u + 2 to bf16,
// with a barrier between phases, so that a SIMD's matrix unit works for one
// wave while its vector unit works for the other.  A tile is 512 blocks of
// codes at D = 128: one for each lane, K's for waves 0-3 and V's for waves
// 4-7, held from its load a tile earlier, 16 conversions and four LDS stores.
// LDS is a ring of four stages: tile u + 2 goes where tile u - 2 was, whose
// last reads (M(u - 1) of both groups) lie before pair u of phases.  1560
// queries x 32760 places, 12 heads of 128 in 3 ranges: 287 us, 1.09 PFLOP/s;
// matrix units busy for 42 % of the cycles (48 before waves without a row were
// spared) at 2.1 GHz, which is the power limit of the bf16 attention too.
constexpr int kManyWaves = 8, kManyRows = 32 * kManyWaves, kManyKeys = 64;

template <int D>
__global__ __launch_bounds__(64 * kManyWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_many_kernel(AttnCacheArgs a, AttnCachePlan p)
{
    constexpr int KS = D / 32, DB = D / 16, NBLK = D / 32;
    constexpr int T_BYTES = kManyKeys * D * 2, STAGE = 2 * T_BYTES;  // a K or V tile; both
    __shared__ __attribute__((aligned(1024))) char smem[4 * STAGE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave >> 2, g = lane >> 4, x = lane & 15;
    const Place w = place_of(a, p);
    const int G = a.H / a.c.heads, rows = a.Sq * G;
    const int row0 = w.tile * kManyRows + wave * 32;
    const float c = a.scale * kLog2e;
    const int T = (w.k1 - w.k0 + kManyKeys - 1) / kManyKeys;  // tiles
    const bool ragged = (w.k1 - w.k0) % kManyKeys != 0;

    bf16x8 qf[2][KS];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) load_q<D>(a, w, row0 + qb * 16 + x, G, qf[qb]);
    f32x4 o[DB][2], s[4][2];
    bf16x8 pw[2][2];
    float mref[2] = {kNone, kNone}, lsum[2] = {0.f, 0.f}, rsum[2] = {0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][0] = o[db][1] = f32x4{0.f, 0.f, 0.f, 0.f};

    // this lane's block of a tile: waves 0-3 K's, waves 4-7 V's (at D = 64 the first two of each)
    const int64_t first = ((int64_t)w.b * a.c.heads + w.hk) * a.c.capacity + w.k0;
    const int trow = (int)(threadIdx.x & 255) / NBLK, tblk = threadIdx.x % NBLK;
    const bool mine = trow < kManyKeys;
    const uint8_t *codes = (grp ? a.c.v_codes : a.c.k_codes) + first * (D / 2);  // wave-uniform
    const uint8_t *scales = (grp ? a.c.v_scales : a.c.k_scales) + first * NBLK;
    const uint32_t lofs = trow * NBLK + tblk;
    u32x4 code = {0, 0, 0, 0};
    uint32_t byte = 127;
    auto load = [&](int u) __attribute__((always_inline)) {  // of tile u, zeros past the end
        code = u32x4{0, 0, 0, 0};
        byte = 127;
        if (mine && w.k0 + u * kManyKeys + trow < w.k1) {
            code = *reinterpret_cast<const u32x4 *>(codes + (int64_t)u * (kManyKeys * D / 2) + lofs * 16);
            byte = (scales + (int64_t)u * (kManyKeys * NBLK))[lofs];
        }
    };
    int wofs[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
        wofs[t] = grp ? T_BYTES + trow * D * 2 + v_slot<D>(trow, tblk * 4 + t) * 16
                      : trow * D * 2 + k_slot<D>(trow, tblk * 4 + t) * 16;
    auto stage = [&](int u) __attribute__((always_inline)) {  // the held block of tile u to its place
        if (!mine) return;
        const float sc = scale_bits(byte);
        lds_char *dst = (lds_char *)smem + (u & 3) * STAGE;
#pragma unroll
        for (int t = 0; t < 4; ++t) *(lds_bf16x8 *)(dst + wofs[t]) = decode8(code[t], sc);
    };

    int koff[KS], voff[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = x * D * 2 + k_slot<D>(x, D / 32 * g + ks) * 16;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        const int row = 4 * g + (x >> 2), col = db * 16 + 4 * (x & 3);
        voff[db] = T_BYTES + row * D * 2 + v_slot<D>(row, col >> 3) * 16 + (col & 7) * 2;
    }
    constexpr int NK = 4 * KS, NV = 2 * DB, kAhead = 4;
    auto at = [&](int u) { return (const lds_char *)smem + (u & 3) * STAGE; };
    auto kfrag = [&](const lds_char *t, int i) -> bf16x8 {  // i = ks * 4 + kb
        return *(const lds_bf16x8 *)(t + koff[i >> 2] + (i & 3) * 16 * D * 2);
    };
    auto vfrag = [&](const lds_char *t, int i) -> bf16x8 {  // i = ks * DB + db
        const int ks = i / DB, db = i % DB;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(t + voff[db] + ks * 32 * D * 2));
        const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(t + voff[db] + (ks * 32 + 16) * D * 2));
        return bf16x8{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
    };
    using T_ = std::true_type;
    using F_ = std::false_type;
    bf16x8 r[kAhead];
    // the first fragments of M(u), read before the barrier that starts it
    auto mprefetch = [&](int u, auto do_pv) __attribute__((always_inline)) {
        constexpr int N0 = decltype(do_pv)::value ? NV : 0;
        const lds_char *vt = at(u - 1), *kt = at(u);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) r[j] = j < N0 ? vfrag(vt, j) : kfrag(kt, j - N0);
    };
    auto mphase = [&](int u, auto do_pv, auto do_qk) __attribute__((always_inline)) {
        constexpr bool PV = decltype(do_pv)::value, QK = decltype(do_qk)::value;
        constexpr int N0 = PV ? NV : 0, N = N0 + (QK ? NK : 0);
        const lds_char *vt = at(u - 1), *kt = at(u);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j < N0) {
                const int ks = j / DB, db = j % DB;
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
                    o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[j % kAhead], pw[ks][qb], o[db][qb], 0, 0, 0);
            } else {
                const int ks = (j - N0) >> 2, kb = (j - N0) & 3;
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
                    s[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[j % kAhead], qf[qb][ks],
                                                                       ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[kb][qb], 0,
                                                                       0, 0);
            }
            if (j + kAhead < N) r[j % kAhead] = j + kAhead < N0 ? vfrag(vt, j + kAhead) : kfrag(kt, j + kAhead - N0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // weights of tile u; MASK: places from k1 on have none
    auto vphase = [&](int u, auto mask) __attribute__((always_inline)) {
        constexpr bool MASK = decltype(mask)::value;
        const int key0 = w.k0 + u * kManyKeys;
        auto valid = [&](int kb, int i) { return !MASK || key0 + kb * 16 + g * 4 + i < w.k1; };
        float e_sum[2], r_sum[2];
        auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                const float nm = -mref[qb];
                float a0 = -0.f, a1 = -0.f, ar = -0.f;
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        float e0 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][i], c, nm));
                        float e1 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][i + 1], c, nm));
                        e0 = valid(kb, i) ? e0 : 0.f;
                        e1 = valid(kb, i + 1) ? e1 : 0.f;
                        put_pair(pw[kb >> 1][qb], (kb & 1) * 4 + i, e0, e1, ar);
                        a0 += e0;
                        a1 += e1;
                    }
                e_sum[qb] = a0 + a1;
                r_sum[qb] = ar;
            }
        };
        weights();
        if (__builtin_amdgcn_ballot_w64(!(e_sum[0] <= kSpecLimit) || !(e_sum[1] <= kSpecLimit)) != 0) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                float m = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, valid(kb, i) ? s[kb][qb][i] : -INFINITY);
                m = quad_max(m);
                const float mnew = fmaxf(mref[qb], m == -INFINITY ? kNone : m * c);
                const float alpha = __builtin_amdgcn_exp2f(mref[qb] - mnew);
                mref[qb] = mnew;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db][qb] *= alpha;
                lsum[qb] *= alpha;
                rsum[qb] *= alpha;
            }
            weights();
        }
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) lsum[qb] += e_sum[qb], rsum[qb] += r_sum[qb];
    };
    auto vlast = [&]() __attribute__((always_inline)) {
        if (ragged)
            vphase(T - 1, T_{});
        else
            vphase(T - 1, F_{});
    };
    // nothing moves across a barrier between phases, scores and weights included
    auto phase_barrier = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        __asm__ volatile("" : "+v"(s[0][0]), "+v"(s[0][1]), "+v"(s[1][0]), "+v"(s[1][1]), "+v"(s[2][0]),
                         "+v"(s[2][1]), "+v"(s[3][0]), "+v"(s[3][1]));
        __asm__ volatile("" : "+v"(pw[0][0]), "+v"(pw[0][1]), "+v"(pw[1][0]), "+v"(pw[1][1]));
        __builtin_amdgcn_sched_barrier(0);
    };
    // what a V phase does for the ring: tile u + 2 to LDS, tile u + 3 requested
    auto feed = [&](int u) __attribute__((always_inline)) {
        stage(u + 2);
        load(u + 3);
    };

    if (T > 0) {
        load(0);
        stage(0);
        load(1);
        stage(1);
        load(2);
        __syncthreads();
        // Pairs of phases u = 0 .. T - 1, two barriers each in both groups: group 0 runs M(u) | V(u), group 1
        // V(u - 1) | M(u); then the last M (of weights only) of each group.
        if (row0 >= rows) {
            // A wave past the last row only brings its share of the codes, between the same barriers: energy that the
            // clock of the others gets (305 us, 295 so, at the size above).
            __syncthreads();
            if (grp != 0) __syncthreads();
            for (int u = 0; u < T - 1; ++u) {
                feed(u);
                __syncthreads();
                __syncthreads();
            }
            if (grp == 0) __syncthreads();
        } else if (grp == 0) {
            __asm__ volatile("; group 0");
            mprefetch(0, F_{});
            mphase(0, F_{}, T_{});
            phase_barrier();
            for (int u = 0; u < T - 1; ++u) {
                feed(u);
                vphase(u, F_{});
                mprefetch(u + 1, T_{});
                phase_barrier();
                mphase(u + 1, T_{}, T_{});
                phase_barrier();
            }
            vlast();
            mprefetch(T, T_{});
            phase_barrier();
            __asm__ volatile("; last M, group 0");
            mphase(T, T_{}, F_{});
        } else {
            __asm__ volatile("; group 1");
            mprefetch(0, F_{});
            phase_barrier();
            mphase(0, F_{}, T_{});
            phase_barrier();
            for (int u = 1; u < T; ++u) {
                feed(u - 1);
                vphase(u - 1, F_{});
                mprefetch(u, T_{});
                phase_barrier();
                mphase(u, T_{}, T_{});
                phase_barrier();
            }
            vlast();
            mprefetch(T, T_{});
            __asm__ volatile("; last M, group 1");
            mphase(T, T_{}, F_{});
        }
    }
    // lane indices from a fresh copy of the thread index: none stays live across the key loop
    int tid_e = (int)threadIdx.x;
    __asm__ volatile("" : "+v"(tid_e));
    const int g_e = (tid_e & 63) >> 4, x_e = tid_e & 15;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const float ll = quad_sum(lsum[qb]), rr = quad_sum(rsum[qb]);
        const int row = row0 + qb * 16 + x_e;
        if (row >= rows) continue;
        const bool none = ll == 0.f;
        const float inv = none ? 0.f : 1.0f / rr;
        const float lse2 = none ? -INFINITY : mref[qb] + __builtin_amdgcn_logf(ll);
        const int64_t sq = row / G, h = w.hk * G + row % G;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const f32x4 v = o[db][qb] * inv;
            if (p.key_ranges == 1)
                store_out4(a, w.b, sq, h, db * 16 + 4 * g_e, v);
            else
                *reinterpret_cast<f32x4 *>(part_o(a, w.range, w.b, sq, h) + db * 16 + 4 * g_e) = v;
        }
        if (g_e != 0) continue;
        if (p.key_ranges > 1)
            *part_lse(a, p.key_ranges, w.range, w.b, sq, h) = lse2;
        else if (a.lse != nullptr)
            a.lse[((int64_t)w.b * a.H + h) * a.Sq + sq] = lse2 * kLn2;
    }
}

// The key ranges' partial results joined, in order.  Up to kFewRanges of them:
// D / 4 lanes per (query, head), R >= ranges of them read at once (8 ranges of one
// query: 2.1 us less than one by one).  HBM- or cache-bound where there are many rows
// (3 ranges of 1560 x 12 x 128 in f32: 7.5 us, 34 MB).
constexpr int kFewRanges = 8;
template <int D, int R>
__global__ __launch_bounds__(256) void attn_join_few_kernel(AttnCacheArgs a, int ranges)
{
    constexpr int LPR = D / 4;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR;
    if (id >= (int64_t)a.B * a.Sq * a.H) return;
    const int d = threadIdx.x % LPR * 4;
    const int64_t h = id % a.H, s = id / a.H % a.Sq, b = id / ((int64_t)a.H * a.Sq);
    float lse[R];
    f32x4 part[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {  // past the last range that again, with no weight
        lse[k] = *part_lse(a, ranges, min(k, ranges - 1), b, s, h);
        part[k] = *reinterpret_cast<const f32x4 *>(part_o(a, min(k, ranges - 1), b, s, h) + d);
    }
    float m = lse[0];
#pragma unroll
    for (int k = 1; k < R; ++k) m = fmaxf(m, lse[k]);
    m = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const float f = k < ranges ? __builtin_amdgcn_exp2f(lse[k] - m) : 0.f;
        l += f;
        o += part[k] * f;
    }
    store_out4(a, b, s, h, d, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / l));
    if (d == 0 && a.lse != nullptr)
        a.lse[(b * a.H + h) * a.Sq + s] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// More: a workgroup per (query, head), D / 4 lanes along the channels and 1024 /
// D along the ranges, whose sums meet in LDS (12 rows of 42 ranges: 3.3 us, with
// one lane group per row 18).
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnCacheArgs a, int ranges)
{
    constexpr int LPR = D / 4, SL = 256 / LPR;
    __shared__ float weight[64], total;
    __shared__ f32x4 sum[SL][LPR];
    const int t = threadIdx.x, d = t % LPR, slice = t / LPR;
    const int64_t id = blockIdx.x, h = id % a.H, s = id / a.H % a.Sq, b = id / ((int64_t)a.H * a.Sq);
    // requested before the weights are known
    constexpr int KEEP = 64 / SL;
    f32x4 part[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        part[k] = *reinterpret_cast<const f32x4 *>(part_o(a, min(k * SL + slice, ranges - 1), b, s, h) + d * 4);
    if (t < 64) {
        const float e = t < ranges ? *part_lse(a, ranges, t, b, s, h) : -INFINITY;
        float m = e;
#pragma unroll
        for (int i = 32; i >= 1; i >>= 1) m = fmaxf(m, __shfl_xor(m, i, 64));
        m = m == -INFINITY ? 0.f : m;
        const float f = __builtin_amdgcn_exp2f(e - m);
        weight[t] = f;
        float l = f;
#pragma unroll
        for (int i = 32; i >= 1; i >>= 1) l += __shfl_xor(l, i, 64);
        if (t == 0) {
            total = l;
            if (a.lse != nullptr)
                a.lse[(b * a.H + h) * a.Sq + s] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
    }
    __syncthreads();
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (k * SL + slice < ranges) o += part[k] * weight[k * SL + slice];
    sum[slice][d] = o;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int k = 1; k < SL; ++k) o += sum[k][d];
    store_out4(a, b, s, h, d * 4, total == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / total));
}

template <int D>
hipError_t launch_attn_t(const AttnCacheArgs &a, const AttnCachePlan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.c.heads * p.row_tiles * p.key_ranges));
    switch (p.tile_rows) {
    case 16: hipLaunchKernelGGL((attn_few_kernel<D, 1>), grid, dim3(64 * kFewWaves), 0, stream, a, p); break;
    case 32: hipLaunchKernelGGL((attn_few_kernel<D, 2>), grid, dim3(64 * kFewWaves), 0, stream, a, p); break;
    case kManyRows: hipLaunchKernelGGL((attn_many_kernel<D>), grid, dim3(64 * kManyWaves), 0, stream, a, p); break;
    default: return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.key_ranges == 1) return e;
    const int64_t rows = (int64_t)a.B * a.Sq * a.H;
    const dim3 few((unsigned)((rows * (D / 4) + 255) / 256));
    if (p.key_ranges <= 2)
        hipLaunchKernelGGL((attn_join_few_kernel<D, 2>), few, dim3(256), 0, stream, a, p.key_ranges);
    else if (p.key_ranges <= 4)
        hipLaunchKernelGGL((attn_join_few_kernel<D, 4>), few, dim3(256), 0, stream, a, p.key_ranges);
    else if (p.key_ranges <= kFewRanges)
        hipLaunchKernelGGL((attn_join_few_kernel<D, kFewRanges>), few, dim3(256), 0, stream, a, p.key_ranges);
    else
        hipLaunchKernelGGL((attn_join_kernel<D>), dim3((unsigned)rows), dim3(256), 0, stream, a, p.key_ranges);
    return hipGetLastError();
}

}  // namespace

AttnCachePlan attn_cache_plan(int B, int H, int heads, int Sq, int max_len, int D, int n_cu)
{
    AttnCachePlan p{};
    const int64_t rows = (int64_t)Sq * (H / heads);
    p.tile_rows = rows <= 16 ? 16 : rows <= 128 ? 32 : kManyRows;
    p.row_tiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t units = (int64_t)B * heads * p.row_tiles;
    // As many ranges as fill the compute units, with two workgroups of 16 rows or one of more each (measured at 3120 and
    // 10920 places, 12 to 64 units: more cost up to a fifth, for the joining), of at least two rounds of a workgroup's
    // waves; few rows against few places are not cut, which saves the joining launch: at 768 places 7.5 us against 7.6 in
    // 3 ranges with D = 128, at 1024 6.8 against 7.2 in 4 with D = 64.
    const bool many = p.tile_rows == kManyRows;
    const int64_t slots = (int64_t)n_cu * (p.tile_rows == 16 ? 2 : 1);
    const int64_t most = many ? max_len / 512 : (int64_t)max_len * (D + 128) <= 768 * 256 ? 1 : max_len / 256;
    p.key_ranges = (int32_t)std::max<int64_t>(1, std::min({slots / std::max<int64_t>(1, units), most, (int64_t)64}));
    p.ws_bytes = p.key_ranges > 1 ? p.key_ranges * ((int64_t)B * Sq * H * (D + 1)) * (int64_t)sizeof(float) : 0;
    return p;
}

hipError_t launch_append(const AppendArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)a.S * a.c.heads * (a.c.D / 8);
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)a.c.B);
    if (a.c.D == 128)
        hipLaunchKernelGGL(append_kernel<128>, grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(append_kernel<64>, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <int D>
static hipError_t launch_values_t(const ValuesArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)a.c.capacity * a.c.heads * (D / 8);
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)a.c.B);
    if (a.f32)
        hipLaunchKernelGGL((values_kernel<D, true>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((values_kernel<D, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}
hipError_t launch_values(const ValuesArgs &a, hipStream_t stream)
{
    return a.c.D == 128 ? launch_values_t<128>(a, stream) : launch_values_t<64>(a, stream);
}

hipError_t launch_attn_cache(const AttnCacheArgs &a, int n_cu, hipStream_t stream)
{
    const AttnCachePlan p = attn_cache_plan(a.B, a.H, a.c.heads, a.Sq, a.max_len, a.c.D, n_cu);
    return a.c.D == 128 ? launch_attn_t<128>(a, p, stream) : launch_attn_t<64>(a, p, stream);
}

}  // namespace mx
}  // namespace regenvc
