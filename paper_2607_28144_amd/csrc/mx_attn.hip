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

#include "mx_device.hpp"

namespace regenvc {
namespace mx {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;

// ---------------------------------------------------------------- append, read back
// One lane per eight channels of a token's head; blockIdx.y: k or v.
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    const int per = a.c.D / 8;  // lanes of a head's row
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t n = (int64_t)a.c.B * a.S * a.c.heads * per;
    const bool in = id < n;
    const int64_t at = in ? id : 0;
    const int chunk = (int)(at % per);
    const int h = (int)(at / per % a.c.heads);
    const int i = (int)(at / ((int64_t)per * a.c.heads) % a.S);
    const int b = (int)(at / ((int64_t)per * a.c.heads * a.S));
    const int count = a.count != nullptr ? min(a.count[b], a.S) : a.S;
    const int start = a.start != nullptr ? a.start[b] : 0;
    const bool is_v = blockIdx.y != 0;
    const uint16_t *src = static_cast<const uint16_t *>(is_v ? a.v : a.k) + b * (is_v ? a.v_sb : a.k_sb) +
                          i * (is_v ? a.v_ss : a.k_ss) + h * (is_v ? a.v_sh : a.k_sh) + chunk * 8;
    // of more tokens than the cache holds, only the last ones: no two tokens share a place
    const bool live = in && i < count && (int64_t)i + a.c.capacity >= count && start >= 0;
    float x[8] = {};
    if (live) {
        const bf16x8 q = *reinterpret_cast<const bf16x8 *>(src);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (float)q[k];
    }
    uint32_t code;
    const uint32_t byte = quantize_quad(x, code);
    if (!live) return;
    const int place = (int)(((int64_t)start + i) % a.c.capacity);
    const int64_t token = ((int64_t)b * a.c.heads + h) * a.c.capacity + place;
    *reinterpret_cast<uint32_t *>((is_v ? a.c.v_codes : a.c.k_codes) + token * (a.c.D / 2) + chunk * 4) = code;
    if ((chunk & 3) == 0) (is_v ? a.c.v_scales : a.c.k_scales)[token * (a.c.D / 32) + chunk / 4] = (uint8_t)byte;
}

template <bool F32>
__global__ __launch_bounds__(256) void values_kernel(ValuesArgs a)
{
    const int per = a.c.D / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)a.c.B * a.c.capacity * a.c.heads * per) return;
    const int chunk = (int)(id % per);
    const int h = (int)(id / per % a.c.heads);
    const int64_t tok = id / ((int64_t)per * a.c.heads);  // b * capacity + place
    const int64_t token = (tok / a.c.capacity * a.c.heads + h) * a.c.capacity + tok % a.c.capacity;
    const bool is_v = blockIdx.y != 0;
    const uint32_t code =
        *reinterpret_cast<const uint32_t *>((is_v ? a.c.v_codes : a.c.k_codes) + token * (a.c.D / 2) + chunk * 4);
    const float s = scale_value((is_v ? a.c.v_scales : a.c.k_scales)[token * (a.c.D / 32) + chunk / 4]);
    const bf16x8 v = decode8(code, 1.0f);
    void *out = is_v ? a.v : a.k;
    if constexpr (F32) {
        float *o = static_cast<float *>(out) + id * 8;
#pragma unroll
        for (int h4 = 0; h4 < 2; ++h4)
            *reinterpret_cast<f32x4 *>(o + 4 * h4) = f32x4{(float)v[4 * h4] * s, (float)v[4 * h4 + 1] * s,
                                                           (float)v[4 * h4 + 2] * s, (float)v[4 * h4 + 3] * s};
    } else {
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)((float)v[i] * s);
        *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(out) + id * 8) = o;
    }
}

// ---------------------------------------------------------------- attention
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -3.0e38f;  // a running maximum before any key: below every score, and finite

// x combined over the lanes l, l^16, l^32, l^48 (each gets the result).
__device__ __forceinline__ float quad_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float quad_sum(float x)
{
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

// 16-byte chunk of a V row in LDS (2 D bytes a row) where chunk c of key row r
// is kept: pairs of chunks change places with the row, so that neither the
// stores of whole blocks nor the transposing reads (4 rows by 32 bytes per 16
// lanes) meet in a bank.
template <int D>
__device__ __forceinline__ int v_slot(int r, int c)
{
    return c ^ ((r & (D / 16 - 1)) << 1);
}

// The same for K rows: the fragment reads take one chunk of each of 16 rows.
template <int D>
__device__ __forceinline__ int k_slot(int r, int c)
{
    return c ^ (D == 128 ? r & 15 : (r >> 1) & 7);
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
    int id = blockIdx.x;
    w.range = id % p.key_ranges;
    id /= p.key_ranges;
    w.tile = id % p.row_tiles;
    id /= p.row_tiles;
    w.hk = id % a.c.heads;
    w.b = id / a.c.heads;
    int len = a.lens != nullptr ? a.lens[w.b] : a.max_len;
    w.len = len = max(0, min(len, a.c.capacity));
    const int64_t units = (len + kKeyAlign - 1) / kKeyAlign;
    w.k0 = (int)(units * w.range / p.key_ranges) * kKeyAlign;
    w.k1 = min(len, (int)(units * (w.range + 1) / p.key_ranges) * kKeyAlign);
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

// Weights of 32 keys (8 of them this lane's) for one row: p in bf16, the
// running maximum m (log2 units) raised, alpha the factor for what was summed
// under the old one.
__device__ __forceinline__ void softmax32(const f32x4 (&s)[2], float c, float &m, float &lsum, float &rsum, float &alpha,
                                          bf16x8 &p)
{
    float t = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = fmaxf(t, s[i >> 2][i & 3]);
    t = quad_max(t) * c;
    const float mn = fmaxf(m, t);
    alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    float l = 0.f, r = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c, -mn));
        p[i] = (__bf16)e;
        l += e;
        r += (float)p[i];
    }
    lsum = fmaf(lsum, alpha, l);  // over this lane's keys; the lanes' sums are joined at the end
    rsum = fmaf(rsum, alpha, r);
}

// Few rows (up to 16 MB for a key head): memory-bound.  Every wave walks key
// tiles of its own, 32 keys at a time, with nothing shared: K's codes go from
// memory to registers and the matrix unit; V's through 2 D x 32 bytes of
// wave-private LDS, for the transposition.  The waves' results meet in LDS.
constexpr int kFewWaves = 4;

template <int D, int MB>
__global__ __launch_bounds__(64 * kFewWaves) void attn_few_kernel(AttnCacheArgs a, AttnCachePlan p)
{
    constexpr int KS = D / 32, DB = D / 16, NBLK = D / 32;
    constexpr int V_BYTES = 32 * D * 2;
    constexpr int RED = 16 * MB * D * 4;
    constexpr int LDS = kFewWaves * V_BYTES > RED ? kFewWaves * V_BYTES : RED;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    __shared__ float stat[kFewWaves][3][16 * MB];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, x = lane & 15;
    const Place w = place_of(a, p);
    const int G = a.H / a.c.heads, rows = a.Sq * G;
    const float c = log2_scale(a.scale);

    bf16x8 q[MB][KS];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) load_q<D>(a, w, mb * 16 + x, G, q[mb]);
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
    // of V, one block (16 bytes) of keys lane / NBLK + 64 / NBLK j.  Keys past the end: zeros.
    constexpr int VK = 64 / NBLK, NVJ = 32 / VK;
    u32x4 kcode[2], vcode[NVJ];
    uint32_t kscale[2], vscale[NVJ];
    auto load = [&](int key0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = key0 + 16 * j + x;
            kcode[j] = u32x4{0, 0, 0, 0};
            kscale[j] = 127;
            if (key < w.k1) {
                if constexpr (D == 128) {
                    kcode[j] = *reinterpret_cast<const u32x4 *>(kc + (int64_t)key * 64 + g * 16);
                } else {
                    const u32x2 t = *reinterpret_cast<const u32x2 *>(kc + (int64_t)key * 32 + g * 8);
                    kcode[j][0] = t[0], kcode[j][1] = t[1];
                }
                kscale[j] = ks[(int64_t)key * NBLK + g * NBLK / 4];
            }
        }
#pragma unroll
        for (int j = 0; j < NVJ; ++j) {
            const int key = key0 + lane / NBLK + VK * j;
            vcode[j] = u32x4{0, 0, 0, 0};
            vscale[j] = 127;
            if (key < w.k1) {
                vcode[j] = *reinterpret_cast<const u32x4 *>(vc + (int64_t)key * (D / 2) + lane % NBLK * 16);
                vscale[j] = vs[(int64_t)key * NBLK + lane % NBLK];
            }
        }
    };
    lds_char *vl = (lds_char *)smem + wave * V_BYTES;
    const int step = 32 * kFewWaves;
    int key0 = w.k0 + 32 * wave;
    if (key0 < w.k1) load(key0);
    for (; key0 < w.k1; key0 += step) {
        // V to LDS as bf16
#pragma unroll
        for (int j = 0; j < NVJ; ++j) {
            const int row = lane / NBLK + VK * j, blk = lane % NBLK;
            const float sc = scale_bits(vscale[j]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                *(lds_bf16x8 *)(vl + row * D * 2 + v_slot<D>(row, blk * 4 + t) * 16) = decode8(vcode[j][t], sc);
        }
        f32x4 s[MB][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            bf16x8 kf[KS];
            const float sc = scale_bits(kscale[j]);
#pragma unroll
            for (int t = 0; t < KS; ++t) kf[t] = decode8(kcode[j][t], sc);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                s[mb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    s[mb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], q[mb][t], s[mb][j], 0, 0, 0);
            }
        }
        const int at = key0;
        if (key0 + step < w.k1) load(key0 + step);  // in flight beside the rest of this tile
        if (at + 32 > w.k1) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at + 16 * (i >> 2) + 4 * g + (i & 3) >= w.k1) s[mb][i >> 2][i & 3] = -INFINITY;
        }
        bf16x8 pw[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            float alpha;
            softmax32(s[mb], c, m[mb], l[mb], r[mb], alpha, pw[mb]);
#pragma unroll
            for (int d = 0; d < DB; ++d) o[mb][d] *= alpha;
        }
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
    }
    // the four waves' results, in a fixed order
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        l[mb] = quad_sum(l[mb]);
        r[mb] = quad_sum(r[mb]);
        if (g == 0) stat[wave][0][mb * 16 + x] = m[mb], stat[wave][1][mb * 16 + x] = l[mb], stat[wave][2][mb * 16 + x] = r[mb];
    }
    __syncthreads();  // also: no wave reads V from LDS any more
    float *sum = reinterpret_cast<float *>(smem);  // [row][D]
    for (int k = 0; k < kFewWaves; ++k) {
        if (wave == k) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const int row = mb * 16 + x;
                float mm = stat[0][0][row];
#pragma unroll
                for (int t = 1; t < kFewWaves; ++t) mm = fmaxf(mm, stat[t][0][row]);
                const float f = __builtin_amdgcn_exp2f(m[mb] - mm);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    f32x4 *z = reinterpret_cast<f32x4 *>(sum + row * D + (((d * 4 + g) ^ (x & 7)) * 4));
                    *z = k == 0 ? o[mb][d] * f : *z + o[mb][d] * f;
                }
            }
        }
        __syncthreads();
    }
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
        f32x4 v = *reinterpret_cast<const f32x4 *>(sum + row * D + ((d4 ^ (row & 7)) * 4));
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

// Many rows: matrix-bound.  Four waves of 32 rows share tiles of 64 keys,
// which they bring to bf16 together, a tile ahead, into LDS of two stages; two
// workgroups per compute unit, so that one's exponentials run beside the
// other's matrix instructions.
constexpr int kManyWaves = 4, kManyRows = 32 * kManyWaves, kManyKeys = 64;

template <int D>
__global__ __launch_bounds__(64 * kManyWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_many_kernel(AttnCacheArgs a, AttnCachePlan p)
{
    constexpr int KS = D / 32, DB = D / 16, NBLK = D / 32, MB = 2, KB = kManyKeys / 16;
    constexpr int T_BYTES = kManyKeys * D * 2;  // a K or V tile
    __shared__ __attribute__((aligned(1024))) char smem[4 * T_BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, x = lane & 15;
    const Place w = place_of(a, p);
    const int G = a.H / a.c.heads, rows = a.Sq * G;
    const int row0 = w.tile * kManyRows + wave * 32;
    const float c = log2_scale(a.scale);

    bf16x8 q[MB][KS];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) load_q<D>(a, w, row0 + mb * 16 + x, G, q[mb]);
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

    // a lane's block of a tile (of the first half of the lanes at D = 64)
    const int trow = threadIdx.x / NBLK, tblk = threadIdx.x % NBLK;
    const bool mine = trow < kManyKeys;
    u32x4 kcode, vcode;
    uint32_t kscale, vscale;
    auto load = [&](int key0) {
        const int64_t key = key0 + trow;
        kcode = vcode = u32x4{0, 0, 0, 0};
        kscale = vscale = 127;
        if (mine && key < w.k1) {
            kcode = *reinterpret_cast<const u32x4 *>(kc + key * (D / 2) + tblk * 16);
            vcode = *reinterpret_cast<const u32x4 *>(vc + key * (D / 2) + tblk * 16);
            kscale = ks[key * NBLK + tblk];
            vscale = vs[key * NBLK + tblk];
        }
    };
    auto stage = [&](int st) {
        if (!mine) return;
        lds_char *kl = (lds_char *)smem + st * 2 * T_BYTES, *vl = kl + T_BYTES;
        const float sk = scale_bits(kscale), sv = scale_bits(vscale);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            *(lds_bf16x8 *)(kl + trow * D * 2 + k_slot<D>(trow, tblk * 4 + t) * 16) = decode8(kcode[t], sk);
            *(lds_bf16x8 *)(vl + trow * D * 2 + v_slot<D>(trow, tblk * 4 + t) * 16) = decode8(vcode[t], sv);
        }
    };
    int st = 0;
    if (w.k0 < w.k1) {
        load(w.k0);
        stage(0);
        load(w.k0 + kManyKeys);
    }
    for (int key0 = w.k0; key0 < w.k1; key0 += kManyKeys, st ^= 1) {
        __syncthreads();  // the tile is there; the other stage is no longer read
        const lds_char *kl = (const lds_char *)smem + st * 2 * T_BYTES, *vl = kl + T_BYTES;
        if (key0 + kManyKeys < w.k1) {
            stage(st ^ 1);
            load(key0 + 2 * kManyKeys);
        }
        f32x4 s[MB][KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) s[mb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const int row = kb * 16 + x;
                const bf16x8 kf = *(const lds_bf16x8 *)(kl + row * D * 2 + k_slot<D>(row, D / 32 * g + t) * 16);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    s[mb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[mb][t], s[mb][kb], 0, 0, 0);
            }
        }
        if (key0 + kManyKeys > w.k1) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + 16 * kb + 4 * g + i >= w.k1) s[mb][kb][i] = -INFINITY;
        }
        bf16x8 pw[MB][KB / 2];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            float t = s[mb][0][0];
#pragma unroll
            for (int i = 1; i < 4 * KB; ++i) t = fmaxf(t, s[mb][i >> 2][i & 3]);
            const float mn = fmaxf(m[mb], quad_max(t) * c);
            const float alpha = __builtin_amdgcn_exp2f(m[mb] - mn);
            m[mb] = mn;
            float ll = 0.f, rr = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * KB; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[mb][i >> 2][i & 3], c, -mn));
                const __bf16 pb = (__bf16)e;
                pw[mb][i >> 3][i & 7] = pb;
                ll += e;
                rr += (float)pb;
            }
            l[mb] = fmaf(l[mb], alpha, ll);
            r[mb] = fmaf(r[mb], alpha, rr);
#pragma unroll
            for (int d = 0; d < DB; ++d) o[mb][d] *= alpha;
        }
#pragma unroll
        for (int kk = 0; kk < KB / 2; ++kk)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int row = 32 * kk + 4 * g + (x >> 2), col = d * 16 + 4 * (x & 3);
                const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                    (lds_bf16x4 *)(vl + row * D * 2 + v_slot<D>(row, col >> 3) * 16 + (col & 7) * 2));
                const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                    (lds_bf16x4 *)(vl + (row + 16) * D * 2 + v_slot<D>(row + 16, col >> 3) * 16 + (col & 7) * 2));
                const bf16x8 vf = {lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    o[mb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pw[mb][kk], o[mb][d], 0, 0, 0);
            }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const float ll = quad_sum(l[mb]), rr = quad_sum(r[mb]);
        const int row = row0 + mb * 16 + x;
        if (row >= rows) continue;
        const bool none = ll == 0.f;
        const float inv = none ? 0.f : 1.0f / rr;
        const float lse2 = none ? -INFINITY : m[mb] + __builtin_amdgcn_logf(ll);
        const int64_t sq = row / G, h = w.hk * G + row % G;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const f32x4 v = o[mb][d] * inv;
            if (p.key_ranges == 1)
                store_out4(a, w.b, sq, h, d * 16 + 4 * g, v);
            else
                *reinterpret_cast<f32x4 *>(part_o(a, w.range, w.b, sq, h) + d * 16 + 4 * g) = v;
        }
        if (g != 0) continue;
        if (p.key_ranges > 1)
            *part_lse(a, p.key_ranges, w.range, w.b, sq, h) = lse2;
        else if (a.lse != nullptr)
            a.lse[((int64_t)w.b * a.H + h) * a.Sq + sq] = lse2 * kLn2;
    }
}

// The key ranges' partial results joined, in order: D / 4 lanes per (query, head).
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnCacheArgs a, int ranges)
{
    constexpr int LPR = D / 4;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR;
    if (id >= (int64_t)a.B * a.Sq * a.H) return;
    const int d = threadIdx.x % LPR * 4;
    const int64_t h = id % a.H, s = id / a.H % a.Sq, b = id / ((int64_t)a.H * a.Sq);
    float m = -INFINITY;
    for (int k = 0; k < ranges; ++k) m = fmaxf(m, *part_lse(a, ranges, k, b, s, h));
    const float m0 = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < ranges; ++k) {
        const float e = *part_lse(a, ranges, k, b, s, h);
        const float f = __builtin_amdgcn_exp2f(e - m0);
        l += f;
        o += *reinterpret_cast<const f32x4 *>(part_o(a, k, b, s, h) + d) * f;
    }
    store_out4(a, b, s, h, d, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / l));
    if (d == 0 && a.lse != nullptr)
        a.lse[(b * a.H + h) * a.Sq + s] = l == 0.f ? -INFINITY : (m0 + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D>
hipError_t launch_attn_t(const AttnCacheArgs &a, const AttnCachePlan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.c.heads * p.row_tiles * p.key_ranges));
    switch (p.tile_rows) {
    case 16: hipLaunchKernelGGL((attn_few_kernel<D, 1>), grid, dim3(64 * kFewWaves), 0, stream, a, p); break;
    case 32: hipLaunchKernelGGL((attn_few_kernel<D, 2>), grid, dim3(64 * kFewWaves), 0, stream, a, p); break;
    case 64: hipLaunchKernelGGL((attn_few_kernel<D, 4>), grid, dim3(64 * kFewWaves), 0, stream, a, p); break;
    case kManyRows: hipLaunchKernelGGL((attn_many_kernel<D>), grid, dim3(64 * kManyWaves), 0, stream, a, p); break;
    default: return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.key_ranges == 1) return e;
    const int64_t lanes = (int64_t)a.B * a.Sq * a.H * (D / 4);
    hipLaunchKernelGGL((attn_join_kernel<D>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, a, p.key_ranges);
    return hipGetLastError();
}

}  // namespace

AttnCachePlan attn_cache_plan(int B, int H, int heads, int Sq, int max_len, int D, int n_cu)
{
    AttnCachePlan p{};
    const int64_t rows = (int64_t)Sq * (H / heads);
    p.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : kManyRows;
    p.row_tiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t units = (int64_t)B * heads * p.row_tiles;
    // workgroups side by side; a range is at least two rounds of a workgroup's waves
    const int64_t slots = (int64_t)n_cu * 2;
    const int64_t most = std::max<int64_t>(1, max_len / (p.tile_rows == kManyRows ? 512 : 256));
    p.key_ranges = (int32_t)std::max<int64_t>(1, std::min({slots / std::max<int64_t>(1, units), most, (int64_t)64}));
    p.ws_bytes = p.key_ranges > 1 ? p.key_ranges * ((int64_t)B * Sq * H * (D + 1)) * (int64_t)sizeof(float) : 0;
    return p;
}

hipError_t launch_append(const AppendArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)a.c.B * a.S * a.c.heads * (a.c.D / 8);
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)((n + 255) / 256), 2), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_values(const ValuesArgs &a, hipStream_t stream)
{
    const int64_t n = (int64_t)a.c.B * a.c.capacity * a.c.heads * (a.c.D / 8);
    const dim3 grid((unsigned)((n + 255) / 256), 2);
    if (a.f32)
        hipLaunchKernelGGL(values_kernel<true>, grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(values_kernel<false>, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_attn_cache(const AttnCacheArgs &a, int n_cu, hipStream_t stream)
{
    const AttnCachePlan p = attn_cache_plan(a.B, a.H, a.c.heads, a.Sq, a.max_len, a.c.D, n_cu);
    return a.c.D == 128 ? launch_attn_t<128>(a, p, stream) : launch_attn_t<64>(a, p, stream);
}

}  // namespace mx
}  // namespace regenvc
