// gfx950 attention of new tokens to a bf16 key/value cache in pages: to all
// places of their sequence, or to the pages that a list selects.
//
// Scores are computed transposed, S^T = K Q^T, on v_mfma_f32_16x16x32_bf16: a
// lane's accumulator holds, for one query row, keys 4 g .. 4 g + 3 of 16 (g =
// lane / 16); rounded to bf16, two of them are the B operand of O^T = V^T P^T in
// the key order {4 g + i, 16 + 4 g + i}, which the transposing LDS reads of V
// follow.  The sum over d of K Q^T is taken in the order in which lane group g
// has the D / 4 channels from D / 4 g on.
//
// Query heads that share a key head are rows of one tile: row r is query r / G
// of head G hk + r % G.  Two running sums per row: O is divided by the sum of
// the weights as rounded to bf16, LSE takes that of the unrounded ones.
//
// Keys go by units of 16 places, which always lie in one page.  A wave reads a
// unit's rows through a buffer descriptor that ends with the last place that its
// tile sees: what lies behind it comes back as zeros, whatever memory holds, as
// do pages that do not exist.  The page numbers of a wave's next units are held
// a lane each.
#include "paged_kernels.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_device.hpp"
#include "paged_device.hpp"

namespace regenvc {
namespace paged {
namespace {

using namespace cache_attn;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 16;
constexpr int kNowhere = 0x3fffffff;  // the place of a unit that does not exist: past every limit
constexpr int kKeyAlign = 64;         // ranges of keys begin at multiples of it
constexpr int kMostRanges = 64;       // of a tile's keys

// Sequences of a call whose keys are cut. Each workgroup goes over all of them to find its piece, and over more of them
// that costs more than ranges give. Single tokens of 4 heads over one key head, D = 128, cut or not: 256 sequences of up to
// 2048 places 45 or 40 us, 65 17 or 26, 100 of up to 32768 216 or 376, 256 of up to 1024 with one of 32768 36 or 292.
constexpr int kMostCut = 256;

// What a workgroup works on: `rows` rows (query, head) of a block of queries, from
// its row `row0` on, and of their keys range `range` of `ranges`, [k0, k1) in units
// of 16.  Key i is place i, or with selected pages place i % page of the page that
// entry i / page names.
struct Work {
    Block blk;
    int hk, row0, rows, range, ranges;
    int part;               // first row of the workgroup's partial results
    int k0, k1;
    int see, least;         // places that its last, its first row sees
    const int32_t *pages;   // the sequence's row of the table
    const int32_t *chosen;  // of the block and key head
};

// Sequences of a call differ in length, which only the device knows, and a long
// one would be the last to end: where there are too few tiles to even that out (the
// plan says so), every wave goes over the sequences, 64 at a time, adds up what there
// is to do, and finds the one that workgroup `id` has a piece of.  Of one sequence
// the tiles that fill whole rounds of slots stay whole, and the keys of the rest are
// cut into as many ranges as the last round has room for: with the join, 264 tiles of 64
// rows and 4096 selected places on 256 slots 85 us, all whole 110; 264 of 256 rows and
// 21840 places (D = 64) 496 and 906.  Those of several are cut at 5/4 of what a slot has
// on the average, those with the longest pieces first.  Seven chunks of 1 to 1365 tokens
// behind 0 to 10663 others, 20 heads on 4: 80 us so; when it was chosen 83, cut at 1 or
// 1.5 of the average 87 and 91, in the order of the call 96, cut by a bound that the host
// has 133 (tiles of 256 rows: each workgroup's begin and end are worth six rounds of
// keys, so that finer pieces cost more than they even out).
struct Piece {
    int b, ranges, tile, range, hk;  // tile -1: no such piece
    int first, rows, len;            // of the sequence
};
template <bool SPARSE>
__device__ __forceinline__ Piece piece_of(const AttnArgs &a, const AttnPlan &p, uint32_t id)
{
    const int lane = threadIdx.x & 63, heads = a.c.heads;
    int first = 0, rows = 0, len = 0, tiles = 0, keys = 0;
    float mean = 0.f;  // keys of a row, on the average
    auto look = [&](int c) {
        const int b = c + lane, at = min(b, a.n.B - 1);
        first = first_of(a.n, at);
        rows = max(0, first_of(a.n, at + 1) - first);
        keys = len = places_of(a.n, at, a.c.shift);
        if constexpr (SPARSE) keys = min(keys, a.count << a.c.shift);
        mean = a.causal && !SPARSE ? max(1.f, keys - 0.5f * min(rows, keys)) : (float)keys;
        tiles = b < a.n.B ? (rows + p.block - 1) / p.block * p.tiles : 0;
    };
    float all = 0.f;
    for (int c = 0; c < a.n.B; c += 64) {
        look(c);
        all += tiles * mean;
    }
    all = wave_sum(all) * heads;
    const bool one = a.n.B == 1;
    const float size = fmaxf((float)p.least, all * (one ? 1.f : 1.25f) / p.slots);
    Piece k{0, 1, -1, 0, 0, 0, 0, 0};
    uint32_t before = 0;
    // Of up to 64, those with the longest pieces first, in three classes by their keys, so that none of them begins late.
    // (Beyond 64, whose lengths are not all at hand, in their order.)
    const int classes = one || a.n.B > 64 ? 1 : 3;
    for (int rank = 0; rank < classes; ++rank)
        for (int c = 0; c < a.n.B; c += 64) {
            if (a.n.B > 64) look(c);
            int skip = 0, most = kMostRanges;
            float longest = size;
            if (one) {  // lane 0: the whole tiles, lane 1: those that are cut
                const uint32_t n = (uint32_t)__builtin_amdgcn_readfirstlane(tiles), rounds = n * heads / (uint32_t)p.fill;
                const uint32_t whole = rounds * p.fill / heads, rest = n - whole;
                most = lane == 0 ? 1 : (int)(((rounds + 1) * p.fill / heads - whole) / max(1u, rest));
                tiles = lane == 0 ? whole : lane == 1 ? rest : 0;
                skip = lane == 0 ? rest : 0;
                if (rounds > 0) longest = (float)p.least;
            }
            // of several, the mean of a row: there are workgroups enough
            const int ranges = max(1, min(min(kMostRanges, most), (int)(one ? floorf(keys / longest) : ceilf(mean / size))));
            const float piece = mean / ranges;
            const bool now = classes == 1 || (piece >= 0.7f * size ? rank == 0 : piece >= 0.3f * size ? rank == 1 : rank == 2);
            const uint32_t mine = now ? (uint32_t)tiles * ranges * heads : 0, upto = before + wave_upto(mine);
            const uint64_t done = __builtin_amdgcn_ballot_w64(upto <= id);
            if (done != ~(uint64_t)0) {
                const int at = __popcll(done);  // upto ascends
                k.b = one ? 0 : c + at;
                k.ranges = __builtin_amdgcn_readlane(ranges, at);
                const uint32_t rest = id - (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), at);
                const uint32_t per = (uint32_t)k.ranges * heads;
                const uint32_t t = rest / per, r2 = rest - t * per;
                k.tile = __builtin_amdgcn_readlane(tiles + skip, at) - 1 - (int)t;  // the last first: in a causal call it has the most keys
                k.range = (int)(r2 / (uint32_t)heads);
                k.hk = (int)r2 - k.range * heads;
                k.first = __builtin_amdgcn_readlane(first, at);
                k.rows = __builtin_amdgcn_readlane(rows, at);
                k.len = __builtin_amdgcn_readlane(len, at);
                return k;
            }
            before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
    return k;
}

template <bool SPARSE>
__device__ __forceinline__ Work work_of(const AttnArgs &a, const AttnPlan &p)
{
    Work w;
    const int heads = a.c.heads, G = a.H / heads;
    int64_t j;
    w.rows = w.range = w.part = 0;
    w.ranges = 1;
    w.k0 = w.k1 = w.see = w.least = 0;
    if (p.split) {
        const Piece k = piece_of<SPARSE>(a, p, blockIdx.x);
        if (k.tile < 0) return w;
        const int i = p.tiles == 1 ? k.tile : __builtin_amdgcn_readfirstlane(k.tile / p.tiles), at = i * p.block;  // at < rows: the tile exists
        w.blk.b = __builtin_amdgcn_readfirstlane(k.b);
        w.blk.row = k.first + at;
        w.blk.rows = min(p.block, k.rows - at);
        w.blk.len = k.len;
        w.blk.pos = k.len - k.rows + at;
        j = !SPARSE ? 0 : (p.block == 1 ? k.first : (int64_t)(k.first / p.block)) + w.blk.b + i;
        w.row0 = __builtin_amdgcn_readfirstlane((k.tile - i * p.tiles) * p.tile_rows);
        w.hk = __builtin_amdgcn_readfirstlane(k.hk);
        w.range = __builtin_amdgcn_readfirstlane(k.range);
        w.ranges = __builtin_amdgcn_readfirstlane(k.ranges);
        w.part = (int)blockIdx.x * p.tile_rows;
    } else {
        // key head, then tile, then block, the last block first
        const uint32_t id = gridDim.x - 1 - blockIdx.x, q = id / (uint32_t)heads;
        w.hk = (int)(id - q * heads);
        j = q / (uint32_t)p.tiles;
        w.row0 = (int)(q - j * p.tiles) * p.tile_rows;
        w.blk = block_of(a.n, a.c.shift, p.block, j);
    }
    w.rows = max(0, min(p.tile_rows, w.blk.rows * G - w.row0));
    w.pages = a.n.table + w.blk.b * a.n.table_stride;
    w.chosen = nullptr;
    if (w.rows == 0) return w;
    const int first = w.blk.pos + (w.row0 == 0 ? 0 : w.row0 / G), last = w.blk.pos + (w.row0 + w.rows - 1) / G;
    w.see = a.causal ? max(0, last + 1) : w.blk.len;
    w.least = a.causal ? max(0, first + 1) : w.blk.len;
    int keys = w.see;
    if constexpr (SPARSE) {
        w.chosen = a.selected + (j * heads + w.hk) * a.count;
        keys = a.count << a.c.shift;
    }
    const uint32_t units = ((uint32_t)keys + kKeyAlign - 1) / kKeyAlign;  // < 2^24, ranges <= 64
    w.k0 = w.ranges == 1 ? 0 : (int)(units * w.range / w.ranges) * kKeyAlign;
    w.k1 = w.ranges == 1 ? keys : min(keys, (int)(units * (w.range + 1) / w.ranges) * kKeyAlign);
    return w;
}
// Where the keys end: with selected pages, behind the list's last entry that is not none.  Apart from work_of, so that the
// list is read beside what else a workgroup begins with.
template <bool SPARSE>
__device__ __forceinline__ int end_of(const AttnArgs &a, const Work &w)
{
    if constexpr (!SPARSE) return w.k1;
    int n = 0;
    for (int i = threadIdx.x & 63; i < a.count; i += 64)
        if (w.chosen[i] >= 0) n = i + 1;
    return min(w.k1, (int)__builtin_amdgcn_readfirstlane(wave_max(n)) << a.c.shift);
}

// Where the unit from key i on lies: its page in the pool (-1: nowhere) and its first place.
struct Unit {
    int page, place;
};
template <bool SPARSE>
__device__ __forceinline__ Unit unit_at(const AttnArgs &a, const Work &w, int i)
{
    Unit u{-1, kNowhere};
    if (i >= w.k1) return u;
    int col = i >> a.c.shift, place = i;
    if constexpr (SPARSE) {
        col = w.chosen[col];
        if (col < 0 || col >= a.n.columns) return u;
        place = (col << a.c.shift) + (i & ((1 << a.c.shift) - 1));
    }
    if (place >= w.see) return u;
    const int page = w.pages[col];
    if (page < 0 || page >= a.c.pages) return u;
    u.page = page;
    u.place = place;
    return u;
}

// A buffer descriptor of the unit's rows of one head, as many as its tile sees: loads behind them give zeros.
template <int D>
__device__ __forceinline__ u32x4 rows_of(const AttnArgs &a, const Work &w, uint16_t *base, int page, int place)
{
    const int n = __builtin_amdgcn_readfirstlane(max(0, min(kUnit, w.see - place)));  // uniform as it is, in a scalar
    const int64_t row = (((int64_t)max(page, 0) * a.c.heads + w.hk) << a.c.shift) + (place & ((1 << a.c.shift) - 1));
    const uint64_t at = (uint64_t)(base + row * D);
    return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffff, (uint32_t)(n * D * 2), 0x00027000};
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(u32x4 r)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)r[1] << 32 | r[0]), 0, (int)r[2], (int)r[3]);
}
__device__ __forceinline__ u32x4 load_rows(__amdgpu_buffer_rsrc_t r, int at, int imm)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + imm, 0, 0));
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// N loads of 16 bytes a lane from a descriptor's rows to LDS, lane i's 16 bytes of load j to dst + 1024 j + 16 i from 1024 j
// + at[j] on.  Inline, because the compiler would wait for them before every later LDS read; who reads them waits by
// itself.  The nops: scalars written just before, M0 too.
template <int N>
__device__ __forceinline__ void rows_to_lds(uint32_t dst, const uint32_t (&at)[N], u32x4 r)
{
    static_assert(N == 2 || N == 4, "16 rows of 128 or 256 bytes");
    if constexpr (N == 4)
        __asm__ volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                         "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 lds\n\t"
                         "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 lds\n\t"
                         "buffer_load_dwordx4 %4, %5, 0 offen offset:%6 lds"
                         : : "s"(dst), "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(r), "n"(3 * 1024) : "m0", "memory");
    else
        __asm__ volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                         "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
                         : : "s"(dst), "v"(at[0]), "v"(at[1]), "s"(r) : "m0", "memory");
}
#pragma clang diagnostic pop

// Partial results of the workgroups whose tile has more than one range, in the
// workspace: O (f32, normalized over the range) [workgroup][row of the tile][D],
// then LSE in log2 units [workgroup][row] (-inf: no key), then for each [row of the
// call][head] where its first range is and how many there are (1: the result is in
// place).  Ranges of a tile are as many workgroups apart as there are key heads.
struct Parts {
    int first, ranges;
};
__device__ __forceinline__ float *part_o(const AttnArgs &a, int64_t row)
{
    return reinterpret_cast<float *>(a.ws) + row * a.c.D;
}
__device__ __forceinline__ float *part_lse(const AttnArgs &a, const AttnPlan &p, int64_t row)
{
    return reinterpret_cast<float *>(a.ws) + (int64_t)p.groups * p.tile_rows * a.c.D + row;
}
__device__ __forceinline__ Parts *parts_of(const AttnArgs &a, const AttnPlan &p, int64_t t, int64_t h)
{
    return reinterpret_cast<Parts *>(a.ws + (int64_t)p.groups * p.tile_rows * (a.c.D + 1) * 4) + t * a.H + h;
}
__device__ __forceinline__ void store_out4(const AttnArgs &a, int64_t t, int64_t h, int d, f32x4 v)
{
    const int64_t at = t * a.o_ss + h * a.o_sh + d;
    if (a.f32) {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.o) + at) = v;
    } else {
        const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.o) + at) = o;
    }
}

// LSE of row `row` of the tile, token t and head h.
__device__ __forceinline__ void store_lse(const AttnArgs &a, const AttnPlan &p, const Work &w, int row, int64_t t, int64_t h,
                                          float lse2)
{
    if (p.split && w.range == 0) *parts_of(a, p, t, h) = Parts{w.part + row, w.ranges};
    if (w.ranges > 1)
        *part_lse(a, p, w.part + row) = lse2;
    else if (a.lse != nullptr)
        a.lse[h * a.n.T + t] = lse2 * kLn2;
}

// Row r of the tile: the channels D / 4 g + 8 s + 0..7 of it for s < D / 32, and the places that it sees.
template <int D>
__device__ __forceinline__ int load_q(const AttnArgs &a, const Work &w, int r, int G, bf16x8 (&q)[D / 32])
{
    const int g = (threadIdx.x & 63) >> 4, at = w.row0 + max(0, min(r, w.rows - 1));
    const int query = at / G;
    const uint16_t *p = a.q + (int64_t)(w.blk.row + query) * a.q_ss + (int64_t)(w.hk * G + at - query * G) * a.q_sh + D / 4 * g;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 8 * s);
    return a.causal ? max(0, w.blk.pos + query + 1) : w.blk.len;
}

__device__ __forceinline__ bool finite4(f32x4 v)
{
    return fmaf(v[3], 0.f, fmaf(v[2], 0.f, fmaf(v[1], 0.f, v[0] * 0.f))) == 0.f;
}

// Places that row `row` of a causal tile sees.
__device__ __forceinline__ int sees(const Work &w, int row, int G)
{
    return max(0, w.blk.pos + (w.row0 + row) / G + 1);
}

// One past the last place that some rows of a causal tile see and others do not (at least w.least, before w.see) and whose
// value is not finite in some channel.  Without such a place, w.least or less.  Every lane of the wave takes part and gets
// the answer.  A tile has no more such places than queries.
template <int D, bool SPARSE>
__device__ __forceinline__ int foul_end(const AttnArgs &a, const Work &w)
{
    constexpr int CH = D / 8, VR = 64 / CH, NL = kUnit / VR;  // 16-byte chunks of a row, rows that a load takes, loads
    const int lane = threadIdx.x & 63;
    uint32_t end = 0;
    for (int i0 = SPARSE ? w.k0 : max(w.k0, w.least & -kUnit); i0 < w.k1; i0 += 64 * kUnit) {
        const Unit u = unit_at<SPARSE>(a, w, i0 + lane * kUnit);
        uint64_t mixed = __builtin_amdgcn_ballot_w64(u.page >= 0 && u.place + kUnit > w.least);
        for (; mixed != 0; mixed &= mixed - 1) {
            const int at = __builtin_ctzll(mixed);
            const int page = __builtin_amdgcn_readlane(u.page, at), place = __builtin_amdgcn_readlane(u.place, at);
            const __amdgpu_buffer_rsrc_t r = resource(rows_of<D>(a, w, a.c.v, page, place));  // zeros from w.see on
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const u32x4 x = load_rows(r, lane * 16, j * 1024);
                bool foul = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) foul |= (x[e] & 0x7f80) == 0x7f80 || (x[e] & 0x7f800000) == 0x7f800000;
                if (foul) end = max(end, (uint32_t)(place + VR * j + lane / CH + 1));
            }
        }
    }
    return (int)wave_max(end);
}

// Row `row` of the tile by one wave, a key to a lane, with only the places that it
// sees.  The matrix products of a causal tile take a weight of 0 times the values of
// places that some of its rows do not see: where those hold an infinity or NaN,
// the product is NaN, and the row is done again here.  A row that is not finite
// by what it sees alone is right as it is (foul_end tells the two apart).  Off every
// path of finite values, and slow: a row and 64 keys take about 9 us, a wave's rows one
// after another.  10920 causal queries x 12 heads of 128 with a NaN in the first value 0.55
// ms (all of their rows done again: 135), in the last one 48, in every value 57.
template <int D, bool SPARSE>
__device__ __forceinline__ void redo_row(const AttnArgs &a, const AttnPlan &p, const Work &w, int row)
{
    constexpr int PER = D / 64, kAhead = 8;
    const int lane = threadIdx.x & 63, G = a.H / a.c.heads;
    const int at = w.row0 + row, query = at / G;
    const int64_t tok = w.blk.row + query, h = w.hk * G + at - query * G;
    const int lim = sees(w, row, G);
    const uint16_t *q = a.q + tok * a.q_ss + h * a.q_sh;
    const float c = log2_scale(a.scale);
    auto wide = [](uint32_t u) { return __uint_as_float(u << 16); };
    float m = kNone, l = 0.f, r = 0.f, o[PER] = {};
    for (int i0 = w.k0; i0 < w.k1; i0 += 64) {
        const int i = i0 + lane;
        const Unit u = unit_at<SPARSE>(a, w, i & -kUnit);
        const bool see = u.page >= 0 && u.place + (i & (kUnit - 1)) < lim;
        const int64_t cell = (((int64_t)max(u.page, 0) * a.c.heads + w.hk) << a.c.shift) +
                             (see ? (u.place + (i & (kUnit - 1))) & ((1 << a.c.shift) - 1) : 0);
        float s = -INFINITY;
        if (see) {
            s = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 8) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(q + d), y = *reinterpret_cast<const u32x4 *>(a.c.k + cell * D + d);
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fmaf(wide(x[e] >> 16), wide(y[e] >> 16), fmaf(wide(x[e]), wide(y[e]), s));
            }
        }
        float top = s;
#pragma unroll
        for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        const float mn = fmaxf(m, top * c), alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        const float e = see ? __builtin_amdgcn_exp2f(fmaf(s, c, -m)) : 0.f, er = (float)(__bf16)e;
        l = l * alpha + wave_sum(e);
        r = r * alpha + wave_sum(er);
#pragma unroll
        for (int k = 0; k < PER; ++k) o[k] *= alpha;
        const uint64_t seen = __builtin_amdgcn_ballot_w64(see);
#pragma unroll 1
        for (int k0 = 0; k0 < 64; k0 += kAhead) {
            if ((seen >> k0 & ((1u << kAhead) - 1)) == 0) continue;
            uint16_t v[kAhead][PER];  // of a key that the row does not see: a row of page 0, with no part in the sum
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const uint32_t l = __builtin_amdgcn_readlane((int)cell, k0 + k), h = __builtin_amdgcn_readlane((int)(cell >> 32), k0 + k);
                const uint16_t *from = a.c.v + (int64_t)((uint64_t)h << 32 | l) * D + lane;
#pragma unroll
                for (int n = 0; n < PER; ++n) v[k][n] = from[64 * n];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(er), k0 + k));
                const bool part = seen >> (k0 + k) & 1;
#pragma unroll
                for (int n = 0; n < PER; ++n) o[n] = fmaf(x, part ? wide(v[k][n]) : 0.f, o[n]);
            }
        }
    }
    const bool none = l == 0.f;
#pragma unroll
    for (int n = 0; n < PER; ++n) {
        const int d = lane + 64 * n;
        const float v = none ? 0.f : o[n] / r;
        if (w.ranges > 1)
            part_o(a, w.part + row)[d] = v;
        else if (a.f32)
            static_cast<float *>(a.o)[tok * a.o_ss + h * a.o_sh + d] = v;
        else
            static_cast<__bf16 *>(a.o)[tok * a.o_ss + h * a.o_sh + d] = (__bf16)v;
    }
    if (lane == 0) store_lse(a, p, w, row, tok, h, none ? -INFINITY : m + __builtin_amdgcn_logf(l));
}

// Few rows (tiles of 16 MB): memory-bound.  Every wave walks key tiles of its
// own, 32 keys at a time, with nothing shared: K goes from memory to registers
// and the matrix unit; V through 2 D x 32 bytes of wave-private LDS, for the
// transposition.  The waves' results meet in LDS.
//
// 16 rows: eight waves, so that few places need no second launch to join ranges
// (1024 keys are four rounds); more rows take the registers of two waves each.
// One query against 32760 places x 12 heads of 128 (201 MB): 39 us, 5.1 TB/s, and
// 4.9 for the join of 21 ranges; queries of 16 sequences of 1 to 10920 places, 16
// heads of 64 on 4 (75 MB): 16.1 + 4.0.  16 pages of 64 for one query: 10.9 + 4.0,
// of which a chain of eight dependent loads has most (sequence, list, table, keys).
// 64 rows: 25 blocks of 64 queries x 12 heads with 64 pages of 64 each (629 MB from
// the caches, 321 from HBM): 85 us and 5 for the join, 252 tiles whole and 48 in five
// ranges each, at the rate of what lies behind the L2; all whole it took 111.  The
// next tile's scores beside a tile's weights (142 us instead of 135, with the
// selection) or every tile's keys in three ranges (149) lose.
constexpr int few_waves(int rows) { return attn_threads(rows) / 64; }

template <int D, int MB, bool SPARSE>
__global__ __launch_bounds__(64 * few_waves(16 * MB)) __attribute__((amdgpu_waves_per_eu(MB == 1 ? 2 : 1)))
void attn_few_kernel(AttnArgs a, AttnPlan p)
{
    constexpr int kFewWaves = few_waves(16 * MB);
    constexpr int KS = D / 32, DB = D / 16, CH = D / 8;  // CH: 16-byte chunks of a row
    constexpr int VR = 64 / CH, NVJ = 32 / VR;           // rows of V that a load of the wave takes, and the loads
    constexpr int V_BYTES = 32 * D * 2;
    constexpr int RED = kFewWaves * 16 * MB * D * 4;
    constexpr int LDS = kFewWaves * V_BYTES > RED ? kFewWaves * V_BYTES : RED;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    __shared__ float stat[kFewWaves][3][16 * MB];
    __shared__ int again[16 * MB];
    const int lane = threadIdx.x & 63, g = lane >> 4, x = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Work w = work_of<SPARSE>(a, p);
    if (w.rows <= 0) return;
    const int G = a.H / a.c.heads;
    const float c = log2_scale(a.scale);

    bf16x8 q[MB][KS];
    int lim[MB];  // places that this lane's rows see
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) lim[mb] = load_q<D>(a, w, mb * 16 + x, G, q[mb]);
    f32x4 o[MB][DB];
    float m[MB], l[MB], r[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        m[mb] = kNone, l[mb] = r[mb] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[mb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Units of this wave's tiles i = 0, 1, ... (keys key_of(i) .. + 31), two each: lane 32 h + i % 32 holds half h of tile
    // i of 32, and those of the 32 tiles after them.
    const int step = 32 * kFewWaves, begin = w.k0 + 32 * wave;
    auto units = [&](int i0) { return unit_at<SPARSE>(a, w, begin + (i0 + (lane & 31)) * step + (lane >> 5) * kUnit); };
    Unit now = units(0), later = units(32);
    const int tiles = max(0, (end_of<SPARSE>(a, w) - begin + step - 1) / step);
    struct Piece {
        u32x4 k[2][KS], v[NVJ];
        int place[2];
    };
    // Tile i's rows, asked for in order.  Without a branch (there may be no such tile: zeros, and no memory is read), so that
    // they are counted and not waited for.
    auto load = [&](Piece &t, int i) __attribute__((always_inline)) {
        if ((i & 31) == 0 && i > 0) {
            now = later;
            later = units(i + 32);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = __builtin_amdgcn_readlane(now.page, (i & 31) + 32 * h);
            const int place = __builtin_amdgcn_readlane(now.place, (i & 31) + 32 * h);
            t.place[h] = place;
            const __amdgpu_buffer_rsrc_t rk = resource(rows_of<D>(a, w, a.c.k, page, place));
            const __amdgpu_buffer_rsrc_t rv = resource(rows_of<D>(a, w, a.c.v, page, place));
#pragma unroll
            for (int s = 0; s < KS; ++s) t.k[h][s] = load_rows(rk, x * D * 2 + g * D / 2, s * 16);
#pragma unroll
            for (int j = 0; j < NVJ / 2; ++j) t.v[h * (NVJ / 2) + j] = load_rows(rv, lane * 16, j * 1024);
        }
    };
    lds_char *vl = (lds_char *)smem + wave * V_BYTES;
    // Tile i, and then its registers to tile i + 2: between them and the next one's, two tiles are in flight.
    auto one = [&](Piece &cur, int i) __attribute__((always_inline)) {
        const int place[2] = {cur.place[0], cur.place[1]};
#pragma unroll
        for (int j = 0; j < NVJ; ++j) {
            const int row = lane / CH + VR * j;
            *(__attribute__((address_space(3))) u32x4 *)(vl + row * D * 2 + v_slot<D>(row, lane % CH) * 16) = cur.v[j];
        }
        f32x4 s[MB][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                s[mb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    s[mb][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, cur.k[h][t]), q[mb][t],
                                                                       s[mb][h], 0, 0, 0);
            }
        load(cur, i + 2);
        if (max(place[0], place[1]) + kUnit > w.least) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (place[e >> 2] + 4 * g + (e & 3) >= lim[mb]) s[mb][e >> 2][e & 3] = -INFINITY;
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
                for (int e = 1; e < 8; ++e) t = fmaxf(t, s[mb][e >> 2][e & 3]);
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
    };
    Piece even, odd;
    load(even, 0);
    load(odd, 1);
    for (int i = 0; i < tiles; i += 2) {
        one(even, i);
        if (i + 1 >= tiles) break;
        one(odd, i + 1);
    }
    // the waves' results, in a fixed order
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
        if (row >= w.rows) continue;
#pragma unroll
        for (int d = 0; d < DB; ++d)
            *reinterpret_cast<f32x4 *>(sum + row * D + (((d * 4 + g) ^ (x & 7)) * 4)) = o[mb][d] * f;
    }
    const bool apart = a.causal && w.see > w.least;  // rows of the tile see different places
    if (apart && threadIdx.x < 16 * MB) again[threadIdx.x] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < w.rows * (D / 4); t += 64 * kFewWaves) {
        const int row = t / (D / 4), d4 = t % (D / 4);
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
        const int at = w.row0 + row, query = at / G;  // 32 bits: a division of 64 takes longer than the row
        const int64_t tok = w.blk.row + query, h = w.hk * G + at - query * G;
        if (apart && !finite4(v)) again[row] = 1;
        if (w.ranges == 1)
            store_out4(a, tok, h, d4 * 4, v);
        else
            *reinterpret_cast<f32x4 *>(part_o(a, w.part + row) + d4 * 4) = v;
        if (d4 == 0) store_lse(a, p, w, row, tok, h, lse2);
    }
    if (!apart) return;
    __syncthreads();
    int foul = -1;  // not looked for yet
    for (int row = wave; row < w.rows; row += kFewWaves) {
        if (__builtin_amdgcn_readfirstlane(again[row]) == 0) continue;
        if (foul < 0) foul = foul_end<D, SPARSE>(a, w);
        if (foul > sees(w, row, G)) redo_row<D, SPARSE>(a, p, w, row);
    }
}

// Many rows: matrix- and vector-bound, on the schedule of the other caches'
// attention.  Eight waves of 32 rows, two per SIMD: waves 0-3 and 4-7 alternate, in
// opposite phases, between
//   M(u): matrix instructions only: O^T += V^T P^T of tile u - 1, then S^T = K
//         Q^T of tile u (64 keys), fragments read kAhead of them ahead;
//   V(u): vector instructions only: the weights of tile u, and this wave's part of
//         tile u + 3 (K's for waves 0-3, V's for waves 4-7) asked for, to LDS,
// with a barrier between phases, so that a SIMD's matrix unit works for one
// wave while its vector unit works for the other.  LDS is a ring of four stages:
// tile u + 3 goes where tile u - 1 was.  Its K was last read by M(u - 1) of waves
// 4-7, its V by M(u) of waves 4-7: a barrier before V(u) of the waves that load it.
// Scores of places that a row does not see are set to -inf before one form of the
// weights (with a form for either, 90 registers spilled: 409 us instead of 335).
// 10920 causal queries x 12 heads of 128: 332-352 us from card to card, 1.04-1.10 PFLOP/s,
// matrix units busy for 51 % of the cycles, no LDS conflicts; 1560 queries against 32760
// places: 295-310 us in three ranges and 8 for their join; both at the power limit.
constexpr int kManyWaves = 8, kManyRows = 32 * kManyWaves, kManyKeys = 64;
static_assert(attn_threads(kManyRows) == 64 * kManyWaves, "what the plan counts on");

template <int D, bool SPARSE>
__global__ __launch_bounds__(64 * kManyWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_many_kernel(AttnArgs a, AttnPlan p)
{
    constexpr int KS = D / 32, DB = D / 16, CH = D / 8;  // CH: 16-byte chunks of a row
    constexpr int T_BYTES = kManyKeys * D * 2, STAGE = 2 * T_BYTES;  // a K or V tile; both
    __shared__ __attribute__((aligned(1024))) char smem[4 * STAGE];
    __shared__ int holes[kManyWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave >> 2, g = lane >> 4, x = lane & 15;
    const Work w = work_of<SPARSE>(a, p);
    if (w.rows <= 0) return;
    const int G = a.H / a.c.heads;
    const int row0 = wave * 32;  // of the tile
    const float c = log2_scale(a.scale);

    bf16x8 qf[2][KS];
    int lim[2];  // places that this lane's rows see, less its first key of a unit
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) lim[qb] = load_q<D>(a, w, row0 + qb * 16 + x, G, qf[qb]) - 4 * g;
    f32x4 o[DB][2], s[4][2];
    bf16x8 pw[2][2];
    float mref[2] = {kNone, kNone}, lsum[2] = {0.f, 0.f}, rsum[2] = {0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][0] = o[db][1] = f32x4{0.f, 0.f, 0.f, 0.f};

    // This wave's unit of a tile: K's (waves 0-3) or V's (4-7) rows 16 (wave % 4) .. + 15.  Lane i has where it lies in
    // tile i of 64, and in those of the 64 tiles after them.
    const int mine = (wave & 3) * kUnit;
    uint16_t *const base = grp ? a.c.v : a.c.k;  // wave-uniform
    constexpr int VR = 64 / CH, NL = kUnit / VR;  // rows that a load of the wave takes, and the loads
    auto units = [&](int u0) { return unit_at<SPARSE>(a, w, w.k0 + (u0 + lane) * kManyKeys + mine); };
    Unit now = units(0), later = units(64);
    // Whether a page of those units does not exist: then all waves look every tile's pages up again.
    auto hole = [&](const Unit &x, int u0) {
        return __builtin_amdgcn_ballot_w64(x.page < 0 && w.k0 + (u0 + lane) * kManyKeys + mine < w.k1) != 0;
    };
    if (!SPARSE) holes[wave] = hole(now, 0) || hole(later, 64);
    const int T = max(0, (end_of<SPARSE>(a, w) - w.k0 + kManyKeys - 1) / kManyKeys);  // tiles of keys
    // Where a load of the wave finds what its lanes' places in LDS hold: chunks change places with the row (v_slot, k_slot).
    uint32_t vofs[NL];
#pragma unroll
    for (int j = 0; j < NL; ++j) {
        const int row = VR * j + lane / CH, ch = lane % CH;
        vofs[j] = lane / CH * D * 2 + (grp ? v_slot<D>(row, ch) : k_slot<D>(row, ch)) * 16;
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_char *)smem + (grp ? T_BYTES : 0) + mine * D * 2);
    auto load = [&](int u) __attribute__((always_inline)) {  // tile u to LDS, asked for in order; zeros where there is none
        if ((u & 63) == 0 && u > 0) {
            now = later;
            later = units(u + 64);
            if (!SPARSE && hole(later, u + 64)) holes[wave] = 1;  // read 61 tiles later or more
        }
        const u32x4 r = rows_of<D>(a, w, base, __builtin_amdgcn_readlane(now.page, u & 63),
                                   __builtin_amdgcn_readlane(now.place, u & 63));
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + (u & 3) * STAGE);
        rows_to_lds(dst, vofs, r);
    };
    // the loads of all tiles but the last two asked for have landed
    auto landed = [&]() __attribute__((always_inline)) { __asm__ volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * NL) : "memory"); };
    // The first places of a tile's four units: with selected pages lane i has those of tile i of 64.
    int at4[4] = {kNowhere, kNowhere, kNowhere, kNowhere};
    int gaps = 0;
    auto firsts = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) at4[t] = unit_at<SPARSE>(a, w, w.k0 + (u + lane) * kManyKeys + t * kUnit).place;
    };
    if constexpr (SPARSE) firsts(0);
    auto places = [&](int u, int (&pl)[4]) __attribute__((always_inline)) {
        if constexpr (SPARSE) {
            if ((u & 63) == 0 && u > 0) firsts(u);
#pragma unroll
            for (int t = 0; t < 4; ++t) pl[t] = __builtin_amdgcn_readlane(at4[t], u & 63);
        } else {
            if ((u & 63) == 0) gaps = __builtin_amdgcn_readfirstlane(holes[0] | holes[1] | holes[2] | holes[3]);
#pragma unroll
            for (int t = 0; t < 4; ++t) pl[t] = w.k0 + u * kManyKeys + t * kUnit;
            if (gaps != 0) {
#pragma unroll
                for (int t = 0; t < 4; ++t) pl[t] = __builtin_amdgcn_readfirstlane(unit_at<SPARSE>(a, w, pl[t]).place);
            }
        }
    };

    // Fragments in LDS: chunk D / 32 g + ks of K's row x (and 16, 32, 48 rows on), channels 16 db + 4 (x % 4) of V's row 4 g +
    // x / 4.  ks and db change bits of the address that no other term of it has: an exclusive or instead of a register.
    const uint32_t koff = x * D * 2 + k_slot<D>(x, D / 32 * g) * 16;
    const uint32_t voff = T_BYTES + (4 * g + (x >> 2)) * D * 2 + v_slot<D>(4 * g + (x >> 2), (x & 3) >> 1) * 16 + (x & 1) * 8;
    constexpr int NK = 4 * KS, NV = 2 * DB, kAhead = 4;
    auto at = [&](int u) { return (u & 3) * STAGE; };
    auto kfrag = [&](uint32_t t, int i) -> bf16x8 {  // i = ks * 4 + kb
        return *(const lds_bf16x8 *)((lds_char *)smem + ((t + koff) ^ (i >> 2) * 16) + (i & 3) * 16 * D * 2);
    };
    auto vfrag = [&](uint32_t t, int i) -> bf16x8 {  // i = ks * DB + db
        lds_char *p = (lds_char *)smem + ((t + voff) ^ (i % DB) * 32) + i / DB * 32 * D * 2;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)p);
        const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(p + 16 * D * 2));
        return bf16x8{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
    };
    using T_ = std::true_type;
    using F_ = std::false_type;
    bf16x8 r[kAhead];
    // the first fragments of M(u), read before the barrier that starts it
    auto mprefetch = [&](int u, auto do_pv) __attribute__((always_inline)) {
        constexpr int N0 = decltype(do_pv)::value ? NV : 0;
        const uint32_t vt = at(u - 1), kt = at(u);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) r[j] = j < N0 ? vfrag(vt, j) : kfrag(kt, j - N0);
    };
    auto mphase = [&](int u, auto do_pv, auto do_qk) __attribute__((always_inline)) {
        constexpr bool PV = decltype(do_pv)::value, QK = decltype(do_qk)::value;
        constexpr int N0 = PV ? NV : 0, N = N0 + (QK ? NK : 0);
        const uint32_t vt = at(u - 1), kt = at(u);
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
    // weights of tile u
    auto vphase = [&](int u) __attribute__((always_inline)) {
        int pl[4];
        places(u, pl);
        if (max(max(pl[0], pl[1]), max(pl[2], pl[3])) + kUnit > w.least) {  // some row does not see some place of it
            int end[2] = {lim[0], lim[1]};
            __asm__ volatile("" : "+v"(end[0]), "+v"(end[1]));  // else eight limits are kept across the loop
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int qb = 0; qb < 2; ++qb)
                        if (pl[kb] + i >= end[qb]) s[kb][qb][i] = -INFINITY;
        }
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
                        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][i], c, nm));
                        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][i + 1], c, nm));
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
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, s[kb][qb][i]);
                const float mnew = fmaxf(mref[qb], quad_max(m) * c);
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
    // what a V phase does for the ring: tile u + 3 asked for, tile u + 1 there
    auto feed = [&](int u) __attribute__((always_inline)) {
        load(u + 3);
        landed();
    };

    if (T > 0) {
        load(0);
        load(1);
        load(2);
        landed();
        __syncthreads();
        // Pairs of phases u = 0 .. T - 1, two barriers each in both groups: group 0 runs M(u) | V(u), group 1
        // V(u - 1) | M(u); then the last M (of weights only) of each group.
        if (row0 >= w.rows) {
            // A wave past the last row only brings its share of the keys, between the same barriers.
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
                vphase(u);
                mprefetch(u + 1, T_{});
                phase_barrier();
                mphase(u + 1, T_{}, T_{});
                phase_barrier();
            }
            vphase(T - 1);
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
                vphase(u - 1);
                mprefetch(u, T_{});
                phase_barrier();
                mphase(u, T_{}, T_{});
                phase_barrier();
            }
            vphase(T - 1);
            mprefetch(T, T_{});
            __asm__ volatile("; last M, group 1");
            mphase(T, T_{}, F_{});
        }
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" : : : "memory");  // nothing lands in LDS after the workgroup
    // lane indices from a fresh copy of the thread index: none stays live across the key loop
    int tid_e = (int)threadIdx.x;
    __asm__ volatile("" : "+v"(tid_e));
    const int g_e = (tid_e & 63) >> 4, x_e = tid_e & 15;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const float ll = quad_sum(lsum[qb]), rr = quad_sum(rsum[qb]);
        const int row = row0 + qb * 16 + x_e;
        const bool none = ll == 0.f;
        const float inv = none ? 0.f : 1.0f / rr;
        const float lse2 = none ? -INFINITY : mref[qb] + __builtin_amdgcn_logf(ll);
        const int at = w.row0 + row, query = at / G;  // 32 bits: a division of 64 takes longer than the row
        const int64_t tok = w.blk.row + query, h = w.hk * G + at - query * G;
        bool bad = false;
        if (row < w.rows) {
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const f32x4 v = o[db][qb] * inv;
                bad |= !finite4(v);
                if (w.ranges == 1)
                    store_out4(a, tok, h, db * 16 + 4 * g_e, v);
                else
                    *reinterpret_cast<f32x4 *>(part_o(a, w.part + row) + db * 16 + 4 * g_e) = v;
            }
            if (g_e == 0) store_lse(a, p, w, row, tok, h, lse2);
        }
        uint64_t rows_bad = __builtin_amdgcn_ballot_w64(bad);
        if (rows_bad != 0 && a.causal && w.see > w.least) {
            rows_bad |= rows_bad >> 32, rows_bad |= rows_bad >> 16;  // lane x of a row has it
            // the stores above are this wave's own and come before
            __asm__ volatile("s_waitcnt vmcnt(0)" : : : "memory");
            const int foul = foul_end<D, SPARSE>(a, w);
            for (int i = 0; i < 16; ++i) {
                const int r = row0 + qb * 16 + i;
                if ((rows_bad >> i & 1) && foul > sees(w, r, G)) redo_row<D, SPARSE>(a, p, w, r);
            }
        }
    }
}

// Whether row t belongs to a sequence: no other is written.
__device__ __forceinline__ bool covered(const Batch &n, int64_t t)
{
    return t >= n.first[0] && t < n.first[n.B];
}

constexpr int kFewRows = 2048;

// A row's partial results, where there is more than one range; what lies beyond the
// workspace is none (only of `first` that does not ascend).
__device__ __forceinline__ bool joined(const AttnArgs &a, const AttnPlan &p, int64_t t, int64_t h, Parts &k)
{
    k = *parts_of(a, p, t, h);  // of a row of no sequence: anything
    return covered(a.n, t) && k.ranges > 1 && k.ranges <= kMostRanges && k.first >= 0 &&
           k.first + (int64_t)(k.ranges - 1) * a.c.heads * p.tile_rows < (int64_t)p.groups * p.tile_rows;
}

// The key ranges' partial results joined, in order.  Many rows: D / 4 lanes per
// (row, head), kAtOnce ranges read at once.
constexpr int kAtOnce = 4;
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, AttnPlan p)
{
    constexpr int LPR = D / 4;
    const uint32_t id = blockIdx.x * (256u / LPR) + threadIdx.x / LPR, token = id / (uint32_t)a.H;  // at most 2^29
    if (token >= (uint32_t)a.n.T) return;
    const int d = threadIdx.x % LPR * 4;
    const int64_t h = id - token * a.H, t = token, step = (int64_t)a.c.heads * p.tile_rows;
    Parts k;
    if (!joined(a, p, t, h, k)) return;
    float m = kNone, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < k.ranges; r += kAtOnce) {
        float lse[kAtOnce];
        f32x4 part[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {  // past the last range that again, with no weight
            const int64_t row = k.first + min(r + i, k.ranges - 1) * step;
            lse[i] = *part_lse(a, p, row);
            part[i] = *reinterpret_cast<const f32x4 *>(part_o(a, row) + d);
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) mn = fmaxf(mn, lse[i]);
        const float f0 = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f0;
        o *= f0;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const float f = r + i < k.ranges ? __builtin_amdgcn_exp2f(lse[i] - m) : 0.f;
            l += f;
            o += part[i] * f;
        }
    }
    store_out4(a, t, h, d, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / l));
    if (d == 0 && a.lse != nullptr) a.lse[h * a.n.T + t] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Few rows, of many ranges each: a workgroup per (row, head), D / 4 lanes along the
// channels and 1024 / D along the ranges, whose sums meet in LDS.
template <int D>
__global__ __launch_bounds__(256) void attn_join_few_kernel(AttnArgs a, AttnPlan p)
{
    constexpr int LPR = D / 4, SL = 256 / LPR, KEEP = kMostRanges / SL;
    __shared__ float weight[kMostRanges], total;
    __shared__ f32x4 sum[SL][LPR];
    const int i = threadIdx.x, d = i % LPR, slice = i / LPR;
    const uint32_t token = blockIdx.x / (uint32_t)a.H;
    const int64_t h = blockIdx.x - token * a.H, t = token, step = (int64_t)a.c.heads * p.tile_rows;
    Parts k;
    if (!joined(a, p, t, h, k)) return;
    f32x4 part[KEEP];  // requested before the weights are known
#pragma unroll
    for (int n = 0; n < KEEP; ++n) {
        part[n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (n * SL < k.ranges)
            part[n] = *reinterpret_cast<const f32x4 *>(part_o(a, k.first + min(n * SL + slice, k.ranges - 1) * step) + d * 4);
    }
    if (i < 64) {
        const float e = i < k.ranges ? *part_lse(a, p, k.first + i * step) : -INFINITY;
        float m = e;
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
        m = m == -INFINITY ? 0.f : m;
        const float f = __builtin_amdgcn_exp2f(e - m);
        weight[i] = f;
        const float l = wave_sum(f);
        if (i == 0) {
            total = l;
            if (a.lse != nullptr) a.lse[h * a.n.T + t] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
    }
    __syncthreads();
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < KEEP; ++n)
        if (n * SL + slice < k.ranges) o += part[n] * weight[n * SL + slice];
    sum[slice][d] = o;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int n = 1; n < SL; ++n) o += sum[n][d];
    store_out4(a, t, h, d * 4, total == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.0f / total));
}

template <int D, bool SPARSE>
hipError_t launch_tiles(const AttnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.groups), block((unsigned)attn_threads(p.tile_rows));
    switch (p.tile_rows) {
    case 16: hipLaunchKernelGGL((attn_few_kernel<D, 1, SPARSE>), grid, block, 0, stream, a, p); break;
    case 32: hipLaunchKernelGGL((attn_few_kernel<D, 2, SPARSE>), grid, block, 0, stream, a, p); break;
    case 64: hipLaunchKernelGGL((attn_few_kernel<D, 4, SPARSE>), grid, block, 0, stream, a, p); break;
    case kManyRows: hipLaunchKernelGGL((attn_many_kernel<D, SPARSE>), grid, block, 0, stream, a, p); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    const hipError_t e = a.selected != nullptr ? launch_tiles<D, true>(a, p, stream) : launch_tiles<D, false>(a, p, stream);
    if (e != hipSuccess || !p.split) return e;
    const int64_t rows = (int64_t)a.n.T * a.H;
    if (rows <= kFewRows)
        hipLaunchKernelGGL((attn_join_few_kernel<D>), dim3((unsigned)rows), dim3(256), 0, stream, a, p);
    else
        hipLaunchKernelGGL((attn_join_kernel<D>), dim3((unsigned)((rows * (D / 4) + 255) / 256)), dim3(256), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace

AttnPlan attn_plan(const AttnShape &s, int n_cu)
{
    AttnPlan p{};
    const int64_t G = s.H / s.heads, queries = s.count > 0 ? std::min(s.q_block, s.max_rows) : s.max_rows;
    // rows of a sequence (of a block of queries) that share a key head: at most, and on the average
    const int64_t most = queries * G, mean = s.count > 0 ? most : std::min(most, (s.T + (int64_t)s.B - 1) / s.B * G);
    p.tile_rows = most <= 16 || mean <= 16 ? 16 : most <= 32 || mean <= 32 ? 32 : most <= 64 || mean <= 64 ? 64 : kManyRows;
    // Up to 64 rows in two tiles while those leave compute units free: 64 rows of 12 heads against 10920 places 29 us, in one
    // 34; 25 blocks of 64 queries of 12 heads, 64 pages of 64 each, in one 117 us, in two 236 (all tiles whole).
    const int64_t sequences = s.count > 0 ? (int64_t)s.T / s.q_block + s.B : s.B;
    if (p.tile_rows == 64 && 2 * sequences * s.heads <= n_cu) p.tile_rows = 32;
    p.block = s.count > 0 ? s.q_block : (int)std::max<int64_t>(1, p.tile_rows / G);
    p.tiles = (int)((std::min(p.block, s.T) * G + p.tile_rows - 1) / p.tile_rows);
    // workgroups that run at once: two of 32 rows of 64 channels to a compute unit, or one of any other
    p.slots = n_cu * (p.tile_rows == 32 && s.D == 64 ? 2 : 1);
    p.least = p.tile_rows == kManyRows ? 512 : 256;
    const int64_t blocks = (int64_t)s.T / p.block + s.B, most_blocks = s.B == 1 ? (s.T + (int64_t)p.block - 1) / p.block : blocks;
    const int64_t tiles = std::min<int64_t>(most_blocks, s.T) * p.tiles * s.heads;
    const int64_t keys = s.count > 0 ? std::min<int64_t>(s.max_len, (int64_t)s.count * s.page) : s.max_len;
    // Keys are cut where there are too few tiles for their number to even out the differences, at least into two ranges of
    // `least` keys.  Workgroups: piece_of makes at most one to a tile and one to a slot; of one sequence whole rounds (`fill`)
    // of one to a slot, or two where its tiles may differ much, as those of many rows of a short causal one do.
    const int64_t rounds = s.B > 1 || s.count > 0 || !s.causal || 4 * (int64_t)s.max_rows <= s.max_len ? 1 : 2;
    p.fill = (int)rounds * p.slots;
    const int64_t n = tiles / s.heads, full = s.B == 1 ? tiles / p.fill : 0, whole = full * p.fill / s.heads;
    const bool room = s.B == 1 ? n > whole && ((full + 1) * p.fill / s.heads - whole) / (n - whole) >= 2
                               : tiles < 4 * (int64_t)p.slots && s.B <= kMostCut;
    // Behind whole rounds the join has to be worth a round's saving.  Blocks of 64 queries of 12 heads of 128 with 1024, 2048,
    // 4096 places of a list each, all whole or cut: 324 tiles 54 or 56, 76 or 74, 113 or 100 us; 516 of them 79 or 78, 114 or
    // 104, 169 or 144 (with 512 places 41 or 44, 61 or 64).  Up to four, as partial results of all are in the workspace.
    if (full == 0)
        p.split = room && keys >= (p.tile_rows == 16 && 8 * tiles > p.slots ? 6 : 2) * p.least;
    else
        p.split = room && rounds == 1 && full <= 4 && keys >= 4 * full * p.least;
    p.groups = !p.split ? blocks * p.tiles * s.heads : s.B > 1 ? tiles + p.slots : (full + 1) * p.fill;
    p.ws_bytes = p.split ? (p.groups * p.tile_rows * (int64_t)(s.D + 1) + 2 * (int64_t)s.T * s.H) * (int64_t)sizeof(float) : 0;
    return p;
}

hipError_t launch_attn(const AttnArgs &a, const AttnPlan &p, hipStream_t stream)
{
    return a.c.D == 128 ? launch_d<128>(a, p, stream) : launch_d<64>(a, p, stream);
}

}  // namespace paged
}  // namespace regenvc
