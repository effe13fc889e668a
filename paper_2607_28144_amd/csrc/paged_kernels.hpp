// Internal launch interface of the kernels of a bf16 key/value cache in pages.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace regenvc {
namespace paged {

// Keys and values bf16 [pages, heads, 2^shift, D], means bf16 [pages, heads, D].
struct Pool {
    uint16_t *k, *v, *means;
    int32_t pages, shift, heads, D;
};
// The sequences of a call (int32 in device memory): table [B, columns], first [B + 1], lens [B].
struct Batch {
    const int32_t *table, *first, *lens;
    int64_t table_stride;
    int32_t B, columns, T;
};

// q, k, v, q_out: bf16 [T, heads, D] with strides; H = 0 without q.
struct AppendArgs {
    Pool c;
    Batch n;
    const uint16_t *q, *k, *v, *w_q, *w_k;
    uint16_t *q_out;
    int64_t q_ss, q_sh, k_ss, k_sh, v_ss, v_sh, o_ss, o_sh;
    const double *turns;
    int32_t H, pairs, interleaved;
    float eps, amplitude;
};
hipError_t launch_append(const AppendArgs &a, int n_cu, hipStream_t stream);

// selected: int32 [blocks, heads, count]; n.B = 0: blocks without queries.
struct SelectArgs {
    Pool c;
    Batch n;
    const uint16_t *q;
    int64_t q_ss, q_sh;
    int32_t *selected;
    int32_t H, q_block, count, keep_first, keep_last, causal;
};
constexpr int kMaxSelectColumns = 16384;  // a score of 64 bits each, in LDS
hipError_t launch_select(const SelectArgs &a, int64_t blocks, int n_cu, hipStream_t stream);

struct AttnShape {
    int32_t B, T, H, heads, D, page, q_block, count, max_rows, max_len, causal;  // count 0: every page
};
// Tiles of rows (queries times the heads that share a key head), `block` queries each and `tiles` of them to a block
// (more than one where a query block is larger than a tile).  split: the keys of a tile may be cut into ranges, which the
// device decides by the sequences' lengths; `slots` workgroups run at once, a range has `least` keys or more.  Of one sequence: a round has `fill` pieces.
struct AttnPlan {
    int32_t tile_rows, block, tiles, split, slots, least, fill;
    int64_t groups, ws_bytes;
};
AttnPlan attn_plan(const AttnShape &s, int n_cu);
// Threads of a workgroup with a tile of 16, 32, 64 or 256 rows.
constexpr int attn_threads(int tile_rows) { return tile_rows == 32 || tile_rows == 64 ? 256 : 512; }

// selected null: every page.  o: bf16 or f32; lse: f32 [H, T] or null; ws: the partial results of key ranges.
struct AttnArgs {
    Pool c;
    Batch n;
    const uint16_t *q;
    void *o;
    int64_t q_ss, q_sh, o_ss, o_sh;
    float *lse;
    const int32_t *selected;
    int32_t H, count, causal;
    float scale;
    bool f32;
    char *ws;
};
hipError_t launch_attn(const AttnArgs &a, const AttnPlan &p, hipStream_t stream);

}  // namespace paged
}  // namespace regenvc
