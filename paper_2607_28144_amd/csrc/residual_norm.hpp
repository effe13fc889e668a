// Internal launch interface of the seam between two branches of a block:
// gated residual with a norm before and a norm after it, and its gradients.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace regenvc {

enum NormKind : int32_t { kNormNone = 0, kNormLayer = 1, kNormRms = 2 };

struct NormSpec {
    int32_t kind;
    float eps;
    const uint16_t *w, *b;  // bf16 [C] or null (1 and 0)
};

// Rows r of the batch, group g = r / group_rows of the f32 [C] vectors gate,
// scale and shift (a row of each per group, ldv elements apart; null: 1, 0, 0).
struct ResidualNormArgs {
    const float *x;  // forward: the stream before; backward: after the branch (the forward's x_out)
    const void *y;
    int64_t ldx, ldy;
    NormSpec post, pre;
    const float *gate, *scale, *shift;
    int64_t ldv;
    float alpha;
    int32_t rows, C, group_rows;
    bool f32;  // y, h, gh and dy are f32 (else bf16)
    // forward
    float *x_out;
    void *h;
    int64_t ldxo, ldh;
    // backward
    const void *gh;
    const float *gx;  // or null: 0
    float *dx;
    void *dy;
    int64_t ldgh, ldgx, lddx, lddy;
    // gradients of the vectors, or null: of gate, scale and shift [groups, C], of the weights [C]
    float *dgate, *dscale, *dshift, *dw, *db, *dpost_w, *dpost_b;
    float *ws;
};

hipError_t launch_residual_norm_fwd(const ResidualNormArgs &a, hipStream_t stream);

// How the backward pass deals its rows: `segments` runs of rows, `per_group` of
// each group's, to `blocks` workgroups.  Sums over the rows of a group that
// one segment holds whole go to the output directly; other sums pass through
// the workspace as one f32 row per segment (sums of a group) or workgroup
// (sums of all rows), which a second kernel adds in order.
struct ResidualNormPlan {
    int32_t groups, per_group, blocks;
    int32_t row_waves, rows_at_once;  // of a row, of a workgroup
    __host__ __device__ int64_t segments() const { return (int64_t)groups * per_group; }
};
ResidualNormPlan residual_norm_plan(int rows, int C, int group_rows, int n_cu);
// Workspace bytes for these numbers of sums over a group's and over all rows.
int64_t residual_norm_workspace(const ResidualNormPlan &p, int C, int group_sums, int row_sums);
hipError_t launch_residual_norm_bwd(const ResidualNormArgs &a, int n_cu, hipStream_t stream);

}  // namespace regenvc
