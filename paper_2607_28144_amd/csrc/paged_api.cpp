// C ABI of the kernels of a cache in pages (include/regenvc_paged.h):
// synchronous argument validation before any launch, then the kernels on the
// caller's stream.
#include "regenvc_paged.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "abi_util.hpp"
#include "attn_kernels.hpp"
#include "paged_kernels.hpp"

using regenvc::abi::aligned;
using regenvc::abi::failf;
using regenvc::abi::overlaps;
using regenvc::abi::Range;
using regenvc::abi::range_of;
namespace paged = regenvc::paged;

namespace {

constexpr int32_t kMaxB = 1 << 20, kMaxT = 1 << 26, kMaxPages = 1 << 30;
constexpr int64_t kMaxPoolBytes = (int64_t)1 << 47;  // all that a process can address
constexpr int64_t kMaxPlaces = (int64_t)1 << 30;   // a tile past the last place stays within int32
constexpr int32_t kMaxBlock = 1 << 20, kMaxCount = 16384;
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;  // of a launch: its size has 32 bits
constexpr int64_t kMaxBlocks = kMaxThreads / 256;        // of a choice of pages: so many threads to each of more than a few
constexpr int64_t kMaxRows = (int64_t)1 << 29;  // of query heads: the kernels count a tile's and a block's in 32 bits

regenvc_status done()
{
    regenvc::abi::clear_error();
    return REGENVC_OK;
}

// What the kernels of a call read or write besides its tensors.
struct Ranges {
    Range pool[3], batch[3];
};

bool meets(const Range (&p)[3], const Range &r)
{
    return overlaps(p[0], r) || overlaps(p[1], r) || overlaps(p[2], r);
}

regenvc_status check_pool(const char *fn, const regenvc_page_pool *p, Range (&r)[3])
{
    if (p == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: pool is NULL", fn);
    if (p->pages < 0 || p->heads < 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (pages=%d heads=%d)", fn, p->pages, p->heads);
    if (p->D != 64 && p->D != 128) return failf(REGENVC_ERR_UNSUPPORTED, "%s: D=%d (64 or 128)", fn, p->D);
    if (p->page < 16 || p->page > 1024 || (p->page & (p->page - 1)) != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: pages of %d places (a power of two, 16 to 1024)", fn, p->page);
    if (p->pages >= kMaxPages || p->heads > 65535)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: %d pages of %d heads (below %d, at most 65535)", fn, p->pages, p->heads,
                     kMaxPages);
    const bool any = p->pages > 0 && p->heads > 0;
    if (any && (p->k == nullptr || p->v == nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: a NULL pool pointer", fn);
    if (!aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->means, 16))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: the pool must be 16-byte aligned", fn);
    const int64_t rows = (int64_t)p->pages * p->heads;  // below 2^46, with up to 2^18 bytes each
    if (rows > kMaxPoolBytes / (p->page * p->D * 2))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: keys of more than 2^47 bytes", fn);
    r[0] = range_of(p->k, rows * p->page * p->D * 2);
    r[1] = range_of(p->v, rows * p->page * p->D * 2);
    r[2] = range_of(p->means, p->means != nullptr ? rows * p->D * 2 : 0);
    return REGENVC_OK;
}

regenvc_status check_batch(const char *fn, const regenvc_page_batch *n, int32_t page, Range (&r)[3])
{
    if (n == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: batch is NULL", fn);
    if (n->B < 0 || n->T < 0 || n->columns < 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (B=%d T=%d columns=%d)", fn, n->B, n->T, n->columns);
    if (n->B > kMaxB || n->T >= kMaxT || (int64_t)n->columns * page >= kMaxPlaces)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: B=%d T=%d columns=%d pages of %d places: too many for one call", fn, n->B,
                     n->T, n->columns, page);
    r[0] = r[1] = r[2] = Range{0, 0};
    if (n->B == 0) return REGENVC_OK;
    if ((n->columns > 0 && n->table == nullptr) || n->first == nullptr || n->lens == nullptr)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: table, first or lens is NULL", fn);
    if (!aligned(n->table, 4) || !aligned(n->first, 4) || !aligned(n->lens, 4))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: table, first and lens must be 4-byte aligned", fn);
    if (n->table_stride < 0 || n->table_stride > kMaxPlaces)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: table_stride=%lld", fn, (long long)n->table_stride);
    r[0] = range_of(n->table, ((n->B - 1) * n->table_stride + n->columns) * 4);
    r[1] = range_of(n->first, ((int64_t)n->B + 1) * 4);
    r[2] = range_of(n->lens, (int64_t)n->B * 4);
    return REGENVC_OK;
}

regenvc_status check_heads(const char *fn, int32_t H, int32_t heads)
{
    if (H < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: H=%d < 0", fn, H);
    if (heads < 1 || H % heads != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: H=%d is not a multiple of the pool's %d heads", fn, H, heads);
    return REGENVC_OK;
}

regenvc_status check_rows(const char *fn, int32_t H, int32_t T)
{
    if ((int64_t)H * T > kMaxRows)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: %lld rows, at most 2^29", fn, (long long)((int64_t)H * T));
    return REGENVC_OK;
}

regenvc_status check_block(const char *fn, int32_t q_block, int32_t count)
{
    if (q_block < 1 || q_block > kMaxBlock || count < 1 || count > kMaxCount)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: q_block=%d count=%d (1 to %d, 1 to %d)", fn, q_block, count, kMaxBlock,
                     kMaxCount);
    return REGENVC_OK;
}

// The [T, heads, D] view of a packed tensor: stride_b is not looked at.
regenvc_status packed_range(const char *name, const regenvc_tensor *t, int64_t T, int64_t H, int64_t D, size_t elem, Range *r)
{
    regenvc_tensor u{};
    if (t != nullptr) u = *t;
    u.stride_b = 0;
    return regenvc::abi::view_range(name, t != nullptr ? &u : nullptr, 1, T, H, D, elem, r);
}
bool packed_injective(const regenvc_tensor *t, int64_t T, int64_t H, int64_t D)
{
    regenvc_tensor u = *t;
    u.stride_b = 0;
    return regenvc::abi::view_injective(&u, 1, T, H, D);
}

// Whether two packed bf16 tensors of equal row strides, such as the parts of a
// fused projection, share no element though their ranges cross.
bool interleaved(const regenvc_tensor *a, int64_t Ha, const regenvc_tensor *b, int64_t Hb, int64_t D)
{
    const int64_t row = a->stride_s;
    if (row != b->stride_s || row <= 0 || a->stride_h < 0 || b->stride_h < 0) return false;
    const int64_t wa = a->stride_h * (Ha - 1) + D, wb = b->stride_h * (Hb - 1) + D;
    int64_t apart = ((int64_t)reinterpret_cast<uintptr_t>(b->ptr) - (int64_t)reinterpret_cast<uintptr_t>(a->ptr)) / 2 % row;
    if (apart < 0) apart += row;  // b's row begins this many elements behind one of a's
    return wa <= apart && apart + wb <= row;
}

paged::Pool pool_of(const regenvc_page_pool &p)
{
    return {static_cast<uint16_t *>(p.k), static_cast<uint16_t *>(p.v), static_cast<uint16_t *>(p.means), p.pages,
            __builtin_ctz((unsigned)p.page), p.heads, p.D};
}
paged::Batch batch_of(const regenvc_page_batch &n)
{
    return {n.table, n.first, n.lens, n.table_stride, n.B, n.columns, n.T};
}
const uint16_t *u16(const void *p)
{
    return static_cast<const uint16_t *>(p);
}

regenvc_status check_shape(const char *fn, const regenvc_paged_attn_shape *s)
{
    if (s == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: shape is NULL", fn);
    regenvc_status st = check_heads(fn, s->H, s->heads);
    if (st != REGENVC_OK) return st;
    if (s->B < 0 || s->T < 0 || s->max_rows < 0 || s->max_len < 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: negative size (B=%d T=%d max_rows=%d max_len=%d)", fn, s->B, s->T,
                     s->max_rows, s->max_len);
    if (s->D != 64 && s->D != 128) return failf(REGENVC_ERR_UNSUPPORTED, "%s: D=%d (64 or 128)", fn, s->D);
    if (s->page < 16 || s->page > 1024 || (s->page & (s->page - 1)) != 0)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: pages of %d places (a power of two, 16 to 1024)", fn, s->page);
    if (s->B > kMaxB || s->T >= kMaxT || s->max_len >= kMaxPlaces || s->heads > 65535)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: B=%d T=%d heads=%d max_len=%d: too many for one call", fn, s->B, s->T,
                     s->heads, s->max_len);
    if (s->max_rows > s->T)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: max_rows=%d of T=%d rows", fn, s->max_rows, s->T);
    if (s->count != 0 && (st = check_block(fn, s->q_block, s->count)) != REGENVC_OK) return st;
    return check_rows(fn, s->H, s->T);
}

bool empty(const regenvc_paged_attn_shape &s)
{
    return s.B == 0 || s.T == 0 || s.H == 0;
}

// The plan of a shape that check_shape accepts and that is not empty.
regenvc_status plan_of(const char *fn, const regenvc_paged_attn_shape &s, int n_cu, paged::AttnPlan *p)
{
    *p = paged::attn_plan({s.B, s.T, s.H, s.heads, s.D, s.page, s.q_block, s.count, s.max_rows, s.max_len, s.causal}, n_cu);
    const int64_t most = kMaxThreads / paged::attn_threads(p->tile_rows);
    if (p->groups > most || p->groups * p->tile_rows > INT32_MAX)  // rows of partial results are counted in 32 bits
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: more than %lld workgroups", fn, (long long)most);
    return REGENVC_OK;
}

}  // namespace

extern "C" {

regenvc_status regenvc_paged_append(const regenvc_page_pool *pool, const regenvc_page_batch *batch,
                                    const regenvc_tensor *q, const regenvc_tensor *k, const regenvc_tensor *v,
                                    const void *w_q, const void *w_k, float eps, const regenvc_rotary *rotary,
                                    const regenvc_tensor *q_out, int32_t H, void *stream)
{
    const char *fn = "regenvc_paged_append";
    Ranges r{};
    regenvc_status st = check_pool(fn, pool, r.pool);
    if (st == REGENVC_OK) st = check_batch(fn, batch, pool->page, r.batch);
    if (st != REGENVC_OK) return st;
    if (H < 0 || H > 65535) return failf(REGENVC_ERR_INVALID_ARG, "%s: H=%d (0 to 65535)", fn, H);
    if ((H > 0) != (q != nullptr) || (H > 0) != (q_out != nullptr) || (H == 0 && w_q != nullptr))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: q, q_out and H go together, w_q with them", fn);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return failf(REGENVC_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
    if (rotary != nullptr) {
        if (rotary->pairs < 0 || rotary->pairs % 8 != 0 || 2 * (int64_t)rotary->pairs > pool->D)
            return failf(REGENVC_ERR_UNSUPPORTED, "%s: %d rotated pairs (a multiple of 8, at most %d)", fn, rotary->pairs,
                         pool->D / 2);
        if (rotary->pairs > 0 && rotary->turns == nullptr)
            return failf(REGENVC_ERR_INVALID_ARG, "%s: turns is NULL", fn);
        if (!aligned(rotary->turns, 8)) return failf(REGENVC_ERR_UNSUPPORTED, "%s: turns must be 8-byte aligned", fn);
        if (!std::isfinite(rotary->amplitude))
            return failf(REGENVC_ERR_INVALID_ARG, "%s: the amplitude must be finite", fn);
    }
    if (!aligned(w_q, 16) || !aligned(w_k, 16))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: w_q and w_k must be 16-byte aligned", fn);
    if (batch->B == 0 || batch->T == 0 || (H == 0 && pool->heads == 0)) return done();
    const int D = pool->D, T = batch->T, heads = pool->heads;
    Range rq{0, 0}, ro{0, 0}, rk{0, 0}, rv{0, 0};
    if (H > 0) {
        if ((st = packed_range("q", q, T, H, D, 2, &rq)) != REGENVC_OK) return st;
        if ((st = packed_range("q_out", q_out, T, H, D, 2, &ro)) != REGENVC_OK) return st;
        if (!packed_injective(q_out, T, H, D))
            return failf(REGENVC_ERR_INVALID_ARG, "%s: elements of q_out share an address", fn);
    }
    if (heads > 0) {
        if ((st = packed_range("k", k, T, heads, D, 2, &rk)) != REGENVC_OK) return st;
        if ((st = packed_range("v", v, T, heads, D, 2, &rv)) != REGENVC_OK) return st;
    }
    const Range rt = range_of(rotary != nullptr ? rotary->turns : nullptr, rotary != nullptr ? (int64_t)rotary->pairs * 8 : 0);
    const Range rw[2] = {range_of(w_q, w_q != nullptr ? D * 2 : 0), range_of(w_k, w_k != nullptr ? D * 2 : 0)};
    if (overlaps(r.pool[0], r.pool[1]) || overlaps(r.pool[0], r.pool[2]) || overlaps(r.pool[1], r.pool[2]))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: the pool overlaps itself", fn);
    for (const Range &i : {rq, rk, rv, ro, rt, rw[0], rw[1], r.batch[0], r.batch[1], r.batch[2]})
        if (meets(r.pool, i)) return failf(REGENVC_ERR_INVALID_ARG, "%s: the pool overlaps another argument", fn);
    if (H > 0) {
        const bool in_place = q_out->ptr == q->ptr && (T == 1 || q_out->stride_s == q->stride_s) &&
                              (H == 1 || q_out->stride_h == q->stride_h);
        if ((!in_place && overlaps(ro, rq) && !interleaved(q_out, H, q, H, D)) ||
            (heads > 0 && overlaps(ro, rk) && !interleaved(q_out, H, k, heads, D)) ||
            (heads > 0 && overlaps(ro, rv) && !interleaved(q_out, H, v, heads, D)))
            return failf(REGENVC_ERR_INVALID_ARG, "%s: q_out overlaps an input", fn);
        for (const Range &i : {rt, rw[0], rw[1], r.batch[0], r.batch[1], r.batch[2]})
            if (overlaps(ro, i)) return failf(REGENVC_ERR_INVALID_ARG, "%s: q_out overlaps an input", fn);
    }
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    paged::AppendArgs a{};
    a.c = pool_of(*pool), a.n = batch_of(*batch);
    if (H > 0) {
        a.q = u16(q->ptr), a.q_ss = q->stride_s, a.q_sh = q->stride_h;
        a.q_out = static_cast<uint16_t *>(q_out->ptr), a.o_ss = q_out->stride_s, a.o_sh = q_out->stride_h;
    }
    if (heads > 0) {
        a.k = u16(k->ptr), a.k_ss = k->stride_s, a.k_sh = k->stride_h;
        a.v = u16(v->ptr), a.v_ss = v->stride_s, a.v_sh = v->stride_h;
    }
    a.w_q = u16(w_q), a.w_k = u16(w_k), a.eps = eps, a.H = H, a.amplitude = 1.f;
    if (rotary != nullptr) {
        a.turns = rotary->turns, a.pairs = rotary->pairs, a.interleaved = rotary->interleaved != 0;
        a.amplitude = rotary->amplitude;
    }
    return regenvc::abi::launch_status(paged::launch_append(a, regenvc::device_cu_count(), static_cast<hipStream_t>(stream)),
                                       fn);
}

regenvc_status regenvc_paged_select(const regenvc_tensor *q, const regenvc_page_pool *pool,
                                    const regenvc_page_batch *batch, int32_t H, int32_t q_block, int32_t count,
                                    int32_t keep_first, int32_t keep_last, int32_t causal, int32_t *selected,
                                    void *stream)
{
    const char *fn = "regenvc_paged_select";
    Ranges r{};
    regenvc_status st = check_pool(fn, pool, r.pool);
    if (st == REGENVC_OK) st = check_batch(fn, batch, pool->page, r.batch);
    if (st == REGENVC_OK) st = check_heads(fn, H, pool->heads);
    if (st == REGENVC_OK) st = check_rows(fn, H, batch->T);
    if (st == REGENVC_OK) st = check_block(fn, q_block, count);
    if (st != REGENVC_OK) return st;
    if (keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > count)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: keep_first=%d keep_last=%d of count=%d", fn, keep_first, keep_last, count);
    const int64_t blocks = (int64_t)batch->T / q_block + batch->B;
    if (batch->columns > paged::kMaxSelectColumns || blocks > kMaxBlocks)
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: %d columns, %lld blocks (at most %d, %lld)", fn, batch->columns,
                     (long long)blocks, paged::kMaxSelectColumns, (long long)kMaxBlocks);
    if (blocks == 0) return done();
    const bool any = batch->B > 0 && batch->T > 0 && H > 0;  // else every block is one without queries: -1
    if (any && pool->means == nullptr && pool->pages > 0)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: the pool has no means", fn);
    Range rq{0, 0};
    if (any && (st = packed_range("q", q, batch->T, H, pool->D, 2, &rq)) != REGENVC_OK) return st;
    if (selected == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: selected is NULL", fn);
    if (!aligned(selected, 4)) return failf(REGENVC_ERR_UNSUPPORTED, "%s: selected must be 4-byte aligned", fn);
    const Range rs = range_of(selected, blocks * pool->heads * count * 4);
    for (const Range &i : {rq, r.batch[0], r.batch[1], r.batch[2], r.pool[0], r.pool[1], r.pool[2]})
        if (overlaps(rs, i)) return failf(REGENVC_ERR_INVALID_ARG, "%s: selected overlaps an input", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    paged::SelectArgs a{};
    a.c = pool_of(*pool), a.n = batch_of(*batch);
    if (any)
        a.q = u16(q->ptr), a.q_ss = q->stride_s, a.q_sh = q->stride_h;
    else
        a.n.B = 0;
    a.selected = selected, a.H = H, a.q_block = q_block, a.count = count;
    a.keep_first = keep_first, a.keep_last = keep_last, a.causal = causal != 0;
    return regenvc::abi::launch_status(paged::launch_select(a, blocks, regenvc::device_cu_count(), static_cast<hipStream_t>(stream)),
                                       fn);
}

regenvc_status regenvc_paged_attn_workspace(const regenvc_paged_attn_shape *shape, int32_t n_cu, int64_t *bytes)
{
    const char *fn = "regenvc_paged_attn_workspace";
    if (bytes == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    if (n_cu < 1) return failf(REGENVC_ERR_INVALID_ARG, "%s: n_cu=%d < 1", fn, n_cu);
    regenvc_status st = check_shape(fn, shape);
    if (st != REGENVC_OK) return st;
    paged::AttnPlan p{};
    if (!empty(*shape) && (st = plan_of(fn, *shape, n_cu, &p)) != REGENVC_OK) return st;
    *bytes = p.ws_bytes;
    return done();
}

regenvc_status regenvc_paged_attn_plan_query(const regenvc_paged_attn_shape *shape, int32_t n_cu,
                                             regenvc_paged_attn_plan *plan)
{
    const char *fn = "regenvc_paged_attn_plan_query";
    if (plan == nullptr) return failf(REGENVC_ERR_INVALID_ARG, "%s: plan is NULL", fn);
    if (n_cu < 1) return failf(REGENVC_ERR_INVALID_ARG, "%s: n_cu=%d < 1", fn, n_cu);
    regenvc_status st = check_shape(fn, shape);
    if (st != REGENVC_OK) return st;
    paged::AttnPlan p{};
    if (!empty(*shape) && (st = plan_of(fn, *shape, n_cu, &p)) != REGENVC_OK) return st;
    *plan = regenvc_paged_attn_plan{p.tile_rows, (int32_t)p.groups, p.split};
    return done();
}

regenvc_status regenvc_paged_attn_fwd(const regenvc_tensor *q, const regenvc_page_pool *pool,
                                      const regenvc_page_batch *batch, const int32_t *selected, int32_t q_block,
                                      int32_t count, int32_t causal, int32_t max_rows, int32_t max_len,
                                      const regenvc_tensor *o, regenvc_dtype o_dtype, float *lse, int32_t H,
                                      float softmax_scale, void *workspace, int64_t workspace_bytes, void *stream)
{
    const char *fn = "regenvc_paged_attn_fwd";
    Ranges r{};
    regenvc_status st = check_pool(fn, pool, r.pool);
    if (st == REGENVC_OK) st = check_batch(fn, batch, pool->page, r.batch);
    if (st == REGENVC_OK && selected != nullptr) st = check_block(fn, q_block, count);
    if (st != REGENVC_OK) return st;
    const regenvc_paged_attn_shape s{batch->B,   batch->T, H,       pool->heads, pool->D, pool->page, q_block,
                                     selected != nullptr ? count : 0, max_rows, max_len, causal};
    if ((st = check_shape(fn, &s)) != REGENVC_OK) return st;
    if ((st = regenvc::abi::softmax_scale_ok(softmax_scale)) != REGENVC_OK) return st;
    if (o_dtype != REGENVC_BF16 && o_dtype != REGENVC_F32) return failf(REGENVC_ERR_INVALID_ARG, "%s: dtype %d", fn, o_dtype);
    if (max_len > batch->columns * pool->page)
        return failf(REGENVC_ERR_INVALID_ARG, "%s: max_len=%d, the table has %d places", fn, max_len,
                     batch->columns * pool->page);
    if (workspace_bytes < 0) return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
    if (empty(s)) return done();
    const int D = pool->D, T = batch->T;
    Range rq, ro;
    if ((st = packed_range("q", q, T, H, D, 2, &rq)) != REGENVC_OK) return st;
    if ((st = packed_range("o", o, T, H, D, o_dtype == REGENVC_F32 ? 4 : 2, &ro)) != REGENVC_OK) return st;
    if (!packed_injective(o, T, H, D)) return failf(REGENVC_ERR_INVALID_ARG, "%s: elements of o share an address", fn);
    if (!aligned(lse, 4) || !aligned(selected, 4))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: lse and selected must be 4-byte aligned", fn);
    if (workspace != nullptr && !aligned(workspace, 256))
        return failf(REGENVC_ERR_UNSUPPORTED, "%s: workspace must be 256-byte aligned", fn);
    const Range rl = range_of(lse, lse != nullptr ? (int64_t)H * T * 4 : 0);
    const Range rw = range_of(workspace, workspace != nullptr ? workspace_bytes : 0);
    const Range rs = range_of(selected, selected != nullptr ? ((int64_t)T / q_block + batch->B) * pool->heads * count * 4 : 0);
    for (const Range &x : {ro, rl, rw})
        if (overlaps(x, rq) || overlaps(x, rs) || meets(r.pool, x) || meets(r.batch, x))
            return failf(REGENVC_ERR_INVALID_ARG, "%s: an output or the workspace overlaps an input", fn);
    if (overlaps(ro, rl) || overlaps(ro, rw) || overlaps(rl, rw))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: o, lse and the workspace overlap", fn);
    if ((st = regenvc::abi::device_ok()) != REGENVC_OK) return st;
    paged::AttnPlan p{};
    if ((st = plan_of(fn, s, regenvc::device_cu_count(), &p)) != REGENVC_OK) return st;
    if (p.ws_bytes > 0 && (workspace == nullptr || workspace_bytes < p.ws_bytes))
        return failf(REGENVC_ERR_INVALID_ARG, "%s: workspace of %lld bytes, this call needs %lld", fn,
                     (long long)(workspace != nullptr ? workspace_bytes : 0), (long long)p.ws_bytes);
    const paged::AttnArgs a{pool_of(*pool), batch_of(*batch), u16(q->ptr), o->ptr, q->stride_s, q->stride_h, o->stride_s,
                            o->stride_h,    lse,              selected,    H,      count,       causal != 0, softmax_scale,
                            o_dtype == REGENVC_F32, static_cast<char *>(workspace)};
    return regenvc::abi::launch_status(paged::launch_attn(a, p, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
