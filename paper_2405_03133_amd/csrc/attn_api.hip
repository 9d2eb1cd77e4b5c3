// extern "C" entry points of the attention half: argument validation, launch on the caller's stream.  See include/lory.h
// for the contract of every call.
#include <math.h>

#include "lory_internal.h"

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int64_t kMaxStride = (int64_t)1 << 36;   // elements; times any number of rows it stays far inside 64 bits

// esize of a dtype, 0: unknown
int esize_of(int dtype) { return dtype == LORY_F32 ? 4 : dtype == LORY_BF16 ? 2 : 0; }

int check_heads_dims(int q_heads, int kv_heads, int head_dim)
{
    if (q_heads <= 0 || q_heads > 65535 || kv_heads <= 0 || kv_heads > 65535) return LORY_ERR_SHAPE;
    if (head_dim < 8 || head_dim > 256 || head_dim % 8 != 0) return LORY_ERR_SHAPE;
    return LORY_OK;
}

// A strided tensor: data there and aligned, strides whole 16 bytes (those of a dimension of one entry are not used).
int check_heads(const lory_heads *h, long tokens, long heads, int esize)
{
    if (!h || (tokens > 0 && !h->data)) return LORY_ERR_NULL;
    if (h->token < 0 || h->head < 0 || h->token > kMaxStride || h->head > kMaxStride) return LORY_ERR_SHAPE;
    const int n = 16 / esize;
    if (!aligned(h->data, 16) || (tokens > 1 && h->token % n != 0) || (heads > 1 && h->head % n != 0)) return LORY_ERR_ALIGN;
    return LORY_OK;
}

// The same for one that is written: no two heads share a place.
int check_out(const lory_heads *h, long tokens, long heads, int head_dim, int esize)
{
    const int rc = check_heads(h, tokens, heads, esize);
    if (rc != LORY_OK) return rc;
    long s0 = h->token, n0 = tokens, s1 = h->head, n1 = heads;
    if (n0 <= 1 || (n1 > 1 && s1 < s0)) {   // the shorter stride first
        s0 = h->head;
        n0 = heads;
        s1 = h->token;
        n1 = tokens;
    }
    if (n0 > 1 && s0 < head_dim) return LORY_ERR_OVERLAP;
    if (n1 > 1 && s1 < (n0 > 1 ? s0 * (n0 - 1) : 0) + head_dim) return LORY_ERR_OVERLAP;
    return LORY_OK;
}

int check_rope(const lory_rope_shape *s)
{
    if (!s) return LORY_ERR_NULL;
    if (!esize_of(s->dtype)) return LORY_ERR_DTYPE;
    if (s->tokens < 0 || s->tokens > (1 << 25)) return LORY_ERR_SHAPE;   // tokens index the grid
    const int rc = check_heads_dims(s->q_heads, s->kv_heads, s->head_dim);
    if (rc != LORY_OK) return rc;
    if (s->rot_dim < 0 || s->rot_dim > s->head_dim || s->rot_dim % 16 != 0) return LORY_ERR_SHAPE;
    if (s->interleaved != 0 && s->interleaved != 1) return LORY_ERR_SHAPE;
    if (!(s->eps >= 0.f) || isinf(s->eps)) return LORY_ERR_SHAPE;
    return LORY_OK;
}

// The inputs that all three calls share.
int check_rope_inputs(const lory_rope_shape *s, const lory_heads *q, const lory_heads *k, const int32_t *pos,
                      const double *freq, const void *wq, const void *wk)
{
    int rc = check_rope(s);
    if (rc != LORY_OK) return rc;
    if ((s->tokens > 0 && !pos) || (s->rot_dim > 0 && !freq) || (wq == nullptr) != (wk == nullptr)) return LORY_ERR_NULL;
    if (!aligned(pos, 4) || !aligned(freq, 8) || !aligned(wq, 16) || !aligned(wk, 16)) return LORY_ERR_ALIGN;
    rc = check_heads(q, s->tokens, s->q_heads, esize_of(s->dtype));
    return rc != LORY_OK ? rc : check_heads(k, s->tokens, s->kv_heads, esize_of(s->dtype));
}

int check_cache(const void *k_cache, const void *v_cache, int pages, int page, int kv_heads)
{
    if (!k_cache || !v_cache) return LORY_ERR_NULL;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return LORY_ERR_ALIGN;
    if (pages <= 0 || page <= 0 || (long)pages * page >= (1l << 31) || (long)pages * page * kv_heads >= (1l << 31))
        return LORY_ERR_SHAPE;
    return LORY_OK;
}

int check_paged(const lory_paged_shape *s)
{
    if (!s) return LORY_ERR_NULL;
    if (!esize_of(s->dtype)) return LORY_ERR_DTYPE;
    if (s->rows < 0 || s->rows > (1 << 20)) return LORY_ERR_SHAPE;
    const int rc = check_heads_dims(s->q_heads, s->kv_heads, s->head_dim);
    if (rc != LORY_OK) return rc;
    if (s->q_heads % s->kv_heads != 0) return LORY_ERR_SHAPE;
    if (s->pages <= 0 || s->page <= 0 || s->width <= 0 || s->table_row < s->width || s->table_row > kMaxStride)
        return LORY_ERR_SHAPE;
    if ((long)s->width * s->page > (1l << 30)) return LORY_ERR_SHAPE;
    // the kernel counts the row's blocks of 64 keys in 32 bits
    if (s->rows * ((long)s->width * s->page / 64 + 1) >= (1l << 31)) return LORY_ERR_SHAPE;
    if (!(s->scale > 0.f) || isinf(s->scale)) return LORY_ERR_SHAPE;
    return LORY_OK;
}

struct Range {
    const void *p;
    size_t bytes;
};

bool overlap(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

}  // namespace

extern "C" {

int lory_qk_rope(const lory_rope_shape *shape, const lory_heads *q, const lory_heads *k, const int32_t *pos,
                 const double *freq, const void *wq, const void *wk, const lory_heads *q_out, const lory_heads *k_out,
                 void *stream)
{
    int rc = check_rope_inputs(shape, q, k, pos, freq, wq, wk);
    if (rc == LORY_OK) rc = check_out(q_out, shape->tokens, shape->q_heads, shape->head_dim, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_out(k_out, shape->tokens, shape->kv_heads, shape->head_dim, esize_of(shape->dtype));
    if (rc != LORY_OK || shape->tokens == 0) return rc;
    return lory::qk_rope_launch(*shape, *q, *k, pos, freq, wq, wk, *q_out, k_out, nullptr, (hipStream_t)stream);
}

int lory_qk_rope_cache(const lory_rope_shape *shape, const lory_heads *q, const lory_heads *k, const lory_heads *v,
                       const int32_t *pos, const double *freq, const void *wq, const void *wk, const lory_heads *q_out,
                       void *k_cache, void *v_cache, int32_t pages, int32_t page, const int64_t *slots, void *stream)
{
    int rc = check_rope_inputs(shape, q, k, pos, freq, wq, wk);
    if (rc == LORY_OK) rc = check_heads(v, shape->tokens, shape->kv_heads, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_out(q_out, shape->tokens, shape->q_heads, shape->head_dim, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_cache(k_cache, v_cache, pages, page, shape->kv_heads);
    if (rc != LORY_OK) return rc;
    if (shape->tokens > 0 && !slots) return LORY_ERR_NULL;
    if (!aligned(slots, 8)) return LORY_ERR_ALIGN;
    if (shape->tokens == 0) return LORY_OK;
    const lory::RopeCache cache = {v, k_cache, v_cache, pages, page, slots};
    return lory::qk_rope_launch(*shape, *q, *k, pos, freq, wq, wk, *q_out, nullptr, &cache, (hipStream_t)stream);
}

int lory_qk_rope_workspace_bytes(const lory_rope_shape *shape, size_t *bytes_out)
{
    if (!bytes_out) return LORY_ERR_NULL;
    const int rc = check_rope(shape);
    if (rc == LORY_OK) *bytes_out = lory::qk_rope_bwd_workspace_bytes(*shape);
    return rc;
}

int lory_qk_rope_bwd(const lory_rope_shape *shape, const lory_heads *q, const lory_heads *k, const lory_heads *dq_out,
                     const lory_heads *dk_out, const int32_t *pos, const double *freq, const void *wq, const void *wk,
                     const lory_heads *dq, const lory_heads *dk, float *dwq, float *dwk, void *workspace,
                     size_t workspace_bytes, void *stream)
{
    int rc = check_rope_inputs(shape, q, k, pos, freq, wq, wk);
    for (int i = 0; i < 2 && rc == LORY_OK; ++i) {
        const int n = i ? shape->kv_heads : shape->q_heads, esize = esize_of(shape->dtype);
        rc = check_heads(i ? dk_out : dq_out, shape->tokens, n, esize);
        if (rc == LORY_OK) rc = check_out(i ? dk : dq, shape->tokens, n, shape->head_dim, esize);
    }
    if (rc != LORY_OK) return rc;
    if (wq) {
        const size_t need = lory::qk_rope_bwd_workspace_bytes(*shape);
        if (!dwq || !dwk || (need > 0 && !workspace)) return LORY_ERR_NULL;
        if (!aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(workspace, 16)) return LORY_ERR_ALIGN;
        if (workspace_bytes < need) return LORY_ERR_WORKSPACE;
    } else if (shape->tokens == 0) {
        return LORY_OK;
    }
    return lory::qk_rope_bwd_launch(*shape, *q, *k, *dq_out, *dk_out, pos, freq, wq, wk, *dq, *dk, dwq, dwk, workspace,
                                    (hipStream_t)stream);
}

int lory_kv_plan(const lory_plan_shape *shape, const int32_t *lens, const int32_t *add, int32_t *table, int32_t *free,
                 const int32_t *count, int32_t *lens_new, int32_t *cu, int32_t *positions, int64_t *slots,
                 int32_t *count_new, int32_t *status, void *stream)
{
    if (!shape) return LORY_ERR_NULL;
    const lory_plan_shape &s = *shape;
    if (s.rows < 0 || s.rows > (1 << 20) || s.room < 0 || s.width <= 0 || s.page <= 0 || s.free_size <= 0 ||
        s.table_row < s.width || s.table_row > kMaxStride || (long)s.width * s.page >= (1l << 31))
        return LORY_ERR_SHAPE;
    if (!free || !count || !cu || !count_new || !status || (s.rows > 0 && (!lens || !add || !table || !lens_new)) ||
        (s.room > 0 && (!positions || !slots)))
        return LORY_ERR_NULL;
    const size_t rows = s.rows, room = s.room;
    const Range r[] = {
        {lens, 4 * rows}, {add, 4 * rows}, {count, 4},   // inputs; the rest is written
        {table, s.rows > 0 ? 4 * ((rows - 1) * s.table_row + s.width) : 0}, {free, 4 * (size_t)s.free_size},
        {lens_new, 4 * rows}, {cu, 4 * (rows + 1)}, {positions, 4 * room}, {slots, 8 * room}, {count_new, 4}, {status, 4},
    };
    const int n = sizeof(r) / sizeof(r[0]), inputs = 3;
    for (int i = 0; i < n; ++i)
        if (!aligned(r[i].p, r[i].p == slots ? 8 : 4)) return LORY_ERR_ALIGN;
    for (int i = inputs; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(r[i], r[j])) return LORY_ERR_OVERLAP;
    return lory::kv_plan_launch(s, lens, add, table, free, count, lens_new, cu, positions, slots, count_new, status,
                                (hipStream_t)stream);
}

int lory_paged_attn_workspace_bytes(const lory_paged_shape *shape, size_t *bytes_out)
{
    if (!bytes_out) return LORY_ERR_NULL;
    const int rc = check_paged(shape);
    if (rc == LORY_OK) *bytes_out = lory::paged_attn_workspace_bytes(*shape);
    return rc;
}

int lory_paged_attn(const lory_paged_shape *shape, const lory_heads *q, const void *k_cache, const void *v_cache,
                    const int32_t *table, const int32_t *lens, const lory_heads *out, float *lse, void *workspace,
                    size_t workspace_bytes, void *stream)
{
    int rc = check_paged(shape);
    if (rc == LORY_OK) rc = check_heads(q, shape->rows, shape->q_heads, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_out(out, shape->rows, shape->q_heads, shape->head_dim, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_cache(k_cache, v_cache, shape->pages, shape->page, shape->kv_heads);
    if (rc != LORY_OK) return rc;
    if (!workspace || (shape->rows > 0 && (!table || !lens))) return LORY_ERR_NULL;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(lse, 4) || !aligned(workspace, 16)) return LORY_ERR_ALIGN;
    if (workspace_bytes < lory::paged_attn_workspace_bytes(*shape)) return LORY_ERR_WORKSPACE;
    if (shape->rows == 0) return LORY_OK;
    return lory::paged_attn_launch(*shape, *q, k_cache, v_cache, table, lens, *out, lse, workspace, (hipStream_t)stream);
}

}  // extern "C"
