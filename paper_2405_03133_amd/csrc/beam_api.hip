// extern "C" entry points of several continuations of one prompt: argument validation, launch on the caller's stream.  See
// include/lory.h for the contract of every call.
#include "attn_checks.h"

using namespace lory::check;

namespace {

int check_beam(const lory_beam_shape *s)
{
    if (!s) return LORY_ERR_NULL;
    if (!esize_of(s->dtype)) return LORY_ERR_DTYPE;
    if (s->requests < 0 || s->beams <= 0 || s->beams > 64 || (long)s->requests * s->beams > (1 << 20) || s->vocab <= 0 ||
        s->vocab > (1 << 24) || s->k <= 0 || s->k > 64 || s->row < s->vocab || s->row > kMaxStride)
        return LORY_ERR_SHAPE;
    return LORY_OK;
}

int check_fork(const lory_fork_shape *s)
{
    if (!s) return LORY_ERR_NULL;
    if (s->old_rows < 0 || s->old_rows > (1 << 20) || s->rows < 0 || s->rows > (1 << 20) || s->width <= 0 || s->page <= 0 ||
        s->pages <= 0 || s->free_size <= 0 || (long)s->width * s->page >= (1l << 31) || s->table_row < s->width ||
        s->table_row > kMaxStride || s->new_row < s->width || s->new_row > kMaxStride)
        return LORY_ERR_SHAPE;
    return LORY_OK;
}

int check_prefix(const lory_paged_shape *s, int groups)
{
    const int rc = check_paged(s);
    if (rc != LORY_OK) return rc;
    if (groups < 0 || (s->rows > 0 && groups == 0) || groups > s->rows || (groups > 0 && s->rows % groups != 0)) return LORY_ERR_SHAPE;
    // the kernel counts units of 64 keys, and two more for every row and group, in 32 bits
    if (s->rows * ((long)s->width * s->page / 64 + 4) >= (1l << 31)) return LORY_ERR_SHAPE;
    if (groups > 0 && (long)(s->rows / groups) * (s->q_heads / s->kv_heads) >= (1l << 30)) return LORY_ERR_SHAPE;
    return LORY_OK;
}

// bytes of n rows of `width` elements of 4 bytes
size_t strided(size_t n, int64_t row, int width) { return n > 0 ? 4 * ((n - 1) * row + width) : 0; }

// The arrays from `inputs` on are written: none of them may share a byte with another.
int check_ranges(const Range *r, int n, int inputs)
{
    for (int i = 0; i < n; ++i)
        if (!aligned(r[i].p, 4)) return LORY_ERR_ALIGN;
    for (int i = inputs; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(r[i], r[j])) return LORY_ERR_OVERLAP;
    return LORY_OK;
}

}  // namespace

extern "C" {

int lory_beam_select_workspace_bytes(const lory_beam_shape *shape, size_t *bytes_out)
{
    if (!bytes_out) return LORY_ERR_NULL;
    const int rc = check_beam(shape);
    if (rc == LORY_OK) *bytes_out = lory::beam_select_workspace_bytes(*shape);
    return rc;
}

int lory_beam_select(const lory_beam_shape *shape, const void *logits, const float *score, float *score_out, int32_t *token,
                     int32_t *parent, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_beam(shape);
    if (rc != LORY_OK) return rc;
    const lory_beam_shape &s = *shape;
    if (s.requests == 0) return LORY_OK;
    if (!logits || !score || !score_out || !token || !parent || !workspace) return LORY_ERR_NULL;
    const int esize = esize_of(s.dtype);
    if (!aligned(logits, esize) || !aligned(workspace, 16)) return LORY_ERR_ALIGN;
    const size_t rows = (size_t)s.requests * s.beams, n = (size_t)s.requests * s.k, need = lory::beam_select_workspace_bytes(s);
    const Range r[] = {{score, 4 * rows}, {score_out, 4 * n}, {token, 4 * n}, {parent, 4 * n}, {workspace, need}};
    rc = check_ranges(r, 5, 1);
    if (rc != LORY_OK) return rc;
    const Range x = {logits, ((rows - 1) * s.row + s.vocab) * esize};
    for (int i = 1; i < 5; ++i)
        if (overlap(r[i], x)) return LORY_ERR_OVERLAP;
    if (workspace_bytes < need) return LORY_ERR_WORKSPACE;
    return lory::beam_select_launch(s, logits, score, score_out, token, parent, workspace, (hipStream_t)stream);
}

int lory_kv_fork_workspace_bytes(const lory_fork_shape *shape, size_t *bytes_out)
{
    if (!bytes_out) return LORY_ERR_NULL;
    const int rc = check_fork(shape);
    if (rc == LORY_OK) *bytes_out = lory::kv_fork_workspace_bytes(*shape);
    return rc;
}

int lory_kv_fork(const lory_fork_shape *shape, const int32_t *lens, const int32_t *src, const int32_t *table, int32_t *free,
                 const int32_t *count, int32_t *lens_new, int32_t *table_new, int32_t *count_new, int32_t *copies,
                 int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_fork(shape);
    if (rc != LORY_OK) return rc;
    const lory_fork_shape &s = *shape;
    if (!free || !count || !count_new || !status || !workspace || (s.old_rows > 0 && (!lens || !table)) ||
        (s.rows > 0 && (!src || !lens_new || !table_new || !copies)))
        return LORY_ERR_NULL;
    const size_t old = s.old_rows, rows = s.rows, need = lory::kv_fork_workspace_bytes(s);
    const Range r[] = {
        {lens, 4 * old}, {src, 4 * rows}, {table, strided(old, s.table_row, s.width)}, {count, 4},   // inputs
        {free, 4 * (size_t)s.free_size}, {lens_new, 4 * rows}, {table_new, strided(rows, s.new_row, s.width)}, {count_new, 4},
        {copies, 12 * rows}, {status, 4}, {workspace, need},
    };
    if (!aligned(workspace, 16)) return LORY_ERR_ALIGN;
    rc = check_ranges(r, sizeof(r) / sizeof(r[0]), 4);
    if (rc != LORY_OK) return rc;
    if (workspace_bytes < need) return LORY_ERR_WORKSPACE;
    return lory::kv_fork_launch(s, lens, src, table, free, count, lens_new, table_new, count_new, copies, status, workspace,
                                (hipStream_t)stream);
}

int lory_kv_copy(const lory_copy_shape *shape, void *k_cache, void *v_cache, const int32_t *copies, void *stream)
{
    if (!shape) return LORY_ERR_NULL;
    const lory_copy_shape &s = *shape;
    if (!esize_of(s.dtype)) return LORY_ERR_DTYPE;
    int rc = check_heads_dims(s.kv_heads, s.kv_heads, s.head_dim);
    if (rc != LORY_OK) return rc;
    if (s.n < 0 || s.n > (1 << 20) || s.layers <= 0 || s.layers > 32767) return LORY_ERR_SHAPE;
    rc = check_cache(k_cache, v_cache, s.pages, s.page, s.kv_heads);
    if (rc != LORY_OK) return rc;
    // a page's 16-byte pieces are counted in 32 bits
    if ((long)s.page * s.kv_heads * s.head_dim * esize_of(s.dtype) / 16 >= (1l << 31)) return LORY_ERR_SHAPE;
    if (s.n == 0) return LORY_OK;
    if (!copies) return LORY_ERR_NULL;
    if (!aligned(copies, 4)) return LORY_ERR_ALIGN;
    const size_t bytes = (size_t)s.layers * s.pages * s.page * s.kv_heads * s.head_dim * esize_of(s.dtype);
    const Range r[] = {{copies, 12 * (size_t)s.n}, {k_cache, bytes}, {v_cache, bytes}};
    if (overlap(r[0], r[1]) || overlap(r[0], r[2]) || overlap(r[1], r[2])) return LORY_ERR_OVERLAP;
    return lory::kv_copy_launch(s, k_cache, v_cache, copies, (hipStream_t)stream);
}

int lory_prefix_attn_workspace_bytes(const lory_paged_shape *shape, int32_t groups, size_t *bytes_out)
{
    if (!bytes_out) return LORY_ERR_NULL;
    const int rc = check_prefix(shape, groups);
    if (rc == LORY_OK) *bytes_out = lory::prefix_attn_workspace_bytes(*shape, groups);
    return rc;
}

int lory_prefix_attn(const lory_paged_shape *shape, int32_t groups, const lory_heads *q, const void *k_cache, const void *v_cache,
                     const int32_t *table, const int32_t *lens, const int32_t *shared, const lory_heads *out, float *lse,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_prefix(shape, groups);
    if (rc == LORY_OK) rc = check_heads(q, shape->rows, shape->q_heads, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_out(out, shape->rows, shape->q_heads, shape->head_dim, esize_of(shape->dtype));
    if (rc == LORY_OK) rc = check_cache(k_cache, v_cache, shape->pages, shape->page, shape->kv_heads);
    if (rc != LORY_OK) return rc;
    if (!workspace || (shape->rows > 0 && (!table || !lens || !shared))) return LORY_ERR_NULL;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(shared, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
        return LORY_ERR_ALIGN;
    if (workspace_bytes < lory::prefix_attn_workspace_bytes(*shape, groups)) return LORY_ERR_WORKSPACE;
    if (shape->rows == 0) return LORY_OK;
    return lory::prefix_attn_launch(*shape, groups, *q, k_cache, v_cache, table, lens, shared, *out, lse, workspace,
                                    (hipStream_t)stream);
}

}  // extern "C"
