// Argument checks that the C entries of the attention half share.
#pragma once

#include <math.h>

#include "lory_internal.h"

namespace lory {
namespace check {

inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int64_t kMaxStride = (int64_t)1 << 36;   // elements; times any number of rows it stays far inside 64 bits

// esize of a dtype, 0: unknown
inline int esize_of(int dtype) { return dtype == LORY_F32 ? 4 : dtype == LORY_BF16 ? 2 : 0; }

inline int check_heads_dims(int q_heads, int kv_heads, int head_dim)
{
    if (q_heads <= 0 || q_heads > 65535 || kv_heads <= 0 || kv_heads > 65535) return LORY_ERR_SHAPE;
    if (head_dim < 8 || head_dim > 256 || head_dim % 8 != 0) return LORY_ERR_SHAPE;
    return LORY_OK;
}

// A strided tensor: data there and aligned, strides whole 16 bytes (those of a dimension of one entry are not used).
inline int check_heads(const lory_heads *h, long tokens, long heads, int esize)
{
    if (!h || (tokens > 0 && !h->data)) return LORY_ERR_NULL;
    if (h->token < 0 || h->head < 0 || h->token > kMaxStride || h->head > kMaxStride) return LORY_ERR_SHAPE;
    const int n = 16 / esize;
    if (!aligned(h->data, 16) || (tokens > 1 && h->token % n != 0) || (heads > 1 && h->head % n != 0)) return LORY_ERR_ALIGN;
    return LORY_OK;
}

// The same for one that is written: no two heads share a place.
inline int check_out(const lory_heads *h, long tokens, long heads, int head_dim, int esize)
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

inline int check_cache(const void *k_cache, const void *v_cache, int pages, int page, int kv_heads)
{
    if (!k_cache || !v_cache) return LORY_ERR_NULL;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return LORY_ERR_ALIGN;
    if (pages <= 0 || page <= 0 || (long)pages * page >= (1l << 31) || (long)pages * page * kv_heads >= (1l << 31))
        return LORY_ERR_SHAPE;
    return LORY_OK;
}

inline int check_paged(const lory_paged_shape *s)
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

inline bool overlap(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

}  // namespace check
}  // namespace lory
