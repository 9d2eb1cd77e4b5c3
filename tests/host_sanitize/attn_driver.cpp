// Host layer of the attention operators under sanitizers: refusals and workspace sizes over shapes up to every limit.  No kernel
// is launched: every call either is refused, has nothing to do, or only asks for a size.
#include <stdint.h>
#include <stdio.h>

#include "lory.h"

static int failures = 0;
#define EXPECT(c)                                              \
    do {                                                       \
        if (!(c)) {                                            \
            printf("%s:%d: %s\n", __FILE__, __LINE__, #c);     \
            ++failures;                                        \
        }                                                      \
    } while (0)

static unsigned rng = 7;
static int rnd(int n)
{
    rng = rng * 1664525u + 1013904223u;
    return (int)((rng >> 8) % (unsigned)n);
}
// 1 .. hi, even over the logarithm
static int spread(int hi)
{
    int bits = 0;
    while ((2ll << bits) <= hi) ++bits;
    const int v = 1 << rnd(bits + 1);
    const long long x = v + rnd(v);
    return x < hi ? (int)x : hi;
}

int main()
{
    void *const F = (void *)0x7F0000001000;   // aligned, never read
    size_t n = 0;
    for (int i = 0; i < 200000; ++i) {
        lory_rope_shape s = {spread(1 << 25), spread(65535), spread(65535), 8 * (1 + rnd(32)), 0, rnd(2), rnd(2), 1e-6f};
        s.rot_dim = 16 * rnd(s.head_dim / 16 + 1);
        if (i % 50 == 0) s.tokens = 0;
        EXPECT(lory_qk_rope_workspace_bytes(&s, &n) == LORY_OK);
        EXPECT(n <= (size_t)1024 * 2 * s.head_dim * 4 && (n == 0) == (s.tokens == 0));
        if (n > 0) {   // too little workspace: refused whatever the shape
            const lory_heads q = {F, (int64_t)s.q_heads * s.head_dim, s.head_dim}, k = {F, (int64_t)s.kv_heads * s.head_dim, s.head_dim};
            EXPECT(lory_qk_rope_bwd(&s, &q, &k, &q, &k, (int32_t *)F, (double *)F, F, F, &q, &k, (float *)F, (float *)F, F, n - 1,
                                    NULL) == LORY_ERR_WORKSPACE);
        }
    }
    int ok = 0;
    for (int i = 0; i < 400000; ++i) {
        lory_paged_shape s = {};
        s.rows = i % 50 == 0 ? 0 : spread(1 << 20);
        s.kv_heads = spread(65535);
        s.q_heads = s.kv_heads * spread(65535 / s.kv_heads);
        s.head_dim = 8 * (1 + rnd(32));
        s.pages = spread(1 << 30);
        s.page = spread(1 << 30);
        s.width = spread(1 << 30);
        s.dtype = rnd(2);
        s.table_row = s.width + (int64_t)rnd(3) * (1 << 30);
        s.scale = 0.1f;
        n = 0;
        const int rc = lory_paged_attn_workspace_bytes(&s, &n);
        EXPECT(rc == LORY_OK || rc == LORY_ERR_SHAPE);
        if (rc != LORY_OK) continue;
        ++ok;
        EXPECT(n >= 256 && n % 256 == 0 && n <= (size_t)4 * (s.rows + 65) + 256 + (size_t)1536 * 16 * (s.head_dim + 2) * 4);
        const lory_heads q = {F, (int64_t)s.q_heads * s.head_dim, s.head_dim};
        const int call = lory_paged_attn(&s, &q, F, F, (int32_t *)F, (int32_t *)F, &q, NULL, F, n - 1, NULL);
        EXPECT(call == LORY_ERR_WORKSPACE || call == LORY_ERR_SHAPE);   // SHAPE: more rows of the cache than 31 bits
    }
    EXPECT(ok > 1000);
    for (int i = 0; i < 200000; ++i) {
        lory_plan_shape s = {spread(1 << 20), spread(1 << 30), spread(1 << 30), spread(INT32_MAX), spread(INT32_MAX), 0};
        s.table_row = s.width + (int64_t)rnd(3) * (1 << 30);
        // every array at one address: an overlap unless the shape is refused first
        const int rc = lory_kv_plan(&s, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F,
                                    (int32_t *)F, (int64_t *)F, (int32_t *)F, (int32_t *)F, NULL);
        EXPECT(rc == ((int64_t)s.width * s.page >= (1ll << 31) ? LORY_ERR_SHAPE : LORY_ERR_OVERLAP));
    }
    // strides at the ends of their range
    lory_rope_shape s = {2, 2, 2, 64, 64, 0, LORY_F32, 0.f};
    const lory_heads good = {F, 128, 64};
    const int64_t odd[] = {INT64_MIN, -4, 1, INT64_MAX, INT64_MAX - 3, ((int64_t)1 << 36) + 4};
    for (int i = 0; i < 6; ++i) {
        const lory_heads bad = {F, odd[i], 64}, bad2 = {F, 128, odd[i]};
        EXPECT(lory_qk_rope(&s, &bad, &good, (int32_t *)F, (double *)F, NULL, NULL, &good, &good, NULL) != LORY_OK);
        EXPECT(lory_qk_rope(&s, &good, &good, (int32_t *)F, (double *)F, NULL, NULL, &bad2, &good, NULL) != LORY_OK);
    }
    lory_plan_shape p = {2, 4, 16, 8, 8, INT64_MAX};
    lory_paged_shape a = {2, 2, 2, 64, 4, 16, 4, LORY_F32, INT64_MAX, 0.1f};
    EXPECT(lory_kv_plan(&p, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F, (int32_t *)F,
                        (int64_t *)F, (int32_t *)F, (int32_t *)F, NULL) == LORY_ERR_SHAPE);
    EXPECT(lory_paged_attn_workspace_bytes(&a, &n) == LORY_ERR_SHAPE);
    printf("attention abi sanitizer run: %s (%d failures)\n", failures ? "FAILED" : "ok", failures);
    return failures ? 1 : 0;
}
