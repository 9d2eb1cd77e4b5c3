// Host layer of the operators for several continuations of a prompt under sanitizers: refusals and workspace sizes over shapes up
// to every limit.  No kernel is launched: every call either is refused, has nothing to do, or only asks for a size.
#include <stdint.h>
#include <stdio.h>

#include "lory.h"

static int failures = 0;
#define EXPECT(c)                                              \
    do {                                                       \
        if (!(c)) {                                            \
            printf("%s:%d: %s FAILED\n", __FILE__, __LINE__, #c); \
            ++failures;                                        \
        }                                                      \
    } while (0)

static unsigned rng = 11;
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
    const long long x = (long long)v + rnd(v);
    return x < hi ? (int)x : hi;
}

int main()
{
    char *const F = (char *)0x7F0000001000;   // aligned, never read
    int32_t *const I = (int32_t *)F;
    size_t n = 0;
    int ok = 0;
    for (int i = 0; i < 200000; ++i) {
        lory_beam_shape s = {i % 50 == 0 ? 0 : spread(1 << 20), spread(64), spread(1 << 24), 1 + rnd(64), rnd(2), 0};
        s.row = s.vocab + (int64_t)rnd(3) * (1 << 30);
        const int rc = lory_beam_select_workspace_bytes(&s, &n);
        EXPECT(rc == ((int64_t)s.requests * s.beams > (1 << 20) ? LORY_ERR_SHAPE : LORY_OK));
        if (rc != LORY_OK) continue;
        ++ok;
        EXPECT(n % 256 == 0 && n <= (size_t)s.requests * s.beams * 16 * (16 + 8 * s.k) + 512);
        // workspace too small, nothing to do, or the outputs lie in the logits
        float *const f = (float *)(F + (1ll << 45));
        const int call = lory_beam_select(&s, F, f, f + (1 << 24), I + (1ll << 44), I + (1ll << 44) + (1 << 26), F + (3ll << 45), n ? n - 1 : 0, NULL);
        EXPECT(call == (s.requests == 0 ? LORY_OK : LORY_ERR_WORKSPACE) || call == LORY_ERR_OVERLAP);
    }
    EXPECT(ok > 10000);
    ok = 0;
    for (int i = 0; i < 200000; ++i) {
        lory_fork_shape s = {i % 40 == 0 ? 0 : spread(1 << 20), i % 30 == 0 ? 0 : spread(1 << 20), spread(1 << 30), spread(1 << 30), spread(INT32_MAX),
                             spread(INT32_MAX), 0, 0};
        s.table_row = s.width + (int64_t)rnd(3) * (1 << 30);
        s.new_row = s.width + (int64_t)rnd(3) * (1 << 30);
        const int rc = lory_kv_fork_workspace_bytes(&s, &n);
        EXPECT(rc == ((int64_t)s.width * s.page >= (1ll << 31) ? LORY_ERR_SHAPE : LORY_OK));
        if (rc != LORY_OK) continue;
        ++ok;
        EXPECT(n % 256 == 0 && n >= 2ull * s.pages + 4ull * s.old_rows + 4ull * s.rows);
        // every array at one address: an overlap
        EXPECT(lory_kv_fork(&s, I, I, I, I, I, I, I, I, I, I, F, n, NULL) == LORY_ERR_OVERLAP);
    }
    EXPECT(ok > 10000);
    for (int i = 0; i < 200000; ++i) {
        lory_copy_shape s = {i % 40 == 0 ? 0 : spread(1 << 20), spread(32767), spread(1 << 30), spread(1 << 30), spread(65535), 8 * (1 + rnd(32)), rnd(2)};
        const int rc = lory_kv_copy(&s, F, F, I, NULL);
        EXPECT(rc == LORY_ERR_SHAPE || rc == (s.n == 0 ? LORY_OK : LORY_ERR_OVERLAP));
    }
    ok = 0;
    for (int i = 0; i < 400000; ++i) {
        lory_paged_shape s = {};
        const int groups = i % 50 == 0 ? 0 : spread(1 << 20);
        s.rows = groups > 0 ? groups * spread((1 << 20) / groups) : 0;
        s.kv_heads = spread(65535);
        s.q_heads = s.kv_heads * spread(65535 / s.kv_heads);
        s.head_dim = 8 * (1 + rnd(32));
        s.pages = spread(1 << 30);
        s.page = spread(1 << 30);
        s.width = spread(1 << 30);
        s.dtype = rnd(2);
        s.table_row = s.width + (int64_t)rnd(3) * (1 << 30);
        s.scale = 0.1f;
        const int rc = lory_prefix_attn_workspace_bytes(&s, groups, &n);
        EXPECT(rc == LORY_OK || rc == LORY_ERR_SHAPE);
        if (rc != LORY_OK) continue;
        ++ok;
        EXPECT(n % 256 == 0 && n >= (size_t)s.rows * s.q_heads * s.head_dim * 4);
        const lory_heads q = {F, (int64_t)s.q_heads * s.head_dim, s.head_dim};
        const int call = lory_prefix_attn(&s, groups, &q, F, F, I, I, I, &q, NULL, F, n - 1, NULL);
        EXPECT(call == LORY_ERR_WORKSPACE || call == LORY_ERR_SHAPE);   // SHAPE: more rows of the cache than 31 bits
    }
    EXPECT(ok > 1000);
    if (failures) return 1;
    printf("beam abi sanitizer run: ok\n");
    return 0;
}
