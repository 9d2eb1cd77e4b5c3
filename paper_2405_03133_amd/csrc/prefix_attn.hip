// Attention of one new token per row where groups of rows have their first tokens in common (lory_prefix_attn).
//
// Bound by the bytes of the cache while few rows share a prefix: it is read once for up to 16 NQ queries (rows times query heads of a
// key-value head) of a group, and every row's own tokens once for its query heads.  With hundreds of queries the matrix cores and the
// exponentials bind.
//
// Work.  A wavefront holds NQ blocks of 16 queries and takes 32 (bf16) or 16 (fp32) keys at a time as paged_attn.hip does it; the
// operands of the keys and values, the values' transposition among them, serve all blocks.  A unit is kTile keys of one item: of a
// group's prefix for one key-value head and NQ blocks of queries, or of a row's own tokens for one key-value head and up to 16 of its
// queries.  The units of all prefixes and then of all rows are cut into equal ranges (a prefix unit counts `weight` times), a
// workgroup each; every range leaves the maximum, sum and unnormalised output of each item that it touches in the workspace, and a
// second launch joins an output's pieces in order: those of its group's prefix and those of its row.
//
// Measured (us, both launches): 24 groups of 8 rows, prefixes of 300 to 6000 tokens, 16 heads of 128 on 4: 39.6 + 7.5; 96 rows, 16000
// tokens in common, 32 heads on 8: 117.7 + 7.4; rows of one token of their own beside it 90 + 7.  Queries in registers instead of LDS, one workgroup a
// CU: 50 and 161.  Blocks: of heads of 128 four to a wavefront (one workgroup a CU) 135 where two take 115; of heads of 64 four 80, two 89.
// What an item counts beside its units: 1 150, 2 118, 4 130; the last tokens of every row left to the second launch instead: 31 + 22, 123 + 60.
// Bound now: with few queries by the chain of a unit (page, keys, values: 2 us a step on four wavefronts) and of a piece's start and
// end, 1.5 us; with hundreds by the steps' own instructions and the re-reads of the prefix, 489 MB where 361 are needed.
//
// A row is one of its group's where it has at least the group's shared tokens; a shorter one reads all its tokens by itself.
#include "attn_wave.h"
#include "lory_internal.h"
#include "paged_index.h"

namespace lory {

namespace {

using namespace attn;

constexpr int kCUs = 256;

struct Args {
    const char *q;
    long q_row, q_head;   // bytes
    const char *k, *v;
    const int32_t *table;
    long table_row;
    const int32_t *lens, *shared;
    char *out;
    long out_row, out_head;   // bytes
    float *lse;
    int32_t *gstart, *rstart;   // workspace: units of one head before each group's prefix, each row; with the sum of all behind
    float *part_o;              // pieces: [places][D], a place a query
    float2 *part_ml;            // [places], maximum and sum
    long row_places, more_places;   // first place of the rows' pieces, and of pieces that do not begin an item
    int rows, groups, beams, Hq, Hkv, D, pages, page, width;
    int group, tiles;           // query heads of a key-value head, and blocks of 16 of them
    int queries, chunks;        // of a group and key-value head, and chunks of 16 NQ of them
    int weight;
    int ranges;                 // workgroups
    paged::Divider div;         // by page
    float scale;
};

__device__ __forceinline__ int clamped(const Args &a, int n)
{
    const int most = a.width * a.page;
    return n < 0 ? 0 : n < most ? n : most;
}
__device__ __forceinline__ int length_of(const Args &a, int b) { return clamped(a, a.lens[b]); }
__device__ __forceinline__ int shared_of(const Args &a, int g) { return clamped(a, a.shared[g]); }
// first token that a row reads by itself
__device__ __forceinline__ int own_from(int len, int shared) { return len >= shared ? shared : 0; }

// Units of that many tokens, and what an item of them counts: as many, and kStart for finding its pages and joining its wavefronts.
constexpr int kStart = 2;
template <typename T> __device__ __forceinline__ int units_of(int tokens)
{
    return tokens > 0 ? (tokens + kTile<T> - 1) / kTile<T> + kStart : 0;
}

template <int DP, int NQ> struct Shared {
    u32x4 q[NQ * DP / 32 * 64];    // operands of the queries, DP / 32 pieces of 16 bytes a lane and block of bf16, twice that of fp32
    alignas(16) float o[kWaves][16][DP + 4];   // a wavefront's output of one block, unnormalised
    float m[kWaves][16], l[kWaves][16];
};

// Tokens first .. last of the row whose table is `pages`, for key-value head kvh and nq queries; query(x): address of one, or
// NULL: it takes no part.  The piece goes to the places from `place` on.
template <typename T, int DP, bool PAD, bool STREAM, int NQ, typename Lds, typename Query>
__device__ __forceinline__ void piece(const Args &a, Lds &sh, const int32_t *pages, int kvh, int first, int last, int nq,
                                      long place, const Query &query)
{
    using W = Wave<T, DP, PAD, NQ>;
    constexpr int KEYS = kKeys<T>, STEP = kTile<T>, NS = KEYS / 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, c = lane >> 4;

    W w;
    auto page_of = [&](int at) {
        const int t = at + (lane & (KEYS - 1));
        return t < last ? pages[paged::quotient(a.div, t)] : -1;
    };
    auto row_of = [&](int at, int page) {
        return paged::cache_row(a.div, at + (lane & (KEYS - 1)), page, a.pages, a.Hkv, kvh);
    };
    const int at0 = first + wave * KEYS, page0 = page_of(at0), page1 = page_of(at0 + STEP);
    // the queries' operands lie in LDS: registers are what limits the wavefronts that run
    constexpr int KS = W::KS;
    if (wave < NQ) {
        const char *p = wave * 16 + i < nq ? query(wave * 16 + i) : nullptr;
        typename W::Query q;
        W::load_q(q, p, a.D, c, p != nullptr);
#pragma unroll
        for (int s = 0; s < KS; ++s) sh.q[(wave * KS + s) * 64 + lane] = __builtin_bit_cast(u32x4, q[s]);
    }
    __syncthreads();
    float m[NQ], l[NQ];
    auto walk = [&](auto split, int page, int next) {
        typename W::Keys x;
        int at = at0;
#pragma unroll
        for (int b = 0; b < NQ; ++b) {
#pragma unroll
            for (int t = 0; t < W::NT; ++t) w.o[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[b] = -INFINITY;
            l[b] = 0.f;
        }
        int row = row_of(at, page);
        if (at < last) {
            W::load_k(x, a.k, max(row, 0), a.D, i, c);
            W::template load_v<STREAM>(x, a.v, max(row, 0), a.D, i, c);
        }
        for (; at < last; at += STEP) {
#pragma clang fp contract(off)
            const uint32_t valid = paged::valid_keys(__ballot(row >= 0), KEYS);
            row = row_of(at + STEP, next);
            next = page_of(at + 2 * STEP);
            const bool more = at + STEP < last;

            float s[NQ][NS];
            asm volatile("" ::: "memory");   // the queries are read in every step: kept in registers they would cost others their place
#pragma unroll
            for (int b = 0; b < NQ; ++b) {
                typename W::Query q;
#pragma unroll
                for (int t = 0; t < KS; ++t) q[t] = __builtin_bit_cast(typename std::remove_reference<decltype(q[0])>::type, sh.q[(b * KS + t) * 64 + lane]);
                W::scores(q, x, s[b]);
            }
            if (more) W::load_k(x, a.k, max(row, 0), a.D, i, c);
            const bool full = valid == paged::all_keys(KEYS);
            if (!full) W::clear_v(x, valid, c);
#pragma unroll
            for (int b = 0; b < NQ; ++b) {
#pragma unroll
                for (int n = 0; n < NS; ++n) s[b][n] *= a.scale;
                if (!full) {
#pragma unroll
                    for (int n = 0; n < NS; ++n)
                        if (!((valid >> ((n >> 2) * 16 + 4 * c + (n & 3))) & 1)) s[b][n] = -INFINITY;
                }
                float top = s[b][0];
#pragma unroll
                for (int n = 1; n < NS; ++n) top = fmaxf(top, s[b][n]);
                const float m1 = fmaxf(m[b], xor_max(top));
                const float ref = m1 == -INFINITY ? 0.f : m1;   // nothing but -inf so far: every weight is 0
                if (__any(m1 != m[b])) {
                    const float f = exp_of(m[b] - ref);
                    l[b] *= f;
#pragma unroll
                    for (int t = 0; t < W::NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w.o[b][t][e] *= f;
                }
                m[b] = m1;
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    s[b][n] = exp_of(s[b][n] - ref);
                    l[b] += s[b][n];
                }
            }
            w.template add<decltype(split)::value>(x, s);
            if (more) W::template load_v<STREAM>(x, a.v, max(row, 0), a.D, i, c);
        }
    };
    walk(std::false_type(), page0, page1);
    if constexpr (sizeof(T) == 2) {   // infinite values among these keys: once more, with what they take in every step
        bool odd = false;
#pragma unroll
        for (int b = 0; b < NQ; ++b) odd |= b * 16 + i < nq && w.odd(b);
        if (__builtin_expect(__any(odd), 0)) walk(std::true_type(), page_of(at0), page_of(at0 + STEP));
    }

#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const int n = min(16, nq - 16 * b);
        if (n <= 0) break;
        const float L = xor_sum(l[b]);
        if (c == 0) {
            sh.m[wave][i] = m[b];
            sh.l[wave][i] = L;
        }
        if (i < n) {
#pragma unroll
            for (int t = 0; t < W::NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) sh.o[wave][i][W::dim(t, 4 * c + r)] = w.o[b][t][r];
        }
        __syncthreads();
        const int j = tid / 16;   // 16 threads a query, four dims at a time
        if (j < n) {
            float M = sh.m[0][j];
#pragma unroll
            for (int v = 1; v < kWaves; ++v) M = fmaxf(M, sh.m[v][j]);
            const float ref = M == -INFINITY ? 0.f : M;
            float S = 0.f, f[kWaves];
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                f[v] = exp_of(sh.m[v][j] - ref);
                S = fmaf(f[v], sh.l[v][j], S);
            }
            const long to = place + 16 * b + j;
            float *out = a.part_o + to * a.D;
            for (int d = tid % 16 * 4; d < a.D; d += 64) {
                f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int v = 0; v < kWaves; ++v) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(&sh.o[v][j][d]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[e] = fmaf(f[v], x[e], O[e]);
                }
                *reinterpret_cast<f32x4 *>(out + d) = O;
            }
            if (tid % 16 == 0) a.part_ml[to] = make_float2(M, S);
        }
        __syncthreads();
    }
}

// Units of all prefixes and rows, and the ranges they are cut into: each is at least as long as one unit counts.
struct Cut {
    long prefix, all;   // cost of the prefixes' units, and of all
    int ranges;
};
__device__ __forceinline__ Cut cut_of(const Args &a, long group_units, long row_units)
{
    Cut c;
    c.prefix = group_units * a.Hkv * a.chunks * a.weight;
    c.all = c.prefix + row_units * a.Hkv * a.tiles;
    const long n = c.all / a.weight;
    c.ranges = n < 1 ? 1 : n < a.ranges ? (int)n : a.ranges;
    return c;
}

// Workgroups of four wavefronts that the registers let a CU hold.
constexpr int resident(int esize, int head_dim, int nq)
{
    return head_dim <= 64 ? (esize == 4 || nq == 1 ? 3 : 2) : head_dim <= 128 ? (nq <= 2 ? 2 : 1) : 1;
}

template <typename T, int DP, bool PAD, bool STREAM, int NQ>
__global__ __launch_bounds__(kThreads, resident(sizeof(T), DP, NQ)) void prefix_attn_kernel(Args a)
{
    __shared__ Shared<DP, (sizeof(T) / 2) * NQ> sh;
    __shared__ int wsum[2][kWaves];
    __shared__ struct { int item, rest_units; long rest; } from[2];   // group or row of the range's first unit, and units of it before that
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // units of one head, of the thread's chunk of groups and of rows: its own, then those before and those of all
    const int gchunk = (a.groups + kThreads - 1) / kThreads, g0 = min(tid * gchunk, a.groups), g1 = min(g0 + gchunk, a.groups);
    const int rchunk = (a.rows + kThreads - 1) / kThreads, r0 = min(tid * rchunk, a.rows), r1 = min(r0 + rchunk, a.rows);
    auto row_units = [&](int b) {
        const int len = length_of(a, b);
        return units_of<T>(len - own_from(len, shared_of(a, b / a.beams)));
    };
    int gown = 0, rown = 0;
    for (int g = g0; g < g1; ++g) gown += units_of<T>(shared_of(a, g));
    for (int b = r0; b < r1; ++b) rown += row_units(b);
    int gupto = gown, rupto = rown;
    for (int m = 1; m < 64; m <<= 1) {
        const int g = __shfl_up(gupto, m, 64), r = __shfl_up(rupto, m, 64);
        if (lane >= m) {
            gupto += g;
            rupto += r;
        }
    }
    if (lane == 63) {
        wsum[0][wave] = gupto;
        wsum[1][wave] = rupto;
    }
    __syncthreads();
    int gall = 0, rall = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) {
            gupto += wsum[0][w];
            rupto += wsum[1][w];
        }
        gall += wsum[0][w];
        rall += wsum[1][w];
    }
    if (blockIdx.x == 0) {   // for the launch that joins
        int n = gupto - gown;
        for (int g = g0; g < g1; ++g) {
            a.gstart[g] = n;
            n += units_of<T>(shared_of(a, g));
        }
        n = rupto - rown;
        for (int b = r0; b < r1; ++b) {
            a.rstart[b] = n;
            n += row_units(b);
        }
        if (tid == 0) {
            a.gstart[a.groups] = gall;
            a.rstart[a.rows] = rall;
        }
    }
    const Cut cut = cut_of(a, gall, rall);
    // neighbouring ranges on one of the eight XCDs, as they read the same prefix for other queries
    const int w = cut.ranges == a.ranges ? (blockIdx.x % 8) * (a.ranges / 8) + blockIdx.x / 8 : blockIdx.x;
    if (w >= cut.ranges || cut.all == 0) return;
    const long x0 = paged::range_begin(w, cut.all, cut.ranges), x1 = paged::range_begin(w + 1, cut.all, cut.ranges);
    const int gheads = a.Hkv * a.chunks, rheads = a.Hkv * a.tiles;
    long u = min((x0 + a.weight - 1) / a.weight, (long)gall * gheads), v = max(0l, x0 - cut.prefix);
    const long uend = min((x1 + a.weight - 1) / a.weight, (long)gall * gheads), vend = max(0l, x1 - cut.prefix);

    if (u < uend && (long)(gupto - gown) * gheads <= u && u < (long)gupto * gheads) {   // one thread's chunk has the first unit
        long rest = u - (long)(gupto - gown) * gheads;
        int g = g0, n = units_of<T>(shared_of(a, g));
        for (; g < g1 - 1 && rest >= (long)n * gheads; n = units_of<T>(shared_of(a, ++g))) rest -= (long)n * gheads;
        from[0] = {g, n, rest};
    }
    if (v < vend && (long)(rupto - rown) * rheads <= v && v < (long)rupto * rheads) {
        long rest = v - (long)(rupto - rown) * rheads;
        int b = r0, n = row_units(b);
        for (; b < r1 - 1 && rest >= (long)n * rheads; n = row_units(++b)) rest -= (long)n * rheads;
        from[1] = {b, n, rest};
    }
    __syncthreads();

    if (u < uend) {
        int g = from[0].item, units = from[0].rest_units;
        int h = (int)paged::quotient64(from[0].rest, units), tile = (int)(from[0].rest - (long)h * units);
        while (u < uend) {
            const int shared = shared_of(a, g), stop = (int)(uend - u < units - tile ? tile + (uend - u) : units);
            const int t0 = max(0, tile - kStart), t1 = stop - kStart;
            // a row that has all of the prefix: its table is read
            int has = INT32_MAX;
            for (int r = lane; r < a.beams; r += 64)
                if (length_of(a, g * a.beams + r) >= shared) has = min(has, r);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) has = min(has, __shfl_xor(has, o, 64));
            has = __builtin_amdgcn_readfirstlane(has);
            const int kvh = a.chunks == 1 ? h : h / a.chunks, q0 = (h - kvh * a.chunks) * 16 * NQ;
            if (has != INT32_MAX && t0 < t1) {
                auto query = [&](int x) -> const char * {
                    const int r = (q0 + x) / a.group, b = g * a.beams + r;
                    if (length_of(a, b) < shared) return nullptr;
                    return a.q + b * a.q_row + (kvh * a.group + (q0 + x) - r * a.group) * a.q_head;
                };
                piece<T, DP, PAD, false, NQ>(a, sh, a.table + ((long)g * a.beams + has) * a.table_row, kvh, t0 * kTile<T>,
                                              min(t1 * kTile<T>, shared), min(16 * NQ, a.queries - q0),
                                              t0 == 0 ? ((long)g * gheads + h) * 16 * NQ : a.more_places + (long)w * 16 * NQ, query);
            }
            u += stop - tile;
            tile = 0;
            if (stop == units && ++h == gheads && u < uend) {
                h = 0;
                do units = units_of<T>(shared_of(a, ++g)); while (units == 0);
            }
        }
    }
    if (v < vend) {
        int b = from[1].item, units = from[1].rest_units;
        int h = (int)paged::quotient64(from[1].rest, units), tile = (int)(from[1].rest - (long)h * units);
        while (v < vend) {
            const int stop = (int)(vend - v < units - tile ? tile + (vend - v) : units);
            const int t0 = max(0, tile - kStart), t1 = stop - kStart;
            const int len = length_of(a, b), start = own_from(len, shared_of(a, b / a.beams));
            const int kvh = a.tiles == 1 ? h : h / a.tiles, head = kvh * a.group + (h - kvh * a.tiles) * 16;
            const int nq = min(16, (kvh + 1) * a.group - head), most = min(16, a.group);
            auto query = [&](int x) -> const char * { return a.q + b * a.q_row + (head + x) * a.q_head; };
            if (t0 < t1)
                piece<T, DP, PAD, STREAM, 1>(a, sh, a.table + b * a.table_row, kvh, start + t0 * kTile<T>,
                                         min(start + t1 * kTile<T>, len), nq,
                                         t0 == 0 ? a.row_places + ((long)b * rheads + h) * most : a.more_places + (long)w * 16 * NQ, query);
            v += stop - tile;
            tile = 0;
            if (stop == units && ++h == rheads && v < vend) {
                h = 0;
                do units = row_units(++b); while (units == 0);
            }
        }
    }
}

// Joins the pieces of one row's head, grid (heads, rows): every thread takes four dims of one query over a share of the pieces,
// and the shares are added in order.
template <typename T> __global__ __launch_bounds__(kJoinThreads) void prefix_attn_join_kernel(Args a, int NQ)
{
    __shared__ f32x4 so[kJoinThreads];
    __shared__ float2 sml[kJoinThreads];
    const int h = blockIdx.x, tid = threadIdx.x;
    const int kvh = a.tiles == 1 ? h : h / a.tiles, first = (h - kvh * a.tiles) * 16;   // query head of the key-value head
    const int nq = min(16, a.group - first), most = min(16, a.group);
    const int gheads = a.Hkv * a.chunks, rheads = a.Hkv * a.tiles, chunk = 16 * NQ;
    const Cut cut = cut_of(a, a.gstart[a.groups], a.rstart[a.rows]);
    for (int b = blockIdx.y; b < a.rows; b += gridDim.y) {
        const int g = b / a.beams, len = length_of(a, b), shared = shared_of(a, g);
        const int gspan = a.gstart[g + 1] - a.gstart[g], runits = a.rstart[b + 1] - a.rstart[b], gunits = len >= shared ? gspan : 0;
        int rw0 = 0, rparts = 0;
        if (runits > 0) {
            const long u = cut.prefix + (long)a.rstart[b] * rheads + (long)h * runits;
            rw0 = paged::owner(u + kStart, cut.all, cut.ranges);
            rparts = paged::owner(u + runits - 1, cut.all, cut.ranges) - rw0 + 1;
        }
        const int quads = a.D / 4, all = nq * quads;
        int per = 16;   // threads that share a piece
        while (per < all && per < kJoinThreads) per <<= 1;
        const int shares = kJoinThreads / per, share = tid / per;
        for (int x0 = 0; x0 < all; x0 += per) {
            const int x = x0 + tid % per;
            const bool on = x < all;
            const int j = on ? x / quads : 0, d = on ? x - j * quads : 0;
            const int query = (b - g * a.beams) * a.group + first + j, c = query / chunk, at = query - c * chunk;
            int gw0 = 0, gparts = 0;
            if (gunits > 0) {
                const long u = (long)a.gstart[g] * gheads + (long)(kvh * a.chunks + c) * gunits;
                gw0 = paged::owner((u + kStart) * a.weight, cut.all, cut.ranges);
                gparts = paged::owner((u + gunits - 1) * a.weight, cut.all, cut.ranges) - gw0 + 1;
            }
            const int parts = gparts + rparts;
            auto place_of = [&](int p) -> long {
                if (p < gparts) return (p == 0 ? ((long)g * gheads + kvh * a.chunks + c) * chunk : a.more_places + (long)(gw0 + p) * chunk) + at;
                p -= gparts;
                return (p == 0 ? a.row_places + ((long)b * rheads + h) * most : a.more_places + (long)(rw0 + p) * chunk) + j;
            };
            float M = -INFINITY, L = 0.f;
            f32x4 O = {0.f, 0.f, 0.f, 0.f};
            auto take = [&](float m, float l, f32x4 o) {
                const float M1 = fmaxf(M, m), ref = M1 == -INFINITY ? 0.f : M1;
                const float f = exp_of(M - ref), e = exp_of(m - ref);
                L = L * f + l * e;
#pragma unroll
                for (int n = 0; n < 4; ++n) O[n] = O[n] * f + o[n] * e;
                M = M1;
            };
            // eight pieces at a time, all under way at once; where there are fewer, the last ones are empty
            for (int p0 = share; on && p0 < parts; p0 += 8 * shares) {
                float2 ml[8];
                f32x4 o[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    ml[n] = make_float2(-INFINITY, 0.f);
                    o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (p0 + n * shares < parts) {
                        const long from = place_of(p0 + n * shares);
                        ml[n] = a.part_ml[from];
                        o[n] = *reinterpret_cast<const f32x4 *>(a.part_o + from * 4 * quads + 4 * d);
                    }
                }
#pragma unroll
                for (int n = 0; n < 8; ++n) take(ml[n].x, ml[n].y, o[n]);
            }
            if (shares > 1) {
                so[tid] = O;
                sml[tid] = make_float2(M, L);
                __syncthreads();
                if (share == 0)
                    for (int n = 1; n < shares; ++n) take(sml[n * per + tid].x, sml[n * per + tid].y, so[n * per + tid]);
                __syncthreads();
            }
            if (share == 0 && on) {
                const float ref = M == -INFINITY ? 0.f : M, n = L == 0.f ? 1.f : L;
                const int head = kvh * a.group + first + j;
                char *p = a.out + b * a.out_row + head * a.out_head + 4 * d * (int)sizeof(T);
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<gemm::u32x2 *>(p) = gemm::u32x2{gemm::cvt_pk_bf16(O[0] / n, O[1] / n), gemm::cvt_pk_bf16(O[2] / n, O[3] / n)};
                else
                    *reinterpret_cast<f32x4 *>(p) = f32x4{O[0] / n, O[1] / n, O[2] / n, O[3] / n};
                if (d == 0 && a.lse) a.lse[(long)b * a.Hq + head] = fmaf(log2f(L), kLn2, ref);
            }
        }
    }
}

// Blocks of 16 queries that a wavefront holds: as many as the rows of a group have, and as leave room for two workgroups on a CU
// (measured on both sides, above).
int blocks(const lory_paged_shape &s, int groups)
{
    const long n = groups > 0 ? (long)(s.rows / groups) * (s.q_heads / s.kv_heads) : 1;
    int most = s.head_dim > 128 ? 1 : s.dtype == LORY_F32 || s.head_dim > 64 ? 2 : 4;
    while (most > 1 && n <= 8 * most) most /= 2;
    return most;
}

struct Sizes {
    int nq, ranges, chunks, tiles, most;
    long row_places, more_places, places;
    size_t gstart, rstart, o, ml;
    Sizes(const lory_paged_shape &s, int groups)
    {
        const int group = s.q_heads / s.kv_heads;
        nq = blocks(s, groups);
        ranges = kCUs * resident(s.dtype == LORY_F32 ? 4 : 2, s.head_dim, nq);
        const long n = groups > 0 ? (long)(s.rows / groups) * group : 0;
        chunks = (int)((n + 16 * nq - 1) / (16 * nq));
        tiles = (group + 15) / 16;
        most = group < 16 ? group : 16;
        row_places = (long)groups * s.kv_heads * chunks * 16 * nq;
        more_places = row_places + (long)s.rows * s.kv_heads * tiles * most;
        places = more_places + (long)ranges * 16 * nq;
        gstart = align_up(((size_t)groups + 1) * 4, 256);
        rstart = align_up(((size_t)s.rows + 1) * 4, 256);
        o = (size_t)places * s.head_dim * 4;
        ml = (size_t)places * 8;
    }
    size_t all() const { return align_up(gstart + rstart + o + ml, 256); }
};

template <typename T, int DP, bool PAD, int NQ> void launch4(const Args &a, bool stream, hipStream_t st)
{
    if (stream)
        hipLaunchKernelGGL((prefix_attn_kernel<T, DP, PAD, true, NQ>), dim3(a.ranges), dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((prefix_attn_kernel<T, DP, PAD, false, NQ>), dim3(a.ranges), dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL((prefix_attn_join_kernel<T>), dim3(a.Hkv * a.tiles, a.rows < 32768 ? a.rows : 32768), dim3(kJoinThreads), 0, st, a, NQ);
}

template <typename T, int DP, bool PAD> void launch3(const Args &a, int nq, bool stream, hipStream_t st)
{
    constexpr int most = DP > 128 ? 1 : sizeof(T) == 4 || DP > 64 ? 2 : 4;
    if (nq == 1) return launch4<T, DP, PAD, 1>(a, stream, st);
    if constexpr (most >= 2) {
        if (nq == 2) return launch4<T, DP, PAD, 2>(a, stream, st);
    }
    if constexpr (most >= 4) launch4<T, DP, PAD, 4>(a, stream, st);
}

template <typename T, int DP> void launch2(const Args &a, int nq, bool stream, hipStream_t st)
{
    if (a.D == DP)
        launch3<T, DP, false>(a, nq, stream, st);
    else
        launch3<T, DP, true>(a, nq, stream, st);
}

template <typename T> void launch1(const Args &a, int nq, bool stream, hipStream_t st)
{
    if (a.D <= 64)
        launch2<T, 64>(a, nq, stream, st);
    else if (a.D <= 128)
        launch2<T, 128>(a, nq, stream, st);
    else
        launch2<T, 256>(a, nq, stream, st);
}

}  // namespace

size_t prefix_attn_workspace_bytes(const lory_paged_shape &s, int groups) { return Sizes(s, groups).all(); }

int prefix_attn_launch(const lory_paged_shape &s, int groups, const lory_heads &q, const void *k_cache, const void *v_cache,
                       const int32_t *table, const int32_t *lens, const int32_t *shared, const lory_heads &out, float *lse, void *ws,
                       hipStream_t st)
{
    const int esize = s.dtype == LORY_F32 ? 4 : 2;
    const Sizes z(s, groups);
    Args a = {};
    a.q = (const char *)q.data;
    a.q_row = q.token * esize;
    a.q_head = q.head * esize;
    a.k = (const char *)k_cache;
    a.v = (const char *)v_cache;
    a.table = table;
    a.table_row = s.table_row;
    a.lens = lens;
    a.shared = shared;
    a.out = (char *)out.data;
    a.out_row = out.token * esize;
    a.out_head = out.head * esize;
    a.lse = lse;
    a.gstart = (int32_t *)ws;
    a.rstart = (int32_t *)((char *)ws + z.gstart);
    a.part_o = (float *)((char *)ws + z.gstart + z.rstart);
    a.part_ml = (float2 *)((char *)ws + z.gstart + z.rstart + z.o);
    a.row_places = z.row_places;
    a.more_places = z.more_places;
    a.rows = s.rows;
    a.groups = groups;
    a.beams = s.rows / groups;
    a.Hq = s.q_heads;
    a.Hkv = s.kv_heads;
    a.D = s.head_dim;
    a.pages = s.pages;
    a.page = s.page;
    a.width = s.width;
    a.group = s.q_heads / s.kv_heads;
    a.tiles = z.tiles;
    a.queries = a.beams * a.group;
    a.chunks = z.chunks;
    // A unit of four blocks takes longer than a row's of one.  Heads of 64, rows / tokens in common / of their own, us with a weight of 1, 2, 3:
    // 96 / 16000 / 1500 81, 73, 88; 96 / 4000 / 1500 58, 46, 52; 8 groups of 16 / 1000-8000 / 150 32, 27, 25; 6 of 40 / 3000 / 2000 81, 70, 76; 200 /
    // 30000 / 300 94, 87, 96.  Units of one and two blocks count as a row's: with 1.5 the 24
    // groups above take 35 for 40, but the long prefix 145 for 118.
    a.weight = z.nq == 4 ? 2 : 1;
    a.ranges = z.ranges;
    a.div = paged::divider(s.page);
    a.scale = s.scale;
    prof::Range r(st, prof::kPrefixAttn, 0.0, 0.0);   // the lengths are on the device
    // rows' own values of large caches past them, from where paged_attn.hip measured it; a prefix may be read by several workgroups
    const bool stream = 2 * (long)s.pages * s.kv_heads * s.page * s.head_dim * esize > (64l << 20);
    if (s.dtype == LORY_F32)
        launch1<float>(a, z.nq, stream, st);
    else
        launch1<__hip_bfloat16>(a, z.nq, stream, st);
    return launch_status();
}

}  // namespace lory
