// Attention of one new token per row over a paged key-value cache (lory_paged_attn).
//
// Bound by the bytes of the cache: every key and value is read once for up to 16 query heads that share it, and again for
// every 16 more.
//
// Work.  A unit is kTile keys of one key-value head of one row (of up to 16 of its query heads).  Short rows are a workgroup
// each, or every row is cut into the same number of ranges; else the units of all rows and heads, in order, are cut into as
// many equal ranges as workgroups run at a time, whatever the rows' lengths, which only the device knows: every workgroup takes the
// sums over the lengths for itself (the choice: plan, below).  A range ends inside a row's units as it comes; such a piece leaves
// its maximum, sum and unnormalised output in the workspace (at most two pieces a workgroup: the first and the
// last), and a second launch joins the pieces of a row in order.  Rows that lie in one range are written directly.
//
// A wavefront takes 32 (bf16) or 16 (fp32) keys at a time, straight from memory to the operands of the matrix cores:
//   S^T [keys x queries] = K Q^T   A = K: lane (i, c) holds pieces of 16 bytes of key i
//   O^T [dims x queries] += V^T P^T
// S^T leaves a lane with the scores of its query (column i) and of keys 4c .. 4c+3, which is the layout of P^T as the
// other product's operand if its keys are taken in that order, so the probabilities never move between lanes.  V rows are
// read whole by 16 lanes; lane i holds dims nt i .. nt i + nt - 1 of eight keys, and a v_perm per pair of keys gives the operand of
// one matrix instruction per dim: row i of output tile t is dim nt i + t.  fp32 needs no transposition (one key per lane and instruction).
// The probabilities go in as two bf16 terms (p = hi + lo, error 2^-16): one alone would round every weight of the sum to
// 2^-8, and the matrix cores wait for memory anyway.  An infinite value would be NaN with the second term; a wavefront whose
// sums are not finite takes its keys again and leaves it out there (the check costs 0.1 to 0.3 us a call).
//
// Pages: the lane that owns a key looks its page up two steps ahead; the others fetch the row by a lane permute.
//
// Measured: four rows of 50000 to 131072 tokens, 32 query heads on 8, heads of 128, bf16: 216 us + 5.8 for the join, 6.5 TB/s
// (a pass that only reads reaches 6.7); 48 rows of 1 to 9000 tokens 22.8 + 5.2 us, 4.5 TB/s; HBM traffic is the cache's
// bytes and 1 MB of pieces.  One CU takes in about 60 bytes per ns however many loads are under way (a second step in flight,
// 16 wavefronts instead of eight or steps of 16 keys change nothing), so a short row costs 4 us and its bytes at that
// rate.  Joining in the workgroup that finishes last instead of a second launch was tried: with fences between the XCDs
// a ragged batch takes 55 us instead of 31, with agent-scope loads and stores 34.
#include <hip/hip_bf16.h>

#include <type_traits>

#include "gemm_bf16.h"
#include "lory_internal.h"
#include "paged_index.h"

namespace lory {

namespace {

using gemm::bf16x8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4, kJoinThreads = 256;
constexpr int kCUs = 256;
// Workgroups of four wavefronts that the registers let a CU hold (heads of up to 64, 128, 256): 100 rows of 100 to 4000 tokens,
// 8 heads of 64, in 512 ranges 58.8 us, in 768 52.2.
constexpr int resident(int head_dim) { return head_dim <= 64 ? 3 : head_dim <= 128 ? 2 : 1; }
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
    const char *q;
    long q_row, q_head;   // bytes
    const char *k, *v;
    const int32_t *table;
    long table_row;
    const int32_t *lens;
    char *out;
    long out_row, out_head;   // bytes
    float *lse;
    int32_t *starts;          // workspace: units of one head before each row, [rows + 1]
    float2 *part_o;           // pieces: [slots][part_rows][D / 2]
    float2 *part_ml;          // [slots][part_rows], maximum and sum
    int part_rows;
    int rows, Hq, Hkv, D, pages, page, width;
    int group, tiles;         // query heads of a key-value head, and blocks of 16 of them
    int groups;               // ranges that share the units
    paged::Divider div;       // by page
    float scale;
};

// Values are read past the caches where the key-value cache is too large to be found in the memory-side cache (256 MB, of which
// other layers want their share) when it is read again: from 64 MB on.  us with and without: four rows of 50000 to
// 131072 tokens 220 / 246, 16 rows of 500 to 3000, 16 heads of 128 36.6 / 42, a ragged batch of 103 MB 28.0 / 30.3; 25 MB that
// were read just before 10.1 / 9.0.  Keys are not: their lines are read by two instructions each (37.8 there).
// The size is that of all pages, a sign of what else the program reads, and not what the call can reach: rows of 1000 tokens, 8 heads
// of 128, in pages spread over 6 GB, read in turn with seven like calls 24 MB 12.1 / 11.9, 48 MB 17.1 / 19.1, 64 MB 19.1 / 21.5,
// 128 MB 25.8 / 27.6; read again at once, which a program of several layers does not, 10.3 / 10.3, 16.0 / 14.7, 17.0 / 15.2, 22.9 / 22.6.
// Nor does it matter that several workgroups read a value, for more than 16 query heads on a key-value head: 164 MB, 32 on one
// 48.8 / 50.7, 64 on one 69.4 / 68.9, 123 MB, 128 on one 87.8 / 87.5 (called again at once 48.0 / 40.7, 67.8 / 58.6, 86.3 / 79.3).
constexpr long kStreamBytes = 64l << 20;

template <bool STREAM, typename V> __device__ __forceinline__ V load_value(const char *p)
{
    if constexpr (STREAM)
        return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else
        return *reinterpret_cast<const V *>(p);
}

template <typename T> constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;   // of a wavefront's step
template <typename T> constexpr int kTile = kKeys<T> * kWaves;

__device__ __forceinline__ int length_of(const Args &a, int b)
{
    const int n = a.lens[b], most = a.width * a.page;
    return n < 0 ? 0 : n < most ? n : most;
}

template <typename T> __device__ __forceinline__ int units_of(int len)
{
    return len <= kTile<T> ? 1 : (len + kTile<T> - 1) / kTile<T>;   // an empty row has one, which writes its zeros
}

// e^x for x <= 0
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ float xor_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float xor_sum(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// One row's head for one wavefront: the operand of Q, the running softmax and the output.
// DP: head_dim rounded up to 64, 128 or 256.  PAD: head_dim < DP (pieces behind it are zeros that nothing loads).
template <typename T, int DP, bool PAD> struct Wave;

template <int DP, bool PAD> struct Wave<__hip_bfloat16, DP, PAD> {
    static constexpr int KS = DP / 32;     // K steps of a product over the dims
    static constexpr int NT = DP / 16;     // output tiles
    static constexpr int VW = NT < 8 ? NT : 8;   // dims of a V load
    static constexpr int VL = NT / VW;     // V loads of a key
    struct Keys {   // of a step
        u32x4 k[2][KS];
        uint32_t v[8][VL][VW / 2];
    };
    bf16x8 q[KS];
    f32x4 o[NT];

    // dim of row i of output tile t
    static __device__ int dim(int t, int i) { return (t / VW) * 16 * VW + VW * i + t % VW; }

    __device__ void load_q(const char *p, int D, int c, bool on)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u32x4 r = {0, 0, 0, 0};
            if (on && (!PAD || (4 * s + c) * 8 < D)) r = *reinterpret_cast<const u32x4 *>(p + (4 * s + c) * 16);
            q[s] = __builtin_bit_cast(bf16x8, r);
        }
    }
    // row: of the lane's own key of the step (lane & 31)
    __device__ static void load_k(Keys &x, const char *base, int row, int D, int i, int c)
    {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const uint32_t r = __shfl(row, kt * 16 + i, 64);
            const char *p = base + (uint64_t)r * (uint32_t)(PAD ? D * 2 : DP * 2) + c * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (PAD) x.k[kt][s] = u32x4{0, 0, 0, 0};
                if (!PAD || (4 * s + c) * 8 < D) x.k[kt][s] = *reinterpret_cast<const u32x4 *>(p + s * 64);
            }
        }
    }
    template <bool STREAM> __device__ static void load_v(Keys &x, const char *base, int row, int D, int i, int c)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = __shfl(row, (j >> 2) * 16 + 4 * c + (j & 3), 64);
            const char *p = base + (uint64_t)r * (uint32_t)(PAD ? D * 2 : DP * 2) + i * (VW * 2);
#pragma unroll
            for (int m = 0; m < VL; ++m) {
                if constexpr (VW == 8) {
                    u32x4 y = {0, 0, 0, 0};
                    if (!PAD || (16 * m + i) * 8 < D) y = load_value<STREAM, u32x4>(p + m * 256);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[j][m][e] = y[e];
                } else {
                    gemm::u32x2 y = {0, 0};
                    if (!PAD || i * 4 < D) y = load_value<STREAM, gemm::u32x2>(p);
                    x.v[j][m][0] = y[0];
                    x.v[j][m][1] = y[1];
                }
            }
        }
    }
    // s[n]: score of the lane's query with key (n / 4) * 16 + 4c + n % 4
    __device__ void scores(const Keys &x, float (&s)[8])
    {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KS; ++t)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[kt][t]), q[t], acc, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[kt * 4 + r] = acc[r];
        }
    }
    // the values of keys that are left out have no bits that may enter a product
    __device__ static void clear_v(Keys &x, uint32_t valid, int c)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool on = (valid >> ((j >> 2) * 16 + 4 * c + (j & 3))) & 1;
#pragma unroll
            for (int m = 0; m < VL; ++m)
#pragma unroll
                for (int e = 0; e < VW / 2; ++e) x.v[j][m][e] = on ? x.v[j][m][e] : 0;
        }
    }
    // SPLIT: an infinite value counts with hi alone (a lo of 0 or of the other sign would make NaN of it)
    template <bool SPLIT> __device__ void add(const Keys &x, const float (&p)[8])
    {
        u32x4 hi, lo;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            hi[n] = gemm::cvt_pk_bf16(p[2 * n], p[2 * n + 1]);
            lo[n] = gemm::cvt_pk_bf16(p[2 * n] - __uint_as_float(hi[n] << 16), p[2 * n + 1] - __uint_as_float(hi[n] & 0xffff0000u));
        }
        const bf16x8 bh = __builtin_bit_cast(bf16x8, hi), bl = __builtin_bit_cast(bf16x8, lo);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4 y;
#pragma unroll
            for (int n = 0; n < 4; ++n)
                y[n] = __builtin_amdgcn_perm(x.v[2 * n + 1][t / VW][(t % VW) / 2], x.v[2 * n][t / VW][(t % VW) / 2],
                                             (t & 1) ? 0x07060302u : 0x05040100u);
            const bf16x8 af = __builtin_bit_cast(bf16x8, y);
            o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af, bh, o[t], 0, 0, 0);
            if constexpr (SPLIT) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if ((y[n] & 0x7f80u) == 0x7f80u) y[n] &= 0xffff0000u;
                    if ((y[n] & 0x7f800000u) == 0x7f800000u) y[n] &= 0xffffu;
                }
            }
            o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y), bl, o[t], 0, 0, 0);
        }
    }
    // the lane's sums have an infinity or NaN among them (or are large enough to make one)
    __device__ bool odd() const
    {
        f32x4 v = o[0];
#pragma unroll
        for (int t = 1; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += o[t][e];
        return !(fabsf((v[0] + v[1]) + (v[2] + v[3])) < INFINITY);
    }
};

template <int DP, bool PAD> struct Wave<float, DP, PAD> {
    static constexpr int KS = DP / 16;   // 16-byte pieces of a key per lane
    static constexpr int NT = DP / 16;
    static constexpr int VL = DP / 64;
    struct Keys {   // of a step
        f32x4 k[KS];
        f32x4 v[4][VL];
    };
    f32x4 q[KS];
    f32x4 o[NT];

    static __device__ int dim(int t, int i) { return (t / 4) * 64 + 4 * i + t % 4; }

    __device__ void load_q(const char *p, int D, int c, bool on)
    {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (on && (!PAD || (4 * s + c) * 4 < D)) q[s] = *reinterpret_cast<const f32x4 *>(p + (4 * s + c) * 16);
        }
    }
    __device__ static void load_k(Keys &x, const char *base, int row, int D, int i, int c)
    {
        const uint32_t r = __shfl(row, i, 64);
        const char *p = base + (uint64_t)r * (uint32_t)(PAD ? D * 4 : DP * 4) + c * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (PAD) x.k[s] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (!PAD || (4 * s + c) * 4 < D) x.k[s] = *reinterpret_cast<const f32x4 *>(p + s * 64);
        }
    }
    template <bool STREAM> __device__ static void load_v(Keys &x, const char *base, int row, int D, int i, int c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t r = __shfl(row, 4 * c + j, 64);
            const char *p = base + (uint64_t)r * (uint32_t)(PAD ? D * 4 : DP * 4) + i * 16;
#pragma unroll
            for (int m = 0; m < VL; ++m) {
                if (PAD) x.v[j][m] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (!PAD || (16 * m + i) * 4 < D) x.v[j][m] = load_value<STREAM, f32x4>(p + m * 256);
            }
        }
    }
    __device__ void scores(const Keys &x, float (&s)[4])
    {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[t][e], q[t][e], acc, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = acc[r];
    }
    __device__ static void clear_v(Keys &x, uint32_t valid, int c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool on = (valid >> (4 * c + j)) & 1;
#pragma unroll
            for (int m = 0; m < VL; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) x.v[j][m][e] = on ? x.v[j][m][e] : 0.f;
        }
    }
    template <bool> __device__ void add(const Keys &x, const float (&p)[4])
    {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[j][t / 4][t % 4], p[j], o[t], 0, 0, 0);
    }
};

// LDS of a workgroup of NW wavefronts.
template <int DP, int NW> struct Shared {
    float o[NW][16][DP + 4];   // a wavefront's output, unnormalised
    float m[NW][16], l[NW][16];
};

// Dims d and d + 1 of a query head's result from the sums relative to ref, and its lse with dim 0.
template <typename T> __device__ __forceinline__ void write_out(const Args &a, int b, int head, int d, float ref, float L, float O0, float O1)
{
    const float n = L == 0.f ? 1.f : L;
    char *p = a.out + b * a.out_row + head * a.out_head + d * (int)sizeof(T);
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint32_t *>(p) = gemm::cvt_pk_bf16(O0 / n, O1 / n);
    else
        *reinterpret_cast<float2 *>(p) = make_float2(O0 / n, O1 / n);
    if (d == 0 && a.lse) a.lse[(long)b * a.Hq + head] = fmaf(log2f(L), kLn2, ref);
}

// Tiles t0 .. t1 of head h (a block of up to 16 query heads of a key-value head) of row b, whose length is len: the
// wavefronts take turns of kKeys keys and join in LDS.  `whole`: the piece is all of the row, its result goes to out; else
// it goes to slot `slot` of the workspace.
template <typename T, int DP, bool PAD, bool STREAM, int NW>
__device__ __forceinline__ void piece(const Args &a, Shared<DP, NW> &sh, int b, int h, int t0, int t1, int len, bool whole, int slot)
{
    using W = Wave<T, DP, PAD>;
    constexpr int KEYS = kKeys<T>, STEP = KEYS * NW, NS = KEYS / 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, c = lane >> 4;
    const int kvh = a.tiles == 1 ? h : h / a.tiles, first = kvh * a.group + (h - kvh * a.tiles) * 16;   // first query head
    const int nq = min(16, (kvh + 1) * a.group - first);
    const int last = min(t1 * kTile<T>, len);

    W w;
    // page of the lane's key of the step at `at`, -1 where there is none
    const int32_t *pages = a.table + b * a.table_row;
    auto page_of = [&](int at) {
        const int t = at + (lane & (KEYS - 1));
        return t < last ? pages[paged::quotient(a.div, t)] : -1;
    };
    auto row_of = [&](int at, int page) {
        return paged::cache_row(a.div, at + (lane & (KEYS - 1)), page, a.pages, a.Hkv, kvh);
    };
    const int at0 = t0 * kTile<T> + wave * KEYS, page0 = page_of(at0), page1 = page_of(at0 + STEP);
    w.load_q(a.q + b * a.q_row + (first + i) * a.q_head, a.D, c, i < nq);
    float m, l;
    auto walk = [&](auto split, int page, int next) {
        typename W::Keys x;
        int at = at0;
#pragma unroll
        for (int t = 0; t < W::NT; ++t) w.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        l = 0.f;

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

            float s[NS];
            w.scores(x, s);
            if (more) W::load_k(x, a.k, max(row, 0), a.D, i, c);

            // rounded before the maximum is taken off: equal scores of any size stay equal (a fused product would not); to
            // base 2 only then, so that a score counts as long as fp32 holds it and its product
#pragma unroll
            for (int n = 0; n < NS; ++n) s[n] *= a.scale;
            if (valid != paged::all_keys(KEYS)) {
                W::clear_v(x, valid, c);
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    if (!((valid >> ((n >> 2) * 16 + 4 * c + (n & 3))) & 1)) s[n] = -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int n = 1; n < NS; ++n) top = fmaxf(top, s[n]);
            const float m1 = fmaxf(m, xor_max(top));
            const float ref = m1 == -INFINITY ? 0.f : m1;   // nothing but -inf so far: every weight is 0
            if (__any(m1 != m)) {
                const float f = exp_of(m - ref);
                l *= f;
#pragma unroll
                for (int t = 0; t < W::NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w.o[t][e] *= f;
            }
            m = m1;
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                s[n] = exp_of(s[n] - ref);
                l += s[n];
            }
            w.template add<decltype(split)::value>(x, s);
            if (more) W::template load_v<STREAM>(x, a.v, max(row, 0), a.D, i, c);
        }
    };
    walk(std::false_type(), page0, page1);
    if constexpr (sizeof(T) == 2) {   // infinite values among these keys: once more, with what they take in every step
        if (__builtin_expect(__any(i < nq && w.odd()), 0)) walk(std::true_type(), page_of(at0), page_of(at0 + STEP));
    }
    l = xor_sum(l);

    if (c == 0) {
        sh.m[wave][i] = m;
        sh.l[wave][i] = l;
    }
    if (i < nq) {
#pragma unroll
        for (int t = 0; t < W::NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sh.o[wave][i][W::dim(t, 4 * c + r)] = w.o[t][r];
    }
    __syncthreads();
    const int pairs = a.D / 2;
    for (int x = tid; x < nq * pairs; x += 64 * NW) {
        const int j = x / pairs, d = (x - j * pairs) * 2;
        float M = sh.m[0][j];
#pragma unroll
        for (int n = 1; n < NW; ++n) M = fmaxf(M, sh.m[n][j]);
        const float ref = M == -INFINITY ? 0.f : M;
        float L = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
        for (int n = 0; n < NW; ++n) {
            const float f = exp_of(sh.m[n][j] - ref);
            L = fmaf(f, sh.l[n][j], L);
            O0 = fmaf(f, sh.o[n][j][d], O0);
            O1 = fmaf(f, sh.o[n][j][d + 1], O1);
        }
        if (whole) {
            write_out<T>(a, b, first + j, d, ref, L, O0, O1);
        } else {
            const long at = (long)slot * a.part_rows + j;
            a.part_o[at * pairs + d / 2] = make_float2(O0, O1);
            if (d == 0) a.part_ml[at] = make_float2(M, L);
        }
    }
    __syncthreads();
}

// A row's units in equal ranges, a workgroup each: grid (ranges, heads, rows).  One range: all of the row, and nothing is left
// to join.
template <typename T, int DP, bool PAD, bool STREAM, int NW> __global__ __launch_bounds__(64 * NW) void paged_attn_rows_kernel(Args a)
{
    __shared__ Shared<DP, NW> sh;
    const int s = blockIdx.x, S = gridDim.x, h = blockIdx.y;
    for (int b = blockIdx.z; b < a.rows; b += gridDim.z) {
        const int len = length_of(a, b), units = units_of<T>(len);
        const int t0 = S == 1 ? 0 : (int)paged::range_begin(s, units, S), t1 = S == 1 ? units : (int)paged::range_begin(s + 1, units, S);
        if (t0 < t1) piece<T, DP, PAD, STREAM, NW>(a, sh, b, h, t0, t1, len, t0 == 0 && t1 == units, (int)(((unsigned)b * gridDim.y + h) * S + s));
    }
}

// Equal ranges of the units of all rows and heads.
template <typename T, int DP, bool PAD, bool STREAM> __global__ __launch_bounds__(kThreads) void paged_attn_kernel(Args a)
{
    __shared__ Shared<DP, kWaves> sh;
    __shared__ int wsum[kWaves];
    __shared__ struct { int row, len; long rest; } at;   // row of the range's first unit, and units of it before that
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int heads = a.Hkv * a.tiles;

    // units of one head: of the thread's chunk of rows, then before it and of all rows
    const int chunk = (a.rows + kThreads - 1) / kThreads, row0 = min(tid * chunk, a.rows), row1 = min(row0 + chunk, a.rows);
    int own = 0;
    for (int b = row0; b < row1; ++b) own += units_of<T>(length_of(a, b));
    int upto = own;
    for (int m = 1; m < 64; m <<= 1) {
        const int v = __shfl_up(upto, m, 64);
        if (lane >= m) upto += v;
    }
    if (lane == 63) wsum[wave] = upto;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) upto += wsum[w];
        total += wsum[w];
    }
    if (blockIdx.x == 0) {   // for the launch that joins
        int n = upto - own;
        for (int b = row0; b < row1; ++b) {
            a.starts[b] = n;
            n += units_of<T>(length_of(a, b));
        }
        if (tid == 0) a.starts[a.rows] = total;
    }
    const long U = (long)total * heads;
    constexpr int groups = kCUs * resident(DP);
    long u = paged::range_begin(blockIdx.x, U, groups);
    const long end = paged::range_begin(blockIdx.x + 1, U, groups);
    if (u >= end) return;
    if ((long)(upto - own) * heads <= u && u < (long)upto * heads) {   // one thread's chunk has the range's first unit
        long rest = u - (long)(upto - own) * heads;
        int b = row0, len = length_of(a, b);
        for (; b < row1 - 1 && rest >= (long)units_of<T>(len) * heads; len = length_of(a, ++b)) rest -= (long)units_of<T>(len) * heads;
        at = {b, len, rest};
    }
    __syncthreads();
    int b = at.row, len = at.len, units = units_of<T>(len);
    int h = (int)paged::quotient64(at.rest, units), tile = (int)(at.rest - (long)h * units);

    while (u < end) {
        const int stop = (int)(end - u < units - tile ? tile + (end - u) : units);
        piece<T, DP, PAD, STREAM, kWaves>(a, sh, b, h, tile, stop, len, tile == 0 && stop == units, 2 * blockIdx.x + (tile == 0 ? 1 : 0));
        u += stop - tile;
        tile = 0;
        if (stop == units && ++h == heads && u < end) {
            h = 0;
            ++b;
            len = length_of(a, b);
            units = units_of<T>(len);
        }
    }
}

// Joins the pieces of one row's head, grid (heads, rows): every thread takes four dims of one query over a share of the pieces,
// maximum, sum and output at once (one read of memory behind the row's place), and the shares are added in order.  BY_ROW:
// the pieces are those of paged_attn_rows_kernel.
template <typename T, bool BY_ROW> __global__ __launch_bounds__(kJoinThreads) void paged_attn_join_kernel(Args a)
{
    __shared__ f32x4 so[kJoinThreads];
    __shared__ float2 sml[kJoinThreads];
    const int h = blockIdx.x, heads = gridDim.x, tid = threadIdx.x;
    for (int b = blockIdx.y; b < a.rows; b += gridDim.y) {
        const int units = BY_ROW ? units_of<T>(length_of(a, b)) : a.starts[b + 1] - a.starts[b];
        const long U = BY_ROW ? units : (long)a.starts[a.rows] * heads;
        const long u0 = BY_ROW ? 0 : (long)a.starts[b] * heads + (long)h * units;
        const int w0 = paged::owner(u0, U, a.groups), w1 = paged::owner(u0 + units - 1, U, a.groups);
        if (w0 == w1) continue;   // written already
        // pieces lie with consecutive ranges, or with those that have a unit at all
        const bool dense = U >= a.groups;
        const int parts = dense ? w1 - w0 + 1 : units;
        auto slot_of = [&](int p) {
            const int w = dense ? w0 + p : (int)(((uint32_t)(u0 + p + 1) * a.groups - 1) / (uint32_t)U);   // owner, of fewer units
            return BY_ROW ? (b * heads + h) * a.groups + w : 2 * w + (p == 0);
        };
        const int kvh = a.tiles == 1 ? h : h / a.tiles, first = kvh * a.group + (h - kvh * a.tiles) * 16;
        const int nq = min(16, (kvh + 1) * a.group - first);

        const int quads = a.D / 4, all = nq * quads;
        int per = 16;   // threads that share a piece
        while (per < all && per < kJoinThreads) per <<= 1;
        const int shares = kJoinThreads / per, share = tid / per;
        for (int x0 = 0; x0 < all; x0 += per) {
            const int x = x0 + tid % per;
            const bool on = x < all;
            const int j = on ? x / quads : 0, d = on ? x - j * quads : 0;
            float M = -INFINITY, L = 0.f;
            f32x4 O = {0.f, 0.f, 0.f, 0.f};
            auto take = [&](float m, float l, f32x4 o) {
                const float M1 = fmaxf(M, m), ref = M1 == -INFINITY ? 0.f : M1;
                const float f = exp_of(M - ref), g = exp_of(m - ref);
                L = L * f + l * g;
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] = O[e] * f + o[e] * g;
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
                        const long at = (long)slot_of(p0 + n * shares) * a.part_rows + j;
                        ml[n] = a.part_ml[at];
                        o[n] = *reinterpret_cast<const f32x4 *>(a.part_o + at * 2 * quads + 2 * d);
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
                const float ref = M == -INFINITY ? 0.f : M;
                write_out<T>(a, b, first + j, 4 * d, ref, L, O[0], O[1]);
                write_out<T>(a, b, first + j, 4 * d + 2, ref, L, O[2], O[3]);
            }
        }
    }
}

struct Plan {
    int ranges;    // of every row, 0: ranges over all rows
    int slots;     // pieces that the workspace has room for
};

// How the units are cut, from the longest rows that the table allows (the lengths are on the device).  One workgroup takes
// in about 60 bytes per ns, the second launch and the pieces cost 5 us:
//  - a workgroup per row and head where that is at most 256 KB of keys and values, or up to 512 KB with so many rows that
//    they fill the chip (us, one launch / cut; bf16, heads of 128: 2 heads of 512 tokens 8.8 / 8.7, of 1024 12.6 / 9.2; 64 of
//    512 9.7 / 12.7, of 1024 14.3 / 14.6; 160 of 1024 16.6 / 21.9.  Beyond that the two are near each other, the cut
//    behind where all rows are long and ahead where few are: 200 rows of 2048 42 / 50; 800 heads of 64 over 100 to 4000
//    tokens 62 / 52);
//  - every row cut alike where the ranges fill the chip once at most and the longest is short, so that it does not matter whose
//    row is long (28 heads of up to 3001 tokens, fp32: 18.1 us, 20.4 with ranges over all rows, both before full steps went
//    without masks; with longer ranges a ragged batch of 48 rows takes 46 us against 31);
//  - else equal ranges over all rows, which costs the sums over their lengths.
Plan plan(const lory_paged_shape &s)
{
    const int esize = s.dtype == LORY_F32 ? 4 : 2, tile = s.dtype == LORY_F32 ? kTile<float> : kTile<__hip_bfloat16>;
    const int group = s.q_heads / s.kv_heads;
    const long items = (long)s.rows * s.kv_heads * ((group + 15) / 16), most = ((long)s.width * s.page + tile - 1) / tile;
    const long row_bytes = 2 * most * tile * s.head_dim * esize, KB = 1024;
    if (most == 1 || row_bytes <= 256 * KB || row_bytes <= (items < 64 ? items * 8 * KB : 512 * KB)) return {1, 0};
    const long n = items > 0 ? (2 * kCUs / items < most ? 2 * kCUs / items : most) : 1;
    if (n > 1 && row_bytes <= n * 256 * KB) return {(int)n, (int)(n * items)};
    return {0, 2 * kCUs * resident(s.head_dim)};
}

template <typename T, int DP, bool PAD, bool STREAM> void launch4(const Args &a, const Plan &p, hipStream_t st)
{
    const dim3 join(a.Hkv * a.tiles, a.rows < 32768 ? a.rows : 32768);
    Args g = a;
    if (p.ranges) {
        g.groups = p.ranges;
        const long all = (long)a.rows * a.Hkv * a.tiles * p.ranges;
        const dim3 grid(p.ranges, a.Hkv * a.tiles, a.rows < 65535 ? a.rows : 65535);
        bool wide = false;
        if constexpr (DP <= 128) {   // eight wavefronts of the widest heads would spill
            wide = all <= 256;
            if (wide) hipLaunchKernelGGL((paged_attn_rows_kernel<T, DP, PAD, STREAM, 8>), grid, dim3(512), 0, st, g);
        }
        if (!wide) hipLaunchKernelGGL((paged_attn_rows_kernel<T, DP, PAD, STREAM, 4>), grid, dim3(256), 0, st, g);
        if (p.ranges > 1) hipLaunchKernelGGL((paged_attn_join_kernel<T, true>), join, dim3(kJoinThreads), 0, st, g);
        return;
    }
    g.groups = kCUs * resident(DP);
    hipLaunchKernelGGL((paged_attn_kernel<T, DP, PAD, STREAM>), dim3(g.groups), dim3(kThreads), 0, st, g);
    hipLaunchKernelGGL((paged_attn_join_kernel<T, false>), join, dim3(kJoinThreads), 0, st, g);
}

template <typename T, int DP, bool PAD> void launch3(const Args &a, const Plan &p, hipStream_t st)
{
    if (2 * (long)a.pages * a.Hkv * a.page * a.D * (long)sizeof(T) > kStreamBytes)
        launch4<T, DP, PAD, true>(a, p, st);
    else
        launch4<T, DP, PAD, false>(a, p, st);
}

template <typename T, int DP> void launch2(const Args &a, const Plan &p, hipStream_t st)
{
    if (a.D == DP)
        launch3<T, DP, false>(a, p, st);
    else
        launch3<T, DP, true>(a, p, st);
}

template <typename T> void launch1(const Args &a, const Plan &p, hipStream_t st)
{
    if (a.D <= 64)
        launch2<T, 64>(a, p, st);
    else if (a.D <= 128)
        launch2<T, 128>(a, p, st);
    else
        launch2<T, 256>(a, p, st);
}

size_t starts_bytes(const lory_paged_shape &s, const Plan &p)
{
    return p.ranges ? 0 : align_up(((size_t)s.rows + 1) * sizeof(int32_t), 256);
}

// queries of a piece
int part_rows(const lory_paged_shape &s)
{
    const int group = s.q_heads / s.kv_heads;
    return group < 16 ? group : 16;
}

}  // namespace

size_t paged_attn_workspace_bytes(const lory_paged_shape &s)
{
    const Plan p = plan(s);
    const size_t n = starts_bytes(s, p) + (size_t)p.slots * part_rows(s) * (s.head_dim + 2) * sizeof(float);
    return align_up(n > 0 ? n : 1, 256);
}

int paged_attn_launch(const lory_paged_shape &s, const lory_heads &q, const void *k_cache, const void *v_cache,
                      const int32_t *table, const int32_t *lens, const lory_heads &out, float *lse, void *ws, hipStream_t st)
{
    const int esize = s.dtype == LORY_F32 ? 4 : 2;
    Args a = {};
    a.q = (const char *)q.data;
    a.q_row = q.token * esize;
    a.q_head = q.head * esize;
    a.k = (const char *)k_cache;
    a.v = (const char *)v_cache;
    a.table = table;
    a.table_row = s.table_row;
    a.lens = lens;
    a.out = (char *)out.data;
    a.out_row = out.token * esize;
    a.out_head = out.head * esize;
    a.lse = lse;
    const Plan p = plan(s);
    a.starts = (int32_t *)ws;
    a.part_rows = part_rows(s);
    a.part_o = (float2 *)((char *)ws + starts_bytes(s, p));
    a.part_ml = a.part_o + (size_t)p.slots * a.part_rows * (s.head_dim / 2);
    a.rows = s.rows;
    a.Hq = s.q_heads;
    a.Hkv = s.kv_heads;
    a.D = s.head_dim;
    a.pages = s.pages;
    a.page = s.page;
    a.width = s.width;
    a.group = s.q_heads / s.kv_heads;
    a.tiles = (a.group + 15) / 16;
    a.div = paged::divider(s.page);
    a.scale = s.scale;
    prof::Range r(st, prof::kPagedAttn, 0.0, 0.0);   // the lengths are on the device
    if (s.dtype == LORY_F32)
        launch1<float>(a, p, st);
    else
        launch1<__hip_bfloat16>(a, p, st);
    return launch_status();
}

}  // namespace lory
