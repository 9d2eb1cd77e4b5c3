// The best continuations over beams and vocabulary (lory_beam_select).
//
//   z[b][v] = score[b] + (x[b][v] - log sum_u exp x[b][u]),  the k largest of a request, equal ones by beam and token
//
// Bound by the bytes of the logits, read once; four operations each, one of them an exponential (a quarter of the others' rate).  A request's
// k best are among the k best of each of its beams, and within a beam they are those of the logits themselves, whatever the sum is: so
// a workgroup streams a chunk of one beam's logits, adds its exponentials and keeps its k largest logits, and a second launch forms
// the sums, ranks what the chunks of a request left, and writes.  Sums of a lane (32 terms of bf16, 16 of fp32) are fp32, all others and the
// ranking fp64: candidates of different beams may be as near each other as the sums are accurate.
//
// The k largest of a chunk: of its first part every two lanes' largest logit goes to LDS, and the k-th of these 128 is a bound that at
// least k logits reach and few more.  While the rest goes by, the 16-byte vectors that reach it are only noted in LDS (a hundred of
// them); at the end their logits are looked at, a vector a thread, and ranked by counting.  Where more reach it than there
// is room for (logits in ascending order, thousands of equal ones), those that are noted give a higher bound, and the chunk is
// read once more with a bound that rises as it goes.
// Measured: 48 requests of 8 beams, 128000 bf16 logits each (98 MB): 27.5 + 9.1 us, 3.6 TB/s in the first launch, of which 19 us are a
// workgroup's own (768 of them): 4.2 until its first logits, 1.8 for the bound, 7.4 streaming, 0.7 for its sum, 4.6 for the choice.
// 2^21 fp32 logits in ascending order, read twice: 289 us, in descending order 27; read again for every thousand vectors 1101.  Before: a chunk
// held in registers 47.7 + 24.4; every logit that reaches the bound collected as it goes by 34; candidates of a second level in the second
// launch's bound 51 -> 9.4.  Chunks: 768 workgroups 26.6, 384 37.9, 1152 27.8, 1920 32, 4992 45.  Loads past the caches: no change.
#include <hip/hip_bf16.h>

#include "gemm_bf16.h"
#include "lory_internal.h"

namespace lory {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMost = 4 * kThreads;   // vectors, and logits, of a chunk that LDS holds
constexpr int kFew = 2 * kThreads;    // that are ranked by counting
constexpr int kResident = 1024;       // workgroups that run at a time
constexpr int kChunks = 16;           // of a row at most
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kHead = 4;              // vectors of a thread that give the bound, and of a step

struct Entry {
    float x;
    int32_t token;   // -1: none
};

struct Stat {
    double sum, top;   // sum of exp(x - top)
};

struct Args {
    const char *logits;
    long row;                // bytes
    const float *score;
    int requests, beams, vocab, k;
    int chunks, vectors;     // of a row; 16-byte vectors of a chunk
    Stat *stats;             // workspace: [rows][chunks]
    Entry *entries;          // [rows][chunks][k]
    float *score_out;
    int32_t *token, *parent;
};

// Unsigned numbers in the order of values, and of (value, lower index first).
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);   // -0 is 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }

template <int CONTROL> __device__ __forceinline__ float dpp(float v)
{
    const int x = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(x, x, CONTROL, 0xf, 0xf, false));
}

// Over all lanes, in all of them: neighbours, pairs, halves of eight and sixteen by lane permutes inside the vector unit.
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, dpp<0xb1>(v));
    v = fmaxf(v, dpp<0x4e>(v));
    v = fmaxf(v, dpp<0x141>(v));
    v = fmaxf(v, dpp<0x140>(v));
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

template <typename T> constexpr int kVec = 16 / sizeof(T);   // logits of a vector

template <typename T> __device__ __forceinline__ float element(const gemm::u32x4 &v, int j)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[j]);
    return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
}

// 16 bytes at an address that is a multiple of the type's size.
template <typename T> __device__ __forceinline__ gemm::u32x4 load(const char *p)
{
    typedef uint32_t Vector2 __attribute__((ext_vector_type(4), aligned(2)));
    typedef uint32_t Vector4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef typename std::conditional<sizeof(T) == 2, Vector2, Vector4>::type Vector;
    const Vector v = *reinterpret_cast<const Vector *>(p);
    return gemm::u32x4{v[0], v[1], v[2], v[3]};
}

// Vector v of a row of `vocab` logits: what lies behind the row is -inf.  Vectors start where the row does, at any address: what a lane
// adds, and so a sum's last bits, do not depend on it, and beams with the same logits tie.
template <typename T> __device__ __forceinline__ gemm::u32x4 fetch(const char *row, int v, int end, int vocab)
{
    constexpr int N = kVec<T>;
    constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    if (v >= end) return gemm::u32x4{none, none, none, none};
    const char *p = row + (long)v * 16;
    const int n = vocab - v * N;
    if (n >= N) return load<T>(p);
    uint64_t w[2] = {(uint64_t)none << 32 | none, (uint64_t)none << 32 | none};
    constexpr int bits = 8 * sizeof(T), half = N / 2;
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
        const uint64_t e = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t *>(p + 4 * j) : *reinterpret_cast<const uint16_t *>(p + 2 * j);
        const int at = bits * (j < half ? j : j - half);
        const uint64_t mask = ~(((1ull << bits) - 1) << at);
        if (j < half)
            w[0] = (w[0] & mask) | e << at;
        else
            w[1] = (w[1] & mask) | e << at;
    }
    return gemm::u32x4{(uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32)};
}

__device__ __forceinline__ Entry entry_of(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return Entry{__uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o), (int32_t)~(uint32_t)key};
}

// Largest of a vector's logits that are numbers, and of m.
template <typename T> __device__ __forceinline__ float max_of(const gemm::u32x4 &y, float m)
{
#pragma unroll
    for (int j = 0; j < kVec<T>; j += 2)   // fmaxf would make every operand canonical first
        asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m) : "v"(element<T>(y, j)), "v"(element<T>(y, j + 1)));
    return m;
}

// A wavefront's reference of its exponentials, which are 2^(x log2e - c): relative to c / log2e with the fp32 constant, whatever the rounding of
// c.  Where c would pass fp32 they are formed from x - ref.
struct Ref {
    float ref, c;   // ref: -inf before the first logit
    bool far;
    __device__ void set(float m)
    {
        ref = m;
        far = fabsf(m) > 1e38f && fabsf(m) < INFINITY;
        c = m == -INFINITY ? 0.f : m * kLog2e;
    }
    __device__ double top() const { return ref == -INFINITY ? 0.0 : far ? (double)ref : (double)c / (double)kLog2e; }
};

template <typename T> __global__ __launch_bounds__(kThreads, kResident / 256) void beam_scan_kernel(Args a)
{
    constexpr int N = kVec<T>;
    __shared__ uint64_t keys[kMost], thread_keys[kThreads];
    __shared__ gemm::u32x4 hit_vectors[kMost];
    __shared__ int32_t hits[kMost];
    __shared__ float4 groups[kThreads / 8];
    __shared__ float bound[kWaves];
    __shared__ double sums[kWaves], tops[kWaves];
    __shared__ uint64_t limit;
    __shared__ int noted, found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunk = blockIdx.y;
    const long row = blockIdx.x;
    const char *p = a.logits + row * a.row;
    const int v0 = chunk * a.vectors + tid, end = min((chunk + 1) * a.vectors, (a.vocab + N - 1) / N);

    // whole steps of kHead vectors a thread, and what is left behind them
    constexpr int kStep = kHead * kThreads;
    const int steps = max(0, min(end, a.vocab / N) - (v0 - tid)) / kStep, rest0 = v0 + steps * kStep;
    auto fetch_step = [&](gemm::u32x4 (&y)[kHead], int step) {
#pragma unroll
        for (int i = 0; i < kHead; ++i) y[i] = load<T>(p + (long)(v0 + step * kStep + i * kThreads) * 16);
    };
    gemm::u32x4 rest[kHead], x[kHead], y[kHead];   // x, y: two steps under way, where there is one
    if (steps > 0) {
        fetch_step(x, 0);
        fetch_step(y, min(1, steps - 1));
    }
#pragma unroll
    for (int i = 0; i < kHead; ++i) rest[i] = fetch<T>(p, rest0 + i * kThreads, end, a.vocab);
    if (tid == 0) noted = found = 0;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kHead; ++i) m = max_of<T>(rest[i], m);
    if (steps > 0) {
#pragma unroll
        for (int i = 0; i < kHead; ++i) m = max_of<T>(x[i], m);
    }
    Ref ref;
    ref.set(wave_max(m));
    m = fmaxf(m, dpp<0xb1>(m));
    float *const group = reinterpret_cast<float *>(groups);
    if ((tid & 1) == 0) group[tid >> 1] = m;
    __syncthreads();
    if (tid < kThreads / 2) {   // the largest value that k of them reach
        const float mine = group[tid];
        int reach = 0;
#pragma unroll 8
        for (int i = 0; i < kThreads / 8; ++i) {
            const float4 g = groups[i];
            reach += (g.x >= mine) + (g.y >= mine) + (g.z >= mine) + (g.w >= mine);
        }
        const float w = wave_max(reach >= a.k ? mine : -INFINITY);
        if (lane == 0) bound[wave] = w;
    }
    __syncthreads();
    float least = fmaxf(bound[0], bound[1]);
    int least_at = INT32_MAX;   // of those that equal the bound, tokens up to this one

    // vectors noted with this one, 0: it is not
    auto note = [&](float mx, const gemm::u32x4 &y, int v) {
        if (!(mx >= least && mx > -INFINITY && (mx > least || v * N <= least_at))) return 0;
        const int at = atomicAdd(&noted, 1);
        if (at < kMost) {
            hits[at] = v;
            hit_vectors[at] = y;
        }
        return at + 1;
    };
    // Two questions to a vector, asked as one: does it reach the bound, and has its wavefront's reference to be raised?  The second does not
    // follow from the first: the bound is the workgroup's, the reference the wavefront's own, which may have seen nothing but barred tokens.
    float gate = fminf(least, ref.ref + 64.f);
    double sum = 0.0;
    auto take = [&](const gemm::u32x4 (&x)[kHead], int v) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kHead; ++i) {
            const float mx = max_of<T>(x[i], -INFINITY);
            if (__any(mx >= gate && mx > -INFINITY)) {
                if (__any(mx > ref.ref + 64.f)) {   // a wavefront's sum stays far inside fp32
                    const double old = ref.top();
                    const bool none = ref.ref == -INFINITY;   // so far 0, or NaN where a logit was that: it stays
                    ref.set(wave_max(mx));
                    gate = fminf(least, ref.ref + 64.f);
                    sum = none ? sum + s : (sum + s) * exp(old - ref.top());
                    s = 0.f;
                }
                note(mx, x[i], v + i * kThreads);
            }
            if (__builtin_expect(ref.far, 0)) {
#pragma unroll 1
                for (int j = 0; j < N; ++j) {
                    const uint32_t w = j * (int)sizeof(T) < 8 ? (j * (int)sizeof(T) < 4 ? x[i][0] : x[i][1]) : (j * (int)sizeof(T) < 12 ? x[i][2] : x[i][3]);
                    const float e = __uint_as_float(sizeof(T) == 4 ? w : j & 1 ? w & 0xffff0000u : w << 16);
                    s += __builtin_amdgcn_exp2f((e - ref.ref) * kLog2e);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f(fmaf(element<T>(x[i], j), kLog2e, -ref.c));
            }
        }
        sum += s;
    };
    take(rest, rest0);
    if (steps > 0) {   // behind the last step it is read again, so that no load hangs on a condition
        for (int i = 0; i < steps; i += 2) {
            take(x, v0 + i * kStep);
            fetch_step(x, min(i + 2, steps - 1));
            if (i + 1 == steps) break;
            take(y, v0 + (i + 1) * kStep);
            fetch_step(y, min(i + 3, steps - 1));
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) {
        tops[wave] = ref.top();
        sums[wave] = sum;
    }
    __syncthreads();

    // the thread whose key is the k-th largest of the threads' says the next bound; every thread has one, and no two the same
    auto raise = [&](uint64_t best) {
        thread_keys[tid] = best;
        __syncthreads();
        int rank = 0;
        for (int i = 0; i < kThreads; ++i) rank += thread_keys[i] > best;
        if (rank == a.k - 1) limit = best;
        if (tid == 0) noted = found = 0;
        __syncthreads();
        const Entry e = entry_of(limit);
        least = e.x;
        least_at = e.token;
    };
    int n = noted;
    if (__builtin_expect(n > kMost, 0)) {
        // More reach the bound than there is room for.  Those that are noted give a higher one, and the chunk is read once more, a vector a
        // thread at a time; before there is no room for another of each thread, the bound is raised to what the k threads with the largest
        // noted logits reach, and only their vectors stay, 4 k <= kThreads.
        bool again = false;
        int v = v0;
        for (int all = kMost; all > 0;) {   // kThreads at least: every thread has one
            uint64_t best = 0;
#pragma unroll 1
            for (int i = tid; i < all; i += kThreads) {
                const gemm::u32x4 y = hit_vectors[i];
                const int token = hits[i] * N;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const uint64_t key = key_of(element<T>(y, j), token + j);
                    if (element<T>(y, j) > -INFINITY && key > best) best = key;
                }
            }
            raise(best);
#pragma unroll 1
            for (int i = tid; again && i - tid < all; i += kThreads) {   // none is written before it is read
                const int at = i < all ? hits[i] : -1;
                const gemm::u32x4 y = hit_vectors[i];
                __syncthreads();
                if (at >= 0) note(max_of<T>(y, -INFINITY), y, at);
            }
            __syncthreads();
            again = true;
            all = 0;
            for (; v - tid < end && all == 0; v += kThreads) {
                const gemm::u32x4 y = fetch<T>(p, v, end, a.vocab);
                if (__syncthreads_or(note(max_of<T>(y, -INFINITY), y, v) > kMost - kThreads)) all = noted;
            }
        }
        n = noted;
    }
    const int vectors = n;
    auto collect = [&]() {
        for (int i = tid; i < vectors; i += kThreads) {
            const gemm::u32x4 y = hit_vectors[i];
            const int token = hits[i] * N;
            uint32_t some = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float e = element<T>(y, j);
                some |= (uint32_t)((e > least) | ((e == least) & (e > -INFINITY) & (token + j <= least_at))) << j;
            }
            int at = atomicAdd(&found, __popc(some));
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (some >> j & 1) {
                    if (at < kMost) keys[at] = key_of(element<T>(y, j), token + j);
                    ++at;
                }
        }
    };
    collect();
    __syncthreads();
    n = found;
    while (n > kFew) {
        uint64_t mine[kMost / kThreads], best = 0;
#pragma unroll
        for (int i = 0; i < kMost / kThreads; ++i) {
            mine[i] = i * kThreads + tid < n ? keys[i * kThreads + tid] : 0;
            best = mine[i] > best ? mine[i] : best;
        }
        raise(best);
        if (n <= kMost) {
            const uint64_t lim = limit;
#pragma unroll
            for (int i = 0; i < kMost / kThreads; ++i)
                if (mine[i] >= lim) keys[atomicAdd(&found, 1)] = mine[i];   // at most k threads' keys
        } else {
            collect();
        }
        __syncthreads();
        n = found;
    }
    Entry *out = a.entries + (row * a.chunks + chunk) * a.k;
    for (int e = tid; e < n; e += kThreads) {
        const uint64_t mine = keys[e];
        int rank = 0;
#pragma unroll 8
        for (int i = 0; i < n; ++i) rank += keys[i] > mine;
        if (rank < a.k) out[rank] = entry_of(mine);
    }
    for (int e = n + tid; e < a.k; e += kThreads) out[e] = Entry{-INFINITY, -1};
    if (wave == 0) {   // the chunk's sum from its wavefronts'; one without a logit has the sum 0
        const double sw = lane < kWaves ? sums[lane] : 0.0, tw = lane < kWaves && sw != 0.0 ? tops[lane] : -(double)INFINITY;
        double R = tw;
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) R = fmax(R, __shfl_xor(R, o, 64));
        double S = sw != 0.0 ? sw * exp(tw - R) : 0.0;
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) S += __shfl_xor(S, o, 64);
        if (lane == 0) a.stats[row * a.chunks + chunk] = Stat{S, R};
    }
}

// One request: a list of k candidates from every chunk of every beam, each sorted; THREADS >= lists.
template <int THREADS> __global__ __launch_bounds__(THREADS) void beam_join_kernel(Args a)
{
    constexpr int kCap = 4096, kAhead = 4;
    __shared__ double z[kCap];
    __shared__ uint64_t tie[kCap];
    __shared__ int32_t tokens[kCap];
    __shared__ double tops[THREADS], term[THREADS], lse[64], add[64], level[2 * THREADS], bounds[THREADS / 64];
    __shared__ uint64_t least_tie;
    __shared__ int found, places[64];
    const int tid = threadIdx.x, lane = tid & 63, r = blockIdx.x, lists = a.beams * a.chunks, k = a.k, all = lists * k;
    const long row0 = (long)r * a.beams;
    const Entry *entries = a.entries + row0 * a.chunks * k;
    const bool on = tid < lists;
    // Level s: entry 2^s - 1 of every list.  Where k / 2^s of them reach a value, k candidates do.
    int levels = 1;
    while ((1 << (levels - 1)) < k && (levels + 1) * lists <= 2 * THREADS) ++levels;
    auto level_entry = [&](int x) {
        const int s = x / lists;
        return entries[(x - s * lists) * k + min(1 << s, k) - 1];
    };
    // all loads under way at once
    Entry ahead[kAhead], first[2];
    int ahead_beam[kAhead], first_beam[2];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = tid + i * THREADS < all ? entries[tid + i * THREADS] : Entry{-INFINITY, -1};
#pragma unroll
    for (int i = 0; i < 2; ++i) first[i] = tid + i * THREADS < levels * lists ? level_entry(tid + i * THREADS) : Entry{-INFINITY, -1};
    const Stat st = on ? a.stats[row0 * a.chunks + tid] : Stat{0.0, -(double)INFINITY};
    const float score = tid < a.beams ? a.score[row0 + tid] : 0.f;
    const int beam = on ? tid / a.chunks : 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead_beam[i] = min((tid + i * THREADS) / k / a.chunks, a.beams - 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) first_beam[i] = (tid + i * THREADS) % lists / a.chunks;
    if (tid < a.beams) add[tid] = score;
    tops[tid] = st.top;
    if (tid < 64) places[tid] = 0;
    if (tid == 0) found = 0;
    __syncthreads();
    double R = -INFINITY;
    if (on)
        for (int c = 0; c < a.chunks; ++c) R = fmax(R, tops[beam * a.chunks + c]);
    term[tid] = st.sum != 0.0 ? st.sum * exp(st.top - R) : 0.0;
    __syncthreads();
    if (on && tid == beam * a.chunks) {
        double S = 0.0;
        for (int c = 0; c < a.chunks; ++c) S += term[tid + c];
        lse[beam] = R + log(S);       // -inf or NaN for a beam without a distribution: its candidates become NaN
    }
    __syncthreads();
    auto value = [&](const Entry &e, int b) {   // -inf: none
        const double v = ((double)e.x - lse[b]) + add[b];
        return e.token >= 0 && v > -INFINITY ? v : -(double)INFINITY;
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) level[tid + i * THREADS] = value(first[i], first_beam[i]);
    __syncthreads();
    double l = -INFINITY;   // a value that k candidates reach
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int x = tid + i * THREADS;
        if (x >= levels * lists) continue;
        const int s = x / lists;
        const double v = level[x];
        int reach = 0;
#pragma unroll 8
        for (int j = 0; j < lists; ++j) reach += level[s * lists + j] >= v;
        if (reach << s >= k) l = fmax(l, v);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l = fmax(l, __shfl_xor(l, o, 64));
    if (lane == 0) bounds[tid >> 6] = l;
    __syncthreads();
    l = bounds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) l = fmax(l, bounds[w]);

    // Order of equal values, the least first: by beam, in a beam by logit (a far score makes different ones equal), then by place,
    // list * k + rank in the list, of 16 bits.
    auto tie_of = [&](float x, int b, int at) { return (uint64_t)b << 48 | (uint64_t)~order_of(x) << 16 | (uint32_t)at; };
    uint64_t lt = ~0ull;
    auto take = [&](const Entry &e, int b, int i) {
        const double v = value(e, b);
        if (!(v > -INFINITY && v >= l)) return;
        const uint64_t t = tie_of(e.x, b, i);
        if (v == l && t > lt) return;
        const int n = atomicAdd(&found, 1);
        if (n < kCap) {
            z[n] = v;
            tie[n] = t;
            tokens[n] = e.token;
        }
    };
    auto take_all = [&]() {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (tid + i * THREADS < all) take(ahead[i], ahead_beam[i], tid + i * THREADS);
        for (int i = tid + kAhead * THREADS; i < all; i += THREADS) take(entries[i], i / k / a.chunks, i);
    };
    take_all();
    __syncthreads();
    int n = found;
    if (n > kCap) {   // thousands of equal candidates: k lists or more.  What k lists' first entries come before is left out: k k remain
        const double v = on ? level[tid] : 0.0;
        const uint64_t t = on ? tie_of(first[0].x, beam, tid * k) : 0;
        term[tid] = __longlong_as_double((long long)t);   // only kept there
        __syncthreads();
        int rank = 0;
        if (on)
            for (int i = 0; i < lists; ++i) rank += level[i] > v || (level[i] == v && (uint64_t)__double_as_longlong(term[i]) < t);
        if (on && rank == k - 1) {
            bounds[0] = v;
            least_tie = t;
        }
        if (tid == 0) found = 0;
        __syncthreads();
        l = bounds[0];
        lt = least_tie;
        take_all();
        __syncthreads();
        n = found;
    }
    auto write = [&](int e, int rank) {
        const long o = (long)r * k + rank;
        a.score_out[o] = (float)z[e];
        a.token[o] = tokens[e];
        a.parent[o] = (int32_t)(row0 + (int)(tie[e] >> 48));
    };
    // ranks by value; where two are equal the order of their ties is looked at, for all
    int ranks = k;
    bool twice = n > THREADS;
    if (!twice && tid < n) {
        const double v = z[tid];
        ranks = 0;
#pragma unroll 8
        for (int i = 0; i < n; ++i) ranks += z[i] > v;
        if (ranks < k) twice = atomicAdd(places + ranks, 1) > 0;
    }
    if (!__syncthreads_or(twice)) {
        if (ranks < k) write(tid, ranks);
    } else {
        for (int e = tid; e < n; e += THREADS) {
            const double v = z[e];
            const uint64_t t = tie[e];
            int rank = 0;
            for (int i = 0; i < n; ++i) rank += z[i] > v || (z[i] == v && tie[i] < t);
            if (rank < k) write(e, rank);
        }
    }
    for (int e = n + tid; e < k; e += THREADS) {
        const long o = (long)r * k + e;
        a.score_out[o] = -INFINITY;
        a.token[o] = a.parent[o] = -1;
    }
}

// Chunks of a row, and 16-byte vectors of a chunk: as many workgroups as run at a time (four a CU) where the rows alone are fewer,
// of one vector a thread at least.
struct Plan {
    int chunks, vectors;
};

Plan plan(const lory_beam_shape &s)
{
    const int n = s.dtype == LORY_F32 ? 4 : 8;
    const long rows = (long)s.requests * s.beams, vectors = ((long)s.vocab + n - 1) / n;
    long want = rows > 0 ? kResident / rows : 1;
    const long most = (vectors + kThreads - 1) / kThreads;
    if (want > most) want = most;
    if (want > kChunks) want = kChunks;
    if (want < 1) want = 1;
    return {(int)want, (int)((vectors + want - 1) / want)};
}

template <typename T> void launch(const Args &a, long rows, hipStream_t st)
{
    hipLaunchKernelGGL((beam_scan_kernel<T>), dim3((unsigned)rows, a.chunks), dim3(kThreads), 0, st, a);
    if (a.beams * a.chunks <= 256)
        hipLaunchKernelGGL((beam_join_kernel<256>), dim3(a.requests), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((beam_join_kernel<1024>), dim3(a.requests), dim3(1024), 0, st, a);
}

size_t stats_bytes(const lory_beam_shape &s, const Plan &p)
{
    return align_up((size_t)s.requests * s.beams * p.chunks * sizeof(Stat), 256);
}

}  // namespace

size_t beam_select_workspace_bytes(const lory_beam_shape &s)
{
    const Plan p = plan(s);
    return stats_bytes(s, p) + align_up((size_t)s.requests * s.beams * p.chunks * s.k * sizeof(Entry), 256);
}

int beam_select_launch(const lory_beam_shape &s, const void *logits, const float *score, float *score_out, int32_t *token,
                       int32_t *parent, void *ws, hipStream_t st)
{
    const Plan p = plan(s);
    const int esize = s.dtype == LORY_F32 ? 4 : 2;
    const long rows = (long)s.requests * s.beams;
    Args a = {(const char *)logits, (long)s.row * esize, score, s.requests, s.beams, s.vocab, s.k, p.chunks, p.vectors,
              (Stat *)ws, (Entry *)((char *)ws + stats_bytes(s, p)), score_out, token, parent};
    prof::Range r(st, prof::kBeamSelect, 4.0 * rows * s.vocab, (double)rows * s.vocab * esize);
    if (s.dtype == LORY_F32)
        launch<float>(a, rows, st);
    else
        launch<__hip_bfloat16>(a, rows, st);
    return launch_status();
}

}  // namespace lory
