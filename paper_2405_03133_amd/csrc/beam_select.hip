// The best continuations over beams and vocabulary (lory_beam_select).
//
//   z[b][v] = score[b] + (x[b][v] - log sum_u exp x[b][u]),  the k largest of a request, equal ones by beam and token
//
// Bound by the bytes of the logits, read once; four operations each, one of them an exponential.  A request's k best are among the k best
// of each of its beams, and within a beam they are those of the logits themselves, whatever the sum is: so a workgroup takes a
// chunk of one beam's logits into registers, adds its exponentials and finds its k largest logits, and a second launch forms the
// sums, ranks what the chunks of a request left, and writes.  Sums of a lane (64 terms at most) are fp32, all others and
// the ranking fp64: candidates of different beams may be as near each other as the sums are accurate.
//
// The k largest of a chunk: every wavefront takes its lanes' largest values off one after the other until it has had k / 8
// of them; the smallest of the eight last ones is a bound that at least k logits of the chunk reach, and that few others do.  Those
// that reach it go to LDS and are ranked by counting.  A chunk in which more reach it than LDS holds (thousands of equal logits)
// takes its largest off one by one instead.
#include <hip/hip_bf16.h>

#include "gemm_bf16.h"
#include "lory_internal.h"

namespace lory {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kMost = 2048;           // logits of a chunk that LDS holds
constexpr int kPer = 64;              // logits of a thread at most: chunks of up to 32768
constexpr int kChunks = 16;           // of a row at most

struct Entry {
    float x;
    int32_t token;   // -1: none
};

struct Stat {
    double sum;      // of exp(x - top)
    float top, pad;
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

// Unsigned keys in the order of (value, lower index first).
__device__ __forceinline__ uint64_t key_of(float x, int index)
{
    const uint32_t u = __float_as_uint(x + 0.f);   // -0 is 0
    const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (uint64_t)o << 32 | (uint32_t)~index;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
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

// VPT: vectors of a thread
template <typename T, int VPT> __global__ __launch_bounds__(kThreads) void beam_scan_kernel(Args a)
{
    constexpr int N = kVec<T>;
    __shared__ uint64_t keys[kMost];
    __shared__ float bound[kWaves], top[kWaves];
    __shared__ double sums[kWaves];
    __shared__ uint64_t best[kWaves];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunk = blockIdx.y;
    const long row = blockIdx.x;
    const char *p = a.logits + row * a.row;
    const int v0 = chunk * a.vectors, v1 = min(v0 + a.vectors, (a.vocab + N - 1) / N);
    if (tid == 0) found = 0;

    // Vectors start where the row does, at any address: what a lane adds, and so a sum's last bits, do not depend on it, and
    // beams with the same logits tie.
    gemm::u32x4 x[VPT];
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;   // -inf
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = v0 + i * kThreads + tid, t = v * N;
        x[i] = gemm::u32x4{kNone, kNone, kNone, kNone};
        if (v < v1) {
            if (t + N <= a.vocab) {
                x[i] = load<T>(p + (long)v * 16);
            } else {   // the row ends inside the vector
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (t + j >= a.vocab) continue;
                    if constexpr (sizeof(T) == 4) {
                        x[i][j] = *reinterpret_cast<const uint32_t *>(p + (long)v * 16 + 4 * j);
                    } else {
                        const uint32_t h = *reinterpret_cast<const uint16_t *>(p + (long)v * 16 + 2 * j);
                        x[i][j >> 1] = j & 1 ? (x[i][j >> 1] & 0xffffu) | h << 16 : (x[i][j >> 1] & 0xffff0000u) | h;
                    }
                }
            }
        }
    }

    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, element<T>(x[i], j));
    const float wm = wave_max(m), ref = wm == -INFINITY ? 0.f : wm;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f((element<T>(x[i], j) - ref) * 1.4426950408889634f);
    double sum = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);

    // the wavefront's value that `each` of its lanes reach
    const int each = (a.k + kWaves - 1) / kWaves;
    float mine = m, last = wm;
    for (int n = 1; n < each; ++n) {
        const uint64_t at = __ballot(mine == last);
        if (at && lane == __ffsll((unsigned long long)at) - 1) mine = -INFINITY;
        last = wave_max(mine);
    }
    if (lane == 0) {
        top[wave] = ref;
        sums[wave] = sum;
        bound[wave] = last;
    }
    __syncthreads();
    float least = bound[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) least = fminf(least, bound[w]);

    // what reaches the bound
    if (m >= least && m > -INFINITY) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float e = element<T>(x[i], j);
                if (e >= least && e > -INFINITY) {
                    const int at = atomicAdd(&found, 1);
                    if (at < kMost) keys[at] = key_of(e, (v0 + i * kThreads + tid) * N + j);
                }
            }
    }
    __syncthreads();
    const int n = found;
    Entry *out = a.entries + (row * a.chunks + chunk) * a.k;
    auto entry = [&](uint64_t key) {
        const uint32_t o = (uint32_t)(key >> 32);
        return Entry{__uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o), (int32_t)~(uint32_t)key};
    };
    if (n <= kMost) {
        for (int e = tid; e < n; e += kThreads) {
            const uint64_t mine_key = keys[e];
            int rank = 0;
            for (int i = 0; i < n; ++i) rank += keys[i] > mine_key;
            if (rank < a.k) out[rank] = entry(mine_key);
        }
        for (int e = n + tid; e < a.k; e += kThreads) out[e] = Entry{-INFINITY, -1};
    } else {
        uint64_t prev = ~0ull;   // more than any key
        for (int r = 0; r < a.k; ++r) {
            uint64_t b = 0;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float e = element<T>(x[i], j);
                    const uint64_t key = key_of(e, (v0 + i * kThreads + tid) * N + j);
                    if (e > -INFINITY && key < prev && key > b) b = key;
                }
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint64_t y = __shfl_xor((unsigned long long)b, o, 64);
                if (y > b) b = y;
            }
            if (lane == 0) best[wave] = b;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                if (best[w] > b) b = best[w];
            if (tid == 0) out[r] = entry(b);   // more than kMost >= k logits are there
            prev = b;
            __syncthreads();
        }
    }
    if (wave == 0) {   // the chunk's sum from its wavefronts'; one without a logit has the sum 0
        const double sw = lane < kWaves ? sums[lane] : 0.0;
        const float tw = lane < kWaves && sw != 0.0 ? top[lane] : -INFINITY, R = wave_max(tw);
        double S = sw != 0.0 ? sw * exp((double)tw - (double)R) : 0.0;
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) S += __shfl_xor(S, o, 64);
        if (lane == 0) a.stats[row * a.chunks + chunk] = Stat{S, R, 0.f};
    }
}

// One request: a list of k candidates from every chunk of every beam, each sorted; THREADS >= lists.
template <int THREADS> __global__ __launch_bounds__(THREADS) void beam_join_kernel(Args a)
{
    constexpr int kCap = 4096;
    __shared__ double z[kCap];
    __shared__ int32_t place[kCap];          // of a candidate: list * k + its rank there
    __shared__ double lse[64], add[64];
    __shared__ double heads[THREADS];
    __shared__ double least;
    __shared__ int least_at, found;
    const int tid = threadIdx.x, r = blockIdx.x, lists = a.beams * a.chunks, k = a.k;
    const long row0 = (long)r * a.beams;
    if (tid < a.beams) {
        const Stat *st = a.stats + (row0 + tid) * a.chunks;
        float R = -INFINITY;
        for (int c = 0; c < a.chunks; ++c) R = fmaxf(R, st[c].top);
        double S = 0.0;
        for (int c = 0; c < a.chunks; ++c)
            if (st[c].sum != 0.0) S += st[c].sum * exp((double)st[c].top - (double)R);
        lse[tid] = (double)R + log(S);       // -inf or NaN for a beam without a distribution: its candidates become NaN
        add[tid] = a.score[row0 + tid];
    }
    if (tid == 0) {
        found = 0;
        least = -INFINITY;
        least_at = INT32_MAX;
    }
    __syncthreads();
    const Entry *list = a.entries + (row0 * a.chunks + tid) * k;
    const int beam = tid / a.chunks;
    auto value = [&](int i) {   // -inf: none
        const Entry e = list[i];
        const double v = ((double)e.x - lse[beam]) + add[beam];
        return e.token >= 0 && v > -INFINITY ? v : -(double)INFINITY;
    };
    const bool on = tid < lists;
    // a bound that k candidates reach: with k lists or more the k-th of their first entries, else the least of the lists'
    // entries at a depth that makes k together
    const bool many = lists >= k;
    const double head = on ? value(many ? 0 : (k + lists - 1) / lists - 1) : -(double)INFINITY;
    heads[tid] = head;
    __syncthreads();
    if (on) {
        int rank = 0;
        for (int i = 0; i < lists; ++i) rank += heads[i] > head || (heads[i] == head && i < tid);
        if (rank == (many ? k : lists) - 1) {
            least = head;
            least_at = many ? tid : INT32_MAX;
        }
    }
    __syncthreads();
    if (on) {
        const double l = least;
        const int at = least_at;
        for (int i = 0; i < k; ++i) {
            const double v = value(i);
            if (!(v > -INFINITY) || v < l || (v == l && tid > at)) break;
            const int n = atomicAdd(&found, 1);
            z[n] = v;
            place[n] = tid * k + i;
        }
    }
    __syncthreads();
    const int n = found;
    for (int e = tid; e < n; e += THREADS) {
        const double v = z[e];
        const int at = place[e];
        int rank = 0;
        for (int i = 0; i < n; ++i) rank += z[i] > v || (z[i] == v && place[i] < at);
        if (rank < k) {
            const int l = at / k;
            const long o = (long)r * k + rank;
            a.score_out[o] = (float)v;
            a.token[o] = a.entries[(row0 * a.chunks + l) * k + (at - l * k)].token;
            a.parent[o] = (int32_t)(row0 + l / a.chunks);
        }
    }
    for (int e = n + tid; e < k; e += THREADS) {
        const long o = (long)r * k + e;
        a.score_out[o] = -INFINITY;
        a.token[o] = a.parent[o] = -1;
    }
}

// Chunks of a row, and 16-byte vectors of a chunk: as many workgroups as run at a time (two a CU) where the rows alone are fewer,
// chunks of eight thousand logits at least, and of what a workgroup's registers hold at most.
struct Plan {
    int chunks, vectors;
};

Plan plan(const lory_beam_shape &s)
{
    const int n = s.dtype == LORY_F32 ? 4 : 8;
    const long rows = (long)s.requests * s.beams, vectors = ((long)s.vocab + n - 1) / n;
    const long need = (vectors * n + (long)kThreads * kPer - 1) / ((long)kThreads * kPer);
    long want = rows > 0 ? (512 + rows - 1) / rows : 1;
    const long most = (s.vocab + 8191) / 8192;
    if (want > most) want = most;
    if (want < need) want = need;
    if (want > kChunks) want = kChunks;
    return {(int)want, (int)((vectors + want - 1) / want)};
}

template <typename T> void launch(const Args &a, long rows, hipStream_t st)
{
    constexpr int F = sizeof(T) == 4 ? 2 : 1;
    const dim3 grid((unsigned)rows, a.chunks);
    const int per = (a.vectors + kThreads - 1) / kThreads;   // vectors of a thread
    if (per <= 2 * F)
        hipLaunchKernelGGL((beam_scan_kernel<T, 2 * F>), grid, dim3(kThreads), 0, st, a);
    else if (per <= 4 * F)
        hipLaunchKernelGGL((beam_scan_kernel<T, 4 * F>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((beam_scan_kernel<T, 8 * F>), grid, dim3(kThreads), 0, st, a);
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
