// Device code shared by the head norm + position rotation (qk_rope.hip) and its gradient (qk_rope_bwd.hip).
//
// A head of D values is D/VEC chunks of 16 bytes; LPH lanes (the power of two from D/VEC on) hold a head, a lane one chunk, so a
// wavefront takes 64/LPH heads of one token with one 16-byte load per lane.  The rotation pairs value i of the first half
// of the turning part with value i of the second: their chunks lie a fixed number of lanes apart and change places by a
// lane permute (neighbouring pairs stay inside a lane).  Written for a lane's value x_e, its partner p_e and the
// turning part's factors,  y_e = x_e c_e + p_e s_e,  where s_e carries the sign of the half; values behind
// the turning part have c = 1, s = 0 and themselves as partner, so no lane branches.
#pragma once

#include "elem_io.h"
#include "gemm_bf16.h"
#include "lory_internal.h"

namespace lory {
namespace rope {

constexpr int kWaves = 4;        // wavefronts of a workgroup
constexpr int kMaxPairs = 128;   // rot_dim / 2 of the widest head

struct Heads {   // strides in bytes
    char *p;
    long token, head;
};

inline Heads heads(const lory_heads &h, int esize) { return {(char *)h.data, h.token * esize, h.head * esize}; }

// The wavefront's number as a scalar, so that what follows from it (token, pointers) takes no vector registers.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// A 16-byte chunk as it lies in memory.
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));

// Results are written past the caches (their readers are other launches, mostly on other XCDs): prompts of 12001 tokens into
// the cache 38.4 -> 28.0 us, 16384 tokens of 32 heads of 128 55.5 -> 52.2.  Loads past them: the gradient's (99 -> 83 us
// there when it came in, 84 -> 80 now; 74 MB of fp32 18.5 -> 19.0) and those of large forward calls.
__device__ __forceinline__ void store_once(char *p, Chunk v) { __builtin_nontemporal_store(v, reinterpret_cast<Chunk *>(p)); }
template <bool STREAM> __device__ __forceinline__ Chunk load(const char *p)
{
    if constexpr (STREAM)
        return __builtin_nontemporal_load(reinterpret_cast<const Chunk *>(p));
    else
        return *reinterpret_cast<const Chunk *>(p);
}

template <typename T> __device__ __forceinline__ void widen(Chunk r, float (&v)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    }
}

template <typename T> __device__ __forceinline__ Chunk narrow(const float (&v)[16 / sizeof(T)])
{
    Chunk r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = gemm::cvt_pk_bf16(v[2 * i], v[2 * i + 1]);
    }
    return r;
}

// cos and sin of pos * freq.  The product is taken to turns and reduced to an eighth of a turn in fp64 (exact to
// |pos| 2^-53 turns), so that fp32 holds the rest to half a step whatever the position; sincospif needs no
// reduction there.
__device__ __forceinline__ float2 turn_of(double pos, double freq)
{
    const double t = pos * (freq * 0.15915494309189533577);   // 1 / (2 pi)
    const double quarter = rint(4.0 * t);
    const float f = (float)(t - 0.25 * quarter);
    float s, c;
    sincospif(2.0f * f, &s, &c);
    const int k = (int)(quarter - 4.0 * floor(0.25 * quarter));   // 0 .. 3
    const float cc = (k & 1) ? s : c, ss = (k & 1) ? c : s;
    return make_float2((k == 1 || k == 2) ? -cc : cc, (k >= 2) ? -ss : ss);
}

// The wavefront's LDS writes are done before its reads that follow; other wavefronts use other parts.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Sum over the LPH lanes of a head, the same bits in each.
template <int LPH> __device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int m = 1; m < LPH; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// What a lane does with its chunk of every head.
struct Lane {
    int chunk, sub;     // chunk of the head, head of the wavefront's group
    int partner;        // chunk it pairs with
    bool on, low;       // the chunk exists; it is in the first half of the turning part
    int turn;           // first pair of the chunk, -1: it does not turn
};

template <typename T, int LPH, bool INTER> __device__ __forceinline__ Lane lane_of(int lane, int D, int rot)
{
    constexpr int VEC = 16 / sizeof(T);
    Lane l;
    l.chunk = lane & (LPH - 1);
    l.sub = lane / LPH;
    l.on = l.chunk * VEC < D;
    l.partner = l.chunk;
    l.low = false;
    l.turn = -1;
    const int first = l.chunk * VEC, half = rot >> 1;
    if (first < rot) {
        if constexpr (INTER) {
            l.turn = first >> 1;
        } else {
            l.low = first < half;
            l.turn = l.low ? first : first - half;
            l.partner = l.low ? l.chunk + half / VEC : l.chunk - half / VEC;
        }
    }
    return l;
}

// Factors of the lane's values from the token's table of (cos, sin); sign -1 turns back.
template <typename T, bool INTER>
__device__ __forceinline__ void factors(const Lane &l, const float2 *table, float sign, float (&c)[16 / sizeof(T)],
                                        float (&s)[16 / sizeof(T)])
{
    constexpr int VEC = 16 / sizeof(T);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const float2 a = l.turn < 0 ? make_float2(1.f, 0.f) : table[INTER ? l.turn + e / 2 : l.turn + e];
        c[e] = a.x;
        s[e] = ((INTER ? (e & 1) == 0 : l.low) ? -sign : sign) * a.y;
    }
}

// The partner's chunk of every lane; 0 for chunks that do not turn (their factor is 0, which an infinity would not stand).
template <typename T, int LPH, bool INTER> __device__ __forceinline__ Chunk exchange(const Lane &l, Chunk r)
{
    if constexpr (INTER) {
        Chunk o;
        if constexpr (sizeof(T) == 4) {
            o[0] = r[1]; o[1] = r[0]; o[2] = r[3]; o[3] = r[2];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbit(r[i], r[i], 16);
        }
        return l.turn < 0 ? Chunk{0, 0, 0, 0} : o;
    } else {
        Chunk o;
        const int from = (l.sub * LPH + l.partner) << 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)r[i]);
        return l.turn < 0 ? Chunk{0, 0, 0, 0} : o;
    }
}

// Weights of the lane's chunk (or of its partner's values); 1 without weights.
template <typename T, bool INTER>
__device__ __forceinline__ void weights(const Lane &l, const T *w, bool partner, float (&v)[16 / sizeof(T)])
{
    constexpr int VEC = 16 / sizeof(T);
    if (w == nullptr || !l.on) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = 1.f;
        return;
    }
    float own[VEC];
    widen<T>(*reinterpret_cast<const Chunk *>(w + (partner ? l.partner : l.chunk) * VEC), own);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = own[INTER && partner ? (e ^ 1) : e];
}

// Lanes a head takes: a template parameter of every kernel here.
template <typename T> int lanes_per_head(int D)
{
    const int chunks = D * (int)sizeof(T) / 16;
    return chunks <= 8 ? 8 : chunks <= 16 ? 16 : chunks <= 32 ? 32 : 64;
}

}  // namespace rope
}  // namespace lory
