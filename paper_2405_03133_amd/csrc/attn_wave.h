// A wavefront's part of attention over a paged key-value cache: operands straight from memory to the matrix cores, for NQ blocks of
// 16 queries.  What a step of keys does with them stands in paged_attn.hip.
#pragma once

#include <hip/hip_bf16.h>

#include <type_traits>

#include "gemm_bf16.h"

namespace lory {
namespace attn {

using gemm::bf16x8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4, kJoinThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <bool STREAM, typename V> __device__ __forceinline__ V load_value(const char *p)
{
    if constexpr (STREAM)
        return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
    else
        return *reinterpret_cast<const V *>(p);
}

template <typename T> constexpr int kKeys = sizeof(T) == 2 ? 32 : 16;   // of a wavefront's step
template <typename T> constexpr int kTile = kKeys<T> * kWaves;

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

// One key-value head for one wavefront: operands of keys, values and queries (16 of them), and the outputs.
// DP: head_dim rounded up to 64, 128 or 256.  PAD: head_dim < DP (pieces behind it are zeros that nothing loads).
template <typename T, int DP, bool PAD, int NQ = 1> struct Wave;

template <int DP, bool PAD, int NQ> struct Wave<__hip_bfloat16, DP, PAD, NQ> {
    static constexpr int KS = DP / 32;     // K steps of a product over the dims
    static constexpr int NT = DP / 16;     // output tiles
    static constexpr int VW = NT < 8 ? NT : 8;   // dims of a V load
    static constexpr int VL = NT / VW;     // V loads of a key
    struct Keys {   // of a step
        u32x4 k[2][KS];
        uint32_t v[8][VL][VW / 2];
    };
    typedef bf16x8 Query[KS];
    Query q[NQ];
    f32x4 o[NQ][NT];

    // dim of row i of output tile t
    static __device__ int dim(int t, int i) { return (t / VW) * 16 * VW + VW * i + t % VW; }

    __device__ static void load_q(Query &q, const char *p, int D, int c, bool on)
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
    __device__ static void scores(const bf16x8 (&q)[KS], const Keys &x, float (&s)[8])
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
    template <bool SPLIT> __device__ void add(const Keys &x, const float (&p)[NQ][8])
    {
        bf16x8 bh[NQ], bl[NQ];
#pragma unroll
        for (int b = 0; b < NQ; ++b) {
            u32x4 hi, lo;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                hi[n] = gemm::cvt_pk_bf16(p[b][2 * n], p[b][2 * n + 1]);
                lo[n] = gemm::cvt_pk_bf16(p[b][2 * n] - __uint_as_float(hi[n] << 16),
                                          p[b][2 * n + 1] - __uint_as_float(hi[n] & 0xffff0000u));
            }
            bh[b] = __builtin_bit_cast(bf16x8, hi);
            bl[b] = __builtin_bit_cast(bf16x8, lo);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4 y;
#pragma unroll
            for (int n = 0; n < 4; ++n)
                y[n] = __builtin_amdgcn_perm(x.v[2 * n + 1][t / VW][(t % VW) / 2], x.v[2 * n][t / VW][(t % VW) / 2],
                                             (t & 1) ? 0x07060302u : 0x05040100u);
            const bf16x8 af = __builtin_bit_cast(bf16x8, y);
#pragma unroll
            for (int b = 0; b < NQ; ++b) o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af, bh[b], o[b][t], 0, 0, 0);
            if constexpr (SPLIT) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if ((y[n] & 0x7f80u) == 0x7f80u) y[n] &= 0xffff0000u;
                    if ((y[n] & 0x7f800000u) == 0x7f800000u) y[n] &= 0xffffu;
                }
            }
            const bf16x8 al = __builtin_bit_cast(bf16x8, y);
#pragma unroll
            for (int b = 0; b < NQ; ++b) o[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(al, bl[b], o[b][t], 0, 0, 0);
        }
    }
    // the lane's sums have an infinity or NaN among them (or are large enough to make one)
    __device__ bool odd(int b) const
    {
        f32x4 v = o[b][0];
#pragma unroll
        for (int t = 1; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += o[b][t][e];
        return !(fabsf((v[0] + v[1]) + (v[2] + v[3])) < INFINITY);
    }
};

template <int DP, bool PAD, int NQ> struct Wave<float, DP, PAD, NQ> {
    static constexpr int KS = DP / 16;   // 16-byte pieces of a key per lane
    static constexpr int NT = DP / 16;
    static constexpr int VL = DP / 64;
    struct Keys {   // of a step
        f32x4 k[KS];
        f32x4 v[4][VL];
    };
    typedef f32x4 Query[KS];
    Query q[NQ];
    f32x4 o[NQ][NT];

    static __device__ int dim(int t, int i) { return (t / 4) * 64 + 4 * i + t % 4; }

    __device__ static void load_q(Query &q, const char *p, int D, int c, bool on)
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
    __device__ static void scores(const f32x4 (&q)[KS], const Keys &x, float (&s)[4])
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
    template <bool> __device__ void add(const Keys &x, const float (&p)[NQ][4])
    {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int b = 0; b < NQ; ++b)
                    o[b][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[j][t / 4][t % 4], p[b][j], o[b][t], 0, 0, 0);
    }
};

}  // namespace attn
}  // namespace lory
