// Norm of the query and key heads and the position rotation, with the keys into their own tensor or, with the values
// beside them, into a paged cache (lory_qk_rope, lory_qk_rope_cache).
//
// HBM-bound: every head is read and written once, 9 flops a value.  A wavefront takes one token (all its heads where there
// are enough tokens to fill the chip, a share of them otherwise), so the token's angles are formed once, one pair
// per lane, and stay in registers as the factors of the lane's values, with the norm's weights multiplied in:
//   y_e = r (x_e (w_e c_e) + p_e (w'_e s_e)),   r = 1 / sqrt(mean + eps).
// Four groups of heads are loaded at a time; two or eight were slower (16384 tokens of 32 heads of 128, bf16: 55.4 and 54.9 us
// against 52.1), and so was loading queries, keys and values before the angles are formed (57.4: the registers for it cost two
// of six wavefronts per SIMD).
// Measured: those 16384 tokens 48.5 us, 5.5 TB/s; prompts of 12001 tokens (16 + 4 heads) into the cache 25.8 us, 5.7 TB/s; 4093
// fp32 tokens (16 heads of 80, 20 of 32 lanes in use) 11.0 us, 3.8 TB/s; 48 tokens into the cache 4.2 us, of which a launch
// that does nothing takes 1.8.  HBM traffic is that of the heads alone (134.9 + 134.2 MB of 268.5).
#include "qk_rope.h"

namespace lory {

namespace {

using namespace rope;

struct Args {
    Heads q, k, v, q_out, k_out;
    const int32_t *pos;
    const double *freq;
    const void *wq, *wk;
    const int64_t *slots;
    char *k_cache, *v_cache;
    long slots_end;         // pages * page
    int page;
    int tokens, Hq, Hkv, D, rot;
    float eps;
};

// STREAM: the heads are read past the caches.
template <typename T, int LPH, bool INTER, bool STORE, bool STREAM> __global__ __launch_bounds__(64 * kWaves) void qk_rope_kernel(Args a)
{
    constexpr int VEC = 16 / sizeof(T), HPW = 64 / LPH;   // heads of a group: one load of the wavefront
    constexpr int U = 4;                                  // groups in flight
    __shared__ float2 table[kWaves][kMaxPairs];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int t = blockIdx.x * kWaves + wave;
    if (t >= a.tokens) return;   // wavefronts share nothing

    const Lane l = lane_of<T, LPH, INTER>(lane, a.D, a.rot);
    const int gq = (a.Hq + HPW - 1) / HPW, gk = (a.Hkv + HPW - 1) / HPW;
    const int groups = gq + gk + (STORE ? gk : 0);
    // this wavefront's share of the token's groups
    const int g0 = (int)((long)blockIdx.y * groups / gridDim.y), g1 = (int)((long)(blockIdx.y + 1) * groups / gridDim.y);

    char *krow = nullptr, *vrow = nullptr;
    long khead = a.k_out.head;
    bool kept = true;
    if constexpr (STORE) {
        const int64_t slot = a.slots[t];
        kept = slot >= 0 && slot < a.slots_end;
        const unsigned page = kept ? (unsigned)(slot / a.page) : 0;
        const unsigned row = kept ? (unsigned)(slot - (int64_t)page * a.page) : 0;
        khead = (long)a.page * a.D * sizeof(T);
        const long at = (long)page * a.Hkv * khead + (long)row * a.D * sizeof(T);
        krow = a.k_cache + at;
        vrow = a.v_cache + at;
    } else {
        krow = a.k_out.p + t * a.k_out.token;
    }

    if (g0 < gq + gk) {
        const double pos = a.pos[t];
        for (int i = lane; i < (a.rot >> 1); i += 64) table[wave][i] = turn_of(pos, a.freq[i]);
        wave_sync();
        float c[VEC], s[VEC];
        factors<T, INTER>(l, table[wave], 1.f, c, s);

        auto section = [&](int lo, int hi, int H, const char *src, long src_head, char *dst, long dst_head, const T *w,
                           bool write) {
            if (lo >= hi) return;
            float A[VEC], B[VEC];
            {
                float own[VEC], other[VEC];
                weights<T, INTER>(l, w, false, own);
                weights<T, INTER>(l, w, true, other);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    A[e] = own[e] * c[e];
                    B[e] = other[e] * s[e];
                }
            }
            for (int g = lo; g < hi; g += U) {
                Chunk raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = (g + u) * HPW + l.sub;
                    raw[u] = Chunk{0, 0, 0, 0};
                    if (g + u < hi && h < H && l.on)
                        raw[u] = load<STREAM>(src + h * src_head + l.chunk * 16);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (g + u >= hi) break;
                    const int h = (g + u) * HPW + l.sub;
                    float x[VEC], p[VEC], y[VEC], r = 1.f;
                    widen<T>(raw[u], x);
                    widen<T>(exchange<T, LPH, INTER>(l, raw[u]), p);
                    if (w) {
                        float ss = 0.f;
#pragma unroll
                        for (int e = 0; e < VEC; ++e) ss = fmaf(x[e], x[e], ss);
                        r = rsqrtf(head_sum<LPH>(ss) / (float)a.D + a.eps);
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[e] = r * fmaf(x[e], A[e], p[e] * B[e]);
                    if (h < H && l.on && write)
                        store_once(dst + h * dst_head + l.chunk * 16, narrow<T>(y));
                }
            }
        };
        section(g0, g1 < gq ? g1 : gq, a.Hq, a.q.p + t * a.q.token, a.q.head, a.q_out.p + t * a.q_out.token, a.q_out.head,
                (const T *)a.wq, true);
        section((g0 > gq ? g0 : gq) - gq, (g1 < gq + gk ? g1 : gq + gk) - gq, a.Hkv, a.k.p + t * a.k.token, a.k.head, krow, khead,
                (const T *)a.wk, kept);
    }
    if constexpr (STORE) {
        const int lo = g0 > gq + gk ? g0 - gq - gk : 0;
        if (!kept || !l.on) return;
        const char *src = a.v.p + t * a.v.token + l.chunk * 16;
#pragma unroll 4
        for (int g = lo; g < g1 - gq - gk; ++g) {
            const int h = g * HPW + l.sub;
            if (h < a.Hkv)
                store_once(vrow + h * khead + l.chunk * 16, load<STREAM>(src + h * a.v.head));
        }
    }
}

// Heads of more than 96 MB are read past the caches: less is what the 256 MB memory-side cache may still hold from the
// projection (us with and without: 134 MB read 49.7 / 52.3, 165 MB 45.7 / 46.7; 74 MB 30.7 / 26.2, 21 MB 13.9 / 11.3, just written).
constexpr long kStreamBytes = 96l << 20;

template <typename T, int LPH, bool STORE> void launch2(const Args &a, bool inter, hipStream_t st)
{
    constexpr int HPW = 64 / LPH;
    const int gq = (a.Hq + HPW - 1) / HPW, gk = (a.Hkv + HPW - 1) / HPW;
    const int groups = gq + gk * (STORE ? 2 : 1), blocks = (a.tokens + kWaves - 1) / kWaves;
    // a token's heads over several wavefronts until there are 4096 of them (four per SIMD; 48 tokens of 40 heads take 4.2 us
    // so, and more wavefronts cost larger calls the angles again: 4093 fp32 tokens 15.7 us against 11.3)
    int ny = (1024 + blocks - 1) / blocks;
    if (ny > groups) ny = groups;
    const dim3 grid(blocks, ny), block(64 * kWaves);
    const bool stream = (long)a.tokens * (a.Hq + (STORE ? 2 : 1) * a.Hkv) * a.D * (long)sizeof(T) > kStreamBytes;
    if (inter && stream)
        hipLaunchKernelGGL((qk_rope_kernel<T, LPH, true, STORE, true>), grid, block, 0, st, a);
    else if (inter)
        hipLaunchKernelGGL((qk_rope_kernel<T, LPH, true, STORE, false>), grid, block, 0, st, a);
    else if (stream)
        hipLaunchKernelGGL((qk_rope_kernel<T, LPH, false, STORE, true>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((qk_rope_kernel<T, LPH, false, STORE, false>), grid, block, 0, st, a);
}

template <typename T, bool STORE> void launch1(const Args &a, bool inter, hipStream_t st)
{
    switch (lanes_per_head<T>(a.D)) {
    case 8: launch2<T, 8, STORE>(a, inter, st); break;
    case 16: launch2<T, 16, STORE>(a, inter, st); break;
    case 32: launch2<T, 32, STORE>(a, inter, st); break;
    default:
        if constexpr (sizeof(T) == 4) launch2<T, 64, STORE>(a, inter, st);
    }
}

}  // namespace

int qk_rope_launch(const lory_rope_shape &s, const lory_heads &q, const lory_heads &k, const int32_t *pos, const double *freq,
                   const void *wq, const void *wk, const lory_heads &q_out, const lory_heads *k_out, const RopeCache *cache,
                   hipStream_t st)
{
    const int esize = s.dtype == LORY_F32 ? 4 : 2;
    Args a = {};
    a.q = heads(q, esize);
    a.k = heads(k, esize);
    a.q_out = heads(q_out, esize);
    a.pos = pos;
    a.freq = freq;
    a.wq = wq;
    a.wk = wk;
    a.tokens = s.tokens;
    a.Hq = s.q_heads;
    a.Hkv = s.kv_heads;
    a.D = s.head_dim;
    a.rot = s.rot_dim;
    a.eps = s.eps;
    if (cache) {
        a.v = heads(*cache->v, esize);
        a.slots = cache->slots;
        a.k_cache = (char *)cache->k_cache;
        a.v_cache = (char *)cache->v_cache;
        a.slots_end = (long)cache->pages * cache->page;
        a.page = cache->page;
    } else {
        a.k_out = heads(*k_out, esize);
    }
    const double values = (double)s.tokens * (s.q_heads + s.kv_heads) * s.head_dim;
    prof::Range r(st, prof::kQkRope, 9.0 * values,
                  2.0 * esize * (values + (cache ? (double)s.tokens * s.kv_heads * s.head_dim : 0.0)) +
                      (cache ? 12.0 : 4.0) * s.tokens);
    const bool inter = s.interleaved != 0;
    if (s.dtype == LORY_F32)
        cache ? launch1<float, true>(a, inter, st) : launch1<float, false>(a, inter, st);
    else
        cache ? launch1<__hip_bfloat16, true>(a, inter, st) : launch1<__hip_bfloat16, false>(a, inter, st);
    return launch_status();
}

}  // namespace lory
