// Gradient of the head norm and rotation (lory_qk_rope_bwd).
//
// HBM-bound: heads and their gradients are read once, the input gradients written once.  With g = the gradient turned back,
//   dx = r g w - x r^3 / D * sum(g w x),   dw += g x r,
// so both sums of a head (x^2 and g w x) come from the same registers.  Wavefronts walk over tokens and keep dw of their
// chunk in registers; every workgroup adds its wavefronts in LDS and leaves one row of partial sums, and a second
// launch adds the rows in order: the same bits on every run.  A few tokens take one workgroup, and that launch only (qk_rope_plan.h).
// 128 registers, four wavefronts per SIMD and 1024 workgroups, all resident at once: with 141 registers a quarter of them
// waited for a second round (99 us against 79 for 16384 tokens of 32 heads of 128, bf16).  Workgroups of eight or 16 wavefronts leave
// fewer rows to add but measured the same or slower (79.6, 86).
// Measured: those 16384 tokens 73.7 us, 5.5 TB/s, and 4.5 us for the rows; 2999 fp32 tokens of 24 + 8 heads of 64 16.7 + 3.8 us.
#include "qk_rope.h"
#include "qk_rope_plan.h"

namespace lory {

namespace {

using namespace rope;

constexpr int kMaxBlocks = 1024;   // rows of partial sums

struct Args {
    Heads q, k, dyq, dyk, dq, dk;
    const int32_t *pos;
    const double *freq;
    const void *wq, *wk;
    float *part;   // [blocks][2][D]
    float *dwq, *dwk;
    int tokens, shares, Hq, Hkv, D, rot;
    float eps;
};

// WAVES wavefronts a workgroup: kWaves, or kAlone for a launch of one workgroup, which writes dw itself.
template <typename T, int LPH, bool INTER, bool NORM, int WAVES> __global__ __launch_bounds__(64 * WAVES, 4) void qk_rope_bwd_kernel(Args a)
{
    constexpr int VEC = 16 / sizeof(T), HPW = 64 / LPH;
    constexpr int U = sizeof(T) == 4 ? 4 : 2;   // groups in flight, what the registers allow
    __shared__ float2 table[WAVES][kMaxPairs];
    __shared__ float sums[WAVES][2 * LPH * VEC];
    const int lane = threadIdx.x & 63, wave = wave_index();
    const Lane l = lane_of<T, LPH, INTER>(lane, a.D, a.rot);
    const int gq = (a.Hq + HPW - 1) / HPW, gk = (a.Hkv + HPW - 1) / HPW, groups = gq + gk;

    float accq[VEC], acck[VEC], wq[VEC], wk[VEC];
    weights<T, INTER>(l, (const T *)a.wq, false, wq);
    weights<T, INTER>(l, (const T *)a.wk, false, wk);
#pragma unroll
    for (int e = 0; e < VEC; ++e) accq[e] = acck[e] = 0.f;

    // an item is a share of a token's heads
    const long items = (long)a.tokens * a.shares;
    for (long item = (long)blockIdx.x * WAVES + wave; item < items; item += (long)gridDim.x * WAVES) {
        const int t = (int)(item / a.shares), share = (int)(item - (long)t * a.shares);
        const int g0 = share * groups / a.shares, g1 = (share + 1) * groups / a.shares;
        const double pos = a.pos[t];
        wave_sync();   // the table's last readers are done
        for (int i = lane; i < (a.rot >> 1); i += 64) table[wave][i] = turn_of(pos, a.freq[i]);
        wave_sync();
        float c[VEC], s[VEC];
        factors<T, INTER>(l, table[wave], -1.f, c, s);

        auto section = [&](int lo, int hi, int H, const char *src, long src_head, const char *grad, long grad_head, char *dst,
                           long dst_head, const float (&w)[VEC], float (&acc)[VEC]) {
            for (int g = lo; g < hi; g += U) {
                Chunk rx[U], rg[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = (g + u) * HPW + l.sub;
                    rx[u] = rg[u] = Chunk{0, 0, 0, 0};
                    if (g + u < hi && h < H && l.on) {
                        if constexpr (NORM) rx[u] = load<true>(src + h * src_head + l.chunk * 16);
                        rg[u] = load<true>(grad + h * grad_head + l.chunk * 16);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (g + u >= hi) break;
                    const int h = (g + u) * HPW + l.sub;
                    float dy[VEC], p[VEC], y[VEC];
                    widen<T>(rg[u], dy);
                    widen<T>(exchange<T, LPH, INTER>(l, rg[u]), p);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[e] = fmaf(dy[e], c[e], p[e] * s[e]);
                    if constexpr (NORM) {
                        // not 0 where no head is: an infinite r, without eps, would make NaN of its zeros
                        float x[VEC], xx = h < H ? 0.f : 1.f, gx = 0.f;
                        widen<T>(rx[u], x);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            xx = fmaf(x[e], x[e], xx);
                            gx = fmaf(y[e] * w[e], x[e], gx);
                        }
                        const float r = rsqrtf(head_sum<LPH>(xx) / (float)a.D + a.eps);
                        const float m = head_sum<LPH>(gx) / (float)a.D * r * r;
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            acc[e] = fmaf(y[e], x[e] * r, acc[e]);
                            y[e] = r * fmaf(-x[e], m, y[e] * w[e]);
                        }
                    }
                    if (h < H && l.on) store_once(dst + h * dst_head + l.chunk * 16, narrow<T>(y));
                }
            }
        };
        section(g0, g1 < gq ? g1 : gq, a.Hq, a.q.p + t * a.q.token, a.q.head, a.dyq.p + t * a.dyq.token, a.dyq.head,
                a.dq.p + t * a.dq.token, a.dq.head, wq, accq);
        section((g0 > gq ? g0 : gq) - gq, g1 - gq, a.Hkv, a.k.p + t * a.k.token, a.k.head, a.dyk.p + t * a.dyk.token, a.dyk.head,
                a.dk.p + t * a.dk.token, a.dk.head, wk, acck);
    }
    if constexpr (NORM) {
        // the heads of a wavefront's groups, then the wavefronts, in order
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
#pragma unroll
            for (int m = LPH; m < 64; m <<= 1) {
                accq[e] += __shfl_xor(accq[e], m, 64);
                acck[e] += __shfl_xor(acck[e], m, 64);
            }
            if (l.sub == 0) {
                sums[wave][l.chunk * VEC + e] = accq[e];
                sums[wave][(LPH + l.chunk) * VEC + e] = acck[e];
            }
        }
        __syncthreads();
        float *dst = a.part + (size_t)blockIdx.x * 2 * a.D;
        for (int i = threadIdx.x; i < 2 * a.D; i += 64 * WAVES) {
            const int j = i < a.D ? i : i - a.D + LPH * VEC;
            float v = sums[0][j];
#pragma unroll
            for (int n = 1; n < WAVES; ++n) v += sums[n][j];
            if constexpr (WAVES == kWaves)
                dst[i] = v;
            else
                (i < a.D ? a.dwq : a.dwk)[i < a.D ? i : i - a.D] = v;
        }
    }
}

// dw from the rows of partial sums, 16 columns a workgroup: a thread takes every 64th row of its column, the 64 sums of a column
// are added in order, a quarter per lane, and the quarters last.  1024 rows of 2 x 128: 4.6 us, a launch and three latencies.
constexpr int kDwColumns = 16;

__global__ __launch_bounds__(1024) void qk_rope_dw_kernel(const float *part, int rows, int D, float *dwq, float *dwk)
{
    __shared__ float sums[64][kDwColumns];
    const int c = threadIdx.x % kDwColumns, g = threadIdx.x / kDwColumns;
    const int col = blockIdx.x * kDwColumns + c;   // below 2 D, which is a multiple of 16
    float x[kMaxBlocks / 64], v = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxBlocks / 64; ++i) {   // all under way at once
        x[i] = 0.f;
        if (g + 64 * i < rows) x[i] = part[(size_t)(g + 64 * i) * 2 * D + col];
    }
#pragma unroll
    for (int i = 0; i < kMaxBlocks / 64; ++i) v += x[i];
    sums[g][c] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) total += sums[16 * g + i][c];
    total += __shfl_xor(total, 16, 64);
    total += __shfl_xor(total, 32, 64);
    if (g == 0) (col < D ? dwq : dwk)[col < D ? col : col - D] = total;
}

struct Plan {
    int shares, blocks;
};

// Groups of a token's heads: loads of a wavefront.
int groups_of(const lory_rope_shape &s)
{
    const int lph = s.dtype == LORY_F32 ? lanes_per_head<float>(s.head_dim) : lanes_per_head<__hip_bfloat16>(s.head_dim);
    const int hpw = 64 / lph;
    return (s.q_heads + hpw - 1) / hpw + (s.kv_heads + hpw - 1) / hpw;
}

// A token's heads over as many wavefronts as end first: rounds of the items over 4 kMaxBlocks wavefronts, each as long as
// its groups and about one more for the angles.
Plan plan(const lory_rope_shape &s)
{
    const int groups = groups_of(s), waves = kWaves * kMaxBlocks;
    Plan p = {1, 0};
    if (s.tokens <= 0) return p;
    long best = 0;
    for (int n = 1; n <= groups && (n == 1 || (long)s.tokens * (n - 1) < 4 * waves); ++n) {
        const long cost = ((long)s.tokens * n + waves - 1) / waves * ((groups + n - 1) / n + 1);
        if (n == 1 || cost < best) {
            best = cost;
            p.shares = n;
        }
    }
    const long blocks = ((long)s.tokens * p.shares + kWaves - 1) / kWaves;
    p.blocks = (int)(blocks < kMaxBlocks ? blocks : kMaxBlocks);
    return p;
}

template <typename T, int LPH, bool INTER> void launch3(const Args &a, int blocks, bool norm, bool alone, hipStream_t st)
{
    if (alone)
        hipLaunchKernelGGL((qk_rope_bwd_kernel<T, LPH, INTER, true, kAlone>), dim3(1), dim3(64 * kAlone), 0, st, a);
    else if (norm)
        hipLaunchKernelGGL((qk_rope_bwd_kernel<T, LPH, INTER, true, kWaves>), dim3(blocks), dim3(64 * kWaves), 0, st, a);
    else
        hipLaunchKernelGGL((qk_rope_bwd_kernel<T, LPH, INTER, false, kWaves>), dim3(blocks), dim3(64 * kWaves), 0, st, a);
}

template <typename T, int LPH> void launch2(const Args &a, int blocks, bool inter, bool norm, bool alone, hipStream_t st)
{
    if (inter)
        launch3<T, LPH, true>(a, blocks, norm, alone, st);
    else
        launch3<T, LPH, false>(a, blocks, norm, alone, st);
}

template <typename T> void launch1(const Args &a, int blocks, bool inter, bool norm, bool alone, hipStream_t st)
{
    switch (lanes_per_head<T>(a.D)) {
    case 8: launch2<T, 8>(a, blocks, inter, norm, alone, st); break;
    case 16: launch2<T, 16>(a, blocks, inter, norm, alone, st); break;
    case 32: launch2<T, 32>(a, blocks, inter, norm, alone, st); break;
    default:
        if constexpr (sizeof(T) == 4) launch2<T, 64>(a, blocks, inter, norm, alone, st);
    }
}

}  // namespace

size_t qk_rope_bwd_workspace_bytes(const lory_rope_shape &s)
{
    return align_up((size_t)plan(s).blocks * 2 * s.head_dim * sizeof(float), 256);
}

int qk_rope_bwd_launch(const lory_rope_shape &s, const lory_heads &q, const lory_heads &k, const lory_heads &dq_out,
                       const lory_heads &dk_out, const int32_t *pos, const double *freq, const void *wq, const void *wk,
                       const lory_heads &dq, const lory_heads &dk, float *dwq, float *dwk, void *ws, hipStream_t st)
{
    const int esize = s.dtype == LORY_F32 ? 4 : 2;
    const Plan p = plan(s);
    Args a = {};
    a.q = heads(q, esize);
    a.k = heads(k, esize);
    a.dyq = heads(dq_out, esize);
    a.dyk = heads(dk_out, esize);
    a.dq = heads(dq, esize);
    a.dk = heads(dk, esize);
    a.pos = pos;
    a.freq = freq;
    a.wq = wq;
    a.wk = wk;
    a.part = (float *)ws;
    a.dwq = dwq;
    a.dwk = dwk;
    a.tokens = s.tokens;
    a.shares = p.shares;
    a.Hq = s.q_heads;
    a.Hkv = s.kv_heads;
    a.D = s.head_dim;
    a.rot = s.rot_dim;
    a.eps = s.eps;
    const double values = (double)s.tokens * (s.q_heads + s.kv_heads) * s.head_dim;
    prof::Range r(st, prof::kQkRopeBwd, 17.0 * values, (wq ? 3.0 : 2.0) * esize * values + 4.0 * s.tokens);
    const bool inter = s.interleaved != 0, norm = wq != nullptr;
    const bool alone = norm && rope::alone(s.tokens, (long)s.tokens * (s.q_heads + s.kv_heads) * s.head_dim);
    if (alone) {
        const int groups = groups_of(s), shares = kAlone / s.tokens;
        a.shares = shares < groups ? shares : groups;
    }
    if (p.blocks > 0) {
        if (s.dtype == LORY_F32)
            launch1<float>(a, p.blocks, inter, norm, alone, st);
        else
            launch1<__hip_bfloat16>(a, p.blocks, inter, norm, alone, st);
    }
    if (norm && !alone)
        hipLaunchKernelGGL(qk_rope_dw_kernel, dim3(2 * s.head_dim / kDwColumns), dim3(1024), 0, st, (const float *)ws, p.blocks,
                           s.head_dim, dwq, dwk);
    return launch_status();
}

}  // namespace lory
