// Plan of a generating step (lory_kv_plan): pages, positions and slots of the new tokens from the requests' lengths.
//
// Latency-bound: at most 12 bytes a token and a few reads a row.  One launch: every workgroup takes the prefix sums over all
// rows for itself (8 bytes a row from L2, cheaper than a second launch or a wait between workgroups) and then fills
// its share of the outputs.  A token, a page that a row takes and a page that comes back each find their row by a
// binary search over the sums of chunks of rows in LDS and a walk inside the chunk.  Pages that come back are never read from
// where another workgroup may just write them: place j of the grown stack is free[j] below the old top and the
// page table's own entry above it, entries that no workgroup changes.  Tokens and pages are one list, a thread each: one
// loop after the other took 9.0 us where this takes 6.7 (1000 rows, 88000 new tokens).  64 rows with a token each: 3.8 us, a
// launch that does nothing 1.8.
#include "lory_internal.h"

namespace lory {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

struct Args {
    const int32_t *lens, *add;
    int32_t *table, *free;
    const int32_t *count;
    int32_t *lens_new, *cu, *positions;
    int64_t *slots;
    int32_t *count_new, *status;
    long table_row;
    int rows, width, page, free_size, room;
    int chunk;   // rows of a thread's chunk
};

// Sums that pass 32 bits stay at the largest value: any limit they are compared with is smaller.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t page) { return tokens ? (tokens - 1) / page + 1 : 0; }

struct Row {
    uint32_t n, old, take, give;   // new tokens; pages it has, takes, gives back
    uint32_t flags;
    int64_t len_new;
};

__device__ __forceinline__ Row row_of(const Args &a, int32_t len, int32_t add)
{
    Row r;
    const int64_t most = (int64_t)a.width * a.page;   // below 2^31
    const bool ended = add < 0;
    r.flags = (len < 0 || (ended && len > most)) ? 16 : 0;
    const uint32_t l = len < 0 ? 0 : (uint32_t)len;
    r.n = ended ? 0 : (uint32_t)add;
    r.len_new = ended ? 0 : (int64_t)l + r.n;
    if (r.len_new > most) r.flags |= 2;
    r.old = pages_of(l, (uint32_t)a.page);
    r.take = ended ? 0 : pages_of(l + r.n, (uint32_t)a.page) - r.old;
    r.give = ended ? r.old : 0;
    return r;
}

__global__ __launch_bounds__(kThreads) void kv_plan_kernel(Args a)
{
    // sums before each chunk of rows: new tokens, pages taken, pages given back
    __shared__ uint32_t pn[kThreads + 1], pt[kThreads + 1], pg[kThreads + 1];
    __shared__ uint32_t wn[kWaves], wt[kWaves], wg[kWaves], wf[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int first = tid * a.chunk, last = min(first + a.chunk, a.rows);
    const int32_t count = a.count[0];

    uint32_t n = 0, t = 0, g = 0, flags = 0;
    for (int b = first; b < last; ++b) {
        const Row r = row_of(a, a.lens[b], a.add[b]);
        n = add_sat(n, r.n);
        t = add_sat(t, r.take);
        g = add_sat(g, r.give);
        flags |= r.flags;
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t un = __shfl_up(n, m, 64), ut = __shfl_up(t, m, 64), ug = __shfl_up(g, m, 64);
        if (lane >= m) {
            n = add_sat(n, un);
            t = add_sat(t, ut);
            g = add_sat(g, ug);
        }
    }
    uint32_t all_flags = 0;
#pragma unroll
    for (int bit = 1; bit <= 16; bit <<= 1) all_flags |= __ballot(flags & bit) ? bit : 0;
    if (lane == 63) {
        wn[wave] = n;
        wt[wave] = t;
        wg[wave] = g;
        wf[wave] = all_flags;
    }
    __syncthreads();
    uint32_t bn = 0, bt = 0, bg = 0;
    flags = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) {
            bn = add_sat(bn, wn[w]);
            bt = add_sat(bt, wt[w]);
            bg = add_sat(bg, wg[w]);
        }
        flags |= wf[w];
    }
    pn[tid + 1] = add_sat(n, bn);
    pt[tid + 1] = add_sat(t, bt);
    pg[tid + 1] = add_sat(g, bg);
    if (tid == 0) pn[0] = pt[0] = pg[0] = 0;
    __syncthreads();

    const uint32_t tokens = pn[kThreads], taken = pt[kThreads], given = pg[kThreads];
    const int64_t top = (int64_t)count + given;
    if (count < 0 || count > a.free_size) flags |= 16;
    if (tokens > (uint32_t)a.room) flags |= 1;
    if ((int64_t)taken > top) flags |= 4;
    if (top > a.free_size) flags |= 8;
    const bool ok = flags == 0;
    const long step = (long)gridDim.x * kThreads, me = (long)blockIdx.x * kThreads + tid;

    // last chunk whose sum before it is not above i
    auto chunk_of = [&](const uint32_t *sums, uint32_t i) {
        int lo = 0, hi = kThreads;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sums[mid] <= i) lo = mid; else hi = mid;
        }
        return lo;
    };
    // place j of the stack with the pages that come back on top
    auto stack = [&](int64_t j) -> int32_t {
        if (j < count) return a.free[j];
        uint32_t i = (uint32_t)(j - count);
        const int ch = chunk_of(pg, i);
        i -= pg[ch];
        int b = ch * a.chunk;
        for (const int end = min(b + a.chunk, a.rows) - 1; b < end; ++b) {
            const uint32_t give = row_of(a, a.lens[b], a.add[b]).give;
            if (i < give) break;
            i -= give;
        }
        return a.table[(long)b * a.table_row + i];
    };

    if (blockIdx.x == 0) {
        if (tid == 0) {
            *a.status = (int32_t)flags;
            *a.count_new = ok ? (int32_t)(top - taken) : count;
            a.cu[0] = 0;
        }
        uint32_t before = pn[tid];
        for (int b = first; b < last; ++b) {
            const int32_t len = a.lens[b];
            const Row r = row_of(a, len, a.add[b]);
            before = add_sat(before, r.n);
            a.lens_new[b] = ok ? (int32_t)r.len_new : len;
            a.cu[b + 1] = ok ? (int32_t)before : 0;
        }
    }

    // one list of work: positions and slots, pages that rows take, places of the stack that pages come back to
    const long back = ok && top - taken > count ? top - taken - count : 0, pages = ok ? taken : 0, all = a.room + pages + back;
    for (long x = me; x < all; x += step) {
        if (x >= a.room + pages) {
            const int64_t j = count + (x - a.room - pages);
            a.free[j] = stack(j);
            continue;
        }
        // the row of a token or of a page that is taken: rest items of it come before
        const bool token = x < a.room;
        const uint32_t i = (uint32_t)(token ? x : x - a.room);
        if (token && (!ok || i >= tokens)) {
            a.positions[i] = 0;
            a.slots[i] = -1;
            continue;
        }
        const int ch = token ? chunk_of(pn, i) : chunk_of(pt, i);
        uint32_t rest = i - (token ? pn[ch] : pt[ch]), took = pt[ch];
        int b = ch * a.chunk;
        const int end = min(b + a.chunk, a.rows) - 1;
        int32_t len = a.lens[b];
        Row r = row_of(a, len, a.add[b]);
        while (b < end && rest >= (token ? r.n : r.take)) {
            rest -= token ? r.n : r.take;
            took += r.take;
            ++b;
            len = a.lens[b];
            r = row_of(a, len, a.add[b]);
        }
        int32_t *row = a.table + (long)b * a.table_row;
        if (token) {
            const int32_t at = len + (int32_t)rest;
            const uint32_t c = (uint32_t)at / (uint32_t)a.page;
            const int32_t page = c < r.old ? row[c] : stack(top - 1 - took - (c - r.old));
            a.positions[i] = at;
            a.slots[i] = (int64_t)page * a.page + (at - (int32_t)(c * a.page));
        } else {
            row[r.old + rest] = stack(top - 1 - i);
        }
    }
}

}  // namespace

int kv_plan_launch(const lory_plan_shape &s, const int32_t *lens, const int32_t *add, int32_t *table, int32_t *free,
                   const int32_t *count, int32_t *lens_new, int32_t *cu, int32_t *positions, int64_t *slots, int32_t *count_new,
                   int32_t *status, hipStream_t st)
{
    Args a = {lens, add, table, free, count, lens_new, cu, positions, slots, count_new, status,
              (long)s.table_row, s.rows, s.width, s.page, s.free_size, s.room, (s.rows + kThreads - 1) / kThreads};
    // a thread for every token, page that can be taken and place that one can come back to, two workgroups a CU at most
    const long items = (long)s.room + s.room / s.page + s.rows + s.free_size;
    long blocks = (items + kThreads - 1) / kThreads;
    if (blocks > 512) blocks = 512;
    prof::Range r(st, prof::kKvPlan, 0.0, 12.0 * s.room + 16.0 * s.rows);
    hipLaunchKernelGGL(kv_plan_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a);
    return launch_status();
}

}  // namespace lory
