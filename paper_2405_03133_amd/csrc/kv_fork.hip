// Rows of a paged cache that go on from other rows (lory_kv_fork), and copies of its pages (lory_kv_copy).
//
// lory_kv_fork is latency-bound: 4 bytes of the table's entries in and out.  Which pages come back needs no counts of
// their owners kept between calls: a page comes back if an old row without children has it and no row with children does.  Every old row is
// marked once, in two sets over the pool; the sums over rows and over words of the sets then say which page goes to which place of
// the stack or, above its new top, to the row that takes it.
//
// Small tables are one workgroup's, with the sets as bits in LDS.  Larger ones take three launches: the first children of the old rows, and
// the sets cleared; the marks and the new tables; the sums, by one workgroup.  There the sets are bytes, set by plain stores: bits
// need atomic operations that all XCDs see, 41 us for 512 rows of 95 pages where the bytes take 4.2.
// Measured: 16 rows of up to 94 pages in one launch 5.3 us (three took 9.7 and two more starts); 512 rows of up to 260 pages 2.1 + 4.2 +
// 5.6, 240 rows of up to 1600 2.0 + 5.0 + 6.1; the last launch is a chain of reads and two sums over its threads.
//
// lory_kv_copy is bound by HBM: 3001 pages of 128 KB 158.6 us, 4.96 TB/s read and written together, a large copy's rate.
#include "lory_internal.h"

namespace lory {

namespace {

constexpr int kThreads = 256, kLast = 1024;
constexpr int kSmallRows = 2048, kSmallPages = 1 << 17;      // whose sets and first children LDS holds
// Entries of both tables up to which one workgroup is faster, us called eagerly, one launch / three: 1024 5.5 / 10.6, 4416 7.4 / 10.2,
// 8832 9.7 / 10.2, 17664 15.0 / 10.6, 33792 23.7 / 12.5.
constexpr int kSmallEntries = 9000;
constexpr int kFirstRows = 8192;                             // old rows of a workgroup that finds first children
constexpr int kLocalWords = 8192;                            // of 32 pages, that the last launch packs by itself

struct Args {
    const int32_t *lens, *src, *table;
    int32_t *free;
    const int32_t *count;
    int32_t *lens_new, *table_new, *count_new, *copies, *status;
    long table_row, new_row;
    int old_rows, rows, width, page, pages, free_size;
    // workspace
    uint8_t *ended, *kept;   // by page: an old row without children has it, one with children does
    uint32_t *back;          // bits: pages that come back
    int32_t *first;          // first child of every old row, INT32_MAX: none
    int32_t *got;            // pages that come back and are taken again, by taker
    int32_t *flags;
    int words;               // of 32 pages
};

__device__ __forceinline__ int pages_of(const Args &a, int len)   // of a length inside its limits
{
    return (int)(((uint32_t)len + a.page - 1) / (uint32_t)a.page);
}
__device__ __forceinline__ bool bad_length(const Args &a, int len) { return len < 0 || len > (long)a.width * a.page; }

// Workgroups 0 .. groups - 1: first children; the others clear the sets.
__global__ __launch_bounds__(kLast) void kv_fork_begin_kernel(Args a, int groups)
{
    __shared__ int32_t first[kFirstRows];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < groups) {
        const int r0 = blockIdx.x * kFirstRows, n = min(kFirstRows, a.old_rows - r0);
        for (int i = tid; i < n; i += kLast) first[i] = INT32_MAX;
        __syncthreads();
        for (int b = tid; b < a.rows; b += kLast) {
            const int r = a.src[b];
            if (r >= r0 && r < r0 + n) atomicMin(first + (r - r0), b);
        }
        __syncthreads();
        for (int i = tid; i < n; i += kLast) a.first[r0 + i] = first[i];
        return;
    }
    const long step = (long)(gridDim.x - groups) * kLast, me = (long)(blockIdx.x - groups) * kLast + tid;
    uint4 *e = reinterpret_cast<uint4 *>(a.ended), *k = reinterpret_cast<uint4 *>(a.kept);
    for (long i = me; i < 2l * a.words; i += step) e[i] = k[i] = make_uint4(0, 0, 0, 0);
    if (me == 0) *a.flags = 0;
}

// grid (column blocks, rows): old rows first, then new ones
__global__ __launch_bounds__(kThreads) void kv_fork_mark_kernel(Args a)
{
    const int c0 = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
    for (long y = blockIdx.y; y < (long)a.old_rows + a.rows; y += gridDim.y) {
        const bool old = y < a.old_rows;
        const int b = (int)(y - a.old_rows), row = old ? (int)y : a.src[b];
        if (!old && row < 0) continue;
        if (row >= a.old_rows) {
            if (c0 == 0) atomicOr(a.flags, 16);
            continue;
        }
        const int len = a.lens[row], child = a.first[row];
        if (old && child != INT32_MAX) continue;   // its first child marks its pages
        if (bad_length(a, len)) {
            if (c0 == 0) atomicOr(a.flags, 16);
            continue;
        }
        const int used = pages_of(a, len);
        const int32_t *from = a.table + row * a.table_row;
        uint8_t *set = old ? a.ended : child == b ? a.kept : nullptr;
        int32_t *to = a.table_new + b * a.new_row;
        bool bad = false;
        for (int c = c0; c < used; c += step) {
            const int page = from[c];
            if (!old) to[c] = page;
            if ((uint32_t)page >= (uint32_t)a.pages)
                bad = true;
            else if (set)
                set[page] = 1;
        }
        if (bad) atomicOr(a.flags, 16);
    }
}

// Bit i of the result: byte i of two 16-byte pieces is set in `e` and not in `k`.
__device__ __forceinline__ uint32_t bits_of(const uint8_t *e, const uint8_t *k)
{
    uint32_t r = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 x = reinterpret_cast<const uint4 *>(e)[h], y = reinterpret_cast<const uint4 *>(k)[h];
        const uint32_t w[4] = {x.x & ~y.x, x.y & ~y.y, x.z & ~y.z, x.w & ~y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) r |= (w[i] * 0x01020408u >> 24 & 15u) << (16 * h + 4 * i);   // bytes are 0 or 1: no carries
    }
    return r;
}

// Pools of more pages than the last launch packs by itself.
__global__ __launch_bounds__(kThreads) void kv_fork_pack_kernel(Args a)
{
    const int w = blockIdx.x * kThreads + threadIdx.x;
    if (w < a.words) a.back[w] = bits_of(a.ended + 32l * w, a.kept + 32l * w);
}

// Sum before this thread's and of all; kLast threads.
__device__ __forceinline__ uint32_t scan(uint32_t own, uint32_t *sums, uint32_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t v = own;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t u = __shfl_up(v, m, 64);
        if (lane >= m) v += u;
    }
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kLast / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    __syncthreads();
    all = total;
    return before + v - own;
}

// What is left once the pages that come back are known (bits, in words): by one workgroup.  first: of the old rows; got: room for a page of
// every new row; flags: the same in all threads.
__device__ __forceinline__ void finish(const Args &a, int flags, const uint32_t *back, const int32_t *first, int32_t *got, uint32_t *sums)
{
    const int tid = threadIdx.x;
    const int chunk = (a.rows + kLast - 1) / kLast, b0 = min(tid * chunk, a.rows), b1 = min(b0 + chunk, a.rows);
    const int wchunk = (a.words + kLast - 1) / kLast, w0 = min(tid * wchunk, a.words), w1 = min(w0 + wchunk, a.words);
    const int count = *a.count;
    if (count < 0 || count > a.free_size) flags |= 16;

    // the row that b goes on from, or -1; copies: it needs a page of its own
    auto parent = [&](int b, int &len, bool &copies) {
        const int r = a.src[b];
        len = r >= 0 ? a.lens[r] : 0;
        copies = r >= 0 && len % a.page != 0 && first[r] != b;
        return r;
    };
    uint32_t takes = 0, gives = 0;
    if (!(flags & 16)) {
        for (int b = b0; b < b1; ++b) {
            int len;
            bool copies;
            parent(b, len, copies);
            takes += copies;
        }
        for (int w = w0; w < w1; ++w) gives += __popc(back[w]);
    }
    uint32_t taken, given;
    const uint32_t taker0 = scan(takes, sums, taken), back0 = scan(gives, sums, given);
    const long top = (long)count + given, left = top - taken;
    if (!(flags & 16)) {
        if (left < 0) flags |= 4;
        if (top > a.free_size) flags |= 8;
    }
    const bool ok = flags == 0;
    if (tid == 0) {
        *a.status = flags;
        *a.count_new = ok ? (int)left : count;
    }
    if (ok) {
        long at = count + back0;
        for (int w = w0; w < w1; ++w) {
            for (uint32_t bits = back[w]; bits; bits &= bits - 1, ++at) {
                const int page = w * 32 + __ffs(bits) - 1;
                if (at < left)
                    a.free[at] = page;
                else
                    got[top - 1 - at] = page;
            }
        }
    }
    __syncthreads();
    uint32_t taker = taker0;
    for (int b = b0; b < b1; ++b) {
        int len = 0, from = -1, to = -1, part = 0;
        bool copies = false;
        if (ok) {
            const int r = parent(b, len, copies);
            if (copies) {
                const int c = len / a.page;
                part = len - c * a.page;
                from = a.table[r * a.table_row + c];
                to = taker < given ? got[taker] : a.free[top - 1 - taker];
                a.table_new[b * a.new_row + c] = to;
                ++taker;
            }
        }
        a.lens_new[b] = len;
        a.copies[b] = from;
        a.copies[(long)a.rows + b] = to;
        a.copies[2l * a.rows + b] = part;
    }
}

// LOCAL: packs the sets by itself
template <bool LOCAL> __global__ __launch_bounds__(kLast) void kv_fork_last_kernel(Args a)
{
    __shared__ uint32_t sums[kLast / 64], back[LOCAL ? kLocalWords : 1];
    const int flags = *a.flags;
    if constexpr (LOCAL) {
        for (int w = threadIdx.x; w < a.words; w += kLast) back[w] = bits_of(a.ended + 32l * w, a.kept + 32l * w);
        __syncthreads();
        finish(a, flags, back, a.first, a.got, sums);
    } else {
        finish(a, flags, a.back, a.first, a.got, sums);
    }
}

// All of it, for at most kSmallRows old and new rows each and kSmallPages pages.
__global__ __launch_bounds__(kLast) void kv_fork_small_kernel(Args a)
{
    __shared__ uint32_t sums[kLast / 64], ended[kSmallPages / 32], kept[kSmallPages / 32];
    __shared__ int32_t first[kSmallRows], got[kSmallRows], source[kSmallRows];
    __shared__ int flags;
    const int tid = threadIdx.x;
    for (int w = tid; w < a.words; w += kLast) ended[w] = kept[w] = 0;
    for (int r = tid; r < a.old_rows; r += kLast) first[r] = INT32_MAX;
    if (tid == 0) flags = 0;
    __syncthreads();
    bool bad = false;
    for (int b = tid; b < a.rows; b += kLast) {
        const int r = a.src[b];
        source[b] = r < a.old_rows ? r : -1;
        if (r >= a.old_rows)
            bad = true;
        else if (r >= 0)
            atomicMin(first + r, b);
    }
    for (int r = tid; r < a.old_rows; r += kLast) bad |= bad_length(a, a.lens[r]);
    __syncthreads();
    const int old = a.old_rows * a.width, all = old + a.rows * a.width;
    for (int e = tid; e < all; e += kLast) {
        const bool mark = e < old;
        const int y = (mark ? e : e - old) / a.width, c = (mark ? e : e - old) - y * a.width, r = mark ? y : source[y];
        if (r < 0) continue;
        const int len = a.lens[r];
        if (bad_length(a, len) || c >= pages_of(a, len)) continue;
        const int page = a.table[r * a.table_row + c];
        if (!mark)
            a.table_new[y * a.new_row + c] = page;
        else if ((uint32_t)page >= (uint32_t)a.pages)
            bad = true;
        else
            atomicOr((first[r] == INT32_MAX ? ended : kept) + (page >> 5), 1u << (page & 31));
    }
    if (bad) atomicOr(&flags, 16);
    __syncthreads();
    for (int w = tid; w < a.words; w += kLast) ended[w] &= ~kept[w];
    const int f = flags;
    __syncthreads();
    finish(a, f, ended, first, got, sums);
}

// Copies: grid (blocks of a pair's 16-byte pieces, pairs, layers x (keys, values)).
struct CopyArgs {
    char *k, *v;
    long layer;               // bytes from layer to layer
    const int32_t *copies;
    int n, pages, page, heads, vectors;   // vectors of a token of one head
};

constexpr int kPieces = 4;    // of a thread

__global__ __launch_bounds__(kThreads) void kv_copy_kernel(CopyArgs a)
{
    for (long i = blockIdx.y; i < a.n; i += gridDim.y) {
        const int from = a.copies[i], to = a.copies[(long)a.n + i], rows = min(a.copies[2l * a.n + i], a.page);
        if ((uint32_t)from >= (uint32_t)a.pages || (uint32_t)to >= (uint32_t)a.pages || from == to || rows <= 0) continue;
        const uint32_t per = (uint32_t)rows * a.vectors, all = per * a.heads, whole = (uint32_t)a.page * a.vectors;
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        char *base = (blockIdx.z & 1 ? a.v : a.k) + (blockIdx.z >> 1) * a.layer;
        const char *s = base + (long)from * a.heads * whole * 16;
        char *d = base + (long)to * a.heads * whole * 16;
        for (uint32_t x0 = blockIdx.x * kThreads * kPieces + threadIdx.x; x0 < all; x0 += gridDim.x * kThreads * kPieces) {
            u32x4 y[kPieces];
            long at[kPieces];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const uint32_t x = x0 + j * kThreads, h = x / per;
                at[j] = ((long)h * whole + (x - h * per)) * 16;
                if (x < all) y[j] = *reinterpret_cast<const u32x4 *>(s + at[j]);
            }
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                if (x0 + j * kThreads < all) *reinterpret_cast<u32x4 *>(d + at[j]) = y[j];
        }
    }
}

bool small(const lory_fork_shape &s)
{
    return s.old_rows <= kSmallRows && s.rows <= kSmallRows && s.pages <= kSmallPages &&
           ((long)s.old_rows + s.rows) * s.width <= kSmallEntries;
}

struct Sizes {
    size_t words, bytes, back, first, got, flags;
    explicit Sizes(const lory_fork_shape &s)
        : words(((size_t)s.pages + 31) / 32), bytes(align_up(32 * words, 256)), back(words > kLocalWords ? align_up(4 * words, 256) : 0),
          first(align_up((size_t)s.old_rows * 4, 256)), got(align_up((size_t)s.rows * 4, 256)), flags(256)
    {
    }
    size_t all() const { return 2 * bytes + back + first + got + flags; }
};

}  // namespace

size_t kv_fork_workspace_bytes(const lory_fork_shape &s) { return Sizes(s).all(); }

int kv_fork_launch(const lory_fork_shape &s, const int32_t *lens, const int32_t *src, const int32_t *table, int32_t *free,
                   const int32_t *count, int32_t *lens_new, int32_t *table_new, int32_t *count_new, int32_t *copies,
                   int32_t *status, void *ws, hipStream_t st)
{
    const Sizes z(s);
    char *p = (char *)ws;
    Args a = {lens, src, table, free, count, lens_new, table_new, count_new, copies, status, (long)s.table_row, (long)s.new_row,
              s.old_rows, s.rows, s.width, s.page, s.pages, s.free_size};
    a.ended = (uint8_t *)p;
    a.kept = (uint8_t *)(p += z.bytes);
    a.back = (uint32_t *)(p += z.bytes);
    a.first = (int32_t *)(p += z.back);
    a.got = (int32_t *)(p += z.first);
    a.flags = (int32_t *)(p += z.got);
    a.words = (int)z.words;
    prof::Range r(st, prof::kKvFork, 0.0, 8.0 * s.rows);
    if (small(s)) {
        hipLaunchKernelGGL(kv_fork_small_kernel, dim3(1), dim3(kLast), 0, st, a);
        return launch_status();
    }
    const int groups = (s.old_rows + kFirstRows - 1) / kFirstRows;
    const long clear = (2l * a.words + kLast - 1) / kLast;
    hipLaunchKernelGGL(kv_fork_begin_kernel, dim3((unsigned)(groups + (clear < 512 ? clear : 512))), dim3(kLast), 0, st, a, groups);
    const long rows = (long)s.old_rows + s.rows, columns = ((long)s.width + kThreads - 1) / kThreads;
    if (rows > 0)
        hipLaunchKernelGGL(kv_fork_mark_kernel, dim3((unsigned)(columns < 64 ? columns : 64), (unsigned)(rows < 65535 ? rows : 65535)),
                           dim3(kThreads), 0, st, a);
    if (a.words <= kLocalWords) {
        hipLaunchKernelGGL(kv_fork_last_kernel<true>, dim3(1), dim3(kLast), 0, st, a);
    } else {
        hipLaunchKernelGGL(kv_fork_pack_kernel, dim3((unsigned)((a.words + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(kv_fork_last_kernel<false>, dim3(1), dim3(kLast), 0, st, a);
    }
    return launch_status();
}

int kv_copy_launch(const lory_copy_shape &s, void *k_cache, void *v_cache, const int32_t *copies, hipStream_t st)
{
    const long vectors = (long)s.head_dim * (s.dtype == LORY_F32 ? 4 : 2) / 16, bytes = (long)s.kv_heads * s.page * vectors * 16;
    const CopyArgs a = {(char *)k_cache, (char *)v_cache, bytes * s.pages, copies, s.n, s.pages, s.page, s.kv_heads, (int)vectors};
    const long blocks = (bytes / 16 + kThreads * kPieces - 1) / (kThreads * kPieces);
    prof::Range r(st, prof::kKvCopy, 0.0, 0.0);   // what is copied is on the device
    hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)(s.n < 65535 ? s.n : 65535), 2 * s.layers),
                       dim3(kThreads), 0, st, a);
    return launch_status();
}

}  // namespace lory
