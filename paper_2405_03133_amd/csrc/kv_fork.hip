// Rows of a paged cache that go on from other rows (lory_kv_fork), and copies of its pages (lory_kv_copy).
//
// lory_kv_fork is latency-bound: 4 bytes of the table's entries in and out.  Which pages come back needs no counts of
// their owners kept between calls: a page comes back if an old row has it and no new row does, and two bitmaps over the pool say
// that.  One launch clears them; the second copies the tables and sets the bits, with the first child of every old row; the third, one
// workgroup, takes the sums over rows and over words of the bitmaps, gives pages back in the order of their numbers, and hands
// pages to the rows that need one.  A page that comes back goes to the stack or, above its new top, to the row that takes it.
#include "lory_internal.h"

namespace lory {

namespace {

constexpr int kThreads = 256, kLast = 1024;

struct Args {
    const int32_t *lens, *src, *table;
    int32_t *free;
    const int32_t *count;
    int32_t *lens_new, *table_new, *count_new, *copies, *status;
    long table_row, new_row;
    int old_rows, rows, width, page, pages, free_size;
    // workspace
    uint32_t *old_bits, *kept_bits;   // a bit for every page that an old row has, that a new row goes on with
    int32_t *first;                   // first child of every old row
    int32_t *got;                     // pages that come back and are taken again, by taker
    int32_t *flags;
    int words;
};

__device__ __forceinline__ int pages_of(const Args &a, int len)   // of a length inside its limits
{
    return (int)(((uint32_t)len + a.page - 1) / (uint32_t)a.page);
}
__device__ __forceinline__ bool bad_length(const Args &a, int len) { return len < 0 || len > (long)a.width * a.page; }

__global__ __launch_bounds__(kThreads) void kv_fork_clear_kernel(Args a)
{
    const long step = (long)gridDim.x * kThreads, me = (long)blockIdx.x * kThreads + threadIdx.x;
    for (long i = me; i < a.words; i += step) a.old_bits[i] = a.kept_bits[i] = 0;
    for (long i = me; i < a.old_rows; i += step) a.first[i] = INT32_MAX;
    if (me == 0) *a.flags = 0;
}

__device__ __forceinline__ void set_bit(const Args &a, uint32_t *bits, int page)
{
    if ((uint32_t)page >= (uint32_t)a.pages) {
        atomicOr(a.flags, 16);
        return;
    }
    const uint32_t bit = 1u << (page & 31);
    if (!(bits[page >> 5] & bit)) atomicOr(bits + (page >> 5), bit);   // rows share most pages
}

// grid (column blocks, rows): old rows first, then new ones
__global__ __launch_bounds__(kThreads) void kv_fork_mark_kernel(Args a)
{
    const int c0 = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
    for (long y = blockIdx.y; y < (long)a.old_rows + a.rows; y += gridDim.y) {
        const bool old = y < a.old_rows;
        const int row = old ? (int)y : a.src[y - a.old_rows];
        if (!old && row < 0) continue;
        if (row >= a.old_rows) {
            if (c0 == 0) atomicOr(a.flags, 16);
            continue;
        }
        const int len = a.lens[row];
        if (bad_length(a, len)) {
            if (c0 == 0) atomicOr(a.flags, 16);
            continue;
        }
        const int used = pages_of(a, len);
        const int32_t *from = a.table + row * a.table_row;
        if (old) {
            for (int c = c0; c < used; c += step) set_bit(a, a.old_bits, from[c]);
            continue;
        }
        const int b = (int)(y - a.old_rows);
        if (c0 == 0) atomicMin(a.first + row, b);
        int32_t *to = a.table_new + b * a.new_row;
        for (int c = c0; c < used; c += step) {
            const int page = from[c];
            to[c] = page;
            set_bit(a, a.kept_bits, page);
        }
    }
}

// Sum before this thread's and of all; THREADS threads.
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
    for (int w = 0; w < kLast / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    __syncthreads();
    all = total;
    return before + v - own;
}

__global__ __launch_bounds__(kLast) void kv_fork_last_kernel(Args a)
{
    __shared__ uint32_t sums[kLast / 64];
    const int tid = threadIdx.x;
    const int chunk = (a.rows + kLast - 1) / kLast, b0 = min(tid * chunk, a.rows), b1 = min(b0 + chunk, a.rows);
    const int wchunk = (a.words + kLast - 1) / kLast, w0 = min(tid * wchunk, a.words), w1 = min(w0 + wchunk, a.words);
    const int count = *a.count;
    int flags = *a.flags;
    if (count < 0 || count > a.free_size) flags |= 16;

    // the row that b goes on from, or -1; copies: it needs a page of its own
    auto parent = [&](int b, int &len, bool &copies) {
        const int r = a.src[b];
        len = r >= 0 ? a.lens[r] : 0;
        copies = r >= 0 && len % a.page != 0 && a.first[r] != b;
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
        for (int w = w0; w < w1; ++w) gives += __popc(a.old_bits[w] & ~a.kept_bits[w]);
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
            for (uint32_t bits = a.old_bits[w] & ~a.kept_bits[w]; bits; bits &= bits - 1, ++at) {
                const int page = w * 32 + __ffs(bits) - 1;
                if (at < left)
                    a.free[at] = page;
                else
                    a.got[top - 1 - at] = page;
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
                to = taker < given ? a.got[taker] : a.free[top - 1 - taker];
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

struct Sizes {
    size_t bits, first, got, flags;
    explicit Sizes(const lory_fork_shape &s)
        : bits(align_up(((size_t)s.pages + 31) / 32 * 4, 256)), first(align_up((size_t)s.old_rows * 4, 256)),
          got(align_up((size_t)s.rows * 4, 256)), flags(256)
    {
    }
    size_t all() const { return 2 * bits + first + got + flags; }
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
              s.old_rows, s.rows, s.width, s.page, s.pages, s.free_size, (uint32_t *)p, (uint32_t *)(p + z.bits),
              (int32_t *)(p + 2 * z.bits), (int32_t *)(p + 2 * z.bits + z.first), (int32_t *)(p + 2 * z.bits + z.first + z.got),
              (int)((s.pages + 31l) / 32)};
    prof::Range r(st, prof::kKvFork, 0.0, 8.0 * s.rows);
    const long items = a.words > s.old_rows ? a.words : s.old_rows;
    const long clear = (items + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(kv_fork_clear_kernel, dim3((unsigned)(clear < 1 ? 1 : clear < 1024 ? clear : 1024)), dim3(kThreads), 0, st, a);
    const long rows = (long)s.old_rows + s.rows, columns = ((long)s.width + kThreads - 1) / kThreads;
    if (rows > 0)
        hipLaunchKernelGGL(kv_fork_mark_kernel, dim3((unsigned)(columns < 64 ? columns : 64), (unsigned)(rows < 65535 ? rows : 65535)),
                           dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL(kv_fork_last_kernel, dim3(1), dim3(kLast), 0, st, a);
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
