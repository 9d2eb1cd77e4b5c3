// Index arithmetic of the paged attention, for the host and the device: which page and row a token has, and which range of
// the work is whose.
#pragma once

#include <stdint.h>

#ifndef __HIPCC__
#define LORY_HD inline
#else
#include <hip/hip_runtime.h>
#define LORY_HD __host__ __device__ __forceinline__
#endif

namespace lory {
namespace paged {

// t / page for 0 <= t < 2^31 as t * magic >> shift: magic = ceil(2^shift / page) with shift = 31 + ceil(log2(page)) is at
// most 2^32 - 1, and its excess over 2^shift / page, below 1, times t stays below 2^31 <= 2^shift / page.
struct Divider {
    uint32_t magic;
    int shift, page;
};

inline Divider divider(int page)
{
    int bits = 0;
    while ((1ll << bits) < page) ++bits;
    Divider d;
    d.shift = 31 + bits;
    d.magic = (uint32_t)((((uint64_t)1 << d.shift) + page - 1) / page);
    d.page = page;
    return d;
}

LORY_HD uint32_t quotient(const Divider &d, uint32_t t) { return (uint32_t)(((uint64_t)t * d.magic) >> d.shift); }

// Row of the cache [pages, heads, page] that holds token t, which lies on page number `at`; -1: that is no page of it.
LORY_HD int cache_row(const Divider &d, uint32_t t, int at, int pages, int heads, int head)
{
    return (uint32_t)at < (uint32_t)pages ? (at * heads + head) * d.page + (int)(t - quotient(d, t) * d.page) : -1;
}

// Keys of a wavefront's step that have a page, as bits: its lanes' ballot, in which lanes behind the step's keys (16 of 64 in
// fp32, 32 in bf16) repeat them.
LORY_HD uint32_t all_keys(int keys) { return (uint32_t)(((uint64_t)1 << keys) - 1); }
LORY_HD uint32_t valid_keys(uint64_t ballot, int keys) { return (uint32_t)ballot & all_keys(keys); }

// a / b for 0 <= a, 0 < b; the 64-bit division takes some 150 instructions, the 32-bit one 30.
LORY_HD long quotient64(long a, long b)
{
    return ((uint64_t)(a | b) >> 32) == 0 ? (long)((uint32_t)a / (uint32_t)b) : a / b;
}

// Units of work 0 .. U - 1 in `groups` ranges: range w starts at unit w U / groups, and unit u belongs to the last
// range that starts at or before it.
LORY_HD long range_begin(int w, long U, int groups) { return quotient64((long)w * U, groups); }
LORY_HD int owner(long u, long U, int groups) { return (int)quotient64((u + 1) * groups - 1, U); }

}  // namespace paged
}  // namespace lory
