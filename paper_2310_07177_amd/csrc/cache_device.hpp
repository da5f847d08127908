// cache_device.hpp -- what the operators on the paged cache share: the place of
// a token, the ancestors of a tree's nodes, rows of bf16 or fp32 values.
#pragma once

#include "osd_device.hpp"
#include "osd_internal.hpp"

namespace osd {

// The page of token j >= 0 of sequence b, and its slot there; -1 outside the
// table or the cache.
__device__ inline int cache_page(const CachePages& c, int b, int j, int* slot) {
    if (j >= c.capacity) return -1;
    const int at = int((uint64_t(uint32_t(j)) * c.magic) >> c.shift);
    *slot = j - at * c.page_size;
    const int page = c.table[int64_t(b) * c.table_len + at];
    return uint32_t(page) < uint32_t(c.pages) ? page : -1;
}

// Byte offset of head 0 of token j, -1 without a place.
__device__ inline int64_t cache_place(const CachePages& c, int b, int j) {
    int slot;
    const int page = cache_page(c, b, j, &slot);
    return page < 0 ? -1 : int64_t(page) * c.page_bytes + int64_t(slot) * c.row_bytes;
}

// Nodes 0 .. n-1 of a tree of at most 64, lane i holding node i: the set of its
// ancestors and itself.  By pointer doubling: after r rounds a lane holds its
// nearest 2^r, six rounds of lane exchanges instead of a walk of up to 63
// dependent steps.  Sets *ok false on an invalid tree.
__device__ inline uint64_t wave_ancestors(const int32_t* parent, int n, bool* ok) {
    const int lane = int(threadIdx.x) & (kWave - 1);
    uint64_t mine = uint64_t(1) << lane;
    if (!parent) {
        *ok = true;
        return mine | (mine - 1);
    }
    int p = lane > 0 && lane < n ? parent[lane] : 0;
    *ok = __ballot(lane > 0 && lane < n && uint32_t(p) >= uint32_t(lane)) == 0;
    p &= kWave - 1;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        mine |= uint64_t(__shfl(static_cast<unsigned long long>(mine), p));
        p = __shfl(p, p);
    }
    return mine;
}

// Whether c new tokens behind a context of len fit a table, n of N given.
__device__ inline bool cache_fits(const CachePages& c, int len, int n, int N) {
    return n >= 0 && n <= N && len <= c.capacity - n;
}

}  // namespace osd
