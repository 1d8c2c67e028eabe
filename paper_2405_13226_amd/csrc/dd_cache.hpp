// dd_cache.hpp -- a paged cache of keys and values on the device: where a
// sequence's slots lie, and which rows of a ragged chunk are whose.
//
// Pages are bf16 [pages][Hkv][page][D] (the slots of one head of a page are
// contiguous); table [B][per] names each sequence's pages in order, so slot j
// of sequence b is row j % page of page table[b][j / page].  Sequence b has
// lens[b] slots in use before a call and the rows cu[b] .. cu[b + 1] - 1 of
// the chunk: its new token i is in slot lens[b] + i and sees the slots up to
// that one.
//
// Everything read from device memory is clamped before it forms an address:
// malformed contents give unspecified results, never an access outside the
// tensors.
#pragma once

#include "dd_device.hpp"

namespace dd {

struct CacheView {
    const int32_t *table, *lens, *cu;
    int T, B, Hkv, pages, shift, per;  // page = 1 << shift slots

    __host__ __device__ int page() const { return 1 << shift; }
    __host__ __device__ int slots() const { return per << shift; }  // of a sequence, < 2^30
};

// A sequence: its first row in the chunk, its new tokens, the slots in use
// before the call and with the new tokens (those that have a slot).
struct CacheSeq {
    int row0, n, len, total;
};

// An element of an array that the kernel only reads: a scalar load where the
// index is the same in all lanes.
__device__ __forceinline__ int constant(const int32_t *p, long long i)
{
    typedef const __attribute__((address_space(4))) int32_t *pointer;
    return ((pointer)(p))[i];
}

__device__ __forceinline__ int cache_cu(const CacheView &c, int b)
{
    return min(max(constant(c.cu, b), 0), c.T);
}

__device__ __forceinline__ CacheSeq cache_seq(const CacheView &c, int b)
{
    CacheSeq s;
    s.row0 = cache_cu(c, b);
    s.n = max(cache_cu(c, b + 1) - s.row0, 0);
    s.len = min(max(constant(c.lens, b), 0), c.slots());
    s.total = min(s.len + s.n, c.slots());
    return s;
}

// The sequence of row t of the chunk: the last b with cu[b] <= t.
__device__ __forceinline__ int cache_seq_of(const CacheView &c, int t)
{
    int lo = 0, hi = c.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (constant(c.cu, mid) <= t)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// The page of a slot, or -1 where the table names none.
__device__ __forceinline__ int cache_page(const CacheView &c, int b, int slot)
{
    const int id = constant(c.table, static_cast<long long>(b) * c.per + (slot >> c.shift));
    return id >= 0 && id < c.pages ? id : -1;
}

// Row (in units of D elements) of a slot of head h in page `id`.
__device__ __forceinline__ long long cache_row(const CacheView &c, int id, int h, int slot)
{
    return ((static_cast<long long>(id) * c.Hkv + h) << c.shift) + (slot & (c.page() - 1));
}

}  // namespace dd
