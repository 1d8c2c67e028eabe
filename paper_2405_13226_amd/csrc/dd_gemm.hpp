// dd_gemm.hpp -- what the matrix product kernels share: waits joined with the
// workgroup's barrier, the swizzle of sub-tiles read along rows, and the order
// of the tiles.
#pragma once

#include <algorithm>

#include "dd_device.hpp"

namespace dd {

// Waits until at most N of this wave's vector-memory operations are in
// flight and all its LDS reads have returned, then joins the workgroup's
// barrier.
template <int N>
__device__ __forceinline__ void wait_and_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ void plain_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Chunk swizzle of the sub-tiles that are read along rows: 64 lanes read 16
// consecutive rows at four neighbouring chunks, and the LDS serves them in
// groups of 16 lanes that are not consecutive (lanes 0-3, 12-15, 20-23,
// 24-27 and so on).  With swz<64>, made for 32 rows at two chunks, such a
// read has two-way bank conflicts.
__device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }

// Tile of block `id`.  Workgroups are dispatched round-robin over the 8 XCDs
// (block id % 8), each with its own L2.  XCD x takes every xm-th tile row
// from row x % xm on and one of 8 / xm blocks of columns, in bands of kGR of
// its rows; a band is walked in groups of 32 tiles (one per CU of the XCD),
// each group column by column, so the tiles that run at the same time share
// their A and B panels in one L2.  xm = 0: row by row (tile_rows_step).
constexpr int kGR = 4;

__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int xm, int &tm, int &tn)
{
    if (xm == 0) {
        tm = id / tiles_n;
        tn = id - tm * tiles_n;
        return;
    }
    const int x = id % kXcds, k = id / kXcds;
    const int rows_x = tiles_m / xm, cols_x = tiles_n * xm / kXcds;
    const int band = k / (kGR * cols_x), rem = k - band * kGR * cols_x;
    const int gr = min(kGR, rows_x - band * kGR);  // rows of this band
    const int gc = 32 / gr, grp = rem / (gr * gc), w = rem - grp * gr * gc;
    tm = (band * kGR + w % gr) * xm + x % xm;
    tn = x / xm * cols_x + grp * gc + w / gr;
}

// xm of tile_of: the one whose groups of 32 tiles read the fewest panels per
// tile, of those that divide the tiles evenly (0: none does).  Eight tile rows
// of a weight gradient, taken a row per XCD, read 24 B panels for 24 tiles
// (2048 x 6144, K = 16,384: 430 us); as 4 x 6 tiles per XCD 400 us.
inline int tile_rows_step(int tiles_m, int tiles_n)
{
    int best = 0;
    double least = 0;
    for (int xm = kXcds; xm >= 1; xm /= 2) {
        if (tiles_m % xm || tiles_n * xm % kXcds)
            continue;
        const double gr = std::min(kGR, tiles_m / xm);
        const double gc = std::min(32 / gr, static_cast<double>(tiles_n * xm / kXcds));
        const double panels = (gr + gc) / (gr * gc);
        if (best == 0 || panels < least) {
            best = xm;
            least = panels;
        }
    }
    return best;
}

// A matrix for buffer loads: byte offsets from `p` at which `bytes` or more
// have passed read as zeros, in memory and as direct loads to LDS.  `bytes`
// is capped at kBufferEnd, which so is out of range in every matrix; it is
// beyond the largest tile offset (256 rows of less than 2^23 bytes each).
constexpr uint32_t kBufferEnd = 1u << 31;

__device__ __forceinline__ u32x4 buffer_of(const void *p, long long bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const long long n = bytes < 0 ? 0 : bytes < kBufferEnd ? bytes : kBufferEnd;
    return u32x4{static_cast<uint32_t>(a), static_cast<uint32_t>(a >> 32) & 0xffffu,
                 static_cast<uint32_t>(n), 0x00020000u};
}

// Direct load of 16 bytes per lane, as dma_b128_off (dd_tile.hpp).  The
// descriptor has to come from scalar arithmetic: the hardware does not wait
// for a scalar register that the vector unit has just written.
__device__ __forceinline__ void dma_b128_buf(u32x4 buf, uint32_t off, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(lds_base), "v"(off), "s"(buf)
                 : "m0", "memory");
}

// The same with 4 bytes per lane.
__device__ __forceinline__ void dma_b32_buf(u32x4 buf, uint32_t off, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(lds_base), "v"(off), "s"(buf)
                 : "m0", "memory");
}

// The same value, of which the compiler does not know it: what is formed from
// it stays where it is used, and is not kept in registers around the K loop.
__device__ __forceinline__ int fresh(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

}  // namespace dd
