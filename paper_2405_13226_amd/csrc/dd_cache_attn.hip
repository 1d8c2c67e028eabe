// dd_cache_attn.hip -- attention of a ragged chunk of new tokens over a paged
// cache (dd_cache.hpp), and the attention weight of each cached slot.
//
//   O[t, h]   = sum_j p_j V_j,  p = softmax over j <= len + i of q K_j / sqrt(D)
//   W[b, g, j] += sum of p_j over the sequence's new tokens and the heads that
//               share key head g
//
// A sequence's rows for one key head are its new tokens times the G = H / Hkv
// heads that share it, token-major: row r is token r / G, head r % G.  A wave
// holds 32 rows as matrix-core B operands and keeps a running maximum and sum
// (log2 domain, fp32); S^T = K Q^T puts a row in a lane column, P^T stays in
// registers as the B operand of O^T += V^T P^T.  Two kernels differ in who
// reads the keys:
//
//   tile_kernel  many rows: four waves (128 rows) share 64-key tiles,
//                double-buffered in LDS
//   few_kernel   few rows (generation): every wave walks key tiles of its own
//                (32 keys, its own LDS stages, no barrier), the waves' sums are
//                joined through LDS at the end
//
// Either splits the keys over workgroups where there are too few rows to fill
// the chip; finish_kernel adds the parts.  The weights need the rows' final
// sums: where a sequence has few rows their scores are kept (4 bytes a slot and
// row, against 2 D bytes of K), else S is formed once more (weights_kernel).
// Tiles arrive by direct global->LDS loads; one load instruction covers rows of
// one page (pages hold at least 16 slots), whose number is a scalar load.
//
// Few rows are bound by the cache's bytes: 32 sequences of up to 8,192 slots, 16
// heads of 128, a token each: 1,564 MB in 273 us and 5 us for the parts, 5.6 TB/s
// (a copy of 2 GiB: 4.9).  Many by the matrix cores and the exponentials: 4 x 2,048
// tokens over 14,336 slots and each other, 16 heads of 128: 1.03 TFLOP in 1,000 to
// 1,058 us on different cards, 0.97-1.03 PFLOP/s (the library's largest products
// 1.37); matrix cores busy 57% of the time, no LDS conflicts.
//
// Slots behind a sequence's last are never read (a tile's rows are clamped to
// it).  A slot that a row may not see leaves no trace in it, whatever it
// holds: its score is replaced, and where a boundary tile holds values that
// are not finite its keys are added one by one, each only to the rows that see
// it (zero times infinity would not be zero).
#include "dd_cache.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_tile.hpp"
#include "dd_attn.h"

#include <algorithm>
#include <cmath>

namespace dd {

namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

// Rescaling of the accumulator is skipped until the running maximum has grown
// by this many log2 units (probabilities stay below 2^8).
constexpr float kSlack = 8.0f;
constexpr int kMaxSplits = 64;
constexpr size_t kMaxScores = 256UL << 20;  // bytes of scores kept for the weights

struct AttnRows {
    const uint16_t *Q, *K, *V;
    uint16_t *O;
    float *LSE;
    float *part_o, *part_lse;  // [splits][T * H][D], [splits][T * H] (log2), splits > 1
    float *scores;             // [T * H][slots] q K_j, or NULL
    long long ldq;
    int H, G, tiles, splits;
    float scale_log2;
};

template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// One tile of NB x 32 keys for the wave's 32 rows.  MASKED: the lane's row sees
// the tile's keys 0 .. hi_r only (boundary tiles).  `scores` (optional)
// receives the lane's row of q K_j, `room` of them (a multiple of 4).  Where a
// boundary tile holds values that are not finite: EXACT adds its keys one by
// one, each only to the rows that see it; otherwise the result is true, and the
// sums are not to be used.
template <int D, int NB, bool MASKED, bool EXACT, bool SCORES = false>
__device__ __forceinline__ bool
attend_tile(const uint16_t *kt, const uint16_t *vt, const bf16x8 (&qf)[D / 16],
            const int (&koff)[D / 16], const int (&voff)[D / 32][2], int hi_r, int g,
            float scale_log2, f32x16 (&acc)[D / 32], float &m_i, float &l_i,
            float *scores = nullptr, int room = 0)
{
    constexpr int KK = D / 16, DB = D / 32;
    f32x16 s[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
        s[kb] = f32x16{};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
            s[kb] = mfma32(lds_row8(kt + kb * 32 * D + koff[kk]), qf[kk], s[kb]);
    }
    if constexpr (MASKED) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[kb][r] = kb * 32 + 8 * (r >> 2) + (r & 3) <= hi_r - 4 * g ? s[kb][r] : -INFINITY;
    }
    if constexpr (SCORES) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int rg = 0; rg < 4; ++rg)
                if (kb * 32 + 8 * rg + 4 * g < room)
                    *reinterpret_cast<f32x4 *>(scores + kb * 32 + 8 * rg + 4 * g) =
                        f32x4{s[kb][4 * rg], s[kb][4 * rg + 1], s[kb][4 * rg + 2], s[kb][4 * rg + 3]};
    }
    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            m4[r & 3] = fmaxf(m4[r & 3], s[kb][r]);
    const float mc = halves_max(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]))) * scale_log2;
    if (__any(mc > m_i + kSlack)) {
        const float m_new = fmaxf(m_i, mc);
        const float alpha = fast_exp2(m_i - (m_new == -INFINITY ? 0.f : m_new));
        l_i *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            acc[db] *= alpha;
        m_i = m_new;
    }
    // A wave that has its scores goes before one that forms them: two on a SIMD
    // then alternate between the vector unit and the matrix cores (1,000 us instead
    // of 1,095 for 4 x 2,048 tokens over 14,336, 119 instead of 139 for 8 x up to
    // 512 over 4,000; with the products V P alone before the others 1,068 and 130).
    __builtin_amdgcn_s_setprio(1);
    const float neg_m = m_i == -INFINITY ? 0.f : -m_i;
    float psum = 0.f;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = fast_exp2(fmaf(s[kb][r], scale_log2, neg_m));
            s[kb][r] = p;
            psum += p;
        }
    l_i += psum;

    // The one rounding to fewer bits before the output's: the matrix cores take P in
    // V's type, and its roundings, one a key, average out where many keys count
    // (o of one token over 1,024 slots is 0.00164 from float64, relative, and 0.00161
    // if only o itself is rounded; of 4 x 2,048 tokens over 14,336 0.00168 and
    // 0.00167).  The row's sum is of the fp32 values.
    bf16x8 pb[NB][2];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
            pb[kb][t2] = pack8(s[kb], 8 * t2);
    auto value = [&](int kb, int t2, int db) __attribute__((always_inline)) {
        const uint16_t *vr = vt + (kb * 32 + 16 * t2) * D;
        return join(lds_tr4(vr + voff[db][0]), lds_tr4(vr + voff[db][1]));
    };
    if constexpr (MASKED && EXACT) {
        u16x8 top = {};
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const u32x4 a = __builtin_bit_cast(u32x4, value(kb, t2, db)) & 0x7fff7fffu;
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x8, a));
                }
        if (__any(__builtin_reduce_max(top) >= 0x7f80)) {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll 1
                    for (int x = 0; x < 16; ++x) {
                        // slot e of half gx: key 16 t2 + 8 (e / 4) + 4 gx + e % 4
                        const int gx = x >> 3, e = x & 7;
                        const bool sees =
                            kb * 32 + 16 * t2 + 8 * (e >> 2) + 4 * gx + (e & 3) <= hi_r;
                        const uint32_t half = gx == g ? (e & 1 ? 0xffff0000u : 0xffffu) : 0u;
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            u32x4 a = __builtin_bit_cast(u32x4, value(kb, t2, db));
#pragma unroll
                            for (int w = 0; w < 4; ++w)
                                a[w] &= w == e >> 1 ? half : 0u;
                            const f32x16 one = mfma32(as_bf16x8(a), pb[kb][t2], f32x16{});
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                acc[db][r] += sees ? one[r] : 0.f;
                        }
                    }
            __builtin_amdgcn_s_setprio(0);
            return false;
        }
    }
    u16x8 top = {};
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x8 a = value(kb, t2, db);
                if constexpr (MASKED && !EXACT)
                    top = __builtin_elementwise_max(
                        top, __builtin_bit_cast(u16x8, __builtin_bit_cast(u32x4, a) & 0x7fff7fffu));
                acc[db] = mfma32(a, pb[kb][t2], acc[db]);
            }
    __builtin_amdgcn_s_setprio(0);
    return MASKED && !EXACT && __any(__builtin_reduce_max(top) >= 0x7f80);
}

// A work item: BM rows of one sequence and key head, and the part of the key
// tiles (of BN keys) that it takes.
struct AttnItem {
    CacheSeq s;
    int b, h, row, rows;  // first row, rows of the sequence
    int t0, t1;           // key tiles [t0, t1)
    int split;
};

// A value that is the same in every lane, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The sequences' row tiles lie one after the other: those of sequence b start
// at cu[b] G / BM + b, which leaves room for each of its parts of BM rows.
template <int BM, int BN>
__device__ __forceinline__ bool attn_item(const CacheView &c, const AttnRows &a, AttnItem &it)
{
    int h, j;
    block_slice(static_cast<int>(blockIdx.x), a.tiles * a.splits, c.Hkv, h, j);
    it.h = uniform(h);
    j = uniform(j);
    if (it.h >= c.Hkv || j >= a.tiles * a.splits)
        return false;
    const int tile = a.splits == 1 ? j : uniform(j / a.splits);
    it.split = j - tile * a.splits;
    const int from_end = a.tiles - 1 - tile;  // a sequence's last rows see the most keys
    auto first = [&](int b) __attribute__((always_inline)) {
        return static_cast<int>(static_cast<unsigned long long>(cache_cu(c, b)) * a.G / BM) + b;
    };
    int lo = 0, hi = c.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(mid) <= from_end)
            lo = mid;
        else
            hi = mid - 1;
    }
    it.b = lo;
    it.s = cache_seq(c, lo);
    it.rows = it.s.n * a.G;
    it.row = (from_end - first(lo)) * BM;
    if (it.row < 0 || it.row >= it.rows)
        return false;
    const int last = min(it.row + BM, it.rows) - 1;
    const int keys = min(it.s.len + uniform(last / a.G) + 1, it.s.total);
    // (tiles: below 2^25 of them, splits at most 64)
    const int tiles = (keys + BN - 1) / BN;
    it.t0 = a.splits == 1 ? 0 : uniform(static_cast<int>(static_cast<unsigned>(tiles) * it.split / a.splits));
    it.t1 = a.splits == 1
                ? tiles
                : uniform(static_cast<int>(static_cast<unsigned>(tiles) * (it.split + 1) / a.splits));
    return true;
}

// Direct loads of one tile of ROWS slots from slot j0 on, shared by NW waves.
// RPI rows per instruction lie in one page.
template <int D, int ROWS, int NW>
struct PagedTile {
    static constexpr int CPR = D / 8, RPI = 64 / CPR, PER = ROWS / RPI / NW;

    static __device__ __forceinline__ void issue(const CacheView &c, const uint16_t *X, uint16_t *lds,
                                                 const AttnItem &it, int j0, int wave, int lane)
    {
        const int w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave);
        const uint32_t slot0 = lds_base_sgpr(lds) + 1024u * static_cast<uint32_t>(w);
        const int32_t *table = c.table + static_cast<long long>(it.b) * c.per;
        const int lr = lane / CPR;
        const int end = it.s.total - 1;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r0 = (w + NW * k) * RPI;  // row of the tile
            // an instruction behind the last slot reads the last slot's rows
            const int first = __builtin_amdgcn_readfirstlane(min(j0 + r0, end & -RPI));
            const uint32_t id = min(static_cast<uint32_t>(constant(table, first >> c.shift)),
                                    static_cast<uint32_t>(c.pages - 1));
            const uint16_t *base = X + cache_row(c, static_cast<int>(id), it.h, first) * D;
            const int row = min(lr, end - first);
            const int x = (lane % CPR) ^ swz<D>(r0 + lr);
            dma_b128_off(base, static_cast<uint32_t>((row * D + x * 8) * 2), slot0 + 1024u * NW * k);
        }
    }
};

// Row r of the sequence (the last one, where it has fewer) in the outputs: its
// token times H plus its head.
__device__ __forceinline__ long long row_out(const AttnRows &a, const AttnItem &it, int r)
{
    const int last = min(r, it.rows - 1), i = last / a.G;
    return static_cast<long long>(it.s.row0 + i) * a.H + it.h * a.G + last - i * a.G;
}

// The wave's 32 rows from `row` on: its query fragments, and the last slot the
// lane's row sees.  Rows behind the last read the last one's.
template <int D>
__device__ __forceinline__ void load_rows(const AttnRows &a, const AttnItem &it, int row, int l32,
                                          int g, bf16x8 (&qf)[D / 16], int &hi)
{
    const int r = min(row + l32, it.rows - 1), i = r / a.G, h = it.h * a.G + r - i * a.G;
    hi = min(it.s.len + i, it.s.total - 1);
    const uint16_t *src = a.Q + (it.s.row0 + i) * a.ldq + h * D + g * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
        qf[kk] = as_bf16x8(*reinterpret_cast<const u32x4 *>(src + kk * 16));
}

template <int D>
__device__ __forceinline__ void tile_offsets(int lane, int (&koff)[D / 16], int (&voff)[D / 32][2])
{
    const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
        koff[kk] = tile_off<D>(l32, kk * 16 + g * 8);
    const int q = lane >> 4, e = (lane & 15) >> 2, x = lane & 3;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
            voff[db][hh] = tile_off<D>(8 * hh + 4 * g + e, db * 32 + 16 * (q & 1) + 4 * x);
}

// O and the LSE of the lane's row (the sequence's row `row`, if it has that
// many), or a split's part.
template <int D>
__device__ __forceinline__ void store_rows(const CacheView &c, const AttnRows &a, const AttnItem &it,
                                           int row, int g, const f32x16 (&acc)[D / 32],
                                           float m_i, float l_i)
{
    const float l = halves_sum(l_i);
    const bool ok = row < it.rows;
    const long long out = row_out(a, it, row);
    if (a.splits == 1) {
        const float inv = 1.0f / l;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
            store_block_bf16(a.O + out * D + db * 32, acc[db], inv, g, ok);
        if (ok && g == 0)
            a.LSE[out] = (m_i + log2f(l)) * kLn2;
        return;
    }
    const long long at = static_cast<long long>(it.split) * c.T * a.H + out;
    const float inv = l == 0.f ? 0.f : 1.0f / l;  // no key in this part
    if (!ok)
        return;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = acc[db][4 * rg + e] * inv;
            *reinterpret_cast<f32x4 *>(a.part_o + at * D + db * 32 + 8 * rg + 4 * g) = v;
        }
    if (g == 0)
        a.part_lse[at] = m_i + log2f(l);
}

// At D = 64 values that are not finite in a boundary tile make the item start
// over in a loop of its own: within the main one they cost it a wave per SIMD
// (4 x 2,048 tokens over 8,192 slots of 16 heads 341-349 us instead of 370; at
// D = 128 it is the other way round, 1,185 instead of 1,110 over 16,384).
template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) tile_kernel(AttnRows a, CacheView c)
{
    constexpr int BM = 128, BN = 64, TILE = BN * D, KK = D / 16, DB = D / 32;
    constexpr bool EXACT = D == 128;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[4 * TILE];
    AttnItem it;
    if (!attn_item<BM, BN>(c, a, it))
        return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
    const int row = it.row + wave * 32;
    const bool on = __builtin_amdgcn_readfirstlane(row < it.rows);

    bf16x8 qf[KK];
    int hi;
    load_rows<D>(a, it, row, l32, g, qf, hi);
    const int hi_first = __builtin_amdgcn_readlane(hi, 0), hi_last = __builtin_amdgcn_readlane(hi, 31);
    int koff[KK], voff[DB][2];
    tile_offsets<D>(lane, koff, voff);
    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
        acc[db] = f32x16{};
    float m_i = -INFINITY, l_i = 0.f;

    auto issue = [&](int t, uint16_t *stage) __attribute__((always_inline)) {
        PagedTile<D, BN, 4>::issue(c, a.K, stage, it, t * BN, wave, lane);
        PagedTile<D, BN, 4>::issue(c, a.V, stage + TILE, it, t * BN, wave, lane);
    };
    if (it.t0 < it.t1)
        issue(it.t0, lds);
    wait_vmem();
    __syncthreads();
    // The last slot the lane's row sees, formed anew for each boundary tile, as
    // the row's place is for the results: held over the loop they would spill.
    auto place = [&]() __attribute__((always_inline)) {
        int tid = static_cast<int>(threadIdx.x);
        asm volatile("" : "+v"(tid));
        return it.row + (tid >> 6) * 32 + (tid & 31);
    };
    auto last_seen = [&]() __attribute__((always_inline)) {
        return min(it.s.len + min(place(), it.rows - 1) / a.G, it.s.total - 1);
    };
    bool again = false;
    auto step = [&](int t, auto bufc) __attribute__((always_inline)) {
        constexpr int BUF = decltype(bufc)::value;
        const uint16_t *kt = lds + BUF * 2 * TILE;
        if (t + 1 < it.t1)
            issue(t + 1, lds + (1 - BUF) * 2 * TILE);
        const int j0 = t * BN;
        if (on && j0 <= hi_last) {
            if (j0 + BN - 1 <= hi_first)
                attend_tile<D, 2, false, false>(kt, kt + TILE, qf, koff, voff, 0, g, a.scale_log2,
                                                acc, m_i, l_i);
            else
                again |= attend_tile<D, 2, true, EXACT>(kt, kt + TILE, qf, koff, voff,
                                                        last_seen() - j0, g, a.scale_log2, acc, m_i,
                                                        l_i);
        }
        wait_vmem();
        __syncthreads();
    };
    // (the stages as constants: with one body for both 6% slower at 2,048 new
    // tokens over 16,384 slots)
    for (int t = it.t0; t < it.t1; t += 2) {
        step(t, IC<0>{});
        if (t + 1 < it.t1)
            step(t + 1, IC<1>{});
    }
    if constexpr (!EXACT) {
        if (__syncthreads_or(again)) {  // from the start
#pragma unroll
            for (int db = 0; db < DB; ++db)
                acc[db] = f32x16{};
            m_i = -INFINITY;
            l_i = 0.f;
#pragma unroll 1
            for (int t = it.t0; t < it.t1; ++t) {
                issue(t, lds);
                wait_vmem();
                __syncthreads();
#pragma unroll 1
                for (int p = 0; p < 2; ++p) {
                    const uint16_t *kt = lds + p * 32 * D;
                    const int j0 = t * BN + p * 32;
                    if (!on || j0 > hi_last)
                        continue;
                    if (j0 + 31 <= hi_first)
                        attend_tile<D, 1, false, true>(kt, kt + TILE, qf, koff, voff, 0, g,
                                                       a.scale_log2, acc, m_i, l_i);
                    else
                        attend_tile<D, 1, true, true>(kt, kt + TILE, qf, koff, voff,
                                                      last_seen() - j0, g, a.scale_log2, acc, m_i,
                                                      l_i);
                }
                __syncthreads();
            }
        }
    }
    if (on)
        store_rows<D>(c, a, it, place(), g, acc, m_i, l_i);
}

template <int D, int NW, bool SCORES>
__global__ void __launch_bounds__(64 * NW) few_kernel(AttnRows a, CacheView c)
{
    constexpr int BN = 32, TILE = BN * D, KK = D / 16, DB = D / 32;
    constexpr int LOADS = 2 * PagedTile<D, BN, 1>::PER;  // of a tile's K and V
    __shared__ __attribute__((aligned(1024))) uint16_t lds[NW * 4 * TILE];
    AttnItem it;
    if (!attn_item<32, BN>(c, a, it))
        return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
    uint16_t *const mine = lds + wave * 4 * TILE;

    int t = it.t0 + wave;
    auto issue = [&](int at, int buf) __attribute__((always_inline)) {
        uint16_t *stage = mine + buf * 2 * TILE;
        PagedTile<D, BN, 1>::issue(c, a.K, stage, it, at * BN, 0, lane);
        PagedTile<D, BN, 1>::issue(c, a.V, stage + TILE, it, at * BN, 0, lane);
    };
    if (t < it.t1)
        issue(t, 0);
    if (t + NW < it.t1)
        issue(t + NW, 1);

    bf16x8 qf[KK];
    int hi;
    load_rows<D>(a, it, it.row, l32, g, qf, hi);
    const int hi_first = __builtin_amdgcn_readlane(hi, 0);
    int koff[KK], voff[DB][2];
    tile_offsets<D>(lane, koff, voff);
    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
        acc[db] = f32x16{};
    float m_i = -INFINITY, l_i = 0.f;

    float *const scores = SCORES ? a.scores + row_out(a, it, it.row + l32) * c.slots() : nullptr;
    const bool mine_ok = it.row + l32 < it.rows;
    int buf = 0;
    for (; t < it.t1; t += NW, buf ^= 1) {
        if (t + NW < it.t1)
            wait_vm<LOADS>();
        else
            wait_vm<0>();
        const uint16_t *kt = mine + buf * 2 * TILE;
        const int j0 = t * BN;
        const int room = mine_ok ? c.slots() - j0 : 0;
        if (j0 + BN - 1 <= hi_first)
            attend_tile<D, 1, false, true, SCORES>(kt, kt + TILE, qf, koff, voff, 0, g, a.scale_log2,
                                             acc, m_i, l_i, scores + j0, room);
        else
            attend_tile<D, 1, true, true, SCORES>(kt, kt + TILE, qf, koff, voff, hi - j0, g,
                                            a.scale_log2, acc, m_i, l_i, scores + j0, room);
        if (t + 2 * NW < it.t1) {
            // the stage's last reads have returned before it is filled again
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
            issue(t + 2 * NW, buf);
        }
    }

    // The waves' sums on a common maximum, through LDS (every wave is done with
    // its stages): each wave adds up and stores every NW-th piece of 4 values.
    constexpr int NS = 1 + 4 * DB;
    float *x = reinterpret_cast<float *>(lds) + lane * 4;
    __syncthreads();
    float *y = x + wave * NS * 256;
    *reinterpret_cast<f32x4 *>(y) = f32x4{m_i, l_i, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 4 * DB; ++r) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = acc[r >> 2][4 * (r & 3) + e];
        *reinterpret_cast<f32x4 *>(y + (r + 1) * 256) = v;
    }
    __syncthreads();
    float scale[NW], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        scale[w] = x[w * NS * 256];
        m = fmaxf(m, scale[w]);
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        scale[w] = fast_exp2(scale[w] - ref);
        l += scale[w] * x[w * NS * 256 + 1];
    }
    l = halves_sum(l);
    const int row = it.row + l32;
    const bool one = a.splits == 1;
    // (a part without a key of the row has l = 0)
    const float inv = !one && l == 0.f ? 0.f : 1.0f / l;
    const long long out = row_out(a, it, row);
    const long long part = static_cast<long long>(it.split) * c.T * a.H + out;
#pragma unroll
    for (int i = 0; i < 4 * DB / NW; ++i) {
        const int r = wave + i * NW;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w)
            v += scale[w] * *reinterpret_cast<const f32x4 *>(x + (w * NS + r + 1) * 256);
        v *= inv;
        const int at = 8 * r + 4 * g;
        if (row >= it.rows)
            continue;
        if (one)
            *reinterpret_cast<bf16x4 *>(a.O + out * D + at) = pack4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<f32x4 *>(a.part_o + part * D + at) = v;
    }
    if (wave == 0 && g == 0 && row < it.rows) {
        if (one)
            a.LSE[out] = (m + log2f(l)) * kLn2;
        else
            a.part_lse[part] = m + log2f(l);
    }
}

struct WeightRows {
    const uint16_t *Q, *K;
    const float *LSE, *W;
    float *Wout;
    long long ldq;
    int H, G;
    float scale_log2;
};

// Blocks below `joins`: rows' parts on a common maximum, D / 4 lanes per row.
// The others (where scores were kept): the weights of 1024 slots of one key
// head, from its rows' scores; each block forms its rows' sums itself.
template <int D>
__global__ void __launch_bounds__(256) finish_kernel(AttnRows a, WeightRows w, CacheView c, int joins)
{
    constexpr int LANES = D / 4, ROWS = 256 / LANES, SETS = kMaxSplits / LANES;
    constexpr int AT_ONCE = 64;
    __shared__ float lse2[AT_ONCE];
    const long long n = static_cast<long long>(c.T) * a.H;
    if (static_cast<int>(blockIdx.x) < joins) {
        const long long row = static_cast<long long>(blockIdx.x) * ROWS + threadIdx.x / LANES;
        const int x = threadIdx.x % LANES;
        if (row < static_cast<long long>(cache_cu(c, 0)) * a.H ||
            row >= static_cast<long long>(cache_cu(c, c.B)) * a.H)
            return;  // (whole groups of lanes)
        // (the first parts are on their way while the sums are joined)
        constexpr int BATCH = 8;
        f32x4 v[BATCH];
        auto load = [&](int s0) __attribute__((always_inline)) {
            const float *part = a.part_o + row * D + 4 * x;
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                v[i] = *reinterpret_cast<const f32x4 *>(part + min(s0 + i, a.splits - 1) * n * D);
        };
        load(0);
        float ls[SETS], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const int s = i * LANES + x;
            ls[i] = s < a.splits ? a.part_lse[s * n + row] : -INFINITY;
            m = fmaxf(m, ls[i]);
        }
#pragma unroll
        for (int o = LANES / 2; o >= 1; o >>= 1)
            m = fmaxf(m, __shfl_xor(m, o));
        const float ref = m == -INFINITY ? 0.f : m;
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            ls[i] = fast_exp2(ls[i] - ref);
            l += ls[i];
        }
#pragma unroll
        for (int o = LANES / 2; o >= 1; o >>= 1)
            l += __shfl_xor(l, o);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < a.splits; s0 += BATCH) {
            float w = ls[0];  // of the batch's parts, and others
#pragma unroll
            for (int i = 1; i < SETS; ++i)
                w = s0 / LANES == i ? ls[i] : w;
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (s0 + i < a.splits)
                    o += __shfl(w, s0 % LANES + i, LANES) * v[i];
            if (s0 + BATCH < a.splits)
                load(s0 + BATCH);
        }
        const float inv = 1.0f / l;
        const bf16x4 y = pack4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        *reinterpret_cast<u32x2 *>(a.O + row * D + 4 * x) = __builtin_bit_cast(u32x2, y);
        if (x == 0)
            a.LSE[row] = (m + log2f(l)) * kLn2;
        return;
    }
    const int blocks = (c.slots() + 1023) / 1024, id = static_cast<int>(blockIdx.x) - joins;
    const int bh = id / blocks, b = bh / c.Hkv, h = bh % c.Hkv;
    const CacheSeq s = cache_seq(c, b);
    const int key = (id % blocks * 256 + static_cast<int>(threadIdx.x)) * 4;
    if (id % blocks * 1024 >= s.total)
        return;
    const bool in = key < s.total;
    const int rows = s.n * a.G, lane = threadIdx.x & 63;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < rows; r0 += AT_ONCE) {
        __syncthreads();
        for (int r = r0 + (threadIdx.x >> 6); r < min(r0 + AT_ONCE, rows); r += 4) {
            const long long out = static_cast<long long>(s.row0 + r / a.G) * a.H + h * a.G + r % a.G;
            float z;
            if (a.splits == 1) {
                z = a.LSE[out] * kLog2e;
            } else {
                const float p = lane < a.splits ? a.part_lse[lane * n + out] : -INFINITY;
                float m = p;
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1)
                    m = fmaxf(m, __shfl_xor(m, o));
                float l = fast_exp2(p - (m == -INFINITY ? 0.f : m));
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1)
                    l += __shfl_xor(l, o);
                z = m + log2f(l);
            }
            if (lane == 0)
                lse2[r - r0] = z;
        }
        __syncthreads();
        if (in)
#pragma unroll 4
            for (int r = r0; r < min(r0 + AT_ONCE, rows); ++r) {
                const int i = r / a.G, hi = min(s.len + i, s.total - 1);
                const long long out = static_cast<long long>(s.row0 + i) * a.H + h * a.G + r - i * a.G;
                const f32x4 q = *reinterpret_cast<const f32x4 *>(a.scores + out * c.slots() + key);
                const float z = lse2[r - r0];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum[e] += key + e <= hi ? fast_exp2(fmaf(q[e], a.scale_log2, -z)) : 0.f;
            }
    }
    const long long at = static_cast<long long>(bh) * c.slots() + key;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (key + e < s.total)
            w.Wout[at + e] = (key + e < s.len ? w.W[at + e] : 0.f) + sum[e];
}

// ---------------------------------------------------------------------------

// The weights of KB x 128 slots of one key head, from Q and K again (where scores
// would be more to keep): KB x 32 slots per wave, their K rows in registers as B
// operands.  S = Q K^T puts a slot in a lane column, so a slot's sum stays in
// its lane; the sequence's rows pass 32 at a time through LDS, three tiles on
// their way while one is used, and their sums 1024 at a time.
template <int D, int KB>
__global__ void __launch_bounds__(256) weights_kernel(WeightRows a, CacheView c)
{
    constexpr int KK = D / 16, CPR = D / 8, PER = 32 * CPR / 64 / 4, TILE = 32 * D;
    constexpr int STAGES = 4, ROWS = 1024;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[STAGES * TILE];
    __shared__ __attribute__((aligned(16))) float lse2[ROWS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
    const int b = static_cast<int>(blockIdx.y) / c.Hkv, h = static_cast<int>(blockIdx.y) % c.Hkv;
    const CacheSeq s = cache_seq(c, b);
    const int block0 = static_cast<int>(blockIdx.x) * KB * 128;
    const int key0 = block0 + wave * KB * 32;
    if (block0 >= s.total)
        return;
    const int rows = s.n * a.G;
    // the first row that sees a slot
    auto first = [&](int key) __attribute__((always_inline)) {
        return static_cast<int>(min(static_cast<long long>(max(key - s.len, 0)) * a.G,
                                    static_cast<long long>(rows)));
    };
    bf16x8 kf[KB][KK];
    int sees[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const int key = key0 + kb * 32 + l32, at = min(key, s.total - 1);
        const int id = max(cache_page(c, b, at), 0);
        const uint16_t *kp = a.K + cache_row(c, id, h, at) * D + g * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
            kf[kb][kk] = as_bf16x8(*reinterpret_cast<const u32x4 *>(kp + kk * 16));
        sees[kb] = first(key);
    }
    const int wave_first = first(key0), wave_all = first(key0 + KB * 32 - 1);
    const int begin = first(block0) & ~31;

    // The next tile's rows of the lane: their tokens and heads, stepped from tile
    // to tile (divisions cost 7 ragged sequences with 4 heads a key head 2 us of 35).
    // Behind the last token they are rows of that one.
    int token[PER], head[PER];
    const int step_token = 32 / a.G, step_head = 32 - step_token * a.G;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int r = begin + ((wave + 4 * k) * 64 + lane) / CPR;
        token[k] = r / a.G;
        head[k] = r - token[k] * a.G;
    }
    auto issue = [&](int buf) __attribute__((always_inline)) {
        const uint32_t slot = lds_base_sgpr(lds) + static_cast<uint32_t>(buf * TILE * 2 + 1024 * wave);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int q = (wave + 4 * k) * 64 + lane, tr = q / CPR, x = (q % CPR) ^ swz<D>(tr);
            dma_b128(a.Q + (s.row0 + min(token[k], s.n - 1)) * a.ldq + (h * a.G + head[k]) * D +
                         x * 8,
                     slot + 4096u * k);
            head[k] += step_head;
            token[k] += step_token + (head[k] >= a.G ? 1 : 0);
            head[k] -= head[k] >= a.G ? a.G : 0;
        }
    };
    int koff[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
        koff[kk] = tile_off<D>(l32, kk * 16 + g * 8);
    float sum[KB] = {};
    for (int c0 = begin; c0 < rows; c0 += ROWS) {
        const int end = min(c0 + ROWS, rows);
        __syncthreads();  // the sums before have been read
        for (int r = c0 + static_cast<int>(threadIdx.x); r < c0 + ROWS; r += 256) {
            const int i = min(r, rows - 1) / a.G;
            const long long at =
                static_cast<long long>(s.row0 + i) * a.H + h * a.G + min(r, rows - 1) - i * a.G;
            lse2[r - c0] = r < rows ? a.LSE[at] * kLog2e : INFINITY;
        }
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t)
            if (c0 + 32 * t < end)
                issue(t);
        int buf = 0;
        for (int r0 = c0; r0 < end; r0 += 32, buf = (buf + 1) % STAGES) {
            // this tile's loads, and at most two later tiles' outstanding
            if (r0 + 64 < end)
                wait_vm<2 * PER>();
            else if (r0 + 32 < end)
                wait_vm<PER>();
            else
                wait_vm<0>();
            __syncthreads();  // every wave's loads; and the stage before is free
            if (r0 + 32 * (STAGES - 1) < end)
                issue((buf + STAGES - 1) % STAGES);
            if (r0 + 32 <= wave_first)
                continue;
            const uint16_t *qt = lds + buf * TILE;
            f32x16 p[KB] = {};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const bf16x8 q = lds_row8(qt + koff[kk]);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    p[kb] = mfma32(q, kf[kb][kk], p[kb]);
            }
            auto add = [&](auto wholec) __attribute__((always_inline)) {
                constexpr bool WHOLE = decltype(wholec)::value != 0;
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) {
                    const f32x4 z =
                        *reinterpret_cast<const f32x4 *>(&lse2[r0 - c0 + 8 * rg + 4 * g]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int rr = r0 + 8 * rg + 4 * g + e;
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) {
                            const float v = fast_exp2(fmaf(p[kb][4 * rg + e], a.scale_log2, -z[e]));
                            sum[kb] += WHOLE || (rr >= sees[kb] && rr < rows) ? v : 0.f;
                        }
                    }
                }
            };
            if (r0 >= wave_all && r0 + 32 <= rows)
                add(IC<1>{});
            else
                add(IC<0>{});
        }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const float t = halves_sum(sum[kb]);
        const int key = key0 + kb * 32 + l32;
        if (key < s.total && g == 0) {
            const long long at = static_cast<long long>(blockIdx.y) * c.slots() + key;
            a.Wout[at] = (key < s.len ? a.W[at] : 0.f) + t;
        }
    }
}

CacheView view(const CacheShape &c)
{
    return CacheView{c.table, c.lens, c.cu_new, c.T, c.B, c.Hkv, c.pages, c.shift, c.per};
}

// Up to so many rows per sequence on the average go to few_kernel, more to
// tile_kernel.  In us by rows per sequence, few_kernel / tile_kernel, 16 heads of
// 4,096 slots (the last: 8,192):
//            16            24            32            48            96
//   D = 128, 1 sequence
//       19.1 / 20.0               19.7 / 20.3   19.9 / 21.2   32 / 24
//   16   108 / 102     109 / 103   112 / 104     150 / 110     211 / 121
//   32   416 / 363     429 / 364
//   D = 64, 1 sequence
//       14.1 / 15.4               15.1 / 15.6   14.4 / 16.4   19 / 18
//   16    55 / 57       56 / 57     67 / 58       67 / 61      111 / 67
//   32   200 / 194     207 / 228
constexpr int few_rows(int D) { return D == 64 ? 24 : 16; }

// Waves of a workgroup with few rows: 64 KB of LDS, two workgroups per CU.  (At
// D = 128 four waves, one workgroup per CU, read 8 x 8,192 slots of 8 key heads
// in 46-56 us instead of 41-43: nothing runs while a workgroup begins or ends.)
// Twice as many where a sequence's slots are few enough to be one part, which
// saves the launch that joins parts and the memory for them (1,024 slots, 12
// heads of 64: 8.5 us instead of 5.5 + 3.8 in two launches).
template <int D>
constexpr int few_waves = D == 64 ? 4 : 2;
constexpr long long kOnePart = 256 << 10;  // bytes of K and V

// How a call runs: by what the host knows of it (rows, sequences, slots).
struct AttnPlan {
    bool few, scores, wide;
    int tiles, splits;
    size_t rows, part_bytes, bytes;  // of the parts, and of the whole workspace
};

// Parts of a sequence's keys for few rows, `work` of them to be split: the time of
// `work` x p workgroups, 512 at once, is estimated for those p that fill 1, 2, 3
// ... rounds.  Together they read 5.6 TB/s, one alone up to 17 GB/s; a round costs
// a microsecond to begin and end, ragged sequences a quarter of one (within one
// round the others go faster instead), the join a launch and its bytes.  (32 x
// 8,192 slots of 16 heads of 128 in 2, 4, 8 and 16 parts: 314, 293, 281 and 293
// us; 8 sequences and 8 key heads in 4, 8 and 16: 64, 52 and 53; 6 and 8 in 10
// and 11: 43 and 60.)
int few_parts(long long work, long long slots, int D, long long rows)
{
    const int most = static_cast<int>(std::clamp<long long>(slots / 128, 1, kMaxSplits));
    int best = 1;
    double least = 0;
    for (int m = 0; m <= 16; ++m) {
        const int p = static_cast<int>(std::clamp<long long>(512 * m / work, 1, most));
        const long long n = work * p, full = n / 512, rest = n % 512;
        const double bytes = static_cast<double>(slots) * D * 4 / p, round = bytes * 512 / 5.6e6;
        const double us = static_cast<double>(full) * round +
                          (rest ? bytes / std::min(17e3, 5.6e6 / static_cast<double>(rest)) : 0) +
                          (n > 512 ? 0.25 : 0.06) * round + static_cast<double>(full + (rest > 0)) +
                          (p > 1 ? 2 + static_cast<double>(p) * rows * D * 8 / 5.6e6 : 0);
        if (m == 0 || us < least) {
            best = p;
            least = us;
        }
        if (p == most)
            break;
    }
    return best;
}

AttnPlan attn_plan(const CacheShape &c, int H, bool weights)
{
    AttnPlan p;
    const long long rows = static_cast<long long>(c.T) * (H / c.Hkv);
    p.few = rows <= static_cast<long long>(few_rows(c.D)) * c.B;
    const int bm = p.few ? 32 : 128;
    p.tiles = static_cast<int>(rows / bm) + c.B;
    // workgroups with work in them, if the rows are spread evenly
    const long long each = (rows + c.B - 1) / c.B;
    const long long work = std::min<long long>(c.B, c.T) * ((each + bm - 1) / bm) * c.Hkv;
    const long long slots = static_cast<long long>(c.per) << c.shift;
    // Many rows: enough workgroups, of 512 slots or more; at D = 64, where 768 run
    // at once and a part's sums are half as many bytes, two rounds of them where
    // they keep 2,048 slots, for ragged sequences (in us with 1 and 2-3 parts, up to
    // so many new tokens: 3 x 1,399 over 7,053 slots of one key head with 16 124 and
    // 88, 16 x 256 over 8,000 of 16 207 and 156; at D = 128 192 and 179 at best, but
    // 124 and 140, 295 and 342).
    p.wide = p.few && slots * c.D * 4 <= kOnePart && work < 512;
    long long want = std::min(512 / work, slots / 512);
    if (c.D == 64)
        want = std::max(want, std::min((1536 + work / 2) / work, slots / 2048));
    if (p.few && !p.wide)
        want = few_parts(work, slots, c.D, rows);
    p.splits = p.wide ? 1 : static_cast<int>(std::clamp<long long>(want, 1, kMaxSplits));
    p.rows = static_cast<size_t>(c.T) * H;
    p.part_bytes = p.splits == 1 ? 0 : p.splits * p.rows * (c.D + 1) * sizeof(float);
    p.part_bytes = (p.part_bytes + 15) / 16 * 16;
    const size_t score_bytes = p.rows * slots * sizeof(float);
    // Scores are kept where they are at most half of K's bytes, written and read
    // (8 sequences of 8,192 slots, 8 key heads with 4 heads each, a token: 65 us in
    // all, 91 with S formed once more), and where a launch has as many workgroups of
    // 256 as finish_kernel takes (below 2^32 threads, half of them for the joins).
    p.scores = weights && p.few && rows * 8 <= static_cast<long long>(c.D) * c.B &&
               score_bytes <= kMaxScores &&
               static_cast<long long>(c.B) * c.Hkv * ((slots + 1023) / 1024) < 1 << 23;
    p.bytes = p.part_bytes + (p.scores ? score_bytes : 0);
    return p;
}

template <int D>
int launch_attn_d(const CacheAttnArgs &a)
{
    const AttnPlan p = attn_plan(a.c, a.H, a.Wout != nullptr);
    const CacheView c = view(a.c);
    char *ws = static_cast<char *>(a.workspace);
    float *parts = reinterpret_cast<float *>(ws);
    const float scale_log2 = kLog2e / std::sqrt(static_cast<float>(D));
    const AttnRows r{static_cast<const uint16_t *>(a.Q), static_cast<const uint16_t *>(a.Kp),
                     static_cast<const uint16_t *>(a.Vp), static_cast<uint16_t *>(a.O), a.LSE,
                     parts, p.splits > 1 ? parts + p.splits * p.rows * D : nullptr,
                     p.scores ? reinterpret_cast<float *>(ws + p.part_bytes) : nullptr, a.ldq, a.H,
                     a.H / a.c.Hkv, p.tiles, p.splits, scale_log2};
    const WeightRows w{r.Q, r.K, a.LSE, a.W, a.Wout, a.ldq, a.H, r.G, scale_log2};
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    const long long items = static_cast<long long>(p.tiles) * p.splits * a.c.Hkv;
    const unsigned grid = static_cast<unsigned>((items + kXcds - 1) / kXcds * kXcds);
    constexpr int NW = few_waves<D>, WIDE = 2 * NW;
    auto kern = p.scores ? few_kernel<D, NW, true> : few_kernel<D, NW, false>;
    if (p.wide)
        kern = p.scores ? few_kernel<D, WIDE, true> : few_kernel<D, WIDE, false>;
    if (!p.few)
        kern = tile_kernel<D>;
    hipError_t e = launch_kernel(kern, dim3(grid),
                                 dim3(static_cast<unsigned>(p.wide ? 64 * WIDE : p.few ? 64 * NW : 256)),
                                 st, r, c);
    constexpr int ROWS = 256 / (D / 4);
    const unsigned joins = p.splits > 1 ? static_cast<unsigned>((p.rows + ROWS - 1) / ROWS) : 0;
    const unsigned heads = static_cast<unsigned>(a.c.B * a.c.Hkv);
    const unsigned more = p.scores ? heads * static_cast<unsigned>((c.slots() + 1023) / 1024) : 0;
    if (e == hipSuccess && joins + more)
        e = launch_kernel(finish_kernel<D>, dim3(joins + more), dim3(256), st, r, w, c,
                          static_cast<int>(joins));
    if (e == hipSuccess && a.Wout && !p.scores) {
        // 128 slots a workgroup, or 256 where that still fills the chip twice
        // over (7 ragged sequences, 4 key heads, 3,000 slots: 35 against 46 us)
        const unsigned two = static_cast<unsigned>((c.slots() + 255) / 256);
        const bool wide = static_cast<unsigned long long>(two) * heads >= 2048;
        e = launch_kernel(wide ? weights_kernel<D, 2> : weights_kernel<D, 1>,
                          dim3(wide ? two : static_cast<unsigned>((c.slots() + 127) / 128), heads),
                          dim3(256), st, w, c);
    }
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace

size_t cache_attn_workspace_bytes(const CacheShape &c, int H, bool weights)
{
    return attn_plan(c, H, weights).bytes;
}

int launch_cache_attn(const CacheAttnArgs &a)
{
    return a.c.D == 64 ? launch_attn_d<64>(a) : launch_attn_d<128>(a);
}

}  // namespace dd
