// dd_cache.hip -- writing and thinning out a paged cache (dd_cache.hpp).
//
// Append: a ragged chunk's keys and values into their slots, keys (and the
// chunk's queries) rotated at their positions (dd_rope.hpp: bit-identical to a
// dd_rope pass at these positions).  One workgroup per token: thread t holds
// the 8-element chunk t % (D/8) of its heads, so an angle is formed once per
// token and thread.  Bytes only: each row is read and written once (24,863 tokens
// of 16 heads of 128 with their queries: 611 MB in 115 us, 5.3 TB/s; a copy of
// 2 GiB reaches 4.9).
//
// Eviction: per sequence and key head, the `budget` slots of most weight stay
// (slots of the last `recent` positions before all others; equal ones by the
// lowest slot).  Attention does not depend on the order of the slots, keys
// carry their rotation, and every kept slot is older than any later token, so
// nothing is shifted: the n-th evicted slot below the budget receives the n-th
// kept slot behind it.  Sources and targets are disjoint, so rows move in any
// order, and no more of them than the result needs.
//   select: one workgroup per (sequence, head) finds the weight of rank
//           `budget` by three histograms of 11, 11 and 10 bits of the ordered
//           weights, then lists holes and survivors in slot order.  A thread
//           holds 16 consecutive slots in registers: the weights are read once,
//           and a prefix sum over the workgroup orders equal ones, another the
//           lists.  (Beyond 16,384 slots per sequence they are read again for
//           each histogram and for the lists.)
//   move:   the listed rows (by the workgroup that found them, where they are
//           few: one launch, no memory for the lists)
// 16 sequences of 8,192 slots, 16 heads of 128, thinned out to 4,096: 17 us for
// the lists, bound by the latency of three histograms and two prefix sums, and 87
// for the rows, 4.6 TB/s (a copy 4.9; pieces of 256 bytes at random).
#include "dd_cache.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_rope.hpp"
#include "dd_attn.h"

#include <algorithm>

namespace dd {

namespace {

struct AppendRows {
    const uint16_t *Q, *K, *V;
    uint16_t *Qrot, *Kp, *Vp;
    int32_t *P;
    const int32_t *start;
    long long ldq, ldk, ldv;
    int H;
};

template <int D, bool ROPE>
__global__ void __launch_bounds__(256)
append_kernel(AppendRows a, CacheView c, RopeEpi rt)
{
    constexpr int CG = D / 8, ROWS = 256 / CG;
    const int t = static_cast<int>(blockIdx.x);
    const int cg = threadIdx.x % CG, r0 = threadIdx.x / CG;
    const int b = cache_seq_of(c, t);
    const CacheSeq s = cache_seq(c, b);
    const int i = t - s.row0;
    if (i < 0 || i >= s.n)  // behind the last sequence
        return;
    const int slot = s.len + i;
    const int pos = (a.start ? a.start[b] : s.len) + i;
    const int id = slot < c.slots() ? cache_page(c, b, slot) : -1;

    float sn[4], cs[4];
    if constexpr (ROPE) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            rope_sincos(rope_theta_j(rt, cg * 4 + e), pos, sn[e], cs[e]);
    }
    auto rotated = [&](u32x4 u) __attribute__((always_inline)) {
        if constexpr (ROPE) {
            float f[8];
            unpack8(u, f);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                rope_pair<false>(f[2 * e], f[2 * e + 1], sn[e], cs[e]);
            u = pack8f(f);
        }
        return u;
    };
    if (a.Q != nullptr) {
        const uint16_t *q = a.Q + t * a.ldq + cg * 8;
        uint16_t *y = a.Qrot + static_cast<long long>(t) * a.H * D + cg * 8;
        for (int h = r0; h < a.H; h += ROWS)
            *reinterpret_cast<u32x4 *>(y + h * D) =
                rotated(*reinterpret_cast<const u32x4 *>(q + h * D));
    }
    if (id < 0)
        return;
    const uint16_t *k = a.K + t * a.ldk + cg * 8, *v = a.V + t * a.ldv + cg * 8;
    for (int h = r0; h < c.Hkv; h += ROWS) {
        const long long at = cache_row(c, id, h, slot) * D + cg * 8;
        const u32x4 kh = *reinterpret_cast<const u32x4 *>(k + h * D);
        const u32x4 vh = *reinterpret_cast<const u32x4 *>(v + h * D);
        *reinterpret_cast<u32x4 *>(a.Kp + at) = rotated(kh);
        *reinterpret_cast<u32x4 *>(a.Vp + at) = vh;
        if (a.P != nullptr && cg == 0)
            a.P[(static_cast<long long>(b) * c.Hkv + h) * c.slots() + slot] = pos;
    }
}

template <int D>
int launch_append_d(const CacheAppendArgs &a)
{
    const AppendRows r{static_cast<const uint16_t *>(a.Q), static_cast<const uint16_t *>(a.K),
                       static_cast<const uint16_t *>(a.V), static_cast<uint16_t *>(a.Qrot),
                       static_cast<uint16_t *>(a.Kp), static_cast<uint16_t *>(a.Vp), a.P, a.start,
                       a.ldq, a.ldk, a.ldv, a.H};
    const CacheView c{a.c.table, a.c.lens, a.c.cu_new, a.c.T, a.c.B, a.c.Hkv, a.c.pages,
                      a.c.shift, a.c.per};
    const bool rope = a.rope_base > 0.0;
    const hipError_t e = launch_kernel(
        rope ? append_kernel<D, true> : append_kernel<D, false>, dim3(static_cast<unsigned>(a.c.T)),
        dim3(256), static_cast<hipStream_t>(a.stream), r, c,
        rope ? rope_epi(a.rope_base, D) : RopeEpi{});
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

// ---------------------------------------------------------------------------

struct EvictRows {
    const float *W;
    const int32_t *P, *seen;
    float *Wout;
    int32_t *Pout, *lens_out;
    int32_t *count;     // [B * Hkv] rows to move
    int32_t *to, *from; // [B * Hkv][list] their targets and sources
    uint16_t *Kp, *Vp;
    int budget, recent, list;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// Weights in order as unsigned numbers: a NaN below all, the slots that stay
// in any case above all.
__device__ __forceinline__ uint32_t weight_key(float w, bool stays)
{
    const uint32_t u = __float_as_uint(w + 0.0f);  // -0 as 0
    const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
    return stays ? 0xffffffffu : w != w ? 0u : k;
}

// Exclusive prefix sum of x over the workgroup's NT threads, and its total.
template <int NT>
__device__ __forceinline__ uint32_t block_prefix(uint32_t x, uint32_t *waves, uint32_t &total)
{
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(static_cast<int>(s), o);
        s += lane >= o ? y : 0u;
    }
    __syncthreads();  // `waves` of the call before have been read
    if (lane == 63)
        waves[wave] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const uint32_t w = waves[i];
        before += i < wave ? w : 0u;
        all += w;
    }
    total = all;
    return before + s - x;
}

// Entries of a list that stays in LDS, for the workgroup that made it to move the
// rows.  (12 heads of 1,100 slots, up to 100 of them moved: 9.4 us, 8.6 + 4.0 in
// two launches; with longer lists one workgroup per head moves too slowly.)
constexpr int kFewMoves = 512;

// Moves rows r0, r0 + step, ... of n: row to[r] receives row from[r].
template <int D>
__device__ __forceinline__ void move_rows(const EvictRows &a, const CacheView &c, int bh,
                                          const int32_t *to, const int32_t *from, int n, int r0,
                                          int step)
{
    const int b = bh / c.Hkv, h = bh % c.Hkv, cg = threadIdx.x % (D / 8);
    const long long base = static_cast<long long>(bh) * c.slots();
    for (int r = r0; r < n; r += step) {
        const int d = to[r], s = from[r];
        const int pd = cache_page(c, b, d), ps = cache_page(c, b, s);
        if (pd >= 0 && ps >= 0) {
            const long long rd = cache_row(c, pd, h, d) * D + cg * 8;
            const long long rs = cache_row(c, ps, h, s) * D + cg * 8;
            const u32x4 k = *reinterpret_cast<const u32x4 *>(a.Kp + rs);
            const u32x4 v = *reinterpret_cast<const u32x4 *>(a.Vp + rs);
            *reinterpret_cast<u32x4 *>(a.Kp + rd) = k;
            *reinterpret_cast<u32x4 *>(a.Vp + rd) = v;
        }
        if (cg == 0) {
            a.Wout[base + d] = a.W[base + s];
            a.Pout[base + d] = a.P[base + s];
        }
    }
}

// A thread holds HELD consecutive slots; ONE: the sequence's slots are at most
// NT * HELD.  MOVE (D, or 0): the workgroup moves its rows too; lens_out is not
// lens then (other heads' workgroups still read that).
template <int NT, int HELD, bool ONE, int MOVE = 0>
__global__ void __launch_bounds__(NT) select_kernel(EvictRows a, CacheView c)
{
    constexpr int BINS = 2048, SPAN = NT * HELD;
    __shared__ uint32_t hist[BINS];
    __shared__ uint32_t waves[NT / 64];
    __shared__ uint32_t found[2];
    __shared__ int32_t lists[MOVE ? 2 * kFewMoves : 1];
    const int bh = static_cast<int>(blockIdx.x), b = bh / c.Hkv, tid = threadIdx.x;
    const int n = min(max(c.lens[b], 0), c.slots());
    const long long base = static_cast<long long>(bh) * c.slots();
    const float *W = a.W + base;
    const int32_t *P = a.P + base;
    float *Wout = a.Wout + base;
    int32_t *Pout = a.Pout + base;
    if (MOVE && tid == 0 && bh % c.Hkv == 0)
        a.lens_out[b] = min(n, a.budget);
    if (n <= a.budget) {
        if (!MOVE && tid == 0)
            a.count[bh] = 0;
        if (Wout != W || Pout != P)
            for (int j = tid; j < min(a.budget, c.slots()); j += NT) {
                Wout[j] = W[j];
                Pout[j] = P[j];
            }
        return;
    }
    // the first position that stays in any case (or the lowest number)
    const int first = static_cast<int>(
        max(static_cast<long long>(a.seen[b]) - a.recent, static_cast<long long>(INT32_MIN)));
    const bool copy = Wout != W || Pout != P;

    // The keys of the thread's slots from j0 on; those below the budget are
    // copied on the way (evicted ones are written over by the moves).
    uint32_t key[HELD];
    auto load = [&](int j0, bool keep) __attribute__((always_inline)) {
        f32x4_any w[HELD / 4];
        i32x4_any p[HELD / 4];
#pragma unroll
        for (int q = 0; q < HELD / 4; ++q) {  // (slots: a multiple of 16)
            const int j = min(j0 + 4 * q, c.slots() - 4);
            w[q] = *reinterpret_cast<const f32x4_any *>(W + j);
            p[q] = *reinterpret_cast<const i32x4_any *>(P + j);
        }
#pragma unroll
        for (int q = 0; q < HELD / 4; ++q) {
            const int j = j0 + 4 * q;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                key[4 * q + e] = weight_key(w[q][e], p[q][e] >= first);
            if (!keep)
                continue;
            if (j + 4 <= a.budget) {
                *reinterpret_cast<f32x4_any *>(Wout + j) = w[q];
                *reinterpret_cast<i32x4_any *>(Pout + j) = p[q];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < a.budget) {
                        Wout[j + e] = w[q][e];
                        Pout[j + e] = p[q][e];
                    }
            }
        }
    };

    // The key of rank `budget` (counted from the largest), from its leading
    // bits on, and how many keys equal to it stay.
    uint32_t prefix = 0, need = static_cast<uint32_t>(a.budget);
    if (ONE && tid * HELD < n)
        load(tid * HELD, copy);
#pragma unroll
    for (int part = 0; part < 3; ++part) {
        const int low = part == 0 ? 21 : part == 1 ? 10 : 0, bits = part == 2 ? 10 : 11;
        const uint32_t mask = (1u << bits) - 1;
        for (int i = tid; i < BINS; i += NT)
            hist[i] = 0;
        __syncthreads();
        for (int j0 = tid * HELD; j0 < n; j0 += SPAN) {
            if constexpr (!ONE)
                load(j0, false);
#pragma unroll
            for (int e = 0; e < HELD; ++e)
                if (j0 + e < n && (part == 0 || key[e] >> (low + bits) == prefix))
                    atomicAdd(&hist[(key[e] >> low) & mask], 1u);
        }
        __syncthreads();
        // bins from the largest key down, some per thread
        constexpr int EACH = BINS / NT;
        uint32_t h[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            h[i] = hist[BINS - 1 - tid * EACH - i];
            sum += h[i];
        }
        uint32_t all, above = block_prefix<NT>(sum, waves, all);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (above < need && need <= above + h[i]) {
                found[0] = BINS - 1 - tid * EACH - i;
                found[1] = need - above;
            }
            above += h[i];
        }
        __syncthreads();
        prefix = prefix << bits | found[0];
        need = found[1];
        __syncthreads();
    }

    // Holes and survivors in slot order.
    int32_t *to = MOVE ? lists : a.to + static_cast<long long>(bh) * a.list;
    int32_t *from = MOVE ? lists + kFewMoves : a.from + static_cast<long long>(bh) * a.list;
    uint32_t equal = 0, holes = 0, extra = 0;  // so far
    for (int s0 = 0; s0 < n; s0 += SPAN) {
        const int j0 = s0 + tid * HELD;
        if constexpr (!ONE)
            load(min(j0, c.slots() - HELD), copy && j0 < n);
        uint32_t eq = 0, all;
        if (j0 < n)
#pragma unroll
            for (int e = 0; e < HELD; ++e)
                eq += j0 + e < n && key[e] == prefix ? 1u : 0u;
        uint32_t before = equal + block_prefix<NT>(eq, waves, all);
        equal += all;
        uint32_t hole = 0, moved = 0;  // bits of the thread's slots
        if (j0 < n) {
            uint32_t keep = 0;
#pragma unroll
            for (int e = 0; e < HELD; ++e) {
                const bool same = key[e] == prefix;
                keep |= (key[e] > prefix || (same && before < need) ? 1u : 0u) << e;
                before += same ? 1u : 0u;
            }
            auto below = [&](int end) __attribute__((always_inline)) {
                return (1u << min(max(end - j0, 0), HELD)) - 1;
            };
            hole = ~keep & below(a.budget);  // (the budget is below n)
            moved = keep & below(n) & ~below(a.budget);
        }
        // (of either at most SPAN <= 2^14 in a step)
        const uint32_t place =
            block_prefix<NT>(__popc(hole) | __popc(moved) << 16, waves, all);
        uint32_t at = holes + (place & 0xffffu);
        for (; hole; hole &= hole - 1)
            to[at++] = j0 + __ffs(hole) - 1;
        at = extra + (place >> 16);
        for (; moved; moved &= moved - 1)
            from[at++] = j0 + __ffs(moved) - 1;
        holes += all & 0xffffu;
        extra += all >> 16;
    }
    if constexpr (MOVE != 0) {
        // (the barrier also orders the copies of evicted weights before the moves)
        __syncthreads();
        move_rows<MOVE>(a, c, bh, to, from, static_cast<int>(holes), tid / (MOVE / 8), NT / (MOVE / 8));
    } else if (tid == 0) {
        a.count[bh] = static_cast<int>(holes);
    }
}

template <int D>
__global__ void __launch_bounds__(256) move_kernel(EvictRows a, CacheView c)
{
    constexpr int ROWS = 256 / (D / 8);
    const int bh = static_cast<int>(blockIdx.y), b = bh / c.Hkv;
    if (blockIdx.x == 0 && bh % c.Hkv == 0 && threadIdx.x == 0)
        a.lens_out[b] = min(min(max(c.lens[b], 0), c.slots()), a.budget);
    const long long list = static_cast<long long>(bh) * a.list;
    move_rows<D>(a, c, bh, a.to + list, a.from + list, a.count[bh],
                 static_cast<int>(blockIdx.x) * ROWS + threadIdx.x / (D / 8),
                 static_cast<int>(gridDim.x) * ROWS);
}

// Entries of a list: holes lie below the budget, survivors behind it.
int evict_list(const CacheShape &c, int budget)
{
    return std::max(std::min(budget, (c.per << c.shift) - budget), 0);
}

// As many threads as hold the sequence's slots, where that is possible.
template <int MOVE>
hipError_t launch_select(const EvictRows &r, const CacheView &c, hipStream_t st)
{
    const int slots = c.slots();
    auto kern = select_kernel<1024, 16, false, MOVE>;
    if (slots <= 2048)
        kern = select_kernel<256, 8, true, MOVE>;
    else if (slots <= 8192)
        kern = select_kernel<1024, 8, true, MOVE>;
    else if (slots <= 16384)
        kern = select_kernel<1024, 16, true, MOVE>;
    return launch_kernel(kern, dim3(static_cast<unsigned>(c.B * c.Hkv)),
                         dim3(slots <= 2048 ? 256u : 1024u), st, r, c);
}

}  // namespace

int launch_cache_append(const CacheAppendArgs &a)
{
    return a.c.D == 64 ? launch_append_d<64>(a) : launch_append_d<128>(a);
}

size_t cache_evict_workspace_bytes(const CacheShape &c, int budget, bool in_place)
{
    if (evict_list(c, budget) <= kFewMoves && !in_place)
        return 0;
    return static_cast<size_t>(c.B) * c.Hkv * (1 + 2 * static_cast<size_t>(evict_list(c, budget))) *
           sizeof(int32_t);
}

int launch_cache_evict(const CacheEvictArgs &a)
{
    const CacheView c{a.c.table, a.c.lens, nullptr, 0, a.c.B, a.c.Hkv, a.c.pages, a.c.shift,
                      a.c.per};
    const int bh = a.c.B * a.c.Hkv, list = evict_list(a.c, a.budget);
    int32_t *ws = static_cast<int32_t *>(a.workspace);
    const EvictRows r{a.W, a.P, a.seen, a.Wout, a.Pout, a.lens_out, ws, ws + bh,
                      ws + bh + static_cast<size_t>(bh) * list, static_cast<uint16_t *>(a.Kp),
                      static_cast<uint16_t *>(a.Vp), a.budget, a.recent, list};
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    if (list <= kFewMoves && a.lens_out != a.c.lens) {
        const bool narrow = a.c.D == 64;
        const hipError_t e = narrow ? launch_select<64>(r, c, st) : launch_select<128>(r, c, st);
        return e == hipSuccess ? DD_OK : DD_ERR_HIP;
    }
    hipError_t e = launch_select<0>(r, c, st);
    if (e != hipSuccess)
        return DD_ERR_HIP;
    const int rows = 256 / (a.c.D / 8);
    const unsigned parts = static_cast<unsigned>(std::clamp((list + 4 * rows - 1) / (4 * rows), 1, 64));
    e = launch_kernel(a.c.D == 64 ? move_kernel<64> : move_kernel<128>,
                      dim3(parts, static_cast<unsigned>(bh)), dim3(256), st, r, c);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
