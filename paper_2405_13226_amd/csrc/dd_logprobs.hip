// dd_logprobs.hip -- log probabilities of given tokens from logits, with the
// entropy and the most likely alternatives, and the gradient of the logits.
//
// Row x of V logits, given token t:
//   lse  = log sum_j e^x_j            logp = x_t - lse
//   H    = lse - sum_j p_j x_j        p_j  = e^(x_j - lse)
//   dx_j = p_j [(g_lse - g_logp) - g_H (x_j - lse + H)] + g_logp [j = t]
//
// Forward: one pass over the row.  A thread keeps a reference m, s = sum
// e^(x - m) and u = sum e^(x - m) (x - m) in fp32; m follows the largest logit
// only when that passes it by more than kSlack (the sums stay far inside
// fp32's range, and a change of reference costs a branch of the whole wave).
// Alternatives: a thread also keeps its largest logit, the piece of 8 that has
// it, and the largest of its other pieces.  Where k lanes of a wave hold a logit
// of at least c, the row's k largest are no less than c: the largest such c of
// the workgroup's waves is a floor that few logits reach.  The pieces that
// reach it are read once more (one of a thread as a rule; all of them where its
// other pieces reach it too), what is not below the floor goes into a list in
// LDS as 64-bit keys of logit and index, and their ranks are the result.  A
// list that does not fit is found by k passes instead, each for the largest key
// below the last: many equal logits at the floor, or so many masked ones that no
// wave has k lanes with another (the floor is the mask then; 16 x 50,432 with 30
// logits that are not -inf and 8 alternatives 77 us, with 300 of them 13.7).
// Both join over a workgroup's waves, and over the workgroups of a row where
// there are few rows.
//
// Backward: elementwise, each logit read and each gradient written once (rows
// whose lse lies far from zero are read twice, see kNearLse).
//
// Both are bound by the logits' bytes: 1,501 x 50,277 in fp32 with 5 alternatives
// 302 MB in 59 us, 5.1 TB/s; 16,384 x 50,432 in bf16 296 us forward, 5.6 TB/s, and
// 556 back, 5.9 (what the cache still holds of the forward's among it; a copy of
// 2 GiB 4.9).  16 rows with 8 alternatives, 11.7 us, by latency: the sums 5, the
// alternatives 7.
#include "dd_device.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_attn.h"

#include <algorithm>
#include <cfloat>

namespace dd {

namespace {

typedef uint32_t piece16 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float piece16f __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kSlack = 10.0f;
// Keys of a workgroup's list (without a floor there are below 8 k of them).
template <int NT>
constexpr int kList = NT < 256 ? 8 * NT : 2048;
constexpr int kMaxTop = 64;

// Eight logits from element `at` on, of which those below `end` exist; -inf
// for the others.
__device__ __forceinline__ f32x8 load_logits(const uint16_t *x, int at, int end)
{
    f32x8 f;
    if (at + 8 <= end) {
        const bf16x8 u = as_bf16x8(*reinterpret_cast<const piece16 *>(x + at));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = static_cast<float>(u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = at + i < end ? __uint_as_float(static_cast<uint32_t>(x[at + i]) << 16) : -INFINITY;
    }
    return f;
}
__device__ __forceinline__ f32x8 load_logits(const float *x, int at, int end)
{
    f32x8 f;
    if (at + 8 <= end) {
        const piece16f a = *reinterpret_cast<const piece16f *>(x + at);
        const piece16f b = *reinterpret_cast<const piece16f *>(x + at + 4);
        f = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = at + i < end ? x[at + i] : -INFINITY;
    }
    return f;
}
__device__ __forceinline__ float load_logit(const uint16_t *x, long long at)
{
    return __uint_as_float(static_cast<uint32_t>(x[at]) << 16);
}
__device__ __forceinline__ float load_logit(const float *x, long long at) { return x[at]; }

// Running sums of a thread (or of several, joined).  The reference starts at
// the lowest finite number, so differences from it are never infinite minus
// infinite; a difference is bounded where it multiplies (zero times infinity).
struct Sums {
    float m, s, u;
};
constexpr float kFar = -1e30f;

__device__ __forceinline__ void rebase(Sums &a, float m)
{
    const float d = fmaxf(a.m - m, kFar), f = fast_exp2(d * kLog2e);
    a.u = f * fmaf(d, a.s, a.u);
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    rebase(a, m);
    rebase(b, m);
    return Sums{m, a.s + b.s, a.u + b.u};
}

// Pairs in order as keys: larger logits first, then lower indices; a NaN last.
__device__ __forceinline__ uint64_t pair_key(float x, int index)
{
    const uint32_t u = __float_as_uint(x + 0.0f);  // -0 as 0
    const uint32_t k = x != x ? 0u : u >> 31 ? ~u : u | 0x80000000u;
    return static_cast<uint64_t>(k) << 32 | ~static_cast<uint32_t>(index);
}
__device__ __forceinline__ float key_logit(uint64_t key)
{
    const uint32_t k = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : k ? ~k : 0x7fc00000u);
}

// The largest c, of multiples of 2^LOW, that at least k lanes hold a larger or
// equal x than; 0 if none.
template <int LOW>
__device__ __forceinline__ uint32_t wave_floor(uint32_t x, int k)
{
    uint32_t c = 0;
#pragma unroll
    for (int b = 31; b >= LOW; --b)
        if (__popcll(__ballot(x >= (c | 1u << b))) >= k)
            c |= 1u << b;
    return c;
}

struct LogitRows {
    const void *X;
    const int64_t *targets;
    float *logp, *entropy, *lse, *top_logp;
    int64_t *top_ids;
    Sums *part;           // [rows][splits]
    uint64_t *part_keys;  // [rows][splits][top]
    long long ldx;
    int rows, V, top, splits;
};

// A row's outputs from its joined sums (one thread).  Log probabilities are
// formed as (x - m) - log s: the lse, m + log s, is rounded to m's size.
struct RowLog {
    float m, ls;
    __device__ float of(float x) const { return (x - m) - ls; }
};

template <typename T>
__device__ __forceinline__ RowLog finish_row(const LogitRows &a, int row, const Sums &s)
{
    const RowLog l{s.m, logf(s.s)};
    const int64_t t = a.targets[row];
    float lp = 0.f;  // ignored
    if (t >= 0)
        lp = t < a.V ? l.of(load_logit(static_cast<const T *>(a.X) + row * a.ldx, t)) : NAN;
    a.logp[row] = lp;
    a.entropy[row] = l.ls - s.u / s.s;
    a.lse[row] = l.m + l.ls;
    return l;
}

// The `top` largest of a workgroup's n keys (in LDS; none twice, 0 for none),
// in order, to the row's alternatives or, where `list` is given, to a part's.
__device__ __forceinline__ void rank_keys(const LogitRows &a, int row, const uint64_t *keys, int n,
                                          const RowLog &row_log, uint64_t *list)
{
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t key = keys[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j)
            rank += keys[j] > key ? 1 : 0;
        if (key == 0 || rank >= a.top)
            continue;
        if (list) {
            list[rank] = key;
        } else {
            const long long o = static_cast<long long>(row) * a.top + rank;
            a.top_logp[o] = row_log.of(key_logit(key));
            a.top_ids[o] = static_cast<int64_t>(~static_cast<uint32_t>(key));
        }
    }
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT) logits_kernel(LogitRows a)
{
    constexpr int NW = NT / 64;
    __shared__ uint64_t keys[TOP ? kList<NT> : 1];
    __shared__ int some[TOP ? NT : 1], full[TOP ? NT : 1];
    __shared__ Sums waves[NW];
    __shared__ uint32_t floors[NW];
    __shared__ int n_some, n_full, n_keys;
    __shared__ RowLog row_log;
    const int row = static_cast<int>(blockIdx.x / a.splits);
    const int split = static_cast<int>(blockIdx.x % a.splits);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *x = static_cast<const T *>(a.X) + row * a.ldx;
    // a split's logits, whole pieces of 8
    const long long pieces = (a.V + 7) / 8;
    const int lo = static_cast<int>(pieces * split / a.splits) * 8;
    const int hi = min(static_cast<int>(pieces * (split + 1) / a.splits) * 8, a.V);
    if (TOP && tid == 0)
        n_some = n_full = n_keys = 0;

    Sums s{-FLT_MAX, 0.f, 0.f};
    // the largest logit (a NaN if there are none but NaN), its piece, and the
    // largest of the other pieces
    float most = NAN, next = NAN;
    int where = 0;
    auto take = [&](f32x8 f) __attribute__((always_inline)) {
        const float mx = fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])),
                               fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
        if (__any(mx > s.m + kSlack))
            rebase(s, fmaxf(s.m, mx));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = f[i] - s.m, e = fast_exp2(d * kLog2e);
            s.s += e;
            s.u = fmaf(e, fmaxf(d, kFar), s.u);
        }
        return mx;
    };
    auto note = [&](float mx, int at) __attribute__((always_inline)) {
        const bool more = !(mx <= most);
        next = more ? most : fmaxf(next, mx);
        where = more ? at : where;
        most = more ? fmaxf(most, mx) : most;
    };
    // (two pieces of a thread are on their way at once)
    for (int at = lo + tid * 8; at < hi; at += NT * 16) {
        const f32x8 f0 = load_logits(x, at, hi), f1 = load_logits(x, at + NT * 8, hi);
        const float m0 = take(f0), m1 = take(f1);
        if constexpr (TOP) {
            note(m0, at);
            if (at + NT * 8 < hi)
                note(m1, at + NT * 8);
        }
    }
    const uint32_t reach = TOP ? static_cast<uint32_t>(pair_key(most, 0) >> 32) : 0u;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        s = joined(s, Sums{__shfl_xor(s.m, o), __shfl_xor(s.s, o), __shfl_xor(s.u, o)});
    if constexpr (TOP) {
        // (bf16 logits differ in their upper halves only)
        const uint32_t c = wave_floor<sizeof(T) == 2 ? 16 : 0>(reach, a.top);
        if (lane == 0)
            floors[wave] = c;
    }
    if (lane == 0)
        waves[wave] = s;
    __syncthreads();
    const long long part = static_cast<long long>(row) * a.splits + split;
    if (wave == 0) {
        s = waves[lane % NW];
#pragma unroll
        for (int o = NW / 2; o >= 1; o >>= 1)
            s = joined(s, Sums{__shfl_xor(s.m, o), __shfl_xor(s.s, o), __shfl_xor(s.u, o)});
        if (lane == 0) {
            if (a.splits == 1)
                row_log = finish_row<T>(a, row, s);
            else
                a.part[part] = s;
        }
    }
    if constexpr (TOP) {
        uint32_t floor = floors[0];
#pragma unroll
        for (int i = 1; i < NW; ++i)
            floor = max(floor, floors[i]);
        if (lo + tid * 8 < hi && reach >= floor) {
            if (floor == 0 || static_cast<uint32_t>(pair_key(next, 0) >> 32) >= floor)
                full[atomicAdd(&n_full, 1)] = tid;
            else
                some[atomicAdd(&n_some, 1)] = where;
        }
        uint64_t *list = a.splits == 1 ? nullptr : a.part_keys + part * a.top;
        if (list && tid < a.top)
            list[tid] = 0;  // a part may have fewer
        __syncthreads();
        const int steps = (hi - lo + NT * 8 - 1) / (NT * 8);
        for (int i = tid; i < n_some + n_full * steps; i += NT) {
            const int j = i - n_some;
            const int at = j < 0 ? some[i] : lo + (j / n_full * NT + full[j % n_full]) * 8;
            const f32x8 f = load_logits(x, at, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint64_t key = pair_key(f[e], at + e);
                if (at + e < hi && static_cast<uint32_t>(key >> 32) >= floor) {
                    const int k = atomicAdd(&n_keys, 1);
                    if (k < kList<NT>)
                        keys[k] = key;
                }
            }
        }
        __syncthreads();
        int n = n_keys;
        if (n > kList<NT>) {
            // k passes: each thread's largest key below the last, then the row's
            uint64_t last = ~0ull;
            for (n = 0; n < a.top; ++n) {
                uint64_t best = 0;
                for (int at = lo + tid * 8; at < hi; at += NT * 8) {
                    const f32x8 f = load_logits(x, at, hi);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint64_t key = pair_key(f[j], at + j);
                        if (at + j < hi && key < last && key > best)
                            best = key;
                    }
                }
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1) {
                    const uint64_t other = __shfl_xor(static_cast<unsigned long long>(best), o);
                    best = other > best ? other : best;
                }
                __syncthreads();  // the pass before has read
                if (lane == 0)
                    keys[kMaxTop + wave] = best;
                __syncthreads();
                last = keys[kMaxTop];
                for (int i = 1; i < NW; ++i)
                    last = keys[kMaxTop + i] > last ? keys[kMaxTop + i] : last;
                if (tid == 0)
                    keys[n] = last;
            }
            __syncthreads();
        }
        rank_keys(a, row, keys, n, row_log, list);
    }
}

// A row's parts, one workgroup per row.
constexpr int kMaxParts = 64, kMaxPartKeys = 1024;

template <typename T>
__global__ void __launch_bounds__(256) join_logits_kernel(LogitRows a)
{
    __shared__ uint64_t keys[kMaxPartKeys];
    __shared__ RowLog row_log;
    const int row = static_cast<int>(blockIdx.x), tid = threadIdx.x;
    if (tid < 64) {
        const long long part = static_cast<long long>(row) * a.splits;
        Sums s = tid < a.splits ? a.part[part + tid] : Sums{-FLT_MAX, 0.f, 0.f};
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1)
            s = joined(s, Sums{__shfl_xor(s.m, o), __shfl_xor(s.s, o), __shfl_xor(s.u, o)});
        if (tid == 0)
            row_log = finish_row<T>(a, row, s);
    }
    const int n = a.splits * a.top;
    for (int i = tid; i < n; i += 256)
        keys[i] = a.part_keys[static_cast<long long>(row) * n + i];
    __syncthreads();
    if (n)
        rank_keys(a, row, keys, n, row_log, nullptr);
}

// ---------------------------------------------------------------------------

struct GradRows {
    const void *X;
    const int64_t *targets;
    const float *lse, *entropy, *g_logp, *g_entropy, *g_lse;
    void *dX;
    long long ldx, lddx;
    int rows, V, blocks;  // workgroups per row
};

// STREAM: past the caches.
template <bool STREAM, typename V>
__device__ __forceinline__ void store_piece(V *p, V v)
{
    if constexpr (STREAM)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}
template <bool STREAM>
__device__ __forceinline__ void store_grads(uint16_t *y, int at, int end, f32x8 f)
{
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        b[i] = static_cast<__bf16>(f[i]);
    const piece16 u = __builtin_bit_cast(u32x4, b);
    if (at + 8 <= end) {
        store_piece<STREAM>(reinterpret_cast<piece16 *>(y + at), u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < end)
                y[at + i] = static_cast<uint16_t>(u[i >> 1] >> 16 * (i & 1));
    }
}
template <bool STREAM>
__device__ __forceinline__ void store_grads(float *y, int at, int end, f32x8 f)
{
    if (at + 8 <= end) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            store_piece<STREAM>(reinterpret_cast<piece16f *>(y + at + 4 * h),
                                piece16f{f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]});
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < end)
                y[at + i] = f[i];
    }
}

// Gradients past this size leave the last-level cache (256 MB) before anyone
// reads them: they are stored past it (16,384 x 50,432, in turn with the forward:
// 599 us through the cache and 345 for the next forward, past it 579 and 320; rows
// taken from the last one on 566 and 316).
constexpr long long kStreamBytes = 256LL << 20;
constexpr int kGradPieces = 4;  // of 8 logits per thread

// Below this log p there is no p (e^-1000 is 0 in fp32): what multiplies that 0
// stays finite for a g_entropy of up to 1e35.
constexpr float kNone = -1000.0f;

// The lse is rounded to its own size, and every p_j = e^(x_j - lse) carries that
// rounding.  Up to this |lse| it is at most 2^-18 of p.  Beyond it the row's first
// workgroup takes the whole row: S = sum_j e^(x_j - lse), which the rounding moved
// away from 1, then p_j = e^(x_j - lse) / S.  (All of the row is read before any
// of it is written, as the gradient may take the logits' place.  16,384 x 50,432
// by itself, no row and every row beyond it: 626 and 792 us in bf16, 1,272 and
// 1,849 in fp32.)
constexpr float kNearLse = 64.0f;

template <typename T, bool STREAM>
__global__ void __launch_bounds__(256) logits_grad_kernel(GradRows a)
{
    __shared__ float waves[4];
    // from the last row on: what the forward read last is still in the cache
    const int row = a.rows - 1 - static_cast<int>(blockIdx.x / a.blocks);
    const int block = static_cast<int>(blockIdx.x % a.blocks), tid = static_cast<int>(threadIdx.x);
    const T *x = static_cast<const T *>(a.X) + row * a.ldx;
    T *y = static_cast<T *>(a.dX) + row * a.lddx;
    const float lse = a.lse[row], h = a.entropy[row];
    const int64_t t = a.targets[row];
    // (a target of V or more has no log probability: its row becomes NaN)
    const float g_t = a.g_logp && t >= 0 ? (t < a.V ? a.g_logp[row] : NAN) : 0.f;
    const float g_h = a.g_entropy ? a.g_entropy[row] : 0.f;
    const float g_p = (a.g_lse ? a.g_lse[row] : 0.f) - g_t;
    const int64_t given = g_t != 0.f ? t : -1;
    if (fabsf(lse) > kNearLse) {
        if (block)
            return;
        float s = 0.f;
        for (int at = tid * 8; at < a.V; at += 2048) {
            const f32x8 f = load_logits(x, at, a.V);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s += fast_exp2((f[i] - lse) * kLog2e);
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1)
            s += __shfl_xor(s, o);
        if ((tid & 63) == 0)
            waves[tid >> 6] = s;
        __syncthreads();
        s = (waves[0] + waves[1]) + (waves[2] + waves[3]);
        // (half a step of the lse, or little more; further off, the lse is that of a
        // row of which these columns are a part, and counts as it is)
        const float off = logf(s);
        const bool rounding = fabsf(off) <= fabsf(lse) * 0x1p-21f;
        const float scale = rounding ? 1.f / s : 1.f, log_s = rounding ? off : 0.f;
        for (int at = tid * 8; at < a.V; at += 2048) {
            f32x8 f = load_logits(x, at, a.V);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = f[i] - lse, p = fast_exp2(d * kLog2e) * scale;
                const float v = p * (g_p - g_h * (fmaxf(d - log_s, kNone) + h));
                f[i] = at + i == given ? v + g_t : v;
            }
            store_grads<STREAM>(y, at, a.V, f);
        }
        return;
    }
    f32x8 f[kGradPieces];
    const int at0 = (block * kGradPieces * 256 + tid) * 8;
#pragma unroll
    for (int k = 0; k < kGradPieces; ++k)
        if (at0 + k * 2048 < a.V)
            f[k] = load_logits(x, at0 + k * 2048, a.V);
#pragma unroll
    for (int k = 0; k < kGradPieces; ++k) {
        const int at = at0 + k * 2048;
        if (at >= a.V)
            return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = f[k][i] - lse, p = fast_exp2(d * kLog2e);
            const float v = p * (g_p - g_h * (fmaxf(d, kNone) + h));
            f[k][i] = at + i == given ? v + g_t : v;
        }
        store_grads<STREAM>(y, at, a.V, f[k]);
    }
}

// Few long rows: a row is one workgroup of 1024 threads, or several of them where
// it is very long.  Otherwise it is a wave, up to a length that grows with the
// number of rows (a wave takes long over its row, and many rows hide that), or a
// workgroup of 256.  In us with a wave, 256 and 1024 threads, without
// alternatives / with 8:
//      16 x 50,432   31 / 38     11 / 15     7.3 / 11.2
//     512 x 50,432   47 / 55     17 / 20      14 / 18
//     768 x 50,432   49 / 56     19 / 23      18 / 25
//      16 x  1,000  3.3 / 5.6   3.5 / 6.0    3.7 / 6.2
//      16 x  8,000  7.3 / 10.0  4.2 / 7.1    4.8 / 8.3
//   2,048 x  4,000  7.6 / 10.3  7.6 / 11.0    16 / 28
//   2,048 x  8,000   12 / 15     10 / 14      21 / 35
//  16,384 x  1,000   13 / 20     29 / 49
//  16,384 x 16,000  102 / 111   101 / 124
//  16,384 x 24,000  144 / 154   138 / 163
// (16 x 50,432 in 12 parts of 256 threads and a join: 7.4 + 3.6, and a launch.)
constexpr int kFewRows = 512;

int row_threads(int rows, int V)
{
    if (rows <= kFewRows && V > 8192)
        return 1024;
    return V <= std::clamp(2 * rows, 1024, 16384) ? 64 : 256;
}

int split_rows(int rows, int V, int top)
{
    if (rows > kFewRows)
        return 1;
    const int most = std::min(top ? kMaxPartKeys / top : kMaxParts, kFewRows / rows);
    return std::clamp((V + 65535) / 65536, 1, most);
}

template <typename T>
int launch_logprobs_t(const LogprobArgs &a)
{
    const int splits = split_rows(a.rows, a.V, a.top);
    const size_t parts = static_cast<size_t>(a.rows) * splits;
    uint64_t *keys = static_cast<uint64_t *>(a.workspace);
    const LogitRows r{a.X, a.targets, a.logp, a.entropy, a.lse, a.top_logp, a.top_ids,
                      reinterpret_cast<Sums *>(keys + parts * a.top), keys, a.ldx, a.rows, a.V,
                      a.top, splits};
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    const int nt = row_threads(a.rows, a.V);
    auto kern = nt == 1024 ? (a.top ? logits_kernel<T, 1024, true> : logits_kernel<T, 1024, false>)
                : nt == 256 ? (a.top ? logits_kernel<T, 256, true> : logits_kernel<T, 256, false>)
                            : (a.top ? logits_kernel<T, 64, true> : logits_kernel<T, 64, false>);
    hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(parts)),
                                 dim3(static_cast<unsigned>(nt)), st, r);
    if (e == hipSuccess && splits > 1)
        e = launch_kernel(join_logits_kernel<T>, dim3(static_cast<unsigned>(a.rows)), dim3(256), st,
                          r);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace

size_t logprobs_workspace_bytes(int rows, int V, int top)
{
    const int splits = split_rows(rows, V, top);
    return splits == 1 ? 0 : static_cast<size_t>(rows) * splits * (sizeof(Sums) + 8 * top);
}

int launch_logprobs(const LogprobArgs &a)
{
    return a.f32 ? launch_logprobs_t<float>(a) : launch_logprobs_t<uint16_t>(a);
}

int launch_logprobs_bwd(const LogprobBackArgs &a)
{
    const int blocks = (a.V + 2048 * kGradPieces - 1) / (2048 * kGradPieces);
    const GradRows r{a.X, a.targets, a.lse, a.entropy, a.g_logp, a.g_entropy, a.g_lse, a.dX, a.ldx,
                     a.lddx, a.rows, a.V, blocks};
    const bool stream = static_cast<long long>(a.rows) * a.V * (a.f32 ? 4 : 2) > kStreamBytes;
    const hipError_t e = launch_kernel(
        a.f32 ? (stream ? logits_grad_kernel<float, true> : logits_grad_kernel<float, false>)
              : (stream ? logits_grad_kernel<uint16_t, true> : logits_grad_kernel<uint16_t, false>),
        dim3(static_cast<unsigned>(a.rows) * static_cast<unsigned>(blocks)), dim3(256),
        static_cast<hipStream_t>(a.stream), r);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
