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
// Alternatives: a wave keeps a list of its largest (logit, lowest index) pairs
// as 64-bit keys and the key of rank k in it; a piece whose largest logit is
// below that one is passed over, which after the first pieces are nearly all.
// Both join over a workgroup's waves, and over the workgroups of a row where
// there are few rows.
//
// Backward: elementwise, each logit read and each gradient written once.
#include "dd_device.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_attn.h"

#include <algorithm>
#include <cfloat>

namespace dd {

namespace {

typedef uint32_t piece16 __attribute__((ext_vector_type(4), aligned(2)));
typedef float piece16f __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kSlack = 10.0f;
constexpr int kList = 128;  // keys of a wave's list: kMaxTop + 64 at most
constexpr int kMaxTop = 64;

// Eight logits from element `at` on, of which those below `end` exist; -inf
// for the others.
__device__ __forceinline__ void load_logits(const uint16_t *x, int at, int end, float (&f)[8])
{
    if (at + 8 <= end) {
        const u32x4 u = *reinterpret_cast<const piece16 *>(x + at);
        unpack8(u, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = at + i < end ? __uint_as_float(static_cast<uint32_t>(x[at + i]) << 16) : -INFINITY;
    }
}
__device__ __forceinline__ void load_logits(const float *x, int at, int end, float (&f)[8])
{
    if (at + 8 <= end) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const piece16f u = *reinterpret_cast<const piece16f *>(x + at + 4 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                f[4 * h + i] = u[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = at + i < end ? x[at + i] : -INFINITY;
    }
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

// A wave's list: `n` keys, of which none is at or below `floor` (its key of
// rank k once there are k).
struct Best {
    uint64_t *keys;
    int n, k;
    uint64_t floor;
    float logit;  // of floor; -inf before
};

// Keeps the k largest keys, in order.
__device__ __forceinline__ void compact(Best &t)
{
    const int lane = threadIdx.x & 63;
    uint64_t mine[kList / 64];
    int rank[kList / 64] = {};
#pragma unroll
    for (int i = 0; i < kList / 64; ++i)
        mine[i] = i * 64 + lane < t.n ? t.keys[i * 64 + lane] : 0u;
    for (int j = 0; j < t.n; ++j) {
        const uint64_t other = t.keys[j];
#pragma unroll
        for (int i = 0; i < kList / 64; ++i)
            rank[i] += other > mine[i] ? 1 : 0;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < kList / 64; ++i)
        if (i * 64 + lane < t.n && rank[i] < t.k)
            t.keys[rank[i]] = mine[i];
    __builtin_amdgcn_wave_barrier();
    if (t.n >= t.k) {
        t.n = t.k;
        t.floor = t.keys[t.k - 1];
        t.logit = key_logit(t.floor);
        if (t.logit != t.logit)
            t.logit = -INFINITY;
    }
}

__device__ __forceinline__ void offer(Best &t, const float (&f)[8], int at, int end)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint64_t key = pair_key(f[i], at + i);
        const bool add = at + i < end && key > t.floor;
        const uint64_t who = __ballot(add);
        if (who == 0)
            continue;
        const int more = __popcll(who);
        if (t.n + more > kList)
            compact(t);
        if (add)
            t.keys[t.n + __popcll(who & ((1ull << lane) - 1))] = key;
        __builtin_amdgcn_wave_barrier();
        t.n += more;
    }
    // a floor as soon as there is one
    if (t.n >= t.k && (t.floor == 0 || t.n > kList - 64))
        compact(t);
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
    __shared__ uint64_t lists[TOP ? NW * kList : 1];
    __shared__ uint64_t tops[TOP ? NW * kMaxTop : 1];
    __shared__ Sums waves[NW];
    __shared__ RowLog row_log;
    const int row = static_cast<int>(blockIdx.x / a.splits);
    const int split = static_cast<int>(blockIdx.x % a.splits);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *x = static_cast<const T *>(a.X) + row * a.ldx;
    // a split's logits, whole pieces of 8
    const long long pieces = (a.V + 7) / 8;
    const int lo = static_cast<int>(pieces * split / a.splits) * 8;
    const int hi = min(static_cast<int>(pieces * (split + 1) / a.splits) * 8, a.V);

    Sums s{-FLT_MAX, 0.f, 0.f};
    Best best{lists + (TOP ? wave * kList : 0), 0, a.top, 0, -INFINITY};
    for (int w0 = lo + wave * 512; w0 < hi; w0 += NT * 8) {
        const int at = w0 + lane * 8;
        float f[8];
        load_logits(x, at, hi, f);
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
        if constexpr (TOP)
            if (__any(!(mx < best.logit)))
                offer(best, f, at, hi);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        s = joined(s, Sums{__shfl_xor(s.m, o), __shfl_xor(s.s, o), __shfl_xor(s.u, o)});
    if (lane == 0)
        waves[wave] = s;
    if constexpr (TOP) {
        compact(best);
        if (lane < a.top)
            tops[wave * a.top + lane] = lane < best.n ? best.keys[lane] : 0;
    }
    __syncthreads();
    const long long part = static_cast<long long>(row) * a.splits + split;
    if (tid == 0) {
        for (int i = 1; i < NW; ++i)
            s = joined(s, waves[i]);
        if (a.splits == 1)
            row_log = finish_row<T>(a, row, s);
        else
            a.part[part] = s;
    }
    if constexpr (TOP) {
        uint64_t *list = a.splits == 1 ? nullptr : a.part_keys + part * a.top;
        if (list && tid < a.top)
            list[tid] = 0;  // a part may have fewer
        __syncthreads();
        rank_keys(a, row, tops, NW * a.top, row_log, list);
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

__device__ __forceinline__ void store_grads(uint16_t *y, int at, int end, const float (&f)[8])
{
    const u32x4 u = pack8f(f);
    if (at + 8 <= end) {
        *reinterpret_cast<piece16 *>(y + at) = u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < end)
                y[at + i] = static_cast<uint16_t>(u[i >> 1] >> 16 * (i & 1));
    }
}
__device__ __forceinline__ void store_grads(float *y, int at, int end, const float (&f)[8])
{
    if (at + 8 <= end) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<piece16f *>(y + at + 4 * h) =
                piece16f{f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < end)
                y[at + i] = f[i];
    }
}

constexpr int kGradPieces = 4;  // of 8 logits per thread

template <typename T>
__global__ void __launch_bounds__(256) logits_grad_kernel(GradRows a)
{
    const int row = static_cast<int>(blockIdx.x / a.blocks);
    const int block = static_cast<int>(blockIdx.x % a.blocks);
    const T *x = static_cast<const T *>(a.X) + row * a.ldx;
    T *y = static_cast<T *>(a.dX) + row * a.lddx;
    const float lse = a.lse[row], h = a.entropy[row];
    const int64_t t = a.targets[row];
    const float g_t = a.g_logp && t >= 0 ? a.g_logp[row] : 0.f;
    const float g_h = a.g_entropy ? a.g_entropy[row] : 0.f;
    const float g_p = (a.g_lse ? a.g_lse[row] : 0.f) - g_t;
    const int64_t given = g_t != 0.f ? t : -1;
    float f[kGradPieces][8];
    const int at0 = (block * kGradPieces * 256 + static_cast<int>(threadIdx.x)) * 8;
#pragma unroll
    for (int k = 0; k < kGradPieces; ++k)
        if (at0 + k * 2048 < a.V)
            load_logits(x, at0 + k * 2048, a.V, f[k]);
#pragma unroll
    for (int k = 0; k < kGradPieces; ++k) {
        const int at = at0 + k * 2048;
        if (at >= a.V)
            return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = f[k][i] - lse, p = fast_exp2(d * kLog2e);
            const float v = p * (g_p - g_h * (fmaxf(d, kFar) + h));
            f[k][i] = at + i == given ? v + g_t : v;
        }
        store_grads(y, at, a.V, f[k]);
    }
}

int split_rows(int rows, int V, int top)
{
    const int most = std::min({kMaxParts, V / 4096, top ? kMaxPartKeys / top : kMaxParts});
    return std::clamp(512 / rows, 1, std::max(most, 1));
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
    hipError_t e = launch_kernel(a.top ? logits_kernel<T, 256, true> : logits_kernel<T, 256, false>,
                                 dim3(static_cast<unsigned>(parts)), dim3(256), st, r);
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
    const hipError_t e = launch_kernel(
        a.f32 ? logits_grad_kernel<float> : logits_grad_kernel<uint16_t>,
        dim3(static_cast<unsigned>(a.rows) * static_cast<unsigned>(blocks)), dim3(256),
        static_cast<hipStream_t>(a.stream), r);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
