// dd_rms.hip -- rows into 8 bits: RMSNorm (with the residual's addition, its
// output in bf16 or as codes, and its backward), and the codes of any matrix's
// rows and back.  All are passes over [rows, d] tensors with fp32 arithmetic,
// bound by HBM, or at a few rows by latency.
//
// RMSNorm:   h = bf16(x + r), rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd w.
// Codes:     a row z with largest magnitude A is held as int8 codes
//            q = the integer nearest to 127 z / A (ties to even) and one fp32
//            scale; the row's values are scale q.
// For the norm's codes z = h w: rstd cancels out of the codes, so they need no
// sum over the row, and h w is exact in fp32 (two 8-bit significands) unless it
// leaves fp32's range: rows with A outside 2^-60 .. 2^60 take it in fp64.  The
// scale is A rstd / 127.
//
// Backward, with xh = h rstd and g = dy w:
//            dx = rstd (g - xh mean(g xh)) (+ dres),  dw = sum over rows dy xh.
//
// 65,536 x 2048, us (TB/s; a plain copy's rate is 4.8): norm with a residual 188
// (5.7), with codes 167-172 (5.6), backward 215-217 (5.0), quantizing 75 call after
// call (5.4) and 65 after other kernels (6.2), dequantizing 70 (5.8).  One row of
// 2048: 2.3, 2.8 with codes.
#include "dd_device.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_attn.h"

#include <algorithm>

namespace dd {

namespace {

enum RowKind { kNorm, kNormCodes, kCodes };

// Row `row` of a matrix belongs to TPR threads of a workgroup: a wave or a part
// of one (several rows per workgroup of 256 threads), or a whole workgroup of
// 256 or 1024.  Thread t holds the 8-element chunks t, t + TPR, ... of it, CH of
// them.
template <int TPR>
struct RowThreads {
    static constexpr int THREADS = TPR <= 64 ? 256 : TPR;
    static constexpr int ROWS = THREADS / TPR;
    static constexpr int WAVES = TPR <= 64 ? 1 : TPR / 64;  // per row
};

// Pieces of rows at any element's address (the hardware takes unaligned
// vectors).
typedef uint32_t piece16 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t codes8 __attribute__((ext_vector_type(2), aligned(1)));

// Eight elements from `p`, of which `left` (or more) exist; zeros for the
// others.  WHOLE: left is a multiple of 8.
template <bool WHOLE>
__device__ __forceinline__ u32x4 load8(const uint16_t *p, int left)
{
    u32x4 u = {0u, 0u, 0u, 0u};
    if (WHOLE ? left > 0 : left >= 8) {
        u = *reinterpret_cast<const piece16 *>(p);
    } else if (!WHOLE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left)
                u[i >> 1] |= static_cast<uint32_t>(p[i]) << 16 * (i & 1);
    }
    return u;
}

template <bool WHOLE>
__device__ __forceinline__ void load8(const uint16_t *p, int left, float (&f)[8])
{
    unpack8(load8<WHOLE>(p, left), f);
}

template <bool WHOLE>
__device__ __forceinline__ void store8(uint16_t *p, int left, const float (&f)[8])
{
    const u32x4 u = pack8f(f);
    if (WHOLE ? left > 0 : left >= 8) {
        *reinterpret_cast<piece16 *>(p) = u;
    } else if (!WHOLE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left)
                p[i] = static_cast<uint16_t>(u[i >> 1] >> 16 * (i & 1));
    }
}

// The sum of s and the maximum of m over a row's threads, in each of them.
// `red` is LDS of 2 x WAVES floats and as many words; `flip` alternates from
// row to row, so that one barrier a row is enough.
template <int TPR>
__device__ __forceinline__ void row_reduce(float &s, uint32_t &m, float *red, int flip)
{
    constexpr int W = RowThreads<TPR>::WAVES;
#pragma unroll
    for (int o = TPR < 64 ? TPR / 2 : 32; o >= 1; o >>= 1) {
        s += __shfl_xor(s, o);
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o)));
    }
    if constexpr (W > 1) {
        float *rs = red + flip * 2 * W;
        uint32_t *rm = reinterpret_cast<uint32_t *>(rs + W);
        if ((threadIdx.x & 63) == 0) {
            rs[threadIdx.x >> 6] = s;
            rm[threadIdx.x >> 6] = m;
        }
        __syncthreads();
        s = rs[0];
        m = rm[0];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            s += rs[i];
            m = max(m, rm[i]);
        }
    }
}

// How a row's codes are formed from its largest magnitude.  z is first
// multiplied by `fit`, a power of two that keeps every step below normal and
// finite (1 for ordinary rows).  A row of zeros has codes and scale 0; one
// that holds a NaN or an infinity has codes 0 (`keep`) and a NaN scale, so
// that all its values are NaN.
struct CodeScale {
    float fit, amax, inv, scale;
    uint32_t keep;

    __device__ __forceinline__ explicit CodeScale(uint32_t amax_bits)
    {
        const float a = __uint_as_float(amax_bits);
        fit = a < 0x1p-60f ? 0x1p64f : a > 0x1p60f ? 0x1p-64f : 1.0f;
        amax = a * fit;
        inv = 127.0f / amax;
        scale = a / 127.0f;
        keep = ~0u;
        if (amax_bits == 0 || amax_bits >= 0x7f800000u) {
            fit = amax = 1.0f;
            inv = 0.0f;
            keep = 0u;
            scale = amax_bits == 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        }
    }
    // The codes of eight values, a byte each.  z inv is off by less than 127
    // 2^-23 (two roundings), so the integer nearest to it is the one nearest to
    // 127 z / A unless it is further than 1/2 - 2^-14 from it; then 127 z - q
    // amax, which is exact in fp32 (z and amax have at most 16 significant
    // bits, q and 127 seven), tells the side.  Adding 1.5 2^23 rounds to an
    // integer, ties to even, and leaves its low byte in the bits.
    __device__ __forceinline__ u32x2 codes(const float (&z)[8]) const
    {
        constexpr float kRound = 12582912.0f;
        float t[8], worst = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = z[i] * inv;
            t[i] = v + kRound;
            worst = fmaxf(worst, fabsf(v - (t[i] - kRound)));
        }
        if (worst > 0.5f - 0x1p-14f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float q = t[i] - kRound;
                const float r = fmaf(-q, amax, 127.0f * z[i]), r2 = 2.0f * fabsf(r);
                if (r2 > amax || (r2 == amax && (__float_as_uint(t[i]) & 1)))
                    t[i] += r > 0.f ? 1.0f : -1.0f;
            }
        }
        u32x2 u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                b[e] = __float_as_uint(t[4 * i + e]);
            // Bytes 0-3 of a permutation's selector are its second operand's.
            u[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u),
                                         __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u),
                                         0x05040100u);
        }
        return u;
    }
};

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <bool WHOLE>
__device__ __forceinline__ void store_codes(int8_t *p, int left, const u32x2 &u)
{
    if (WHOLE ? left > 0 : left >= 8) {
        *reinterpret_cast<codes8 *>(p) = u;
    } else if (!WHOLE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left)
                p[i] = static_cast<int8_t>(u[i >> 2] >> 8 * (i & 3));
    }
}

}  // namespace

// One pass over the rows: the row stays in registers from its load to its
// stores.  H and Y have a row stride of d.
struct RowOperands {
    const uint16_t *X, *R, *W;
    uint16_t *H, *Y;
    int8_t *Q;
    float *scales, *rstd;
    long long ldx, ldr, ldq;
    int rows, d;
    float eps;
};

// Element i of h w in fp64, which holds every product of two bf16 numbers: 16
// significant bits, so that the high word alone tells a magnitude.
__device__ __forceinline__ double product_at(const RowOperands &op, long long row, int i)
{
    auto at = [](const uint16_t *p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); };
    float h = at(op.X + row * op.ldx + i);
    if (op.R != nullptr)
        h = static_cast<float>(static_cast<__bf16>(h + at(op.R + row * op.ldr + i)));
    return static_cast<double>(h) * at(op.W + i);
}

// The codes and the scale of a row of the norm whose largest magnitude A by its
// fp32 products is 0, below 2^-60, above 2^60 or not finite.  Zeros are looked up
// as such; else A and the codes come from products in fp64, an element at a time:
// the integer nearest to a quotient of two numbers of at most 23 bits, which fp64
// does not round onto a border.  (In the other rows a product that has lost bits,
// below 2^-126, has code 0 either way.)  65,536 rows of 2048: zeros 133 us,
// extreme values 544, ordinary rows 167.
template <int TPR>
__device__ __forceinline__ void extreme_row(const RowOperands &op, long long row, float rstd,
                                            int t, uint32_t m, float *red, int &flip)
{
    // Nothing is shared with the ordinary rows' way, whose registers it would take.
    asm volatile("" : "+v"(t), "+v"(row));
    const int d = op.d;
    int8_t *q = op.Q + row * op.ldq;
    float none = 0.f;
    if (m == 0 && d >= 8) {
#pragma unroll 1
        for (int i = 8 * t; i < d; i += 8 * TPR) {
            const int col = min(i, d - 8);
            u32x4 u = *reinterpret_cast<const piece16 *>(op.X + row * op.ldx + col);
            if (op.R != nullptr)
                u |= *reinterpret_cast<const piece16 *>(op.R + row * op.ldr + col);
            m |= (u[0] | u[1] | u[2] | u[3]) & 0x7fff7fffu;
        }
        flip ^= 1;
        row_reduce<TPR>(none, m, red, flip);
        if (m == 0) {
            for (int i = 8 * t; i < d; i += 8 * TPR)
                *reinterpret_cast<codes8 *>(q + min(i, d - 8)) = u32x2{0u, 0u};
            if (t == 0)
                op.scales[row] = 0.0f;
            return;
        }
    }
    m = 0;
#pragma unroll 1
    for (int i = t; i < d; i += TPR)
        m = max(m, static_cast<uint32_t>(__double2hiint(product_at(op, row, i))) & 0x7fffffffu);
    flip ^= 1;
    row_reduce<TPR>(none, m, red, flip);
    const bool values = m != 0 && m < 0x7ff00000u;
    const double amax = __hiloint2double(static_cast<int>(m), 0);
    if (t == 0)
        op.scales[row] = values   ? static_cast<float>(amax * rstd / 127.0)
                         : m == 0 ? 0.0f
                                  : __uint_as_float(0x7fc00000u);
#pragma unroll 1
    for (int i = t; i < d; i += TPR)
        q[i] = values ? static_cast<int8_t>(__double2int_rn(127.0 * product_at(op, row, i) / amax))
                      : 0;
}

// Six waves per SIMD for a wave's rows: the norm's codes of rows of 2048 take
// 172 us a 65,536-token step instead of 185 with four (its registers else).
// Eight for rows of 1024 threads: two workgroups per CU (8192 x 16,384, codes,
// 165 us; with one 196).
template <int TPR, int CH, bool WHOLE, int KIND>
__global__ void __launch_bounds__(RowThreads<TPR>::THREADS, TPR <= 64 ? 6 : TPR == 1024 ? 8 : 1)
row_kernel(RowOperands op)
{
    using T = RowThreads<TPR>;
    __shared__ float red[T::WAVES > 1 ? 4 * T::WAVES : 1];
    const int t = threadIdx.x % TPR, d = op.d;
    const int step = static_cast<int>(gridDim.x) * T::ROWS;
    int flip = 0;
    for (long long row = static_cast<long long>(blockIdx.x) * T::ROWS + threadIdx.x / TPR;
         row < op.rows; row += step, flip ^= 1) {
        float v[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (t + TPR * c) * 8;
            load8<WHOLE>(op.X + row * op.ldx + col, d - col, v[c]);
        }
        if (KIND != kCodes && op.R != nullptr) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (t + TPR * c) * 8;
                float r[8];
                load8<WHOLE>(op.R + row * op.ldr + col, d - col, r);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = static_cast<float>(static_cast<__bf16>(v[c][i] + r[i]));
                store8<WHOLE>(op.H + row * d + col, d - col, v[c]);
            }
        }
        float s = 0.f;
        uint32_t m = 0;
        float w[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (t + TPR * c) * 8;
            if constexpr (KIND != kCodes)
                load8<WHOLE>(op.W + col, d - col, w[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (KIND != kCodes)
                    s += v[c][i] * v[c][i];
                if constexpr (KIND == kNormCodes)
                    v[c][i] *= w[c][i];
                if constexpr (KIND != kNorm)
                    m = max(m, abs_bits(v[c][i]));
            }
        }
        row_reduce<TPR>(s, m, red, flip);
        float rstd = 1.f;
        if constexpr (KIND != kCodes) {
            rstd = 1.0f / sqrtf(s / d + op.eps);
            if (t == 0)
                op.rstd[row] = rstd;
        }
        if constexpr (KIND == kNorm) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (t + TPR * c) * 8;
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[i] = v[c][i] * rstd * w[c][i];
                store8<WHOLE>(op.Y + row * d + col, d - col, y);
            }
        } else {
            if constexpr (KIND == kNormCodes) {
                if (m < __float_as_uint(0x1p-60f) || m > __float_as_uint(0x1p60f)) {
                    extreme_row<TPR>(op, row, rstd, t, m, red, flip);
                    continue;
                }
            }
            const CodeScale cs(m);
            if (t == 0)
                op.scales[row] =
                    KIND == kNormCodes ? __uint_as_float(m) * rstd / 127.0f : cs.scale;
            if (cs.fit != 1.0f) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[c][i] *= cs.fit;
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (t + TPR * c) * 8;
                const u32x2 u = cs.codes(v[c]);
                store_codes<WHOLE>(op.Q + row * op.ldq + col, d - col, u32x2{u[0] & cs.keep, u[1] & cs.keep});
            }
        }
    }
}

// Codes to bf16, 8 per lane and load: TPR threads (a wave or less) per row and
// 32 TPR columns.
template <int TPR, bool WHOLE>
__global__ void __launch_bounds__(256)
dequantize_kernel(const int8_t *__restrict__ Q, long long ldq, const float *__restrict__ scales,
                  uint16_t *__restrict__ Y, long long ldy, int rows, int d)
{
    using T = RowThreads<TPR>;
    const int t = threadIdx.x % TPR;
    const int step = static_cast<int>(gridDim.x) * T::ROWS;
    for (long long row = static_cast<long long>(blockIdx.x) * T::ROWS + threadIdx.x / TPR;
         row < rows; row += step) {
        const float s = scales[row];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int col = (static_cast<int>(blockIdx.y) * 4 * TPR + t + TPR * c) * 8;
            const int left = d - col;
            const int8_t *q = Q + row * ldq + col;
            u32x2 u = {0u, 0u};
            if (WHOLE ? left > 0 : left >= 8) {
                u = *reinterpret_cast<const codes8 *>(q);
            } else if (!WHOLE) {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < left)
                        u[i >> 2] |= static_cast<uint32_t>(q[i] & 255) << 8 * (i & 3);
            }
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = s * static_cast<float>(static_cast<int8_t>(u[i >> 2] >> 8 * (i & 3)));
            store8<WHOLE>(Y + row * ldy + col, left, f);
        }
    }
}

// Backward of per_wg rows per workgroup: dx of each, and their column sums of
// dy xh into row blockIdx.x of an fp32 workspace.
struct RmsBackOperands {
    const uint16_t *H, *W, *dY, *dRes;
    const float *rstd;
    uint16_t *dX;
    float *part;
    int rows, d, per_wg;
};

template <int TPR, int CH, bool WHOLE>
__global__ void __launch_bounds__(RowThreads<TPR>::THREADS)
rms_bwd_kernel(RmsBackOperands op)
{
    using T = RowThreads<TPR>;
    constexpr int COLS = TPR * CH * 8;
    // Several rows at once: each one's column sums; else the reductions.
    __shared__ float red[T::ROWS > 1 ? T::ROWS * COLS : 4 * T::WAVES];
    const int t = threadIdx.x % TPR, d = op.d;
    u32x4 w[CH];
    float dw[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (t + TPR * c) * 8;
        w[c] = load8<WHOLE>(op.W + col, d - col);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            dw[c][i] = 0.f;
    }
    const long long row0 = static_cast<long long>(blockIdx.x) * op.per_wg;
    const int n = static_cast<int>(min(static_cast<long long>(op.per_wg), op.rows - row0));
    int flip = 0;
    for (int rr = threadIdx.x / TPR; rr < n; rr += T::ROWS, flip ^= 1) {
        const long long row = row0 + rr, base = row * d;
        const float rstd = op.rstd[row];
        u32x4 h[CH], dy[CH], res[CH];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (t + TPR * c) * 8;
            h[c] = load8<WHOLE>(op.H + base + col, d - col);
            dy[c] = load8<WHOLE>(op.dY + base + col, d - col);
        }
        if (op.dRes != nullptr) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (t + TPR * c) * 8;
                res[c] = load8<WHOLE>(op.dRes + base + col, d - col);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float x[8], y[8], v[8];
            unpack8(h[c], x);
            unpack8(dy[c], y);
            unpack8(w[c], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = y[i] * (x[i] * rstd);
                dw[c][i] += p;
                s += p * v[i];
            }
        }
        uint32_t none = 0;
        row_reduce<TPR>(s, none, red, flip);
        const float mean = s / d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (t + TPR * c) * 8;
            float x[8], y[8], v[8], out[8];
            unpack8(h[c], x);
            unpack8(dy[c], y);
            unpack8(w[c], v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                out[i] = rstd * (y[i] * v[i] - x[i] * rstd * mean);
            if (op.dRes != nullptr) {
                float r[8];
                unpack8(res[c], r);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    out[i] += r[i];
            }
            store8<WHOLE>(op.dX + base + col, d - col, out);
        }
    }
    float *dst = op.part + static_cast<long long>(blockIdx.x) * d;
    if constexpr (T::ROWS > 1) {
        float *mine = red + threadIdx.x / TPR * COLS;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                mine[(t + TPR * c) * 8 + i] = dw[c][i];
        __syncthreads();
        for (int col = threadIdx.x; col < d; col += T::THREADS) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < T::ROWS; ++k)
                sum += red[k * COLS + col];
            dst[col] = sum;
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((t + TPR * c) * 8 + i < d)
                    dst[(t + TPR * c) * 8 + i] = dw[c][i];
    }
}

// Sums of the columns of `part` [n][d]: 16 waves sum 64 columns over the rows
// of chunk blockIdx.y (`per` rows); the result goes to `sums` (fp32, one row
// per chunk), or rounded to bf16 to `dw`.
__global__ void __launch_bounds__(1024)
rms_columns_kernel(const float *__restrict__ part, int n, int per, int d, float *__restrict__ sums,
                   uint16_t *__restrict__ dw)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = static_cast<int>(blockIdx.x) * 64 + lane;
    const int p0 = static_cast<int>(blockIdx.y) * per, p1 = min(p0 + per, n);
    float s = 0.f;
    if (col < d) {
#pragma unroll 4
        for (int p = p0 + wave; p < p1; p += 16)
            s += part[static_cast<long long>(p) * d + col];
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < d) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w)
            sum += red[w][lane];
        if (dw != nullptr)
            dw[col] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(sum));
        else
            sums[static_cast<long long>(blockIdx.y) * d + col] = sum;
    }
}

namespace {

// Rows per workgroup of the backward.  Every workgroup leaves a row of column
// sums; at most kRmsOneStage of those are summed in one launch, more go through
// kRmsChunks chunk sums in two.  So one workgroup per CU for few rows, two for
// many, and four for short rows, of which a workgroup has few in flight.  us
// with 256 / 512 / 1024 workgroups: 2048 x 1024 7.9 / 8.9 / 8.9, 4096 x 2048 18.7
// / 19.9 / 22.3, 16,384 x 5632 172.7 / 166.5 / 170.8, 65,536 x 2048 220.5 / 217.3
// / 217.5, 65,536 x 512 72.7 / 50.2 / 48.4.
constexpr int kRmsOneStage = 256, kRmsChunks = 32;

int rms_rows_per_wg(int rows, int d)
{
    const int wgs = d <= 512 ? 1024 : rows <= 8192 ? 256 : 512;
    const int per = static_cast<int>((rows + wgs - 1LL) / wgs + 3) / 4 * 4;
    return std::max(per, 8);
}

// Threads per row and chunks per thread for rows of d elements: a wave or less
// where that holds the row (65,536 rows of 64: 20.0 us with a wave each), a
// workgroup for longer rows and for few of them, whose latency counts.
struct RowShape {
    int tpr, ch;
};

RowShape row_shape(int rows, int d)
{
    const int tpr = d <= 128                              ? 16
                    : d <= 256                            ? 32
                    : d <= 512 || (d <= 2048 && rows >= 512) ? 64
                    : d <= 8192                           ? 256
                                                          : 1024;
    return RowShape{tpr, (d + 8 * tpr - 1) / (8 * tpr)};
}

// Calls f(IC<TPR>, IC<CH>) for the shape.
template <typename F>
auto with_shape(RowShape s, F f)
{
    if (s.tpr == 16)
        return f(IC<16>{}, IC<1>{});
    if (s.tpr == 32)
        return f(IC<32>{}, IC<1>{});
    if (s.tpr == 64)
        return s.ch == 1   ? f(IC<64>{}, IC<1>{})
               : s.ch == 2 ? f(IC<64>{}, IC<2>{})
               : s.ch == 3 ? f(IC<64>{}, IC<3>{})
                           : f(IC<64>{}, IC<4>{});
    if (s.tpr == 256)
        return s.ch == 1   ? f(IC<256>{}, IC<1>{})
               : s.ch == 2 ? f(IC<256>{}, IC<2>{})
               : s.ch == 3 ? f(IC<256>{}, IC<3>{})
                           : f(IC<256>{}, IC<4>{});
    return f(IC<1024>{}, IC<2>{});
}

// Workgroups of a grid over `n` units: below 2^20, the kernels walk further.
unsigned grid_of(long long n) { return static_cast<unsigned>(std::min<long long>(n, 1 << 20)); }

}  // namespace

int launch_rows(const RowArgs &a)
{
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    const RowOperands op{static_cast<const uint16_t *>(a.X), static_cast<const uint16_t *>(a.R),
                         static_cast<const uint16_t *>(a.w), static_cast<uint16_t *>(a.H),
                         static_cast<uint16_t *>(a.Y),       static_cast<int8_t *>(a.Q),
                         a.scales, a.rstd, a.ldx, a.ldr, a.ldq, a.rows, a.d, a.eps};
    const bool whole = a.d % 8 == 0;
    const hipError_t e = with_shape(row_shape(a.rows, a.d), [&](auto tpr, auto ch) {
        using T = RowThreads<decltype(tpr)::value>;
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        auto run = [&](auto kind) {
            constexpr int K = decltype(kind)::value;
            return launch_kernel(whole ? row_kernel<TPR, CH, true, K> : row_kernel<TPR, CH, false, K>,
                                 dim3(grid_of((a.rows + T::ROWS - 1LL) / T::ROWS)),
                                 dim3(T::THREADS), st, op);
        };
        return a.w == nullptr ? run(IC<kCodes>{}) : a.Q ? run(IC<kNormCodes>{}) : run(IC<kNorm>{});
    });
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

int launch_dequantize(const DequantizeArgs &a)
{
    const bool whole = a.d % 8 == 0;
    auto run = [&](auto tpr) {
        constexpr int TPR = decltype(tpr)::value, ROWS = RowThreads<TPR>::ROWS;
        const dim3 grid(grid_of((a.rows + ROWS - 1LL) / ROWS),
                        static_cast<unsigned>((a.d + 32 * TPR - 1) / (32 * TPR)));
        return launch_kernel(whole ? dequantize_kernel<TPR, true> : dequantize_kernel<TPR, false>,
                             grid, dim3(256), static_cast<hipStream_t>(a.stream),
                             static_cast<const int8_t *>(a.Q), a.ldq, a.scales,
                             static_cast<uint16_t *>(a.Y), a.ldy, a.rows, a.d);
    };
    const hipError_t e = a.d <= 512 ? run(IC<16>{}) : run(IC<64>{});
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

size_t rmsnorm_workspace_bytes(int rows, int d)
{
    const int per = rms_rows_per_wg(rows, d);
    const long long parts = (rows + per - 1LL) / per;
    return static_cast<size_t>(parts + kRmsChunks) * d * sizeof(float);
}

int launch_rmsnorm_bwd(const RmsBackArgs &a)
{
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    const int per = rms_rows_per_wg(a.rows, a.d), parts = static_cast<int>((a.rows + per - 1LL) / per);
    auto *part = static_cast<float *>(a.workspace);
    auto *dw = static_cast<uint16_t *>(a.dw);
    const RmsBackOperands op{static_cast<const uint16_t *>(a.H), static_cast<const uint16_t *>(a.w),
                             static_cast<const uint16_t *>(a.dY), static_cast<const uint16_t *>(a.dRes),
                             a.rstd, static_cast<uint16_t *>(a.dX), part, a.rows, a.d, per};
    const bool whole = a.d % 8 == 0;
    hipError_t e = with_shape(row_shape(a.rows, a.d), [&](auto tpr, auto ch) {
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        return launch_kernel(whole ? rms_bwd_kernel<TPR, CH, true> : rms_bwd_kernel<TPR, CH, false>,
                             dim3(static_cast<unsigned>(parts)), dim3(RowThreads<TPR>::THREADS), st,
                             op);
    });
    if (e != hipSuccess)
        return DD_ERR_HIP;
    const unsigned cols = static_cast<unsigned>((a.d + 63) / 64);
    const float *from = part;
    int n = parts;
    if (parts > kRmsOneStage) {
        float *sums = part + static_cast<long long>(parts) * a.d;
        const int rows = (parts + kRmsChunks - 1) / kRmsChunks;
        e = launch_kernel(rms_columns_kernel, dim3(cols, kRmsChunks), dim3(1024), st, from, parts,
                          rows, a.d, sums, nullptr);
        if (e != hipSuccess)
            return DD_ERR_HIP;
        from = sums;
        n = kRmsChunks;
    }
    e = launch_kernel(rms_columns_kernel, dim3(cols, 1), dim3(1024), st, from, n, n, a.d, nullptr,
                      dw);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
