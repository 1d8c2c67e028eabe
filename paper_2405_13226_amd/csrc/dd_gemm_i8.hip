// dd_gemm_i8.hip -- products of 8-bit integers on the matrix cores:
//   C[m, n] = bf16( sa[m] sb[n] sum over k of A[m, k] B[n, k]  (+ R[m, n]) ),
// A [M][K] and B [N][K] int8 with K innermost, sa an fp32 scale per row of A (a
// token), sb one per row of B (an output channel).  The sum is exact in int32
// (K < 2^17); it is scaled and the residual added in fp32, with one rounding to
// bf16 at the end.  Any M, N and K (a multiple of 16).
#include "dd_device.hpp"
#include "dd_tile.hpp"
#include "dd_gemm.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_routes.hpp"
#include "dd_attn.h"

#include <algorithm>

namespace dd {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// v_mfma_i32_16x16x64_i8: lane l holds the 16 bytes k = 16 (l / 16) .. +15 of
// row l % 16 of A, and of column l % 16 of B; in C rows 4 (l / 16) .. +3 of
// column l % 16.
__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Pieces of rows at any bf16 address (the hardware takes unaligned vectors).
typedef uint32_t piece16 __attribute__((ext_vector_type(4), aligned(2)));

struct GemmI8Operands {
    const int8_t *A, *B;
    const float *sa, *sb;
    const uint16_t *R;
    uint16_t *C;
    long long lda, ldb, ldc;
    int M, N, K, tiles_m, tiles_n, xm;
};

__device__ __forceinline__ float bf16_at(const uint16_t *p)
{
    return __uint_as_float(static_cast<uint32_t>(*p) << 16);
}

// Two accumulators' (j = 0 and 1 of a row block) scaled values of eight
// neighbouring columns: the lanes of neighbouring g exchange halves, after
// which a lane holds the columns from 16 (g % 2) + 8 (g / 2) on.
__device__ __forceinline__ void scale8(i32x4 a0, i32x4 a1, float ra, const float (&rb)[8],
                                       float (&c)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const auto p = __builtin_amdgcn_permlane16_swap(a0[e], a1[e], false, false);
        c[e] = static_cast<float>(static_cast<int>(p[0])) * ra * rb[e];
        c[e + 4] = static_cast<float>(static_cast<int>(p[1])) * ra * rb[e + 4];
    }
}

// c += the eight bf16 values of a piece.
__device__ __forceinline__ void add8(float (&c)[8], const u32x4 &r)
{
    float v[8];
    unpack8(r, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c[e] += v[e];
}

// Stores the first `left` (or all) of eight values at element `o` of C, with
// the residual.
__device__ __forceinline__ void store_edge(const GemmI8Operands &op, long long o, int left,
                                           const float (&c)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) {
            const float v = op.R != nullptr ? c[e] + bf16_at(op.R + o + e) : c[e];
            op.C[o + e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
        }
}

// The direct loads of both operands of a tile.  Every 64 rows x 128 bytes of
// an operand are a sub-tile of 8 KiB in LDS, whose 16-byte chunk x of row r
// sits at x ^ row_swz(r); one instruction of wave w loads its rows 8 w .. +7.
// Rows behind the matrix and bytes behind K read as zeros.
struct I8Loads {
    u32x4 a, b;
    uint32_t va, vb;     // this lane's byte offset in a sub-tile of the step
    uint32_t sa, sb;     // from sub-tile to sub-tile
    int kx, k, K;        // this lane's first k in a step, the next step, the end

    __device__ __forceinline__ void init(const GemmI8Operands &op, int m0, int n0, int wave,
                                         int lane)
    {
        a = buffer_of(op.A + m0 * op.lda, (op.M - 1LL - m0) * op.lda + op.K);
        b = buffer_of(op.B + n0 * op.ldb, (op.N - 1LL - n0) * op.ldb + op.K);
        const int r = 8 * wave + (lane >> 3);
        kx = ((lane & 7) ^ row_swz(r)) * 16;
        va = static_cast<uint32_t>(r * op.lda + kx);
        vb = static_cast<uint32_t>(r * op.ldb + kx);
        sa = static_cast<uint32_t>(64 * op.lda);
        sb = static_cast<uint32_t>(64 * op.ldb);
        k = 0;
        K = op.K;
    }
    // Sub-tile s of the step's A (B) to LDS address l.
    __device__ __forceinline__ void load_a(int s, uint32_t l) const
    {
        dma_b128_buf(a, kx + k < K ? va + (s * sa + k) : kBufferEnd, l);
    }
    __device__ __forceinline__ void load_b(int s, uint32_t l) const
    {
        dma_b128_buf(b, kx + k < K ? vb + (s * sb + k) : kBufferEnd, l);
    }
};

// 256 x 256 tiles, K in steps of 128: the loop of the bf16 product (dd_gemm.hip,
// which has its phases), since an int8 product instruction takes the bytes and
// the time of a bf16 one with twice the k.  A tile is so half as many steps, and
// its start and end weigh twice as much: a workgroup walks tiles blockIdx.x,
// blockIdx.x + gridDim.x, ... as one sequence of steps, the loads running ahead
// across tiles, and the accumulators go to memory straight from registers.
// 65,536 x 5632 over 2048: 601-625 us (2,420-2,515 TOPS), in a process's first
// calls up to 709; 8192^3 373-386 (2,850-2,950).  With a residual 65,536 x 2048
// over 2048 292-389 and 30,000 x 5000 over 1008, whose rows of 10,000 bytes end
// inside a tile, 275-328 (by the profiler, 50 calls).
// The matrix pipes are busy 61% of the time at 2.0 GHz; without the stores 620 us
// where the whole took 667.
struct I8Walk {
    I8Loads ld;
    int tile, count;   // of the next step to load: its tile, how many before it
    int tm, tn, base;  // lane i: the place of the walk's tile base + i
    u32x4 sa, sb;      // the scales of the tile's rows and columns

    // A tile's place comes from the lanes' table: its divisions, made at every
    // tile by every wave, were 2 us of it.
    __device__ __forceinline__ int m0(int n) const
    {
        return __builtin_amdgcn_readlane(tm, n - base) * 256;
    }
    __device__ __forceinline__ int n0(int n) const
    {
        return __builtin_amdgcn_readlane(tn, n - base) * 256;
    }
    __device__ __forceinline__ void places(const GemmI8Operands &op, int from, int lane)
    {
        base = from;
        tile_of(walk_tile(static_cast<int>(blockIdx.x), from + lane, static_cast<int>(gridDim.x),
                          op.tiles_m * op.tiles_n),
                op.tiles_m, op.tiles_n, op.xm, tm, tn);
    }
    __device__ __forceinline__ void start(const GemmI8Operands &op, int wave, int lane,
                                          uint32_t scales)
    {
        if (tile < op.tiles_m * op.tiles_n) {
            if (count - base == 64)  // the tile computed is at most three behind
                places(op, count - 3, lane);
            const int m = m0(count), n = n0(count);
            ld.init(op, m, n, wave, lane);
            sa = buffer_of(op.sa + m, (op.M - m) * 4LL);
            sb = buffer_of(op.sb + n, (op.N - n) * 4LL);
        } else {  // nothing left: the loads read zeros
            ld.k = 0;
            ld.a[2] = ld.b[2] = sa[2] = sb[2] = 0;
        }
        // 256 + 256 scales, 64 per wave, to one of four places in LDS.
        const uint32_t l = scales + 2048u * (count & 3) + 256u * wave;
        if (wave < 4)
            dma_b32_buf(sa, 4u * (64 * wave + lane), l);
        else
            dma_b32_buf(sb, 4u * (64 * (wave - 4) + lane), l);
    }
    __device__ __forceinline__ void next(const GemmI8Operands &op, int wave, int lane,
                                         uint32_t scales)
    {
        ld.k += 128;
        if (ld.k >= op.K) {
            tile += static_cast<int>(gridDim.x);
            ++count;
            start(op, wave, lane, scales);
        }
    }
};

__global__ void __launch_bounds__(512, 1)
gemm_i8_kernel(GemmI8Operands op)
{
    constexpr int SUB = 64 * 128, HALF = 2 * SUB, SIDE = 4 * HALF;  // bytes
    __shared__ __attribute__((aligned(1024))) int8_t lds[2 * SIDE + 4 * 2048];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int wm = wave >> 2, wn = wave & 3;
    const int tiles = op.tiles_m * op.tiles_n, nkt = (op.K + 127) / 128;
    const uint32_t lds0 = lds_base_sgpr(lds), scales = lds0 + 2 * SIDE;
    I8Walk at;
    at.tile = static_cast<int>(blockIdx.x);
    at.count = 0;
    at.places(op, 0, lane);
    at.start(op, wave, lane, scales);
    auto load_a = [&](int h, int S) __attribute__((always_inline)) {
        const uint32_t l = lds0 + 1024u * wave + (2 * h + S) * HALF;
        at.ld.load_a(2 * h, l);
        at.ld.load_a(2 * h + 1, l + SUB);
    };
    auto load_b = [&](int h, int S) __attribute__((always_inline)) {
        const uint32_t l = lds0 + 1024u * wave + SIDE + (2 * h + S) * HALF;
        at.ld.load_b(2 * h, l);
        at.ld.load_b(2 * h + 1, l + SUB);
    };
    const int8_t *fa[2], *fb[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        const int x = ((4 * kk + g) ^ row_swz(l16)) * 16;
        fa[kk] = lds + wm * SUB + 128 * l16 + x;
        fb[kk] = lds + SIDE + (wn >> 1) * SUB + 128 * (32 * (wn & 1) + l16) + x;
    }
    u32x4 a0[4][2], a1[4][2], b0[2][2], b1[2][2];
    auto read_a = [&](u32x4 (&f)[4][2], int h, int S) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
                f[i][kk] = *reinterpret_cast<const u32x4 *>(fa[kk] + ((2 * h + S) * HALF + 2048 * i));
    };
    auto read_b = [&](u32x4 (&f)[2][2], int h, int S) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
                f[j][kk] = *reinterpret_cast<const u32x4 *>(fb[kk] + ((2 * h + S) * HALF + 2048 * j));
    };
    i32x4 acc[2][2][4][2];  // [A half][B half][i][j]
    // c += b a, or in a tile's first step c = b a.
    auto products = [&](i32x4 (&c)[4][2], const u32x4 (&a)[4][2], const u32x4 (&b)[2][2],
                        bool first) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    c[i][j] = mfma_i8(b[j][kk], a[i][kk],
                                      first && kk == 0 ? i32x4{} : c[i][j]);  // rows n, columns m
        __builtin_amdgcn_s_setprio(0);
        plain_barrier();
    };
    // Six halves of loads (12) stay in flight, as in the bf16 product; in the
    // six phases after a whole tile's 16 stores, which no load waits for, those
    // too.  (A tile's scales are one load more: the waits are then one tighter.)
    bool stored = false;
    auto wait = [&](bool first) __attribute__((always_inline)) {
        if (first && stored)
            wait_and_barrier<28>();
        else
            wait_and_barrier<12>();
    };
    // One step from stage S, its tile's first (FIRST 2), second (1) or a later
    // one.
    auto step = [&](auto stage, auto first) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value, FIRST = decltype(first)::value;
        read_b(b0, 0, S);
        load_a(0, S);
        wait(FIRST > 0);
        products(acc[0][0], a0, b0, FIRST == 2);
        read_b(b1, 1, S);
        load_b(0, S);
        wait(FIRST > 0);
        products(acc[0][1], a0, b1, FIRST == 2);
        read_a(a1, 1, S);
        load_b(1, S);
        wait(FIRST > 1);
        products(acc[1][1], a1, b1, FIRST == 2);
        read_a(a0, 0, 1 - S);  // of the next step
        load_a(1, S);
        at.next(op, wave, lane, scales);
        wait(FIRST > 1);
        products(acc[1][0], a1, b0, FIRST == 2);
    };
    auto load_step = [&](int S) __attribute__((always_inline)) {
        load_a(0, S);
        load_b(0, S);
        load_b(1, S);
        load_a(1, S);
        at.next(op, wave, lane, scales);
    };
    load_step(0);
    load_step(1);
    wait_and_barrier<8>();
    read_a(a0, 0, 0);
    // Phase 1 refills the half just read: only after a barrier that every wave
    // reaches with its reads returned.
    wait_and_barrier<8>();
    // Waves 4-7 run half a phase behind waves 0-3.
    if (wm == 1)
        plain_barrier();
    int tile = static_cast<int>(blockIdx.x), done = 0;
    // A tile whose first step is in stage S; with an odd number of steps the
    // next tile's is in the other.
    auto whole_tile = [&](auto stage) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value;
        step(IC<S>{}, IC<2>{});
        if (nkt > 1) {
            step(IC<1 - S>{}, IC<1>{});
            for (int kt = 2; kt + 1 < nkt; kt += 2) {
                step(IC<S>{}, IC<0>{});
                step(IC<1 - S>{}, IC<0>{});
            }
            if (nkt & 1)
                step(IC<S>{}, IC<0>{});
        }
        // Accumulator (ha, hb, i, j), register e: row m = 128 ha + 64 wm + 16 i
        // + l16, column n = 128 hb + 32 wn + 16 j + 4 g + e of the tile; eight
        // neighbouring columns per lane by scale8.
        const int m0 = at.m0(done), n0 = at.n0(done);
        const bool whole = m0 + 256 <= op.M && n0 + 256 <= op.N;
        const float *sc = reinterpret_cast<const float *>(lds + 2 * SIDE + 2048 * (done & 3));
        const int el = fresh(lane), row = 64 * wm + (el & 15);
        const int col = 32 * wn + 16 * ((el >> 4) & 1) + 8 * (el >> 5);
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
            const int n = n0 + 128 * hb + col;
            // Of the lane's first row; from there 32 bits (ldc < 2^23).
            const long long at0 = (m0 + row) * op.ldc + n;
            const uint32_t ld = fresh(static_cast<int>(op.ldc));
            float rb[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                rb[e] = sc[256 + 128 * hb + col + e];
            // The residual's pieces first, together: a wait for one also waits
            // for what is in flight.
            u32x4 res[8];
            if (op.R != nullptr) {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int r = 128 * (x >> 2) + 16 * (x & 3), m = m0 + r + row;
                    res[x] = u32x4{0u, 0u, 0u, 0u};
                    if (whole || (m < op.M && n + 8 <= op.N))
                        res[x] = *reinterpret_cast<const piece16 *>(op.R + at0 + r * ld);
                }
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const int ha = x >> 2, i = x & 3, r = 128 * ha + 16 * i, m = m0 + r + row;
                const float ra = sc[r + row];
                float c[8];
                scale8(acc[ha][hb][i][0], acc[ha][hb][i][1], ra, rb, c);
                const long long o = at0 + r * ld;
                if (whole || (m < op.M && n + 8 <= op.N)) {
                    if (op.R != nullptr)
                        add8(c, res[x]);
                    *reinterpret_cast<piece16 *>(op.C + o) = pack8f(c);
                } else if (m < op.M) {
                    store_edge(op, o, op.N - n, c);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        stored = whole;
        tile += static_cast<int>(gridDim.x);
        ++done;
    };
    while (tile < tiles) {
        whole_tile(IC<0>{});
        if ((nkt & 1) && tile < tiles)
            whole_tile(IC<1>{});
    }
    if (wm == 0)
        plain_barrier();
    // The loads behind the last tile still write to this workgroup's LDS.
    wait_vmem();
}

// 128 x 128 tiles, two workgroups per CU (80 KiB each), whose starts and ends
// the other one's products fill.  K in steps of 64, five stages of which four
// are in flight; eight waves, 64 x 32 each, one barrier a step.  What the end
// needs is loaded before the loop.  (One workgroup per CU, four stages of 128
// and two wave groups half a phase apart, with the tile's image through LDS:
// 16,384 x 500 over 512 14.7 us, here 12.1; 65,536 x 512 over 512 51.2 and
// 34.9; 4096 x 2048 over 2048 with a residual 32.2 and 27.7; at one tile per CU
// or fewer the same within 8%.)
__global__ void __launch_bounds__(512, 4)
gemm_i8_small_kernel(GemmI8Operands op)
{
    constexpr int SIDE = 128 * 64, STAGE = 2 * SIDE, NST = 5;  // bytes
    __shared__ __attribute__((aligned(1024))) int8_t lds[NST * STAGE];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int wm = wave >> 2, wn = wave & 3;
    int tm, tn;
    tile_of(static_cast<int>(blockIdx.x), op.tiles_m, op.tiles_n, op.xm, tm, tn);
    const int m0 = tm * 128, n0 = tn * 128;
    const int nkt = (op.K + 63) / 64;

    // A wave loads 16 rows of 64 bytes of each side.  Chunk x of row r sits at
    // x ^ (-(r / 4) mod 4): the 16 lanes that the LDS serves together (rows r,
    // r + 12 of chunk x, r + 4, r + 8 of chunk x + 1, r < 4, and so on) then read
    // all banks.
    const int swz = -(lane >> 4) & 3;
    const int kx = ((lane & 3) ^ swz) * 16;
    const u32x4 ba = buffer_of(op.A + m0 * op.lda, (op.M - 1LL - m0) * op.lda + op.K);
    const u32x4 bb = buffer_of(op.B + n0 * op.ldb, (op.N - 1LL - n0) * op.ldb + op.K);
    const uint32_t va = static_cast<uint32_t>((16 * wave + (lane >> 2)) * op.lda + kx);
    const uint32_t vb = static_cast<uint32_t>((16 * wave + (lane >> 2)) * op.ldb + kx);
    const uint32_t lds0 = lds_base_sgpr(lds) + 1024u * wave;
    auto load = [&](int kt, int st) __attribute__((always_inline)) {
        const int k = kt * 64;
        dma_b128_buf(ba, kx + k < op.K ? va + k : kBufferEnd, lds0 + STAGE * st);
        dma_b128_buf(bb, kx + k < op.K ? vb + k : kBufferEnd, lds0 + STAGE * st + SIDE);
    };
    const int x = (g ^ (-(l16 >> 2) & 3)) * 16;
    const int fa = (64 * wm + l16) * 64 + x, fb = SIDE + (32 * wn + l16) * 64 + x;

    // The lane's rows and columns in the end (gemm_i8_kernel).
    const int row = m0 + 64 * wm + l16, n = n0 + 32 * wn + 16 * (g & 1) + 8 * (g >> 1);
    float ra[4], rb[8];
    u32x4 res[4];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        rb[e] = op.sb[min(n + e, op.N - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = row + 16 * i;
        ra[i] = op.sa[min(m, op.M - 1)];
        res[i] = u32x4{0u, 0u, 0u, 0u};
        if (op.R != nullptr && m < op.M && n + 8 <= op.N)
            res[i] = *reinterpret_cast<const piece16 *>(op.R + m * op.ldc + n);
    }

    i32x4 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            acc[i][j] = i32x4{};
    for (int kt = 0; kt < NST - 1; ++kt)
        load(kt, kt);  // (behind K: zeros)
    int rs = 0, ws = NST - 1;  // the stages read and refilled by a step
    for (int kt = 0; kt < nkt; ++kt) {
        // This step's loads are there, and every wave has read the stage of the
        // step before.
        wait_and_barrier<2 * (NST - 2)>();
        load(kt + NST - 1, ws);
        const int8_t *st = lds + rs * STAGE;
        u32x4 a[4], b[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            b[j] = *reinterpret_cast<const u32x4 *>(st + fb + 1024 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = *reinterpret_cast<const u32x4 *>(st + fa + 1024 * i);
        ws = rs;
        rs = rs + 1 == NST ? 0 : rs + 1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = mfma_i8(b[j], a[i], acc[i][j]);  // rows n, columns m
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = row + 16 * i;
        float c[8];
        scale8(acc[i][0], acc[i][1], ra[i], rb, c);
        const long long o = m * op.ldc + n;
        if (m < op.M && n + 8 <= op.N) {
            add8(c, res[i]);
            *reinterpret_cast<piece16 *>(op.C + o) = pack8f(c);
        } else if (m < op.M) {
            store_edge(op, o, op.N - n, c);
        }
    }
    // The loads behind the last step still write to this workgroup's LDS.
    wait_vmem();
}

// At most 64 tokens: the weights are read once, straight into registers, 16
// NB rows of them per workgroup; its eight waves share K in turns of 64 and add
// their sums through LDS.  MB blocks of 16 tokens.  Bound by the weights' bytes
// (1 x 50,432 over 2048 18.1 us, 5.7 TB/s) or the latency of one pass (1 x 6144
// over 2048 4.4 us, of which the bytes are 2.6).
template <int MB, int NB>
__global__ void __launch_bounds__(512)
gemm_i8_few_kernel(GemmI8Operands op)
{
    constexpr int UN = MB * NB > 4 ? 2 : 4;  // turns whose loads are in flight
    __shared__ __attribute__((aligned(16))) int sums[8][MB * NB][4][64];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int n0 = static_cast<int>(blockIdx.x) * 16 * NB;
    const int8_t *pa[MB], *pb[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
        pa[i] = op.A + min(16 * i + l16, op.M - 1) * op.lda + 16 * g;
#pragma unroll
    for (int j = 0; j < NB; ++j)
        pb[j] = op.B + min(n0 + 16 * j + l16, op.N - 1) * op.ldb + 16 * g;
    i32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            acc[i][j] = i32x4{};
    for (int k0 = wave * 64; k0 < op.K; k0 += 512 * UN) {
        u32x4 a[UN][MB], b[UN][NB];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int k = k0 + 512 * u;
            const bool in = k + 16 * g < op.K;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                b[u][j] = in ? *reinterpret_cast<const u32x4 *>(pb[j] + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < MB; ++i)
                a[u][i] = in ? *reinterpret_cast<const u32x4 *>(pa[i] + k) : u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    acc[i][j] = mfma_i8(b[u][j], a[u][i], acc[i][j]);  // rows n, columns m
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sums[wave][i * NB + j][e][lane] = acc[i][j][e];
    __syncthreads();
    // Element (m, n) of the workgroup: block (m / 16, n / 16), register n % 4
    // of lane 16 (n % 16 / 4) + m % 16.
    for (int idx = tid; idx < 256 * MB * NB; idx += 512) {
        const int m = idx / (16 * NB), c = idx % (16 * NB), n = n0 + c;
        if (m >= op.M || n >= op.N)
            continue;
        const int blk = (m >> 4) * NB + (c >> 4), ln = 16 * ((c & 15) >> 2) + (m & 15);
        int s = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w)
            s += sums[w][blk][c & 3][ln];
        const long long at = m * op.ldc + n;
        float v = static_cast<float>(s) * op.sa[m] * op.sb[n];
        if (op.R != nullptr)
            v += bf16_at(op.R + at);
        op.C[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
}

int launch_gemm_i8(const GemmI8Args &a)
{
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    GemmI8Operands op{static_cast<const int8_t *>(a.A), static_cast<const int8_t *>(a.B), a.sa,
                      a.sb, static_cast<const uint16_t *>(a.R), static_cast<uint16_t *>(a.C),
                      a.lda, a.ldb, a.ldc, a.M, a.N, a.K, 0, 0, 0};
    GemmI8Tile tile = gemm_i8_tile(a.M, a.N, a.K, device_cu_count());
    if (tile == GemmI8Tile::kLarge && a.ldc >= 1 << 23)  // its offsets in a tile of C
        tile = GemmI8Tile::kSmall;
    // Weight rows per workgroup of few tokens; a dispatch holds fewer than 2^32
    // work-items.
    const bool two = a.N > 16 * 1024;
    const int cols = two ? 32 : 16;
    if (tile == GemmI8Tile::kFew && (a.N + cols - 1LL) / cols >= 1 << 23)
        tile = GemmI8Tile::kSmall;
    if (tile == GemmI8Tile::kFew) {
        const int mb = (a.M + 15) / 16;
        auto run = [&](auto m) {
            constexpr int MB = decltype(m)::value;
            return launch_kernel(two ? gemm_i8_few_kernel<MB, 2> : gemm_i8_few_kernel<MB, 1>,
                                 dim3(static_cast<unsigned>((a.N + cols - 1) / cols)), dim3(512),
                                 st, op);
        };
        const hipError_t e = mb == 1 ? run(IC<1>{}) : mb == 2 ? run(IC<2>{}) : run(IC<4>{});
        return e == hipSuccess ? DD_OK : DD_ERR_HIP;
    }
    const int edge = tile == GemmI8Tile::kLarge ? 256 : 128;
    op.tiles_m = (a.M + edge - 1) / edge;
    op.tiles_n = (a.N + edge - 1) / edge;
    op.xm = tile_rows_step(op.tiles_m, op.tiles_n);
    const dim3 grid(static_cast<unsigned>(op.tiles_m) * static_cast<unsigned>(op.tiles_n));
    // The large tiles' workgroups, one per CU, walk them; a multiple of the
    // XCDs, so that each keeps its XCD's tiles (tile_of).
    const unsigned cus = static_cast<unsigned>(std::max(device_cu_count() / kXcds * kXcds, kXcds));
    const hipError_t e =
        tile == GemmI8Tile::kLarge
            ? launch_kernel(gemm_i8_kernel, dim3(std::min(grid.x, cus)), dim3(512), st, op)
            : launch_kernel(gemm_i8_small_kernel, grid, dim3(512), st, op);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
