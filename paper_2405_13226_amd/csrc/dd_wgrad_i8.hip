// dd_wgrad_i8.hip -- the weight gradient of a linear layer whose input was kept
// in 8 bits:  dW[m, n] = sum over t of X[t, m] dY[t, n],  X = bf16(scales Q);
// up to three dY at once (projections that share their input).
//
// The restored input is bf16, as the activation that was saved; the products
// are bf16 matrix-core products with fp32 sums.  Any T, M and N (M and N
// multiples of 8).
//
// Two launches, or three.  The first restores X, transposed: XT [M][T] in the
// workspace, T padded with zeros to whole K steps.  The product then reads XT
// along its rows and dY, as it is stored, transposed, with the loop of the
// bf16 product (dd_gemm.hip).  Tiles that several workgroups share (WgradPlan)
// leave fp32 parts in the workspace, which a last launch adds in a fixed order.
//
// 65,536 tokens, 2048 x 5632, us: a call 1183 (1,278 TFLOP/s; median, in turn with
// dd_gemm from bf16 activations, 1256; forming the codes, 75, is not in it).  Its
// kernels under the profiler, mean and least of 50: restoring 76 and 70 (5.8 TB/s),
// product 1151 and 1070, sum 22 and 21.  Power bounds the product: pipes 81-84%
// busy at 1.4-1.65 GHz.  What its uneven tiles cost beside that: 256 whole ones
// (2048 x 8192) keep the pipes 90% busy and read 3.2 GB from behind L2, these 176
// with their pieces 6.5-6.8.  Converting the codes inside the loop, which would save
// the restoring, has not been built: counted, it moves 48 KiB more through an LDS
// that moves 256 a step of 2,400 clocks.
#include "dd_device.hpp"
#include "dd_tile.hpp"
#include "dd_gemm.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_routes.hpp"
#include "dd_attn.h"

#include <algorithm>

namespace dd {

typedef uint32_t codes16 __attribute__((ext_vector_type(4), aligned(8)));

// XT[m][t] = bf16(scales[t] Q[t][m]), zeros for T <= t < Tp.  One 128 x 128
// tile per workgroup: rows of codes into LDS as bf16, then its transposing
// reads, eight tokens of a column per lane.  Bound by HBM.
__global__ void __launch_bounds__(256)
restore_kernel(const int8_t *__restrict__ Q, long long ldq, const float *__restrict__ scales,
               uint16_t *__restrict__ XT, long long Tp, int T, int M)
{
    // Four sub-tiles of 64 columns x 64 tokens.
    __shared__ __attribute__((aligned(16))) uint16_t lds[4 * 64 * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long t0 = static_cast<long long>(blockIdx.x) * 128;
    const int m0 = static_cast<int>(blockIdx.y) * 128;
    const int c = (tid & 7) * 16;
    u32x4 q[4];
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long t = t0 + (tid >> 3) + 32 * i;
        const int8_t *p = Q + t * ldq + m0 + c;
        q[i] = u32x4{0u, 0u, 0u, 0u};
        s[i] = 0.f;
        if (t < T) {
            s[i] = scales[t];
            if (m0 + c + 16 <= M) {
                q[i] = *reinterpret_cast<const codes16 *>(p);
            } else if (m0 + c + 8 <= M) {
                const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
                q[i][0] = v[0];
                q[i][1] = v[1];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = (tid >> 3) + 32 * i;  // token of the tile
        uint16_t *sub = lds + (2 * (r >> 6) + (c >> 6)) * 4096;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                f[e] = s[i] * static_cast<float>(static_cast<int8_t>(q[i][2 * h + (e >> 2)] >> 8 * (e & 3)));
            *reinterpret_cast<u32x4 *>(sub + tile_off<64>(r & 63, (c & 63) + 8 * h)) = pack8f(f);
        }
    }
    __syncthreads();
    // 128 columns x 16 pieces of eight tokens; 16 columns and four pieces per
    // wave instruction.
    const int l16 = lane & 15, g = lane >> 4, e4 = l16 >> 2, c4 = l16 & 3;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int blk = wave * 2 + (i & 1), piece = (i >> 1) * 4 + g;  // columns 16 blk ..
        const uint16_t *sub = lds + (2 * (piece >> 3) + (blk >> 2)) * 4096;
        const int r = 8 * (piece & 7) + e4, col = 16 * (blk & 3) + 4 * c4;
        const bf16x8 v =
            join(lds_tr4(sub + tile_off<64>(r, col)), lds_tr4(sub + tile_off<64>(r + 4, col)));
        const int m = m0 + 16 * blk + l16;
        const long long t = t0 + 8 * piece;
        if (m < M && t < Tp)
            *reinterpret_cast<bf16x8 *>(XT + m * Tp + t) = v;
    }
}

// dW[i] = X^T dY[i] for up to three dY.  Their tiles are one grid of tiles_m x
// tiles_n, `cols` columns of it each.  P: fp32 parts of the shared tiles (of
// WgradPlan): `firsts` = heads x shared, one of each tile's first `head` steps,
// one of its next and so on, then `most` for each of the tails.
struct WgradOperands {
    const uint16_t *XT, *dY[3];
    uint16_t *dW[3];
    float *P;
    long long Tp, ldy, ldw;
    int T, M, N, tiles_m, tiles_n, cols, xm, whole, shared, firsts, steps, head, rest, most;
};

// Where a tile is: its gradient and its first row and column in that.
struct WgradPlace {
    int i, m0, n0;
};

template <int EDGE>
__device__ __forceinline__ WgradPlace wgrad_place(const WgradOperands &op, int tile)
{
    int tm, tn;
    tile_of(tile, op.tiles_m, op.tiles_n, op.xm, tm, tn);
    const int i = (tn >= op.cols) + (tn >= 2 * op.cols);
    return WgradPlace{i, tm * EDGE, (tn - i * op.cols) * EDGE};
}

// One of three pointers; an array in the kernel's arguments that is indexed
// at run time would be copied to memory.
template <typename P>
__device__ __forceinline__ P pick3(P const (&p)[3], int i)
{
    return i == 0 ? p[0] : i == 1 ? p[1] : p[2];
}

// The parts of tiles that workgroup `id` computes, one after the other: steps
// `first` .. first + count - 1 of `tile`, stored to part `slot`, or as the
// result (slot < 0).
struct WgradParts {
    int tile, first, count, slot;
    int at, end;  // in the shared tiles' rests, laid out one after the other

    __device__ __forceinline__ void init(const WgradOperands &op, int id)
    {
        at = end = 0;
        if (id < op.whole) {
            tile = id;
            first = 0;
            count = op.steps;
            slot = -1;
        } else if (id < op.whole + op.firsts) {
            slot = id - op.whole;
            const int j = slot / op.shared;
            tile = id - j * op.shared;
            first = j * op.head;
            count = min(op.head, op.steps - first);
        } else {
            const int w = id - op.whole - op.firsts;
            at = w * op.head;
            end = min(at + op.head, op.shared * op.rest);
            slot = op.firsts + w * op.most - 1;
            next(op);
        }
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void next(const WgradOperands &op)
    {
        const int i = at / op.rest, skip = at - i * op.rest;
        tile = op.whole + i;
        first = op.steps - op.rest + skip;
        count = min(op.rest - skip, end - at);
        at += count;
        ++slot;
    }
};

// Direct loads of a tile's K steps.  XT: 64 columns (rows of XT) of a step are
// a sub-tile, 128-byte rows in chunks swizzled for row reads; dY: the step's
// 64 tokens x 64 columns, swizzled for transposing reads.  Tokens behind T
// are zeros in XT and read as zeros in dY; what is read in columns behind M
// (XT has room for whole tiles) and N is not stored.
struct WgradLoads {
    const uint16_t *a;
    u32x4 buf;            // dY from the rows of the step and column n0 on
    long long b_left;     // its bytes
    uint32_t va, vb, b_step;
    long long a_step;     // from sub-tile to sub-tile (elements)

    __device__ __forceinline__ void init(const WgradOperands &op, const WgradPlace &p, long long kbeg,
                                         int wave, int lane)
    {
        const int r = 8 * wave + (lane >> 3);
        a = op.XT + p.m0 * op.Tp + kbeg;
        a_step = 64 * op.Tp;
        va = static_cast<uint32_t>(r * op.Tp * 2 + ((lane & 7) ^ row_swz(r)) * 16);
        b_left = ((op.T - 1LL - kbeg) * op.ldy + op.N - p.n0) * 2;
        b_step = static_cast<uint32_t>(64 * op.ldy * 2);
        vb = static_cast<uint32_t>((r * op.ldy + ((lane & 7) ^ swz<64>(r)) * 8) * 2);
        buf = buffer_of(pick3(op.dY, p.i) + kbeg * op.ldy + p.n0, b_left);
    }
    __device__ __forceinline__ void next()
    {
        a += 64;
        b_left -= b_step;
        const uint64_t b = (static_cast<uint64_t>(buf[1]) << 32 | buf[0]) + b_step;
        buf = buffer_of(reinterpret_cast<const void *>(b), b_left);
    }
    __device__ __forceinline__ void load_a(int s, uint32_t l) const
    {
        dma_b128_off(a + s * a_step, va, l);
    }
    __device__ __forceinline__ void load_b(int s, uint32_t l) const
    {
        dma_b128_buf(buf, vb + 128u * s, l);
    }
};

__device__ __forceinline__ f32x4 mfma16w(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Element offset of (row r, column c) in the LDS image of the finished tile.
template <int BN>
__device__ __forceinline__ int wgrad_off(int r, int c)
{
    return r * BN + 4 * ((c >> 2) ^ (2 * (r & 15)));
}

template <int BM, int BN>
__device__ __forceinline__ void wgrad_store(const uint16_t *lds, const WgradOperands &op,
                                            const WgradPlace &p, int tid)
{
    constexpr int CPR = BN / 8;
    uint16_t *dW = pick3(op.dW, p.i);
#pragma unroll 4
    for (int it = 0; it < BM * CPR / 512; ++it) {
        const int idx = it * 512 + tid, r = idx / CPR, c = idx % CPR * 8;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + wgrad_off<BN>(r, c));
        if (p.m0 + r < op.M && p.n0 + c < op.N)
            *reinterpret_cast<u32x4 *>(dW + (p.m0 + r) * op.ldw + p.n0 + c) = v;
    }
}

// What becomes of a part's accumulators, which `each` hands to a function of
// (row, column, the values of four columns): an fp32 part, or the result.
template <int EDGE, typename F>
__device__ __forceinline__ void finish_part(const WgradOperands &op, const WgradParts &part,
                                            uint16_t *lds, const WgradPlace &place, int tid,
                                            F each)
{
    if (part.slot >= 0) {
        float *dst = op.P + static_cast<long long>(part.slot) * (EDGE * EDGE);
        each([&](int r, int c, const f32x4 &v) __attribute__((always_inline)) {
            *reinterpret_cast<f32x4 *>(dst + r * EDGE + c) = v;
        });
    } else {
        __syncthreads();
        each([&](int r, int c, const f32x4 &v) __attribute__((always_inline)) {
            *reinterpret_cast<bf16x4 *>(lds + wgrad_off<EDGE>(r, c)) = pack4(v[0], v[1], v[2], v[3]);
        });
        __syncthreads();
        wgrad_store<EDGE, EDGE>(lds, op, place, fresh(tid));
    }
}

// 256 x 256 tiles, the phases of dd_gemm.hip.
__global__ void __launch_bounds__(512, 1)
wgrad_kernel(WgradOperands op)
{
    constexpr int SUB = 64 * 64, HALF = 2 * SUB, SIDE = 4 * HALF;  // elements
    __shared__ __attribute__((aligned(1024))) uint16_t lds[2 * SIDE];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int wm = wave >> 2, wn = wave & 3;
    WgradLoads at;
    const uint32_t lds0 = lds_base_sgpr(lds) + 1024u * wave;
    auto load_a = [&](int h, int S) __attribute__((always_inline)) {
        const uint32_t l = lds0 + 2u * (2 * h + S) * HALF;
        at.load_a(2 * h, l);
        at.load_a(2 * h + 1, l + 2u * SUB);
    };
    auto load_b = [&](int h, int S) __attribute__((always_inline)) {
        const uint32_t l = lds0 + 2u * (SIDE + (2 * h + S) * HALF);
        at.load_b(2 * h, l);
        at.load_b(2 * h + 1, l + 2u * SUB);
    };
    const int e4 = l16 >> 2, c4 = l16 & 3;
    const uint16_t *fa[2], *fb[4];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
        fa[kk] = lds + wm * SUB + 64 * l16 + (((4 * kk + g) ^ row_swz(l16)) << 3);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        fb[j] = lds + SIDE + (wn >> 1) * SUB +
                tile_off<64>(8 * g + 4 * (j & 1) + e4, 32 * (wn & 1) + 16 * (j >> 1) + 4 * c4);
    bf16x8 a0[4][2], a1[4][2], b0[2][2], b1[2][2];
    auto read_a = [&](bf16x8 (&f)[4][2], int h, int S) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
                f[i][kk] = lds_row8(fa[kk] + ((2 * h + S) * HALF + 1024 * i));
    };
    auto read_b = [&](bf16x8 (&f)[2][2], int h, int S) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const int o = (2 * h + S) * HALF + 2048 * kk;
                f[j][kk] = join(lds_tr4(fb[2 * j] + o), lds_tr4(fb[2 * j + 1] + o));
            }
    };
    f32x4 acc[2][2][4][2];  // [A half][B half][i][j]
    auto multiply = [&](f32x4 (&c)[4][2], const bf16x8 (&a)[4][2],
                        const bf16x8 (&b)[2][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    c[i][j] = mfma16w(b[j][kk], a[i][kk], c[i][j]);  // rows n, columns m
    };
    auto products = [&](f32x4 (&c)[4][2], const bf16x8 (&a)[4][2],
                        const bf16x8 (&b)[2][2]) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
        multiply(c, a, b);
        __builtin_amdgcn_s_setprio(0);
        plain_barrier();
    };
    // One K step from stage S.  MODE 0: also starts the loads of the step
    // after the next one; 1, 2: the last step but one, the last step.
    auto step = [&](auto stage, auto mode) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value, MODE = decltype(mode)::value;
        read_b(b0, 0, S);
        if constexpr (MODE == 0)
            load_a(0, S);
        wait_and_barrier<MODE == 0 ? 12 : MODE == 1 ? 10 : 2>();
        products(acc[0][0], a0, b0);
        read_b(b1, 1, S);
        if constexpr (MODE == 0)
            load_b(0, S);
        wait_and_barrier<MODE == 0 ? 12 : MODE == 1 ? 8 : 0>();
        products(acc[0][1], a0, b1);
        read_a(a1, 1, S);
        if constexpr (MODE == 0)
            load_b(1, S);
        wait_and_barrier<MODE == 0 ? 12 : MODE == 1 ? 6 : 0>();
        products(acc[1][1], a1, b1);
        if constexpr (MODE != 2)
            read_a(a0, 0, 1 - S);
        if constexpr (MODE == 0) {
            load_a(1, S);
            at.next();
        }
        wait_and_barrier<MODE == 0 ? 12 : MODE == 1 ? 4 : 0>();
        products(acc[1][0], a1, b0);
    };
    auto load_step = [&](int S) __attribute__((always_inline)) {
        load_a(0, S);
        load_b(0, S);
        load_b(1, S);
        load_a(1, S);
        at.next();
    };
    WgradParts part;
    part.init(op, static_cast<int>(blockIdx.x));
    for (;;) {
        const WgradPlace place = wgrad_place<256>(op, part.tile);
        const int nkt = part.count;
        at.init(op, place, part.first * 64LL, wave, fresh(lane));
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[x >> 1][x & 1][i][j] = f32x4{};
        if (nkt == 1) {
            load_step(0);
            wait_and_barrier<0>();
            read_a(a0, 0, 0);
            read_b(b0, 0, 0);
            multiply(acc[0][0], a0, b0);
            read_b(b1, 1, 0);
            multiply(acc[0][1], a0, b1);
            read_a(a1, 1, 0);
            multiply(acc[1][1], a1, b1);
            multiply(acc[1][0], a1, b0);
        } else {
            const int s0 = nkt & 1;
            load_step(s0);
            load_step(1 - s0);
            wait_and_barrier<8>();
            read_a(a0, 0, s0);
            // Phase 1 refills the half just read: only after a barrier that every
            // wave reaches with its reads returned.
            wait_and_barrier<8>();
            // Waves 4-7 run half a phase behind waves 0-3.
            if (wm == 1)
                plain_barrier();
            for (int kt = 2 - s0; kt < nkt; kt += 2) {
                if (kt > 1)
                    step(IC<0>{}, IC<0>{});
                step(IC<1>{}, IC<0>{});
            }
            step(IC<0>{}, IC<1>{});
            step(IC<1>{}, IC<2>{});
            if (wm == 0)
                plain_barrier();
        }

        // Accumulator (ha, hb, i, j), register e: row m = 128 ha + 64 wm + 16 i +
        // l16, column n = 128 hb + 32 wn + 16 j + 4 g + e of the tile.
        const int el = fresh(lane), el16 = el & 15, eg = el >> 4;
        auto finish = [&](auto put) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int ha = x >> 3, i = (x >> 1) & 3, hb = x & 1;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    put(128 * ha + 64 * wm + 16 * i + el16, 128 * hb + 32 * wn + 16 * j + 4 * eg,
                        acc[ha][hb][i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        finish_part<256>(op, part, lds, place, tid, finish);
        if (!part.more())
            return;
        part.next(op);
        __syncthreads();
    }
}

// 128 x 128 tiles for gradients whose large tiles would leave CUs idle: a
// phase of 16 products of every wave per K step, four stages of which three
// are in flight (128 KiB).
__global__ void __launch_bounds__(512, 1)
wgrad_small_kernel(WgradOperands op)
{
    constexpr int SUB = 64 * 64, STAGE = 4 * SUB, NST = 4;  // elements
    __shared__ __attribute__((aligned(1024))) uint16_t lds[NST * STAGE];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int wm = wave >> 2, wn = wave & 3;
    WgradLoads at;
    const uint32_t lds0 = lds_base_sgpr(lds) + 1024u * wave;
    auto load_step = [&](int st) __attribute__((always_inline)) {
        const uint32_t l = lds0 + 2u * STAGE * st;
        at.load_a(0, l);
        at.load_a(1, l + 2u * SUB);
        at.load_b(0, l + 4u * SUB);
        at.load_b(1, l + 6u * SUB);
        at.next();
    };
    const int e4 = l16 >> 2, c4 = l16 & 3;
    int fa[2], fb[4];  // element offsets in a stage
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
        fa[kk] = wm * SUB + 64 * l16 + (((4 * kk + g) ^ row_swz(l16)) << 3);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        fb[j] = (2 + (wn >> 1)) * SUB +
                tile_off<64>(8 * g + 4 * (j & 1) + e4, 32 * (wn & 1) + 16 * (j >> 1) + 4 * c4);
    f32x4 acc[4][2];
    WgradParts part;
    part.init(op, static_cast<int>(blockIdx.x));
    for (;;) {
        const WgradPlace place = wgrad_place<128>(op, part.tile);
        const int nkt = part.count;
        at.init(op, place, part.first * 64LL, wave, fresh(lane));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = f32x4{};
        const int first = min(nkt, NST - 1);
        for (int kt = 0; kt < first; ++kt)
            load_step(kt);
        if (nkt > NST - 2)
            wait_and_barrier<4 * (NST - 2)>();
        else
            wait_and_barrier<0>();
        if (wm == 1)
            plain_barrier();
        int rs = 0, ws = NST - 1;  // the stages read and refilled by a step
        for (int kt = 0; kt < nkt; ++kt) {
            const uint16_t *st = lds + rs * STAGE;
            bf16x8 a[4][2], b[2][2];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    b[j][kk] = join(lds_tr4(st + fb[2 * j] + 2048 * kk),
                                    lds_tr4(st + fb[2 * j + 1] + 2048 * kk));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i][kk] = lds_row8(st + fa[kk] + 1024 * i);
            }
            // The stage that the step before has read is refilled; before the
            // next step starts, its own loads have to be there (the steps after
            // it may be in flight).
            const int ahead = nkt - 1 - kt;  // steps after this one
            if (ahead >= NST - 1) {
                load_step(ws);
                wait_and_barrier<4 * (NST - 2)>();
            } else if (ahead == 2) {
                wait_and_barrier<4>();
            } else {
                wait_and_barrier<0>();
            }
            ws = rs;
            rs = rs + 1 == NST ? 0 : rs + 1;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = mfma16w(b[j][kk], a[i][kk], acc[i][j]);  // rows n, columns m
            __builtin_amdgcn_s_setprio(0);
            plain_barrier();
        }
        if (wm == 0)
            plain_barrier();

        // Accumulator (i, j), register e: row m = 64 wm + 16 i + l16, column n =
        // 32 wn + 16 j + 4 g + e of the tile.
        const int el = fresh(lane), el16 = el & 15, eg = el >> 4;
        auto finish = [&](auto put) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    put(64 * wm + 16 * i + el16, 32 * wn + 16 * j + 4 * eg, acc[i][j]);
        };
        finish_part<128>(op, part, lds, place, tid, finish);
        if (!part.more())
            return;
        part.next(op);
        __syncthreads();
    }
}

// dW of the shared tiles: the sum of a tile's parts, 8 elements per thread.
template <int EDGE>
__global__ void __launch_bounds__(256)
wgrad_sum_kernel(WgradOperands op)
{
    constexpr int PER = EDGE * EDGE / 8 / 256;  // workgroups per tile
    const int tile = static_cast<int>(blockIdx.x) / PER;
    const int v = static_cast<int>(blockIdx.x) % PER * 256 + threadIdx.x;
    const WgradPlace place = wgrad_place<EDGE>(op, op.whole + tile);
    const int m = place.m0 + v / (EDGE / 8), n = place.n0 + v % (EDGE / 8) * 8;
    if (m >= op.M || n >= op.N)
        return;
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
    auto add = [&](int slot) {
        const float *p = op.P + static_cast<long long>(slot) * (EDGE * EDGE) + v * 8;
        s0 += *reinterpret_cast<const f32x4 *>(p);
        s1 += *reinterpret_cast<const f32x4 *>(p + 4);
    };
    for (int slot = tile; slot < op.firsts; slot += op.shared)
        add(slot);
    // The tails that touch this tile, and which of their parts it is.
    if (op.rest > 0) {
        const int w0 = tile * op.rest / op.head, w1 = ((tile + 1) * op.rest - 1) / op.head;
        for (int w = w0; w <= w1; ++w)
            add(op.firsts + w * op.most + tile - w * op.head / op.rest);
    }
    *reinterpret_cast<bf16x8 *>(pick3(op.dW, place.i) + m * op.ldw + n) =
        join(pack4(s0[0], s0[1], s0[2], s0[3]), pack4(s1[0], s1[1], s1[2], s1[3]));
}

namespace {

// The workspace's parts, in bytes: XT, then the parts of the shared tiles.
struct WgradSpace {
    WgradPlan plan;
    size_t restored, partials;
};

WgradSpace wgrad_space(int T, int M, int N, int n)
{
    const WgradPlan p = wgrad_plan(T, M, N, n, device_cu_count());
    return WgradSpace{p, static_cast<size_t>(p.tiles_m) * p.edge * p.steps * 128,
                      static_cast<size_t>(p.partials()) * p.edge * p.edge * sizeof(float)};
}

}  // namespace

size_t wgrad_i8_workspace_bytes(int T, int M, int N, int n)
{
    const WgradSpace w = wgrad_space(T, M, N, n);
    return w.restored + w.partials;
}

int launch_wgrad_i8(const WgradI8Args &a)
{
    hipStream_t st = static_cast<hipStream_t>(a.stream);
    const WgradSpace w = wgrad_space(a.T, a.M, a.N, a.n);
    const WgradPlan &p = w.plan;
    const long long Tp = p.steps * 64LL;
    auto *xt = static_cast<uint16_t *>(a.workspace);
    auto *parts = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + w.restored);
    hipError_t e = launch_kernel(restore_kernel,
                                 dim3(static_cast<unsigned>((Tp + 127) / 128),
                                      static_cast<unsigned>((a.M + 127) / 128)),
                                 dim3(256), st, static_cast<const int8_t *>(a.Q), a.ldq, a.scales,
                                 xt, Tp, a.T, a.M);
    if (e != hipSuccess)
        return DD_ERR_HIP;
    const int shared = p.heads ? p.shared() : 0;
    WgradOperands op{};
    op.XT = xt;
    for (int i = 0; i < a.n; ++i) {
        op.dY[i] = static_cast<const uint16_t *>(a.dY[i]);
        op.dW[i] = static_cast<uint16_t *>(a.dW[i]);
    }
    op.P = parts;
    op.Tp = Tp;
    op.ldy = a.ldy;
    op.ldw = a.ldw;
    op.T = a.T;
    op.M = a.M;
    op.N = a.N;
    op.tiles_m = p.tiles_m;
    op.tiles_n = p.tiles_n;
    op.cols = p.tiles_n / a.n;
    op.xm = tile_rows_step(p.tiles_m, p.tiles_n);
    op.whole = p.whole;
    op.shared = shared;
    op.firsts = p.heads * shared;
    op.steps = p.steps;
    op.head = p.head;
    op.rest = p.rest();
    op.most = p.most();
    const unsigned wgs = static_cast<unsigned>(p.whole + op.firsts + p.tails);
    e = launch_kernel(p.edge == 256 ? wgrad_kernel : wgrad_small_kernel, dim3(wgs), dim3(512), st, op);
    if (e != hipSuccess || !shared)
        return e == hipSuccess ? DD_OK : DD_ERR_HIP;
    e = p.edge == 256 ? launch_kernel(wgrad_sum_kernel<256>, dim3(shared * 32u), dim3(256), st, op)
                      : launch_kernel(wgrad_sum_kernel<128>, dim3(shared * 8u), dim3(256), st, op);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
