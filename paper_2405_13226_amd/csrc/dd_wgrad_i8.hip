// dd_wgrad_i8.hip -- the weight gradient of a linear layer whose input was kept
// in 8 bits:  dW[m, n] = sum over t of X[t, m] dY[t, n],  X = bf16(scales Q).
//
// The restored input is bf16, as the activation that was saved; the products
// are bf16 matrix-core products with fp32 sums.  Any T, M and N (M and N
// multiples of 8).
#include "dd_device.hpp"
#include "dd_tile.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_attn.h"

namespace dd {

struct WgradI8Operands {
    const int8_t *Q;
    const float *scales;
    const uint16_t *dY;
    uint16_t *dW;
    long long ldq, ldy, ldw;
    int T, M, N, tiles_n;
};

// One workgroup per 64 x 64 tile, 32 x 32 per wave, 64 tokens a step: both
// operands row by row (tokens) into LDS, read transposed.
__global__ void __launch_bounds__(256)
wgrad_i8_kernel(WgradI8Operands op)
{
    __shared__ __attribute__((aligned(16))) uint16_t xs[64 * 64], ys[64 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
    const int e4 = l16 >> 2, c4 = l16 & 3;
    const int m0 = static_cast<int>(blockIdx.x) / op.tiles_n * 64;
    const int n0 = static_cast<int>(blockIdx.x) % op.tiles_n * 64;
    f32x4 acc[2][2] = {};
    for (int t0 = 0; t0 < op.T; t0 += 64) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = (threadIdx.x >> 3) + 32 * i, c = (threadIdx.x & 7) * 8, t = t0 + r;
            float x[8] = {};
            u32x4 y = {0u, 0u, 0u, 0u};
            if (t < op.T && m0 + c < op.M) {
                const float s = op.scales[t];
                const u32x2 u = *reinterpret_cast<const u32x2 *>(op.Q + t * op.ldq + m0 + c);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = s * static_cast<float>(static_cast<int8_t>(u[e >> 2] >> 8 * (e & 3)));
            }
            if (t < op.T && n0 + c < op.N)
                y = *reinterpret_cast<const u32x4 *>(op.dY + t * op.ldy + n0 + c);
            *reinterpret_cast<u32x4 *>(xs + tile_off<64>(r, c)) = pack8f(x);
            *reinterpret_cast<u32x4 *>(ys + tile_off<64>(r, c)) = y;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 32 * kk + 8 * g + e4;
                const int cm = 32 * (wave >> 1) + 16 * i + 4 * c4, cn = 32 * (wave & 1) + 16 * i + 4 * c4;
                a[i] = join(lds_tr4(xs + tile_off<64>(r, cm)), lds_tr4(xs + tile_off<64>(r + 4, cm)));
                b[i] = join(lds_tr4(ys + tile_off<64>(r, cn)), lds_tr4(ys + tile_off<64>(r + 4, cn)));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = m0 + 32 * (wave >> 1) + 16 * i + l16;
            const int n = n0 + 32 * (wave & 1) + 16 * j + 4 * g;
            const f32x4 v = acc[i][j];
            if (m < op.M && n < op.N)
                *reinterpret_cast<bf16x4 *>(op.dW + m * op.ldw + n) = pack4(v[0], v[1], v[2], v[3]);
        }
}

size_t wgrad_i8_workspace_bytes(int, int, int) { return 0; }

int launch_wgrad_i8(const WgradI8Args &a)
{
    const WgradI8Operands op{static_cast<const int8_t *>(a.Q), a.scales,
                             static_cast<const uint16_t *>(a.dY), static_cast<uint16_t *>(a.dW),
                             a.ldq, a.ldy, a.ldw, a.T, a.M, a.N, (a.N + 63) / 64};
    const dim3 grid(static_cast<unsigned>((a.M + 63) / 64) * op.tiles_n);
    const hipError_t e =
        launch_kernel(wgrad_i8_kernel, grid, dim3(256), static_cast<hipStream_t>(a.stream), op);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
