// dd_gemm_i8.hip -- products of 8-bit integers on the matrix cores:
//   C[m, n] = bf16( sa[m] sb[n] sum over k of A[m, k] B[n, k]  (+ R[m, n]) ),
// A [M][K] and B [N][K] int8 with K innermost, sa an fp32 scale per row of A (a
// token), sb one per row of B (an output channel).  The sum is exact in int32
// (K < 2^17); it is scaled and the residual added in fp32, with one rounding to
// bf16 at the end.  Any M, N and K (a multiple of 16).
#include "dd_device.hpp"
#include "dd_internal.h"
#include "dd_launch.hpp"
#include "dd_attn.h"

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

struct GemmI8Operands {
    const int8_t *A, *B;
    const float *sa, *sb;
    const uint16_t *R;
    uint16_t *C;
    long long lda, ldb, ldc;
    int M, N, K, tiles_n;
};

// One workgroup per 64 x 64 tile, 32 x 32 per wave, operands straight from
// memory.
__global__ void __launch_bounds__(256)
gemm_i8_kernel(GemmI8Operands op)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
    const int m0 = static_cast<int>(blockIdx.x) / op.tiles_n * 64 + (wave >> 1) * 32;
    const int n0 = static_cast<int>(blockIdx.x) % op.tiles_n * 64 + (wave & 1) * 32;
    const int8_t *pa[2], *pb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        pa[i] = op.A + min(m0 + 16 * i + l16, op.M - 1) * op.lda;
        pb[i] = op.B + min(n0 + 16 * i + l16, op.N - 1) * op.ldb;
    }
    i32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < op.K; k0 += 64) {
        const int k = k0 + 16 * g;
        u32x4 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = b[i] = u32x4{0u, 0u, 0u, 0u};
            if (k < op.K) {
                a[i] = *reinterpret_cast<const u32x4 *>(pa[i] + k);
                b[i] = *reinterpret_cast<const u32x4 *>(pb[i] + k);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = mfma_i8(b[j], a[i], acc[i][j]);  // rows n, columns m
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = m0 + 16 * i + l16, n = n0 + 16 * j + 4 * g + e;
                if (m >= op.M || n >= op.N)
                    continue;
                const long long at = m * op.ldc + n;
                float c = static_cast<float>(acc[i][j][e]) * op.sa[m] * op.sb[n];
                if (op.R != nullptr)
                    c += __uint_as_float(static_cast<uint32_t>(op.R[at]) << 16);
                op.C[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(c));
            }
}

int launch_gemm_i8(const GemmI8Args &a)
{
    const GemmI8Operands op{static_cast<const int8_t *>(a.A), static_cast<const int8_t *>(a.B),
                            a.sa, a.sb, static_cast<const uint16_t *>(a.R),
                            static_cast<uint16_t *>(a.C), a.lda, a.ldb, a.ldc, a.M, a.N, a.K,
                            (a.N + 63) / 64};
    const dim3 grid(static_cast<unsigned>((a.M + 63) / 64) * op.tiles_n);
    const hipError_t e =
        launch_kernel(gemm_i8_kernel, grid, dim3(256), static_cast<hipStream_t>(a.stream), op);
    return e == hipSuccess ? DD_OK : DD_ERR_HIP;
}

}  // namespace dd
