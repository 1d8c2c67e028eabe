// dd_api8.cpp -- the C ABI entry points of the 8-bit operators (include/dd_attn.h):
// RMSNorm, codes and their values, int8 products, weight gradients from codes.
//
// Host-only C++, as dd_api.cpp: every check runs before any launch, so an
// invalid call leaves all outputs untouched.
#include "dd_attn.h"
#include "dd_check.hpp"
#include "dd_internal.h"

#include <cmath>
#include <initializer_list>

using namespace dd::check;

namespace {

// Row strides below this keep a tile's per-lane byte offsets in 32 bits.
constexpr long long kMaxStride = 1LL << 23;
// 64 x 64 tiles of the largest grids (at most 512 work-items per tile, fewer
// than 2^32 in a dispatch).
constexpr long long kMaxTiles = (1LL << 23) - 1;

long long tiles64(long long M, long long N) { return (M + 63) / 64 * ((N + 63) / 64); }

bool rows_ok(int rows, int d)
{
    return rows >= 1 && d >= 1 && d <= 16384 && static_cast<long long>(rows) * d < (1LL << 40);
}

// Outputs apart from inputs and from each other.
int check_apart(std::initializer_list<Range> ins, std::initializer_list<Range> outs)
{
    for (const Range *o = outs.begin(); o != outs.end(); ++o) {
        for (Range in : ins)
            if (overlaps(*o, in))
                return DD_ERR_ALIAS;
        for (const Range *p = outs.begin(); p != o; ++p)
            if (overlaps(*o, *p))
                return DD_ERR_ALIAS;
    }
    return DD_OK;
}

bool aligned_all(std::initializer_list<const void *> ps, uintptr_t n)
{
    for (const void *p : ps)
        if (!aligned(p, n))
            return false;
    return true;
}

// The two forms of the norm: Y, or Q and scales.
int norm_checked(const void *X, long long ldx, const void *R, long long ldr, const void *w, void *H,
                 void *Y, int8_t *Q, long long ldq, float *scales, float *rstd, int rows, int d,
                 float eps, void *stream)
{
    if (!X || !w || !rstd || (R == nullptr) != (H == nullptr))
        return DD_ERR_NULL;
    if (!rows_ok(rows, d) || ldx < d || (R && ldr < d) || (Q && ldq < d) ||
        !(std::isfinite(eps) && eps > 0.0f))
        return DD_ERR_SHAPE;
    if (!aligned_all({X, R, w, H, Y}, 2) || !aligned_all({rstd, scales}, 4))
        return DD_ERR_ALIGN;
    const size_t tb = matrix_bytes(rows, d, d, 2), sb = static_cast<size_t>(rows) * 4;
    const int st = check_apart(
        {range_of(X, matrix_bytes(rows, d, ldx, 2)),
         range_of(R, R ? matrix_bytes(rows, d, ldr, 2) : 0), range_of(w, d * 2UL)},
        {range_of(H, H ? tb : 0), range_of(Y, Y ? tb : 0),
         range_of(Q, Q ? matrix_bytes(rows, d, ldq, 1) : 0), range_of(scales, scales ? sb : 0),
         range_of(rstd, sb)});
    if (st != DD_OK)
        return st;
    return dd::launch_rows(dd::RowArgs{X, R, w, H, Y, Q, scales, rstd, ldx, R ? ldr : 0, Q ? ldq : 0,
                                       rows, d, eps, stream});
}

}  // namespace

extern "C" {

int dd_rmsnorm_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *w,
                   void *H, void *Y, float *rstd, int rows, int d, float eps, void *stream)
{
    if (!Y)
        return DD_ERR_NULL;
    return norm_checked(X, ldx, R, ldr, w, H, Y, nullptr, 0, nullptr, rstd, rows, d, eps, stream);
}

int dd_rmsnorm_int8_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *w,
                        void *H, int8_t *Q, long long ldq, float *scales, float *rstd, int rows,
                        int d, float eps, void *stream)
{
    if (!Q || !scales)
        return DD_ERR_NULL;
    return norm_checked(X, ldx, R, ldr, w, H, nullptr, Q, ldq, scales, rstd, rows, d, eps, stream);
}

size_t dd_rmsnorm_bwd_workspace_bytes(int rows, int d)
{
    return rows_ok(rows, d) ? dd::rmsnorm_workspace_bytes(rows, d) : 0;
}

int dd_rmsnorm_bwd(const void *H, const void *w, const float *rstd, const void *dY,
                   const void *dRes, void *dX, void *dw, int rows, int d, void *workspace,
                   size_t workspace_bytes, void *stream)
{
    if (!H || !w || !rstd || !dY || !dX || !dw)
        return DD_ERR_NULL;
    if (!rows_ok(rows, d))
        return DD_ERR_SHAPE;
    const size_t need = dd::rmsnorm_workspace_bytes(rows, d);
    if (!workspace || workspace_bytes < need)
        return DD_ERR_WORKSPACE;
    if (!aligned_all({H, w, dY, dRes, dX, dw}, 2) || !aligned_all({rstd, workspace}, 4))
        return DD_ERR_ALIGN;
    const size_t tb = matrix_bytes(rows, d, d, 2);
    const int st = check_apart({range_of(H, tb), range_of(w, d * 2UL),
                                range_of(rstd, static_cast<size_t>(rows) * 4), range_of(dY, tb),
                                range_of(dRes, dRes ? tb : 0)},
                               {range_of(dX, tb), range_of(dw, d * 2UL), range_of(workspace, need)});
    if (st != DD_OK)
        return st;
    return dd::launch_rmsnorm_bwd(
        dd::RmsBackArgs{H, w, dY, dRes, rstd, dX, dw, workspace, rows, d, stream});
}

int dd_quantize(const void *X, long long ldx, int8_t *Q, long long ldq, float *scales, int rows,
                int d, void *stream)
{
    if (!X || !Q || !scales)
        return DD_ERR_NULL;
    if (!rows_ok(rows, d) || ldx < d || ldq < d)
        return DD_ERR_SHAPE;
    if (!aligned(X, 2) || !aligned(scales, 4))
        return DD_ERR_ALIGN;
    const int st = check_apart({range_of(X, matrix_bytes(rows, d, ldx, 2))},
                               {range_of(Q, matrix_bytes(rows, d, ldq, 1)),
                                range_of(scales, static_cast<size_t>(rows) * 4)});
    if (st != DD_OK)
        return st;
    return dd::launch_rows(dd::RowArgs{X, nullptr, nullptr, nullptr, nullptr, Q, scales, nullptr,
                                       ldx, 0, ldq, rows, d, 0.0f, stream});
}

int dd_dequantize(const int8_t *Q, long long ldq, const float *scales, void *Y, long long ldy,
                  int rows, int d, void *stream)
{
    if (!Q || !scales || !Y)
        return DD_ERR_NULL;
    if (!rows_ok(rows, d) || ldq < d || ldy < d)
        return DD_ERR_SHAPE;
    if (!aligned(Y, 2) || !aligned(scales, 4))
        return DD_ERR_ALIGN;
    const int st = check_apart({range_of(Q, matrix_bytes(rows, d, ldq, 1)),
                                range_of(scales, static_cast<size_t>(rows) * 4)},
                               {range_of(Y, matrix_bytes(rows, d, ldy, 2))});
    if (st != DD_OK)
        return st;
    return dd::launch_dequantize(dd::DequantizeArgs{Q, scales, Y, ldq, ldy, rows, d, stream});
}

int dd_gemm_i8(const int8_t *A, long long lda, const float *sa, const int8_t *B, long long ldb,
               const float *sb, const void *R, void *C, long long ldc, int M, int N, int K,
               void *stream)
{
    if (!A || !sa || !B || !sb || !C)
        return DD_ERR_NULL;
    if (M < 1 || N < 1 || K < 16 || K % 16 || K >= (1 << 17) || tiles64(M, N) > kMaxTiles ||
        lda < K || ldb < K || ldc < N || lda >= kMaxStride || ldb >= kMaxStride)
        return DD_ERR_SHAPE;
    if (lda % 16 || ldb % 16 || !aligned_all({A, B}, 16) || !aligned_all({sa, sb}, 4) ||
        !aligned_all({R, C}, 2))
        return DD_ERR_ALIGN;
    const Range c = range_of(C, matrix_bytes(M, N, ldc, 2)), r = range_of(R, R ? c.hi - c.lo : 0);
    int st = check_apart({range_of(A, matrix_bytes(M, K, lda, 1)),
                          range_of(B, matrix_bytes(N, K, ldb, 1)),
                          range_of(sa, static_cast<size_t>(M) * 4),
                          range_of(sb, static_cast<size_t>(N) * 4)},
                         {c});
    if (st == DD_OK && R != C)
        st = check_apart({r}, {c});
    if (st != DD_OK)
        return st;
    return dd::launch_gemm_i8(
        dd::GemmI8Args{A, B, R, sa, sb, C, lda, ldb, ldc, M, N, K, stream});
}

namespace {

// T: the restored input's rows have to keep 32-bit offsets too (64 of them).
// M: a grid over its parts of 128 in y, fewer than 2^16.
bool wgrad_ok(int T, int M, int N, int n)
{
    return n >= 1 && n <= 3 && T >= 1 && T <= (1 << 25) - 64 && M >= 8 && N >= 8 && M % 8 == 0 &&
           M <= (1 << 23) - 128 && N % 8 == 0 && n * tiles64(M, N) <= kMaxTiles;
}

}  // namespace

size_t dd_gemm_i8_wgrad_workspace_bytes(int T, int M, int N, int n)
{
    return wgrad_ok(T, M, N, n) ? dd::wgrad_i8_workspace_bytes(T, M, N, n) : 0;
}

int dd_gemm_i8_wgrad(const int8_t *Q, long long ldq, const float *scales, const void *const *dY,
                     long long ldy, void *const *dW, long long ldw, int n, int T, int M, int N,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q || !scales || !dY || !dW)
        return DD_ERR_NULL;
    if (!wgrad_ok(T, M, N, n) || ldq < M || ldy < N || ldw < N || ldq >= kMaxStride ||
        ldy >= kMaxStride)
        return DD_ERR_SHAPE;
    for (int i = 0; i < n; ++i)
        if (!dY[i] || !dW[i])
            return DD_ERR_NULL;
    if (ldq % 8 || ldy % 8 || ldw % 8 || !aligned(Q, 8) || !aligned(scales, 4))
        return DD_ERR_ALIGN;
    for (int i = 0; i < n; ++i)
        if (!aligned_all({dY[i], dW[i]}, 16))
            return DD_ERR_ALIGN;
    const size_t need = dd::wgrad_i8_workspace_bytes(T, M, N, n);
    if (need && (!workspace || workspace_bytes < need))
        return DD_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16))
        return DD_ERR_ALIGN;
    const Range q = range_of(Q, matrix_bytes(T, M, ldq, 1)),
                sc = range_of(scales, static_cast<size_t>(T) * 4), ws = range_of(workspace, need);
    const size_t wb = matrix_bytes(M, N, ldw, 2);
    int st = check_apart({q, sc}, {ws});
    for (int i = 0; i < n && st == DD_OK; ++i) {
        const Range w = range_of(dW[i], wb), y = range_of(dY[i], matrix_bytes(T, N, ldy, 2));
        st = check_apart({q, sc, ws}, {w});
        if (st == DD_OK)
            st = check_apart({y}, {ws});
        for (int j = 0; j < n && st == DD_OK; ++j) {
            const Range v = range_of(dW[j], wb);
            if (overlaps(v, y))
                st = DD_ERR_ALIAS;
            // Outputs may be column slices of one matrix: they are apart if
            // their columns are.
            if (j < i && overlaps(v, w)) {
                const long long shift =
                    static_cast<long long>(w.lo < v.lo ? v.lo - w.lo : w.lo - v.lo) / 2 % ldw;
                if (shift < N || shift + N > ldw)
                    st = DD_ERR_ALIAS;
            }
        }
    }
    if (st != DD_OK)
        return st;
    dd::WgradI8Args a{Q, {}, scales, {}, workspace, ldq, ldy, ldw, n, T, M, N, stream};
    for (int i = 0; i < n; ++i) {
        a.dY[i] = dY[i];
        a.dW[i] = dW[i];
    }
    return dd::launch_wgrad_i8(a);
}

}  // extern "C"
