// dd_api_cache.cpp -- the C ABI entry points of the paged cache and of the
// log probabilities (include/dd_attn.h).
//
// Host-only C++, as dd_api.cpp: every check runs before any launch, so an
// invalid call leaves all outputs untouched.
#include "dd_attn.h"
#include "dd_check.hpp"
#include "dd_internal.h"

#include <cmath>
#include <vector>

using namespace dd::check;

namespace {

// DD_OK, or what is wrong with the sizes of a cache and a chunk (T >= 1).
int shape_status(int T, int B, int H, int Hkv, int D, int pages, int page, int per)
{
    if (D != 64 && D != 128)
        return DD_ERR_HEADDIM;
    if (T < 1 || B < 1 || H < 1 || Hkv < 1 || H % Hkv || pages < 1 || per < 1 || page < 16 ||
        page > 1024 || (page & (page - 1)))
        return DD_ERR_SHAPE;
    if (T > (1 << 23) || static_cast<long long>(T) * H > (1LL << 26) ||
        static_cast<long long>(H) * D >= (1LL << 23) ||
        static_cast<long long>(B) * Hkv > 65535 ||
        static_cast<long long>(per) * page >= (1LL << 30))
        return DD_ERR_SHAPE;
    return DD_OK;
}

dd::CacheShape shape(const int32_t *table, const int32_t *lens, const int32_t *cu_new, int T, int B,
                     int Hkv, int D, int pages, int page, int per)
{
    int shift = 0;
    while (1 << shift < page)
        ++shift;
    return dd::CacheShape{table, lens, cu_new, T, B, Hkv, D, pages, shift, per};
}

Range pages_of(const void *p, int Hkv, int D, int pages, int page)
{
    return range_of(p, static_cast<size_t>(pages) * Hkv * page * D * 2);
}

Range words(const void *p, long long n) { return range_of(p, p ? static_cast<size_t>(n) * 4 : 0); }

template <int NI, int NO>
int check_apart(const Range (&ins)[NI], const Range (&outs)[NO])
{
    for (int o = 0; o < NO; ++o) {
        for (const Range &in : ins)
            if (overlaps(outs[o], in))
                return DD_ERR_ALIAS;
        for (int p = 0; p < o; ++p)
            if (overlaps(outs[o], outs[p]))
                return DD_ERR_ALIAS;
    }
    return DD_OK;
}

bool rows_ok(int rows, int V, int top, long long ldx)
{
    return rows >= 1 && rows <= (1 << 23) && V >= 1 && V <= (1 << 30) && top >= 0 && top <= 64 &&
           top <= V && ldx >= V && ldx < (1LL << 40) &&
           rows * ((V + 8191LL) / 8192) < (1LL << 24);
}

}  // namespace

extern "C" {

int dd_cache_check(const int32_t *host_table, const int32_t *host_lens, const int32_t *host_cu_new,
                   int T, int B, int pages, int page, int per)
{
    if (!host_table || !host_lens)
        return DD_ERR_NULL;
    if (T < 0 || B < 1 || pages < 1 || per < 1 || page < 16 || page > 1024 || (page & (page - 1)) ||
        static_cast<long long>(per) * page >= (1LL << 30))
        return DD_ERR_SHAPE;
    if (host_cu_new && (host_cu_new[0] != 0 || host_cu_new[B] > T))
        return DD_ERR_CACHE;
    for (int b = 0; b < B; ++b) {
        const long long n =
            host_cu_new ? static_cast<long long>(host_cu_new[b + 1]) - host_cu_new[b] : 0;
        if (n < 0 || host_lens[b] < 0 || host_lens[b] + n > static_cast<long long>(per) * page)
            return DD_ERR_CACHE;
    }
    // every page in use once
    try {
        std::vector<bool> used(static_cast<size_t>(pages), false);
        for (int b = 0; b < B; ++b) {
            const long long n = host_cu_new ? host_cu_new[b + 1] - host_cu_new[b] : 0;
            const long long slots = host_lens[b] + n;
            for (long long i = 0; i * page < slots; ++i) {
                const int32_t id = host_table[static_cast<long long>(b) * per + i];
                if (id < 0 || id >= pages || used[static_cast<size_t>(id)])
                    return DD_ERR_CACHE;
                used[static_cast<size_t>(id)] = true;
            }
        }
    } catch (...) {  // no memory for the marks
        return DD_ERR_SHAPE;
    }
    return DD_OK;
}

int dd_cache_append(const void *Q, long long ldq, const void *K, long long ldk, const void *V,
                    long long ldv, void *Qrot, void *Kp, void *Vp, int32_t *positions,
                    const int32_t *table, const int32_t *lens, const int32_t *start,
                    const int32_t *cu_new, int T, int B, int H, int Hkv, int D, int pages, int page,
                    int per, float rope_base, void *stream)
{
    if (!K || !V || !Kp || !Vp || !table || !lens || !cu_new || (Q == nullptr) != (Qrot == nullptr))
        return DD_ERR_NULL;
    const int st0 = shape_status(T, B, H, Hkv, D, pages, page, per);
    if (st0 != DD_OK)
        return st0;
    const long long dq = static_cast<long long>(H) * D, dk = static_cast<long long>(Hkv) * D;
    const bool rope = rope_base != 0.0f;
    if ((Q && (ldq < dq || ldq >= (1LL << 31))) || ldk < dk || ldv < dk || ldk >= (1LL << 31) ||
        ldv >= (1LL << 31) || (Q && !rope) ||
        (rope && !(std::isfinite(rope_base) && rope_base > 0.0f)))
        return DD_ERR_SHAPE;
    if ((Q && ldq % 8) || ldk % 8 || ldv % 8 || !aligned(Q, 16) || !aligned(Qrot, 16) ||
        !aligned(K, 16) || !aligned(V, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) ||
        !aligned(positions, 4) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(start, 4) ||
        !aligned(cu_new, 4))
        return DD_ERR_ALIGN;
    const Range q = range_of(Q, Q ? matrix_bytes(T, dq, ldq, 2) : 0);
    const Range qr = range_of(Qrot, Qrot ? matrix_bytes(T, dq, dq, 2) : 0);
    const bool in_place = Q && Q == Qrot && ldq == dq;
    const int st = check_apart(
        {in_place ? Range{0, 0} : q, range_of(K, matrix_bytes(T, dk, ldk, 2)),
         range_of(V, matrix_bytes(T, dk, ldv, 2)), words(table, static_cast<long long>(B) * per),
         words(lens, B), words(start, B), words(cu_new, B + 1)},
        {qr, pages_of(Kp, Hkv, D, pages, page), pages_of(Vp, Hkv, D, pages, page),
         words(positions, static_cast<long long>(B) * Hkv * per * page)});
    if (st != DD_OK)
        return st;
    return dd::launch_cache_append(
        dd::CacheAppendArgs{shape(table, lens, cu_new, T, B, Hkv, D, pages, page, per), Q, K, V,
                            Qrot, Kp, Vp, positions, start, ldq, ldk, ldv, H, rope_base, stream});
}

size_t dd_cache_attn_workspace_bytes(int T, int B, int H, int Hkv, int D, int page, int per,
                                     int weights)
{
    if (shape_status(T, B, H, Hkv, D, 1, page, per) != DD_OK)
        return 0;
    return dd::cache_attn_workspace_bytes(
        shape(nullptr, nullptr, nullptr, T, B, Hkv, D, 1, page, per), H, weights != 0);
}

int dd_cache_attn_fwd(const void *Q, long long ldq, const void *Kp, const void *Vp,
                      const int32_t *table, const int32_t *lens, const int32_t *cu_new, void *O,
                      float *LSE, const float *W_in, float *W_out, int T, int B, int H, int Hkv,
                      int D, int pages, int page, int per, void *workspace, size_t workspace_bytes,
                      void *stream)
{
    if (!Q || !Kp || !Vp || !table || !lens || !cu_new || !O || !LSE ||
        (W_in == nullptr) != (W_out == nullptr))
        return DD_ERR_NULL;
    const int st0 = shape_status(T, B, H, Hkv, D, pages, page, per);
    if (st0 != DD_OK)
        return st0;
    const long long dq = static_cast<long long>(H) * D;
    if (ldq < dq || ldq >= (1LL << 31))
        return DD_ERR_SHAPE;
    if (ldq % 8 || !aligned(Q, 16) || !aligned(Kp, 16) || !aligned(Vp, 16) || !aligned(O, 16) ||
        !aligned(LSE, 4) || !aligned(W_in, 4) || !aligned(W_out, 4) || !aligned(table, 4) ||
        !aligned(lens, 4) || !aligned(cu_new, 4))
        return DD_ERR_ALIGN;
    const dd::CacheShape c = shape(table, lens, cu_new, T, B, Hkv, D, pages, page, per);
    const size_t need = dd::cache_attn_workspace_bytes(c, H, W_out != nullptr);
    if (need && (!workspace || workspace_bytes < need))
        return DD_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16))
        return DD_ERR_ALIGN;
    const long long slots = static_cast<long long>(B) * Hkv * per * page;
    const int st = check_apart(
        {range_of(Q, matrix_bytes(T, dq, ldq, 2)), pages_of(Kp, Hkv, D, pages, page),
         pages_of(Vp, Hkv, D, pages, page), words(table, static_cast<long long>(B) * per),
         words(lens, B), words(cu_new, B + 1),
         W_in == W_out ? Range{0, 0} : words(W_in, slots)},
        {range_of(O, matrix_bytes(T, dq, dq, 2)), words(LSE, static_cast<long long>(T) * H),
         words(W_out, slots), need ? range_of(workspace, need) : Range{0, 0}});
    if (st != DD_OK)
        return st;
    return dd::launch_cache_attn(
        dd::CacheAttnArgs{c, Q, Kp, Vp, O, LSE, W_in, W_out, ldq, H, workspace, stream});
}

size_t dd_cache_evict_workspace_bytes(int B, int Hkv, int D, int page, int per, int budget,
                                      int in_place)
{
    if (shape_status(1, B, Hkv, Hkv, D, 1, page, per) != DD_OK || budget < 1)
        return 0;
    return dd::cache_evict_workspace_bytes(
        shape(nullptr, nullptr, nullptr, 1, B, Hkv, D, 1, page, per), budget, in_place != 0);
}

int dd_cache_evict(void *Kp, void *Vp, const int32_t *table, const int32_t *lens, const float *W_in,
                   const int32_t *P_in, const int32_t *seen, float *W_out, int32_t *P_out,
                   int32_t *lens_out, int B, int Hkv, int D, int pages, int page, int per,
                   int budget, int recent, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Kp || !Vp || !table || !lens || !W_in || !P_in || !seen || !W_out || !P_out || !lens_out)
        return DD_ERR_NULL;
    const int st0 = shape_status(1, B, Hkv, Hkv, D, pages, page, per);
    if (st0 != DD_OK)
        return st0;
    if (budget < 1 || recent < 0 || recent > budget)
        return DD_ERR_SHAPE;
    if (!aligned(Kp, 16) || !aligned(Vp, 16) || !aligned(table, 4) || !aligned(lens, 4) ||
        !aligned(W_in, 4) || !aligned(P_in, 4) || !aligned(seen, 4) || !aligned(W_out, 4) ||
        !aligned(P_out, 4) || !aligned(lens_out, 4))
        return DD_ERR_ALIGN;
    const dd::CacheShape c = shape(table, lens, nullptr, 1, B, Hkv, D, pages, page, per);
    const size_t need = dd::cache_evict_workspace_bytes(c, budget, lens == lens_out);
    if (need && (!workspace || workspace_bytes < need))
        return DD_ERR_WORKSPACE;
    if (need && !aligned(workspace, 4))
        return DD_ERR_ALIGN;
    const long long slots = static_cast<long long>(B) * Hkv * per * page;
    // each state in place, or apart
    const Range none{0, 0};
    const int st = check_apart(
        {words(table, static_cast<long long>(B) * per), lens == lens_out ? none : words(lens, B),
         W_in == W_out ? none : words(W_in, slots), P_in == P_out ? none : words(P_in, slots),
         words(seen, B)},
        {pages_of(Kp, Hkv, D, pages, page), pages_of(Vp, Hkv, D, pages, page), words(W_out, slots),
         words(P_out, slots), words(lens_out, B), need ? range_of(workspace, need) : Range{0, 0}});
    if (st != DD_OK)
        return st;
    return dd::launch_cache_evict(dd::CacheEvictArgs{c, Kp, Vp, W_in, P_in, seen, W_out, P_out,
                                                     lens_out, budget, recent, workspace, stream});
}

size_t dd_logprobs_workspace_bytes(int rows, int V, int top)
{
    return rows_ok(rows, V, top, V) ? dd::logprobs_workspace_bytes(rows, V, top) : 0;
}

int dd_logprobs_fwd(const void *X, long long ldx, int f32, const int64_t *targets, float *logp,
                    float *entropy, float *lse, float *top_logp, int64_t *top_ids, int rows, int V,
                    int top, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !targets || !logp || !entropy || !lse || (top > 0 && (!top_logp || !top_ids)))
        return DD_ERR_NULL;
    if (!rows_ok(rows, V, top, ldx))
        return DD_ERR_SHAPE;
    const int size = f32 ? 4 : 2;
    if (!aligned(X, size) || !aligned(targets, 8) || !aligned(logp, 4) || !aligned(entropy, 4) ||
        !aligned(lse, 4) || (top && (!aligned(top_logp, 4) || !aligned(top_ids, 8))))
        return DD_ERR_ALIGN;
    const size_t need = dd::logprobs_workspace_bytes(rows, V, top);
    if (need && (!workspace || workspace_bytes < need))
        return DD_ERR_WORKSPACE;
    if (need && !aligned(workspace, 8))
        return DD_ERR_ALIGN;
    const long long n = static_cast<long long>(rows) * top;
    const int st = check_apart(
        {range_of(X, matrix_bytes(rows, V, ldx, size)), words(targets, 2LL * rows)},
        {words(logp, rows), words(entropy, rows), words(lse, rows), words(top ? top_logp : nullptr, n),
         words(top ? top_ids : nullptr, 2 * n), need ? range_of(workspace, need) : Range{0, 0}});
    if (st != DD_OK)
        return st;
    return dd::launch_logprobs(dd::LogprobArgs{X, targets, logp, entropy, lse, top_logp, top_ids,
                                               ldx, rows, V, top, f32 != 0, workspace, stream});
}

int dd_logprobs_bwd(const void *X, long long ldx, int f32, const int64_t *targets, const float *lse,
                    const float *entropy, const float *g_logp, const float *g_entropy,
                    const float *g_lse, void *dX, long long lddx, int rows, int V, void *stream)
{
    if (!X || !targets || !lse || !entropy || !dX)
        return DD_ERR_NULL;
    if (!rows_ok(rows, V, 0, ldx) || lddx < V || lddx >= (1LL << 40))
        return DD_ERR_SHAPE;
    const int size = f32 ? 4 : 2;
    if (!aligned(X, size) || !aligned(dX, size) || !aligned(targets, 8) || !aligned(lse, 4) ||
        !aligned(entropy, 4) || !aligned(g_logp, 4) || !aligned(g_entropy, 4) || !aligned(g_lse, 4))
        return DD_ERR_ALIGN;
    const Range x = range_of(X, matrix_bytes(rows, V, ldx, size));
    const int st = check_apart({X == dX && ldx == lddx ? Range{0, 0} : x, words(targets, 2LL * rows),
                                words(lse, rows), words(entropy, rows), words(g_logp, rows),
                                words(g_entropy, rows), words(g_lse, rows)},
                               {range_of(dX, matrix_bytes(rows, V, lddx, size))});
    if (st != DD_OK)
        return st;
    return dd::launch_logprobs_bwd(dd::LogprobBackArgs{X, targets, lse, entropy, g_logp, g_entropy,
                                                       g_lse, dX, ldx, lddx, rows, V, f32 != 0,
                                                       stream});
}

}  // extern "C"
