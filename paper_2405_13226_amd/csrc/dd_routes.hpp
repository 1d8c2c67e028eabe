// dd_routes.hpp -- which kernel form a call takes: an attention call by the
// number of its 128-row blocks, the row length L, the mask and the number of
// CUs, a product by its sizes.  Plain C++, so that a host program can ask where
// a shape goes.
//
// Attention: groups of waves share a block's tiles.  The workgroups of a small
// grid are all resident at once, so the heaviest block's chain of tiles is the
// launch's time, and the groups shorten it.  A larger grid is balanced by dispatch (or
// by the persistent forms' walk), and the groups cost it their final sum and
// their share of a CU.  That balance is what the causal mask makes uneven and
// documents more so: without the causal mask every block has the same work, a
// grid that covers the CUs gains nothing, and the groups stop at one block per
// CU or two.
//
// The figures of the attention rules are graph-replayed times with two (or four) groups over
// those with one, per row length and blocks, causal / not causal / causal with
// documents (log-normal lengths, median 600); a rule takes the groups where
// they gain.
#pragma once

#include <algorithm>
#include <cmath>

namespace dd {

// Blocks up to which the groups pay under the causal mask: two per CU, with
// documents two and a half.  D = 128 forward: 512 blocks of 4096 0.78, 640 of
// 4096 1.10, with documents 0.77.
inline bool causal_small_grid(long long blocks, bool docs, long long cus)
{
    return 2 * blocks <= (docs ? 5 : 4) * cus;
}

// Forward: groups over a query block's key tiles.
// D = 64, up to a block per CU: L = 64 (one tile) 1.14 / 1.14 / 1.12, 128 0.97 /
// 1.06 / 0.98, 160 1.02 / 1.03 / 1.02, 256 0.92 / 0.98 / 0.92, 512 0.84 / 0.89 /
// 0.84; four groups from 769 on (L = 2048 0.70 / 0.73 / 0.69).  Up to two: L =
// 256 1.06 / 1.10 / 1.04, 300 1.00 / 1.03 / 1.03, 512 0.96 / 1.03 / 0.97, 700
// 0.87 / 0.93 / 0.86.  Beyond: L = 1536 1.09 / 1.00 / 1.05 (768), 2048 0.84 /
// 0.98 / 0.99 (768) and 1.00 / 1.01 / 1.03 (1280), 4096 0.76 / 0.95 / 0.76 (768)
// and 0.91 / 0.99 / 0.80 (1280), 8192 1.00 / 1.03 / 0.71 (1280).
// D = 128, up to a block per CU: L = 64 1.21 / 1.24 / 1.21, 160 1.07 / 1.12 /
// 1.05, 256 1.00 / 1.07 / 0.96, 300 0.92 / 0.93 / 0.93, 2048 0.82 / 0.84 /
// 0.76.  Beyond: L = 4096 0.79 / 1.14 / 0.70 (320), 0.78 / 1.08 / 0.74 (512);
// L = 2048 1.23 times faster at 320, equal from 480 on: not taken.
inline int fwd_key_groups(int D, long long blocks, int L, bool causal, bool docs, long long cus)
{
    if (D == 64) {
        if (L <= 192)
            return 1;
        if (blocks <= cus)
            return L > 768 ? 4 : 2;
        if (blocks <= 2 * cus)
            return L > (causal ? 384 : 512) ? 2 : 1;
        return L >= 2048 && blocks <= (!causal ? 3 : L > 2048 ? 5 : 4) * cus ? 2 : 1;
    }
    if (blocks <= cus)
        return L > 256 ? 2 : 1;
    return causal && L > 2048 && causal_small_grid(blocks, docs, cus) ? 2 : 1;
}

// dQ: groups over a query block's key tiles, where it runs by itself (the
// ratios are of the whole backward).
// D = 64, up to a block per CU 0.93 / 0.97 / 0.92 (L = 300); with RoPE, which
// has no one-kernel backward, dQ and dK/dV together L = 64 1.20, 128 and 160
// 1.05, 200 0.95.  Up to two: L = 300
// 1.02 / 1.05 / 1.03, 512 1.02 / 1.02 / 1.01, 700 0.94 / 0.98 / 0.96, 1024 0.97 /
// 0.98 / 0.97; four groups over two (512 blocks): L = 8192 0.89 for 0.93 / 0.98
// for 0.95 / 0.83 for 0.85.  Beyond: L = 4096 0.88 / 1.00 / 0.90 (1024), 0.98 /
// 1.01 / 0.90 (1280); L = 3000 1.09 / 1.02 / 1.04 (2040).
// D = 128: L = 4096 0.93 / 1.04 / 0.94 (384), 0.89 / 1.01 / 0.88 (512), 1.01 /
// 0.99 / 0.90 (640), 1.03 / 1.01 / 0.98 (768); L = 1024 0.96 / 1.01 / 0.93 (256).
inline int dq_key_groups(int D, long long blocks, int L, bool causal, bool docs, long long cus)
{
    if (D == 64) {
        if (L <= 512)
            return L > 192 && blocks <= cus ? 2 : 1;
        if (blocks <= 2 * cus)
            return L > 2048 && causal ? 4 : 2;
        return L > 2048 && blocks <= 6 * cus ? 2 : 1;
    }
    return (L > 768 && blocks <= cus) || (L > 2048 && causal && causal_small_grid(blocks, docs, cus))
               ? 2
               : 1;
}

// dK/dV at D = 64: groups over a key block's query tiles.  Up to a block per
// CU 0.92 / 0.94 / 0.86 (L = 2048), not for the shortest rows (see dQ).  L =
// 4096: 0.85 / 1.07 / 0.86 (512), 1.00 / 0.99 / 0.84 (640), 1.04 / 1.00 / 0.93
// (768); L = 3000 1.05 / 0.99 / 0.87 (648).  (At D = 128 the paired waves fill
// a CU's registers with one group.)
inline int dkdv_query_groups(long long blocks, int L, bool causal, bool docs, long long cus)
{
    return (L > 192 && blocks <= cus) ||
                   (L > 2048 && causal && causal_small_grid(blocks, docs, cus))
               ? 2
               : 1;
}

// Whether dK/dV and dQ run as one launch (blocks of each).  Its workgroups
// fill a CU, so it pays while both kernels' blocks fit the chip once; longer
// rows, whose heaviest blocks take longer than the average ones, gain further.
// One launch over the other route.  128 blocks: D = 64 L = 160 0.90 / 0.86 /
// 0.90, 256 0.68 / 0.50 / 0.66; D = 128 L = 64 0.94 / 0.98 / 0.91, 512 0.66 /
// 0.71 / 0.65.  144: D = 64 L = 256 1.08 / 0.80 / 1.07, 300 0.84 / 1.01 / 0.84,
// 512 0.75 / 1.07 / 0.77; D = 128 L = 256 1.12 / 1.16 / 1.07, 300 0.81 / 1.13 /
// 0.82, 512 0.68 / 1.10 / 0.70.  160: D = 64 L = 512 1.05 / 1.05 / 0.90, 600
// 0.65 / 0.77 / 0.81; D = 128 L = 512 1.03 / 1.08 / 0.86, 600 0.74 / 0.89 / 0.91.
// 320, L = 4096: D = 64 0.65 / 0.87 / 0.46, D = 128 0.83 / 0.83 / 0.54; 228, L =
// 1536, D = 128: 0.71 / 1.04 / 0.63.  At D = 64 the one-kernel backward keeps
// rows of at most 128 tokens.
inline bool bwd_together(int D, long long blocks, int L, bool causal, bool rope, long long cus)
{
    if (D == 64 && !rope && L <= 128)
        return false;
    return 2 * blocks <= cus || (causal && L > 256 && 16 * blocks <= 9 * cus) ||
           (L > 512 && 8 * blocks <= 5 * cus) ||
           (L > (causal ? 1024 : 2048) && 4 * blocks <= 5 * cus);
}

// How a product of these sizes runs: on tiles of 256 x 256, 256 x 128 or
// 128 x 128 (the value is log2 of the tiles per 256 x 256), with the K axis in
// `splits` parts (1: none; more need the workspace).
struct GemmPlan {
    enum Tile { kLarge, kTall, kSmall } tile;
    int splits;
};

// Estimated time (us) of `tiles` tiles with `splits` K parts: rounds of
// workgroups over the CUs (one per CU), each a start-up and tail plus its K
// steps, then the partial sums' write and read.  The constants are fits to
// graph-replayed products.  One round of large, tall and small tiles: 2048 x
// 1024 at K = 1024 takes 21 / 15-17 / 12.5-13 us, at K = 5632 88 / 58 / 42-47
// (with two splits 59 / 44 / 40); 2048 x 2816 at K = 1024 (88, 176 and 352
// workgroups) 23 / 17 / 23.  A full chip runs slower, large tiles for their
// power: 8192 x 2048 at K = 2048 (256, 512, 1024 workgroups) 54 / 69 / 86.
inline double gemm_cost(double tiles, double cus, double steps, double splits, double mn,
                        int tile)
{
    const double wgs = tiles * splits, rounds = std::ceil(wgs / cus);
    const double part = std::min(wgs / cus, 1.0);  // CUs in use
    const double step = tile == GemmPlan::kSmall  ? (part < 1 ? 0.42 : 0.55)
                        : tile == GemmPlan::kTall ? (part < 1 ? 0.60 + 0.15 * part : 0.95)
                                                  : (part < 1 ? 1.02 + 0.2 * part : 1.4);
    const double reduce = splits > 1 ? 6.0 + splits * mn * 8.0 / 4.0e6 : 0.0;
    return rounds * (std::ceil(steps / splits) * step + 6.0) + reduce;
}

// The cheapest tile and number of K splits (1, 2, 4, ...) for a product of
// M x N (all groups' columns together) over K.  Splits are multiples of 64
// and at least 1024 long, and more of them than two large tiles per CU are
// never needed.
inline GemmPlan gemm_plan(int M, long long N, long long K, bool may_split, int cus)
{
    cus = std::max(cus, 1);
    const long long tiles = static_cast<long long>(M / 256) * (N / 256);
    GemmPlan best{GemmPlan::kLarge, 1};
    double cost = -1;
    for (int s = 1;; s *= 2) {
        for (const GemmPlan::Tile tile : {GemmPlan::kLarge, GemmPlan::kTall, GemmPlan::kSmall}) {
            const double c = gemm_cost(static_cast<double>(tiles << tile), cus, K / 64.0, s,
                                       static_cast<double>(M) * N, tile);
            if (cost < 0 || c < cost) {
                cost = c;
                best = GemmPlan{tile, s};
            }
        }
        if (!may_split || tiles * s >= 2LL * cus || K / (2 * s) < 1024 ||
            (K / (2 * s)) % 64 != 0)
            return best;
    }
}

// How an int8 product of M x N over K runs: few tokens with the weights
// straight into registers, or on tiles of 128 x 128 or 256 x 256.
enum class GemmI8Tile { kFew, kSmall, kLarge };

inline GemmI8Tile gemm_i8_tile(int M, int N, int K, int cus)
{
    cus = std::max(cus, 1);
    const double steps = std::ceil(K / 128.0);
    auto tiles = [&](int edge) {
        return std::ceil(M / static_cast<double>(edge)) * std::ceil(N / static_cast<double>(edge)) / cus;
    };
    // us.  Small tiles, of which a CU has two at once: a third one starts when
    // the first is done.  One to four per CU of 16 steps 14.3, 26.0, 37.4, 47.3;
    // 352 and 384 on 256 CUs 21.9 and 21.2; 2048 of 4 steps 34.9.
    const double s = tiles(128), rounds = std::max(1.0, std::min(std::ceil(s), s + 0.25));
    const double small = 3.0 + rounds * (1.7 + steps * 0.62);
    // Large ones: each its own start and end and its K steps, which a full
    // chip's power makes longer (16 steps, one tile on each of 256 CUs 32, 16 of
    // them 24; 22 rounds 610), and what it takes to store parts of tiles (8192
    // x 700 over 1008 23.4, small 15.5; 1500 x 5632 over 2048 27.6 and 34.0).
    auto round = [&](double used) { return 6.5 + steps * (0.9 + 0.55 * used); };
    const double l = tiles(256), full = std::floor(l);
    const double large = 3.0 + (N % 256 ? 6.0 : 0.0) + full * round(1.0) +
                         (l > full ? round(l - full) : 0.0);
    if (M <= 64) {
        // The weights once, and the tokens again for every 16 or 32 rows of
        // them, from L2 (6144 x 2048 for 1, 20 and 64 tokens 4.3, 6.9 and 12.1,
        // on small tiles 12; 50,432 x 2048 18.1, 26.0 and 46.1, 20 to 22).
        const double again = std::ceil(N / (N > 16384 ? 32.0 : 16.0)) * M * K;
        const double few = 2.3 + K / 1365.0 + static_cast<double>(N) * K / 5.8e6 + again / 1.0e7;
        if (few < std::min(small, large))
            return GemmI8Tile::kFew;
    }
    return small < large ? GemmI8Tile::kSmall : GemmI8Tile::kLarge;
}

// Tile `i` of workgroup `wg`'s walk through `tiles` tiles: wg, wg + grid, ...  Behind
// the last one it is the last one: a place formed from an id that no tile has
// (tile_of) would be a division by zero.
constexpr int walk_tile(int wg, int i, int grid, int tiles)
{
    return std::min(wg + i * grid, tiles - 1);
}

// How `n` weight gradients of M x N over T tokens run: on tiles of 256 x 256 or
// 128 x 128 (`edge`; tiles_n of all n), T in `steps` of 64 tokens.  The first
// `whole` tiles are a workgroup's each.  The others, fewer than the CUs, are
// shared out so that every workgroup has `head` steps: `heads` workgroups per
// tile take its first parts, and the rest of the tiles, one after the other,
// is cut into pieces for `tails` further workgroups.  (In parts of equal length
// 176 tiles of 1024 steps, 2048 x 5632 over 65,536 tokens, would be 2.75 rounds
// of 256 CUs at four parts each, which takes three.)  The heads of all tiles
// read the same tokens at the same time, the tails do not: 44 tiles of 1024
// steps with one head each and the rest in pieces took 478 us, as five heads
// and pieces 421.
struct WgradPlan {
    int edge, tiles_m, tiles_n, whole, steps, heads, head, tails;

    int shared() const { return tiles_m * tiles_n - whole; }
    int rest() const { return std::max(steps - heads * head, 0); }  // of a shared tile
    // Parts of tiles that one of the `tails` can touch.
    int most() const { return (head - 1) / std::max(rest(), 1) + 2; }
    long long partials() const
    {
        return heads ? static_cast<long long>(heads) * shared() + static_cast<long long>(tails) * most()
                     : 0;
    }
};

inline WgradPlan wgrad_plan(int T, int M, int N, int n, int cus)
{
    cus = std::max(cus, 1);
    const int steps = static_cast<int>((T + 63LL) / 64);
    WgradPlan best{};
    double cost = -1;
    auto consider = [&](const WgradPlan &p, double c) {
        if (cost < 0 || c < cost) {
            cost = c;
            best = p;
        }
    };
    for (const int edge : {256, 128}) {
        const long long tm = (M + edge - 1LL) / edge, tn = (N + edge - 1LL) / edge * n, tiles = tm * tn;
        // us a step: with few workgroups its latency, with a full chip its
        // power (2048 x 5632, 65,536 tokens: 176 workgroups of 1024 steps
        // 1235 us, 256 of 704 steps 1154; 256 x 256, one workgroup of 1024
        // steps per tile: 938 us, 542 on 128 x 128 tiles).
        auto step = [&](double wgs) {
            const double used = std::min(wgs / cus, 1.0);
            return edge == 256 ? std::max(1.03, 0.35 + 1.24 * used) : std::max(0.50, 0.58 * used);
        };
        const long long over = tiles % cus, full = tiles / cus;
        const double whole = full * (steps * step(cus) + 6.0);
        WgradPlan p{edge, static_cast<int>(tm), static_cast<int>(tn), static_cast<int>(tiles), steps,
                    0, 0, 0};
        consider(p, over ? whole + steps * step(over) + 6.0 : whole);
        // Shared: with as many heads as there are CUs for, or one; of equal
        // parts, or with the rest in pieces.  Parts of at least 8 steps: shorter
        // ones are mostly start-up, 2.5 us of every part.  (3001 x 1040 x 1416:
        // two equal heads 34 us, two and pieces of 7 steps 38.)
        if (over == 0 || steps < 16)
            continue;
        p.whole = static_cast<int>(tiles - over);
        for (const long long most : {cus / over, 1LL})
            for (const bool pieces : {false, true}) {
                p.heads = static_cast<int>(std::min<long long>(most, steps / 8));
                p.head = pieces ? static_cast<int>(std::max((over * steps + cus - 1) / cus, 8LL))
                                : (steps + p.heads - 1) / p.heads;
                p.heads = std::min(p.heads, (steps + p.head - 1) / p.head);  // each has steps
                p.tails = static_cast<int>((over * p.rest() + p.head - 1) / p.head);
                const long long parts = over * p.heads + p.tails;
                if (parts > cus || p.head >= steps)
                    continue;
                const int starts = p.tails ? (p.head + p.rest() - 1) / p.rest() : 0;
                // The tiles' first parts share what they read, the pieces do not.
                const double traffic = (static_cast<double>(p.heads) * p.head * (tm + tn) +
                                        2.0 * over * p.rest()) * edge * 128.0 / 6.0e6;
                consider(p, whole + std::max(p.head * step(parts), traffic) + 12.0 + 2.5 * starts +
                                static_cast<double>(parts + (p.tails ? over : 0)) * edge * edge *
                                    8.0 / 1.0e7);
            }
    }
    return best;
}

}  // namespace dd
