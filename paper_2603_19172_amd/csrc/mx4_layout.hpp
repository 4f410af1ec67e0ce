// Workspace layouts of the products in microscaled 4-bit floating point (host side).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "expert_plan.hpp"

namespace dymoe {

constexpr int kMx4TileCols = 256;     // columns of a tile of the weights: four matrix instructions
constexpr int kMx4SmallRows = 32;     // token rows of a tile where experts meet few tokens: one fragment
constexpr int kMx4TallRows = 128;     // and where they meet many
constexpr long kMx4SplitPairs = 8192; // pairs up to which the down projection's K may be cut into parts
constexpr int kMx4MostSplits = 4;     // parts at most
constexpr long kMx4MostCus = 256;     // compute units of the whole chip

static inline size_t mx4_round(size_t v, size_t m) { return (v + m - 1) / m * m; }

// Parts of the down projection's K in tall tiles: while its tiles are fewer than two for each compute unit, and each part has four tiles of K.  More
// pairs take no more parts, more compute units no fewer.
static inline int mx4_ffn_parts(long P, long H, long F, long E, long num_cu)
{
    const long cus = num_cu < kMx4MostCus ? num_cu : kMx4MostCus;
    const long units = (P / kMx4TallRows + (E < P ? E : P)) * ((H + 255) / 256), steps = (F + kMx4TileCols - 1) / kMx4TileCols;
    int parts = 1;
    while (P <= kMx4SplitPairs && parts < kMx4MostSplits && units * parts < 2 * cus && steps / (2 * parts) >= 4) parts *= 2;
    return parts;
}

// Rows of outputs that P pairs' parts need at most, as many at least as fewer pairs' do: a workspace of the largest batch has to do for smaller ones.
static inline long mx4_part_rows(long P, long H, long F, long E)
{
    long rows = P;
    for (int parts = 2; parts <= kMx4MostSplits; parts *= 2) {
        long lo = 0, hi = P < kMx4SplitPairs ? P : kMx4SplitPairs;         // the most pairs that take so many
        while (lo < hi) {
            const long mid = (lo + hi + 1) / 2;
            if (mx4_ffn_parts(mid, H, F, E, kMx4MostCus) >= parts) lo = mid;
            else hi = mid - 1;
        }
        if (lo * parts > rows) rows = lo * parts;
    }
    return rows;
}

struct Mx4FfnLayout {
    size_t Hp, Fp;     // columns of the codes' rows: whole tiles
    size_t xq, xs;     // [Hp / 256, T, 128] codes and [Hp / 256, T, 8] exponents of the activations
    size_t hq, hs;     // codes and exponents of the SwiGLU intermediate, row by row by position (pairs sorted by expert) or in tiles, see below
    size_t part;       // parts of [P, H up to a multiple of 8] outputs of the pairs, by position, fp32: mx4_part_rows rows
    size_t plan;       // int32, see ExpertPlan
    size_t total;
    int max_tiles;
};

static inline Mx4FfnLayout mx4_ffn_layout(long T, long H, long F, long E, long k)
{
    Mx4FfnLayout L;
    const size_t P = (size_t)T * (size_t)k;
    L.Hp = mx4_round((size_t)H, kMx4TileCols);
    L.Fp = mx4_round((size_t)F, kMx4TileCols);
    L.max_tiles = (int)(P / kMx4SmallRows + ((size_t)E < P ? (size_t)E : P));
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += mx4_round(bytes, 256); return here; };
    L.xq = take((size_t)T * L.Hp / 2);
    L.xs = take((size_t)T * L.Hp / 32);
    // Strips: by position.  Tall tiles: in tiles of 32 rows as the weights are, an expert's pairs from a tile's first row on: the expert whose first position is f and whose first
    // tile is number j begins at tile f / 32 + j: the next has at least j + 1, and (f + n) / 32 + 1 >= f / 32 + n / 32 rounded up.  The
    // last ends before P / 32 + P / 128 + the number of experts.
    const size_t held = mx4_round(P + P / 4 + 32 * ((size_t)E < P ? (size_t)E : P), 32);
    L.hq = take(held * L.Fp / 2);
    L.hs = take(held * L.Fp / 32);
    L.part = take((size_t)mx4_part_rows((long)P, H, F, E) * mx4_round((size_t)H, 8) * 4);
    L.plan = take(expert_plan_bytes(P, (size_t)L.max_tiles));
    L.total = at;
    return L;
}

struct Mx4MatLayout {
    size_t Kp;
    size_t xq, xs;     // codes and exponents of the activations, whole tiles of 32 rows
    size_t total;
};

static inline Mx4MatLayout mx4_mat_layout(long T, long K)
{
    Mx4MatLayout L;
    L.Kp = mx4_round((size_t)K, kMx4TileCols);
    L.xq = 0;
    const size_t rows = mx4_round((size_t)T, 32);
    L.xs = rows * L.Kp / 2;
    L.total = L.xs + rows * L.Kp / 32;
    return L;
}

}  // namespace dymoe
