// Which shape a product in microscaled 4-bit floating point is computed in (host side).  Shapes differ in the order of their fp32 sums: the rules
// go by sizes alone, so that the same call has the same order.
#pragma once
#include "mx4_layout.hpp"

namespace dymoe {

constexpr long kMx4FuseBytes = 64 * 1024;       // rows in LDS at most

// bytes of rows in LDS: Kp / 2 + 16 of codes (16 bytes of other banks from row to row) and Kp / 32 of exponents each
static inline long mx4_fuse_bytes(long rows, size_t Kp) { return rows * ((long)Kp / 2 + 16 + (long)Kp / 32); }

enum class Mx4MatShape {
    kSmall,        // strips of 32 weight rows, tiles of 32 rows, K dealt to a workgroup's wavefronts
    kTile32,       // tiles of 32 rows x 128 columns
    kTile64,       // 64 x 128
    kTile64w,      // 64 x 256
    kTile128       // 128 x 256
};

struct Mx4MatChoice {
    Mx4MatShape shape;
    bool fuse;     // kSmall: the workgroups convert the rows
    int waves;     // kSmall: that K is dealt to
};

// Times in us with the conversion of the rows (T x N x K).
static inline Mx4MatChoice mx4_mat_choice(long T, long N, long K, bool coded, long num_cu)
{
    const long strips = (N + 31) / 32, t32 = (T + 31) / 32, t64 = (T + 63) / 64, t128 = (T + 127) / 128, n128 = (N + 127) / 128, n256 = (N + 255) / 256;
    // The conversion inside saves a launch while it is little: 1 x 4096 x 4096 6.1 and 7.7 with a launch of its own, 4 rows 7.0 / 7.9, 8 rows 8.4 / 7.9;
    // 8 x 1536 x 2048 5.8 / 6.8, 16 rows 7.2 / 7.0.
    const bool inside = T <= 32 && T * K <= 16 << 10 && mx4_fuse_bytes(T, mx4_round((size_t)K, kMx4TileCols)) <= kMx4FuseBytes;
    // Eight wavefronts while the strips are fewer than 400: 1 x 4096 x 14336 13.2 and 15.4 with four, 61 x 1536 x 2048 7.4 / 7.2; kernels alone, codes made
    // before, 1 x 14336 x 4096 7.8 / 7.3, 2 x 33000 x 2100 10.8 / 9.5.  But always where rows are converted inside (1 x 14336 x 4096 7.4 / 8.0,
    // 32 x 14336 x 512 5.6 / 5.95, 2 x 33000 x 2100 12.1 / 11.7), and for codes of such rows, so that the order of the sums is the sizes' and not x's type's.
    const Mx4MatChoice small = {Mx4MatShape::kSmall, inside && !coded, inside || strips * t32 < 400 ? 8 : 4};
    // Strips while tiles of 32 x 128 are few, so that each strip has a compute unit (64 x 4096 x 4096, 64 of them: 8.6 and 9.5 in tiles; 256 x 798 x 7548, 56:
    // 13.3 / 13.8; 222 x 1295 x 9025, 77: 23.2 / 15.6; 96 x 4096 x 4096, 96: 11.4 / 10.2), or somewhat more with a short K (512 x 768 x 2048, 96: 7.8 / 8.5;
    // 128 x 4096 x 4096, 128: 11.8 / 9.8); then the largest tiles that still are one for each compute unit, two of 64 x 128 (256 x 4096 x 4096 in tiles of
    // 32 11.3, of 64 12.1, of 128 x 256 22; 512 x 4096 x 4096 15.7, 13.9, 23; 2047 x 2048 x 2048 18.7, 15.7, of 64 x 256 16.3, of 128 20.5;
    // 512 x 14336 x 4096 35, 28.6, 27.4, 28.2; 2047 x 4096 x 4096 42, 32.4, 31.3, 30.9).
    if (T <= 32 || t32 * n128 <= num_cu / 4 || (t32 * n128 <= num_cu * 3 / 8 && K <= 2048)) return small;
    if (t32 * n128 <= num_cu) return {Mx4MatShape::kTile32, false, 0};
    if (t64 * n128 <= 2 * num_cu) return {Mx4MatShape::kTile64, false, 0};
    return {t128 * n256 < num_cu ? Mx4MatShape::kTile64w : Mx4MatShape::kTile128, false, 0};
}

enum class Mx4FfnShape {
    kThin,         // a few pairs: two launches
    kSmall,        // few pairs an expert: strips of 32 weight rows
    kTall          // tiles of 128 rows
};

struct Mx4FfnChoice {
    Mx4FfnShape shape;
    int up_waves, down_waves;      // kSmall: that K is dealt to
    int splits;                    // kTall: parts of the down projection's K
};

// How many wavefronts share a strip: as few as make 2048 of them, and no more than there are tiles of K.  Down projections of 768 x 2048, 61 tokens'
// 8 of 128 experts 18.7 us with one, 20.2 two, 21.9 four; of 14336 x 4096, one token's two experts 35.8, 20.8, 13.7 and 11.7 with eight.
static inline int mx4_strip_waves(long strips, long tiles, int most)
{
    int n = 1;
    while (2 * n <= most && strips * n < 2048 && 2 * n <= tiles) n *= 2;
    return n;
}

static inline Mx4FfnChoice mx4_ffn_choice(long T, long H, long F, long E, long k, long num_cu)
{
    const long P = T * k;
    const size_t Hp = mx4_round((size_t)H, kMx4TileCols), Fp = mx4_round((size_t)F, kMx4TileCols);
    // Two launches instead of four, but a token's workgroups read its experts' W2 for themselves: one token on 2 of 8 experts of 14336 x 4096 35 us and 41.5,
    // two tokens 63 / 64.5, four 108 / 95; on 8 of 128 experts of 768 x 2048, one token 12.3 / 18.9, four 22.3 / 26.8.
    if (P <= 64 && (T <= 2 || 4 * P <= E) && T <= 32 && mx4_fuse_bytes(T, Hp) <= kMx4FuseBytes && mx4_fuse_bytes(k, Fp) <= kMx4FuseBytes)
        return {Mx4FfnShape::kThin, 0, 0, 1};
    // Strips while an expert meets 20 pairs or fewer on average (or never more than 32): 64 tokens, 2 of 8 experts of 14336 x 4096 (16) 131 us and 153 in
    // tall tiles, 96 (24) 148 / 158, 128 (32) 221 / 159; 8 of 128 experts of 768 x 2048, 256 tokens (16) 75 / 78, 384 (24) 86 / 83, 512 107 / 87.
    const long tiles = P / kMx4SmallRows + (E < P ? E : P);
    if (T <= 32 || P <= 20 * E)
        return {Mx4FfnShape::kSmall, mx4_strip_waves(tiles * ((F + 31) / 32), (long)Hp / kMx4TileCols, 4),
                mx4_strip_waves(tiles * ((H + 31) / 32), (long)Fp / kMx4TileCols, 8), 1};
    return {Mx4FfnShape::kTall, 0, 0, mx4_ffn_parts(P, H, F, E, num_cu)};
}

}  // namespace dymoe
