// Which shape an 8-bit integer product is computed in (host side).  Every shape gives the same bits: the rules are for time alone.
#pragma once
#include "int8_layout.hpp"

namespace dymoe {

// Up to 8 rows any matrix, up to 16 while the outputs are few (a workgroup reads its rows' codes for 16 weight rows only): 16 rows of 4096
// values, N = 4096 8.8 us here and 10.0 in the shapes below, N = 14336 18.6 / 20.3, N = 32000 31 / 31.5, N = 64000 58.6 / 52.6.
constexpr int kI8ThinRows = 16;
constexpr long kI8ThinOut = 3 << 18;
// Tokens up to which the experts' workgroups quantise rows themselves: two launches instead of five, but every workgroup of the down
// projection reads its token's intermediate, and an expert that two tokens share is read for each.  One token on 8 of 128 experts of 768 x 2048
// 18.1 us and 25.1 in five launches, two 26.3 / 30.3, three 38.9 / 36.7, four 42.4 / 39.8; 2 of 8 experts of 14336 x 4096: 66 / 75,
// 113 / 114, 163 / 140, 188 / 155.
constexpr int kI8FuseRows = 2;
constexpr long kI8FuseBytes = 64 * 1024;        // the codes' bytes in LDS at most
// The plain product's workgroups quantise where that is less than a launch of its own: T * K values for a workgroup, and all
// workgroups' together.  With T = 8, N = 1536, K = 2048 5.1 us and 5.9 with the launch, T = 16 6.9 / 6.3; T = 1 on 4096 x 14336 13.5 / 16.7, T = 4
// 21.8 / 17.1; T = 2 on 4096 x 4096 6.8 / 7.8, T = 4 8.2 / 7.9; T = 2 on 14336 x 4096 14.8 / 14.2.
constexpr long kI8FuseRow = 16 << 10;
constexpr long kI8FuseReads = 4 << 20;

enum class I8MatShape {
    kThin,         // a few rows: 16 weight rows a workgroup
    kSmall32,      // strips of 32 weight rows, one fragment of 32 rows
    kSmall64,      // two
    kSplit4,       // tiles of 128 x 128, K split over four groups of wavefronts
    kSplit2,       // over two
    kOne,          // one strip a wavefront
    kTwo           // two
};

struct I8MatChoice {
    I8MatShape shape;
    bool fuse;     // the product's workgroups quantise the rows
};

// strips of 32 outputs for tiles of 64 rows
static inline long i8_strip_units(long T, long N) { return (T + 63) / 64 * ((N + 31) / 32); }

static inline I8MatChoice i8_mat_choice(long T, long N, long K, bool coded, long num_cu)
{
    if (T <= kI8ThinRows && (T <= 8 || T * N <= kI8ThinOut))
        return {I8MatShape::kThin, !coded && T * K <= kI8FuseRow && (N + 15) / 16 * T * K < kI8FuseReads};
    // Strips of 32 columns: up to 1.25 of them a compute unit, beyond which they come in two rounds; T = 128, N = K = 4096: 13.9 us and 21.8 in
    // tiles of 128 x 128 with K split; T = 100, N = 14336, K = 4096: 39 and 22.
    if (i8_strip_units(T, N) <= num_cu * 5 / 4) return {T <= 32 ? I8MatShape::kSmall32 : I8MatShape::kSmall64, false};
    // K split in four up to a tile a compute unit: 256 x 4096 x 4096 22 us, unsplit 26.8, as 32-column strips 24.7.  In two a little beyond.
    // Two strips a wavefront from two workgroups a compute unit on, where K is long enough for their longer start: 8192 x 8192 x 8192
    // 492 us, one strip 551; 4096 x 9000 x 700 67 and 57.
    const long tiles = (T + kI8TileRows - 1) / kI8TileRows, units2 = tiles * ((N + 255) / 256), units1 = tiles * ((N + 127) / 128);
    const long Kp = (long)i8_round((size_t)K, 128);
    if (units1 <= num_cu && Kp >= 1024) return {I8MatShape::kSplit4, false};
    if (units1 <= num_cu * 5 / 4) return {I8MatShape::kSplit2, false};
    return {units2 < 2 * num_cu || Kp < 2048 ? I8MatShape::kOne : I8MatShape::kTwo, false};
}

enum class I8FfnShape {
    kThin,         // one or two tokens: two launches
    kSmall,        // few pairs an expert: strips of 32 weight rows
    kGrouped       // tall and wide tiles
};

static inline I8FfnShape i8_ffn_choice(long T, long H, long F, long E, long k)
{
    const long P = T * k, Hp = (long)i8_round((size_t)H, 128), Fp = (long)i8_round((size_t)F, 128);
    if (T <= kI8FuseRows && P <= 64 && T * (Hp + 16) <= kI8FuseBytes && k * (Fp + 16) <= kI8FuseBytes) return I8FfnShape::kThin;
    // Tiles of 32 rows and a sum in LDS while an expert meets 20 pairs or fewer on average (or never more than 32): 64 tokens, 2 of 8 experts of
    // 14336 x 4096 (16 pairs an expert) 241 us and 262 in wide tiles, 80 tokens (20) 251 / 266, 96 (24) 266 / 268, 128 (32) 379 / 280; 8 of 128 experts
    // of 768 x 2048, 256 tokens (16) 124 / 138, 320 (20) 132 / 142, 384 (24) 143 / 146, 512 (32) 182 / 156; 32 tokens on all of 8 such experts
    // 26.6 / 28.9.
    return T <= 32 || P <= 20 * E ? I8FfnShape::kSmall : I8FfnShape::kGrouped;
}

}  // namespace dymoe
