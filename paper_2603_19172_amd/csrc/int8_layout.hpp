// Workspace layouts of the 8-bit integer products (host side).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace dymoe {

constexpr int kI8TileRows = 128;      // token rows of a tile of the grouped products
constexpr int kI8TileWide = 160;      // of a tile where the weights' bytes bound the call
constexpr int kI8TileSmall = 32;      // of a tile where experts meet few tokens: one fragment

static inline size_t i8_round(size_t v, size_t m) { return (v + m - 1) / m * m; }

struct I8FfnLayout {
    size_t Hp, Fp;     // columns of the codes' rows: multiples of a K-tile
    size_t xq, xs;     // [T, Hp] codes and [T] scales of the activations
    size_t h;          // [P, Fp] SwiGLU intermediate, by position (pairs sorted by expert)
    size_t hq, hs;     // [P, Fp] its codes, [P] their scales
    size_t part;       // [P, Hp] outputs of the pairs, by position
    size_t plan;       // int32, see I8Plan
    size_t total;
    int max_tiles;
};

static inline I8FfnLayout i8_ffn_layout(long T, long H, long F, long E, long k)
{
    I8FfnLayout L;
    const size_t P = (size_t)T * (size_t)k;
    L.Hp = i8_round((size_t)H, 128);
    L.Fp = i8_round((size_t)F, 128);
    L.max_tiles = (int)(P / kI8TileSmall + ((size_t)E < P ? (size_t)E : P));
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += i8_round(bytes, 256); return here; };
    L.xq = take((size_t)T * L.Hp);
    L.xs = take((size_t)T * 4);
    L.h = take(P * L.Fp * 4);
    L.hq = take(P * L.Fp);
    L.hs = take(P * 4);
    L.part = take(P * L.Hp * 4);
    L.plan = take((8 + i8_round(2 * P, 4) + 16 * (size_t)L.max_tiles) * 4);        // (a tile's record: 64 bytes)
    L.total = at;
    return L;
}

struct I8MatLayout {
    size_t Kp;
    size_t xq, xs;     // [T up to a multiple of 32, Kp] codes and [T] scales of the activations
    size_t total;
};

static inline I8MatLayout i8_mat_layout(long T, long K)
{
    I8MatLayout L;
    L.Kp = i8_round((size_t)K, 128);
    L.xq = 0;
    L.xs = i8_round(i8_round((size_t)T, 32) * L.Kp, 256);
    L.total = L.xs + i8_round((size_t)T * 4, 256);
    return L;
}

}  // namespace dymoe
