// Which kernel of q4_kernels.h serves a product with 4-bit weights, by what launches of them take (host code; sizes and the type of x are all it goes by).
#pragma once
#include "fscnn.h"

namespace fscnn {

constexpr int kQ4MostRows = (1 << 27) - 16;  // weight rows: 512 threads for 16 of them, fewer than 2^32 in a launch
constexpr int kQ4LaunchRows = 1 << 18;       // rows of x a launch, at most
// The rows of x a launch: its tiles, at worst 512 threads for 32 x 32 outputs, are fewer than 2^32 threads
inline int q4_launch_rows(int K)
{
    int rows = kQ4LaunchRows;
    while (rows > 32 && rows / 32 * ((K + 31LL) / 32) * 512 > 0xffffffffLL) rows /= 2;
    return rows;
}

struct Q4Choice {
    enum Kernel { kRows, kStaged, kTiles } kernel;
    int waves;                               // kRows, kStaged: of a work-group
    int shape;                               // kTiles, 16 and 8 bits: of kTiles or kLoose below; 32-bit floats: rows of a tile, 32 or 64
    int parts;                               // work-groups that divide the columns
    double us;
};

// Columns divided over `parts` work-groups cost a second launch, and the sums' way to memory and back (us)
inline double sums_us(double M, double tiles, int parts) { return parts > 1 ? 2.5 + parts * 1.28e-4 * M * tiles / 3 : 0; }

// How 32-bit floats are served: kernel, and work-groups that divide the columns, at most `most` of them.  (tiles: of 16 weight rows; blocks: of 128 columns)
inline Q4Choice f32_choice(long long tiles, int blocks, int M, int most)
{
    // every row's three parts in one operand; else a wave's own parts (few rows, little work) or a tile's, made once for 256 rows of weights
    // (25088 -> 4096, one row: 14.1 us staged, 30 with a wave's own parts)
    if (M * 3 <= 16) return {Q4Choice::kStaged, blocks >= 64 && tiles <= 256 ? 16 : 8, 0, 1, 0.0};
    // times of launches as TileCost has them; divided columns cost a launch and the sums' way to memory and back
    const double wide = (double)((tiles + 15) / 16);   // work-groups of a part of 32 or 64 rows
    Q4Choice best = {Q4Choice::kTiles, 0, 32, 1, 1e30};
    // (up to 384 columns stores are what counts: 4096 rows to 16384 of 384 take 198 us in tiles of 32 rows, 254 in tiles of 64)
    for (int rows = 32; rows <= (blocks < 4 ? 32 : 64); rows *= 2)
        for (int p = 1; p == 1 || (p <= most && p <= 16 && blocks / p >= 4); p *= 2) {
            const double n = __builtin_ceil(wide * ((M + rows - 1) / rows) * p / 256);
            const double t = 4 + n * ((blocks + p - 1) / p) * (rows == 32 ? 1.45 : 2.65) + sums_us(M, (double)tiles, p);
            if (t < best.us) best = {Q4Choice::kTiles, 0, rows, p, t};
        }
    if (M <= 16)
        if (const double t = 4 + __builtin_ceil(tiles / 256.0) * (blocks / 32.0) * (4 + 0.3 * M); t < best.us) return {Q4Choice::kRows, 8, 0, 1, t};
    return best;
}

// Time of a launch of tiles in us: 4 and, for every turn (a block a set of waves), `one` while a CU has a work-group, `many` times the work-groups of a CU
// beyond that; `parts` work-groups divide the columns
struct TileCost {
    int rows, cols, sets;
    float one, many;
    double us(double M, double K, int blocks, int parts) const
    {
        const double groups = __builtin_ceil(M / rows) * __builtin_ceil(K / cols) * parts, n = __builtin_ceil(groups / 256);
        return 4 + ((blocks + parts - 1) / parts + sets - 1) / sets * (n > 1 && many * n > one ? many * n : one);
    }
};

// x in 16 or 8 bits (ints).  The fastest of seven shapes of tile_kernel, in 8 bits five, by what launches of them take (fitted to 1 to 4096 rows, 1024 to
// 16384 columns, 1024 to 12288 weight rows, within 15 %; in 16 bits the choice is 0.4 % behind the fastest in the mean, in 8 bits 2.4): many sets
// where few work-groups are there, whose sums through LDS cost more than they bring where they are many (bf16, 4096 -> 4096: 64 rows of x 9.3 us
// with 32 x 32 in 8 sets, 28 with 64 x 128 in one; 1024 rows 117 and 45), and the shape whose work-groups leave the fewest CUs idle (200 rows
// 17.4 us with 64 x 64 in 4 sets, 19.4 with the best of the others; 700 rows 33.3 with 96 x 128 in 2 sets and 39.2).  Rows of x that
// are not 16 bytes aligned (`dma` is false) come by way of registers and have four shapes (fp16, 4097 -> 4096: 64 rows 15.4 us with 32 x 32 in 8
// sets, 36 with 64 x 128 in one; 2048 rows 407 and 94).  Up to 16 rows also staged_kernel and, for one or two rows, whose operand is
// not worth a barrier, rows_kernel (bf16, 4096 -> 4096: one row 3.7 us, 4.1 staged; 8 rows 5.5 and 4.9).  Sixteen waves where a wave of
// eight had eight blocks or more (one row of 16384: 8.3 us, 10.3 with eight; of 4096: 3.9 and 3.7).
inline Q4Choice narrow_choice(bool ints, int M, int K, int blocks, int parts, bool dma)
{
    static constexpr TileCost kTiles[2][7] = {{{32, 32, 8, 1.3f, 1.55f}, {32, 64, 4, 1.0f, 0.93f}, {64, 128, 2, 1.3f, 1.2f}, {64, 128, 1, 0.8f, 0.62f},
                                               {128, 128, 1, 1.25f, 1.08f}, {64, 64, 4, 1.6f, 1.72f}, {96, 128, 2, 1.65f, 1.78f}},
                                              {{32, 32, 8, 0.68f, 0.8f}, {32, 64, 4, 0.6f, 0.6f}, {64, 128, 2, 0.8f, 0.79f}, {64, 128, 1, 0.52f, 0.41f},
                                               {128, 128, 1, 0.9f, 0.72f}, {}, {}}};
    static constexpr TileCost kLoose[2][4] = {{{32, 32, 8, 2.1f, 2.5f}, {32, 64, 4, 1.28f, 1.04f}, {64, 128, 2, 1.54f, 1.6f}, {64, 128, 1, 1.0f, 0.69f}},
                                              {{32, 32, 8, 1.5f, 1.3f}, {32, 64, 4, 1.05f, 0.82f}, {64, 128, 2, 1.26f, 1.42f}, {64, 128, 1, 0.8f, 0.56f}}};
    Q4Choice best = {Q4Choice::kTiles, 0, 0, parts, 1e30};
    for (int i = 0; i < (!dma ? 4 : ints ? 5 : 7); ++i)
        if (const double t = (dma ? kTiles[ints][i] : kLoose[ints][i]).us(M, K, blocks, parts); t < best.us) best.shape = i, best.us = t;
    if (M <= 16 && parts == 1) {
        const int n = ((K + 15LL) / 16 + 255) / 256, waves = blocks >= 64 && n == 1 ? 16 : 8;
        const double t = 2.9f + n * (blocks / 32.0f) * (0.95f + 0.13f * M);
        if (M <= 4 || t <= best.us) return {M > 2 ? Q4Choice::kStaged : Q4Choice::kRows, waves, 0, 1, t};
    }
    return best;
}

// Work-groups that divide the columns, at most `most`: where few weight rows leave CUs without one (64 rows, 20000 -> 300:
// bf16 29.6 us, 11.2 in 16 parts; 200 rows, 25088 -> 512 35.4 and 22.6 in 8; int8 19.6 and 12.3 in 8)
inline int narrow_parts(bool ints, int M, long long tiles, int K, int blocks, int most)
{
    int best = 1;
    double us = narrow_choice(ints, M, K, blocks, 1, true).us;
    for (int p = 2; p <= most && p <= 16 && blocks / p >= 4; p *= 2)
        if (const double t = narrow_choice(ints, M, K, blocks, p, true).us + sums_us(M, (double)tiles, p); t < us) {
            us = t;
            best = p;
        }
    return best;
}

// Work-groups that may divide the columns of a call
inline int q4_parts(int x_type, int M, int K, int C)
{
    // (a launch's rows of x: the sums' room is for one launch, and bounded)
    constexpr double kMostBytes = 64 << 20;
    if (M <= (x_type == FSCNN_F32 ? 0 : 16) || M > kQ4LaunchRows) return 1;
    const long long tiles = (K + 15LL) / 16;
    const int blocks = (C + 127) / 128, most = (int)(kMostBytes / (64.0 * tiles * M));
    if (x_type == FSCNN_F32) return f32_choice(tiles, blocks, M, most > 1 ? most : 1).parts;
    return narrow_parts(x_type == FSCNN_I8, M, tiles, K, blocks, most);
}

}  // namespace fscnn
