// Which kernel serves a product of 4-bit matrices, by its sizes alone, and the room that goes with it: plain C++.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

enum { MX_ROWS = 32, MX_COLS = 128, MX_BLOCK = 32, MX_TILE_BYTES = 2048, MX_SCALE_ROWS = 64, MX_SCALE_TILE_BYTES = 256,
       MX_MOST_TILES = 1 << 22 };      // (a grid has less than 2^32 threads)

enum { MX_PARTED_TILES = 100, MX_PARTED_STEPS = 36, MX_PART_STEPS = 12, MX_MOST_PARTS = 8, MX_PART_GROUPS = 384 };     // see sl_mx4_choose

struct SlMx4Choice {
    int tile;                            // 0: 64 x 64, 1: 128 x 128, 2: 128 x 256
    int parts;                           // of the contraction
};

// Tenths of a round (see below) that so many of the larger tiles take.
inline int64_t sl_mx4_rounds10(int64_t tiles) { return tiles / 512 * 10 + (tiles % 512 == 0 ? 0 : tiles % 512 <= 256 ? 6 : 10); }

// By how many tiles there are for the 256 compute units (us, 64 x 64 / 128 x 128 / 128 x 256):
//   few: every one gets a tile as soon as they are small - 1024 x 1024 x 4096 7.3 / 11.0 / 17.8, 256 x 8192 x 2048 7.0 / 7.8 / 11.6 -
//   until 64 x 64 are more than two to a compute unit: 2388 x 956 x 16,370 (570) 46 / 34 / 58, 1024 x 4096 x 1024 8.8 / 6.8 / 9.1, 2048 cubed
//   11.8 / 8.7 / 12.5;
//   many: 512 workgroups of either larger tile run at a time, two to a compute unit, and a round of 128 x 256 takes 1.75 times as long as one of
//   128 x 128 (it reads LDS less for the same products, and power is what bounds them); up to 256 tiles that are left over run one to a unit,
//   in 0.6 of a round.  So the rounds decide: 8192 x 2048 x 16,384 (512 and 1024 tiles) - / 138 / 128, 8575 x 1866 x 3815 (536 and 1005) 72 / 41 / 48,
//   517 x 50,257 x 2048 (985 and 1965) 72 / 46 / 40.5, 12,688 x 1510 x 323 (600 and 1200) 21.4 / 15.6 / 16.4, 5054 x 4236 x 5982 (680 and 1360)
//   124 / 77 / 72.
// A long contraction on very few tiles is cut: parts of 12 steps, of more where there would be more than eight or than 384 workgroups; the steps are
// then shared out evenly, and a second launch adds the parts' results.  In a graph, whole / four / five / eight parts: 100 x 1000 x 16,384 (32 tiles, 128 steps; the rule makes
// eight) 19.1 / 10.3 / 10.0 / 10.2; 55 x 613 x 6252 (10 tiles, 49 steps; five) 8.7 / 7.1 / 7.2 / 7.7; 2378 x 67 x 11,212 (76 tiles, 88 steps; five)
// 14.6 / 11.9 / 11.6 / 13.5; from 128 tiles on it gains nothing (256 x 2048 x 8192 11.0 / 13.9 / 16.0 / 19.0, two parts 11.4 and 11.6).
// (Over 60 sizes drawn from 16 .. 16,384 x 16 .. 8192 x 16 .. 16,384 the rule's choice takes 1 to 2 % longer than the best of the three sizes in
// one, two, four or eight parts.)
inline SlMx4Choice sl_mx4_choose(int64_t m, int64_t n, int64_t k)
{
    const int64_t small = ((m + 63) / 64) * ((n + 63) / 64), middle = ((m + 127) / 128) * ((n + 127) / 128),
                  large = ((m + 127) / 128) * ((n + 255) / 256), steps = (k + MX_COLS - 1) / MX_COLS;
    if (small > 512) return SlMx4Choice{7 * sl_mx4_rounds10(large) < 4 * sl_mx4_rounds10(middle) ? 2 : 1, 1};
    if (small > MX_PARTED_TILES || steps < MX_PARTED_STEPS) return SlMx4Choice{0, 1};
    const int64_t per = std::max<int64_t>({MX_PART_STEPS, (steps + MX_MOST_PARTS - 1) / MX_MOST_PARTS, (steps * small + MX_PART_GROUPS - 1) / MX_PART_GROUPS});
    return SlMx4Choice{0, (int)((steps + per - 1) / per)};
}

// Elements from one row of a part's result to the next.
inline int64_t sl_mx4_part_pitch(int64_t n) { return (n + 3) / 4 * 4; }

// Elements of room for the parts' results that serve every product whose m, n and k are no larger: fewer rows can mean more room, where they are
// few enough tiles that the contraction is cut.  For each number of tiles that is cut, the most parts that sl_mx4_choose makes of it (every
// term of its `per` gives a bound) times the largest result.
inline int64_t sl_mx4_parts_room(int64_t m, int64_t n, int64_t k)
{
    const int64_t steps = (k + MX_COLS - 1) / MX_COLS, rows = (m + 63) / 64, cols = (n + 63) / 64;
    if (steps < MX_PARTED_STEPS) return 0;
    int64_t room = 0;
    for (int64_t r = 1; r <= rows && r <= MX_PARTED_TILES; ++r)
        for (int64_t c = 1; c <= cols && r * c <= MX_PARTED_TILES; ++c) {
            const int64_t parts = std::min<int64_t>({MX_MOST_PARTS, (steps + MX_PART_STEPS - 1) / MX_PART_STEPS, (MX_PART_GROUPS + r * c - 1) / (r * c)});
            room = std::max(room, parts * std::min(64 * r, m) * sl_mx4_part_pitch(std::min(64 * c, n)));
        }
    return room;
}

// Where it is not quicker to quantise x once, in a launch of its own: up to 640 steps of 128 in x's rows together (us, this kernel / two
// launches: 8 rows, k = 8192 9.9 / 14.8, 16 rows, k = 2048 6.6 / 8.6, 16 rows, k = 8192 22.5 / 14.8).  That is at most 52 KB of LDS.
inline bool sl_mx4_few_rows(int64_t m, int64_t k) { return m <= 16 && m * ((k + MX_COLS - 1) / MX_COLS) <= 640; }

// Waves that share a tile of 16 columns of the few rows' result, as a power of two: about 2048 waves in all (us, 1 / 2 / 4 / 8 waves to a tile, k = 2048,
// 512 tiles: 4.5 / 3.8 / 3.5 / 4.2; k = 8192, 128 tiles: 10.1 / 6.8 / 5.2 / 4.4; k = 2048, 3142 tiles: 11.1 / 12.0 / 14.1 / 17.8).
inline int sl_mx4_few_waves_log2(int64_t n)
{
    int log2 = 0;
    while (log2 < 3 && ((n + 15) / 16 << log2) < 2048) ++log2;
    return log2;
}
