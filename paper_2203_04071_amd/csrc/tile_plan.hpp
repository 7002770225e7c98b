// Which tile a dense product of tile_product.hpp takes.  Host only.
#pragma once
#include <stddef.h>

namespace adapt_api {

enum TileKind { TILE_256x256, TILE_256x128, TILE_128x128, TILE_128x128_TWO, TILE_128x64, TILE_64x64, TILE_KINDS };       // _TWO: on a compute unit at a time

struct TilePlan {
    TileKind kind;
    int tm, tn;
    long long tiles_i, tiles_j;
    int split;                  // workgroups that share a tile, each with a part of the rows
    long long kb_split;         // bytes of a row in a part (whole stages)
};

// Times in microseconds: a stage (128 bytes of every row) of a workgroup that has a compute unit to itself, everything else of a tile
// (first requests, outputs), workgroups that a compute unit's LDS holds.  Measured on 2048 x 512 outputs over 300 stages (stages) and
// 6400 x 2048 fp32 outputs over 4 (the rest).  Whole products:
//                                          256x256  256x128  128x128  _TWO  128x64  64x64
//     8192 x 8192, 64 stages int8 -> bf16     469      487      596    707     804    881 us
//     4096 x 4096, 128 stages bf16            210      221      248    321     361     -
//     2048 x 512, 300 stages bf16             309      161      104    160      83     -
//     6400 x 512, 96 stages bf16              107       62       43     55      62     -
//     1111 x 999, 32 stages int8               50       28       18     20      14    13
//     6400 x 2048, 4 stages int8 -> fp32       21       22       24     18      26    19
struct TileCost {
    int tm, tn;
    double stage, rest;
    int per_cu;
};
constexpr TileCost TILE_COST[TILE_KINDS] = {{256, 256, 1.03, 14.0, 1}, {256, 128, 0.54, 7.5, 1}, {128, 128, 0.35, 4.2, 1},
                                            {128, 128, 0.54, 4.0, 2},  {128, 64, 0.27, 2.3, 1},  {64, 64, 0.17, 1.1, 2}};

// Kb: bytes of a row.  max_split > 1: the rows may be split into that many parts of at least eight stages, whose fp32 sums are
// written, read and added afterwards (3 us, 4 TB/s).
inline TilePlan tile_plan(long long I, long long J, long long Kb, int cus, int max_split) {
    TilePlan best{};
    double best_us = 0.0;
    const long long stages = (Kb + 127) / 128;
    for (int k = 0; k < TILE_KINDS; ++k) {
        const TileCost &c = TILE_COST[k];
        const long long ti = (I + c.tm - 1) / c.tm, tj = (J + c.tn - 1) / c.tn, tiles = ti * tj;
        for (int split = 1; split <= max_split; ++split) {
            const long long part = (stages + split - 1) / split;
            if (split > 1 && (part < 8 || (stages + part - 1) / part != split)) continue;
            const long long groups = tiles * split, slots = (long long)cus * c.per_cu, rounds = (groups + slots - 1) / slots;
            // two workgroups on a compute unit share what one has
            const double shared = c.per_cu == 1 ? 1.0 : (groups <= cus ? 1.0 : (groups >= slots ? 2.0 : (double)groups / cus));
            double us = (double)rounds * ((double)part * c.stage * shared + c.rest);
            if (split > 1) us += 3.0 + (double)(I * J) * 4.0 * (2 * split) / 4.0e6;
            if (best_us == 0.0 || us < best_us) {
                best_us = us;
                best = TilePlan{(TileKind)k, c.tm, c.tn, ti, tj, split, split > 1 ? part * 128 : Kb};
            }
        }
    }
    return best;
}

}  // namespace adapt_api
