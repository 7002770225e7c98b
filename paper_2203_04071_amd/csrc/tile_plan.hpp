// Which tile a dense product of tile_product.hpp takes.  Host only.
#pragma once
#include <stddef.h>

namespace adapt_api {

enum TileKind { TILE_256x256, TILE_256x128, TILE_128x128, TILE_128x128_TWO, TILE_128x64, TILE_64x64, TILE_64x64_SIX, TILE_KINDS };       // _TWO, _SIX: on a compute unit at a time

struct TilePlan {
    TileKind kind;
    int tm, tn;
    long long tiles_i, tiles_j;
    int split;                  // workgroups that share a tile, each with a part of the rows
    long long kb_split;         // bytes of a row in a part (whole stages)
};

// Times in microseconds: a stage (128 bytes of every row) of a workgroup that has a compute unit to itself, everything else of a tile
// (first requests, outputs), workgroups that a compute unit's LDS holds.  Small tiles hide the outputs of one behind the sums of others, large ones
// read the operands less often.  Measured on 2048 x 512 outputs over 300 stages (stages) and 6400 x 2048 fp32 outputs over 4 (the rest); those with
// several on a compute unit fitted to 177 drawn int8 products, for which the plan is 1.0 % slower than the best kind (6 % without _SIX).
//                                          256x256  256x128  128x128  _TWO  128x64  64x64  _SIX
//     8192 x 8192, 64 stages int8 -> bf16     469      487      596    707     804    881     -  us
//     4096 x 4096, 32 stages int8 -> bf16      63       63       72     80      98    106   152
//     2048 x 512, 300 stages bf16             309      161      104    160      83     -      -
//     6400 x 512, 96 stages bf16              107       62       43     55      62     -      -
//     1111 x 999, 32 stages int8               50       28       18     20      14    13     21
//     6400 x 2048, 4 stages int8 -> fp32       20       22       24     19      29    24     21
//     1300 x 9615, 2 stages int8 -> fp32       29       24       23     23      27    21     16
//     20000 x 512, 1 stage int8 -> fp16        13       14       13     11      15    13    9.6
struct TileCost {
    int tm, tn;
    double stage, rest;
    int per_cu;
    double alone;       // times of a stage that it takes however few workgroups share a compute unit
};
constexpr TileCost TILE_COST[TILE_KINDS] = {{256, 256, 1.03, 14.0, 1, 1.0}, {256, 128, 0.54, 7.5, 1, 1.0}, {128, 128, 0.35, 4.2, 1, 1.0},
                                            {128, 128, 0.59, 2.6, 2, 1.0},  {128, 64, 0.27, 2.3, 1, 1.0},  {64, 64, 0.20, 1.9, 2, 1.0},
                                            {64, 64, 0.22, 0.5, 6, 3.0}};

// A way to share a product out: tiles of a kind, rows in `split` parts of `part` stages, `groups` workgroups.
struct TileWay {
    long long ti, tj, part, groups;
    int split;
    double join;        // microseconds: fp32 sums written, read and added (3 us and a tenth a part, 4 TB/s)
};

// numbers of parts: the few that even out the last round, then those that fill the chip from a tile or two
constexpr int TILE_SPLITS[] = {1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 24, 32, 48, 64};
constexpr int TILE_WAYS = sizeof(TILE_SPLITS) / sizeof(int);

// The ways for one kind.  split > 0: that many parts; 0: any, parts of at least eight stages and up to two workgroups for every one that
// runs at a time.
inline int tile_ways(const TileCost &c, long long I, long long J, long long stages, int cus, int split, TileWay *ways) {
    const long long ti = (I + c.tm - 1) / c.tm, tj = (J + c.tn - 1) / c.tn, limit = 2ll * cus * c.per_cu;
    int n = 0;
    for (const int z : TILE_SPLITS) {
        const long long part = (stages + z - 1) / z;
        if (split && z != split) continue;
        if (!split && z > 1) {
            if (part < 8 || ti * tj * z > limit) break;
            if ((stages + part - 1) / part != z) continue;
        }
        ways[n++] = TileWay{ti, tj, part, ti * tj * z, z, z > 1 ? 3.0 + 0.1 * z + (double)(I * J) * 4.0 * (2 * z) / 4.0e6 : 0.0};
    }
    return n;
}
inline TilePlan tile_plan_of(int kind, const TileWay &w, long long Kb) {
    return TilePlan{(TileKind)kind, TILE_COST[kind].tm, TILE_COST[kind].tn, w.ti, w.tj, w.split, w.split > 1 ? w.part * 128 : Kb};
}
// workgroups on a compute unit share what one has; _SIX's have too little on its way to take it all
inline double tile_shared(const TileCost &c, long long groups, int cus) {
    const double n = groups >= (long long)c.per_cu * cus ? c.per_cu : (double)groups / cus;
    return n > c.alone ? n : c.alone;
}

// Kb: bytes of a row; split as above
inline TilePlan tile_plan(long long I, long long J, long long Kb, int cus, int split, double *us_out = nullptr) {
    TilePlan best{};
    double best_us = 0.0;
    TileWay ways[TILE_WAYS];
    for (int k = 0; k < TILE_KINDS; ++k) {
        const TileCost &c = TILE_COST[k];
        const int n = tile_ways(c, I, J, (Kb + 127) / 128, cus, split, ways);
        for (int i = 0; i < n; ++i) {
            const TileWay &w = ways[i];
            const long long slots = (long long)cus * c.per_cu;
            const double us = (double)((w.groups + slots - 1) / slots) * ((double)w.part * c.stage * tile_shared(c, w.groups, cus) + c.rest) + w.join;
            if (best_us == 0.0 || us < best_us) {
                best_us = us;
                best = tile_plan_of(k, w, Kb);
            }
        }
    }
    if (us_out) *us_out = best_us;
    return best;
}

// The end of n0 workgroups of t0 microseconds followed by n1 of t1 on so many slots, each taken by the next one as soon as it is free.
inline double tile_end(long long n0, double t0, long long n1, double t1, long long slots) {
    const long long rounds = n0 / slots, late = n0 % slots;         // `late` slots are free at a, the others at b
    const double b = (double)rounds * t0, a = late ? b + t0 : b;
    if (n1 <= 0) return a;
    auto whole = [](double x) { return x > 0.0 ? (long long)(x + 1e-9) : 0ll; };
    if (n1 <= (slots - late) * whole((a - b) / t1)) return a;
    // no slot waits: not before `least`; every slot loses less than one workgroup's time by that
    const double least = ((double)n1 * t1 + (double)late * a + (double)(slots - late) * b) / (double)slots;
    double best = least + t1;
    for (int of_b = 0; of_b < 2; ++of_b) {
        const double from = of_b ? b : a, end = from + (double)whole((least - from) / t1 + 1.0 - 2e-9) * t1;
        if (end >= a && late * whole((end - a) / t1) + (slots - late) * whole((end - b) / t1) >= n1 && end < best) best = end;
    }
    return best;
}

// Two products, in one launch of one kind of tile or one after the other.  One launch fills the last rounds of both and saves 3 us, but is one
// kind for two shapes.  Whole gradients in two launches and in one: 1000 x 1000 -> 1000 bf16 39.4 and 30.6 us, 6400 x 512 -> 2048 fp32 119.7 and 115.3, 3386 x 3066
// -> 408 bf16 90 and 68, 55 x 14134 -> 16177 fp32 593 and 641, 41 x 12179 -> 12837 bf16 366 and 390, 76 x 8301 -> 7271 bf16 170 and 155.  Above 40 us estimates
// decide by 2 % only; over 36 drawn gradients the plan is 0.5 % slower than one launch for all and 9 % faster than two (one of the last three sizes
// goes the wrong way).  The estimates are made for int8 products: those of fp16 numbers come out a quarter too short (6400 x 512 -> 2048 fp32 44 us,
// measured 60), which both sides of the comparison share.
struct TilePairPlan {
    TilePlan plan[2];
    bool joint;
    int first;          // which one's workgroups come first: the longer ones
};
inline TilePairPlan tile_pair_plan(const long long I[2], const long long J[2], const long long Kb[2], int cus) {
    TilePairPlan best{};
    double us0, us1;
    best.plan[0] = tile_plan(I[0], J[0], Kb[0], cus, 0, &us0);
    best.plan[1] = tile_plan(I[1], J[1], Kb[1], cus, 0, &us1);
    double best_us = us0 + us1 < 40.0 ? us0 + us1 + 3.0 : 0.98 * (us0 + us1);
    TileWay ways[2][TILE_WAYS];
    for (int k = 0; k < TILE_KINDS; ++k) {
        const TileCost &c = TILE_COST[k];
        const long long slots = (long long)cus * c.per_cu;
        int n[2];
        for (int x = 0; x < 2; ++x) n[x] = tile_ways(c, I[x], J[x], (Kb[x] + 127) / 128, cus, 0, ways[x]);
        for (int i = 0; i < n[0]; ++i)
            for (int j = 0; j < n[1]; ++j) {
                const TileWay &w0 = ways[0][i], &w1 = ways[1][j];
                const double shared = c.stage * tile_shared(c, w0.groups + w1.groups, cus);
                const double t0 = (double)w0.part * shared + c.rest, t1 = (double)w1.part * shared + c.rest;
                const bool swap = t1 > t0;
                const double us = (swap ? tile_end(w1.groups, t1, w0.groups, t0, slots) : tile_end(w0.groups, t0, w1.groups, t1, slots)) + w0.join + w1.join;
                if (us < best_us) {
                    best_us = us;
                    best.plan[0] = tile_plan_of(k, w0, Kb[0]);
                    best.plan[1] = tile_plan_of(k, w1, Kb[1]);
                    best.joint = true;
                    best.first = swap;
                }
            }
    }
    return best;
}

}  // namespace adapt_api
