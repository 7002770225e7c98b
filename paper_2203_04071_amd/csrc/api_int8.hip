// C ABI, part 5: the exact 8-bit product with a scale for each token and channel, and its gradients.
#include "api_common.hpp"
#include "int8_gradient.hpp"
#include "int8_linear.hpp"
#include "tile_plan.hpp"

using namespace adapt_api;

namespace {

bool off_by(const void *p, size_t align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int INT8_MAX_K = 131071;              // (-128)^2 K < 2^31
constexpr long long MAX_TILES = 1ll << 24;      // a launch is limited to 2^32 threads
constexpr int TOKENS_GROUPS = 1 << 23;         // the same for workgroups of 512
constexpr int GRAD_MAX = 2097152;               // 256 rows of its pieces (4 bytes an element) are addressed with 32 bits

int int8_args(const char *who, int M, int K, int N, int type) {
    if (M < 0 || K < 0 || N < 0) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: negative size", who);
    if (!adapt::element_size(type)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: element type %d is none of ADAPT_F32, ADAPT_F16, ADAPT_BF16", who, type);
    return ADAPT_OK;
}

int grad_limits(const char *who, int M, int K, int N) {
    if (M > GRAD_MAX || K > GRAD_MAX || N > GRAD_MAX) return fail(ADAPT_ERR_UNSUPPORTED, "%s: a size above %d", who, GRAD_MAX);
    // (three matrices in blocks of 64 x 64, a workgroup of 256 each, in one launch of less than 2^32 threads)
    if ((long long)M * K >> 34 || (long long)N * K >> 34 || (long long)M * N >> 34) return fail(ADAPT_ERR_UNSUPPORTED, "%s: a matrix of 2^34 elements or more", who);
    return ADAPT_OK;
}

void set_tiles(adapt::TileParams &p, const TilePlan &t, size_t element) {
    p.tiles_i = (int)t.tiles_i;
    p.tiles_j = (int)t.tiles_j;
    p.Kb_split = (int)t.kb_split;
    p.stream = (double)p.I * (double)p.J * (double)element > 32.0e6;
}

template <class E, int TM, int TN, int SB, int NB, bool DMA, bool TANH = false>
void launch_tile(adapt::TileParams p, const TilePlan &t, hipStream_t s) {
    set_tiles(p, t, sizeof(typename E::mem));
    adapt::tile_product_kernel<adapt::TileI8, E, TM, TN, SB, NB, DMA, TANH><<<(unsigned)(t.tiles_i * t.tiles_j), adapt::TILE_THREADS, 0, s>>>(p);
}
template <class E, int TM, int TN, int SB, int NB, bool DMA>
void launch_tile(const adapt::TilePair &p, unsigned groups, hipStream_t s) {
    adapt::tile_product_kernel<adapt::TileF16, E, TM, TN, SB, NB, DMA><<<groups, adapt::TILE_THREADS, 0, s>>>(p);
}

// whole stages go from memory to LDS by themselves: rows of 16-byte pieces.  `t`: a plan, or the number of workgroups
template <class E, class Params, class Tiles>
void launch_tiles(TileKind kind, const Params &p, const Tiles &t, hipStream_t s) {
    switch (kind) {
        case TILE_256x256: launch_tile<E, 256, 256, 64, 4, true>(p, t, s); break;
        case TILE_256x128: launch_tile<E, 256, 128, 128, 3, true>(p, t, s); break;
        case TILE_128x128: launch_tile<E, 128, 128, 128, 4, true>(p, t, s); break;
        case TILE_128x128_TWO: launch_tile<E, 128, 128, 64, 3, true>(p, t, s); break;
        case TILE_128x64: launch_tile<E, 128, 64, 128, 4, true>(p, t, s); break;
        case TILE_64x64: launch_tile<E, 64, 64, 128, 4, true>(p, t, s); break;
        default: launch_tile<E, 64, 64, 64, 3, true>(p, t, s); break;
    }
}

TilePlan one_tile(long long I, long long J, long long Kb, int tm, int tn) {
    return TilePlan{TILE_KINDS, tm, tn, (I + tm - 1) / tm, (J + tn - 1) / tn, 1, Kb};
}

template <class E, int MT, bool TANH = false>
void launch_tokens(const adapt::Int8Params &p, hipStream_t s) {
    const dim3 grid((unsigned)(((long long)p.N + 15) / 16), (unsigned)((p.M + 16 * MT - 1) / (16 * MT)));
    if (p.K % 4) adapt::int8_tokens_kernel<E, MT, 8, true, TANH><<<grid, 512, 0, s>>>(p);
    else adapt::int8_tokens_kernel<E, MT, 8, false, TANH><<<grid, 512, 0, s>>>(p);
}

// Rows that no 16-byte piece divides: 64 x 64 outputs in stages of 64 bytes, several on a compute unit.  Fewer requests an output where the tiles are many
// and the sums not short (128 x 128) or the sums long (128 x 64 in stages of 128 bytes).  64 x 64, 128 x 64, 128 x 128 (us):
//     1111 x 777 -> 999 fp32       10.4  11.5  14.1        4000 x 1999 -> 2000 fp32    66   50   44
//     5952 x 167 -> 4096 fp16      36    43    34          4000 x 4001 -> 4000 bf16   227  164  140
//     7633 x 113 -> 5504 fp32      53    64    60          1111 x 4095 -> 999 bf16     31   26   38
//     20000 x 100 -> 500 fp16      12.5  15.2  17.9        556 x 2885 -> 576 fp32      14   19   25
template <class E>
void launch_ragged(const adapt::TileParams &p, hipStream_t s) {
    const TilePlan large = one_tile(p.I, p.J, p.Kb, 128, 128), middle = one_tile(p.I, p.J, p.Kb, 128, 64);
    if (p.Kb >= 512 && 2 * large.tiles_i * large.tiles_j >= 3 * device_cus()) launch_tile<E, 128, 128, 64, 2, false>(p, large, s);
    else if (p.Kb >= 2048 && middle.tiles_i * middle.tiles_j >= device_cus() / 2) launch_tile<E, 128, 64, 128, 2, false>(p, middle, s);
    else launch_tile<E, 64, 64, 64, 2, false>(p, one_tile(p.I, p.J, p.Kb, 64, 64), s);
}

// Few tokens, or few tiles: the kernel without LDS tiles (int8_tokens_kernel) reads 16 (MT + 1) K bytes per workgroup of 16 x 16 MT outputs, at about
// 13 TB/s from L2; a tile of 64 x 64 takes K / 128 stages of 0.15 us whatever the number of tiles, up to two per compute unit.  They meet where
// (MT + 1) times the number of workgroups is 900: 32 x 4096 x 4096 8.1 us against 10.4, 64 x 4096 x 4096 11.6 against 10.1, 64 x 8192 -> 256
// 9.1 against 17, 8 x 4096 -> 16384 17 against 12.  Rows that are no multiple of 16 bytes (up to 64 tokens): always.
int tokens_kernel_mt(int M, int N, bool dma) {
    const long long n16 = ((long long)N + 15) / 16;
    if (n16 >= TOKENS_GROUPS) return 0;
    const int mts[3] = {1, 2, 4};
    int best = 0;
    long long best_cost = 0;
    for (int mt : mts) {
        const long long cost = (mt + 1) * n16 * ((M + 16 * mt - 1) / (16 * mt));
        if (!best || cost < best_cost) {
            best = mt;
            best_cost = cost;
        }
    }
    // (few workgroups: smaller ones, to have more)
    for (int mt : mts) {
        const long long groups = n16 * ((M + 16 * mt - 1) / (16 * mt));
        if (mt < best && (mt + 1) * groups < 450) {
            best = mt;
            best_cost = (mt + 1) * groups;
            break;
        }
    }
    return best_cost < 900 || (!dma && M <= 64) ? best : 0;
}

template <class E>
void launch_int8(const adapt::Int8Params &q, hipStream_t s) {
    const bool dma = q.K % 16 == 0 && aligned16(q.a) && aligned16(q.w);
    adapt::TileParams p{};
    p.a = reinterpret_cast<const char *>(q.a);
    p.b = reinterpret_cast<const char *>(q.w);
    p.I = q.M;
    p.J = q.N;
    p.Kb = q.K;
    p.lda = p.ldb = (uint32_t)q.K;
    p.s_i = q.s_a;
    p.s_j = q.s_w;
    p.bias = q.bias;
    p.act = q.act;
    p.c = q.y;
    const TilePlan small = one_tile(p.I, p.J, p.Kb, 64, 64);
    // (tanh: one kernel for each way of reading.  6400 x 512 -> 2048 fp32 35 us where the plain product takes 19, 8192^3 bf16 925 against 477, up to 40 tokens the same)
    if (q.act == 2) {
        if (q.M <= 16 && q.N <= 16 * (TOKENS_GROUPS - 1)) launch_tokens<E, 1, true>(q, s);
        else if (dma) launch_tile<E, 64, 64, 128, 4, true, true>(p, small, s);
        else launch_tile<E, 64, 64, 64, 2, false, true>(p, small, s);
        return;
    }
    switch (tokens_kernel_mt(q.M, q.N, dma)) {
        case 1: launch_tokens<E, 1>(q, s); return;
        case 2: launch_tokens<E, 2>(q, s); return;
        case 4: launch_tokens<E, 4>(q, s); return;
    }
    if (dma) {
        const TilePlan t = tile_plan(p.I, p.J, p.Kb, device_cus(), 1);
        launch_tiles<E>(t.kind, p, t, s);
    } else {
        launch_ragged<E>(p, s);
    }
}

int grad_whole(long long R) { return (int)((R + adapt::GRAD_STAGE - 1) / adapt::GRAD_STAGE * adapt::GRAD_STAGE); }

// Workspace of one gradient c [I][J], the sums over R: rows of the pieces of dy s [I], rows of codes [J], the rows' exponents, partial sums of
// a split product.
struct GradPlan {
    int Rp;                     // R in whole stages
    long long row, row_b;       // bytes of a row of pieces, of codes
    TilePlan tile;
    size_t b, exps, part, bytes;    // offsets (a at 0)
};
// (the tile comes from grad_plans)
GradPlan grad_plan(long long I, long long J, long long R, const TilePlan &tile) {
    GradPlan g{};
    g.Rp = grad_whole(R);
    g.row = 2ll * adapt::GRAD_PIECES * g.Rp;
    g.row_b = 2ll * g.Rp;
    g.tile = tile;
    g.b = round256((size_t)I * (size_t)g.row);
    g.exps = g.b + round256((size_t)J * (size_t)g.row_b);
    g.part = g.exps + round256((size_t)I * 4);
    g.bytes = g.part + (g.tile.split > 1 ? round256((size_t)g.tile.split * (size_t)I * (size_t)J * 4) : 0);
    return g;
}

// partial results of the columns, sums and largest elements: rows that a block takes, blocks, bytes
int column_rows(int M) {
    const int share = (M + adapt::GRAD_BLOCKS - 1) / adapt::GRAD_BLOCKS;
    return share <= adapt::GRAD_ROWS ? adapt::GRAD_ROWS : (share + adapt::GRAD_ROWS - 1) / adapt::GRAD_ROWS * adapt::GRAD_ROWS;
}
int column_blocks(int M) { return (int)((M + (long long)column_rows(M) - 1) / column_rows(M)); }
size_t column_bytes(int M, int N) { return 2 * round256((size_t)(M ? column_blocks(M) : 1) * (size_t)N * 4); }

// Workspace of a call: what dx needs, what dw needs, the columns' partial results.
struct GradPlans {
    GradPlan x, w;              // all zeros where the gradient is not wanted
    bool joint;                 // their products are one launch
    int first;                  // 1: dw's workgroups come first
    size_t bytes;
};
GradPlans grad_plans(int M, int K, int N, bool want_dx, bool want_dw) {
    const int cus = device_cus();
    const long long I[2] = {M, N}, J[2] = {K, K}, Kb[2] = {2ll * adapt::GRAD_PIECES * grad_whole(N), 2ll * adapt::GRAD_PIECES * grad_whole(M)};
    // (a gradient has the same bits whatever else is asked for: the number of parts is the pair's, the tile that which is best for it alone)
    TilePairPlan t = tile_pair_plan(I, J, Kb, cus);
    if (!want_dx || !want_dw) {
        t.joint = false;
        for (int x = 0; x < 2; ++x) t.plan[x] = tile_plan(I[x], J[x], Kb[x], cus, t.plan[x].split);
    }
    GradPlans g{};
    if (want_dx) g.x = grad_plan(M, K, N, t.plan[0]);
    if (want_dw) g.w = grad_plan(N, K, M, t.plan[1]);
    g.joint = t.joint;
    g.first = t.first;
    g.bytes = g.x.bytes + g.w.bytes + column_bytes(M, N);
    return g;
}

adapt::TileParams grad_params(const GradPlan &g, char *ws, int I, int J, void *c, size_t element) {
    adapt::TileParams p{};
    p.a = ws;
    p.b = ws + g.b;
    p.exp_i = reinterpret_cast<const int *>(ws + g.exps);
    p.I = I;
    p.J = J;
    p.Kb = (int)g.row;
    p.Kb_b = (int)g.row_b;
    p.lda = (uint32_t)g.row;
    p.ldb = (uint32_t)g.row_b;
    p.parts = g.tile.split > 1;
    p.c = p.parts ? ws + g.part : c;
    set_tiles(p, g.tile, p.parts ? 4 : element);
    return p;
}
unsigned grad_groups(const GradPlan &g) { return (unsigned)(g.tile.tiles_i * g.tile.tiles_j * g.tile.split); }

template <class E>
void grad_join(const GradPlan &g, const char *ws, int I, int J, void *c, hipStream_t s) {
    if (g.tile.split == 1) return;
    const size_t n = (size_t)I * (size_t)J;
    adapt::grad_join_kernel<E><<<ew_grid(n / 4 + 1), 256, 0, s>>>(reinterpret_cast<const float *>(ws + g.part), g.tile.split, n, static_cast<typename E::mem *>(c));
}

// a wave per row up to 1024 elements, a workgroup up to 8192 (quantize_tokens has the like); a workgroup takes several rows, whose scales of the
// columns it reads once
template <class E>
void prepare(const adapt::GradPrep &p, unsigned groups, hipStream_t s) {
    constexpr int T = adapt::GRAD_THREADS;
    if (p.Np <= 512) adapt::grad_prepare_kernel<E, 64, 1><<<groups, T, 0, s>>>(p);
    else if (p.Np <= 1024) adapt::grad_prepare_kernel<E, 64, 2><<<groups, T, 0, s>>>(p);
    else if (p.Np <= 2048) adapt::grad_prepare_kernel<E, T, 1><<<groups, T, 0, s>>>(p);
    else if (p.Np <= 4096) adapt::grad_prepare_kernel<E, T, 2><<<groups, T, 0, s>>>(p);
    else if (p.Np <= 8192) adapt::grad_prepare_kernel<E, T, 4><<<groups, T, 0, s>>>(p);
    else adapt::grad_prepare_kernel<E, 0, 0><<<groups, T, 0, s>>>(p);
}

template <class E>
void gradients(const adapt::Int8Params &q, const GradPlans &plans, const void *dy, void *dx, void *dw, void *db_dev, char *ws, hipStream_t s) {
    typedef typename E::mem mem;
    mem *const db = static_cast<mem *>(db_dev);
    const GradPlan &gx = plans.x, &gw = plans.w;
    char *const wx = ws, *const ww = ws + gx.bytes, *const wc = ww + gw.bytes;
    auto blocks = [](int n) { return (uint32_t)((n + 63) / 64); };
    adapt::GradPrep p{};
    p.dy = dy;
    p.s_a = q.s_a;
    p.s_w = q.s_w;
    p.a = q.a;
    p.w = q.w;
    p.M = q.M;
    p.K = q.K;
    p.N = q.N;
    p.Np = gx.Rp;
    p.Mp = gw.Rp;
    p.rows = column_rows(q.M);
    p.dy_rows = reinterpret_cast<_Float16 *>(wx);
    p.w_codes = reinterpret_cast<_Float16 *>(wx + gx.b);
    p.row_exps = reinterpret_cast<int *>(wx + gx.exps);
    p.a_codes = reinterpret_cast<_Float16 *>(ww + gw.b);
    p.sum = db ? reinterpret_cast<float *>(wc) : nullptr;
    p.big = dw ? reinterpret_cast<float *>(wc + column_bytes(q.M, q.N) / 2) : nullptr;
    if (dx) {
        const uint32_t rows = p.Np <= 1024 ? ((uint32_t)q.M + 3) / 4 : (uint32_t)q.M;
        p.row_groups = rows < 2048 ? rows : 2048;
        p.w_blocks = (uint32_t)gx.Rp / 64;
        p.w_groups = p.w_blocks * blocks(q.K);
    }
    if (dw || db) {
        p.column_blocks = (uint32_t)column_blocks(q.M);
        p.column_groups = p.column_blocks * blocks(q.N);
    }
    uint32_t a_groups = 0;
    if (dw) {
        p.a_blocks = (uint32_t)gw.Rp / 64;
        a_groups = p.a_blocks * blocks(q.K);
    }
    const uint32_t groups = p.row_groups + p.w_groups + p.column_groups + a_groups;
    if (groups) prepare<E>(p, groups, s);
    adapt::TileParams px{}, pw{};
    if (dx) px = grad_params(gx, wx, q.M, q.K, dx, sizeof(mem));
    if (dw) pw = grad_params(gw, ww, q.N, q.K, dw, sizeof(mem));
    const unsigned nx = grad_groups(gx), nw = grad_groups(gw);
    if (dx && !plans.joint) launch_tiles<E>(gx.tile.kind, adapt::TilePair{{px, px}, nx}, nx, s);
    if (dw && gw.Rp) {
        adapt::grad_turned_rows_kernel<E><<<dim3((unsigned)gw.Rp / 64, blocks(q.N)), 256, 0, s>>>(
            static_cast<const mem *>(dy), q.s_a, p.sum, p.big, db, reinterpret_cast<int *>(ww + gw.exps), reinterpret_cast<_Float16 *>(ww), q.M, q.N, gw.Rp,
            column_blocks(q.M));
    } else {
        if (dw) adapt::fill_u32_kernel<<<ew_grid((size_t)q.N), 256, 0, s>>>(reinterpret_cast<uint32_t *>(ww + gw.exps), 0u, (size_t)q.N);
        if (db) adapt::grad_bias_kernel<E><<<blocks(q.N), adapt::GRAD_THREADS, 0, s>>>(p.sum, db, column_blocks(q.M), q.N);
    }
    if (plans.joint) launch_tiles<E>(gx.tile.kind, plans.first ? adapt::TilePair{{pw, px}, nw} : adapt::TilePair{{px, pw}, nx}, nx + nw, s);
    else if (dw) launch_tiles<E>(gw.tile.kind, adapt::TilePair{{pw, pw}, nw}, nw, s);
    if (dx) grad_join<E>(gx, wx, q.M, q.K, dx, s);
    if (dw) grad_join<E>(gw, ww, q.N, q.K, dw, s);
}

}  // namespace

extern "C" {

int adapt_int8_linear(const int8_t *a_dev, const float *s_a_dev, const int8_t *w_dev, const float *s_w_dev, const float *bias_dev, int act,
                      void *y_dev, int y_type, int M, int K, int N, void *stream) {
    const char *who = "adapt_int8_linear";
    if (int rc = int8_args(who, M, K, N, y_type)) return rc;
    if (act < 0 || act > 2) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: act=%d not in [0,2]", who, act);
    if (!M || !N) return ADAPT_OK;
    if (!s_a_dev || !s_w_dev || !y_dev || (K && (!a_dev || !w_dev))) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL pointer", who);
    if (off_by(s_a_dev, 4) || off_by(s_w_dev, 4) || off_by(bias_dev, 4) || off_by(y_dev, (size_t)adapt::element_size(y_type)))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (is_one_of(y_dev, {a_dev, w_dev, s_a_dev, s_w_dev, bias_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: in-place not possible", who);
    if (K > INT8_MAX_K) return fail(ADAPT_ERR_UNSUPPORTED, "%s: K=%d above %d, sums could pass 32 bits", who, K, INT8_MAX_K);
    if ((((long long)M + 63) / 64) * (((long long)N + 63) / 64) >= MAX_TILES) return fail(ADAPT_ERR_UNSUPPORTED, "%s: 2^24 blocks of 64 x 64 outputs or more", who);
    const adapt::Int8Params p{a_dev, w_dev, s_a_dev, s_w_dev, bias_dev, y_dev, M, K, N, act};
    ADAPT_FOR_TYPE(y_type, E, launch_int8<E>(p, (hipStream_t)stream));
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

int adapt_int8_linear_backward_workspace(int M, int K, int N, int type, int want_dx, int want_dw, size_t *bytes) {
    const char *who = "adapt_int8_linear_backward_workspace";
    if (!bytes) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: bytes is NULL", who);
    *bytes = 0;
    if (int rc = int8_args(who, M, K, N, type)) return rc;
    if (int rc = grad_limits(who, M, K, N)) return rc;
    *bytes = grad_plans(M, K, N, want_dx && M && K, want_dw && N && K).bytes;
    return ADAPT_OK;
}

int adapt_int8_linear_backward(const void *dy_dev, int type, const int8_t *a_dev, const float *s_a_dev, const int8_t *w_dev, const float *s_w_dev,
                               int M, int K, int N, void *dx_dev, void *dw_dev, void *db_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
    const char *who = "adapt_int8_linear_backward";
    if (int rc = int8_args(who, M, K, N, type)) return rc;
    const size_t e = (size_t)adapt::element_size(type);
    const bool want_dx = dx_dev && M > 0 && K > 0, want_dw = dw_dev && N > 0 && K > 0, want_db = db_dev && N > 0;
    if (!want_dx && !want_dw && !want_db) return ADAPT_OK;
    if (M > 0 && N > 0 && !dy_dev) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL dy_dev", who);
    if (want_dx && N > 0 && (!w_dev || !s_w_dev)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL w_dev / s_w_dev", who);
    if (want_dw && M > 0 && (!a_dev || !s_a_dev)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL a_dev / s_a_dev", who);
    for (const void *q : {dy_dev, (const void *)dx_dev, (const void *)dw_dev, (const void *)db_dev})
        if (off_by(q, e)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (off_by(s_a_dev, 4) || off_by(s_w_dev, 4)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    for (const void *g : {dx_dev, dw_dev, db_dev})
        if (is_one_of(g, {dy_dev, a_dev, w_dev, s_a_dev, s_w_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: a gradient must not alias an input", who);
    if (is_one_of(dx_dev, {dw_dev, db_dev}) || is_one_of(dw_dev, {db_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: gradients must not alias each other", who);
    if (is_one_of(workspace_dev, {dy_dev, a_dev, w_dev, s_a_dev, s_w_dev, dx_dev, dw_dev, db_dev}))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: the workspace must not alias an operand or a gradient", who);
    if (int rc = grad_limits(who, M, K, N)) return rc;
    const GradPlans plans = grad_plans(M, K, N, want_dx, want_dw);
    const size_t need = plans.bytes;
    if (need && (!workspace_dev || workspace_bytes < need || off_by(workspace_dev, 256)))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: workspace of %zu bytes, aligned to 256, is needed", who, need);
    const adapt::Int8Params p{a_dev, w_dev, s_a_dev, s_w_dev, nullptr, nullptr, M, K, N, 0};
    char *const ws = static_cast<char *>(workspace_dev);
    void *const dx = want_dx ? dx_dev : nullptr, *const dw = want_dw ? dw_dev : nullptr, *const db = want_db ? db_dev : nullptr;
    hipStream_t s = (hipStream_t)stream;
    ADAPT_FOR_TYPE(type, E, gradients<E>(p, plans, dy_dev, dx, dw, db, ws, s));
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

}  // extern "C"
