// The dense product of the token-wise operators, c[i][j] = sum over r of a[i][r] b[j][r], on rows of int8 codes or of fp16 numbers: both
// matrix instructions take 16 bytes of a row per lane and 32 bytes per step, so one kernel in bytes serves both.
#pragma once
#include <type_traits>

#include "element.hpp"
#include "elementwise.hpp"

namespace adapt {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef float tile_f32x16_t __attribute__((ext_vector_type(16)));
typedef float tile_f32x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr int TILE_THREADS = 256;       // four waves, 2 x 2 over the tile

struct TileParams {
    const char *a, *b;
    int I, J, Kb;               // Kb: bytes of a row that are summed over
    int Kb_b;                   // fp16: bytes of a row of b (whole stages), which meets a's again and again
    const int *exp_i;           // fp16: a row of sums is worth times 2^exp_i
    uint32_t lda, ldb;          // bytes from row to row
    int tiles_i, tiles_j;
    // int8: rescaling by row and column, bias, activation
    const float *s_i, *s_j, *bias;
    int act;
    int Kb_split;               // fp16: bytes of a row that a workgroup sums over: number y takes the ones from y Kb_split, into c + y I J
    bool parts;                 // fp16: c is fp32 whatever E, sums of parts
    int stream;                 // c is larger than the caches: written past them
    void *c;                    // [I][J]
};

// One product, or two of fp16 numbers (a layer's two gradients) in one launch.
struct TilePair {
    TileParams p[2];
    uint32_t first;             // workgroups of the first one
};

struct TileI8 {
    typedef i32x16_t acc_t;
    typedef TileParams args_t;
    static constexpr bool INT = true;
    static __device__ __forceinline__ acc_t mfma(i32x4_t a, i32x4_t b, acc_t c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
struct TileF16 {
    typedef tile_f32x16_t acc_t;
    typedef TilePair args_t;
    static constexpr bool INT = false;
    static __device__ __forceinline__ acc_t mfma(i32x4_t a, i32x4_t b, acc_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
};

// What becomes of a sum: rescaled, the bias added (0 for none), the activation.  `floor`: 0 for a ReLU, NaN for none (a maximum with
// NaN is the other number, NaN included).  TANH: the instantiations that also know tanh (its code, once per output of a lane, is
// longer than all the rest).
template <bool TANH>
__device__ __forceinline__ float int8_finish(int acc, float s_a, float s_w, float bias, float floor, int act) {
    const float y = __builtin_fmaxf(((float)acc * s_a) * s_w + bias, floor);
    return TANH && act == 2 ? tanh_spec(y) : y;
}
__device__ __forceinline__ float int8_floor(int act) {
    float f = act == 1 ? 0.0f : __builtin_nanf("");
    asm("" : "+v"(f));                      // (else the maximum becomes a comparison and a selection)
    return f;
}

// 16 bytes k .. k + 15 of a row of K, zeros beyond its end; nothing outside the row is read.  From 16 bytes on without a branch (the
// last 16 of the row, moved down), so that several requests are on their way together.
__device__ __forceinline__ i32x4_t row_piece(const char *__restrict__ row, int k, int K) {
    unsigned __int128 t = 0;
    if (K >= 16) {
        const int at = min(k, K - 16), down = k - at;
        __builtin_memcpy(&t, row + at, 16);
        t = down < 16 ? t >> (8 * (down & 15)) : 0;
    } else {
        for (int i = K - 1; i >= k; --i) t = t << 8 | (uint8_t)row[i];
    }
    i32x4_t v;
    __builtin_memcpy(&v, &t, 16);
    return v;
}

__device__ __forceinline__ bool tile_second(const TileParams &) { return false; }
__device__ __forceinline__ bool tile_second(const TilePair &a) { return blockIdx.x >= a.first; }
__device__ __forceinline__ const TileParams &tile_params(const TileParams &a, bool) { return a; }
__device__ __forceinline__ const TileParams &tile_params(const TilePair &a, bool second) { return a.p[second]; }

// Which tile a workgroup computes.  Consecutive workgroups go to different XCDs, each with an L2 of its own: an XCD gets a contiguous
// range of tiles, and the range runs through groups of four rows of tiles, so that the tiles in flight on an XCD share operands.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_i, uint32_t tiles_j, uint32_t &ti, uint32_t &tj) {
    const uint32_t n = tiles_i * tiles_j, q = n / 8, r = n % 8, xcd = id % 8;
    const uint32_t t = xcd * q + min(xcd, r) + id / 8;
    const uint32_t group = 4 * tiles_j, g = t / group, first = g * 4, rows = min(4u, tiles_i - first), in = t - g * group;
    ti = first + in % rows;
    tj = in / rows;
}

// columns of a wave's outputs that turn through LDS at a time
template <class E, int WJ>
constexpr int turn_columns = WJ * (int)sizeof(typename E::mem) < 256 ? WJ : 256 / (int)sizeof(typename E::mem);
template <class E, int TM, int TN>
constexpr int turn_bytes = 2 * TM * (turn_columns<E, TN / 2> * (int)sizeof(typename E::mem) + 16);
constexpr int tile_larger(int a, int b) { return a > b ? a : b; }

// Register v of lane l holds column 8 (v / 4) + 4 (l / 32) + v % 4 of row l % 32 of a 32 x 32 block.  A wave turns its outputs through
// LDS, up to 256 bytes of every row at a time, so that a store is 16 bytes of a lane and a row's pieces lie together.
template <class Op, class E, int TM, int TN, bool TANH, int LDS_BYTES>
__device__ __forceinline__ void tile_output(const TileParams &p, const typename Op::acc_t (&acc)[TM / 64][TN / 64], char *lds, const float *side, int i0, int j0, uint32_t part) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = (wave & 1) * (TM / 2), wj = (wave >> 1) * (TN / 2);
    constexpr int BI = TM / 64, BJ = TN / 64, WI = TM / 2, WJ = TN / 2, SIZE = (int)sizeof(typename E::mem);
    constexpr int CB = turn_columns<E, WJ>;                        // columns at a time
    constexpr int ROW = CB * SIZE + 16;                            // (rows start in different banks)
    constexpr int PL = piece_len<E>, LANES = CB / PL;              // lanes that store a row
    static_assert(4 * WI * ROW <= LDS_BYTES, "the turned outputs of four waves");
    char *const turn = lds + wave * (WI * ROW);
    typename E::mem *const c = static_cast<typename E::mem *>(p.c) + (size_t)part * (size_t)p.I * (size_t)p.J;
    const float floor = int8_floor(p.act);
    const bool whole = i0 + TM <= p.I && j0 + TN <= p.J;
#pragma unroll
    for (int cb = 0; cb < WJ / CB; ++cb) {
#pragma unroll
        for (int bi = 0; bi < BI; ++bi) {
            const float s_i = side[wi + 32 * bi + (lane & 31)];
#pragma unroll
            for (int bj = cb * (CB / 32); bj < (cb + 1) * (CB / 32); ++bj) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int col = 32 * bj + 8 * g + 4 * (lane >> 5);
                    float y[4];
                    if constexpr (Op::INT) {
                        const tile_f32x4_t sv = *reinterpret_cast<const tile_f32x4_t *>(&side[TM + wj + col]);
                        const tile_f32x4_t bv = *reinterpret_cast<const tile_f32x4_t *>(&side[TM + TN + wj + col]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) y[v] = int8_finish<TANH>(acc[bi][bj][4 * g + v], s_i, sv[v], bv[v], floor, p.act);
                    } else {
#pragma unroll
                        for (int v = 0; v < 4; ++v) y[v] = __builtin_amdgcn_ldexpf(acc[bi][bj][4 * g + v], __float_as_int(s_i));
                    }
                    typedef typename E::mem quad_t __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<quad_t *>(turn + (32 * bi + (lane & 31)) * ROW + (col - cb * CB) * SIZE) =
                        quad_t{E::store(y[0]), E::store(y[1]), E::store(y[2]), E::store(y[3])};
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");       // (a wave's own outputs: no barrier)
        const int r0 = lane / LANES, col = (lane % LANES) * PL, j = j0 + wj + cb * CB + col;
        const char *from = turn + r0 * ROW + col * SIZE;
        typename E::mem *to = c + (size_t)(i0 + wi + r0) * (size_t)p.J + (size_t)j;
        const size_t next = (size_t)(64 / LANES) * (size_t)p.J;
        typedef i32x4_t piece_t __attribute__((aligned(2)));       // (a row starts at any element)
        if (whole && p.stream) {        // (outputs beyond the caches: 6400 x 512 -> 2048 fp32 20.0 -> 18.2 us)
#pragma unroll 8
            for (int u = 0; u < WI * LANES / 64; ++u, from += 64 / LANES * ROW, to += next)
                __builtin_nontemporal_store(*reinterpret_cast<const i32x4_t *>(from), reinterpret_cast<piece_t *>(to));
        } else if (whole) {
#pragma unroll 8
            for (int u = 0; u < WI * LANES / 64; ++u, from += 64 / LANES * ROW, to += next) *reinterpret_cast<piece_t *>(to) = *reinterpret_cast<const i32x4_t *>(from);
        } else {
#pragma unroll 1
            for (int i = i0 + wi + r0; i < min(p.I, i0 + wi + WI); i += 64 / LANES, from += 64 / LANES * ROW, to += next) {
                if (j + PL <= p.J) {
                    *reinterpret_cast<piece_t *>(to) = *reinterpret_cast<const i32x4_t *>(from);
                } else {
#pragma unroll 1
                    for (int x = 0; j + x < p.J; ++x) to[x] = reinterpret_cast<const typename E::mem *>(from)[x];
                }
            }
        }
        if (cb + 1 < WJ / CB) asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    }
}

// TM x TN outputs per workgroup, (TM / 2) x (TN / 2) per wave in blocks of 32 x 32; NB LDS buffers (stages) of SB bytes of every row.  A row's pieces
// of 16 bytes lie in an order that depends on the row, so that 16 neighbouring lanes (16 rows, one piece) read 64 different banks.
//
// Bounded by the matrix pipe: a step of 32 bytes is 16 instructions of 32 clocks for a wave of the largest tile, over which it issues eight
// LDS reads and four requests to memory.  256 x 256 outputs in four waves, one per SIMD, keep LDS at 1/4 of its rate (eight waves of
// 128 x 64 would read 1.5 times as much) and leave 512 registers a lane, half of them sums.
//
// DMA: rows are multiples of 16 bytes and 16-byte aligned; pieces go from memory to LDS without registers, requested NB - 1 stages ahead, one
// barrier a stage.  8192 x 8192 x 8192 int8 -> bf16 466 - 478 us, 2.3 POP/s; on all compute units the clock falls to 1.8 GHz, at which the matrix
// pipe is busy for 3/4 of the time (alone on the chip a workgroup keeps it busy for 83 %).
// Otherwise (rows of any length and address): pieces pass through registers, three stages ahead, which also put zeros behind a row's end.  Bounded by
// the memory pipe, which takes longer over 16 bytes at an odd address: 1111 x 4096 -> 999 21 us against 14, 4095 26 us.
template <class Op, class E, int TM, int TN, int SB, int NB, bool DMA, bool TANH = false>
__global__ __launch_bounds__(TILE_THREADS) void tile_product_kernel(const typename Op::args_t args) {
    const bool second = tile_second(args);
    const TileParams &p = tile_params(args, second);
    uint32_t id = blockIdx.x, part = 0;
    if constexpr (!Op::INT) {
        if (second) id -= args.first;
        const uint32_t tiles = (uint32_t)p.tiles_i * (uint32_t)p.tiles_j;
        part = id / tiles;
        id -= part * tiles;
    }
    const int k0 = Op::INT ? 0 : (int)part * p.Kb_split, Kb = Op::INT ? p.Kb : min(p.Kb - k0, p.Kb_split);
    constexpr int BI = TM / 64, BJ = TN / 64, NR = BI + BJ, NS = BI * BJ;
    constexpr int PIECES = SB / 16, RQ = 64 / PIECES;              // pieces of a row in a stage, rows of a request
    constexpr int QA = TM / RQ / 4, QB = TN / RQ / 4, NQ = QA + QB;         // 1 KB requests of a wave per stage
    constexpr int STAGE = (TM + TN) * SB, STEPS = SB / 32;
    constexpr int LDS_BYTES = tile_larger(NB * STAGE, tile_larger(turn_bytes<E, TM, TN>, Op::INT ? 0 : turn_bytes<F32, TM, TN>));
    __shared__ __align__(1024) char lds[LDS_BYTES];
    constexpr int SIDE_N = Op::INT ? TM + 2 * TN : TM;
    __shared__ __align__(16) float side[SIDE_N];            // s_i, s_j, bias of the tile, or the bits of exp_i
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t ti, tj;
    tile_of(id, (uint32_t)p.tiles_i, (uint32_t)p.tiles_j, ti, tj);
    const int i0 = (int)ti * TM, j0 = (int)tj * TN;
    const int wi = (wave & 1) * (TM / 2), wj = (wave >> 1) * (TN / 2);

    constexpr int SIDE = (SIDE_N + TILE_THREADS - 1) / TILE_THREADS;
    float side_v[SIDE];                     // (requested now, put into LDS when the sums are done)
#pragma unroll
    for (int u = 0; u < SIDE; ++u) {
        const int x = u * TILE_THREADS + (int)threadIdx.x;
        side_v[u] = 0.0f;
        if constexpr (Op::INT) {
            if (x < TM) side_v[u] = p.s_i[min(i0 + x, p.I - 1)];
            else if (x < TM + TN) side_v[u] = p.s_j[min(j0 + x - TM, p.J - 1)];
            else if (x < TM + 2 * TN && p.bias) side_v[u] = p.bias[min(j0 + x - TM - TN, p.J - 1)];
        } else {
            if (x < TM) side_v[u] = __int_as_float(p.exp_i[min(i0 + x, p.I - 1)]);
        }
    }

    // requests: number q of a wave covers RQ rows from RQ (4 q + wave) on, lane l row l / PIECES and the piece that belongs at place l % PIECES
    static_assert(SB == 64 || SB == 128, "places of a row's pieces");
    auto swizzle = [](int row) { return SB == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
    const int prow = lane / PIECES, piece16 = ((lane % PIECES) ^ swizzle(RQ * wave + prow)) * 16;
    const char *abase = p.a + (size_t)i0 * p.lda + k0, *bbase = p.b + (size_t)j0 * p.ldb;
    uint32_t voff[NQ];
#pragma unroll
    for (int q = 0; q < QA; ++q) voff[q] = (uint32_t)min(RQ * (4 * q + wave) + prow, p.I - 1 - i0) * p.lda + (DMA ? (uint32_t)piece16 : 0u);
#pragma unroll
    for (int q = 0; q < QB; ++q) voff[QA + q] = (uint32_t)min(RQ * (4 * q + wave) + prow, p.J - 1 - j0) * p.ldb + (DMA ? (uint32_t)piece16 : 0u);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    auto place = [&](int q) { return (q < QA ? (4 * q + wave) * 1024 : TM * SB + (4 * (q - QA) + wave) * 1024); };

    // fragments: block b of a wave, lane l: row 32 b + l % 32, piece 2 step + l / 32
    const char *const frag_a = lds + (wi + (lane & 31)) * SB, *const frag_b = lds + TM * SB + (wj + (lane & 31)) * SB;
    i32x4_t f[2][NR];
    auto read1 = [&](i32x4_t(&to)[NR], int r, int buf, int step) {
        const int at = buf * STAGE + (((2 * step + (lane >> 5)) ^ swizzle(lane)) << 4);
        to[r] = r < BI ? *reinterpret_cast<const i32x4_t *>(frag_a + at + r * 32 * SB) : *reinterpret_cast<const i32x4_t *>(frag_b + at + (r - BI) * 32 * SB);
    };
    typename Op::acc_t acc[BI][BJ] = {};

    const int full = Kb / SB, rest = Kb - full * SB;
    const int total = full + (rest ? 1 : 0);        // (rows of fp16 are made in whole stages)

    if constexpr (DMA) {
        int dma_s = 0;          // stage that is requested next
        const int Kb_b = p.Kb_b;        // (a copy: the parameters of a pair would be read again in every stage)
        int kb = Op::INT || total == 0 ? 0 : k0 % Kb_b;        // (no sums: no rows of b either)
        const char *da = abase, *db = bbase + kb;
        auto dma_begin = [&]() {        // where the last stage is not whole, lanes whose piece lies behind the end fetch its first piece instead
            if (Op::INT && dma_s == full && piece16 >= rest)
#pragma unroll
                for (int q = 0; q < NQ; ++q) voff[q] -= (uint32_t)piece16;
        };
        auto dma1 = [&](int q, int buf) {
            const uint32_t to = lds0 + (uint32_t)(buf * STAGE + place(q));
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(voff[q]), "s"(q < QA ? da : db) : "memory", "m0");
        };
        auto dma_end = [&]() {
            da += SB;
            db += SB;
            ++dma_s;
            if constexpr (!Op::INT) {
                kb += SB;
                if (kb == Kb_b) {
                    kb = 0;
                    db = bbase;
                }
            }
        };
        auto dma_stage = [&](int buf) {
            dma_begin();
#pragma unroll
            for (int q = 0; q < NQ; ++q) dma1(q, buf);
            dma_end();
        };
        // one step: the matrix instructions of `cur`, between them the reads of `next` and a share of a stage's requests.  (All of a
        // stage's requests in one step kept the four waves waiting for the memory pipe, which takes 64 bytes a clock.)
        auto step = [&](const i32x4_t(&cur)[NR], i32x4_t(&next)[NR], int rbuf, int rstep, auto request, auto share, int dbuf) {
            constexpr int Q0 = share.value * NQ / STEPS, Q1 = request.value ? (share.value + 1) * NQ / STEPS : Q0;
#pragma unroll
            for (int k = 0; k < NS; ++k) {
                // (the reads are back before the next step begins)
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    if (NS >= 2 * NR ? r == k : r >= 2 * k && (r < 2 * k + 2 || k == NS - 1)) read1(next, r, rbuf, rstep);
#pragma unroll
                for (int q = Q0 + k * (Q1 - Q0) / NS; q < Q0 + (k + 1) * (Q1 - Q0) / NS; ++q) dma1(q, dbuf);
                acc[k / BJ][k % BJ] = Op::mfma(cur[BI + k % BJ], cur[k / BJ], acc[k / BJ][k % BJ]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Stage s + NB - 1 is requested while stage s is multiplied, into the buffer of stage s - 1.  At the end of stage s (before its last
        // step, whose fragments are there) stage s + 1 has landed when nothing behind the requests since is outstanding.
        auto stage = [&](int buf, auto request) {
            const int next = buf + 1 == NB ? 0 : buf + 1, before = buf == 0 ? NB - 1 : buf - 1;
            if constexpr (request.value) dma_begin();
            step(f[0], f[1], buf, 1, request, std::integral_constant<int, 0>{}, before);
            if constexpr (STEPS == 4) {
                step(f[1], f[0], buf, 2, request, std::integral_constant<int, 1>{}, before);
                step(f[0], f[1], buf, 3, request, std::integral_constant<int, 2>{}, before);
            }
            if constexpr (request.value) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((NB - 3) * NQ + NQ * (STEPS - 1) / STEPS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" : : : "memory");
            step(f[1], f[0], next, 0, request, std::integral_constant<int, STEPS - 1>{}, before);       // (behind the last stage: reads of no use)
            if constexpr (request.value) dma_end();
            return next;
        };
        if (total > 0) {
#pragma unroll
            for (int b = 0; b < NB - 1; ++b)
                if (b < total) dma_stage(b);
            if (total >= NB - 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"((NB - 2) * NQ) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" : : : "memory");
#pragma unroll
            for (int r = 0; r < NR; ++r) read1(f[0], r, 0, 0);
        }
        int s = 0, buf = 0;
        for (; s < min(full, total - (NB - 1)); ++s) buf = stage(buf, std::true_type{});
        for (; s < full; ++s) buf = stage(buf, std::false_type{});
        if (Op::INT && rest) {          // the last stage is not whole: its steps one by one, zeros behind the end
            for (int st = 0; 32 * st < rest; ++st) {
                i32x4_t g[NR];
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    read1(g, r, buf, st);
                    if (32 * st + 16 * (lane >> 5) >= rest) g[r] = i32x4_t{0, 0, 0, 0};
                }
#pragma unroll
                for (int k = 0; k < NS; ++k) acc[k / BJ][k % BJ] = Op::mfma(g[BI + k % BJ], g[k / BJ], acc[k / BJ][k % BJ]);
            }
        }
    } else {
        // Three stages are on their way in registers.  Requests are made without a condition, so that they overlap: one behind a row's end
        // fetches the row's last 16 bytes, which are moved down (or out) when they go to LDS.
        i32x4_t reg[3][NQ];
        auto fetch = [&](i32x4_t(&to)[NQ], int s) {
            const int k = min(s * SB + piece16, Kb - 16);
#pragma unroll
            for (int q = 0; q < NQ; ++q) __builtin_memcpy(&to[q], (q < QA ? abase : bbase) + (voff[q] + (uint32_t)k), 16);
        };
        auto stash = [&](i32x4_t(&from)[NQ], int s) {
            if (s >= full) {
                const int down = s * SB + piece16 - (Kb - 16);
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    unsigned __int128 t;
                    __builtin_memcpy(&t, &from[q], 16);
                    t = down < 16 ? t >> (8 * max(down, 0)) : 0;
                    __builtin_memcpy(&from[q], &t, 16);
                }
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) *reinterpret_cast<i32x4_t *>(lds + (s & 1) * STAGE + place(q) + lane * 16) = from[q];
        };
        // (a stage's fragments are requested together: one LDS latency a stage instead of one a step)
        auto multiply = [&](int s) {
            i32x4_t g[STEPS][NR];
#pragma unroll
            for (int st = 0; st < STEPS; ++st)
#pragma unroll
                for (int r = 0; r < NR; ++r) read1(g[st], r, s & 1, st);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int st = 0; st < STEPS; ++st)
#pragma unroll
                for (int k = 0; k < NS; ++k) acc[k / BJ][k % BJ] = Op::mfma(g[st][BI + k % BJ], g[st][k / BJ], acc[k / BJ][k % BJ]);
        };
        // stage s, whose registers are free; `next` holds stage s + 1
        auto stage = [&](i32x4_t(&own)[NQ], i32x4_t(&next)[NQ], int s) {
            fetch(own, s + 3);
            multiply(s);
            stash(next, s + 1);
            __syncthreads();
        };
        if (Kb >= 16) {
            fetch(reg[0], 0);
            fetch(reg[1], 1);
            fetch(reg[2], 2);
            stash(reg[0], 0);
            __syncthreads();
            for (int s = 0; s < total; s += 3) {        // (stages behind the last are zeros)
                stage(reg[0], reg[1], s);
                if (s + 1 >= total) break;
                stage(reg[1], reg[2], s + 1);
                if (s + 2 >= total) break;
                stage(reg[2], reg[0], s + 2);
            }
        } else if (Kb > 0) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) *reinterpret_cast<i32x4_t *>(lds + place(q) + lane * 16) = row_piece((q < QA ? abase : bbase) + voff[q], piece16, Kb);
            __syncthreads();
            multiply(0);
            __syncthreads();
        }
    }

#pragma unroll
    for (int u = 0; u < SIDE; ++u)
        if (u * TILE_THREADS + (int)threadIdx.x < SIDE_N) side[u * TILE_THREADS + threadIdx.x] = side_v[u];
    __syncthreads();                        // (and every wave has read its last fragments)
    if constexpr (!Op::INT && !std::is_same_v<E, F32>) {
        if (p.parts) {
            tile_output<Op, F32, TM, TN, false, LDS_BYTES>(p, acc, lds, side, i0, j0, part);
            return;
        }
    }
    tile_output<Op, E, TM, TN, TANH, LDS_BYTES>(p, acc, lds, side, i0, j0, part);
}

}  // namespace adapt
