// What the gradients of the exact 8-bit product need beside the product itself (tile_product.hpp).
//
//     dx[m][k] = sum_n (dy[m][n] s_w[n]) w[n][k],      dw[n][k] = sum_m (dy[m][n] s_a[m]) a[m][k]
//
// Both are c[i][j] = sum_r t[i][r] q[j][r] with codes q, which are fp16 numbers.  t = dy s becomes fp16 numbers as well: every row i is brought to
// a largest element in [2^14, 2^15) by a power of two, which goes back in on the sums, and is then the sum of two fp16 numbers, t = t0 + t1, t1 the
// rest that t0 leaves: 22 bits, 2^-22 of a term, where an fp32 sum rounds by 2^-24 of itself at every addition.  Elements below 2^-17 of their row's
// largest (2^-3 against 2^14) may keep fewer bits: t1 is then off by half the smallest fp16 number, 2^-25, at most 2^-39 of that largest.  So a gradient is an
// fp16 product with exact partial products and fp32 sums over rows [t1 | t0] that meet the same codes twice, the small pieces first.  (One piece of 11 bits is half the work, 288 us against 508 for 4096^3 bf16, but
// leaves a bf16 gradient none of its 8 bits where the terms of a sum cancel to 2^-12 of themselves.  Three bf16 pieces of 24 bits, without the rows'
// powers of two, took 148 us where this takes 116 for 6400 x 512 -> 2048 fp32.)
//
// Both matrices are written to the workspace with the summed index last, rows in whole stages of 128 bytes.
#pragma once
#include "tile_product.hpp"

namespace adapt {

constexpr int GRAD_STAGE = 64;      // elements of a row that a product takes at a time: pieces are padded to a multiple of them
constexpr int GRAD_THREADS = 256;

// exponent e of a row with largest element m: m 2^-e lies in [2^14, 2^15)
__device__ __forceinline__ int grad_exponent(float m) {
    if (!(m > 0.0f)) return 0;
    return (m < __builtin_inff() ? __builtin_amdgcn_frexp_expf(m) : 128) - 15;
}

// pieces 0 (the smaller) and 1 of eight t 2^-e; next: elements from a piece to the one behind
constexpr int GRAD_PIECES = 2;
__device__ __forceinline__ void store_pieces(const float (&t)[8], int e, _Float16 *out, size_t next) {
    f16x8_t v[GRAD_PIECES];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = __builtin_amdgcn_ldexpf(t[j], -e);
        v[1][j] = (_Float16)x;
        const float hi = (float)v[1][j];
        v[0][j] = fabsf(hi) < __builtin_inff() ? (_Float16)(x - hi) : (_Float16)0.0f;       // (x - hi is exact; infinities and NaN: the larger piece alone)
    }
    *reinterpret_cast<f16x8_t *>(out) = v[0];
    *reinterpret_cast<f16x8_t *>(out + next) = v[1];
}

// eight elements n .. n + 7 of a row of N, zeros beyond its end
template <typename E>
__device__ __forceinline__ void load_eight(const typename E::mem *__restrict__ row, int n, int N, float (&t)[8]) {
    if (n + 8 <= N) {
        load_piece<E, 8>(row + n, t);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = n + j < N ? E::load(row[n + j]) : 0.0f;
    }
}

// out[m][z][n] = piece z of dy[m][n] * s[n], exps[m]; zeros for N <= n < Np.  GROUP lanes share a row, NP times eight elements each, which stay in
// registers between the maximum and the pieces; a lane's columns are the same in every row, their scales are read once.
template <typename E, int GROUP, int NP>
__device__ __forceinline__ void grad_rows(const typename E::mem *__restrict__ dy, const float *__restrict__ s, _Float16 *__restrict__ out, int *__restrict__ exps,
                                          int M, int N, int Np, uint32_t block, uint32_t blocks, float *part) {
    constexpr int WAVES = GROUP / 64;
    const int lane = threadIdx.x % GROUP, stride = (int)blocks * (GRAD_THREADS / GROUP);
    float sc[NP][8];
#pragma unroll
    for (int u = 0; u < NP; ++u) load_eight<F32>(s, (u * GROUP + lane) * 8, N, sc[u]);
    for (int m = (int)block * (GRAD_THREADS / GROUP) + (int)threadIdx.x / GROUP; m < M; m += stride) {
        float t[NP][8], big = 0.0f;
#pragma unroll
        for (int u = 0; u < NP; ++u) load_eight<E>(dy + (size_t)m * (size_t)N, (u * GROUP + lane) * 8, N, t[u]);
#pragma unroll
        for (int u = 0; u < NP; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                t[u][j] = (u * GROUP + lane) * 8 + j < N ? t[u][j] * sc[u][j] : 0.0f;
                big = fmaxf(big, fabsf(t[u][j]));
            }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) big = fmaxf(big, __shfl_xor(big, off, 64));
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = big;
            __syncthreads();
            big = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
            __syncthreads();
        }
        const int e = grad_exponent(big);
        if (lane == 0) exps[m] = e;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const int n = (u * GROUP + lane) * 8;
            if (n < Np) store_pieces(t[u], e, out + (size_t)m * GRAD_PIECES * (size_t)Np + n, (size_t)Np);
        }
    }
}

// The same for rows too long for registers: read twice.
template <typename E>
__device__ __forceinline__ void grad_long_rows(const typename E::mem *__restrict__ dy, const float *__restrict__ s, _Float16 *__restrict__ out, int *__restrict__ exps,
                                               int M, int N, int Np, uint32_t block, uint32_t blocks, float *part) {
    for (int m = (int)block; m < M; m += (int)blocks) {
        float big = 0.0f;
        auto eight = [&](int n, float(&t)[8]) {
            float sc[8];
            load_eight<E>(dy + (size_t)m * (size_t)N, n, N, t);
            load_eight<F32>(s, n, N, sc);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = n + j < N ? t[j] * sc[j] : 0.0f;
        };
        for (int n = threadIdx.x * 8; n < N; n += GRAD_THREADS * 8) {
            float t[8];
            eight(n, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(t[j]));
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) big = fmaxf(big, __shfl_xor(big, off, 64));
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = big;
        __syncthreads();
        big = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        __syncthreads();
        const int e = grad_exponent(big);
        if (threadIdx.x == 0) exps[m] = e;
        for (int n = threadIdx.x * 8; n < Np; n += GRAD_THREADS * 8) {
            float t[8];
            eight(n, t);
            store_pieces(t, e, out + (size_t)m * GRAD_PIECES * (size_t)Np + n, (size_t)Np);
        }
    }
}

// Of 64 columns over `rows` rows (a multiple of GRAD_ROWS): sum[block][n] of dy (sum != nullptr), big[block][n] = max |dy s| (big != nullptr).  A
// thread takes 16 bytes of every 16th (32nd) row.  sums, bigs: [GRAD_THREADS P / 64][64]
constexpr int GRAD_ROWS = 256;
constexpr int GRAD_BLOCKS = 64;         // row blocks at most
template <typename E>
__device__ __forceinline__ void grad_columns(const typename E::mem *__restrict__ dy, const float *__restrict__ s, float *__restrict__ sum, float *__restrict__ big,
                                             int M, int N, int rows, uint32_t row_block, uint32_t column_block, float *sums, float *bigs) {
    constexpr int P = piece_len<E>, LANES = 64 / P, G = GRAD_THREADS / LANES;
    const int c = (threadIdx.x % LANES) * P, n = (int)column_block * 64 + c, g = threadIdx.x / LANES;
    float a[P] = {}, b[P] = {};
    const int first = (int)row_block * rows, last = min(M, first + rows);
    for (int m0 = first; m0 < last; m0 += 8 * G) {
        float t[8][P], sm[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int m = m0 + g + G * u;
            const typename E::mem *const at = dy + (size_t)m * (size_t)N + n;
            sm[u] = big && m < last ? s[m] : 0.0f;
            if (m < last && n + P <= N) {
                load_piece<E, P>(at, t[u]);
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) t[u][j] = m < last && n + j < N ? E::load(at[j]) : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                a[j] += t[u][j];
                b[j] = fmaxf(b[j], fabsf(t[u][j] * sm[u]));
            }
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
        sums[g * 64 + c + j] = a[j];
        bigs[g * 64 + c + j] = b[j];
    }
    __syncthreads();
    const int col = threadIdx.x, at = (int)column_block * 64 + col;
    if (col < 64 && at < N) {
        float x = sums[col], y = bigs[col];
#pragma unroll
        for (int w = 1; w < G; ++w) {
            x += sums[w * 64 + col];
            y = fmaxf(y, bigs[w * 64 + col]);
        }
        if (sum) sum[(size_t)row_block * (size_t)N + at] = x;
        if (big) big[(size_t)row_block * (size_t)N + at] = y;
    }
}

// The row blocks' results of 64 columns together: db[n] (sum != nullptr), and in exponents[64] (big != nullptr) the columns' exponents.  Four waves with
// every fourth block each.  scratch: [4][64]
template <typename E>
__device__ __forceinline__ void grad_columns_join(const float *__restrict__ sum, const float *__restrict__ big, typename E::mem *__restrict__ db, int blocks, int N,
                                                  uint32_t column_block, float (*sums)[64], float (*bigs)[64], int *exponents) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = (int)column_block * 64 + lane;
    float x = 0.0f, y = 0.0f;
    if (n < N) {
#pragma unroll 4
        for (int b = wave; b < blocks; b += 4) {
            if (sum) x += sum[(size_t)b * (size_t)N + n];
            if (big) y = fmaxf(y, big[(size_t)b * (size_t)N + n]);
        }
    }
    sums[wave][lane] = x;
    bigs[wave][lane] = y;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            x += sums[w][lane];
            y = fmaxf(y, bigs[w][lane]);
        }
        if (sum && n < N) db[n] = E::store(x);
        if (big) exponents[lane] = grad_exponent(y);
    }
    __syncthreads();
}
template <typename E>
__global__ __launch_bounds__(GRAD_THREADS) void grad_bias_kernel(const float *__restrict__ sum, typename E::mem *__restrict__ db, int blocks, int N) {
    __shared__ float sums[4][64], bigs[4][64];
    grad_columns_join<E>(sum, nullptr, db, blocks, N, blockIdx.x, sums, bigs, nullptr);
}

// 64 x 64 elements src[r][c] come out as out[c][..][r], padded with zeros to Rp rows: the transposed operands.  A workgroup holds the block in
// LDS as floats; lanes read along c and write along r, 16 bytes a lane.
constexpr int GRAD_LD = 65;
template <typename Write>
__device__ __forceinline__ void grad_transposed(const float (*tile)[GRAD_LD], int C, int r0, int c0, Write &&write) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int c = (threadIdx.x >> 3) + 32 * u, r = (threadIdx.x & 7) * 8;
        if (c0 + c >= C) continue;
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = tile[r + j][c];
        write(c0 + c, r0 + r, t);
    }
}

// out[n][z][m] = piece z of dy[m][n] * s[m] 2^-exps[n], the exponents from the row blocks' maxima; the first workgroup of 64 columns also writes
// exps and, if sum != nullptr, db
template <typename E>
__global__ __launch_bounds__(GRAD_THREADS) void grad_turned_rows_kernel(const typename E::mem *__restrict__ dy, const float *__restrict__ s, const float *__restrict__ sum,
                                                                        const float *__restrict__ big, typename E::mem *__restrict__ db, int *__restrict__ exps,
                                                                        _Float16 *__restrict__ out, int M, int N, int Mp, int blocks) {
    __shared__ float tile[64][GRAD_LD], sums[4][64], bigs[4][64];
    __shared__ int exponents[64];
    const int r0 = blockIdx.x * 64, c = (threadIdx.x & 15) * 4, c0 = blockIdx.y * 64, n = c0 + c;
    float t[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int m = r0 + (threadIdx.x >> 4) + 16 * u;
        const typename E::mem *const at = dy + (size_t)m * (size_t)N + n;
        if (m < M && n + 4 <= N) {
            load_piece<E, 4>(at, t[u]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) t[u][j] = m < M && n + j < N ? E::load(at[j]) : 0.0f;
        }
    }
    const bool first = blockIdx.x == 0;
    grad_columns_join<E>(first ? sum : nullptr, big, db, blocks, N, blockIdx.y, sums, bigs, exponents);
    if (first && threadIdx.x < 64 && c0 + (int)threadIdx.x < N) exps[c0 + threadIdx.x] = exponents[threadIdx.x];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int r = (threadIdx.x >> 4) + 16 * u, m = r0 + r;
        const float sm = m < M ? s[m] : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[r][c + j] = m < M && n + j < N ? t[u][j] * sm : 0.0f;
    }
    __syncthreads();
    grad_transposed(tile, N, r0, c0, [&](int col, int row, const float(&e)[8]) {
        store_pieces(e, exponents[col - c0], out + (size_t)col * GRAD_PIECES * (size_t)Mp + row, (size_t)Mp);
    });
}

// out[c][r] = q[r][c], a block of 64 x 64
__device__ __forceinline__ void grad_codes(const int8_t *__restrict__ q, _Float16 *__restrict__ out, int R, int C, int Rp, uint32_t row_block, uint32_t column_block,
                                           float (*tile)[GRAD_LD]) {
    const int r0 = (int)row_block * 64, c0 = (int)column_block * 64;
    const int rl = threadIdx.x >> 2, c = (threadIdx.x & 3) * 16, r = r0 + rl;
    i32x4_t v = {0, 0, 0, 0};
    if (r < R) {
        const int8_t *const at = q + (size_t)r * (size_t)C + c0 + c;
        if (c0 + c + 16 <= C) {
            __builtin_memcpy(&v, at, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 15; ++j)
                if (c0 + c + j < C) v[j / 4] |= (int)((uint32_t)(uint8_t)at[j] << (8 * (j % 4)));
        }
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) tile[rl][c + j] = (float)(int8_t)(v[j / 4] >> (8 * (j % 4)));
    __syncthreads();
    grad_transposed(tile, C, r0, c0, [&](int col, int row, const float(&t)[8]) {
        f16x8_t b;
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = (_Float16)t[j];
        *reinterpret_cast<f16x8_t *>(out + (size_t)col * (size_t)Rp + row) = b;
    });
}

// Everything that can be made from the operands at once, one launch: the workgroups are dealt out in four ranges, the rows of dy s_w, the codes w,
// the columns' sums and maxima, the codes a.  (A launch each: the whole gradient of 6990 x 227 -> 1706 bf16 takes 98 us instead of 89, that of 1000^3 42 instead of 31.)
struct GradPrep {
    const void *dy;
    const float *s_a, *s_w;
    const int8_t *a, *w;
    int M, K, N, Np, Mp, rows;
    _Float16 *dy_rows, *w_codes, *a_codes;
    int *row_exps;
    float *sum, *big;
    uint32_t row_groups, w_groups, column_groups, w_blocks, column_blocks, a_blocks;    // ranges, the first dimension of three of them
};
// GROUP 0: rows too long for registers
template <typename E, int GROUP, int NP>
__global__ __launch_bounds__(GRAD_THREADS) void grad_prepare_kernel(const GradPrep p) {
    __shared__ float lds[64 * GRAD_LD];
    static_assert(2 * GRAD_THREADS / (64 / piece_len<E>) * 64 <= 64 * GRAD_LD, "column statistics");
    const typename E::mem *const dy = static_cast<const typename E::mem *>(p.dy);
    uint32_t g = blockIdx.x;
    if (g < p.row_groups) {
        if constexpr (GROUP == 0) grad_long_rows<E>(dy, p.s_w, p.dy_rows, p.row_exps, p.M, p.N, p.Np, g, p.row_groups, lds);
        else grad_rows<E, GROUP, NP>(dy, p.s_w, p.dy_rows, p.row_exps, p.M, p.N, p.Np, g, p.row_groups, lds);
        return;
    }
    g -= p.row_groups;
    if (g < p.w_groups) {
        grad_codes(p.w, p.w_codes, p.N, p.K, p.Np, g % p.w_blocks, g / p.w_blocks, reinterpret_cast<float(*)[GRAD_LD]>(lds));
        return;
    }
    g -= p.w_groups;
    if (g < p.column_groups) {
        grad_columns<E>(dy, p.s_a, p.sum, p.big, p.M, p.N, p.rows, g % p.column_blocks, g / p.column_blocks, lds, lds + GRAD_THREADS / (64 / piece_len<E>) * 64);
        return;
    }
    g -= p.column_groups;
    grad_codes(p.a, p.a_codes, p.M, p.K, p.Mp, g % p.a_blocks, g / p.a_blocks, reinterpret_cast<float(*)[GRAD_LD]>(lds));
}

// c[i] = part[0][i] + part[1][i] + ... in that order, rounded to E
template <typename E>
__global__ __launch_bounds__(256) void grad_join_kernel(const float *__restrict__ part, int parts, size_t n, typename E::mem *__restrict__ c) {
    const size_t stride = (size_t)gridDim.x * 256 * 4;
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += stride) {
        if (i + 4 <= n) {
            float s[4], t[4];
            load_piece<F32, 4>(part + i, s);
#pragma unroll 8
            for (int z = 1; z < parts; ++z) {
                load_piece<F32, 4>(part + (size_t)z * n + i, t);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] += t[j];
            }
            store_piece<E, 4>(c + i, s);
        } else {
            for (size_t e = i; e < n; ++e) {
                float s = part[e];
                for (int z = 1; z < parts; ++z) s += part[(size_t)z * n + e];
                c[e] = E::store(s);
            }
        }
    }
}

}  // namespace adapt
