// What the gradients of the exact 8-bit product need beside the product itself (tile_product.hpp).
//
//     dx[m][k] = sum_n (dy[m][n] s_w[n]) w[n][k],      dw[n][k] = sum_m (dy[m][n] s_a[m]) a[m][k]
//
// Codes are bf16 numbers.  dy s is a sum of bf16 numbers, t = t0 + t1 (+ t2), each the rest of the one before it rounded to nearest: 16
// (24) bits.  So a gradient is one bf16 product with exact partial products and fp32 sums, over rows [t1 | t0] that meet the same codes q twice,
// or, where 24 bits are kept, rows [t2 2^16 | t1 2^8 | t0] and [q 2^-16 | q 2^-8 | q]: the powers of two keep the small pieces of small
// gradients above the smallest number (unscaled, fp32 gradients below 2^-110 would lose bits; of a 16-bit type only those below 2^-117 that its results
// do not show).  The small pieces come first.  The matrices are written to the workspace with the summed index last, rows in whole
// stages of 128 bytes.
#pragma once
#include "tile_product.hpp"

namespace adapt {

constexpr int GRAD_STAGE = 64;      // elements of a row that a product takes at a time: pieces are padded to a multiple of them

// numbers a code is written as, P pieces to be met
template <int P>
constexpr int code_copies = P == 3 ? 3 : 1;

// piece z = 0 (the smallest) .. P - 1 of t
template <int P>
__device__ __forceinline__ void split_pieces(float t, __bf16 (&out)[P]) {
    out[P - 1] = (__bf16)t;
    const bool finite = fabsf((float)out[P - 1]) < __builtin_inff();        // (infinities and NaN: the first piece alone)
#pragma unroll
    for (int z = P - 2; z >= 0; --z) {
        t = (t - (float)out[z + 1]) * (P == 3 ? 256.0f : 1.0f);        // exact: the rest has no more bits than t
        if (!finite) t = 0.0f;
        out[z] = (__bf16)t;
    }
}

// out[m][z][n] = piece z of dy[m][n] * s[n], zeros for N <= n < Np; eight elements per thread
template <typename E, int P>
__global__ __launch_bounds__(256) void grad_split_rows_kernel(const typename E::mem *__restrict__ dy, const float *__restrict__ s, __bf16 *__restrict__ out, int M,
                                                              int N, int Np) {
    const int per_row = Np / 8;
    const size_t total = (size_t)M * per_row, stride = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += stride) {
        const size_t m = i / per_row;
        const int n = (int)(i - m * per_row) * 8;
        float t[8];
        const typename E::mem *const row = dy + m * (size_t)N;
        if (n + 8 <= N) {
            load_piece<E, 8>(row + n, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] *= s[n + j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = n + j < N ? E::load(row[n + j]) * s[n + j] : 0.0f;
        }
        bf16x8_t v[P];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            __bf16 q[P];
            split_pieces<P>(t[j], q);
#pragma unroll
            for (int z = 0; z < P; ++z) v[z][j] = q[z];
        }
#pragma unroll
        for (int z = 0; z < P; ++z) *reinterpret_cast<bf16x8_t *>(out + (m * P + z) * (size_t)Np + n) = v[z];
    }
}

// 64 x 64 elements src[r][c] come out as out[c][z][r], padded with zeros to Rp rows: the transposed operands.  A workgroup holds the block in
// LDS as floats; lanes read along c and write along r, 16 bytes a lane.
constexpr int GRAD_LD = 65;
template <typename Write>
__device__ __forceinline__ void grad_transposed(const float (&tile)[64][GRAD_LD], int C, Write &&write) {
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
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

// out[n][z][m] = piece z of dy[m][n] * s[m] (PIECES), and on the way part[block][n] = sum of dy[m][n] over the block's 64 rows (part != nullptr).
// Without PIECES the sums alone, the same ones.
template <typename E, int P, bool PIECES>
__global__ __launch_bounds__(256) void grad_split_columns_kernel(const typename E::mem *__restrict__ dy, const float *__restrict__ s, __bf16 *__restrict__ out,
                                                                 float *__restrict__ part, int M, int N, int Mp) {
    __shared__ float tile[64][GRAD_LD];
    __shared__ float column[16][64];
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, c = (threadIdx.x & 15) * 4, n = c0 + c;
    float t[4][4], sum[4] = {};
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
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int r = (threadIdx.x >> 4) + 16 * u, m = r0 + r;
        const float sm = PIECES && m < M ? s[m] : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum[j] += t[u][j];
            if constexpr (PIECES) tile[r][c + j] = m < M && n + j < N ? t[u][j] * sm : 0.0f;
        }
    }
    if (part)
#pragma unroll
        for (int j = 0; j < 4; ++j) column[threadIdx.x >> 4][c + j] = sum[j];
    __syncthreads();
    if constexpr (PIECES)
        grad_transposed(tile, N, [&](int col, int row, const float(&e)[8]) {
            bf16x8_t v[P];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                __bf16 q[P];
                split_pieces<P>(e[j], q);
#pragma unroll
                for (int z = 0; z < P; ++z) v[z][j] = q[z];
            }
#pragma unroll
            for (int z = 0; z < P; ++z) *reinterpret_cast<bf16x8_t *>(out + ((size_t)col * P + z) * (size_t)Mp + row) = v[z];
        });
    if (part && threadIdx.x < 64 && c0 + (int)threadIdx.x < N) {
        float total = column[0][threadIdx.x];
#pragma unroll
        for (int g = 1; g < 16; ++g) total += column[g][threadIdx.x];
        part[(size_t)blockIdx.x * (size_t)N + c0 + threadIdx.x] = total;
    }
}

// db[n] = the sum of the blocks' sums: 64 columns per workgroup, sixteen waves with every sixteenth block each
template <typename E>
__global__ __launch_bounds__(1024) void grad_bias_kernel(const float *__restrict__ part, typename E::mem *__restrict__ db, int blocks, int N) {
    __shared__ float sum[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (n < N) {
#pragma unroll 8
        for (int b = wave; b < blocks; b += 16) s += part[(size_t)b * (size_t)N + n];
    }
    sum[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && n < N) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += sum[w][lane];
        db[n] = E::store(s);
    }
}

// out[c][z][r] = q[r][c] * 2^(-8 (copies - 1 - z))
template <int P>
__global__ __launch_bounds__(256) void grad_codes_kernel(const int8_t *__restrict__ q, __bf16 *__restrict__ out, int R, int C, int Rp) {
    constexpr int Z = code_copies<P>;
    __shared__ float tile[64][GRAD_LD];
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
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
    grad_transposed(tile, C, [&](int col, int row, const float(&t)[8]) {
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            const float f = z == Z - 1 ? 1.0f : (z == Z - 2 ? 0x1p-8f : 0x1p-16f);
            bf16x8_t b;
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = (__bf16)(t[j] * f);
            *reinterpret_cast<bf16x8_t *>(out + ((size_t)col * Z + z) * (size_t)Rp + row) = b;
        }
    });
}

// c[i] = part[0][i] + part[1][i] + ... in that order, rounded to E
template <typename E>
__global__ __launch_bounds__(256) void grad_join_kernel(const float *__restrict__ part, int parts, size_t n, typename E::mem *__restrict__ c) {
    const size_t stride = (size_t)gridDim.x * 256 * 4;
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += stride) {
        if (i + 4 <= n) {
            float s[4], t[4];
            load_piece<F32, 4>(part + i, s);
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
