// What the gradients of the exact 8-bit product need beside the product itself (tile_product.hpp).
//
//     dx[m][k] = sum_n (dy[m][n] s_w[n]) w[n][k],      dw[n][k] = sum_m (dy[m][n] s_a[m]) a[m][k]
//
// Codes are bf16 numbers.  dy s is a sum of bf16 numbers, t = t0 + t1 (+ t2), each the rest of the one before it rounded to nearest: 16
// (24) bits.  So a gradient is one bf16 product with exact partial products and fp32 sums, over rows [t2 2^16 | t1 2^8 | t0] and
// [q 2^-16 | q 2^-8 | q]: the powers of two keep the small pieces of small gradients above the smallest number (unscaled, gradients below
// 2^-110 would lose bits), and the small pieces come first.  Both matrices are written to the workspace with the summed index last,
// rows in whole stages of 128 bytes.
#pragma once
#include "tile_product.hpp"

namespace adapt {

constexpr int GRAD_STAGE = 64;      // elements of a row that a product takes at a time: pieces are padded to a multiple of them

// piece z = 0 (the smallest) .. P - 1 of t
template <int P>
__device__ __forceinline__ void split_pieces(float t, __bf16 (&out)[P]) {
    out[P - 1] = (__bf16)t;
    const bool finite = fabsf((float)out[P - 1]) < __builtin_inff();        // (infinities and NaN: the first piece alone)
#pragma unroll
    for (int z = P - 2; z >= 0; --z) {
        t = (t - (float)out[z + 1]) * 256.0f;               // exact: the rest has no more bits than t
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
template <typename Load, typename Write>
__device__ __forceinline__ void grad_transpose(int R, int C, Load &&load, Write &&write) {
    __shared__ float tile[64][65];
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
    load(tile, r0, c0);
    __syncthreads();
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

// out[n][z][m] = piece z of dy[m][n] * s[m]
template <typename E, int P>
__global__ __launch_bounds__(256) void grad_split_columns_kernel(const typename E::mem *__restrict__ dy, const float *__restrict__ s, __bf16 *__restrict__ out,
                                                                 int M, int N, int Mp) {
    grad_transpose(
        M, N,
        [&](float(&tile)[64][65], int r0, int c0) {
            const int c = (threadIdx.x & 15) * 4;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = (threadIdx.x >> 4) + 16 * u, m = r0 + r, n = c0 + c;
                float t[4] = {};
                if (m < M) {
                    const typename E::mem *const at = dy + (size_t)m * (size_t)N + n;
                    if (n + 4 <= N) load_piece<E, 4>(at, t);
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (n + j < N) t[j] = E::load(at[j]);
                    const float sm = s[m];
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[j] *= sm;
                    if (n + 4 > N)          // (a scale of infinity times nothing)
#pragma unroll
                        for (int j = 0; j < 4; ++j) t[j] = n + j < N ? t[j] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) tile[r][c + j] = t[j];
            }
        },
        [&](int n, int m, const float(&t)[8]) {
            bf16x8_t v[P];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                __bf16 q[P];
                split_pieces<P>(t[j], q);
#pragma unroll
                for (int z = 0; z < P; ++z) v[z][j] = q[z];
            }
#pragma unroll
            for (int z = 0; z < P; ++z) *reinterpret_cast<bf16x8_t *>(out + ((size_t)n * P + z) * (size_t)Mp + m) = v[z];
        });
}

// out[c][z][r] = q[r][c] * 2^(-8 (P - 1 - z))
template <int P>
__global__ __launch_bounds__(256) void grad_codes_kernel(const int8_t *__restrict__ q, __bf16 *__restrict__ out, int R, int C, int Rp) {
    grad_transpose(
        R, C,
        [&](float(&tile)[64][65], int r0, int c0) {
            const int c = (threadIdx.x & 15) * 4;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int rl = (threadIdx.x >> 4) + 16 * u, r = r0 + rl;
#pragma unroll
                for (int j = 0; j < 4; ++j) tile[rl][c + j] = r < R && c0 + c + j < C ? (float)q[(size_t)r * (size_t)C + c0 + c + j] : 0.0f;
            }
        },
        [&](int c, int r, const float(&t)[8]) {
#pragma unroll
            for (int z = 0; z < P; ++z) {
                const float f = z == P - 1 ? 1.0f : (z == P - 2 ? 0x1p-8f : 0x1p-16f);
                bf16x8_t v;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (__bf16)(t[j] * f);
                *reinterpret_cast<bf16x8_t *>(out + ((size_t)c * P + z) * (size_t)Rp + r) = v;
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

// db[n] = sum_m dy[m][n]: a workgroup adds GRAD_DB_ROWS rows of 64 columns (four threads per column, every fourth row each) to part[block][n];
// grad_join_kernel adds those
constexpr int GRAD_DB_ROWS = 128;
template <typename E>
__global__ __launch_bounds__(256) void grad_bias_kernel(const typename E::mem *__restrict__ dy, float *__restrict__ part, int M, int N) {
    __shared__ float p[4][64];
    const int c = threadIdx.x & 63, ph = threadIdx.x >> 6, n = blockIdx.y * 64 + c, m0 = blockIdx.x * GRAD_DB_ROWS;
    float s = 0.0f;
    if (n < N) {
        const typename E::mem *const at = dy + (size_t)m0 * (size_t)N + n;
        if (m0 + GRAD_DB_ROWS <= M) {
#pragma unroll 8
            for (int r = ph; r < GRAD_DB_ROWS; r += 4) s += E::load(at[(size_t)r * (size_t)N]);
        } else {
            for (int r = ph; m0 + r < M; r += 4) s += E::load(at[(size_t)r * (size_t)N]);
        }
    }
    p[ph][c] = s;
    __syncthreads();
    if (ph == 0 && n < N) part[(size_t)blockIdx.x * N + n] = ((p[0][c] + p[1][c]) + p[2][c]) + p[3][c];
}

}  // namespace adapt
