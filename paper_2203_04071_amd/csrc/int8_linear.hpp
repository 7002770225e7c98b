// The exact product of int8 codes with a scale for each row of both operands, and its gradients.
#pragma once
#include "element.hpp"
#include "elementwise.hpp"

namespace adapt {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

// y[m][n] = act(float(sum_k a[m][k] w[n][k]) * s_a[m] * s_w[n] + bias[n]), rounded to E
struct Int8Params {
    const int8_t *a, *w;
    const float *s_a, *s_w, *bias;
    void *y;
    int M, K, N, act;
};

__device__ __forceinline__ float int8_finish(int acc, float s_a, float s_w, float bias, bool has_bias, int act) {
    float y = ((float)acc * s_a) * s_w;
    if (has_bias) y = y + bias;
    if (act == 1) y = y > 0.0f ? y : 0.0f;
    else if (act == 2) y = tanh_spec(y);
    return y;
}

// 16 codes k .. k + 15 of a row of K, zeros beyond its end; nothing outside the row is read
__device__ __forceinline__ i32x4_t int8_row_piece(const int8_t *__restrict__ row, int k, int K) {
    i32x4_t v = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K) {
        if (K >= 16) {                      // the last 16 of the row, moved down
            unsigned __int128 t;
            __builtin_memcpy(&t, row + K - 16, 16);
            t >>= 8 * (k + 16 - K);
            __builtin_memcpy(&v, &t, 16);
        } else {
            unsigned __int128 t = 0;
            for (int i = K - 1; i >= k; --i) t = t << 8 | (uint8_t)row[i];
            __builtin_memcpy(&v, &t, 16);
        }
    }
    return v;
}

// a wave computes 32 x 32 outputs, its operands come straight from memory; four waves share a tile of 64 x 64
template <typename E>
__global__ __launch_bounds__(256) void int8_linear_kernel(const Int8Params p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tiles_n = (p.N + 63) / 64;
    const int m0 = (int)(blockIdx.x / tiles_n) * 64 + (wave & 1) * 32, n0 = (int)(blockIdx.x % tiles_n) * 64 + (wave >> 1) * 32;
    if (m0 >= p.M || n0 >= p.N) return;
    const int8_t *const ar = p.a + (size_t)min(m0 + (lane & 31), p.M - 1) * (size_t)p.K;
    const int8_t *const wr = p.w + (size_t)min(n0 + (lane & 31), p.N - 1) * (size_t)p.K;
    i32x16_t acc = {};
    for (int k = 0; k < p.K; k += 32)
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(int8_row_piece(ar, k + 16 * (lane >> 5), p.K), int8_row_piece(wr, k + 16 * (lane >> 5), p.K), acc, 0, 0, 0);
    // register v of lane l holds row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32
    const int n = n0 + (lane & 31);
    if (n >= p.N) return;
    const float s_w = p.s_w[n], bias = p.bias ? p.bias[n] : 0.0f;
    typename E::mem *const y = static_cast<typename E::mem *>(p.y);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int m = m0 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
        if (m < p.M) y[(size_t)m * (size_t)p.N + (size_t)n] = E::store(int8_finish(acc[v], p.s_a[m], s_w, bias, p.bias != nullptr, p.act));
    }
}

// c[i][j] = sum_r (a[i sa_i + r sa_r] * s[r]) * q[r][j]: both gradients (a = dy), 32 x 32 outputs per workgroup
template <typename E>
__global__ __launch_bounds__(256) void int8_gradient_kernel(const typename E::mem *__restrict__ a, size_t sa_i, size_t sa_r, const float *__restrict__ s,
                                                            const int8_t *__restrict__ q, typename E::mem *__restrict__ c, int I, int J, int R) {
    __shared__ float As[32][33], Bs[32][33];
    const int tiles_j = (J + 31) / 32;
    const int i0 = (int)(blockIdx.x / tiles_j) * 32, j0 = (int)(blockIdx.x % tiles_j) * 32;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    float acc[4] = {};
    for (int r0 = 0; r0 < R; r0 += 32) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + tx, i = i0 + ty + 8 * u;
            As[ty + 8 * u][tx] = r < R && i < I ? E::load(a[(size_t)i * sa_i + (size_t)r * sa_r]) * s[r] : 0.0f;
            const int rb = r0 + ty + 8 * u, j = j0 + tx;
            Bs[ty + 8 * u][tx] = rb < R && j < J ? (float)q[(size_t)rb * (size_t)J + (size_t)j] : 0.0f;
        }
        __syncthreads();
#pragma unroll 8
        for (int r = 0; r < 32; ++r)
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[u] = __builtin_fmaf(As[ty + 8 * u][r], Bs[r][tx], acc[u]);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = i0 + ty + 8 * u, j = j0 + tx;
        if (i < I && j < J) c[(size_t)i * (size_t)J + (size_t)j] = E::store(acc[u]);
    }
}

// db[n] = sum_m dy[m][n]: 32 columns per workgroup, 8 threads per column
template <typename E>
__global__ __launch_bounds__(256) void int8_bias_grad_kernel(const typename E::mem *__restrict__ dy, typename E::mem *__restrict__ db, int M, int N) {
    __shared__ float part[8][33];
    const int c = threadIdx.x & 31, ph = threadIdx.x >> 5, n = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (n < N)
        for (int m = ph; m < M; m += 8) s += E::load(dy[(size_t)m * (size_t)N + (size_t)n]);
    part[ph][c] = s;
    __syncthreads();
    if (ph == 0 && n < N) {
#pragma unroll
        for (int u = 1; u < 8; ++u) s += part[u][c];
        db[n] = E::store(s);
    }
}

}  // namespace adapt
