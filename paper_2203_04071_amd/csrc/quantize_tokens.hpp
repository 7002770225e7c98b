// Activations to int8 codes with one scale for each row ("token"): the quantiser of Sec. III-A with the range taken from the row
// itself.  s = max |x| / Q, q = clamp(rint(x / s), -Q, Q), every step in fp32; a row of zeros has s = 0 and codes 0.
#pragma once
#include "element.hpp"
#include "elementwise.hpp"

namespace adapt {

constexpr int QT_THREADS = 256;

// max over the workgroup; `part` holds one value per wave
template <int THREADS>
__device__ __forceinline__ float workgroup_max(float m, float *part) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(m, off, 64);
        if (o > m) m = o;
    }
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w)
        if (part[w] > m) m = part[w];
    __syncthreads();
    return m;
}

// one workgroup per row, the row read twice
template <typename E>
__global__ __launch_bounds__(QT_THREADS) void quantize_tokens_kernel(const typename E::mem *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scales,
                                                                     size_t rows, size_t cols, float Q) {
    __shared__ float part[QT_THREADS / 64];
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const typename E::mem *const row = x + r * cols;
        float m = 0.0f;
        for (size_t c = threadIdx.x; c < cols; c += QT_THREADS) {
            const float a = fabsf(E::load(row[c]));
            if (a > m) m = a;               // NaN compares false and is skipped
        }
        m = workgroup_max<QT_THREADS>(m, part);
        const float s = m / Q;
        if (threadIdx.x == 0) scales[r] = s;
        for (size_t c = threadIdx.x; c < cols; c += QT_THREADS) q[r * cols + c] = s > 0.0f ? (int8_t)quant1(E::load(row[c]), s, Q) : (int8_t)0;
    }
}

}  // namespace adapt
