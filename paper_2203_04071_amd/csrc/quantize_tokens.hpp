// Activations to int8 codes with one scale for each row ("token"): the quantiser of Sec. III-A with the range taken from the row
// itself.  s = max |x| * (1 / Q), q = clamp(rint(x / s), -Q, Q), every step in fp32; a row of zeros has s = 0 and codes 0.
// (1 / Q rounded to fp32: within one unit in the last place of max |x| / Q.  Dividing a tensor by a number is this product in torch on the GPU, whose codes
// these are.)
#pragma once
#include "element.hpp"
#include "elementwise.hpp"

namespace adapt {

constexpr int QT_THREADS = 256;

// Codes of N elements of a row with scale s, inv = 1 / s.  rint(x / s) is decided by the product x inv, which is within 127 * 2^-22 < 4e-5 of the
// quotient: adding 1.5 * 2^23 rounds it to an integer (half to even) in the low bits of the sum.  Where the product lies that close to a
// half, or is NaN, the piece is done by IEEE division (`exact`: every piece, for scales whose reciprocal is no ordinary number).  An IEEE
// division is 12 instructions an element, this is 5.  With s within 2^-23 of max |x| / Q no quotient rounds beyond Q.
template <int N>
__device__ __forceinline__ void quantize_piece(const float (&x)[N], float s, float inv, float Q, bool exact, uint32_t (&codes)[N / 4]) {
    constexpr float MAGIC = 12582912.0f;
    bool near = exact;
    uint32_t b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float u = __builtin_fmaf(x[i], inv, MAGIC);
        const float d = __builtin_fmaf(x[i], inv, MAGIC - u);
        near |= !(fabsf(d) <= 0.4999f);
        b[i] = __float_as_uint(u);
    }
    if (near) {
#pragma unroll
        for (int i = 0; i < N; ++i) b[i] = s > 0.0f ? (uint32_t)quant1(x[i], s, Q) : 0u;
    }
#pragma unroll
    for (int w = 0; w < N / 4; ++w) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * w + 1], b[4 * w], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[4 * w + 3], b[4 * w + 2], 0x04000c0cu);
        codes[w] = lo | hi;
    }
}

// GROUP lanes per row (a wave, or the whole workgroup), each with up to NP pieces of 16 bytes that stay in registers between the maximum and
// the codes: x is read once.  Rows of any length and alignment: an element's own alignment is enough for the loads.  Bounded by memory.
template <typename E, int GROUP, int NP>
__global__ __launch_bounds__(QT_THREADS) void quantize_tokens_kernel(const typename E::mem *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scales,
                                                                     size_t rows, uint32_t cols, float Q) {
    constexpr int P = piece_len<E>, WAVES = GROUP / 64;
    __shared__ float part[QT_THREADS / 64];
    const uint32_t lane = threadIdx.x % GROUP;
    const size_t stride = (size_t)gridDim.x * (QT_THREADS / GROUP);
    for (size_t r = (size_t)blockIdx.x * (QT_THREADS / GROUP) + threadIdx.x / GROUP; r < rows; r += stride) {
        const typename E::mem *const row = x + r * cols;
        float v[NP][P];
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const uint32_t c = (u * GROUP + lane) * P;
            if (c + P <= cols) {
                load_piece<E, P>(row + c, v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) v[u][i] = c + i < cols ? E::load(row[c + i]) : 0.0f;
            }
        }
        float m = 0.0f;
#pragma unroll
        for (int u = 0; u < NP; ++u)
#pragma unroll
            for (int i = 0; i < P; ++i) m = fmaxf(m, fabsf(v[u][i]));         // (a maximum with NaN is the other number)
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
            __syncthreads();
            m = part[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, part[w]);
            __syncthreads();
        }
        const float s = m * (1.0f / Q), inv = 1.0f / s;
        const bool exact = !(s > 1.0e-30f && s < 1.0e30f);
        if (lane == 0) scales[r] = s;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const uint32_t c = (u * GROUP + lane) * P;
            if (c >= cols) continue;
            uint32_t codes[P / 4];
            quantize_piece<P>(v[u], s, inv, Q, exact, codes);
            int8_t *const to = q + r * cols + c;
            if (c + P <= cols) {
                __builtin_memcpy(to, codes, P);
            } else {
#pragma unroll
                for (int i = 0; i < P - 1; ++i)
                    if (c + i < cols) to[i] = (int8_t)(codes[i / 4] >> (8 * (i % 4)));
            }
        }
    }
}

// Rows too long for registers: the workgroup reads them twice (the second time mostly from cache).
template <typename E>
__global__ __launch_bounds__(QT_THREADS) void quantize_long_tokens_kernel(const typename E::mem *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scales,
                                                                          size_t rows, size_t cols, float Q) {
    constexpr int P = piece_len<E>;
    __shared__ float part[QT_THREADS / 64];
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const typename E::mem *const row = x + r * cols;
        const size_t whole = cols / P * P;
        float m = 0.0f;
        for (size_t c = (size_t)threadIdx.x * P; c < whole; c += QT_THREADS * P) {
            float v[P];
            load_piece<E, P>(row + c, v);
#pragma unroll
            for (int i = 0; i < P; ++i) m = fmaxf(m, fabsf(v[i]));
        }
        for (size_t c = whole + threadIdx.x; c < cols; c += QT_THREADS) m = fmaxf(m, fabsf(E::load(row[c])));
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
        m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        __syncthreads();
        const float s = m * (1.0f / Q), inv = 1.0f / s;
        const bool exact = !(s > 1.0e-30f && s < 1.0e30f);
        if (threadIdx.x == 0) scales[r] = s;
        for (size_t c = (size_t)threadIdx.x * P; c < whole; c += QT_THREADS * P) {
            float v[P];
            uint32_t codes[P / 4];
            load_piece<E, P>(row + c, v);
            quantize_piece<P>(v, s, inv, Q, exact, codes);
            __builtin_memcpy(q + r * cols + c, codes, P);
        }
        for (size_t c = whole + threadIdx.x; c < cols; c += QT_THREADS) q[r * cols + c] = s > 0.0f ? (int8_t)quant1(E::load(row[c]), s, Q) : (int8_t)0;
    }
}

}  // namespace adapt
