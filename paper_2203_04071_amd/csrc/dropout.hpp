// Dropout whose mask is computed, not stored: element i is kept when word i % 4 of a Philox4x32-10 block is at least p 2^32.  The
// block's counter is (i / 4, offset + *step), its key the seed, so forward and backward, every launch shape and every element type
// see the same mask.
//
// The generator (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds on four words c and
// two key words k,   c' = (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)),   k' = k + (W0, W1).
#pragma once
#include "element.hpp"

namespace adapt {

constexpr int DROP_THREADS = 256;

struct DropoutParams {
    uint64_t seed, offset;
    const uint64_t *step;       // added to the offset; nullptr: nothing
    uint32_t threshold;         // dropped below it
    int none;                   // p = 1: nothing is kept (the threshold would be 2^32)
    float scale;                // 1 / (1 - p)
    size_t n;
};

__device__ __forceinline__ void philox_block(uint64_t block, uint64_t hi, uint64_t seed, uint32_t (&out)[4]) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)hi, c3 = (uint32_t)(hi >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c1, k0, 0x96);       // exclusive or of three
        c1 = (uint32_t)p1;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c3, k1, 0x96);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// A lane takes 16 bytes: one block of the generator for fp32, two for 16-bit types.  Bounded by memory, just: a block is twenty multiplications
// of a quarter of the vector rate and as many other instructions.  64 M bf16 elements take 41 us where half of them lie in the last-level cache, 49 us
// where none do (a copy of as many bytes: 52).
template <typename E>
__global__ __launch_bounds__(DROP_THREADS) void dropout_kernel(const typename E::mem *x, typename E::mem *y, const DropoutParams p) {
    constexpr int P = piece_len<E>;
    const size_t pieces = (p.n + P - 1) / P, stride = (size_t)gridDim.x * DROP_THREADS;
    const uint64_t hi = p.offset + (p.step ? *p.step : 0);
    for (size_t i = (size_t)blockIdx.x * DROP_THREADS + threadIdx.x; i < pieces; i += stride) {
        const size_t at = i * P;
        const bool whole = at + P <= p.n;
        float v[P];
        if (whole) {
            load_piece<E, P>(x + at, v);
        } else {
#pragma unroll
            for (int j = 0; j < P; ++j) v[j] = at + j < p.n ? E::load(x[at + j]) : 0.0f;
        }
        uint32_t r[P / 4][4];
#pragma unroll
        for (int b = 0; b < P / 4; ++b) philox_block(i * (P / 4) + b, hi, p.seed, r[b]);
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = !p.none && r[j / 4][j % 4] >= p.threshold ? v[j] * p.scale : 0.0f;
        if (whole) {
            store_piece<E, P>(y + at, v);
        } else {
#pragma unroll
            for (int j = 0; j < P - 1; ++j)
                if (at + j < p.n) y[at + j] = E::store(v[j]);
        }
    }
}

}  // namespace adapt
