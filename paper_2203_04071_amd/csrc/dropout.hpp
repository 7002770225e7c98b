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
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

template <typename E>
__global__ __launch_bounds__(DROP_THREADS) void dropout_kernel(const typename E::mem *x, typename E::mem *y, const DropoutParams p) {
    const size_t blocks = (p.n + 3) / 4, stride = (size_t)gridDim.x * DROP_THREADS;
    const uint64_t hi = p.offset + (p.step ? *p.step : 0);
    for (size_t b = (size_t)blockIdx.x * DROP_THREADS + threadIdx.x; b < blocks; b += stride) {
        uint32_t r[4];
        philox_block(b, hi, p.seed, r);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (b * 4 + j < p.n) y[b * 4 + j] = E::store(!p.none && r[j] >= p.threshold ? E::load(x[b * 4 + j]) * p.scale : 0.0f);
    }
}

}  // namespace adapt
