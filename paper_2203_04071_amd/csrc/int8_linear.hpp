// Few tokens against many channels: the weights are read once, straight into the matrix instructions.
#pragma once
#include "tile_product.hpp"

namespace adapt {

struct Int8Params {
    const int8_t *a, *w;
    const float *s_a, *s_w, *bias;
    void *y;
    int M, K, N, act;
};

// Rows that do not start at multiples of four bytes: a 16-byte request at an odd address takes the memory pipe two to four times as long as one
// at a multiple of four (8 tokens, 16384 channels of 4095: 48 us; of 4092 16.5).  So the aligned 16 bytes and the word behind them are requested, and the
// bytes moved down when they are used (30 us; 48 x 3001 -> 4096 17.3 -> 12.4).  The last row (the word behind its end may lie outside the matrix), and every
// row of a matrix that itself is not aligned, is read as it lies.
template <bool SHIFT>
struct RowBytes {
    const char *row;            // of the first request
    uint32_t down, word;        // bytes to move, where the word behind is
    __device__ __forceinline__ void set(const char *base, size_t index, size_t last, size_t ld) {
        row = base + index * ld;
        down = SHIFT && index != last && (reinterpret_cast<uintptr_t>(base) & 3u) == 0 ? (uint32_t)(reinterpret_cast<uintptr_t>(row) & 3u) : 0u;
        word = down ? 16 : 0;
        row -= down;
    }
};
// bytes `down` .. `down` + 15 of the 20 in v, word
__device__ __forceinline__ i32x4_t bytes_down(i32x4_t v, uint32_t word, uint32_t down) {
    i32x4_t r;
    r[0] = (int)__builtin_amdgcn_alignbyte((uint32_t)v[1], (uint32_t)v[0], down);
    r[1] = (int)__builtin_amdgcn_alignbyte((uint32_t)v[2], (uint32_t)v[1], down);
    r[2] = (int)__builtin_amdgcn_alignbyte((uint32_t)v[3], (uint32_t)v[2], down);
    r[3] = (int)__builtin_amdgcn_alignbyte(word, (uint32_t)v[3], down);
    return r;
}

// 16 channels x 16 MT tokens per workgroup; its waves share the inner dimension in turns of 64 bytes, so that together they read 64 WAVES
// bytes of 16 rows of weights at a time, and add their sums through LDS (integers: any order).  An instruction takes 16 channels x 64
// bytes and 16 tokens x 64 bytes, 16 bytes a lane; register v of lane l holds channel 4 (l / 16) + v of token l % 16.
template <class E, int MT, int WAVES, bool SHIFT, bool TANH>
__global__ __launch_bounds__(64 * WAVES) void int8_tokens_kernel(const Int8Params p) {
    __shared__ i32x4_t part[WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = (int)blockIdx.x * 16, m0 = (int)blockIdx.y * (16 * MT);
    RowBytes<SHIFT> wr, ar[MT];
    wr.set(reinterpret_cast<const char *>(p.w), (size_t)min(n0 + (lane & 15), p.N - 1), (size_t)p.N - 1, (size_t)p.K);
#pragma unroll
    for (int t = 0; t < MT; ++t) ar[t].set(reinterpret_cast<const char *>(p.a), (size_t)min(m0 + 16 * t + (lane & 15), p.M - 1), (size_t)p.M - 1, (size_t)p.K);
    i32x4_t acc[MT] = {};
    int k = 64 * wave + 16 * (lane >> 4);
    constexpr int U = MT == 1 ? 8 : (MT == 2 ? 4 : 2);          // turns in flight
    auto turn = [&](const i32x4_t &w, const i32x4_t(&a)[MT]) {
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, a[t], acc[t], 0, 0, 0);
    };
    struct Bytes {
        i32x4_t v;
        uint32_t word;
    };
    auto request = [&](const RowBytes<SHIFT> &r, int at) {
        Bytes b;
        __builtin_memcpy(&b.v, r.row + at, 16);
        if constexpr (SHIFT) __builtin_memcpy(&b.word, r.row + at + r.word, 4);
        return b;
    };
    auto bytes = [&](const RowBytes<SHIFT> &r, const Bytes &b) { return SHIFT ? bytes_down(b.v, b.word, r.down) : b.v; };
    auto turns = [&](auto count) {
        constexpr int C = count.value;
        Bytes w[C], a[C][MT];
#pragma unroll
        for (int u = 0; u < C; ++u) w[u] = request(wr, k + u * 64 * WAVES);
#pragma unroll
        for (int u = 0; u < C; ++u)
#pragma unroll
            for (int t = 0; t < MT; ++t) a[u][t] = request(ar[t], k + u * 64 * WAVES);
#pragma unroll
        for (int u = 0; u < C; ++u) {
            i32x4_t at[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) at[t] = bytes(ar[t], a[u][t]);
            turn(bytes(wr, w[u]), at);
        }
    };
    // (k0: the same in the whole wave)
    int k0 = 64 * wave;
    for (; k0 + (U - 1) * 64 * WAVES + 64 <= p.K; k0 += U * 64 * WAVES, k += U * 64 * WAVES) turns(std::integral_constant<int, U>{});
    for (; k0 + 64 <= p.K; k0 += 64 * WAVES, k += 64 * WAVES) turns(std::integral_constant<int, 1>{});
    if (k0 < p.K) {
        const i32x4_t w = row_piece(wr.row + wr.down, k, p.K);
        i32x4_t a[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) a[t] = row_piece(ar[t].row + ar[t].down, k, p.K);
        turn(w, a);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave >= MT) return;
    const int t = wave, m = m0 + 16 * t + (lane & 15), n = n0 + 4 * (lane >> 4);
    if (m >= p.M || n >= p.N) return;
    i32x4_t s = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += part[w][t][lane];
    const float s_a = p.s_a[m], floor = int8_floor(p.act);
    typename E::mem *const y = static_cast<typename E::mem *>(p.y) + (size_t)m * (size_t)p.N + (size_t)n;
    float f[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int c = min(n + v, p.N - 1);
        f[v] = int8_finish<TANH>(s[v], s_a, p.s_w[c], p.bias ? p.bias[c] : 0.0f, floor, p.act);
    }
    if (n + 4 <= p.N) {
        store_piece<E, 4>(y, f);
    } else {
#pragma unroll
        for (int v = 0; v < 3; ++v)
            if (n + v < p.N) y[v] = E::store(f[v]);
    }
}

}  // namespace adapt
