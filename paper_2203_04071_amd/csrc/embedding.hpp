// Embedding lookup with scaling, y[t] = scale * table[tok[t]], and the gradient of the table by sorted tokens,
// dtable[v] = scale * sum over the places t with tok[t] = v of dy[t] (t ascending, fp32).
#pragma once
#include "element.hpp"

namespace adapt {

constexpr int EMB_THREADS = 256;

// a token as a row of the table; V for one that names no row
template <typename Tok>
__device__ __forceinline__ uint32_t embed_row(Tok t, uint32_t V) {
    return t >= 0 && (uint64_t)t < (uint64_t)V ? (uint32_t)t : V;
}

// 2^lg lanes share a row, in pieces of 16 bytes
template <typename E, typename Tok>
__global__ __launch_bounds__(EMB_THREADS) void embedding_kernel(const typename E::mem *__restrict__ table, const Tok *__restrict__ tokens,
                                                                typename E::mem *__restrict__ y, size_t T, uint32_t V, uint32_t D, float scale, int lg) {
    constexpr int P = piece_len<E>;
    const uint32_t lane = threadIdx.x & ((1u << lg) - 1);
    const size_t rows = (size_t)gridDim.x * (EMB_THREADS >> lg);
    for (size_t t = (size_t)blockIdx.x * (EMB_THREADS >> lg) + (threadIdx.x >> lg); t < T; t += rows) {
        const uint32_t v = embed_row(tokens[t], V);
        const typename E::mem *const from = table + (size_t)(v < V ? v : 0) * D;
        typename E::mem *const to = y + t * D;
        for (uint32_t c = lane * P; c < D; c += P << lg) {
            if (c + P <= D) {
                float f[P];
                if (v < V) load_piece<E, P>(from + c, f);
#pragma unroll
                for (int i = 0; i < P; ++i) f[i] = v < V ? f[i] * scale : 0.0f;
                store_piece<E, P>(to + c, f);
            } else {
                for (uint32_t i = c; i < D; ++i) to[i] = E::store(v < V ? E::load(from[i]) * scale : 0.0f);
            }
        }
    }
}

// ---- the gradient: places sorted by token (stable), sums of runs of equal tokens
//
// Least significant digit first, EMB_BITS bits a pass; a workgroup owns EMB_TILE places: count digits, scan the counts, scatter.
constexpr int EMB_BITS = 9;
constexpr int EMB_TILE = 2048;
constexpr int EMB_WAVES = EMB_THREADS / 64;

struct EmbedSort {
    const uint32_t *key_in, *at_in;     // nullptr in the first pass: keys come from the tokens, places are 0, 1, 2 ...
    uint32_t *key_out, *at_out;
    uint32_t *counts;                   // [digit][workgroup]
    uint8_t *used;                      // [V], set in the first pass
    uint32_t T, V;
    int shift, bits;
    int64_t padding;                    // token without a gradient
};

template <typename Tok>
__device__ __forceinline__ uint32_t embed_key(const EmbedSort &p, const Tok *__restrict__ tokens, uint32_t i) {
    if (p.key_in) return p.key_in[i];
    const Tok t = tokens[i];
    return (int64_t)t == p.padding ? p.V : embed_row(t, p.V);
}

// lanes of the wave that hold the same digit (all bits of it), among the active ones
__device__ __forceinline__ uint64_t embed_peers(uint32_t digit, int bits, bool active) {
    uint64_t m = __ballot(active);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        m &= (digit >> b) & 1 ? set : ~set;
    }
    return m;
}

// [wave][digit] counts of this workgroup's places; a wave owns a contiguous quarter of them
template <typename Tok>
__device__ __forceinline__ void embed_count(const EmbedSort &p, const Tok *__restrict__ tokens, uint32_t (*hist)[1 << EMB_BITS], bool mark) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < EMB_WAVES << EMB_BITS; i += EMB_THREADS) hist[i >> EMB_BITS][i & ((1 << EMB_BITS) - 1)] = 0;
    __syncthreads();
    const uint32_t from = blockIdx.x * EMB_TILE + wave * (EMB_TILE / EMB_WAVES);
    for (int u = 0; u < EMB_TILE / EMB_WAVES; u += 64) {
        const uint32_t i = from + u + lane;
        if (i < p.T) {
            const uint32_t key = embed_key(p, tokens, i);
            if (mark && key < p.V) p.used[key] = 1;
            atomicAdd(&hist[wave][(key >> p.shift) & ((1u << p.bits) - 1)], 1u);
        }
    }
    __syncthreads();
}

template <typename Tok>
__global__ __launch_bounds__(EMB_THREADS) void embed_count_kernel(const EmbedSort p, const Tok *__restrict__ tokens) {
    __shared__ uint32_t hist[EMB_WAVES][1 << EMB_BITS];
    embed_count(p, tokens, hist, p.key_in == nullptr);
    for (int d = threadIdx.x; d < 1 << p.bits; d += EMB_THREADS) {
        uint32_t s = 0;
#pragma unroll
        for (int w = 0; w < EMB_WAVES; ++w) s += hist[w][d];
        p.counts[(size_t)d * gridDim.x + blockIdx.x] = s;
    }
}

// exclusive sums of n counts in place; one workgroup
__global__ __launch_bounds__(1024) void embed_scan_kernel(uint32_t *__restrict__ counts, uint32_t n) {
    __shared__ uint32_t wave_sum[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (uint32_t base = 0; base < n; base += 1024) {
        const uint32_t i = base + threadIdx.x;
        const uint32_t own = i < n ? counts[i] : 0u;
        uint32_t incl = own;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = __shfl_up(incl, off, 64);
            if (lane >= off) incl += o;
        }
        if (lane == 63) wave_sum[wave] = incl;
        __syncthreads();
        uint32_t pre = before, total = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) pre += wave_sum[w];
            total += wave_sum[w];
        }
        if (i < n) counts[i] = pre + incl - own;
        before += total;
        __syncthreads();
    }
}

template <typename Tok>
__global__ __launch_bounds__(EMB_THREADS) void embed_scatter_kernel(const EmbedSort p, const Tok *__restrict__ tokens) {
    __shared__ uint32_t hist[EMB_WAVES][1 << EMB_BITS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    embed_count(p, tokens, hist, false);
    for (int d = threadIdx.x; d < 1 << p.bits; d += EMB_THREADS) {        // counts become the wave's next free place
        uint32_t at = p.counts[(size_t)d * gridDim.x + blockIdx.x];
#pragma unroll
        for (int w = 0; w < EMB_WAVES; ++w) {
            const uint32_t c = hist[w][d];
            hist[w][d] = at;
            at += c;
        }
    }
    __syncthreads();
    const uint32_t from = blockIdx.x * EMB_TILE + wave * (EMB_TILE / EMB_WAVES);
    for (int u = 0; u < EMB_TILE / EMB_WAVES; u += 64) {
        const uint32_t i = from + u + lane;
        const bool in = i < p.T;
        const uint32_t key = in ? embed_key(p, tokens, i) : 0u;
        const uint32_t digit = (key >> p.shift) & ((1u << p.bits) - 1);
        const uint64_t peers = embed_peers(digit, p.bits, in);
        const uint32_t rank = __popcll(peers & ((1ull << lane) - 1));
        // (the lanes of a wave run together and its LDS requests are carried out in order: every peer has read the place before the
        // first of them moves it on)
        const uint32_t to = in ? __hip_atomic_load(&hist[wave][digit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT) + rank : 0u;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (in && rank == 0) __hip_atomic_store(&hist[wave][digit], to + (uint32_t)__popcll(peers), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (in) {
            p.key_out[to] = key;
            p.at_out[to] = p.at_in ? p.at_in[i] : i;
        }
    }
}

// Sums.  The sorted places are cut into pieces of C, each summed by 2^lg lanes; a run of equal tokens inside a piece is finished there.
// One that crosses pieces leaves a partial sum in every piece: `head` for the part at a piece's start that began earlier, `tail` for
// the part at its end that goes on; embed_join_kernel adds them in order.
struct EmbedSum {
    const uint32_t *key, *at;
    const uint8_t *used;
    float *head, *tail;                 // [pieces][D]
    uint32_t T, V, D, C, pieces;
    float scale;
    int lg;
    uint32_t sum_blocks;                // workgroups beyond these write the rows without a token
};

template <typename E>
__global__ __launch_bounds__(EMB_THREADS) void embed_sum_kernel(const EmbedSum p, const typename E::mem *__restrict__ dy, typename E::mem *__restrict__ dtable) {
    constexpr int P = piece_len<E>;
    const uint32_t lane = threadIdx.x & ((1u << p.lg) - 1), per = EMB_THREADS >> p.lg;
    if (blockIdx.x >= p.sum_blocks) {
        const uint32_t rows = (gridDim.x - p.sum_blocks) * per;
        for (size_t v = (size_t)(blockIdx.x - p.sum_blocks) * per + (threadIdx.x >> p.lg); v < p.V; v += rows) {
            if (p.used[v]) continue;
            for (uint32_t c = lane; c < p.D; c += 1u << p.lg) dtable[v * p.D + c] = E::store(0.0f);
        }
        return;
    }
    const uint32_t piece = blockIdx.x * per + (threadIdx.x >> p.lg);
    if (piece >= p.pieces) return;
    const uint32_t first = piece * p.C, last = min(first + p.C, p.T);       // (pieces cover T: first < T)
    for (uint32_t c = lane * P; c < p.D; c += (uint32_t)P << p.lg) {
        const int len = (int)min((uint32_t)P, p.D - c);
        float acc[P] = {};
        uint32_t key = p.key[first];
        bool open = first > 0 && p.key[first - 1] == key;       // the run began in an earlier piece
        for (uint32_t i = first; i < last; ++i) {
            if (key >= p.V) break;                              // (places without a gradient come last)
            const typename E::mem *const from = dy + (size_t)p.at[i] * p.D + c;
            if (len == P) {
                float f[P];
                load_piece<E, P>(from, f);
#pragma unroll
                for (int j = 0; j < P; ++j) acc[j] += f[j];
            } else {
                for (int j = 0; j < len; ++j) acc[j] += E::load(from[j]);
            }
            const uint32_t next = i + 1 < p.T ? p.key[i + 1] : ~0u;
            if (next == key && i + 1 < last) continue;
            // the run ends, or the piece does
            if (open || next == key) {
                float *const part = (open ? p.head : p.tail) + (size_t)piece * p.D + c;
                for (int j = 0; j < len; ++j) part[j] = acc[j];
            } else {
                for (int j = 0; j < len; ++j) dtable[(size_t)key * p.D + c + j] = E::store(acc[j] * p.scale);
            }
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] = 0.0f;
            open = false;
            key = next;
        }
    }
}

// one workgroup per piece; it works if a run begins in the piece and goes on in the next
template <typename E>
__global__ __launch_bounds__(EMB_THREADS) void embed_join_kernel(const EmbedSum p, typename E::mem *__restrict__ dtable) {
    const uint32_t piece = blockIdx.x, first = piece * p.C, end = first + p.C;
    if (end >= p.T) return;
    const uint32_t key = p.key[end - 1];
    if (key >= p.V || p.key[end] != key) return;
    if (p.key[first] == key && first > 0 && p.key[first - 1] == key) return;        // it began earlier
    for (uint32_t c = threadIdx.x; c < p.D; c += EMB_THREADS) {
        float s = p.tail[(size_t)piece * p.D + c];
        for (uint32_t j = piece + 1; j < p.pieces && p.key[j * p.C] == key; ++j) s += p.head[(size_t)j * p.D + c];
        dtable[(size_t)key * p.D + c] = E::store(s * p.scale);
    }
}

}  // namespace adapt
