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

// Where the piece of P elements at c of a row of D is taken: the last one ends with the row, and does again what the one before it does in part
// (the same numbers, written twice).  Rows shorter than a piece: element by element.
template <int P>
__device__ __forceinline__ uint32_t embed_piece(uint32_t c, uint32_t D) { return c + P <= D || D < P ? c : D - P; }

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
            const uint32_t at = embed_piece<P>(c, D);
            if (at + P <= D) {
                float f[P];
                if (v < V) load_piece<E, P>(from + at, f);
#pragma unroll
                for (int i = 0; i < P; ++i) f[i] = v < V ? f[i] * scale : 0.0f;
                store_piece<E, P>(to + at, f);
            } else {
                for (uint32_t i = at; i < D; ++i) to[i] = E::store(v < V ? E::load(from[i]) * scale : 0.0f);
            }
        }
    }
}

// ---- the gradient: places sorted by token (stable), sums of runs of equal tokens
//
// Least significant digit first, up to EMB_BITS bits a pass, two launches a pass.  At most EMB_BLOCKS workgroups of 16 waves, each with a
// contiguous share of the places, one digit per thread: count, then (every workgroup adds up the counts before its own) scatter.
constexpr int EMB_BITS = 9;
constexpr int EMB_BLOCKS = 128;
constexpr int EMB_SORT_THREADS = 1024;
constexpr int EMB_WAVES = EMB_SORT_THREADS / 64;

struct EmbedSort {
    const uint32_t *key_in, *at_in;     // nullptr in the first pass: keys come from the tokens, places are 0, 1, 2 ...
    uint32_t *key_out, *at_out;
    uint32_t *counts;                   // [workgroup][digit]
    uint32_t *runs;                     // numbers of runs for embed_join_kernel (two), set to 0 in the first pass
    uint32_t T, V, share;               // share: places of a workgroup, a multiple of EMB_SORT_THREADS
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

// Where the lane's place goes: behind the ones of its digit in earlier lanes; `next` (the wave's next free place of each digit) moves on.
// The lanes of a wave run together and its LDS requests are carried out in order: every peer has read the place before the first
// of them moves it on.
__device__ __forceinline__ uint32_t embed_next_place(uint32_t *next, uint32_t digit, int bits, bool active) {
    const uint64_t peers = embed_peers(digit, bits, active);
    const uint32_t rank = __popcll(peers & ((1ull << (threadIdx.x & 63)) - 1));
    const uint32_t to = active ? __hip_atomic_load(&next[digit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT) + rank : 0u;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (active && rank == 0) __hip_atomic_store(&next[digit], to + (uint32_t)__popcll(peers), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return to;
}

// [wave][digit] counts of this workgroup's places; a wave owns a contiguous sixteenth of them
template <typename Tok>
__device__ __forceinline__ void embed_count(const EmbedSort &p, const Tok *__restrict__ tokens, uint32_t (*hist)[1 << EMB_BITS]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < EMB_WAVES << EMB_BITS; i += EMB_SORT_THREADS) hist[i >> EMB_BITS][i & ((1 << EMB_BITS) - 1)] = 0;
    __syncthreads();
    const uint32_t per_wave = p.share / EMB_WAVES, from = blockIdx.x * p.share + wave * per_wave;
    for (uint32_t u = 0; u < per_wave; u += 64) {
        const uint32_t i = from + u + lane;
        if (i < p.T) atomicAdd(&hist[wave][(embed_key(p, tokens, i) >> p.shift) & ((1u << p.bits) - 1)], 1u);
    }
    __syncthreads();
}

template <typename Tok>
__global__ __launch_bounds__(EMB_SORT_THREADS) void embed_count_kernel(const EmbedSort p, const Tok *__restrict__ tokens) {
    __shared__ uint32_t hist[EMB_WAVES][1 << EMB_BITS];
    embed_count(p, tokens, hist);
    const int d = threadIdx.x;
    if (d < 1 << p.bits) {
        uint32_t s = 0;
#pragma unroll
        for (int w = 0; w < EMB_WAVES; ++w) s += hist[w][d];
        p.counts[((size_t)blockIdx.x << p.bits) + d] = s;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) p.runs[threadIdx.x] = 0;
}

template <typename Tok>
__global__ __launch_bounds__(EMB_SORT_THREADS) void embed_scatter_kernel(const EmbedSort p, const Tok *__restrict__ tokens) {
    __shared__ uint32_t hist[EMB_WAVES][1 << EMB_BITS];
    __shared__ uint32_t wave_sum[EMB_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = threadIdx.x;
    const bool mine = d < 1 << p.bits;
    // places of digit d: in all workgroups, in those before this one
    uint32_t all = 0, before = 0;
    if (mine) {
#pragma unroll 8
        for (uint32_t b = 0; b < gridDim.x; ++b) {
            const uint32_t c = p.counts[((size_t)b << p.bits) + d];
            all += c;
            before += b < blockIdx.x ? c : 0u;
        }
    }
    uint32_t incl = all;                // and of the digits before it
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_up(incl, off, 64);
        if (lane >= off) incl += o;
    }
    if (lane == 63) wave_sum[wave] = incl;
    embed_count(p, tokens, hist);       // (ends with a barrier)
    if (mine) {                         // counts become the wave's next free place
        uint32_t at = incl - all + before;
        for (int w = 0; w < wave; ++w) at += wave_sum[w];
#pragma unroll
        for (int w = 0; w < EMB_WAVES; ++w) {
            const uint32_t c = hist[w][d];
            hist[w][d] = at;
            at += c;
        }
    }
    __syncthreads();
    const uint32_t per_wave = p.share / EMB_WAVES, from = blockIdx.x * p.share + wave * per_wave;
    for (uint32_t u = 0; u < per_wave; u += 64) {
        const uint32_t i = from + u + lane;
        const bool in = i < p.T;
        const uint32_t key = in ? embed_key(p, tokens, i) : 0u;
        const uint32_t digit = (key >> p.shift) & ((1u << p.bits) - 1);
        const uint32_t to = embed_next_place(hist[wave], digit, p.bits, in);
        if (in) {
            p.key_out[to] = key;
            p.at_out[to] = p.at_in ? p.at_in[i] : i;
        }
    }
}

// Few places: all passes in one workgroup, keys and places in LDS.  (2048 places, two passes: 9 us against 19 in four launches; from 6400 on the four are faster)
constexpr uint32_t EMB_SMALL = 4096;
template <typename Tok>
__global__ __launch_bounds__(EMB_SORT_THREADS) void embed_sort_small_kernel(const EmbedSort p, const Tok *__restrict__ tokens, int passes) {
    __shared__ uint32_t keys[2][EMB_SMALL];
    __shared__ uint16_t places[2][EMB_SMALL];
    __shared__ uint32_t hist[EMB_WAVES][1 << EMB_BITS];
    __shared__ uint32_t wave_sum[EMB_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = threadIdx.x;
    for (uint32_t i = threadIdx.x; i < p.T; i += EMB_SORT_THREADS) {
        keys[0][i] = embed_key(p, tokens, i);
        places[0][i] = (uint16_t)i;
    }
    if (threadIdx.x < 2) p.runs[threadIdx.x] = 0;
    const uint32_t per_wave = (p.T + EMB_SORT_THREADS - 1) / EMB_SORT_THREADS * 64, from = wave * per_wave;
    const uint32_t mask = (1u << p.bits) - 1;
    int now = 0;
    for (int pass = 0; pass < passes; ++pass, now ^= 1) {
        const int shift = pass * p.bits;
        for (int i = threadIdx.x; i < EMB_WAVES << EMB_BITS; i += EMB_SORT_THREADS) hist[i >> EMB_BITS][i & ((1 << EMB_BITS) - 1)] = 0;
        __syncthreads();
        for (uint32_t u = 0; u < per_wave; u += 64) {
            const uint32_t i = from + u + lane;
            if (i < p.T) atomicAdd(&hist[wave][(keys[now][i] >> shift) & mask], 1u);
        }
        __syncthreads();
        uint32_t all = 0;
        if (d <= (int)mask)
#pragma unroll
            for (int w = 0; w < EMB_WAVES; ++w) all += hist[w][d];
        uint32_t incl = all;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = __shfl_up(incl, off, 64);
            if (lane >= off) incl += o;
        }
        if (lane == 63) wave_sum[wave] = incl;
        __syncthreads();
        if (d <= (int)mask) {
            uint32_t at = incl - all;
            for (int w = 0; w < wave; ++w) at += wave_sum[w];
#pragma unroll
            for (int w = 0; w < EMB_WAVES; ++w) {
                const uint32_t c = hist[w][d];
                hist[w][d] = at;
                at += c;
            }
        }
        __syncthreads();
        for (uint32_t u = 0; u < per_wave; u += 64) {
            const uint32_t i = from + u + lane;
            const bool in = i < p.T;
            const uint32_t key = in ? keys[now][i] : 0u, place = in ? places[now][i] : 0u;
            const uint32_t to = embed_next_place(hist[wave], (key >> shift) & mask, p.bits, in);
            if (in) {
                keys[now ^ 1][to] = key;
                places[now ^ 1][to] = (uint16_t)place;
            }
        }
        __syncthreads();
    }
    for (uint32_t i = threadIdx.x; i < p.T; i += EMB_SORT_THREADS) {
        p.key_out[i] = keys[now][i];
        p.at_out[i] = places[now][i];
    }
}

typedef uint32_t i32x4_raw __attribute__((ext_vector_type(4)));
constexpr uint32_t EMB_LONG = 32;       // see embed_join_kernel

// Sums.  The sorted places are cut into pieces of C, each summed by 2^lg lanes; a run of equal tokens inside a piece is finished there.
// One that crosses pieces leaves a partial sum in every piece: `head` for the part at a piece's start that began earlier, `tail` for
// the part at its end that goes on; embed_join_kernel adds them in order.  Bounded by memory: dy is read once, the table written once.
struct EmbedSum {
    const uint32_t *key, *at;
    // pieces in whose tail a run begins that goes on, in any order: numbers of short and of long ones; short ones from the list's start
    // on, long ones from its end back
    uint32_t *runs, *run;
    float *head, *tail;                 // [pieces][D]
    uint32_t T, V, D, C, pieces;
    float scale;
    int lg;
    uint32_t sum_blocks;                // workgroups beyond these write the rows without a token
};

// Rows without a token: the first EMB_ZERO_ROWS lanes of a wave look for a row each in the sorted keys, then the wave writes the pieces of all
// those that are not there.
constexpr uint32_t EMB_ZERO_ROWS = 16;
template <typename E>
__device__ __forceinline__ void embed_empty_rows(const EmbedSum &p, typename E::mem *__restrict__ dtable) {
    constexpr uint32_t P = piece_len<E>;
    const float zero[P] = {};
    const uint32_t lane = threadIdx.x & 63, waves = (gridDim.x - p.sum_blocks) * (EMB_THREADS / 64), pieces = (p.D + P - 1) / P;
    for (uint64_t v0 = ((uint64_t)(blockIdx.x - p.sum_blocks) * (EMB_THREADS / 64) + (threadIdx.x >> 6)) * EMB_ZERO_ROWS; v0 < p.V;
         v0 += (uint64_t)waves * EMB_ZERO_ROWS) {
        const uint64_t v = v0 + lane;
        uint32_t lo = 0, n = lane < EMB_ZERO_ROWS ? p.T : 0u;        // first place whose key is not below v
        while (n > 0) {
            const uint32_t half = n / 2;
            const bool below = p.key[lo + half] < v;
            lo = below ? lo + half + 1 : lo;
            n = below ? n - half - 1 : half;
        }
        const uint64_t absent = __ballot(lane < EMB_ZERO_ROWS && v < p.V && (lo >= p.T || p.key[lo] != v));
        typename E::mem *const rows = dtable + (size_t)v0 * p.D;
        // (lane by lane through the pieces of the rows: row and piece move on together)
        uint32_t row = lane / pieces, piece = lane % pieces;
        const uint32_t rows_on = 64 / pieces, pieces_on = 64 % pieces;
        while (row < EMB_ZERO_ROWS) {
            if ((absent >> row) & 1) {
                const uint32_t at = embed_piece<P>(piece * P, p.D);
                typename E::mem *const to = rows + (size_t)row * p.D;
                if (at + P <= p.D) store_piece<E, P>(to + at, zero);
                else
                    for (uint32_t i = at; i < p.D; ++i) to[i] = E::store(0.0f);
            }
            row += rows_on;
            piece += pieces_on;
            if (piece >= pieces) {
                piece -= pieces;
                ++row;
            }
        }
    }
}

template <typename E>
__global__ __launch_bounds__(EMB_THREADS) void embed_sum_kernel(const EmbedSum p, const typename E::mem *__restrict__ dy, typename E::mem *__restrict__ dtable) {
    constexpr int P = piece_len<E>;
    if (blockIdx.x >= p.sum_blocks) {
        embed_empty_rows<E>(p, dtable);
        return;
    }
    const uint32_t lane = threadIdx.x & ((1u << p.lg) - 1), per = EMB_THREADS >> p.lg;
    const uint32_t piece = blockIdx.x * per + (threadIdx.x >> p.lg);
    if (piece >= p.pieces) return;
    const uint32_t first = piece * p.C, last = min(first + p.C, p.T);       // (pieces cover T: first < T)
    for (uint32_t c0 = lane * P; c0 < p.D; c0 += (uint32_t)P << p.lg) {
        const uint32_t c = embed_piece<P>(c0, p.D);
        const int len = (int)min((uint32_t)P, p.D - c);
        float acc[P] = {};
        uint32_t key = p.key[first];
        bool open = first > 0 && p.key[first - 1] == key;       // the run began in an earlier piece
        // the sum of a run so far is complete: `next` is the key behind it
        auto close = [&](uint32_t next) {
            if (open || next == key) {
                float *const part = (open ? p.head : p.tail) + (size_t)piece * p.D + c;
                if (len == P) store_piece<F32, P>(part, acc);
                else
                    for (int j = 0; j < len; ++j) part[j] = acc[j];
                if (!open && c0 == 0) {
                    const bool many = piece + EMB_LONG < p.pieces && p.key[(piece + EMB_LONG) * p.C] == key;
                    const uint32_t at = atomicAdd(&p.runs[many], 1u);
                    p.run[many ? p.pieces - 1 - at : at] = piece;
                }
            } else if (len == P) {
#pragma unroll
                for (int j = 0; j < P; ++j) acc[j] *= p.scale;
                store_piece<E, P>(dtable + (size_t)key * p.D + c, acc);
            } else {
                for (int j = 0; j < len; ++j) dtable[(size_t)key * p.D + c + j] = E::store(acc[j] * p.scale);
            }
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] = 0.0f;
            open = false;
            key = next;
        };
        uint32_t i = first;
        // eight places at a time, their rows requested together (one after the other: 56 us instead of 44 for 65536 x 1024 bf16)
        for (; len == P && i + 8 <= last && p.key[i + 7] < p.V; i += 8) {
            uint32_t k[9];
            i32x4_raw row[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                k[u] = p.key[i + u];
                __builtin_memcpy(&row[u], dy + (size_t)p.at[i + u] * p.D + c, 16);
            }
            k[8] = i + 8 < p.T ? p.key[i + 8] : ~0u;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                float f[P];
                load_piece<E, P>(reinterpret_cast<const typename E::mem *>(&row[u]), f);
#pragma unroll
                for (int j = 0; j < P; ++j) acc[j] += f[j];
                if (k[u + 1] != k[u] || (u == 7 && i + 8 == last)) close(k[u + 1]);
            }
        }
        for (; i < last; ++i) {
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
            if (next != key || i + 1 == last) close(next);
        }
    }
}

// Runs that cross pieces, 64 columns each: a short one (up to EMB_LONG parts behind its first) is added by a wave, a long one by the sixteen waves of
// a workgroup, a contiguous sixteenth of its parts each, whose sums the first wave adds in order.  (A run per workgroup of 256 columns, its
// parts one after the other: 124 us for 65536 places of 1024 columns, a fifth of them one token.)
constexpr unsigned EMB_LONG_BLOCKS = 32;
template <typename E>
__global__ __launch_bounds__(1024) void embed_join_kernel(const EmbedSum p, typename E::mem *__restrict__ dtable) {
    __shared__ float sum[16][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 64 + lane;
    // parts of the run that begins in the tail of `piece`: that tail, and the heads of the pieces whose first key is the run's
    auto parts_of = [&](uint32_t piece, uint32_t key) {
        uint32_t end = piece + 1, n = p.pieces - end;
        while (n > 0) {
            const uint32_t half = n / 2;
            const bool in = p.key[(end + half) * p.C] == key;
            end = in ? end + half + 1 : end;
            n = in ? n - half - 1 : half;
        }
        return end - piece;
    };
    auto add = [&](uint32_t piece, uint32_t from, uint32_t to) {
        float s = 0.0f;
        uint32_t j = from;
        for (; j + 8 <= to; j += 8) {
            float t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = (j + u == 0 ? p.tail : p.head)[(size_t)(piece + j + u) * p.D + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += t[u];
        }
        for (; j < to; ++j) s += (j == 0 ? p.tail : p.head)[(size_t)(piece + j) * p.D + c];
        return s;
    };
    if (blockIdx.x < EMB_LONG_BLOCKS) {
        const uint32_t runs = p.runs[1];
        for (uint32_t r = blockIdx.x; r < runs; r += EMB_LONG_BLOCKS) {
            const uint32_t piece = p.run[p.pieces - 1 - r], key = p.key[(piece + 1) * p.C], parts = parts_of(piece, key);
            const uint32_t share = (parts + 15) / 16, from = min(wave * share, parts), to = min(from + share, parts);
            float s = c < p.D ? add(piece, from, to) : 0.0f;
            sum[wave][lane] = s;
            __syncthreads();
            if (wave == 0 && c < p.D) {
#pragma unroll
                for (int w = 1; w < 16; ++w) s += sum[w][lane];
                dtable[(size_t)key * p.D + c] = E::store(s * p.scale);
            }
            __syncthreads();
        }
    } else if (c < p.D) {
        const uint32_t runs = p.runs[0], waves = (gridDim.x - EMB_LONG_BLOCKS) * 16;
        for (uint32_t r = (blockIdx.x - EMB_LONG_BLOCKS) * 16 + wave; r < runs; r += waves) {
            const uint32_t piece = p.run[r], key = p.key[(piece + 1) * p.C];
            dtable[(size_t)key * p.D + c] = E::store(add(piece, 0, parts_of(piece, key)) * p.scale);
        }
    }
}

}  // namespace adapt
