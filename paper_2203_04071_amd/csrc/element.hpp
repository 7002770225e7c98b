// Element types of activations and gradients in the token-wise operators: fp32, fp16 and bf16 in memory, fp32 in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/adapt_mi355.h"

namespace adapt {

struct F32 {
    typedef float mem;
    static __device__ __forceinline__ float load(mem v) { return v; }
    static __device__ __forceinline__ mem store(float v) { return v; }
};
struct F16 {
    typedef _Float16 mem;
    static __device__ __forceinline__ float load(mem v) { return (float)v; }
    // Round to nearest even, overflow to infinity.  (The empty statement keeps the compiler from folding an fp32 product into the
    // conversion, v_fma_mixlo_f16, which rounds once where every other path rounds the fp32 step first.)
    static __device__ __forceinline__ mem store(float v) {
        asm("" : "+v"(v));
        return (mem)v;
    }
};
struct BF16 {
    typedef __bf16 mem;
    static __device__ __forceinline__ float load(mem v) { return (float)v; }
    static __device__ __forceinline__ mem store(float v) { return (mem)v; }         // round to nearest even (v_cvt_pk_bf16_f32)
};

// N elements of E that lie together, read or written in one piece.  Only the alignment of an element is assumed: the hardware takes
// 16-byte requests at any address, and one that crosses a line costs a second line, not a second instruction.
template <typename E, int N>
struct __attribute__((packed, aligned(sizeof(typename E::mem)))) Piece {
    typename E::mem v[N];
};
template <typename E, int N>
__device__ __forceinline__ void load_piece(const typename E::mem *p, float (&out)[N]) {
    Piece<E, N> t;
    __builtin_memcpy(&t, __builtin_assume_aligned(p, sizeof(typename E::mem)), sizeof(t));
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = E::load(t.v[i]);
}
template <typename E, int N>
__device__ __forceinline__ void store_piece(typename E::mem *p, const float (&in)[N]) {
    Piece<E, N> t;
#pragma unroll
    for (int i = 0; i < N; ++i) t.v[i] = E::store(in[i]);
    __builtin_memcpy(__builtin_assume_aligned(p, sizeof(typename E::mem)), &t, sizeof(t));
}

template <typename E>
constexpr int piece_len = 16 / (int)sizeof(typename E::mem);       // elements of one 16-byte request

inline int element_size(int type) { return type == ADAPT_F32 ? 4 : (type == ADAPT_F16 || type == ADAPT_BF16 ? 2 : 0); }

}  // namespace adapt

// f(E) with the element type that `type` names
#define ADAPT_FOR_TYPE(type, E, ...)                                             \
    do {                                                                         \
        if ((type) == ADAPT_F32) { typedef adapt::F32 E; __VA_ARGS__; }          \
        else if ((type) == ADAPT_F16) { typedef adapt::F16 E; __VA_ARGS__; }     \
        else { typedef adapt::BF16 E; __VA_ARGS__; }                             \
    } while (0)
