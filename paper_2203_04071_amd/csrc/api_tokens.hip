// C ABI, part 6: the quantiser with a scale for each token, embedding, dropout.
#include <cmath>

#include "api_common.hpp"
#include "dropout.hpp"
#include "embedding.hpp"
#include "quantize_tokens.hpp"

using namespace adapt_api;

namespace {

bool off_by(const void *p, size_t align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

unsigned cap_grid(size_t g, size_t cap) { return (unsigned)(g < 1 ? 1 : (g > cap ? cap : g)); }

// A wave per row while its pieces fit four registers' worth, then a workgroup per row, up to eight pieces a lane; longer rows are read twice.
// (512 columns fp32, 6400 rows: a workgroup per row 9.7 us, a wave 6.4 us)
template <typename E>
void quantize_tokens(const typename E::mem *x, int8_t *q, float *scales, size_t rows, size_t cols, float Q, hipStream_t s) {
    constexpr int P = adapt::piece_len<E>, T = adapt::QT_THREADS;
    const size_t pieces = (cols + P - 1) / P;
    const unsigned by_wave = cap_grid((rows + 3) / 4, 1u << 20), by_group = cap_grid(rows, 1u << 20);
    const uint32_t c = (uint32_t)cols;
    if (pieces <= 64) adapt::quantize_tokens_kernel<E, 64, 1><<<by_wave, T, 0, s>>>(x, q, scales, rows, c, Q);
    else if (pieces <= 128) adapt::quantize_tokens_kernel<E, 64, 2><<<by_wave, T, 0, s>>>(x, q, scales, rows, c, Q);
    else if (pieces <= 256) adapt::quantize_tokens_kernel<E, 64, 4><<<by_wave, T, 0, s>>>(x, q, scales, rows, c, Q);
    else if (pieces <= 2 * T) adapt::quantize_tokens_kernel<E, T, 2><<<by_group, T, 0, s>>>(x, q, scales, rows, c, Q);
    else if (pieces <= 4 * T) adapt::quantize_tokens_kernel<E, T, 4><<<by_group, T, 0, s>>>(x, q, scales, rows, c, Q);
    else if (pieces <= 8 * T) adapt::quantize_tokens_kernel<E, T, 8><<<by_group, T, 0, s>>>(x, q, scales, rows, c, Q);
    else adapt::quantize_long_tokens_kernel<E><<<by_group, T, 0, s>>>(x, q, scales, rows, cols, Q);
}

struct EmbedPlan {
    uint32_t T, V, D, C, pieces, blocks, share;
    int passes, bits;
    size_t list, counts, run, part, bytes;      // bytes of a list of places (four of them come first), offsets of the other regions
};
EmbedPlan embed_plan(size_t T, int V, int D) {
    EmbedPlan e{};
    e.T = (uint32_t)T;
    e.V = (uint32_t)V;
    e.D = (uint32_t)D;
    // (few places: short pieces, for their latency; many: long ones, for the partial sums that are written and read again)
    e.C = e.T <= 8192 ? 8 : (e.T <= 16384 ? 16 : (e.T <= 32768 ? 32 : 64));
    e.pieces = (e.T + e.C - 1) / e.C;
    e.share = (e.T + adapt::EMB_BLOCKS - 1) / adapt::EMB_BLOCKS;
    e.share = (e.share + adapt::EMB_SORT_THREADS - 1) / adapt::EMB_SORT_THREADS * adapt::EMB_SORT_THREADS;
    e.blocks = e.share ? (e.T + e.share - 1) / e.share : 0;
    int b = 1;
    while ((e.V >> b) != 0) ++b;                // keys 0 .. V
    e.passes = (b + adapt::EMB_BITS - 1) / adapt::EMB_BITS;
    e.bits = (b + e.passes - 1) / e.passes;
    e.list = round256((size_t)e.T * 4);
    e.counts = 4 * e.list;
    e.run = e.counts + round256(((size_t)e.blocks << e.bits) * 4);
    e.part = e.run + round256(((size_t)e.pieces + 2) * 4);
    e.bytes = e.part + 2 * round256((size_t)e.pieces * e.D * 4);
    return e;
}

constexpr int EMBED_MAX_D = 1 << 21;            // the runs' launch stays below 2^32 threads

int embed_args(const char *who, size_t T, int V, int D) {
    if (V < 0 || D < 0) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: negative size", who);
    if (T >= (1ull << 31)) return fail(ADAPT_ERR_UNSUPPORTED, "%s: more than 2^31-1 tokens", who);
    return ADAPT_OK;
}

// lanes that share a row of D elements in 16-byte pieces: 2^lg of them, at most a workgroup
template <typename E>
int lanes_lg(int D) {
    int lg = 0;
    while (lg < 8 && ((long long)adapt::piece_len<E> << lg) < D) ++lg;
    return lg;
}


template <typename Tok>
void embed_sort(const EmbedPlan &e, const Tok *tokens, char *ws, int64_t padding, hipStream_t s, const uint32_t **key, const uint32_t **at) {
    adapt::EmbedSort p{};
    p.counts = reinterpret_cast<uint32_t *>(ws + e.counts);
    p.runs = reinterpret_cast<uint32_t *>(ws + e.run);
    p.T = e.T;
    p.V = e.V;
    p.share = e.share;
    p.bits = e.bits;
    p.padding = padding;
    if (e.T <= adapt::EMB_SMALL) {
        p.key_out = reinterpret_cast<uint32_t *>(ws);
        p.at_out = reinterpret_cast<uint32_t *>(ws + e.list);
        adapt::embed_sort_small_kernel<<<1, adapt::EMB_SORT_THREADS, 0, s>>>(p, tokens, e.passes);
        *key = p.key_out;
        *at = p.at_out;
        return;
    }
    for (int pass = 0; pass < e.passes; ++pass) {
        char *const to = ws + (pass & 1 ? 2 * e.list : 0);
        p.key_out = reinterpret_cast<uint32_t *>(to);
        p.at_out = reinterpret_cast<uint32_t *>(to + e.list);
        p.shift = pass * e.bits;
        adapt::embed_count_kernel<<<e.blocks, adapt::EMB_SORT_THREADS, 0, s>>>(p, tokens);
        adapt::embed_scatter_kernel<<<e.blocks, adapt::EMB_SORT_THREADS, 0, s>>>(p, tokens);
        p.key_in = p.key_out;
        p.at_in = p.at_out;
    }
    *key = p.key_in;
    *at = p.at_in;
}

int dropout(const char *who, const void *x_dev, void *y_dev, int type, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t *step_dev, void *stream) {
    const size_t e = (size_t)adapt::element_size(type);
    if (!e) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: element type %d is none of ADAPT_F32, ADAPT_F16, ADAPT_BF16", who, type);
    if (!(p >= 0.0f && p <= 1.0f)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: p must be in [0,1]", who);
    if (!n) return ADAPT_OK;
    if (!x_dev || !y_dev) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL pointer", who);
    if (off_by(x_dev, e) || off_by(y_dev, e) || off_by(step_dev, 8)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (is_one_of(y_dev, {step_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: the result must not be the step", who);
    adapt::DropoutParams q{};
    q.seed = seed;
    q.offset = offset;
    q.step = step_dev;
    const double thr = std::nearbyint((double)p * 4294967296.0);
    q.none = thr >= 4294967296.0;
    q.threshold = q.none ? 0xffffffffu : (uint32_t)thr;
    q.scale = q.none ? 0.0f : (float)(1.0 / (1.0 - (double)p));
    q.n = n;
    const size_t pieces = (n + 16 / e - 1) / (16 / e);
    const unsigned grid = cap_grid((pieces + adapt::DROP_THREADS - 1) / adapt::DROP_THREADS, 256 * 32);
    ADAPT_FOR_TYPE(type, E, adapt::dropout_kernel<E><<<grid, adapt::DROP_THREADS, 0, (hipStream_t)stream>>>(
                                static_cast<const E::mem *>(x_dev), static_cast<E::mem *>(y_dev), q));
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

}  // namespace

extern "C" {

int adapt_quantize_tokens(const void *x_dev, int x_type, int8_t *q_dev, float *scales_dev, size_t tokens, size_t cols, int bits, void *stream) {
    const char *who = "adapt_quantize_tokens";
    const size_t e = (size_t)adapt::element_size(x_type);
    if (!e) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: element type %d is none of ADAPT_F32, ADAPT_F16, ADAPT_BF16", who, x_type);
    if (bits < 2 || bits > 8) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: bits=%d not in [2,8]", who, bits);
    if (!tokens) return ADAPT_OK;
    if (!scales_dev || (cols && (!x_dev || !q_dev))) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL pointer", who);
    if (off_by(x_dev, e) || off_by(scales_dev, 4)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (cols && (is_one_of(x_dev, {q_dev, scales_dev}) || is_one_of(q_dev, {scales_dev}))) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: in-place not possible", who);
    const float Q = (float)((1 << (bits - 1)) - 1);
    ADAPT_FOR_TYPE(x_type, E, quantize_tokens<E>(static_cast<const E::mem *>(x_dev), q_dev, scales_dev, tokens, cols, Q, (hipStream_t)stream));
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

/* ------------------------------------------------------------------ embedding */

int adapt_embedding(const void *table_dev, int type, const void *tokens_dev, int token_bits, void *y_dev, size_t tokens, int V, int D, float scale,
                    void *stream) {
    const char *who = "adapt_embedding";
    const size_t e = (size_t)adapt::element_size(type);
    if (!e) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: element type %d is none of ADAPT_F32, ADAPT_F16, ADAPT_BF16", who, type);
    if (token_bits != 32 && token_bits != 64) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: token_bits=%d is neither 32 nor 64", who, token_bits);
    if (int rc = embed_args(who, tokens, V, D)) return rc;
    if (!tokens || !D) return ADAPT_OK;
    if (!tokens_dev || !y_dev || (V && !table_dev)) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL pointer", who);
    if (off_by(table_dev, e) || off_by(y_dev, e) || off_by(tokens_dev, (size_t)token_bits / 8))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (is_one_of(y_dev, {table_dev, tokens_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: in-place not possible", who);
    hipStream_t s = (hipStream_t)stream;
    ADAPT_FOR_TYPE(type, E, {
        const int lg = lanes_lg<E>(D);
        const unsigned grid = cap_grid((tokens + (adapt::EMB_THREADS >> lg) - 1) / (adapt::EMB_THREADS >> lg), 1u << 16);
        const E::mem *const table = static_cast<const E::mem *>(table_dev);
        if (token_bits == 64)
            adapt::embedding_kernel<E, int64_t><<<grid, adapt::EMB_THREADS, 0, s>>>(table, static_cast<const int64_t *>(tokens_dev), static_cast<E::mem *>(y_dev),
                                                                                  tokens, (uint32_t)V, (uint32_t)D, scale, lg);
        else
            adapt::embedding_kernel<E, int32_t><<<grid, adapt::EMB_THREADS, 0, s>>>(table, static_cast<const int32_t *>(tokens_dev), static_cast<E::mem *>(y_dev),
                                                                                  tokens, (uint32_t)V, (uint32_t)D, scale, lg);
    });
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

int adapt_embedding_backward_workspace(size_t tokens, int V, int D, size_t *bytes) {
    const char *who = "adapt_embedding_backward_workspace";
    if (!bytes) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: bytes is NULL", who);
    *bytes = 0;
    if (int rc = embed_args(who, tokens, V, D)) return rc;
    if (D > EMBED_MAX_D) return fail(ADAPT_ERR_UNSUPPORTED, "%s: rows of more than %d elements", who, EMBED_MAX_D);
    *bytes = embed_plan(tokens, V, D).bytes;
    return ADAPT_OK;
}

int adapt_embedding_backward(const void *dy_dev, int type, const void *tokens_dev, int token_bits, void *dtable_dev, size_t tokens, int V, int D, float scale,
                             int64_t padding_idx, void *workspace_dev, size_t workspace_bytes, void *stream) {
    const char *who = "adapt_embedding_backward";
    const size_t e = (size_t)adapt::element_size(type);
    if (!e) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: element type %d is none of ADAPT_F32, ADAPT_F16, ADAPT_BF16", who, type);
    if (token_bits != 32 && token_bits != 64) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: token_bits=%d is neither 32 nor 64", who, token_bits);
    if (int rc = embed_args(who, tokens, V, D)) return rc;
    if (D > EMBED_MAX_D) return fail(ADAPT_ERR_UNSUPPORTED, "%s: rows of more than %d elements", who, EMBED_MAX_D);
    if (!V || !D) return ADAPT_OK;
    if (!dtable_dev || (tokens && (!tokens_dev || !dy_dev))) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: NULL pointer", who);
    if (off_by(dy_dev, e) || off_by(dtable_dev, e) || off_by(tokens_dev, (size_t)token_bits / 8))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: pointer not aligned to its elements", who);
    if (is_one_of(dtable_dev, {dy_dev, tokens_dev})) return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: the gradient must not alias an input", who);
    if (is_one_of(workspace_dev, {dy_dev, tokens_dev, dtable_dev}))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: the workspace must not alias an operand or the gradient", who);
    const EmbedPlan pl = embed_plan(tokens, V, D);
    if (!workspace_dev || workspace_bytes < pl.bytes || off_by(workspace_dev, 256))
        return fail(ADAPT_ERR_INVALID_ARGUMENT, "%s: workspace of %zu bytes, aligned to 256, is needed", who, pl.bytes);
    hipStream_t s = (hipStream_t)stream;
    char *const ws = static_cast<char *>(workspace_dev);
    adapt::EmbedSum p{};
    if (tokens) {
        if (token_bits == 64) embed_sort(pl, static_cast<const int64_t *>(tokens_dev), ws, padding_idx, s, &p.key, &p.at);
        else embed_sort(pl, static_cast<const int32_t *>(tokens_dev), ws, padding_idx, s, &p.key, &p.at);
    }
    p.runs = reinterpret_cast<uint32_t *>(ws + pl.run);
    p.run = p.runs + 2;
    p.head = reinterpret_cast<float *>(ws + pl.part);
    p.tail = reinterpret_cast<float *>(ws + pl.part + round256((size_t)pl.pieces * pl.D * 4));
    p.T = pl.T;
    p.V = pl.V;
    p.D = pl.D;
    p.C = pl.C;
    p.pieces = pl.pieces;
    p.scale = scale;
    ADAPT_FOR_TYPE(type, E, {
        p.lg = lanes_lg<E>(D);
        const unsigned per = (unsigned)(adapt::EMB_THREADS >> p.lg);
        p.sum_blocks = (pl.pieces + per - 1) / per;
        const unsigned zero_blocks = cap_grid(((size_t)V + 4 * adapt::EMB_ZERO_ROWS - 1) / (4 * adapt::EMB_ZERO_ROWS), 4096);
        adapt::embed_sum_kernel<E><<<p.sum_blocks + zero_blocks, adapt::EMB_THREADS, 0, s>>>(p, static_cast<const E::mem *>(dy_dev), static_cast<E::mem *>(dtable_dev));
        if (pl.pieces > 1)
            adapt::embed_join_kernel<E><<<dim3(adapt::EMB_LONG_BLOCKS + cap_grid((pl.pieces + 15) / 16, 64), ((unsigned)D + 63) / 64), 1024, 0, s>>>(p, static_cast<E::mem *>(dtable_dev));
    });
    HIP_TRY(hipGetLastError());
    return ADAPT_OK;
}

/* ------------------------------------------------------------------ dropout */

int adapt_dropout(const void *x_dev, void *y_dev, int type, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t *step_dev, void *stream) {
    return dropout("adapt_dropout", x_dev, y_dev, type, n, p, seed, offset, step_dev, stream);
}

int adapt_dropout_backward(const void *dy_dev, void *dx_dev, int type, size_t n, float p, uint64_t seed, uint64_t offset, const uint64_t *step_dev,
                           void *stream) {
    return dropout("adapt_dropout_backward", dy_dev, dx_dev, type, n, p, seed, offset, step_dev, stream);
}

}  // extern "C"
