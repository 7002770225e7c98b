"""CPU oracle of the token-wise operators (exact 8-bit product with token and channel scales, its gradients, embedding, dropout):
numpy, from the definitions in the public header, in 64 bits where sums or products are concerned and in fp32 steps where the
definition rounds to fp32.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def quantize_tokens(x, bits):
    """x float [M][K] -> (int8 codes, fp32 scales): the scale a product with the rounded 1 / Q (tests/test_tokens_definitions_host.py: how far that is
    from max / Q), every code by an IEEE fp32 division."""
    x = np.asarray(x, dtype=np.float32)
    q_max = np.float32((1 << (bits - 1)) - 1)
    mag = np.where(np.isnan(x), np.float32(0), np.abs(x))
    s = (mag.max(axis=1) if x.shape[1] else np.zeros(x.shape[0], np.float32)) * (np.float32(1) / q_max)
    s = s.astype(np.float32)
    with np.errstate(all="ignore"):
        r = np.rint(x / s[:, None])
    r = np.where(np.isnan(r) | ~(s[:, None] > 0), np.float32(0), r)
    return np.clip(r, -q_max, q_max).astype(np.int8), s


def int8_sums(a, w):
    """int64 [M][N]"""
    return np.rint(a.astype(np.float64) @ w.astype(np.float64).T).astype(np.int64)       # |sums| < 2^31: exact in fp64


def int8_linear(a, s_a, w, s_w, bias=None, act=0, tanh=None):
    """fp32 [M][N], every step rounded to fp32 in the order of the definition."""
    y = int8_sums(a, w).astype(np.int32).astype(np.float32)
    with np.errstate(all="ignore"):
        y = (y * s_a[:, None].astype(np.float32)) * s_w[None, :].astype(np.float32)
        if bias is not None:
            y = y + bias[None, :].astype(np.float32)
    if act == 1:
        y = np.where(y > 0, y, np.float32(0))
    elif act == 2:
        y = tanh(y)
    return y


def int8_linear_backward(dy, a, s_a, w, s_w):
    """((dx, sum of |terms|), (dw, ...), (db, ...)) in fp64."""
    dy = dy.astype(np.float64)
    wf = w.astype(np.float64) * s_w.astype(np.float64)[:, None]
    af = a.astype(np.float64) * s_a.astype(np.float64)[:, None]
    return ((dy @ wf, np.abs(dy) @ np.abs(wf)), (dy.T @ af, np.abs(dy).T @ np.abs(af)), (dy.sum(0), np.abs(dy).sum(0)))


def embedding(table, tokens, scale):
    V = table.shape[0]
    y = np.zeros(tokens.shape + (table.shape[1],), np.float32)
    ok = (tokens >= 0) & (tokens < V)
    y[ok] = table.astype(np.float32)[tokens[ok]] * np.float32(scale)
    return y


def embedding_backward(dy, tokens, V, scale, padding_idx=-1):
    """(gradient, sum of |terms|, places per token) in fp64."""
    D = dy.shape[-1]
    dy, tokens = dy.reshape(-1, D).astype(np.float64), tokens.reshape(-1)
    ok = (tokens >= 0) & (tokens < V) & (tokens != padding_idx)
    g, m, n = np.zeros((V, D)), np.zeros((V, D)), np.zeros(V, np.int64)
    np.add.at(g, tokens[ok], dy[ok])
    np.add.at(m, tokens[ok], np.abs(dy[ok]))
    np.add.at(n, tokens[ok], 1)
    s = float(np.float32(scale))
    return g * s, m * abs(s), n


def philox4x32(counter, key, rounds=10):
    """counter uint32 [..., 4], key (k0, k1) -> uint32 [..., 4] (Salmon et al. 2011)."""
    c = [counter[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & np.uint64(0xFFFFFFFF),
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & np.uint64(0xFFFFFFFF)]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1).astype(np.uint32)


def dropout_kept(n, p, seed, offset, first=0):
    """bool [n]: elements first .. first + n - 1"""
    i = np.arange(first // 4, (first + n + 3) // 4, dtype=np.uint64)
    offset &= (1 << 64) - 1
    counter = np.stack([(i & np.uint64(0xFFFFFFFF)).astype(np.uint32), (i >> np.uint64(32)).astype(np.uint32),
                        np.full(i.shape, offset & 0xFFFFFFFF, np.uint32), np.full(i.shape, offset >> 32, np.uint32)], axis=-1)
    r = philox4x32(counter, (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)).reshape(-1)[first % 4:][:n]
    return r.astype(np.int64) >= int(np.rint(float(np.float32(p)) * 2.0 ** 32))


def dropout(x, p, seed, offset):
    """fp32: kept elements times 1 / (1 - p) rounded to fp32"""
    p = float(np.float32(p))
    factor = np.float32(1.0 / (1.0 - p)) if p < 1 else np.float32(0)
    kept = dropout_kept(x.size, p, seed, offset).reshape(x.shape)
    with np.errstate(all="ignore"):
        return np.where(kept, x.astype(np.float32) * factor, np.float32(0))
