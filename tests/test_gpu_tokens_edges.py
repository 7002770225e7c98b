"""Token-wise operators where their definition is easiest to miss: sums whose terms cancel, elements far below their row's largest, the order of places."""
import numpy as np
import pytest

import oracle as orc
from oracle import tokens as ot
from test_gpu_tokens import TYPES, U, B, _t, codes, dev, f64, randn, rounded, same_bits, scales, tokens_of, within  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- gradients of the product

def far_below(t, q):
    """What elements far below the largest of their row t[i] may lose in all: 2^-39 of it for every unit of the codes q [r][j].  (The largest is brought to
    2^14 at least, and half of the smallest fp16 number is 2^-25.)"""
    return 2.0 ** -39 * np.abs(t.astype(np.float64)).max(axis=1, initial=0.0)[:, None] * np.abs(q.astype(np.float64)).sum(axis=0)[None, :]


def within_22_bits(got, want, mass, terms, name, lost):
    """A gradient of any type: dy * s to 22 bits (2^-22 of a term), sums of fp32, one rounding to the type at the end.  mass: sum of |terms|."""
    import torch
    fi = torch.finfo(_t(name))
    bound = ((terms + 2) * U + 2.0 ** -22) * mass + lost + 2.0 ** -149 * (terms + 2)
    if name != "f32":
        bound = bound * (1 + fi.eps) + fi.eps / 2 * np.abs(want) + fi.smallest_normal * fi.eps / 2
    bad = ~(np.abs(f64(got) - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), f64(got)[bad][:4], want[bad][:4], np.broadcast_to(bound, want.shape)[bad][:4])


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("M,K,N", [(3, 5, 8), (70, 40, 64), (200, 130, 66)])
def test_gradients_of_sums_whose_terms_cancel(B, name, M, K, N):
    """Pairs of terms that differ by a few units of 2^-12 of themselves and have opposite signs: what is left of the sum keeps the type's bits."""
    rng = np.random.default_rng(M + N)
    # dx: pairs of channels with the same codes and nearly the same scale
    w, s_w = np.repeat(codes(rng, N // 2, K), 2, axis=0), np.repeat(scales(rng, N // 2), 2)
    s_w[1::2] *= (1 + rng.integers(1, 9, N // 2) * 2.0 ** -12).astype(np.float32)
    dy = np.repeat(rng.standard_normal((M, N // 2)), 2, axis=1) * np.where(np.arange(N) % 2, -1.0, 1.0)
    t = rounded(dy.astype(np.float32), name)
    dy = t.float().numpy()
    a, s_a = codes(rng, M, K), scales(rng, M)
    dx, _, _ = B.adapt_int8_linear_backward(t.cuda(), dev(a), dev(s_a), dev(w), dev(s_w))
    (wx, mx), _, _ = ot.int8_linear_backward(dy, a, s_a, w, s_w)
    within_22_bits(dx, wx, mx, N, name, far_below(dy * s_w, w))
    # dw: the same with pairs of tokens (the product's two sides change places)
    _, dw, _ = B.adapt_int8_linear_backward(dev(dy.T).to(_t(name)), dev(w), dev(s_w), dev(a), dev(s_a))
    _, (ww, mw), _ = ot.int8_linear_backward(dy.T, w, s_w, a, s_a)
    within_22_bits(dw, ww, mw, N, name, far_below((dy.T * s_w[:, None]).T, w))


@pytest.mark.parametrize("name", TYPES)
def test_gradients_keep_what_two_terms_leave(B, name):
    """(1 + 2^-13) - 1"""
    near, one = np.array([1 + 2.0 ** -13, 1], np.float32), np.ones(1, np.float32)
    q1, q2 = np.ones((1, 1), np.int8), np.ones((2, 1), np.int8)
    dy = dev(np.array([[1, -1]], np.float32)).to(_t(name))
    dx, _, _ = B.adapt_int8_linear_backward(dy, dev(q1), dev(one), dev(q2), dev(near))
    _, dw, _ = B.adapt_int8_linear_backward(dy.t().contiguous(), dev(q2), dev(near), dev(q1), dev(one))
    assert f64(dx) == 2.0 ** -13 and f64(dw) == 2.0 ** -13


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("far", [1.0, 1.5, 2.0, 3.0, 2.0 ** 10])
@pytest.mark.parametrize("largest", [1.0, 1.9921875])
def test_gradients_lose_at_most_2_to_minus_39_of_the_largest(B, name, far, largest):
    """An element of far * 2^-39 beside the largest, which meets a code of 0.  With a largest of a power of two and far = 1 all of it is lost: no
    smaller bound holds."""
    small = 1.0 if name == "f16" else 2.0 ** -39            # (fp16 has no 2^-39: the scales bring the elements apart)
    scale = np.array([1.0, 2.0 ** -39 / small], np.float32)
    dy = dev(np.array([[largest, far * small]], np.float32)).to(_t(name))
    q, one = np.array([[0], [1]], np.int8), np.ones(1, np.float32)
    dx, _, _ = B.adapt_int8_linear_backward(dy, dev(q[:1]), dev(one), dev(q), dev(scale))
    _, dw, _ = B.adapt_int8_linear_backward(dy.t().contiguous(), dev(q), dev(scale), dev(q[:1]), dev(one))
    lost = far * 2.0 ** -39 - np.array([f64(dx).item(), f64(dw).item()])
    step = 2.0 ** -24 if name == "f16" else 0.0             # (nor has its result)
    assert (np.abs(lost) <= 2.0 ** -39 * largest + step / 2).all()
    if far == 1 and largest == 1:
        assert (lost == 2.0 ** -39).all()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("M,K,N", [(0, 8, 9), (7, 300, 0), (5, 0, 6), (0, 1000, 300), (600, 130, 0)])
def test_gradients_of_empty_sums(B, name, M, K, N):
    """No tokens: dw and db are zeros; no channels: dx is; whatever the results' memory held before."""
    import torch
    z = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")
    for want in (("dx", "dw", "db"), ("dx",), ("dw",), ("db",)):
        for _ in range(2):
            junk = [torch.full((n,), float("nan"), dtype=_t(name), device="cuda") for n in (M * K, N * K, N)]
            del junk
            dx, dw, db = B.adapt_int8_linear_backward(torch.ones((M, N), dtype=_t(name), device="cuda"), z(M, K), torch.ones(M, device="cuda"), z(N, K),
                                                      torch.ones(N, device="cuda"), want=want)
            assert dx is None or (dx.shape == (M, K) and (dx == 0).all())
            assert dw is None or (dw.shape == (N, K) and (dw == 0).all())
            assert db is None or (db.shape == (N,) and (db == M).all())


# ---------------------------------------------------------------------------------------------- embedding

@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("T,V,D", [(300, 7, 40), (4096, 100, 33), (40000, 50000, 64), (70001, 12, 40)])
def test_embedding_gradient_does_not_depend_on_where_the_places_lie(B, name, T, V, D):
    """Tokens in another order, the gradients moved with them so that every token's places keep theirs: the same sums in the same order, the same bits."""
    rng = np.random.default_rng(T)
    tok = tokens_of(rng, "zipf", T, V)
    tok[rng.random(T) < 0.4] = 3
    dy, dyd = randn(rng, (T, D), name)
    got = B.adapt_embedding_backward(dyd, dev(tok), V, scale=0.7)
    want, mass, n = ot.embedding_backward(dy, tok, V, 0.7)
    within(got, want, mass, n[:, None], name)
    other = rng.permutation(tok)
    assert (other != tok).any()
    moved = np.empty_like(dy)
    moved[np.argsort(other, kind="stable")] = dy[np.argsort(tok, kind="stable")]
    assert np.array_equal(moved[other == 3], dy[tok == 3])
    same_bits(B.adapt_embedding_backward(rounded(moved, name).cuda(), dev(other), V, scale=0.7), got.cpu())


# ---------------------------------------------------------------------------------------------- product

# few tokens; rows of 16-byte pieces; rows of any length (each of them with and without whole stages and whole tiles)
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("M,K,N", [(1, 512, 2048), (16, 304, 70), (7, 301, 70), (16, 3, 17), (17, 512, 64), (40, 304, 70), (300, 1040, 257), (640, 128, 640),
                                   (17, 15, 64), (40, 300, 70), (300, 513, 130), (2050, 77, 300)])
def test_product_with_tanh(B, name, M, K, N):
    rng = np.random.default_rng(M + K)
    a, w, s_a, s_w = codes(rng, M, K), codes(rng, N, K), scales(rng, M) * 0.1, scales(rng, N) * 0.1
    bias = rng.standard_normal(N).astype(np.float32)
    for b in (None, bias):
        got = B.adapt_int8_linear(dev(a), dev(s_a), dev(w), dev(s_w), bias=None if b is None else dev(b), act=2, dtype=_t(name))
        same_bits(got, rounded(ot.int8_linear(a, s_a, w, s_w, b, 2, tanh=orc.tanh), name))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("M,K,N", [(5, 64, 40), (300, 256, 300), (300, 257, 300)])
def test_tokens_that_hold_an_infinity(B, name, M, K, N):
    """Their scale is infinite, their codes 0: NaN in every channel, which a ReLU turns into 0.  The other tokens do not see them."""
    rng = np.random.default_rng(K)
    x, _ = randn(rng, (M, K), name)
    x[1, 3], x[4, K - 1] = np.inf, -np.inf
    a, s_a = B.adapt_quantize_tokens(dev(x).to(_t(name)))
    w, s_w = codes(rng, N, K), scales(rng, N)
    q, s = ot.quantize_tokens(x, 8)
    assert (q[[1, 4]] == 0).all() and np.isinf(s[[1, 4]]).all()
    for act in (0, 1):
        got = B.adapt_int8_linear(a, s_a, dev(w), dev(s_w), act=act, dtype=_t(name))
        same_bits(got, rounded(ot.int8_linear(q, s, w, s_w, None, act), name))
        rows = f64(got)[[1, 4]]
        assert np.isnan(rows).all() if act == 0 else (rows == 0).all()


# ---------------------------------------------------------------------------------------------- streams

def test_every_operator_on_a_stream_given_to_the_call(B):
    """The same results as on the current stream, whose work they wait for by the caller's own event."""
    import torch
    rng = np.random.default_rng(4)
    M, K, N, V = 500, 96, 120, 70
    a, s_a, w, s_w = dev(codes(rng, M, K)), dev(scales(rng, M)), dev(codes(rng, N, K)), dev(scales(rng, N))
    _, x = randn(rng, (M, K), "bf16")
    _, dy = randn(rng, (M, N), "bf16")
    _, table = randn(rng, (V, K), "bf16")
    tok = dev(tokens_of(rng, "zipf", M, V))
    calls = [lambda **k: B.adapt_quantize_tokens(x, **k), lambda **k: (B.adapt_int8_linear(a, s_a, w, s_w, **k),),
             lambda **k: B.adapt_int8_linear_backward(dy, a, s_a, w, s_w, **k), lambda **k: (B.adapt_embedding(table, tok, **k),),
             lambda **k: (B.adapt_embedding_backward(x, tok, V, **k),), lambda **k: (B.adapt_dropout(x, 0.5, 1, **k),), lambda **k: (B.adapt_dropout_backward(x, 0.5, 1, **k),)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(2):
        got = [c(stream=s) for c in calls]
        s.synchronize()
        for g, v in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(g, v))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("V,D", [(1, 1), (5, 7), (1000, 33), (3, 5000)])
def test_embedding_without_places(B, name, V, D):
    """No tokens: no rows, and a gradient of zeros whatever its memory held."""
    import torch
    for dtype in (torch.int32, torch.int64):
        tok = torch.empty(0, dtype=dtype, device="cuda")
        assert B.adapt_embedding(torch.ones((V, D), dtype=_t(name), device="cuda"), tok).shape == (0, D)
        out = torch.full((V + 1, D), float("nan"), dtype=_t(name), device="cuda")
        B.adapt_embedding_backward(torch.empty((0, D), dtype=_t(name), device="cuda"), tok, V, out=out[:V])
        assert (out[:V] == 0).all() and torch.isnan(out[V]).all()
