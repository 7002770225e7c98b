"""What the definitions of the token-wise operators promise beside the values themselves (no GPU: the oracle, which the kernels match bit for bit)."""
import numpy as np
import pytest

from oracle import tokens as ot


@pytest.mark.parametrize("bits", range(2, 9))
def test_token_scales_are_the_quotient_or_the_number_beside_it(bits):
    """max * (1 / Q), for every significand, against max / Q rounded once: the rule for a calibrated range."""
    q_max = np.float32((1 << (bits - 1)) - 1)
    m = (np.arange(1 << 23, dtype=np.uint32) | np.uint32(127 << 23)).view(np.float32)
    # (a row per number, without its codes: the oracle's scale of a row of one element)
    product = ot.quantize_tokens(m[::4099, None], bits)[1]
    assert (product == m[::4099] * (np.float32(1) / q_max)).all()
    apart = np.abs((m * (np.float32(1) / q_max)).view(np.int32) - (m / q_max).view(np.int32))
    assert apart.max() <= 1 and (bits > 2 or apart.max() == 0)


@pytest.mark.parametrize("bits", range(2, 9))
def test_token_codes_are_those_of_the_quotient_or_one_beside(bits):
    """fp16 values, whose quotients meet halves: a code moves by one at most, and only where x / scale is a half to a few units of fp32."""
    rng = np.random.default_rng(bits)
    x = rng.standard_normal((2000, 300)).astype(np.float16).astype(np.float32)
    q, _ = ot.quantize_tokens(x, bits)
    q_max = np.float32((1 << (bits - 1)) - 1)
    s = np.abs(x).max(axis=1) / q_max
    r = x.astype(np.float64) / s[:, None].astype(np.float64)
    want = np.clip(np.rint(x / s[:, None]), -q_max, q_max).astype(np.int8)
    moved = q != want
    assert np.abs(q.astype(int) - want).max() <= 1
    # the scales differ by 2^-23 of themselves at most, each quotient is rounded once: 3 * 2^-24 of up to Q
    assert (np.abs(np.abs(r[moved]) % 1 - 0.5) <= 3 * 2.0 ** -23 * q_max).all()


# ---------------------------------------------------------------------------------------------- the binding

def test_sizes_that_the_library_takes_as_int_are_not_cut():
    """2^32 + 5 rows are not 5 rows.  (Tensors of no elements, so that the sizes are all there is; refused before the device is touched.)"""
    import torch

    from paper_2203_04071_amd import binding as B
    far = (1 << 32) + 5
    q = lambda *s: torch.empty(s, dtype=torch.int8)
    f = torch.empty
    big = "above 2147483647"
    for a, w in ((q(far, 0), q(3, 0)), (q(3, 0), q(far, 0)), (q(0, far), q(0, far)), (q((1 << 31), 0), q(3, 0))):
        M, N = a.shape[0], w.shape[0]
        with pytest.raises(ValueError, match=big):
            B.adapt_int8_linear(a, f(0), w, f(0))
        if not M * N:
            with pytest.raises(ValueError, match=big):
                B.adapt_int8_linear_backward(f(M, N), a, f(0), w, f(0))
    for M, N in ((far, 0), (0, far)):
        with pytest.raises(ValueError, match=big):
            B.adapt_int8_linear_backward(f(M, N), q(M, 0), f(0), q(N, 0), f(0))
    none = torch.empty(0, dtype=torch.int64)
    for V, D in ((far, 0), (0, far)):
        with pytest.raises(ValueError, match=big):
            B.adapt_embedding(f(V, D), none)
        with pytest.raises(ValueError, match=big):
            B.adapt_embedding_backward(f(0, D), none, V)


def test_product_of_too_many_blocks_is_refused_for_that():
    """The limit counts blocks of 64 x 64 outputs: one row of 2^30 channels is refused, as is 2^18 x 2^18, and told so."""
    import ctypes

    from paper_2203_04071_amd import binding as B
    L, p = B.load(), ctypes.c_void_p(256)
    for M, N in ((1, 1 << 30), (64, (1 << 30) - 63), ((1 << 30) - 63, 1), ((1 << 31) - 1, (1 << 31) - 1), (1 << 18, 1 << 18), ((1 << 18) - 63, (1 << 18) - 63)):
        assert L.adapt_int8_linear(p, p, p, p, None, 0, ctypes.c_void_p(512), 0, M, 4, N, None) == -2
        assert "2^24 blocks of 64 x 64 outputs" in L.adapt_last_error().decode()
