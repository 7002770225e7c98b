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
