"""Every kind of tile of the dense product against the oracle: exact products bit for bit, at the sizes for which
tests/test_tile_plan_host.py shows what kind they take."""
import numpy as np
import pytest

from oracle import tokens as ot
from test_gpu_tokens import TYPES, B, _t, codes, dev, rounded, same_bits, scales  # noqa: F401  (B: the fixture)
from test_tile_plan_host import PRODUCTS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def same_device(B):
    assert B.load().adapt_device_cu_count() == 256, "the sizes were chosen for 256 compute units"


@pytest.mark.parametrize("M,K,N", [s for sizes in PRODUCTS.values() for s in sizes])
def test_exact_product(B, M, K, N):
    rng = np.random.default_rng(M + K + N)
    a, w, s_a, s_w = codes(rng, M, K), codes(rng, N, K), scales(rng, M), scales(rng, N)
    bias = rng.standard_normal(N).astype(np.float32)
    want = ot.int8_linear(a, s_a, w, s_w, bias, 1)
    for name in TYPES:
        same_bits(B.adapt_int8_linear(dev(a), dev(s_a), dev(w), dev(s_w), bias=dev(bias), act=1, dtype=_t(name)), rounded(want, name))
