"""Every kind of tile of the dense product against the oracle: exact products bit for bit, gradients within the bound of their 22 bits, at the sizes for which
tests/test_tile_plan_host.py shows what kind they take."""
import numpy as np
import pytest

from oracle import tokens as ot
from test_gpu_tokens import TYPES, B, _t, codes, dev, randn, rounded, same_bits, scales  # noqa: F401  (B: the fixture)
from test_gpu_tokens_edges import far_below, within_22_bits
from test_tile_plan_host import APART, JOINT, PRODUCTS

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


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("M,K,N", [*JOINT.values(), *APART.values()])
def test_gradients(B, name, M, K, N):
    """Both gradients, then each alone: the same bits."""
    rng = np.random.default_rng(M + 3 * K + 5 * N)
    a, w, s_a, s_w = codes(rng, M, K), codes(rng, N, K), scales(rng, M), scales(rng, N)
    dy, dyd = randn(rng, (M, N), name)
    operands = (dyd, dev(a), dev(s_a), dev(w), dev(s_w))
    dx, dw, db = B.adapt_int8_linear_backward(*operands)
    (wx, mx), (ww, mw), (wb, mb) = ot.int8_linear_backward(dy, a, s_a, w, s_w)
    within_22_bits(dx, wx, mx, N, name, far_below(dy * s_w, w))
    within_22_bits(dw, ww, mw, M, name, far_below((dy * s_a[:, None]).T, a))
    within_22_bits(db, wb, mb, M, name, 0.0)
    same_bits(B.adapt_int8_linear_backward(*operands, want=("dx",))[0], dx.cpu())
    same_bits(B.adapt_int8_linear_backward(*operands, want=("dw", "db"))[1], dw.cpu())
