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


# ---------------------------------------------------------------------------------------------- results that are operands

def test_results_and_workspaces_that_are_operands_or_other_results_are_refused():
    import ctypes

    from paper_2203_04071_amd import binding as B
    L, vp, n = B.load(), ctypes.c_void_p, ctypes.c_size_t()

    def refused(call, good, pairs):
        for a, b in pairs:
            args = dict(good)
            args[a] = args[b]
            assert call(*args.values()) == -1, (a, b)
            text = L.adapt_last_error().decode()
            assert "alias" in text or "in-place" in text or "step" in text, (a, b, text)

    refused(L.adapt_quantize_tokens, dict(x=vp(256), type=0, q=vp(512), scales=vp(768), tokens=4, cols=8, bits=8, stream=None),
            (("q", "x"), ("scales", "x"), ("scales", "q")))
    refused(L.adapt_int8_linear, dict(a=vp(256), s_a=vp(512), w=vp(768), s_w=vp(1024), bias=vp(1280), act=0, y=vp(1536), type=0, M=4, K=8, N=4, stream=None),
            [("y", b) for b in ("a", "s_a", "w", "s_w", "bias")])
    assert L.adapt_int8_linear_backward_workspace(64, 48, 32, 0, 1, 1, ctypes.byref(n)) == 0
    operands, results = ("dy", "a", "s_a", "w", "s_w"), ("dx", "dw", "db")
    refused(L.adapt_int8_linear_backward, dict(dy=vp(256), type=0, a=vp(512), s_a=vp(768), w=vp(1024), s_w=vp(1280), M=64, K=48, N=32, dx=vp(2048),
                                               dw=vp(4096), db=vp(8192), ws=vp(1 << 20), n=n.value, stream=None),
            [(r, o) for r in results + ("ws",) for o in operands] + [("dw", "dx"), ("db", "dx"), ("db", "dw")] + [("ws", r) for r in results])
    refused(L.adapt_embedding, dict(table=vp(256), type=0, tok=vp(512), bits=64, y=vp(1024), T=4, V=8, D=16, scale=1.0, stream=None),
            (("y", "table"), ("y", "tok")))
    assert L.adapt_embedding_backward_workspace(4, 8, 16, ctypes.byref(n)) == 0
    refused(L.adapt_embedding_backward, dict(dy=vp(256), type=0, tok=vp(512), bits=64, out=vp(1024), T=4, V=8, D=16, scale=1.0, pad=-1, ws=vp(4096), n=n.value, stream=None),
            [(r, o) for r in ("out", "ws") for o in ("dy", "tok")] + [("ws", "out")])
    for call in (L.adapt_dropout, L.adapt_dropout_backward):
        refused(call, dict(x=vp(256), y=vp(512), type=0, n=4, p=0.5, seed=1, offset=0, step=vp(1024), stream=None), (("y", "step"),))


def test_a_stream_of_another_device_is_refused():
    from types import SimpleNamespace

    import torch

    from paper_2203_04071_amd import binding as B
    stream = SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=7)
    with pytest.raises(ValueError, match="cuda:1"):
        B._raw_stream(stream, 0)
    assert B._raw_stream(stream, 1) == 7
