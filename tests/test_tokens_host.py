"""Token-wise operators without a GPU: refusals before the device is touched, pins of the oracle, workspace sizes."""
import ctypes

import numpy as np
import pytest

from oracle import tokens as ot

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_2203_04071_amd import binding
    return binding.load()


def _text(lib):
    return lib.adapt_last_error().decode()


def test_quantize_tokens_refusals(lib):
    call = lib.adapt_quantize_tokens
    good = [vp(64), 0, vp(128), vp(192), 4, 8, 8, None]

    def bad(at, v):
        args = list(good)
        args[at] = v
        return call(*args)
    for at in (0, 2, 3):
        assert bad(at, None) == -1 and "NULL" in _text(lib)
    assert bad(1, 3) == -1 and "type" in _text(lib)
    assert bad(6, 1) == -1 and bad(6, 9) == -1
    assert bad(0, vp(66)) == -1 and "aligned" in _text(lib)
    assert bad(3, vp(194)) == -1
    assert bad(2, vp(64)) == -1 and "in-place" in _text(lib)
    assert call(None, 0, None, None, 0, 8, 8, None) == 0            # no tokens: nothing to do


def test_int8_linear_refusals(lib):
    good = [vp(64), vp(64), vp(64), vp(64), None, 0, vp(256), 0, 4, 8, 4, None]

    def bad(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return lib.adapt_int8_linear(*args)
    for at in ("_0", "_1", "_2", "_3", "_6"):
        assert bad(**{at: None}) == -1 and "NULL" in _text(lib)
    assert bad(_5=3) == -1 and bad(_5=-1) == -1
    assert bad(_7=7) == -1 and "type" in _text(lib)
    assert bad(_8=-1) == -1 and bad(_9=-1) == -1 and bad(_10=-1) == -1
    assert bad(_1=vp(66)) == -1 and bad(_3=vp(66)) == -1 and bad(_4=vp(66)) == -1 and bad(_6=vp(258)) == -1
    assert bad(_9=131072) == -2 and "32 bits" in _text(lib)
    assert bad(_8=1 << 20, _10=1 << 20) == -2
    assert bad(_8=0, _6=None) == 0 and bad(_10=0, _6=None) == 0


def test_int8_linear_backward_refusals(lib):
    n = ctypes.c_size_t(1)
    assert lib.adapt_int8_linear_backward_workspace(4, 4, 4, 0, 1, 1, None) == -1
    assert lib.adapt_int8_linear_backward_workspace(-4, 4, 4, 0, 1, 1, ctypes.byref(n)) == -1 and n.value == 0
    assert lib.adapt_int8_linear_backward_workspace(4, 4, 4, 5, 1, 1, ctypes.byref(n)) == -1
    for sizes in (((1 << 21) + 1, 4, 4), (4, (1 << 21) + 1, 4), (4, 4, (1 << 21) + 1), (1 << 20, 1 << 16, 4), (4, 1 << 16, 1 << 20), (1 << 20, 4, 1 << 16)):
        assert lib.adapt_int8_linear_backward_workspace(*sizes, 0, 1, 1, ctypes.byref(n)) == -2 and n.value == 0
    assert lib.adapt_int8_linear_backward_workspace(64, 48, 32, 0, 1, 1, ctypes.byref(n)) == 0
    need = n.value
    good = dict(dy=vp(256), type=0, a=vp(512), s_a=vp(768), w=vp(1024), s_w=vp(1280), M=64, K=48, N=32, dx=vp(2048), dw=vp(4096), db=vp(8192),
                ws=vp(1 << 20), n=need, stream=None)

    def bad(**k):
        return lib.adapt_int8_linear_backward(*{**good, **k}.values())
    for k in ("dy", "a", "s_a", "w", "s_w"):
        assert bad(**{k: None}) == -1 and "NULL" in _text(lib)
    assert bad(type=9) == -1 and bad(M=-1) == -1 and bad(K=-1) == -1 and bad(N=-1) == -1
    assert bad(dy=vp(258)) == -1 and bad(dx=vp(2050)) == -1 and bad(s_a=vp(770)) == -1 and bad(s_w=vp(1282)) == -1
    for k in ("dx", "dw", "db"):
        assert bad(**{k: vp(256)}) == -1 and "alias" in _text(lib)
    assert bad(dx=vp(1024)) == -1 and bad(dw=vp(512)) == -1
    if need:
        assert bad(n=need - 1) == -1 and "workspace" in _text(lib)
        assert bad(ws=None) == -1 and bad(ws=vp((1 << 20) + 128)) == -1
    assert bad(dx=None, dw=None, db=None) == 0                      # nothing wanted
    assert bad(dx=None, dw=None, N=0) == 0


def test_embedding_refusals(lib):
    good = dict(table=vp(256), type=0, tok=vp(512), bits=64, y=vp(1024), T=4, V=8, D=16, scale=1.0, stream=None)

    def bad(**k):
        return lib.adapt_embedding(*{**good, **k}.values())
    for k in ("table", "tok", "y"):
        assert bad(**{k: None}) == -1 and "NULL" in _text(lib)
    assert bad(type=3) == -1 and bad(bits=16) == -1 and bad(V=-1) == -1 and bad(D=-1) == -1
    assert bad(table=vp(257)) == -1 and bad(tok=vp(516)) == -1 and bad(y=vp(1026)) == -1
    assert bad(y=vp(256)) == -1 and "in-place" in _text(lib)
    assert bad(T=1 << 31) == -2
    assert bad(T=0, tok=None, y=None) == 0 and bad(D=0, table=None, y=None) == 0

    n = ctypes.c_size_t(1)
    assert lib.adapt_embedding_backward_workspace(4, 8, 16, None) == -1
    assert lib.adapt_embedding_backward_workspace(4, -8, 16, ctypes.byref(n)) == -1 and n.value == 0
    assert lib.adapt_embedding_backward_workspace(1 << 31, 8, 16, ctypes.byref(n)) == -2
    assert lib.adapt_embedding_backward_workspace(4, 8, (1 << 21) + 1, ctypes.byref(n)) == -2 and n.value == 0
    assert lib.adapt_embedding_backward_workspace(4, 8, 16, ctypes.byref(n)) == 0
    need = n.value
    assert need > 0
    good = dict(dy=vp(256), type=0, tok=vp(512), bits=64, out=vp(1024), T=4, V=8, D=16, scale=1.0, pad=-1, ws=vp(4096), n=need, stream=None)

    def bad(**k):
        return lib.adapt_embedding_backward(*{**good, **k}.values())
    for k in ("dy", "tok", "out", "ws"):
        assert bad(**{k: None}) == -1
    assert bad(type=3) == -1 and bad(bits=8) == -1 and bad(V=-1) == -1 and bad(D=-1) == -1
    assert bad(dy=vp(258)) == -1 and bad(tok=vp(516)) == -1 and bad(out=vp(1026)) == -1 and bad(ws=vp(4097)) == -1
    assert bad(n=need - 1) == -1 and "workspace" in _text(lib)
    assert bad(out=vp(256)) == -1 and "alias" in _text(lib)
    assert bad(T=1 << 31) == -2 and bad(D=(1 << 21) + 1) == -2
    assert bad(V=0, out=None) == 0 and bad(D=0, out=None) == 0


@pytest.mark.parametrize("name", ["adapt_dropout", "adapt_dropout_backward"])
def test_dropout_refusals(lib, name):
    good = dict(x=vp(64), y=vp(128), type=0, n=4, p=0.5, seed=1, offset=0, step=None, stream=None)

    def bad(**k):
        return getattr(lib, name)(*{**good, **k}.values())
    assert bad(x=None) == -1 and bad(y=None) == -1 and bad(type=-1) == -1
    assert bad(p=-0.1) == -1 and bad(p=1.1) == -1 and bad(p=float("nan")) == -1
    assert bad(x=vp(66)) == -1 and bad(y=vp(129)) == -1 and bad(step=vp(4)) == -1
    assert bad(n=0, x=None, y=None) == 0


def test_workspaces_grow_with_the_call(lib):
    """A workspace made for the largest call serves smaller ones of the same table or layer."""
    n = ctypes.c_size_t()

    def emb(T, V, D):
        assert lib.adapt_embedding_backward_workspace(T, V, D, ctypes.byref(n)) == 0
        return n.value
    for V, D in ((1, 1), (511, 16), (512, 33), (50000, 1024), (1 << 30, 8)):
        sizes = [emb(T, V, D) for T in (0, 1, 31, 32, 33, 2047, 2048, 2049, 65536, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[-1] > sizes[0]


def test_int8_linear_backward_workspace_for_both_is_enough_for_one(lib):
    n = ctypes.c_size_t()

    def need(M, K, N, t, dx, dw):
        assert lib.adapt_int8_linear_backward_workspace(M, K, N, t, dx, dw, ctypes.byref(n)) == 0
        return n.value
    sizes = (0, 1, 63, 64, 700, 6400, 100000, 1 << 21)
    for M in sizes:
        for K in (0, 1, 20, 512, 4096):
            for N in sizes:
                if M * N < 1 << 34 and M * K < 1 << 34 and N * K < 1 << 34:
                    for t in (0, 1, 2):
                        both, dx, dw, db = (need(M, K, N, t, x, w) for x, w in ((1, 1), (1, 0), (0, 1), (0, 0)))
                        assert both == dx + dw - db >= max(dx, dw) and db > 0 or not N


# ---- the oracle itself

def test_philox_known_answers():
    """The generator's published known answers (ten rounds)."""
    u = np.uint32
    for ctr, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in ot.philox4x32(np.array(ctr, u), key)) == want


def test_dropout_keeps_its_share():
    kept = ot.dropout_kept(1 << 20, 0.3, 11, 5)
    assert abs(kept.mean() - 0.7) < 5 * (0.21 / (1 << 20)) ** 0.5
    assert (ot.dropout_kept(1000, 0.3, 11, 5, first=333) == kept[333:1333]).all()
    assert ot.dropout_kept(100, 0.0, 1, 1).all() and not ot.dropout_kept(100, 1.0, 1, 1).any()


def test_oracle_product_is_the_exact_table():
    """The same integers as the table of the exact multiplier through the C oracle."""
    import oracle as orc
    from paper_2203_04071_amd import workloads as wl
    rng = np.random.default_rng(3)
    a, w = rng.integers(-128, 128, (9, 37), dtype=np.int8), rng.integers(-128, 128, (11, 37), dtype=np.int8)
    assert (ot.int8_sums(a, w) == orc.approx_linear(wl.exact_lut(8), 8, a, w)).all()


def test_oracle_gradients_against_differences():
    """The forward map is linear in the real operands x = a s_a and v = w s_w: differences of sum(dy * y) are exact up to fp64."""
    rng = np.random.default_rng(4)
    M, K, N = 5, 7, 6
    a, w = rng.integers(-127, 128, (M, K), dtype=np.int8), rng.integers(-127, 128, (N, K), dtype=np.int8)
    s_a, s_w = rng.uniform(0.01, 0.1, M).astype(np.float32), rng.uniform(0.01, 0.1, N).astype(np.float32)
    dy = rng.standard_normal((M, N))
    (dx, _), (dw, _), (db, _) = ot.int8_linear_backward(dy, a, s_a, w, s_w)
    x, v, b = a * s_a.astype(np.float64)[:, None], w * s_w.astype(np.float64)[:, None], np.zeros(N)

    def loss(x, v, b):
        return (dy * (x @ v.T + b)).sum()
    for t, g in ((x, dx), (v, dw), (b, db)):
        for i in np.ndindex(t.shape):
            keep = t[i]
            t[i] = keep + 0.5
            up = loss(x, v, b)
            t[i] = keep - 0.5
            assert abs(up - loss(x, v, b) - g[i]) < 1e-10
            t[i] = keep
    table, tok = rng.standard_normal((9, 4)).astype(np.float32), np.array([3, 0, 3, -1, 9, 8, 3])
    dy = rng.standard_normal((7, 4))
    g, _, n = ot.embedding_backward(dy, tok, 9, 2.0, padding_idx=0)
    assert n.tolist() == [0, 0, 0, 3, 0, 0, 0, 0, 1]
    for i in np.ndindex(table.shape):
        one = np.zeros_like(table)
        one[i] = 1
        want = (dy * ot.embedding(one, tok, 2.0)).sum() if i[0] != 0 else 0.0
        assert abs(g[i] - want) < 1e-12
