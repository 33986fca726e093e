"""CPU checks of the 8-bit entry points: what they refuse, with the documented codes, before a GPU is touched."""
import ctypes as C

import pytest

from paper_2603_05959_b200 import binding as B
from paper_2603_05959_b200 import build as build_mod

BAD, MISALIGNED, UNSUPPORTED = -1, -5, -10
P = 4096                                                 # (an aligned address that is never read)


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.lib()


def _call(f, names, defaults, **over):
    args = dict(defaults, **over)
    return f(*[args[n] for n in names])


NORM = dict(x=P, residual=P, weight=P, bias=P, rows=0, C=64, dtype=1, kind=2, eps=1e-6, sum=P, q=P, scale=P, stream=None)


def test_norm(lib):
    call = lambda **o: _call(lib.ovggt_k_norm_q8, list(NORM), NORM, **o)
    assert call() == 0                                   # no rows: nothing to do
    for over in (dict(x=None), dict(q=None), dict(scale=None), dict(rows=-1), dict(C=0), dict(dtype=2), dict(kind=3), dict(kind=-1),
                 dict(residual=None), dict(kind=0), dict(kind=0, weight=None), dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(**dict(dict(rows=1), **over)) == BAD, over
    for over in (dict(C=24), dict(C=16400)):
        assert call(rows=1, **over) == UNSUPPORTED, over
    for name in ("x", "residual", "weight", "bias", "sum", "q"):
        assert call(rows=1, **{name: P + 8}) == MISALIGNED, name
    assert call(rows=1, scale=P + 2) == MISALIGNED


LINEAR = dict(A=P, a_scale=P, W=P, w_scale=P, M=16, N=24, K=64, outs=(C.c_void_p * 3)(P, P, P), n_outs=3, gelu=0, residual=P, sum=P,
              status=P, stream=None)


def test_linear(lib):
    call = lambda **o: _call(lib.ovggt_k_linear_q8, list(LINEAR), LINEAR, **o)
    assert call(M=0) == 0
    for over in (dict(A=None), dict(a_scale=None), dict(W=None), dict(w_scale=None), dict(status=None), dict(M=-1), dict(N=0), dict(K=0),
                 dict(n_outs=4), dict(n_outs=-1), dict(outs=None), dict(residual=None), dict(sum=None), dict(n_outs=0, residual=None, sum=None),
                 dict(outs=(C.c_void_p * 3)(P, None, P))):
        assert call(**over) == BAD, over
    for over in (dict(K=72), dict(N=28, n_outs=1), dict(N=32), dict(n_outs=2), dict(K=131072), dict(M=0x7FFFFF01), dict(N=0x7FFFFFF8, n_outs=1)):
        assert call(**over) == UNSUPPORTED, over
    for name in ("A", "W", "w_scale", "residual", "sum"):
        assert call(**{name: P + 8}) == MISALIGNED, name
    assert call(a_scale=P + 2) == MISALIGNED
    assert call(outs=(C.c_void_p * 3)(P, P, P + 8)) == MISALIGNED


STORE = dict(k=P, v=P, n_seqs=2, M=3, n_heads=4, dtype=1, start=P, capacity=32, kq=P, kx=P, vq=P, vx=P, stream=None)
LOAD = dict(kq=P, kx=P, vq=P, vx=P, n_seqs=2, n_heads=4, capacity=32, first=0, n=32, dtype=0, k=P, v=P, stream=None)


def test_store_and_load(lib):
    store = lambda **o: _call(lib.ovggt_k_store_q8, list(STORE), STORE, **o)
    load = lambda **o: _call(lib.ovggt_k_load_q8, list(LOAD), LOAD, **o)
    assert store(M=0) == store(n_seqs=0) == load(n=0) == load(n_seqs=0) == 0
    for f, names in ((store, ("k", "v", "kq", "kx", "vq", "vx")), (load, ("kq", "kx", "vq", "vx", "k", "v"))):
        for name in names:
            assert f(**{name: None}) == BAD and f(**{name: P + 8}) == MISALIGNED, name
        for over in (dict(n_seqs=-1), dict(n_heads=0), dict(capacity=0), dict(dtype=2)):
            assert f(**over) == BAD, over
        assert f(capacity=40) == UNSUPPORTED
    assert store(M=-1) == load(n=-1) == load(first=-1) == load(first=1) == BAD
    assert store(start=P + 2) == MISALIGNED


ATTEND = dict(q=P, kq=P, kx=P, vq=P, vx=P, n_seqs=2, M=3, n_heads=8, n_kv_heads=4, capacity=32, lens=P, live=P, out=P, scratch=P, status=P, stream=None)


def test_attention(lib):
    call = lambda **o: _call(lib.ovggt_k_attention_q8, list(ATTEND), ATTEND, **o)
    assert call(M=0) == call(n_seqs=0) == 0
    for name in ("q", "kq", "kx", "vq", "vx", "out", "scratch", "status"):
        assert call(**{name: None}) == BAD, name
    for over in (dict(n_seqs=-1), dict(M=-1), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=6), dict(capacity=0)):
        assert call(**over) == BAD, over
    for over in (dict(capacity=40), dict(M=1 << 30), dict(n_seqs=1 << 20, capacity=1 << 12)):
        assert call(**over) == UNSUPPORTED, over
    for name in ("q", "kq", "kx", "vq", "vx", "live", "out", "scratch"):
        assert call(**{name: P + 8}) == MISALIGNED, name
    assert call(lens=P + 2) == call(status=P + 2) == MISALIGNED


def test_attention_scratch(lib):
    f = lib.ovggt_k_attention_q8_scratch_bytes
    assert f(1, 1, 4, 4, 16) > 0                         # (a CTA takes it all: nothing to keep, but something to point to)
    assert f(1, 1374, 16, 16, 17760) >= 2 * 17760 * 1024 * 2                      # both planes
    assert f(64, 300, 16, 16, 17760) < 2 * f(1, 300, 16, 16, 17760)               # a few sequences at a time
    for bad in ((0, 1, 4, 4, 16), (1, 0, 4, 4, 16), (1, 1, 0, 4, 16), (1, 1, 4, 0, 16), (1, 1, 6, 4, 16), (1, 1, 4, 4, 24), (1, 1, 4, 4, 0), (1, 1 << 30, 4, 4, 16)):
        assert f(*bad) == 0, bad
