"""Refusals of the operators for sampled decoding over a 4-bit cache, one at a time: every
pointer has memory of its own, so that a call passes the host's checks (without a GPU it then
fails with a CUDA error) but for the one change that is refused.  Nothing is dereferenced."""
import ctypes
import inspect

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that pass would run, on addresses of nothing")

INVALID, UNSUPPORTED, CUDA = 1, 2, 5


@pytest.fixture(scope="module")
def lib():
    from paper_2405_18628_gb300 import build, ppd
    build.build()
    return ppd.load()


def at(i, offset=0):
    """The i-th piece of 16 GB of addresses."""
    return ctypes.c_void_p((i + 1 << 34) + offset)


def shifted(p, n):
    return ctypes.c_void_p(p.value + n)


def refused(call, same_place, *changes):
    """The call as it is passes; with each change it is refused.  same_place: pairs (output,
    memory it may not share), tried at the same address and one word into each other."""
    assert call() == CUDA
    given = {k: v.default for k, v in inspect.signature(call).parameters.items()}
    for change in changes:
        assert call(**change) == INVALID, change
    for out, other in same_place:
        for p in (given[other], shifted(given[other], 16)):
            assert call(**{out: p}) == INVALID, (out, other)
        assert call(**{other: shifted(given[out], 16)}) == INVALID, (out, other)


def test_append(lib):
    def call(k_new=at(0), v_new=at(1), k=at(2), ks=at(3), v=at(4), vs=at(5), rows=at(6), start=at(7), n=at(8), L=2, B=8, H=3, T=16, D=64, S=40, dt=0,
             status=at(9)):
        return lib.ppd_kv4_append(k_new, v_new, k, ks, v, vs, rows, start, n, L, B, H, T, D, S, dt, status, None)
    # blocks write rows and statuses while others read where rows go and which they are
    outs = ("k", "ks", "v", "vs", "status")
    pairs = [(o, i) for o in outs for i in ("k_new", "v_new", "rows", "start", "n")]
    pairs += [(a, b) for a in outs for b in outs if a < b]
    refused(call, pairs, *(dict([(x, None)]) for x in ("k_new", "v_new", *outs, "start", "n")),
            *(dict([(x, at(20, 8))]) for x in ("k_new", "v_new", "k", "ks", "v", "vs")), dict(L=0), dict(B=0), dict(H=-1), dict(T=0), dict(D=32),
            dict(D=96), dict(S=0), dict(dt=2))
    assert call(rows=None) == CUDA
    assert call(k_new=at(0), v_new=at(0)) == CUDA      # the same rows as K and V are read alone


@pytest.mark.parametrize("dt", [0, 1])
def test_read(lib, dt):
    def call(cache=at(0), scale=at(1), start=at(2), n=at(3), L=2, B=8, H=3, N=16, D=64, S=40, out=at(4), dt=dt):
        return lib.ppd_kv4_read(cache, scale, start, n, L, B, H, N, D, S, out, dt, None)
    refused(call, [("out", i) for i in ("cache", "scale", "start", "n")], *(dict([(x, None)]) for x in ("cache", "scale", "start", "n", "out")),
            *(dict([(x, at(20, 8))]) for x in ("cache", "scale", "out")), dict(L=0), dict(B=0), dict(H=0), dict(N=0), dict(D=256), dict(S=0), dict(dt=5))
