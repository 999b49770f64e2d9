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


@pytest.mark.parametrize("T,S", [(2, 40), (16, 9000), (40, 90)])
def test_attention(lib, T, S):
    L, B, H, G, D = 1, 8, 3, 2, 64
    n = lib.ppd_kv4_attention_workspace_bytes(L, B, H, G, T, D, S)
    assert (n > 0) == (S == 9000)

    def call(q=at(0), k=at(1), ks=at(2), v=at(3), vs=at(4), kt=at(5), vt=at(6), prefix=at(7), parent=at(8), L=L, B=B, H=H, G=G, T=T, D=D, S=S, dt=0,
             scale=0.0, out=at(9), lse=at(10), status=at(11), ws=at(12), n=n):
        return lib.ppd_tree_attention_kv4(q, k, ks, v, vs, kt, vt, prefix, parent, L, B, H, G, T, D, S, dt, scale, out, lse, status, ws, n, None)
    inputs = ("k", "ks", "v", "vs", "kt", "vt", "prefix", "parent")
    outs = ("out", "lse", "status")
    pairs = [(o, i) for o in outs for i in inputs] + [(o, "q") for o in outs[1:]] + [("out", "lse"), ("out", "status"), ("lse", "status")]
    refused(call, pairs, *(dict([(x, None)]) for x in ("q", *inputs, "out", "status")),
            *(dict([(x, at(20, 8))]) for x in ("q", "k", "ks", "v", "vs", "kt", "vt", "out")), *(dict([(x, 0)]) for x in "LBHGTDS"), dict(T=513),
            dict(D=80), dict(dt=3), dict(scale=float("nan")), dict(lse=at(20, 2)), dict(out=at(0, 16)), dict(q=at(9, 16)), dict(dt=1, out=at(0)))
    if n:      # a workspace that the call uses
        for p in (*inputs, "q", *outs):
            given = inspect.signature(call).parameters[p].default
            assert call(ws=given) == INVALID, p
        assert call(ws=None, n=0) == CUDA
    assert call(out=at(0)) == CUDA         # a block writes the rows that it alone has read
    assert call(lse=None) == CUDA
    assert call(k=at(1), v=at(1), ks=at(2), vs=at(2)) == CUDA


@pytest.mark.parametrize("kv4", [True, False])
def test_weight_add(lib, kv4):
    def call(q=at(0), lse=at(1), k=at(2), ks=at(3) if kv4 else None, kt=at(4), path=at(5), accept=at(6), prefix=at(7), L=2, B=8, H=3, G=2, T=16, D=64,
             S=40, dt=0, scale=0.0, weight=at(8)):
        return lib.ppd_kv_weight_add(q, lse, k, ks, kt, path, accept, prefix, L, B, H, G, T, D, S, dt, scale, weight, None)
    inputs = ("q", "lse", "k", "kt", "path", "accept", "prefix")
    refused(call, [("weight", i) for i in (*inputs, *(("ks",) if kv4 else ()))], *(dict([(x, None)]) for x in (*inputs, "weight")),
            *(dict([(x, at(20, 8))]) for x in ("q", "k", "ks", "kt")), dict(lse=at(20, 2)), dict(weight=at(20, 2)), *(dict([(x, 0)]) for x in "LBHGTDS"),
            dict(T=513), dict(D=100), dict(dt=7), dict(scale=float("inf")))
    # the whole extent of the cache counts: rows of D / 2 bytes with scales, of 2 D without
    rows = 2 * 8 * 3 * 40
    assert call(weight=at(2, rows * (32 if kv4 else 128) - 16)) == INVALID
    assert call(weight=at(2, rows * (32 if kv4 else 128))) == CUDA
