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


def test_evict(lib):
    def call(budget=4, sink=1, recent=1, S_max=10, S_out=10, planes=(at(0).value, at(1).value), outs=(at(2).value, at(3).value), rows=(16, 3), n=None,
             weight=at(4), out_w=at(5), length=at(6), kept=at(7), new_len=at(8), status=at(9), L=1, B=8, H=2):
        k = len(planes)
        src, dst = (ctypes.c_void_p * k)(*planes), (ctypes.c_void_p * k)(*outs)
        return lib.ppd_kv_evict(weight, out_w, src, dst, (ctypes.c_int * k)(*rows), k if n is None else n, length, L, B, H, S_max, S_out, budget,
                                sink, recent, kept, new_len, status, None)
    p0, p1, o0, o1 = (at(i).value for i in range(4))
    own = ("kept", "new_len", "status")
    refused(call, [(o, i) for o in (*own, "out_w") for i in ("length",)] + [(o, w) for o in own for w in ("weight", "out_w")] +
            [("kept", "new_len"), ("kept", "status"), ("new_len", "status")],
            *(dict([(x, None)]) for x in ("weight", "out_w", "length", *own)), dict(budget=0), dict(budget=11), dict(budget=9, S_out=8), dict(sink=-1),
            dict(recent=-1), dict(sink=3, recent=2), dict(sink=5, recent=0), dict(sink=0, recent=5), dict(rows=(0, 3)), dict(rows=(16, 1025)),
            dict(planes=(None, p1)), dict(outs=(o0, None)), dict(n=-1), dict(L=0), dict(B=0), dict(H=0), dict(S_max=0), dict(S_out=0),
            dict(planes=tuple(at(20 + i).value for i in range(9)), outs=tuple(at(30 + i).value for i in range(9)), rows=(4,) * 9),
            dict(outs=(p0 + 16, o1)),                         # over its own source, not in place
            dict(outs=(p0, o1), S_out=8),                     # in place with another capacity
            dict(out_w=at(4), S_out=8),
            dict(outs=(p1, o1)), dict(outs=(o0, p0)),         # over the other's source
            dict(outs=(o0, o0 + 16)), dict(outs=(o0, at(5).value)), dict(outs=(at(4).value, o1)),   # two destinations; the weights'
            *(dict([(x, ctypes.c_void_p(p))]) for x in own for p in (p0, p1, o0, o1)), dict(outs=(at(6).value, o1)), dict(weight=at(20, 2)),
            dict(out_w=at(20, 2)))
    assert lib.ppd_kv_evict(at(4), at(5), None, None, None, 1, at(6), 1, 8, 2, 10, 10, 4, 1, 1, at(7), at(8), at(9), None) == INVALID
    assert call(planes=(), outs=(), rows=()) == CUDA
    assert call(outs=(p0, p1), out_w=at(4)) == CUDA           # in place
    assert call(outs=(p0, o1)) == CUDA
    assert call(budget=8, S_out=8, sink=8, recent=0) == CUDA
    assert call(rows=(1, 1024)) == CUDA


@pytest.mark.parametrize("drawn", [True, False])
def test_sample(lib, drawn):
    def call(logits=at(0), cand=at(1), parent=at(2), prefix=at(3), probs=at(4) if drawn else None, row=at(5) if drawn else None, u=at(6), noise=at(7),
             B=8, T=4, V=100, n_draft=3, S=10, temp=0.7, accept_len=at(8), path=at(9), nxt=at(10), new_len=at(11), prob=at(12), status=at(13)):
        return lib.ppd_sample_accept(logits, cand, parent, prefix, probs, row, u, noise, B, T, V, n_draft, S, temp, accept_len, path, nxt, new_len, prob,
                                     status, None)
    outs = ("accept_len", "path", "nxt", "new_len", "prob", "status")
    required = ("logits", "cand", "parent", "prefix", "u", "noise", *outs[:4], "status")
    given = {k: v.default for k, v in inspect.signature(call).parameters.items()}
    refused(call, [(a, b) for a in outs for b in outs if a < b], *(dict([(x, None)]) for x in required), dict(B=0), dict(T=0), dict(T=513), dict(V=0),
            dict(S=0), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")), dict(temp=1e-39),
            *(dict([(x, at(20, 2))]) for x in ("logits", "u", "noise", "prob")),
            *((dict(probs=None), dict(row=None), dict(n_draft=0), dict(probs=at(20, 2))) if drawn else (dict(probs=at(4)), dict(row=at(5)))))
    # an output per sequence or per node may take the whole place of an input of that size (a
    # sequence's CTAs have all read it by then), and share no other bytes with what is read
    inputs = ("logits", "cand", "parent", "prefix", "u", "noise", *(("probs", "row") if drawn else ()))
    for o in outs:
        for i in inputs:
            same = (o in ("path", "prob") and i in ("cand", "parent", "row", "u")) or (o not in ("path", "prob") and i == "prefix")
            assert call(**{o: given[i]}) == (CUDA if same else INVALID), (o, i)
            assert call(**{o: shifted(given[i], 16)}) == INVALID, (o, i)
            assert call(**{i: shifted(given[o], 16)}) == INVALID, (o, i)
    assert call(prob=None) == CUDA
    assert call(V=8 * 48 * 1024 + 1) == UNSUPPORTED


def test_capacities_that_counters_cannot_hold(lib):
    """Row numbers are 32-bit, with room for the tiles that pass the last row; a call whose tiles are
    past 32 bits in all takes its units whole."""
    most = 2 ** 31 - 1 - 65536
    ws = lib.ppd_kv4_attention_workspace_bytes
    assert ws(1, 1, 1, 1, 1, 64, most) > 0
    assert ws(1, 1, 1, 1, 1, 64, most + 1) == 0
    assert ws(1, 1, 1, 2, 512, 64, 2 ** 20) > 0
    assert ws(1, 1, 1, 128, 512, 64, most) == 0     # 1024 blocks of rows, 16 million tiles each
    far = [ctypes.c_void_p(i << 44) for i in range(1, 14)]
    for S, want in ((most, CUDA), (most + 1, UNSUPPORTED), (2 ** 31 - 1, UNSUPPORTED)):
        assert lib.ppd_kv4_append(*far[:9], 1, 1, 1, 4, 64, S, 0, far[9], None) == want
        assert lib.ppd_kv4_read(*far[:4], 1, 1, 1, 4, 64, S, far[4], 0, None) == want
        assert lib.ppd_tree_attention_kv4(*far[:9], 1, 1, 1, 1, 4, 64, S, 0, 0.0, far[9], None, far[10], None, 0, None) == want
        assert lib.ppd_kv_weight_add(*far[:8], 1, 1, 1, 1, 4, 64, S, 0, 0.0, far[8], None) == want
        assert lib.ppd_kv_evict(far[0], far[1], None, None, None, 0, far[2], 1, 1, 1, S, 10, 4, 1, 1, far[3], far[4], far[5], None) == want
        assert lib.ppd_kv_evict(far[0], far[1], None, None, None, 0, far[2], 1, 1, 1, 10, S, 4, 1, 1, far[3], far[4], far[5], None) == want
