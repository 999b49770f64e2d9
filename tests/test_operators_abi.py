"""Refusals of the operators for sampled decoding over a 4-bit cache: on the host, before
any device work (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2405_18628_gb300 import build, ppd
    build.build()
    return ppd.load()


F, ODD = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100008)   # never dereferenced
S, INVALID, UNSUPPORTED = ctypes.c_void_p(0), 1, 2


def _refused(fn, args, changes, want=INVALID):
    """Each change (argument index -> value) alone is refused."""
    for i, v in changes:
        a = list(args)
        a[i] = v
        assert fn(*a) == want, (i, v)


def test_append(lib):
    #        0..9 pointers  L  B  H  T  D  S  dt
    args = [F] * 9 + [1, 1, 1, 4, 64, 10, 0, F, S]
    _refused(lib.ppd_kv4_append, args, [(i, None) for i in (0, 1, 2, 3, 4, 5, 7, 8, 16)] + [(i, ODD) for i in range(6)] +
             [(9, 0), (10, 0), (11, -1), (12, 0), (13, 32), (13, 96), (14, 0), (15, 2)])


def test_read(lib):
    args = [F] * 4 + [1, 1, 1, 4, 64, 10, F, 0, S]
    _refused(lib.ppd_kv4_read, args, [(i, None) for i in (0, 1, 2, 3, 10)] + [(i, ODD) for i in (0, 1, 10)] +
             [(4, 0), (5, 0), (6, 0), (7, 0), (8, 256), (9, 0), (11, 5)])


def test_attention(lib):
    #       pointers     L  B  H  G  T  D  S  dt scale out lse st ws  n
    args = [F] * 9 + [1, 1, 1, 1, 4, 64, 10, 0, 0.0, F, None, F, None, 0, S]
    _refused(lib.ppd_tree_attention_kv4, args, [(i, None) for i in (*range(9), 18, 20)] + [(i, ODD) for i in (*range(7), 18)] +
             [(19, ctypes.c_void_p(0x100002))] + [(i, 0) for i in range(9, 14)] + [(13, 513), (14, 80), (15, 0), (16, 3), (17, float("nan"))])
    assert lib.ppd_kv4_attention_workspace_bytes(1, 1, 1, 1, 600, 64, 10) == 0
    assert lib.ppd_kv4_attention_workspace_bytes(1, 1, 1, 1, 1, 96, 10) == 0
    assert lib.ppd_kv4_attention_workspace_bytes(1, 1, 2, 1, 1, 128, 100000) > 0


def test_weight_add(lib):
    args = [F] * 8 + [1, 1, 1, 1, 4, 64, 10, 0, 0.0, F, S]
    _refused(lib.ppd_kv_weight_add, args, [(i, None) for i in (0, 1, 2, 4, 5, 6, 7, 17)] + [(i, ODD) for i in (0, 2, 3, 4)] +
             [(i, 0) for i in range(8, 13)] + [(12, 513), (13, 100), (14, 0), (15, 7), (16, float("inf"))])


def test_evict(lib):
    def call(budget=4, sink=1, recent=1, S_max=10, S_out=10, planes=(0x1000000,), outs=(0x2000000,), rows=(16,), n=None, weight=F, out_w=F,
             L=1, length=F, kept=F, new_len=F, status=F):
        k = len(planes)
        src, dst = (ctypes.c_void_p * k)(*planes), (ctypes.c_void_p * k)(*outs)
        return lib.ppd_kv_evict(weight, out_w, src, dst, (ctypes.c_int * k)(*rows), k if n is None else n, length, L, 1, 1, S_max, S_out, budget,
                                sink, recent, kept, new_len, status, S)
    for bad in (dict(budget=0), dict(budget=11), dict(S_out=3), dict(sink=-1), dict(recent=-1), dict(sink=3, recent=2), dict(sink=5, recent=0),
                dict(rows=(0,)), dict(rows=(1025,)), dict(planes=(None,)), dict(outs=(None,)), dict(n=-1), dict(n=9), dict(weight=None), dict(out_w=None),
                dict(length=None), dict(kept=None), dict(new_len=None), dict(status=None), dict(L=0),
                dict(outs=(0x1000010,)),                               # over its own source, not in place
                dict(S_out=8),                                         # weights in place with another capacity
                dict(planes=(0x1000000, 0x3000000), outs=(0x2000000, 0x1000000), rows=(16, 16)),   # over the other's source
                dict(planes=(0x1000000, 0x3000000), outs=(0x2000000, 0x2000010), rows=(16, 16))):
        assert call(**bad) == INVALID, bad
    assert lib.ppd_kv_evict(F, F, None, None, None, 1, F, 1, 1, 1, 10, 10, 4, 1, 1, F, F, F, S) == INVALID


def test_evict_over_its_own_lengths(lib):
    """Every block reads the lengths: an output over them would race."""
    at = [ctypes.c_void_p(0x1000000 * (i + 1)) for i in range(5)]
    weight, length, kept, new_len, status = at
    for over in (dict(new_len=length), dict(status=length), dict(kept=length), dict(kept=ctypes.c_void_p(length.value - 8)),
                 dict(new_len=ctypes.c_void_p(length.value + 4))):
        a = dict(kept=kept, new_len=new_len, status=status) | over
        assert lib.ppd_kv_evict(weight, weight, None, None, None, 0, length, 1, 2, 1, 10, 10, 4, 1, 1, a["kept"], a["new_len"], a["status"],
                                S) == INVALID, over


def test_sample(lib):
    #       logits cand parent prefix probs row  u  noise B T V nd S temp  outputs ...
    args = [F] * 4 + [None, None] + [F] * 2 + [1, 4, 100, 0, 10, 0.7] + [F] * 7
    args[-1] = S
    _refused(lib.ppd_sample_accept, args, [(i, None) for i in (0, 1, 2, 3, 6, 7, 14, 15, 16, 17, 19)] + [(4, F), (5, F)] +
             [(8, 0), (9, 0), (9, 513), (10, 0), (12, 0), (13, 0.0), (13, -1.0), (13, float("nan")), (13, 1e-39), (0, ctypes.c_void_p(0x100002))])
    both = list(args)
    both[4] = both[5] = F
    _refused(lib.ppd_sample_accept, both, [(11, 0)])
    _refused(lib.ppd_sample_accept, args, [(10, 8 * 48 * 1024 + 1)], UNSUPPORTED)


def test_the_binding_names_what_is_wrong():
    from paper_2405_18628_gb300 import ppd
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    c, s = ppd.kv4_cache(1, 1, 2, 8, 64, "cpu")
    att = lambda **k: ppd.ppd_tree_attention_kv4(**{**dict(  # noqa: E731
        q=z(1, 1, 4, 3, 64), k_cache=c, k_scale=s, v_cache=c, v_scale=s, k_tree=z(1, 1, 2, 3, 64), v_tree=z(1, 1, 2, 3, 64), prefix_len=i(1), parent=i(1, 3),
        out=z(1, 1, 4, 3, 64), dev_status=i(1)), **k})
    with pytest.raises(ValueError, match="CUDA"):
        att()
    for bad, err in ((dict(q=z(1, 1, 3, 3, 64)), ValueError), (dict(out=z(1, 1, 4, 3, 64, dt=torch.float32)), TypeError),
                     (dict(k_scale=s[..., :1]), ValueError), (dict(k_tree=z(1, 1, 2, 3, 64, dt=torch.float32)), TypeError),
                     (dict(parent=z(1, 3, dt=torch.int64)), TypeError), (dict(parent=i(1, 4)), ValueError), (dict(k_cache=c.to(torch.int8)), TypeError),
                     (dict(q=z(1, 1, 4, 3, 64, dt=torch.float16)), TypeError)):
        with pytest.raises(err):
            att(**bad)
    with pytest.raises(ValueError, match="together"):
        ppd.ppd_kv_evict(z(1, 1, 1, 8, dt=torch.float32), [], i(1), 4, 0, 0, i(1, 1, 1, 4), i(1), i(1), out_planes=[])
    with pytest.raises(ValueError, match="noise"):
        ppd.ppd_sample_accept(z(1, 2, 9, dt=torch.float32), i(1, 2), i(1, 2), i(1), 10, 1.0, z(1, 2, dt=torch.float32), z(1, 8, dt=torch.float32), i(1), i(1, 2), i(1), i(1), i(1))
