"""Refusals of the operators over a pool of pages, one at a time (no GPU needed): every
pointer has memory of its own, so that a call passes the host's checks (without a GPU it then fails
with a CUDA error) but for the one change that is refused.  Nothing is dereferenced."""
import ctypes
import inspect

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that pass would run, on addresses of nothing")

INVALID, UNSUPPORTED, CUDA = 1, 2, 5
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2405_18628_gb300 import build, ppd
    build.build()
    return ppd.load()


def at(i, offset=0):
    """The i-th piece of 16 GB of addresses."""
    return ctypes.c_void_p((i + 1 << 34) + offset)


def refused(call, apart, invalid, unsupported=(), fine=()):
    given = {k: v.default for k, v in inspect.signature(call).parameters.items()}
    assert call() == CUDA
    for change in fine:
        assert call(**change) == CUDA, change
    for want, changes in ((INVALID, invalid), (UNSUPPORTED, unsupported)):
        for change in changes:
            assert call(**change) == want, change
    for a, b in apart:
        for p in (given[b], ctypes.c_void_p(given[b].value + 4)):
            assert call(**{a: p}) == INVALID, (a, b)


def test_assign(lib):
    def call(old=at(0), new=at(1), B=4, page=16, n_pages=40, max_pages=9, max_slots=100, table=at(2), free=at(3), n_free=at(4), new_n_free=at(5),
             out_len=at(6), slots=at(7), start=at(8), status=at(9)):
        return lib.ppd_page_assign(old, new, B, page, n_pages, max_pages, max_slots, table, free, n_free, new_n_free, out_len, slots, start, status, None)
    outs, ins = ("table", "free", "out_len", "slots", "start", "status"), ("old", "new")
    refused(call, [(o, i) for o in outs for i in ins] + [(a, b) for a in outs for b in outs if a < b],
            [{x: None} for x in (*outs, *ins, "n_free", "new_n_free")] + [{x: 0} for x in ("B", "page", "n_pages", "max_pages", "max_slots")] +
            [dict(new_n_free=at(4)), dict(new_n_free=at(0)), dict(out_len=at(4)), dict(start=at(6, -16)), dict(free=at(2, 4 * 9 * 4 - 4))],
            [dict(page=x) for x in (1, 4, 12, 24, 512)] + [dict(B=8193), dict(max_slots=2 ** 31 - 1), dict(max_pages=2 ** 28), dict(n_pages=2 ** 28)],
            [dict(page=x) for x in (8, 32, 64, 128, 256)] + [dict(B=8192), dict(free=at(2, 4 * 9 * 4)), dict(slots=at(7, 4))])


def test_append(lib):
    def call(k_new=at(0), v_new=at(1), k=at(2), v=at(3), rows=at(4), slots=at(5), start=at(6), L=2, B=3, H=2, T=9, D=64, page=16, n_pages=7, max_slots=50,
             dt=0, status=at(7)):
        return lib.ppd_page_append(k_new, v_new, k, v, rows, slots, start, L, B, H, T, D, page, n_pages, max_slots, dt, status, None)
    ins, outs = ("k_new", "v_new", "rows", "slots", "start"), ("status",)
    pool = 2 * 7 * 2 * 16 * 64 * 2
    refused(call, [("status", i) for i in (*ins, "k", "v")],
            [{x: None} for x in (*(i for i in ins if i != "rows"), "k", "v", "status")] + [{x: at(20, 8)} for x in ("k_new", "v_new", "k", "v")] +
            [{x: 0} for x in ("L", "B", "H", "T", "page", "n_pages", "max_slots")] + [dict(D=96), dict(dt=2), dict(v=at(2)), dict(v=at(2, pool - 16))] +
            [{o: at(i, 16)} for o in ("k", "v") for i in (0, 1, 4, 5)] + [dict(k=at(6)), dict(v=at(6))] + [{i: at(2, pool - 16)} for i in ins] + [dict(n_pages=2 ** 27, page=32)],
            [dict(page=12), dict(page=512, n_pages=2), dict(L=2 ** 15, B=2 ** 15, T=512, k_new=at(2 ** 20), v_new=at(2 ** 21), n_pages=1, k=at(100), v=at(200),
                                                            rows=None, slots=at(300), start=at(400), status=at(500))],
            [dict(rows=None), dict(v=at(2, pool)), dict(v_new=at(0)), dict(dt=1), dict(D=128, page=8)])


@pytest.mark.parametrize("T,M,dt", [(1, 5, 0), (9, 3000, 0), (9, 5, 1), (200, 40, 1)])
def test_attention(lib, T, M, dt):
    L, B, H, G, D, page, N = 1, 6, 3, 2, 64, 16, 90
    n = lib.ppd_paged_attention_workspace_bytes(L, B, H, G, T, D, M * page, dt)
    assert (n > 0) == (dt == 1 or M == 3000)

    def call(q=at(0), k=at(1), v=at(2), table=at(3), kt=at(4), vt=at(5), prefix=at(6), parent=at(7), L=L, B=B, H=H, G=G, T=T, D=D, page=page, N=N, M=M,
             dt=dt, scale=0.0, out=at(8), lse=at(9), status=at(10), ws=at(11) if n else None, n=n):
        return lib.ppd_tree_attention_paged(q, k, v, table, kt, vt, prefix, parent, L, B, H, G, T, D, page, N, M, dt, scale, out, lse, status, ws, n, None)
    ins, outs = ("q", "k", "v", "table", "kt", "vt", "prefix", "parent"), ("lse", "status")
    refused(call, [(o, i) for o in outs for i in ins] + [("lse", "status"), ("lse", "out")],
            [{x: None} for x in (*ins, "out", "status")] + [{x: at(20, 8)} for x in ("q", "k", "v", "kt", "vt", "out")] + [dict(lse=at(20, 2))] +
            [{x: 0} for x in ("L", "B", "H", "G", "T", "page", "N", "M")] + [dict(T=513), dict(D=80), dict(dt=3), dict(scale=NAN), dict(scale=INF)] +
            [dict(out=at(i, 16)) for i in range(8)] + [{i: at(8, 16)} for i in ins] + [dict(N=2 ** 27)] +
            ([dict(ws=at(i)) for i in range(11)] if n else []) + ([dict(ws=None, n=0), dict(n=n - 1), dict(ws=at(20, 16))] if dt else []),
            [dict(page=4), dict(page=48, N=9), dict(page=512, N=9), dict(M=2 ** 27)],
            [dict(lse=None), dict(v=at(1)), dict(scale=0.3)] + ([dict(ws=None, n=0)] if not dt else []))


def test_attention_workspace(lib):
    ws = lib.ppd_paged_attention_workspace_bytes
    assert ws(1, 1, 8, 4, 1, 128, 2 ** 17, 0) > 0          # few slices of long caches are cut
    assert ws(1, 1, 8, 4, 1, 128, 256, 0) == 0
    assert ws(1, 1, 8, 4, 1, 96, 2 ** 17, 0) == 0 and ws(1, 1, 8, 4, 600, 128, 2 ** 17, 0) == 0 and ws(1, 1, 8, 4, 1, 128, 2 ** 31 - 1, 0) == 0
    assert ws(1, 1, 8, 4, 3, 128, 256, 1) >= 8 * (12 + 6) * 128 * 2


@pytest.mark.parametrize("dt", [0, 1])
def test_logprobs(lib, dt):
    def call(logits=at(0), tokens=at(1), rows=at(2), B=3, T=5, V=100, n=4, K=6, dt=dt, temp=0.7, logprob=at(3), entropy=at(4), rank=at(5), top=at(6),
             best=at(7), status=at(8)):
        return lib.ppd_token_logprobs(logits, tokens, rows, B, T, V, n, K, dt, temp, logprob, entropy, rank, top, best, status, None)
    ins, outs = ("logits", "tokens", "rows"), ("logprob", "entropy", "rank", "top", "best", "status")
    refused(call, [(o, i) for o in outs for i in ins] + [(a, b) for a in outs for b in outs if a < b],
            [{x: None} for x in ("logits", "tokens", *outs)] + [{x: 0} for x in ("B", "T", "V", "n")] +
            [dict(K=-1), dict(K=6, V=5), dict(dt=2), dict(rows=None, n=6), dict(logits=at(20, 1)), dict(logprob=at(20, 2)), dict(best=at(20, 2))] +
            [dict(temp=x) for x in (0.0, -1.0, NAN, INF, 1e-39)],
            [dict(K=33), dict(B=2 ** 20, n=2 ** 10, rows=at(900), tokens=at(1000), logprob=at(1100), entropy=at(1200), rank=at(1300), top=at(1400),
                              best=at(1500), status=at(1600), logits=at(1700), T=1, V=40)],
            [dict(K=0, top=None, best=None), dict(rows=None), dict(K=32), dict(n=9), dict(logits=at(20, 4 if dt else 2))])


def test_bindings_refuse_other_types_and_shapes():
    """Before anything of the library is called."""
    from paper_2405_18628_gb300 import ppd
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="new_len is"):
        ppd.ppd_page_assign(i32(3), i32(2), 16, i32(3, 4), i32(9), i32(1), i32(1), i32(3), i32(8), i32(4), i32(3))
    with pytest.raises(TypeError, match="free_pages"):
        ppd.ppd_page_assign(i32(3), i32(3), 16, i32(3, 4), i32(9).long(), i32(1), i32(1), i32(3), i32(8), i32(4), i32(3))
    with pytest.raises(TypeError, match="k_pages"):
        ppd.ppd_page_append(bf(1, 2, 1, 4, 64), bf(1, 2, 1, 4, 64), bf(1, 5, 1, 16, 64).float(), bf(1, 5, 1, 16, 64), i32(8), i32(3), i32(2))
    with pytest.raises(ValueError, match="slot_start"):
        ppd.ppd_page_append(bf(1, 2, 1, 4, 64), bf(1, 2, 1, 4, 64), bf(1, 5, 1, 16, 64), bf(1, 5, 1, 16, 64), i32(8), i32(2), i32(2))
    with pytest.raises(ValueError, match="query heads"):
        ppd.ppd_tree_attention_paged(bf(1, 1, 3, 1, 64), bf(1, 5, 2, 16, 64), bf(1, 5, 2, 16, 64), i32(1, 4), bf(1, 1, 2, 1, 64), bf(1, 1, 2, 1, 64),
                                     i32(1), i32(1, 1), bf(1, 1, 3, 1, 64), i32(1))
    with pytest.raises(ValueError, match="given together"):
        ppd.ppd_token_logprobs(torch.zeros(1, 1, 9), i32(1, 1), 1.0, torch.zeros(1, 1), torch.zeros(1, 1), i32(1, 1), i32(1), top_tokens=i32(1, 1, 2))
    with pytest.raises(ValueError, match="contiguous CUDA"):
        ppd.ppd_token_logprobs(torch.zeros(1, 1, 9), i32(1, 1), 1.0, torch.zeros(1, 1), torch.zeros(1, 1), i32(1, 1), i32(1))
