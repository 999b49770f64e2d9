"""The decode loop's own bookkeeping (lengths, weights, room in the caches), with plain forms
in the place of the kernels: no GPU needed."""
import pytest
import torch

import oracle.operators as O


def _append(k_new, v_new, k_cache, k_scale, v_cache, v_scale, start, n_new, dev_status, rows=None, stream=None):
    L, B, H, T, D = k_new.shape
    for b in range(B):
        s, n = int(start[b]), int(n_new[b])
        dev_status[b] = 0 if s >= 0 and 0 <= n <= T and s + n <= k_cache.shape[3] else 4
        if dev_status[b] or n == 0:
            continue
        at = list(range(n)) if rows is None else rows[b, :n].tolist()
        for x, c, sc in ((k_new, k_cache, k_scale), (v_new, v_cache, v_scale)):
            c[:, b, :, s:s + n], sc[:, b, :, s:s + n] = O.kv4_quantise(x[:, b][:, :, at])


def _evict(weight, planes, length, budget, n_sink, n_recent, kept, new_len, dev_status, out_weight=None, out_planes=None, stream=None):
    L, B, H, S = weight.shape
    for b in range(B):
        n = int(length[b])
        dev_status[b] = 0 if 0 <= n <= S else 4
        new_len[b] = n if dev_status[b] else min(n, budget)
        for l in range(L):
            for h in range(H):
                at = [] if dev_status[b] else O.evict(weight[l, b, h].tolist(), n, budget, n_sink, n_recent)
                kept[l, b, h] = torch.tensor(at + [-1] * (budget - len(at)))
                for x in (*planes, weight):
                    x[l, b, h, :len(at)] = x[l, b, h][at].clone()


def _weight_add(q, lse, k_cache, k_tree, path, accept_len, prefix_len, weight, k_scale=None, scale=0.0, stream=None):
    """Every cached row gets 1 from a step, an accepted one too."""
    for b in range(weight.shape[1]):
        P, n = int(prefix_len[b]), int(accept_len[b])
        weight[:, b, :, :P] += 1
        weight[:, b, :, P:P + n] = 1


@pytest.fixture
def decode(monkeypatch):
    from paper_2405_18628_gb300 import build, ppd, sampled_decode
    build.build()
    monkeypatch.setattr(ppd, "ppd_kv4_append", _append)
    monkeypatch.setattr(ppd, "ppd_kv_evict", _evict)
    monkeypatch.setattr(ppd, "ppd_kv_weight_add", _weight_add)
    return sampled_decode


def _rows(n, seed=0, L=2, B=2, H=1, D=64):
    return torch.randn(L, B, H, n, D, generator=torch.Generator().manual_seed(seed))


def _step(ctx, n, **commit):
    """A step that accepts n[b] nodes."""
    L, B, H, G, T, D = ctx.sizes[:6]
    for b in range(B):
        ctx.accept_len[b] = n[b]
        ctx.path[b] = torch.tensor(list(range(n[b])) + [-1] * (T - n[b]))
    ctx.new_length.copy_(ctx.length + ctx.accept_len)
    ctx.commit(torch.zeros(L, B, H * G, T, D), _rows(T, 1, L, B, H, D), _rows(T, 2, L, B, H, D), **commit)


def test_a_prompt_after_an_eviction_starts_without_weight(decode):
    ctx = decode.LongContext(2, 2, 1, 1, 4, 64, 50, 40, 16, n_sink=1, n_recent=2, device="cpu")
    ctx.prompt(_rows(30), _rows(30))
    assert (ctx.weight == 0).all()
    _step(ctx, [3, 1])
    ctx.weight[:, :, :, :30] += torch.arange(30.0)   # unlike weights, large ones at the end
    ctx.evict()
    assert ctx.length.tolist() == [16, 16]
    old = ctx.weight[..., :16].clone()
    ctx.prompt(_rows(5, 3), _rows(5, 4))
    assert ctx.length.tolist() == [21, 21]
    assert torch.equal(ctx.weight[..., :16], old) and (ctx.weight[..., 16:] == 0).all()
    _step(ctx, [1, 2])
    assert (ctx.weight[..., 16:22] == 1).all()


def test_a_prompt_that_does_not_fit_is_refused(decode):
    """Nothing is written and no length moves; what does fit still enters."""
    ctx = decode.LongContext(1, 2, 1, 1, 4, 64, 50, 40, 36, n_sink=1, n_recent=2, device="cpu")
    with pytest.raises(ValueError, match="41 rows"):
        ctx.prompt(_rows(41, L=1), _rows(41, L=1))
    assert ctx.length.tolist() == [0, 0] and ctx.longest == 0 and (ctx.k == 0).all()
    ctx.prompt(_rows(25, L=1), _rows(25, L=1))
    with pytest.raises(ValueError, match="16 rows"):
        ctx.prompt(_rows(16, L=1), _rows(16, L=1))
    assert ctx.length.tolist() == [25, 25] and ctx.append_status.tolist() == [0, 0]
    ctx.prompt(_rows(10, L=1), _rows(10, L=1))
    assert ctx.length.tolist() == [35, 35] and ctx.append_status.tolist() == [0, 0]


def test_a_prompt_fits_by_what_steps_accepted(decode):
    """The host counts the most that steps can accept; where that leaves no room for a prompt, what
    they did accept decides."""
    ctx = decode.LongContext(1, 2, 1, 1, 4, 64, 50, 40, 30, n_sink=1, n_recent=2, device="cpu")
    ctx.prompt(_rows(20, L=1), _rows(20, L=1))
    for _ in range(3):
        _step(ctx, [1, 2])
    assert ctx.longest == 32 and ctx.length.tolist() == [23, 26]
    ctx.prompt(_rows(10, L=1), _rows(10, L=1))
    assert ctx.length.tolist() == [33, 36] and ctx.longest == 36 and ctx.append_status.tolist() == [0, 0]


def test_room_is_made_for_a_prompt_and_for_the_step_after_it(decode):
    ctx = decode.LongContext(1, 2, 1, 1, 4, 64, 50, 40, 16, n_sink=1, n_recent=2, device="cpu")
    ctx.prompt(_rows(36, L=1), _rows(36, L=1))              # a step of four nodes still fits
    assert ctx.length.tolist() == [36, 36]
    ctx.weight[:, :, :, :36] += torch.arange(36.0)
    ctx.prompt(_rows(10, L=1), _rows(10, L=1))              # after an eviction by weight
    assert ctx.length.tolist() == [26, 26] and ctx.append_status.tolist() == [0, 0]
    assert ctx.weight[0, 0, 0, :16].tolist() == [0.0] + [float(x) for x in range(21, 36)]
    assert (ctx.weight[..., 16:] == 0).all()
    ctx.prompt(_rows(12, L=1), _rows(12, L=1))              # it fits, a step after it would not
    assert ctx.length.tolist() == [16, 16] and ctx.longest == 16
    assert ctx.kept[0, 0, 0, -2:].tolist() == [36, 37]
    _step(ctx, [4, 4])
    assert ctx.length.tolist() == [20, 20] and ctx.append_status.tolist() == [0, 0]
    with pytest.raises(ValueError, match="25 rows"):        # no eviction makes room for it: none happens
        ctx.prompt(_rows(25, L=1), _rows(25, L=1))
    assert ctx.length.tolist() == [20, 20]


def test_budgets_that_leave_no_room_are_refused(decode):
    sizes = (1, 1, 1, 1, 4, 64, 50, 40)
    for bad in (dict(budget=37), dict(budget=41), dict(budget=35, most=6), dict(budget=10, n_sink=5, n_recent=6), dict(budget=0, n_sink=0, n_recent=0),
                dict(budget=10, most=0), dict(budget=20, n_sink=-1)):
        with pytest.raises(ValueError):
            decode.LongContext(*sizes, **{**dict(n_sink=1, n_recent=2, device="cpu"), **bad})
    decode.LongContext(*sizes, 36, n_sink=1, n_recent=2, device="cpu")
    ctx = decode.LongContext(*sizes, 38, n_sink=1, n_recent=2, device="cpu", most=2)   # steps of two nodes
    ctx.prompt(_rows(38, L=1, B=1), _rows(38, L=1, B=1))
    _step(ctx, [2])
    assert ctx.length.tolist() == [38]                      # cut as the step ended


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S_max", [41, 44, 97, 1001])
def test_every_layers_tensors_are_aligned(decode, S_max, D):
    """Attention is called one layer at a time, with 16-byte aligned tensors, whatever the capacity."""
    ctx = decode.LongContext(3, 1, 1, 1, 4, D, 50, S_max, 16, n_sink=1, n_recent=2, device="cpu")
    assert S_max <= ctx.sizes[7] == ctx.weight.shape[3] < S_max + 8
    for layer in range(3):
        for x in (ctx.k, ctx.k_scale, ctx.v, ctx.v_scale, ctx.out):
            assert x[layer:layer + 1].data_ptr() % 16 == 0
