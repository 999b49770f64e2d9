"""Attention weight per cached row and eviction on the GPU, against 64 bits and row by row.

Bound of a weight, from its formula: each exp(score - lse) has the relative error of its
exponent's absolute one, at most D 2^-24 of the sum of the score's magnitudes plus 1e-5
(the exponent's other roundings and exp itself), and the sums add a few units of 2^-24."""
import math

import numpy as np
import pytest
import torch

import oracle.operators as O

pytestmark = pytest.mark.gpu


def _i32(a, dev):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)


@pytest.mark.parametrize("cache", ["kv4", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,B,H,G,T,lens,n", [
    (1, 1, 1, 1, 1, [0], [1]), (1, 1, 2, 1, 8, [33], [3]), (2, 3, 2, 2, 20, [100, 0, 67], [5, 1, 0]),
    (1, 2, 3, 8, 1, [31, 32], [1, 1]), (1, 2, 2, 3, 40, [64, 500], [40, 17]), (1, 1, 1, 2, 512, [129], [300]),
    (1, 1, 2, 1, 6, [3001], [4])])
def test_weights_add_up(cuda_device, cache, D, L, B, H, G, T, lens, n):
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    g = torch.Generator(device=dev)
    g.manual_seed(T)
    S = max(lens) + max(n) + 3
    dt = torch.float32 if T == 20 else torch.bfloat16
    r = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
    q, kt = r(L, B, H * G, T, D).to(dt), r(L, B, H, T, D).to(dt)
    lse = math.log(1 + max(lens)) + 0.3 * r(L, B, H * G, T)
    if cache == "kv4":
        kc, ks = O.kv4_quantise(r(L, B, H, S, D))
        rows = O.kv4_values(kc, ks)
    else:
        kc, ks = r(L, B, H, S, D).to(torch.bfloat16), None
        for b in range(B):
            kc[:, b, :, lens[b]:] = float("nan")     # never used
        rows = kc.double()
    path = [sorted(np.random.default_rng(b).permutation(T)[:n[b]].tolist()) for b in range(B)]
    weight = r(L, B, H, S).abs()
    want = weight.double().clone()
    bound = torch.zeros_like(want)
    for l in range(L):
        for b in range(B):
            for h in range(H):
                hs = slice(h * G, (h + 1) * G)
                if n[b]:
                    want[l, b, h] = O.weight_add(weight[l, b, h], q[l, b, hs], lse[l, b, hs], rows[l, b, h], kt[l, b, h], path[b], lens[b])
                size = max(float((O.bf16(q[l, b, hs]).abs() @ torch.cat([rows[l, b, h, :lens[b]], O.bf16(kt[l, b, h])]).abs().T).max()), 1) / math.sqrt(D)
                bound[l, b, h] = D * 2.0 ** -24 * size + 2e-5
    ppd.ppd_kv_weight_add(q, lse, kc, kt, _i32([p + [-1] * (T - len(p)) for p in path], dev), _i32(n, dev), _i32(lens, dev), weight, k_scale=ks)
    assert ((weight.double() - want).abs() <= bound * want.abs()).all(), float(((weight.double() - want).abs() / want.abs()).max())
    for b in range(B):   # rows past the new ones stay as they were, bit for bit
        assert torch.equal(weight[:, b, :, lens[b] + n[b]:].double(), want[:, b, :, lens[b] + n[b]:])


def test_weights_of_a_step_add_up_to_the_accepted_nodes(cuda_device):
    """The attention's own log-sum-exps: over all rows, each accepted query gives 1."""
    from paper_2405_18628_gb300 import ppd
    dev, T, H, G, D, P = cuda_device, 24, 4, 2, 128, 777
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    r = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
    kc, ks = O.kv4_quantise(r(1, 1, H, P + T, D))
    vc, vs = O.kv4_quantise(r(1, 1, H, P + T, D))
    q, kt, vt = (r(1, 1, h, T, D).to(torch.bfloat16) for h in (H * G, H, H))
    parent = [-1] + [(i - 1) // 2 for i in range(1, T)]
    out = torch.empty(1, 1, H * G, T, D, dtype=torch.bfloat16, device=dev)
    lse = torch.empty(1, 1, H * G, T, device=dev)
    st = torch.empty(1, dtype=torch.int32, device=dev)
    ppd.ppd_tree_attention_kv4(q, kc, ks, vc, vs, kt, vt, _i32([P], dev), _i32([parent], dev), out, st, lse=lse)
    weight = torch.zeros(1, 1, H, P + T, device=dev)
    path = [0, 2, 6, 14]
    ppd.ppd_kv_weight_add(q, lse, kc, kt, _i32([path + [-1] * (T - 4)], dev), _i32([4], dev), _i32([P], dev), weight, k_scale=ks)
    assert (weight.sum(-1) - 4 * G).abs().max() < 1e-3


def _planes(kind, L, B, H, S, D, dev, g):
    if kind == "bf16":
        return [torch.randn(L, B, H, S, D, device=dev, generator=g).to(torch.bfloat16) for _ in "kv"]
    if kind == "none":
        return []
    if kind == "odd":    # rows that no wide load divides
        return [torch.randint(0, 256, (L, B, H, S, w), dtype=torch.uint8, device=dev, generator=g) for w in (3, 6, 72, 1000)]
    return [torch.randint(0, 256, (L, B, H, S, w), dtype=torch.uint8, device=dev, generator=g) for w in (D // 2, D // 32, D // 2, D // 32)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["bf16", "kv4", "odd", "none"])
@pytest.mark.parametrize("L,B,H,D,S,lens,budget,sink,recent", [
    (1, 1, 1, 64, 1, [1], 1, 0, 0), (1, 2, 3, 64, 40, [40, 7], 8, 2, 3), (2, 3, 2, 128, 700, [700, 513, 0], 300, 4, 32),
    (1, 1, 4, 64, 5003, [5001], 5000, 0, 0), (1, 2, 1, 128, 3000, [2999, 40], 1, 0, 0), (1, 1, 2, 128, 2500, [2500], 64, 32, 32),
    (1, 1, 1, 64, 20000, [19997], 9001, 1, 100)])
def test_evict_keeps_the_heaviest_rows(cuda_device, in_place, kind, L, B, H, D, S, lens, budget, sink, recent):
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    g = torch.Generator(device=dev)
    g.manual_seed(S)
    weight = torch.exp(2 * torch.randn(L, B, H, S, device=dev, generator=g))
    weight[0, 0, 0, ::3] = 0.25                                   # many ties
    if S > 30:
        weight[0, 0, 0, 5:9] = torch.tensor([float("nan"), -0.0, 0.0, float("inf")], device=dev)
        weight[0, 0, 0, 20] = -1.0
    planes = _planes(kind, L, B, H, S, D, dev, g)
    host = [p.clone() for p in planes] + [weight.clone()]
    S_out = S if in_place else budget + 5
    outs = planes if in_place else [torch.full((L, B, H, S_out, *p.shape[4:]), 7, dtype=p.dtype, device=dev) for p in planes]
    out_w = weight if in_place else torch.full((L, B, H, S_out), 7.0, device=dev)
    kept = torch.full((L, B, H, budget), 99, dtype=torch.int32, device=dev)
    new_len, status = torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev)
    ppd.ppd_kv_evict(weight, planes, _i32(lens, dev), budget, sink, recent, kept, new_len, status,
                     out_planes=None if in_place else outs, out_weight=None if in_place else out_w)
    assert status.tolist() == [0] * B
    assert new_len.tolist() == [min(x, budget) for x in lens]
    for l in range(L):
        for b in range(B):
            for h in range(H):
                want = O.evict(host[-1][l, b, h].tolist(), lens[b], budget, sink, recent)
                m = len(want)
                assert kept[l, b, h].tolist() == want + [-1] * (budget - m)
                for src, dst in zip(host, outs + [out_w]):
                    raw = lambda t: t.contiguous().flatten().view(torch.uint8)  # noqa: E731
                    at = torch.tensor(want, dtype=torch.long, device=dev)
                    assert torch.equal(raw(dst[l, b, h, :m]), raw(src[l, b, h][at]))
                    if in_place:
                        assert torch.equal(raw(dst[l, b, h, m:]), raw(src[l, b, h, m:]))
                    else:
                        assert (dst[l, b, h, m:] == 7).all()


def test_evict_in_place_of_many_slices_and_long_rows(cuda_device):
    """Shifts of every size, whole columns moved over one another."""
    from paper_2405_18628_gb300 import ppd
    dev, L, B, H, S, D, budget = cuda_device, 2, 4, 40, 1500, 128, 1400
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    planes = _planes("bf16", L, B, H, S, D, dev, g)
    weight = torch.rand(L, B, H, S, device=dev, generator=g)
    host, host_w = [p.clone() for p in planes], weight.clone()
    kept = torch.empty(L, B, H, budget, dtype=torch.int32, device=dev)
    i = [torch.empty(B, dtype=torch.int32, device=dev) for _ in range(2)]
    ppd.ppd_kv_evict(weight, planes, _i32([S] * B, dev), budget, 0, 0, kept, *i)
    top = torch.sort(torch.topk(host_w, budget, -1).indices, -1).values
    assert torch.equal(kept.long(), top)
    for p, h in zip(planes, host):
        assert torch.equal(p[:, :, :, :budget], torch.gather(h, 3, top[..., None].expand(-1, -1, -1, -1, D)))
    assert torch.equal(weight[..., :budget], torch.gather(host_w, 3, top))


def test_evict_reports_bad_lengths(cuda_device):
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    w = torch.rand(1, 3, 2, 20, device=dev)
    before = w.clone()
    kept = torch.empty(1, 3, 2, 4, dtype=torch.int32, device=dev)
    new_len, status = torch.empty(3, dtype=torch.int32, device=dev), torch.empty(3, dtype=torch.int32, device=dev)
    ppd.ppd_kv_evict(w, [], _i32([-1, 21, 20], dev), 4, 1, 1, kept, new_len, status)
    E = ppd.PPD_ERR_CAPACITY
    assert status.tolist() == [E, E, 0] and new_len.tolist() == [-1, 21, 4]
    assert (kept[:, :2] == -1).all() and torch.equal(w[:, :2], before[:, :2])


@pytest.mark.parametrize("ties", [False, True])
def test_evict_of_long_caches(cuda_device, ties):
    """More rows than a block's shared memory holds, and more equal ones than a short list."""
    from paper_2405_18628_gb300 import ppd
    dev, S, budget = cuda_device, 70001, 30011
    g = torch.Generator(device=dev)
    g.manual_seed(9)
    for n in (S, 39999):
        w = torch.rand(1, 1, 2, n, device=dev, generator=g)
        if ties:
            w = (w * 3).floor()
        host = w.clone()
        kept = torch.empty(1, 1, 2, min(budget, n // 2), dtype=torch.int32, device=dev)
        i = [torch.empty(1, dtype=torch.int32, device=dev) for _ in range(2)]
        ppd.ppd_kv_evict(w, [], _i32([n], dev), kept.shape[3], 5, 7, kept, *i)
        key = host.clone()
        key[..., :5] = key[..., n - 7:] = float("inf")
        want = torch.sort(torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :kept.shape[3]], -1).values
        assert torch.equal(kept.long(), want)
        assert torch.equal(w[..., :kept.shape[3]], torch.gather(host, 3, want))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S,lens,budget,sink,recent", [(128, [128, 0, 77, 33], 31, 1, 2), (31, [31, 30, 10, 1], 10, 0, 0), (127, [127, 126, 2, 96], 96, 33, 40)])
def test_evict_of_short_caches(cuda_device, in_place, S, lens, budget, sink, recent):
    """Many heads of a few rows, more than one of them ending anywhere in a warp's rows; rows of 1 to
    1024 bytes."""
    from paper_2405_18628_gb300 import ppd
    dev, L, H = cuda_device, 3, 5
    g = torch.Generator(device=dev)
    g.manual_seed(S)
    weight = (torch.rand(L, 4, H, S, device=dev, generator=g) * 6).floor()
    weight[0, 0, 0, 3] = float("nan")
    planes = [torch.randint(0, 256, (L, 4, H, S, w), dtype=torch.uint8, device=dev, generator=g) for w in (1, 64, 1024, 1000, 38)]
    host = [p.clone() for p in planes] + [weight.clone()]
    outs = planes if in_place else [torch.zeros(L, 4, H, budget, p.shape[4], dtype=torch.uint8, device=dev) for p in planes]
    out_w = weight if in_place else torch.zeros(L, 4, H, budget, device=dev)
    kept = torch.empty(L, 4, H, budget, dtype=torch.int32, device=dev)
    new_len, status = (torch.empty(4, dtype=torch.int32, device=dev) for _ in range(2))
    ppd.ppd_kv_evict(weight, planes, _i32(lens, dev), budget, sink, recent, kept, new_len, status, out_planes=None if in_place else outs,
                     out_weight=None if in_place else out_w)
    assert new_len.tolist() == [min(x, budget) for x in lens] and status.tolist() == [0] * 4
    for l in range(L):
        for b in range(4):
            for h in range(H):
                want = O.evict(host[-1][l, b, h].tolist(), lens[b], budget, sink, recent)
                assert kept[l, b, h].tolist() == want + [-1] * (budget - len(want))
                at = torch.tensor(want, dtype=torch.long, device=dev)
                for src, dst in zip(host, outs + [out_w]):
                    assert torch.equal(dst[l, b, h, :len(want)].nan_to_num(9.0) if dst.is_floating_point() else dst[l, b, h, :len(want)],
                                       src[l, b, h][at].nan_to_num(9.0) if src.is_floating_point() else src[l, b, h][at])


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S,budget,sink,recent", [(1, 1, 0, 0), (31, 10, 2, 3), (64, 63, 0, 0), (100, 40, 0, 40), (128, 31, 1, 2)])
def test_evict_of_many_short_caches(cuda_device, in_place, S, budget, sink, recent):
    """Slices by the hundred, of every length up to the capacity and one outside it."""
    from paper_2405_18628_gb300 import ppd
    dev, L, B, H = cuda_device, 2, 33, 9
    g = torch.Generator(device=dev)
    g.manual_seed(S)
    lens = [int(x) for x in np.linspace(0, S, B - 1)] + [S + 1]
    weight = (torch.rand(L, B, H, S, device=dev, generator=g) * 9).floor()
    planes = [torch.randint(0, 256, (L, B, H, S, w), dtype=torch.uint8, device=dev, generator=g) for w in (64, 4, 1024, 7)]
    host = [p.clone() for p in planes] + [weight.clone()]
    outs = planes if in_place else [torch.zeros(L, B, H, budget, p.shape[4], dtype=torch.uint8, device=dev) for p in planes]
    out_w = weight if in_place else torch.zeros(L, B, H, budget, device=dev)
    before = [x.clone() for x in outs + [out_w]]
    kept = torch.full((L, B, H, budget), 77, dtype=torch.int32, device=dev)
    new_len, status = (torch.empty(B, dtype=torch.int32, device=dev) for _ in range(2))
    ppd.ppd_kv_evict(weight, planes, _i32(lens, dev), budget, sink, recent, kept, new_len, status, out_planes=None if in_place else outs,
                     out_weight=None if in_place else out_w)
    assert new_len.tolist() == [min(x, budget) for x in lens[:-1]] + [S + 1]
    assert status.tolist() == [0] * (B - 1) + [status[-1].item()] and status[-1] != 0
    ranks, got, b = host[-1].tolist(), kept.tolist(), B - 1
    for l in range(L):
        for h in range(H):
            assert got[l][b][h] == [-1] * budget
            for b_ in range(B - 1):
                want = O.evict(ranks[l][b_][h], lens[b_], budget, sink, recent)
                assert got[l][b_][h] == want + [-1] * (budget - len(want))
    at = kept.long().clamp(min=0)
    for src, dst, old in zip(host, outs + [out_w], before):
        rows = torch.take_along_dim(src, at.reshape(*at.shape, *[1] * (src.dim() - 4)), 3)
        live = (kept >= 0).reshape(*kept.shape, *[1] * (src.dim() - 4))
        assert torch.equal(dst[..., :budget, :] if src.dim() == 5 else dst[..., :budget],
                           torch.where(live, rows, old[..., :budget, :] if src.dim() == 5 else old[..., :budget]))


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (1, 3), (2, 4), (3, 7), (5, 9)])
def test_weights_of_infinite_rows(cuda_device, cache, D, G, n):
    """Rows whose every score is -inf get no weight, of +inf infinite weight, of NaN NaN, however many
    queries there are; all others what they get without such rows."""
    from paper_2405_18628_gb300 import ppd
    dev, T, P = cuda_device, 12, 70
    g = torch.Generator(device=dev)
    g.manual_seed(G * 10 + n)
    r = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
    q, kt = r(1, 1, G, T, D).to(torch.bfloat16), r(1, 1, 1, T, D).to(torch.bfloat16)
    q[..., 0] = q[..., 0].abs() + 1                # the scores' sign is that of the rows' first channel
    lse = 4 + 0.3 * r(1, 1, G, T)
    path = sorted(np.random.default_rng(n).permutation(T)[:n].tolist())
    rest = dict(path=_i32([path + [-1] * (T - n)], dev), accept_len=_i32([n], dev), prefix_len=_i32([P], dev))
    if cache == "kv4":
        kc, ks = O.kv4_quantise(r(1, 1, 1, P + T, D))
    else:
        kc, ks = r(1, 1, 1, P + T, D).to(torch.bfloat16), None
    start = r(1, 1, 1, P + T).abs()
    plain, weight = start.clone(), start.clone()
    ppd.ppd_kv_weight_add(q, lse, kc, kt, weight=plain, k_scale=ks, **rest)
    kt[0, 0, 0, path[n // 2], 0] = -math.inf
    want = plain.clone()
    want[..., P + n // 2] = 0
    if cache == "bf16":
        for row, x, w in ((5, -math.inf, start[..., 5]), (31, -math.inf, start[..., 31]), (9, math.inf, math.inf), (66, math.nan, math.nan)):
            kc[..., row, 0] = x
            want[..., row] = w
    ppd.ppd_kv_weight_add(q, lse, kc, kt, weight=weight, k_scale=ks, **rest)
    assert torch.equal(weight.nan_to_num(-7.0), want.nan_to_num(-7.0))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,H,S,budget,sink,recent", [(12, 22, 31, 10, 2, 3), (12, 43, 128, 77, 0, 5), (9, 15, 33, 32, 0, 0), (7, 3, 127, 40, 3, 2)])
def test_evict_of_short_caches_of_any_weights(cuda_device, in_place, B, H, S, budget, sink, recent):
    """NaN, zeros of both signs, negative, tiny and infinite weights, and rows in more pieces than a warp moves at
    once; hundreds of slices, and (the last) too few for a warp each."""
    from paper_2405_18628_gb300 import ppd
    dev, L = cuda_device, 2
    g = torch.Generator(device=dev)
    g.manual_seed(S)
    lens = [int(x) for x in np.linspace(0, S, B)]
    odd = torch.tensor([math.nan, -math.nan, 0.0, -0.0, -1.0, 1.0, math.inf, -math.inf, 1e-42, -1e-42, 3.4e38, 0.5], device=dev)
    weight = odd[torch.randint(0, len(odd), (L, B, H, S), device=dev, generator=g)]
    planes = [torch.randint(0, 256, (L, B, H, S, w), dtype=torch.uint8, device=dev, generator=g) for w in (1023, 64, 513)]
    host = [p.clone() for p in planes] + [weight.clone()]
    outs = planes if in_place else [torch.full((L, B, H, budget, p.shape[4]), 3, dtype=torch.uint8, device=dev) for p in planes]
    out_w = weight if in_place else torch.full((L, B, H, budget), 3.0, device=dev)
    before = [x.clone() for x in outs + [out_w]]
    kept = torch.full((L, B, H, budget), 77, dtype=torch.int32, device=dev)
    new_len, status = (torch.empty(B, dtype=torch.int32, device=dev) for _ in range(2))
    ppd.ppd_kv_evict(weight, planes, _i32(lens, dev), budget, sink, recent, kept, new_len, status, out_planes=None if in_place else outs,
                     out_weight=None if in_place else out_w)
    assert new_len.tolist() == [min(x, budget) for x in lens] and (status == 0).all()
    ranks, got = host[-1].tolist(), kept.tolist()
    for l in range(L):
        for b in range(B):
            for h in range(H):
                want = O.evict(ranks[l][b][h], lens[b], budget, sink, recent)
                assert got[l][b][h] == want + [-1] * (budget - len(want)), (l, b, h)
    at, live = kept.long().clamp(min=0), kept >= 0
    raw = lambda x: x.view(torch.int32) if x.dtype == torch.float32 else x  # noqa: E731
    for src, dst, old in zip(host, outs + [out_w], before):
        src, dst, old = (raw(x).reshape(L, B, H, x.shape[3], -1) for x in (src, dst, old))
        rows = torch.take_along_dim(src, at[..., None], 3)
        assert torch.equal(dst[..., :budget, :], torch.where(live[..., None], rows, old[..., :budget, :]))
