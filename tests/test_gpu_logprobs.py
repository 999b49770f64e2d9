"""Log probabilities, entropy, ranks and alternatives on the GPU against 64 bits.

Ranks and alternatives are whole numbers of the row's values: equal.  With d = (x - m) / temperature, in units
of u = 2^-24: a difference, k = log2(e) / temperature (three roundings) and their product leave d within 5 u
of itself, the reference's temperature included; an exponential is within 4 u and 5 u |d| of itself, so a sum of
them within 4 u + 5 u E|d|, and n_seq + 64 roundings of a thread's and the block's sums (n_seq: entries that a
thread adds up).  E|d| <= entropy.  So ln p is within
    u (5 |d_t| + 5 H + n_seq + 72) + 2^-20   (the logarithm: 2^-21 of a bit, and what products of it round)
and the entropy, whose second sum has the same errors in terms of size |d|, within
    u (5 E d^2 + (n_seq + 80) (H + 1) + 5 H) + 2^-20 (1 + H)."""
import math

import numpy as np
import pytest
import torch

import oracle.pages as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _i32(a, dev):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)


def call(ppd, logits, tokens, temperature, rows=None, K=0, stream=None):
    dev, (B, n) = logits.device, tokens.shape
    r = dict(logprob=torch.full((B, n), 55.0, device=dev), entropy=torch.full((B, n), 55.0, device=dev), rank=_i32(np.full((B, n), -9), dev),
             status=_i32([77] * B, dev))
    if K:
        r.update(top=_i32(np.full((B, n, K), -9), dev), best=torch.full((B, n, K), 55.0, device=dev))
    ppd.ppd_token_logprobs(logits, tokens, temperature, r["logprob"], r["entropy"], r["rank"], r["status"], rows=rows, top_tokens=r.get("top"),
                           top_logprobs=r.get("best"), stream=stream)
    return r


def check_items(r, logits, tokens, temperature, rows, items):
    V = logits.shape[2]
    K = r["top"].shape[2] if "top" in r else 0
    for b, i in items:
        row, t = int(rows[b, i]) if rows is not None else i, int(tokens[b, i])
        x = logits[b, row].double()
        xs = x.tolist()
        lp, H, rank, order = O.logprobs(xs, t, temperature)
        assert int(r["rank"][b, i]) == rank, (b, i)
        if K:
            assert r["top"][b, i].tolist() == order[:K], (b, i)
        got = [(float(r["logprob"][b, i]), lp[t] if t >= 0 else 0.0, t)] if t >= 0 else []
        got += [(float(r["best"][b, i, j]), lp[order[j]], order[j]) for j in range(K)]
        if math.isnan(H):
            assert math.isnan(float(r["entropy"][b, i])) and all(math.isnan(g) for g, _, _ in got)
            continue
        d = (x - x.max()) / temperature
        p = lp.to(d.device).exp()
        sq = float(torch.where(p > 0, p * d * d, 0.0).sum())
        n_seq = V / 256
        for g, w, v in got:
            w = float(w)
            if w < -3.4028234e38 * math.log(2):     # in bits it is past fp32's range: (x - m) k overflows to -inf
                assert g == -math.inf, (b, i, g)
                continue
            assert abs(g - w) <= U * (5 * abs(float(d[v])) + 5 * H + n_seq + 72) + 2.0 ** -20, (b, i, v, g, w)
        assert abs(float(r["entropy"][b, i]) - H) <= U * (5 * sq + (n_seq + 80) * (H + 1) + 5 * H) + 2.0 ** -20 * (1 + H), (b, i)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 5, 31, 32, 33, 100, 1023, 4096, 4099, 9001, 32000, 50257])
def test_vocabularies(cuda_device, V, dtype):
    """Rows at every alignment, from one entry on."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(V)
    B, T = 2, 5
    logits = (3 * torch.randn(B, T, V, device=cuda_device, generator=g)).to(dtype)
    tokens = torch.randint(0, V, (B, T), device=cuda_device, generator=g).int()
    for K in sorted({0, 1, min(V, 5), min(V, 32)}):
        r = call(ppd, logits, tokens, 0.8, K=K)
        check_items(r, logits, tokens, 0.8, None, [(b, i) for b in range(B) for i in range(T)])
        assert (r["status"] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_vocabularies_and_temperatures(cuda_device, dtype):
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(1)
    for V, temperature in ((128256, 0.1), (151937, 1.0), (262144, 30.0), (600011, 0.7)):
        logits = (4 * torch.randn(1, 3, V, device=cuda_device, generator=g)).to(dtype)
        tokens = logits.argmax(-1).int()
        tokens[0, 1] = V - 1
        check_items(call(ppd, logits, tokens, temperature, K=20), logits, tokens, temperature, None, [(0, 0), (0, 1), (0, 2)])


def test_many_rows(cuda_device):
    """One CTA a row, several batches of columns each; a base that is not aligned."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(2)
    for dtype, shift in ((torch.float32, 1), (torch.bfloat16, 3)):
        B, T, V = 3, 250, 20011
        flat = (3 * torch.randn(B * T * V + shift, device=cuda_device, generator=g)).to(dtype)
        logits = flat[shift:].view(B, T, V)
        tokens = torch.randint(0, V, (B, T), device=cuda_device, generator=g).int()
        r = call(ppd, logits, tokens, 0.7, K=7)
        check_items(r, logits, tokens, 0.7, None, [(0, 0), (0, 1), (1, 100), (2, 249), (2, 248)])
        order = torch.sort(logits.float(), dim=-1, descending=True, stable=True).indices[..., :7]
        assert torch.equal(r["top"].long(), order)


def _hard_rows(V, dev):
    """Rows that selections go wrong at."""
    a = torch.arange(V, dtype=torch.float32, device=dev)
    rows = {"equal": torch.zeros(V, device=dev), "rising": a / 8, "falling": -a / 8, "steps": (a / 300).floor(), "two values": (a % 2),
            "zeros of both signs": torch.where(a % 3 == 0, -0.0, 0.0), "lowest": torch.full((V,), -3.4e38, device=dev),
            "one allowed": torch.full((V,), -math.inf, device=dev), "few allowed": torch.full((V,), -math.inf, device=dev),
            "huge": torch.where(a % 7 == 3, 3.0e38, -3.0e38), "tiny": a * 1e-42, "end": torch.full((V,), -5.0, device=dev),
            "lowest and some": torch.where(a < 9, a, -3.4028234e38)}
    rows["one allowed"][V // 2] = 1.5
    rows["few allowed"][[3, V // 3, V - 1]] = torch.tensor([0.5, -2.0, 0.5], device=dev)
    rows["end"][-40:] = 7.0
    for name, at in (("nan", [V // 3, 7]), ("inf", [5, V - 2])):
        rows[name] = torch.sin(a)
        rows[name][at] = math.nan if name == "nan" else math.inf
    rows["nothing"] = torch.full((V,), -math.inf, device=dev)
    return rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 3001, 40000])
def test_ties_infinities_and_nan(cuda_device, V, dtype):
    from paper_2405_18628_gb300 import ppd
    rows = _hard_rows(V, cuda_device)
    logits = torch.stack(list(rows.values()))[None].to(dtype)
    T = len(rows)
    for pick in (0, V // 2, V - 1, 7):
        tokens = _i32([[pick] * T], cuda_device)
        for K in (3, 32):
            r = call(ppd, logits, tokens, 0.9, K=K)
            check_items(r, logits, tokens, 0.9, None, [(0, i) for i in range(T)])


def test_rows_of_paths_and_what_is_not_asked(cuda_device):
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(3)
    B, T, V, n, K = 4, 9, 1000, 12, 4
    logits = 3 * torch.randn(B, T, V, device=cuda_device, generator=g)
    rows = _i32([[0, 3, 8, 8, 0] + [-1] * 7, [-1] * 12, [2] * 12, [5, 9, -2, 1, 2, -1, 2 ** 31 - 1, 0, 0, 0, 0, 0]], cuda_device)
    tokens = torch.randint(0, V, (B, n), device=cuda_device, generator=g).int()
    tokens[2, 3], tokens[2, 4], tokens[3, 3], tokens[3, 4] = -1, 999, 1000, -2
    r = call(ppd, logits, tokens, 1.0, rows=rows, K=K)
    assert r["status"].tolist() == [0, 0, 0, 3]
    asked = [(0, i) for i in range(5)] + [(2, i) for i in range(12)] + [(3, i) for i in (0, 7, 8, 9, 10, 11)]
    check_items(r, logits, tokens, 1.0, rows, asked)
    assert float(r["logprob"][2, 3]) == 0.0 and int(r["rank"][2, 3]) == -1
    for b in range(B):
        for i in range(n):
            if (b, i) not in asked:
                assert float(r["logprob"][b, i]) == 0 and float(r["entropy"][b, i]) == 0 and int(r["rank"][b, i]) == -1
                assert r["top"][b, i].tolist() == [-1] * K and r["best"][b, i].tolist() == [0.0] * K


def test_the_same_again_and_from_a_graph(cuda_device):
    """Sums have one order: results repeat bit for bit, captured or not, on another stream."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(4)
    logits = torch.randn(2, 3, 32003, device=cuda_device, generator=g).to(torch.bfloat16)
    tokens = torch.randint(0, 32003, (2, 3), device=cuda_device, generator=g).int()
    first = call(ppd, logits, tokens, 0.8, K=9)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    second = call(ppd, logits, tokens, 0.8, K=9, stream=side)
    out = {k: torch.zeros_like(v) for k, v in first.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ppd.ppd_token_logprobs(logits, tokens, 0.8, out["logprob"], out["entropy"], out["rank"], out["status"], top_tokens=out["top"], top_logprobs=out["best"])
    graph.replay()
    torch.cuda.synchronize()
    for k, v in first.items():
        assert torch.equal(v, second[k]) and torch.equal(v, out[k]), k


def test_logits_past_32_bits(cuda_device):
    from paper_2405_18628_gb300 import ppd
    V, T = 128257, 40000
    logits = torch.empty(1, T, V, dtype=torch.bfloat16, device=cuda_device)
    g = torch.Generator(device=cuda_device)
    g.manual_seed(6)
    rows = [0, 20001, 36000, T - 1]
    for r in rows:
        logits[0, r] = (3 * torch.randn(V, device=cuda_device, generator=g)).to(torch.bfloat16)
    at, tokens = _i32([rows], cuda_device), _i32([[5, V - 1, 70000, 0]], cuda_device)
    check_items(call(ppd, logits, tokens, 0.7, rows=at, K=4), logits, tokens, 0.7, at, [(0, i) for i in range(4)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [3, 257, 1000, 4096, 8191])
def test_many_short_rows(cuda_device, V, dtype):
    """Rows that single warps take."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(V)
    B, T = 4, 300
    logits = (3 * torch.randn(B, T, V, device=cuda_device, generator=g)).to(dtype)
    logits[0, :5, ::2] = -math.inf
    logits[1, 3, V // 2] = math.nan
    tokens = torch.randint(0, V, (B, T), device=cuda_device, generator=g).int()
    for K in (0, min(V, 8)):
        r = call(ppd, logits, tokens, 0.8, K=K)
        check_items(r, logits, tokens, 0.8, None, [(0, 0), (0, 4), (1, 3), (1, 4), (2, 150), (3, 299)])
        if K:
            clean = logits.float()[2:]
            assert torch.equal(r["top"][2:].long(), torch.sort(clean, dim=-1, descending=True, stable=True).indices[..., :K])
        x = logits.float()[2:]
        t = tokens[2:].long()[..., None]
        xt = x.gather(2, t)
        assert torch.equal(r["rank"][2:].long(), ((x > xt) | ((x == xt) & (torch.arange(V, device=cuda_device) < t))).sum(-1))


@pytest.mark.parametrize("V", [40, 3001])
def test_ties_infinities_and_nan_in_many_rows(cuda_device, V):
    """The hard rows again where single warps take them."""
    from paper_2405_18628_gb300 import ppd
    rows = _hard_rows(V, cuda_device)
    T = len(rows)
    logits = torch.stack(list(rows.values())).repeat(70, 1)[None]
    tokens = _i32([[V - 1] * (70 * T)], cuda_device)
    r = call(ppd, logits, tokens, 0.9, K=8)
    check_items(r, logits, tokens, 0.9, None, [(0, i) for i in range(T)])
    for k in ("logprob", "entropy", "rank", "top", "best"):
        assert torch.equal(torch.nan_to_num(r[k].float())[0, :T], torch.nan_to_num(r[k].float())[0, -T:]), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,K", [(2600, 5001, 0), (2600, 5001, 20), (2600, 5001, 32), (2000, 5001, 5), (2000, 5001, 21), (5200, 5001, 20), (5200, 301, 32), (1000, 2048, 20),
                                   (1000, 4097, 20)])
def test_blocks_of_every_size(cuda_device, n, V, K, dtype):
    """Rows by blocks of every size, batches of every size ending inside them; the hard rows among plain ones."""
    from paper_2405_18628_gb300 import ppd
    g = torch.Generator(device=cuda_device)
    g.manual_seed(V + K)
    hard = torch.stack(list(_hard_rows(V, cuda_device).values()))
    logits = (3 * torch.randn(n, V, device=cuda_device, generator=g)).to(dtype)
    h = len(hard)
    logits[:h] = logits[n - h:] = hard.to(dtype)
    logits, tokens = logits[None], torch.randint(0, V, (1, n), device=cuda_device, generator=g).int()
    tokens[0, n - h:] = tokens[0, :h]
    r = call(ppd, logits, tokens, 0.8, K=K)
    check_items(r, logits, tokens, 0.8, None, [(0, i) for i in [*range(h), h, n // 2, n - h - 1]])
    for k in set(r) - {"status"}:
        assert torch.equal(torch.nan_to_num(r[k].float())[0, :h], torch.nan_to_num(r[k].float())[0, n - h:]), k
    x, t = logits.float()[:, h:n - h], tokens[:, h:n - h].long()[..., None]
    if K:
        assert torch.equal(r["top"][:, h:n - h].long(), torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :K])
    xt = x.gather(2, t)
    assert torch.equal(r["rank"][:, h:n - h].long(), ((x > xt) | ((x == xt) & (torch.arange(V, device=cuda_device) < t))).sum(-1))
