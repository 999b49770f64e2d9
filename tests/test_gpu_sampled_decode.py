"""The operators together, as a decode loop runs them: lengths, weights, rows and eviction over
several steps against the plain 64-bit forms, the GPU's own decisions followed."""
import numpy as np
import pytest
import torch

import oracle.operators as O

pytestmark = pytest.mark.gpu


def test_steps_of_a_decode_loop(cuda_device):
    from paper_2405_18628_gb300 import sampled_decode as S
    dev, L, B, H, G, T, D, V, S_max, budget = cuda_device, 2, 2, 2, 2, 12, 64, 500, 96, 60
    g = torch.Generator(device=dev)
    g.manual_seed(4)
    rng = np.random.default_rng(4)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
    ctx = S.LongContext(L, B, H, G, T, D, V, S_max, budget, n_sink=2, n_recent=5, device=dev)
    kp, vp = n(L, B, H, 70, D), n(L, B, H, 70, D)
    ctx.prompt(kp, vp)
    # the plain state: values and weights of every head's rows
    val = {"k": O.kv4_values(*O.kv4_quantise(kp)), "v": O.kv4_values(*O.kv4_quantise(vp))}
    rows = {(x, l, b, h): list(val[x][l, b, h]) for x in "kv" for l in range(L) for b in range(B) for h in range(H)}
    weight = {(l, b, h): [0.0] * 70 for l in range(L) for b in range(B) for h in range(H)}
    evicted = 0
    for step in range(9):
        parent = [[-1] + [int(rng.integers(0, i)) for i in range(1, T)] for _ in range(B)]
        pt = torch.tensor(parent, dtype=torch.int32, device=dev)
        q, kt, vt = n(L, B, H * G, T, D), n(L, B, H, T, D), n(L, B, H, T, D)
        for l in range(L):
            ctx.attend(l, q[l], kt[l], vt[l], pt)
        logits = 4 * torch.randn(B, T, V, device=dev, generator=g)
        cand = logits.argmax(-1).gather(1, pt.long().clamp(min=0)).int()
        u, noise = torch.rand(B, T, device=dev, generator=g), torch.empty(B, V, device=dev).exponential_(generator=g).clamp_(min=1e-12)
        ctx.accept(logits, cand, pt, 0.8, u, noise)
        paths = [[x for x in p if x >= 0] for p in ctx.path.tolist()]
        for b in range(B):
            assert paths[b][0] == 0 and all(parent[b][y] == x for x, y in zip(paths[b], paths[b][1:]))
        lse = ctx.lse.clone()
        before = ctx.longest
        ctx.commit(q, kt, vt)
        cut = ctx.longest < before
        evicted += cut
        for (l, b, h), w in weight.items():
            P = len(w)
            hs = slice(h * G, (h + 1) * G)
            k, v = torch.stack(rows["k", l, b, h]), torch.stack(rows["v", l, b, h])
            out, want_lse, mass, size = O.attention_kv4(q[l, b, hs], k, v, kt[l, b, h], vt[l, b, h], P, parent[b])
            assert ((ctx.out[l, b, hs].double() - out).abs() <= (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass + 1e-36).all()
            assert float((lse[l, b, hs].double() - want_lse).abs().max()) <= D * 2.0 ** -24 * size + 1e-5
            grown = torch.tensor(w + [0.0] * T, dtype=torch.float64, device=dev)
            grown = O.weight_add(grown, q[l, b, hs], want_lse, k, kt[l, b, h], paths[b], P)[:P + len(paths[b])]
            w[:] = grown.tolist()
            for x, new in (("k", kt), ("v", vt)):
                rows[x, l, b, h] += list(O.kv4_values(*O.kv4_quantise(new[l, b, h][paths[b]])))
            if cut:
                got = [j for j in ctx.kept[l, b, h].tolist() if j >= 0]
                want = O.evict(w, len(w), budget, 2, 5)
                # the kept rows are the heaviest; two of nearly equal weight may change places
                lost, won = sorted(set(want) - set(got)), sorted(set(got) - set(want))
                assert len(got) == len(want) and all(abs(w[i] - w[j]) <= 1e-4 * w[i] for i, j in zip(lost, won))
                w[:] = [w[j] for j in got]
                for x in "kv":
                    rows[x, l, b, h] = [rows[x, l, b, h][j] for j in got]
            m = len(w)
            assert int(ctx.length[b]) == m
            np.testing.assert_allclose(ctx.weight[l, b, h, :m].cpu().numpy(), w, rtol=1e-4, atol=1e-7)
            for x, c, s in (("k", ctx.k, ctx.k_scale), ("v", ctx.v, ctx.v_scale)):
                assert torch.equal(O.kv4_values(c[l, b, h, :m], s[l, b, h, :m]), torch.stack(rows[x, l, b, h]))
    assert evicted >= 1
    for st in (ctx.attend_status, ctx.accept_status, ctx.append_status, ctx.evict_status):
        assert (st == 0).all()


def test_the_command(cuda_device, capsys):
    from paper_2405_18628_gb300 import sampled_decode as S
    assert S.main(["--steps", "24", "--layers", "2"]) == 0
    assert "statuses [0, 0, 0, 0]" in capsys.readouterr().out


def test_a_prompt_after_an_eviction(cuda_device):
    """A second turn's prompt: its rows have no weight, whatever rows an eviction left behind them,
    and the next eviction ranks them by what steps gave them."""
    from paper_2405_18628_gb300 import sampled_decode as S
    dev, L, B, H, G, T, D, V = cuda_device, 2, 3, 2, 1, 8, 64, 100
    g = torch.Generator(device=dev)
    g.manual_seed(6)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
    ctx = S.LongContext(L, B, H, G, T, D, V, 64, 20, n_sink=2, n_recent=3, device=dev)
    parent = torch.tensor([[-1, 0, 1, 2, 3, 4, 5, 6]] * B, dtype=torch.int32, device=dev)

    def step():
        q, kt, vt = n(L, B, H * G, T, D), n(L, B, H, T, D), n(L, B, H, T, D)
        for l in range(L):
            ctx.attend(l, q[l], kt[l], vt[l], parent)
        logits = 3 * torch.randn(B, T, V, device=dev, generator=g)
        cand = logits.argmax(-1).gather(1, parent.long().clamp(min=0)).int()
        ctx.accept(logits, cand, parent, 1.0, torch.rand(B, T, device=dev, generator=g),
                   torch.empty(B, V, device=dev).exponential_(generator=g).clamp_(min=1e-12))
        ctx.commit(q, kt, vt)

    ctx.prompt(n(L, B, H, 40, D), n(L, B, H, 40, D))
    step()
    ctx.weight[:, :, :, 20:] += 1000.0        # heavy rows where the next turn's will be
    ctx.evict()
    assert ctx.length.tolist() == [20] * B
    old = ctx.weight[..., :20].clone()
    assert (ctx.weight[..., 20:28] > 0).all()
    ctx.prompt(n(L, B, H, 11, D), n(L, B, H, 11, D))
    assert torch.equal(ctx.weight[..., :20], old) and (ctx.weight[..., 20:31] == 0).all()
    step()
    # a step's weight: less than its accepted nodes' for each row
    assert (ctx.weight[..., 20:31] < T).all() and (ctx.weight[..., 20:31].sum((0, 1, 2)) > 0).all()
    lens = ctx.length.tolist()
    weight = ctx.weight.tolist()
    ctx.evict()
    for l in range(L):
        for b in range(B):
            for h in range(H):
                assert ctx.kept[l, b, h].tolist() == O.evict(weight[l][b][h], lens[b], 20, 2, 3)
    for st in (ctx.attend_status, ctx.accept_status, ctx.append_status, ctx.evict_status):
        assert (st == 0).all()


def test_layers_of_odd_capacities(cuda_device):
    from paper_2405_18628_gb300 import sampled_decode as S
    dev, D = cuda_device, 64
    g = torch.Generator(device=dev)
    g.manual_seed(7)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
    ctx = S.LongContext(3, 1, 1, 1, 4, D, 50, 97, 50, n_sink=1, n_recent=2, device=dev)
    kp, vp, q, kt, vt = n(3, 1, 1, 60, D), n(3, 1, 1, 60, D), n(3, 1, 1, 4, D), n(3, 1, 1, 4, D), n(3, 1, 1, 4, D)
    ctx.prompt(kp, vp)
    parent = [-1, 0, 0, 1]
    for l in range(3):
        out = ctx.attend(l, q[l], kt[l], vt[l], torch.tensor([parent], dtype=torch.int32, device=dev))
        k, v = (O.kv4_values(*O.kv4_quantise(x[l, 0, 0])) for x in (kp, vp))
        want, _, mass, size = O.attention_kv4(q[l, 0], k, v, kt[l, 0, 0], vt[l, 0, 0], 60, parent)
        assert ((out[0].double() - want).abs() <= (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass + 1e-36).all()
    assert (ctx.attend_status == 0).all()
