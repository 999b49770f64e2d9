"""Acceptance by sampling on the GPU against the plain 64-bit walk on the same random
numbers.  A decision is unique where its sides differ by more than float rounding: an fp32
sum of V terms and a few residuals of it are within about 1e-5, so sequences whose smallest
relative margin (from the 64-bit walk) is above 1e-4 are compared, and almost all are."""
import math

import numpy as np
import pytest
import torch

import oracle.operators as O

pytestmark = pytest.mark.gpu


def _i32(a, dev):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)


def _outputs(B, T, dev):
    i = lambda *s: torch.full(s, 55, dtype=torch.int32, device=dev)  # noqa: E731
    return dict(accept_len=i(B), path=i(B, T), next_token=i(B), new_prefix_len=i(B), dev_status=i(B)), torch.full((B, T), 9.0, device=dev)


def _check(ppd, dev, logits, cand, parent, u, noise, temp, draft_probs=None, draft_row=None, prefix=None, least=0.9):
    B, T, V = logits.shape
    prefix = prefix or [10 + b for b in range(B)]
    o, prob = _outputs(B, T, dev)
    d = {} if draft_probs is None else dict(draft_probs=draft_probs.to(dev), draft_row=_i32(draft_row, dev))
    ppd.ppd_sample_accept(logits.to(dev), _i32(cand, dev), _i32(parent, dev), _i32(prefix, dev), 5000, temp, u.to(dev), noise.to(dev),
                          accept_prob=prob, **o, **d)
    assert o["dev_status"].tolist() == [0] * B
    n = 0
    for b in range(B):
        path, nxt, want, margin = O.sample_accept(logits[b], cand[b], parent[b], u[b].tolist(), noise[b], temp,
                                                  None if draft_probs is None else draft_probs[b], None if draft_row is None else draft_row[b])
        if margin < 1e-4:
            continue
        n += 1
        assert o["path"][b].tolist() == path + [-1] * (T - len(path)), b
        assert int(o["accept_len"][b]) == len(path) and int(o["new_prefix_len"][b]) == prefix[b] + len(path)
        assert int(o["next_token"][b]) == nxt, b
        np.testing.assert_allclose(prob[b].cpu().double().numpy(), want, rtol=1e-4, atol=1e-6)
    assert n >= least * B, (n, B)
    return o


def _trees(rng, B, T):
    parent, prompt = [], []
    for _ in range(B):
        p, q = [-1], [False]
        for i in range(1, T):
            a = int(rng.integers(0, i)) if rng.random() < 0.6 else 0
            p.append(a)
            q.append(bool(q[a] or rng.random() < 0.2))
        parent.append(p)
        prompt.append(q)
    return parent, prompt


def _case(B, T, V, drawn, seed, temp, sharp=3.0):
    """Guesses near the target's top tokens, some chosen, some drawn, some prompt tokens."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    parent, prompt = _trees(rng, B, T)
    logits = sharp * torch.randn(B, 1, V, generator=g) + torch.randn(B, T, V, generator=g)
    probs = torch.softmax((logits[:, [0, min(1, T - 1), min(2, T - 1)]] + 0.5 * torch.randn(B, 3, V, generator=g)) / temp, -1)
    cand = [[0] * T for _ in range(B)]
    row = [[-1] * T for _ in range(B)]
    for b in range(B):
        for i in range(1, T):
            if prompt[b][i]:
                cand[b][i] = -1
            elif drawn and rng.random() < (0.7 if drawn == "some" else 1.0):
                row[b][i] = int(rng.integers(3))
                cand[b][i] = int(torch.multinomial(probs[b, row[b][i]], 1, generator=g))
            else:
                cand[b][i] = int(torch.topk(logits[b, parent[b][i]], min(V, 4)).indices[int(rng.integers(min(V, 4)))])
    u = torch.rand(B, T, generator=g)
    noise = torch.empty(B, V).exponential_(generator=g).clamp_(min=1e-12)
    return logits, cand, parent, u, noise, probs if drawn else None, row if drawn else None


@pytest.mark.parametrize("drawn", ["", "some", "all"])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (3, 2, 2), (4, 9, 33), (2, 64, 1024), (5, 30, 4099), (1, 64, 32000), (40, 16, 700), (2, 512, 517), (1, 20, 128256)])
def test_walks(cuda_device, drawn, B, T, V):
    from paper_2405_18628_gb300 import ppd
    x = _case(B, T, V, drawn, B * 100 + T, 0.7)
    _check(ppd, cuda_device, *x[:5], 0.7, *x[5:], least=0.5 if B < 4 else 0.8)


@pytest.mark.parametrize("temp", [0.05, 1.0, 20.0])
def test_temperatures(cuda_device, temp):
    from paper_2405_18628_gb300 import ppd
    x = _case(12, 24, 300, "some", 7, temp)
    _check(ppd, cuda_device, *x[:5], temp, *x[5:], least=0.8)


def test_the_same_token_guessed_twice_and_a_certain_one(cuda_device):
    from paper_2405_18628_gb300 import ppd
    V = 40
    logits = torch.randn(3, 5, V, generator=torch.Generator().manual_seed(1))
    logits[2, 0, 7] = 1000.0                      # everything is token 7
    cand = [[0, 3, 3, 5, -1], [0, 4, 6, 4, 4], [0, 1, 2, 7, 9]]
    parent = [[-1, 0, 0, 0, 0]] * 3
    u = torch.full((3, 5), 0.999)
    u[2, 3] = 0.9999999
    noise = torch.ones(3, V)
    o = _check(ppd, cuda_device, logits, cand, parent, u, noise, 1.0, least=1.0)
    assert o["path"][2].tolist() == [0, 3, -1, -1, -1]


def test_drafts_that_cover_the_target_leave_its_distribution(cuda_device):
    """q = p: a drawn child is accepted at once; where u says no (it cannot below 1), and all is
    taken away, the whole distribution is drawn from."""
    from paper_2405_18628_gb300 import ppd
    dev, V = cuda_device, 64
    logits = torch.randn(1, 2, V, generator=torch.Generator().manual_seed(2))
    q = torch.softmax(logits[:, :1].double(), -1).float()
    q2 = torch.ones(1, 1, V)                      # no distribution, but it covers everything
    o, prob = _outputs(1, 2, dev)
    args = (logits.to(dev), _i32([[0, 5]], dev), _i32([[-1, 0]], dev), _i32([0], dev), 100, 1.0, torch.full((1, 2), 0.9, device=dev),
            torch.ones(1, V, device=dev))
    ppd.ppd_sample_accept(*args, accept_prob=prob, draft_probs=q.to(dev), draft_row=_i32([[-1, 0]], dev), **o)
    assert o["path"].tolist() == [[0, 1]] and abs(float(prob[0, 1]) - 1) < 1e-5
    ppd.ppd_sample_accept(*args, accept_prob=prob, draft_probs=q2.to(dev), draft_row=_i32([[-1, 0]], dev), **o)
    assert o["path"].tolist() == [[0, -1]] and int(o["next_token"][0]) == int(logits[0, 0].argmax())


def test_rows_without_a_distribution(cuda_device):
    from paper_2405_18628_gb300 import ppd
    V = 1000
    logits = torch.randn(6, 3, V, generator=torch.Generator().manual_seed(3))
    logits[0, 0, [700, 20]] = float("nan")
    logits[1, 0, 999] = float("inf")
    logits[2, 0] = -math.inf
    logits[3, 0, 1:] = -math.inf                  # one token is left: a distribution
    logits[4, 0, 5] = float("nan")                # the guess's own entry
    logits[5, 0, 0:500] = -math.inf
    cand = [[0, 1, 2], [0, 999, 2], [0, 0, 1], [0, 1, 0], [0, 5, 3], [0, 1, 2]]
    u = torch.zeros(6, 3)
    o = _check(ppd, cuda_device, logits, cand, [[-1, 0, 0]] * 6, u, torch.ones(6, V), 1.0, least=1.0)
    assert o["next_token"].tolist()[:3] == [20, 999, 0] and o["path"][3].tolist() == [0, 2, -1]


def test_malformed_sequences_are_reported(cuda_device):
    from paper_2405_18628_gb300 import ppd
    dev, B, T, V = cuda_device, 9, 4, 50
    logits = torch.randn(B, T, V, device=dev)
    parent = [[-1, 0, 1, 2] for _ in range(B)]
    cand = [[0, 1, 2, -1] for _ in range(B)]
    row = [[-1, 0, 0, -7] for _ in range(B)]      # a prompt token's draft row is not looked at
    prefix = [0] * B
    parent[1][2] = 2
    parent[2][0] = 0
    cand[3][1] = V
    cand[4][2] = -2
    cand[5][0] = -1
    row[6][1] = 1
    prefix[7], prefix[8] = -1, 100
    o, prob = _outputs(B, T, dev)
    ppd.ppd_sample_accept(logits, _i32(cand, dev), _i32(parent, dev), _i32(prefix, dev), 100, 1.0, torch.zeros(B, T, device=dev), torch.ones(B, V, device=dev),
                          accept_prob=prob, draft_probs=torch.full((B, 1, V), 1.0 / V, device=dev), draft_row=_i32(row, dev), **o)
    E, C = ppd.PPD_ERR_TREE, ppd.PPD_ERR_CAPACITY
    assert o["dev_status"].tolist() == [0, E, E, E, E, E, E, C, C]
    assert o["accept_len"].tolist() == [3] + [0] * 8 and o["next_token"].tolist()[1:] == [-1] * 8
    assert o["new_prefix_len"].tolist() == [3] + prefix[1:] and (o["path"][1:] == -1).all() and (prob[1:] == -1).all()


def test_emitted_tokens_have_the_targets_distribution(cuda_device):
    """20,000 sequences with the same logits: the first emitted token's counts within 4 standard
    deviations of the target's, for chosen and for drawn guesses."""
    from paper_2405_18628_gb300 import ppd
    dev, B, T, V = cuda_device, 20000, 4, 6
    g = torch.Generator(device=dev)
    g.manual_seed(11)
    row = torch.tensor([0.5, 1.5, -0.3, 0.9, 0.0, -1.0], device=dev)
    logits = row.expand(B, T, V).contiguous()
    p = torch.softmax(row.double() / 0.9, -1)
    q = torch.softmax(torch.tensor([1.0, 0.2, 0.4, -0.5, 0.0, 0.3], device=dev), -1)
    for drawn in (False, True):
        cand = torch.tensor([[0, 3, 0, 2]], device=dev).repeat(B, 1)
        d = {}
        if drawn:
            cand[:, 1:] = torch.multinomial(q, 3 * B, replacement=True, generator=g).view(B, 3)
            d = dict(draft_probs=q.expand(B, 1, V).contiguous(), draft_row=torch.tensor([[-1, 0, 0, 0]], dtype=torch.int32, device=dev).repeat(B, 1))
        o, _ = _outputs(B, T, dev)
        ppd.ppd_sample_accept(logits, cand.int().contiguous(), _i32([[-1, 0, 0, 0]] * B, dev), _i32([0] * B, dev), 100, 0.9,
                              torch.rand(B, T, device=dev, generator=g), torch.empty(B, V, device=dev).exponential_(generator=g).clamp_(min=1e-20), **o, **d)
        second = o["path"][:, 1].long()
        tok = torch.where(second >= 0, torch.gather(cand, 1, second.clamp(min=0)[:, None])[:, 0], o["next_token"].long())
        count = torch.bincount(tok, minlength=V).double()
        sd = (B * p * (1 - p)).sqrt()
        assert ((count - B * p).abs() < 4 * sd).all(), (count.tolist(), (B * p).tolist())


@pytest.mark.parametrize("V", [700, 32000])
def test_outputs_in_the_place_of_inputs(cuda_device, V):
    """New lengths over the lengths, the path over the candidates, probabilities over the random
    numbers: what separate memory gives, failed sequences among them."""
    from paper_2405_18628_gb300 import ppd
    dev, B, T = cuda_device, 9, 16
    logits, cand, parent, u, noise, probs, row = _case(B, T, V, "some", 5, 0.7)
    prefix = [10 + b for b in range(B)]
    prefix[2], prefix[5], parent[7][3] = -1, 5001, 3
    want, prob = _outputs(B, T, dev)
    lg, noise, probs, row = logits.to(dev), noise.to(dev), probs.to(dev), _i32(row, dev)
    ppd.ppd_sample_accept(lg, _i32(cand, dev), _i32(parent, dev), _i32(prefix, dev), 5000, 0.7, u.to(dev), noise, accept_prob=prob, draft_probs=probs,
                          draft_row=row, **want)
    assert [x != 0 for x in want["dev_status"].tolist()] == [b in (2, 5, 7) for b in range(B)]
    o, _ = _outputs(B, T, dev)
    length, c, w = _i32(prefix, dev), _i32(cand, dev), u.to(dev)
    o.update(new_prefix_len=length, path=c)
    ppd.ppd_sample_accept(lg, c, _i32(parent, dev), length, 5000, 0.7, w, noise, accept_prob=w, draft_probs=probs, draft_row=row, **o)
    for k in want:
        assert torch.equal(o[k], want[k]), k
    assert torch.equal(w, prob)
