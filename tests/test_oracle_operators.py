"""Pins of the plain 64-bit operators (oracle/operators.py): known values, closed forms and
the distributions that they have to have."""
import math

import pytest
import torch

import oracle.operators as O


def test_4bit_values_by_hand():
    # one word: channels 0..7 get codes 0..7; nibble p is channel 0 2 4 6 1 3 5 7
    codes = torch.zeros(16, dtype=torch.uint8)
    nib = [0, 2, 4, 6, 1, 3, 5, 7]
    codes[:4] = torch.tensor([nib[0] | nib[1] << 4, nib[2] | nib[3] << 4, nib[4] | nib[5] << 4, nib[6] | nib[7] << 4], dtype=torch.uint8)
    scales = torch.tensor([20 * 8 + 4], dtype=torch.uint8)       # 1.5
    assert O.kv4_values(codes, scales)[:8].tolist() == [1.5 * (c - 8) for c in range(8)]
    assert O.kv4_scale_table()[0] == 2.0 ** -20 and O.kv4_scale_table()[255] == 1.875 * 2.0 ** 11


def test_every_value_is_a_bf16_number():
    codes = torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 16).contiguous()
    for b in range(256):
        v = O.kv4_values(codes, torch.full((256, 1), b, dtype=torch.uint8))
        assert torch.equal(v.to(torch.bfloat16).double(), v)


@pytest.mark.parametrize("size", [1e-7, 1e-3, 1.0, 300.0, 26880.0])
def test_quantisation_error_is_half_a_step(size):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(50, 128, generator=g, dtype=torch.float64) * size / 5
    x = x.clamp(-size, size).float()
    codes, scales = O.kv4_quantise(x)
    s = O.kv4_scale_table()[scales.long()].repeat_interleave(32, -1)
    assert ((O.kv4_values(codes, scales) - x.double()).abs() <= s / 2 * (1 + 1e-6)).all()
    # the scale is the smallest that holds the largest channel
    top = x.double().abs().unflatten(-1, (-1, 32)).amax(-1)
    t = O.kv4_scale_table()
    assert (7 * t[scales.long()] >= top * (1 - 1e-6)).all()
    low = scales.long() - 1
    assert ((7 * t[low.clamp(min=0)] < top * (1 + 1e-6)) | (low < 0)).all()


def test_quantisation_of_odd_values():
    x = torch.zeros(4, 32)
    x[1, 3], x[1, 4] = math.nan, 2.0
    x[2, 0], x[2, 1] = math.inf, -math.inf
    x[3] = 1e30
    codes, scales = O.kv4_quantise(x)
    v = O.kv4_values(codes, scales)
    assert (v[0] == 0).all()
    assert v[1, 3] == 0 and abs(v[1, 4] - 2) <= O.kv4_scale_table()[int(scales[1])] / 2
    assert v[2, 0] == 7 * 3840 and v[2, 1] == -7 * 3840 and (v[2, 2:] == 0).all()
    assert (v[3] == 7 * 3840).all()


def test_attention_weights_of_accepted_nodes_add_up_to_their_number():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
    G, T, D, P = 2, 7, 64, 40
    parent = [-1, 0, 0, 1, 3, 2, 4]
    q, k, kt, vt = n(G, T, D), n(P + T, D).double(), n(T, D), n(T, D)
    _, lse, _, _ = O.attention_kv4(q, k, k, kt, vt, P, parent)
    w = O.weight_add(torch.zeros(P + T), q, lse, k, kt, [0, 1, 3, 4], P)
    assert abs(float(w.sum()) - 4 * G) < 1e-9


def test_eviction_by_hand():
    w = [0.0, 5.0, 1.0, math.nan, 5.0, 2.0, 9.0, 0.1]
    assert O.evict(w, 8, 8, 0, 0) == list(range(8))
    assert O.evict(w, 8, 3, 0, 0) == [1, 3, 6]           # NaN first, then 9, then the first 5
    assert O.evict(w, 8, 4, 1, 1) == [0, 3, 6, 7]
    assert O.evict(w, 5, 2, 0, 0) == [1, 3]
    assert O.evict([-0.0, 0.0, 1.0], 3, 2, 0, 0) == [0, 2]


@pytest.mark.parametrize("drawn", [False, True])
def test_emitted_tokens_have_the_targets_distribution(drawn):
    """The first token after the root, accepted or drawn from what is left, is distributed as
    softmax(logits): 4 standard deviations over 6000 walks."""
    g = torch.Generator().manual_seed(5)
    V, temp, N = 5, 0.8, 6000
    logits = torch.randn(4, V, generator=g) * 1.5
    p = torch.softmax(logits[0].double() / temp, -1)
    q = torch.softmax(torch.randn(V, generator=g), -1)
    parent = [-1, 0, 0, 0]
    count = [0] * V
    for _ in range(N):
        if drawn:
            cand = [0] + torch.multinomial(q, 3, replacement=True, generator=g).tolist()
            args = dict(draft_probs=q[None], draft_row=[-1, 0, 0, 0])
        else:
            cand, args = [0, 4, 2, 2], {}
        u = torch.rand(4, generator=g).tolist()
        noise = torch.empty(V).exponential_(generator=g)
        path, nxt, _, _ = O.sample_accept(logits, cand, parent, u, noise, temp, **args)
        count[cand[path[1]] if len(path) > 1 else nxt] += 1
    for v in range(V):
        sd = math.sqrt(N * float(p[v]) * (1 - float(p[v])))
        assert abs(count[v] - N * float(p[v])) < 4 * sd + 1, (count, (N * p).tolist())


def test_sampling_by_hand():
    logits = torch.log(torch.tensor([[0.5, 0.3, 0.2], [0.1, 0.8, 0.1], [1.0, 1.0, 1.0]]))
    ones = torch.ones(3)
    # the chosen token 1 has probability 0.3 at the root
    path, nxt, prob, _ = O.sample_accept(logits, [0, 1, -1], [-1, 0, 1], [0.0, 0.29, 0.0], ones, 1.0)
    assert path == [0, 1] and nxt == 1 and abs(prob[1] - 0.3) < 1e-6 and prob[2] == -1
    path, nxt, prob, _ = O.sample_accept(logits, [0, 1, 0], [-1, 0, 0], [0.0, 0.31, 0.72], ones, 1.0)
    # after 1 is gone, 0 has 5 / 7 and is rejected: 2 alone is left
    assert path == [0] and nxt == 2 and abs(prob[2] - 5 / 7) < 1e-6
    bad = logits.clone()
    bad[0, 2] = math.nan
    assert O.sample_accept(bad, [0, 1, 0], [-1, 0, 0], [0.0, 0.0, 0.0], ones, 1.0)[:2] == ([0], 2)
