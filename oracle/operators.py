"""Plain 64-bit forms of the operators for sampled decoding over a 4-bit cache (torch, any
device): the definitions of include/ppd.h written out, one sequence and one layer at a time,
without the library's code."""
from __future__ import annotations

import math

import torch

# nibble p of a 32-bit word of codes is this channel of its eight
CHANNEL = [2 * (p % 4) + p // 4 for p in range(8)]


def kv4_scale_table(device="cpu"):
    return torch.tensor([(1 + (b % 8) / 8) * 2.0 ** (b // 8 - 20) for b in range(256)], dtype=torch.float64, device=device)


def kv4_quantise(x):
    """x [..., D] -> codes uint8 [..., D/2], scales uint8 [..., D/32].  The quotient a / 7 is an
    fp32 one by definition; everything else is exact in 64 bits."""
    x = x.double()
    g = x.unflatten(-1, (-1, 32))
    clean = torch.where(torch.isnan(g), torch.zeros_like(g), g)
    a = (clean.abs().amax(-1).float() / torch.tensor(7.0, device=x.device)).double()
    table = kv4_scale_table(x.device)
    b = torch.searchsorted(table, a.contiguous()).clamp(max=255)   # the first scale >= a
    q = torch.round((clean / table[b][..., None]).clamp(-7, 7)).long() + 8
    word = q.reshape(*x.shape[:-1], -1, 8)[..., CHANNEL]           # nibbles in order
    return (word[..., 0::2] | word[..., 1::2] << 4).flatten(-2).to(torch.uint8), b.to(torch.uint8)


def kv4_values(codes, scales):
    """codes [..., D/2], scales [..., D/32] -> float64 [..., D]."""
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double().unflatten(-1, (-1, 8))
    out = torch.empty_like(nib)
    out[..., CHANNEL] = nib
    s = kv4_scale_table(codes.device)[scales.long()]
    return ((out.flatten(-2).unflatten(-1, (-1, 32)) - 8) * s[..., None]).flatten(-2)


def ancestors(parent):
    """bool [T,T]: node j is node i or one of its ancestors."""
    T = len(parent)
    see = torch.eye(T, dtype=torch.bool)
    for i in range(1, T):
        see[i] |= see[parent[i]]
    return see


def bf16(x):
    return x.to(torch.bfloat16).double()


def attention_kv4(q, k_rows, v_rows, k_tree, v_tree, prefix, parent, scale=0.0):
    """One slice: q [G,T,D], rows [>= prefix,D] as float64 values, tree rows [T,D] -> out, lse, and
    sum p |v| and max_j scale sum |q k| (what roundings are measured against)."""
    G, T, D = q.shape
    scale = scale if scale > 0 else 1 / math.sqrt(D)
    k = torch.cat([k_rows[:prefix], bf16(k_tree)])
    v = torch.cat([v_rows[:prefix], bf16(v_tree)])
    x = bf16(q) @ k.T * scale
    size = float((bf16(q).abs() @ k.abs().T).max() * scale)
    x[:, :, prefix:].masked_fill_(~ancestors(parent).to(x.device), -math.inf)
    p = torch.softmax(x, -1)
    return p @ v, torch.logsumexp(x, -1), p @ v.abs(), size


def weight_add(weight, q, lse, k_rows, k_tree, path, prefix, scale=0.0):
    """One slice: weight [S] (returned changed), q [G,T,D], lse [G,T], k_rows [S,D], path the accepted nodes."""
    D, S = q.shape[-1], weight.shape[0]
    scale = scale if scale > 0 else 1 / math.sqrt(D)
    w = weight.double().clone()
    new = [0.0] * len(path)
    for g in range(q.shape[0]):
        for i, a in enumerate(path):
            w[:prefix] += torch.exp(scale * (k_rows[:prefix].double() @ bf16(q[g, a])) - lse[g, a].double())
            for j in range(i + 1):
                new[j] += float(torch.exp(scale * torch.dot(bf16(k_tree[path[j]]), bf16(q[g, a])) - lse[g, a].double()))
    for j, x in enumerate(new):
        if prefix + j < S:
            w[prefix + j] = x
    return w


def evict(weight, length, budget, n_sink, n_recent):
    """The rows kept of one slice: weight [S] list of floats -> ascending indices."""
    if length <= budget:
        return list(range(length))

    def rank(j):
        if j < n_sink or j >= length - n_recent:
            return (0, 0.0, j)
        w = weight[j]
        return (1, 0.0, j) if math.isnan(w) else (2, -w + 0.0, j)
    return sorted(sorted(range(length), key=rank)[:budget])


def sample_accept(logits, cand, parent, u, noise, temperature, draft_probs=None, draft_row=None):
    """One sequence.  Returns path, next_token, accept_prob (-1: not tested) and the smallest
    relative margin of any decision."""
    T, V = logits.shape
    prob, margin = [-1.0] * T, math.inf

    def start(node):
        x = logits[node].double()
        if torch.isnan(x).any() or torch.isposinf(x).any() or torch.isneginf(x).all():
            return None
        return torch.softmax(x / temperature, -1)

    path, r = [0], start(0)
    while True:
        cur, nxt = path[-1], None
        for c in range(cur + 1, T):
            if parent[c] != cur or cand[c] < 0:
                continue
            t, row = cand[c], -1 if draft_row is None else draft_row[c]
            if r is None or float(r.sum()) == 0:
                prob[c] = 0.0
                continue
            z = float(r.sum())
            a = float(r[t]) / z
            if row >= 0:
                qt = float(draft_probs[row][t])
                a = a / qt if qt > 0 else 0.0
            a = min(1.0, a)
            prob[c] = a
            if 0 < a < 1:
                margin = min(margin, abs(u[c] - a) / max(a, 1e-30))
            if u[c] < a:
                nxt = c
                break
            if row >= 0:
                r = (r / z - draft_probs[row].double()).clamp(min=0)
            else:
                r = r.clone()
                r[t] = 0
        if nxt is None:
            break
        path.append(nxt)
        r = start(nxt)
    cur = path[-1]
    if r is None:
        x = logits[cur]
        nan = torch.isnan(x)
        return path, int((nan if nan.any() else x).int().argmax() if nan.any() else x.argmax()), prob, margin
    if float(r.sum()) == 0:
        r = start(cur)
    s = r / noise.double()
    top = torch.topk(s, min(2, V)).values
    if V > 1:
        margin = min(margin, float((top[0] - top[1]) / top[0]))
    return path, int(s.argmax()), prob, margin
