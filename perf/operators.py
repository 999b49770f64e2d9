"""Operators of a decode step that samples, over a long context held in few bits:

  append   rows of K and V quantised into a cache held in 4 bits (those of an accepted
           path, or a prompt's), and read back as the values they stand for
  attend   a token tree's attention over such a cache and its own ancestors
  weigh    the attention weight that the accepted tokens gave each cached row, added up
  evict    a cache cut down to a budget of rows per head by that weight
  verify   drafted tokens checked against the target's probabilities with given random
           numbers, and the token after the last accepted one drawn

Sizes: L layers, B sequences, H key/value heads, G query heads for each, head dim D, cached
tokens P (B > 1: ragged, P the longest), cache capacity S, trees of T tokens, vocabulary V.

The 4-bit rows: D / 2 bytes of codes and D / 32 scales for 32 channels each.  A 32-bit word
holds eight channels: nibble p is channel 2 (p % 4) + p // 4, and a code c stands for
scale * (c - 8).  A scale byte b stands for (1 + (b % 8) / 8) * 2^(b // 8 - 20).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TEMPERATURE = 0.7


def case(name, kind, L=1, B=1, H=1, G=1, D=128, P=64, T=1, n=1, V=0, S=None, budget=0, cache="kv4", dtype="bf16", draft=False):
    c = dict(kind=kind, L=L, B=B, H=H, G=G, D=D, P=P, T=T, n=n, V=V, S=S if S is not None else P + T,
             budget=budget, cache=cache, dtype=dtype, draft=draft)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a test-sized model's step: latency is all there is
        case("attend_tiny", "attend", 1, 1, 4, 1, 64, 128, 48),
        # plain decoding, one layer's call: a token of four sequences, four query heads a K/V head, odd lengths
        case("attend_token_gqa_layer", "attend", 1, 4, 8, 4, 128, 9999, 1, S=10240),
        # one step of a 7B model, the headline size
        case("attend_vicuna7b", "attend", 32, 1, 32, 1, 128, 2048, 64),
        # long contexts, eight ragged sequences, four of the 32 layers: the largest
        case("attend_long_batch8", "attend", 4, 8, 32, 1, 128, 16384, 64),
        # an accepted path of six nodes enters the cache of every layer
        case("append_path", "append", 32, 1, 32, 1, 128, 2048, 64, n=6),
        # an odd prompt of two sequences kept in fp32, D = 64
        case("append_prompt_f32", "append", 8, 2, 16, 1, 64, 0, 1003, n=1003, S=1280, dtype="f32"),
        # the rows' weights after a step of the 7B model that accepted four tokens
        case("weigh_vicuna7b", "weigh", 32, 1, 32, 1, 128, 2048, 64, n=4),
        # long ragged contexts in bf16, two query heads a K/V head, an odd capacity
        case("weigh_long_bf16", "weigh", 4, 8, 16, 2, 128, 16384, 32, n=3, S=16461, cache="bf16"),
        # a short cache of one layer, called as that layer is done
        case("evict_layer_bf16", "evict", 1, 3, 16, 1, 64, 1003, 1, budget=640, cache="bf16"),
        # long caches of eight sequences down to a quarter
        case("evict_long", "evict", 4, 8, 32, 1, 128, 16384, 1, budget=4096),
        # one sequence, guesses taken as the best tokens of each depth
        case("verify_top", "verify", T=64, V=32000),
        # a large batch whose guesses were drawn from their depth's distribution, an odd vocabulary
        case("verify_batch_drawn", "verify", B=80, T=32, V=50257, S=4096, draft=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "weigh", "evict", "verify"])
    if kind == "verify":
        V = rng.choice([1024, 32000, 32003, 50257, 128256])
        T = _log_int(rng, 2, 200)
        B = _log_int(rng, 1, max(1, min(96, int(1.3e8 / (V * T)))))
        return case(None, kind, B=B, T=T, V=V, S=4096, draft=rng.random() < 0.5)
    D = rng.choice([64, 128, 128])
    H = rng.choice([1, 2, 4, 8, 16, 32, 40])
    G = rng.choice([1, 1, 2, 4, 8]) if H <= 16 and kind in ("attend", "weigh") else 1
    B = 1 if rng.random() < 0.6 else _log_int(rng, 2, 64)
    P = _log_int(rng, 1, 16384)
    T = 1 if rng.random() < 0.25 else _log_int(rng, 2, 512)
    n = 1
    if kind == "append":
        T = _log_int(rng, 1, 2000)
        n = T if rng.random() < 0.5 else _log_int(rng, 1, min(T, 16))
    if kind == "weigh":
        n = _log_int(rng, 1, min(T, 12))
    # (layer, sequence, head, key) rows and the products of the largest listed case
    rows = 4 * 8 * 32 * 13000 * 128 / D
    if kind == "attend":
        rows = min(rows, rows * 64 / (G * T))
    if kind in ("weigh", "append"):
        rows /= 2
    P = max(1, min(P, int(rows / (B * H)) - T))
    B = max(1, min(B, int(rows / (H * (P + T)))))
    L = max(1, min(_log_int(rng, 1, 40), int(rows / (B * H * (P + T)))))
    return case(None, kind, L, B, H, G, D, P, T, n=n, S=P + T + rng.choice([0, 0, 1, 63, 250]),
                budget=max(1, int(P * rng.uniform(0.2, 0.95))) if kind == "evict" else 0,
                cache=rng.choice(["kv4", "kv4", "bf16"]) if kind in ("weigh", "evict") else "kv4",
                dtype=rng.choice(["bf16", "f32"]) if kind in ("append", "attend") else "bf16")


# ------------------------------------------------------------------ inputs

def _lens(c):
    """Cached tokens of each sequence: P, or ragged between P / 2 and P."""
    return [c["P"] - (b * 7919) % (c["P"] // 2 + 1) for b in range(c["B"])]


def _tree(rng, T):
    """Parents and prompt-token flags of a tree: a quarter of its nodes (root included) are
    guesses at most six deep, chains of up to three prompt tokens fill the rest."""
    n = max(1, (T + 3) // 4)
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = rng.randrange(i)
        while depth[p] >= 6:
            p = rng.randrange(i)
        parent.append(p)
        depth.append(depth[p] + 1)
    prompt, anchor, left = [False] * n, 0, 0
    while len(parent) < T:
        parent.append(anchor % n if left == 0 else len(parent) - 1)
        prompt.append(True)
        anchor, left = (anchor + 1, 2) if left == 0 else (anchor, left - 1)
    return parent, prompt


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _path(parent, n):
    """A root-to-node path of at most n nodes: the deepest one's first nodes."""
    best = []
    for i in range(len(parent)):
        p = [i]
        while parent[p[-1]] >= 0:
            p.append(parent[p[-1]])
        best = p if len(p) > len(best) else best
    return best[::-1][:n]


def prepare(case, seed):
    c = case
    L, B, H, G, D, T, S, n, V = (c[k] for k in ("L", "B", "H", "G", "D", "T", "S", "n", "V"))
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 17)
    rng = random.Random(seed * 7919 + 5)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    normal = lambda *shape: torch.randn(shape, dtype=dt, device=DEV, generator=g)  # noqa: E731
    empty = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    s = dict(case=c, status=empty(torch.int32, B))
    if c["kind"] == "verify":
        return _prepare_verify(c, s, g, rng)
    if c["kind"] == "append":
        # rows as a model's projections give them: channels of unlike sizes
        size = torch.exp(0.5 * torch.randn(H, 1, D, device=DEV, generator=g))
        s.update(k_new=(normal(L, B, H, T, D) * size).to(dt), v_new=normal(L, B, H, T, D))
        if n < T:
            rows = [sorted(rng.sample(range(1, T), n - 1)) for _ in range(B)]
            s["rows"] = _i32([[0] + r + [-1] * (T - n) for r in rows])
        else:
            s["rows"] = None
        s.update(start=_i32([min(p, S - n) for p in _lens(c)]), n_new=_i32([n] * B))
        for k in ("k", "v"):
            s[k + "_cache"] = torch.zeros(L, B, H, S, D // 2, dtype=torch.uint8, device=DEV)
            s[k + "_scale"] = torch.zeros(L, B, H, S, D // 32, dtype=torch.uint8, device=DEV)
            s[k + "_back"] = empty(torch.bfloat16, L, B, H, n, D)
        return s
    s["prefix_len"] = _i32(_lens(c))
    if c["kind"] == "evict":
        s.update(budget=c["budget"], sink=min(4, c["budget"]), recent=max(0, min(64, c["budget"] - 4) // 2))
        # weights fall off by powers of ten from row to row, as sums of attention weights do
        s["weight"] = torch.exp(2.5 * torch.randn(L, B, H, S, device=DEV, generator=g)) / 100
        s["kept"], s["new_len"] = empty(torch.int32, L, B, H, c["budget"]), empty(torch.int32, B)
        if c["cache"] == "bf16":
            s["planes"] = [normal(L, B, H, S, D), normal(L, B, H, S, D)]
        else:
            s["planes"] = [x for _ in range(2) for x in _kv4_rows(g, L, B, H, S, D)]
        # the rows go into a cache of the budget's size
        s["out_planes"] = [torch.zeros(L, B, H, c["budget"], *x.shape[4:], dtype=x.dtype, device=DEV) for x in s["planes"]]
        s["out_weight"] = torch.zeros(L, B, H, c["budget"], device=DEV)
        return s
    trees = [_tree(rng, T) for _ in range(B)]
    s["parent"] = _i32([p for p, _ in trees])
    s.update(q=normal(L, B, H * G, T, D), k_tree=normal(L, B, H, T, D))
    if c["kind"] == "attend":
        s["k_cache"], s["k_scale"] = _kv4_rows(g, L, B, H, S, D)
        s["v_cache"], s["v_scale"] = _kv4_rows(g, L, B, H, S, D)
        s.update(v_tree=normal(L, B, H, T, D), out=empty(torch.bfloat16, L, B, H * G, T, D), lse=empty(torch.float32, L, B, H * G, T))
        s["workspace"] = empty(torch.uint8, 64 << 20)   # one scratch buffer serves a program's calls
        return s
    paths = [_path(p, n) for p, _ in trees]
    s["path"] = _i32([p + [-1] * (T - len(p)) for p in paths])
    s["accept_len"] = _i32([len(p) for p in paths])
    if c["cache"] == "bf16":
        s["k_cache"], s["k_scale"] = normal(L, B, H, S, D), None
    else:
        s["k_cache"], s["k_scale"] = _kv4_rows(g, L, B, H, S, D)
    # what the attention left: log-sum-exps of scores of unit normal rows, about log P + 1/2
    s["lse"] = torch.log(s["prefix_len"].float())[None, :, None, None] + 0.5 + 0.1 * torch.randn(L, B, H * G, T, device=DEV, generator=g)
    s["weight"] = torch.rand(L, B, H, S, device=DEV, generator=g)
    return s


def _kv4_rows(g, L, B, H, S, D):
    """A 4-bit cache of unit normal rows."""
    codes = torch.empty(L, B, H, S, D // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(L, B, H, S, D // 32, dtype=torch.uint8, device=DEV)
    for l in range(L):
        codes[l], scales[l] = _quantise(torch.randn(B, H, S, D, device=DEV, generator=g))
    return codes, scales


def _prepare_verify(c, s, g, rng):
    B, T, V = c["B"], c["T"], c["V"]
    trees = [_tree(rng, T) for _ in range(B)]
    parent, prompt = [p for p, _ in trees], _i32([q for _, q in trees]) != 0
    depth = [[0] * T for _ in range(B)]
    for b in range(B):
        for i in range(1, T):
            depth[b][i] = depth[b][parent[b][i]] + 1
    # a target whose rows of one depth are alike, as a guess for that depth can foresee
    n_draft = 7
    base = 4.0 * torch.randn(B, n_draft, V, device=DEV, generator=g)
    at = _i32(depth).long().clamp(max=n_draft - 1)
    s["logits"] = torch.empty(B, T, V, device=DEV)
    for b in range(B):
        torch.randn(T, V, device=DEV, generator=g, out=s["logits"][b])
        s["logits"][b] += base[b, at[b]]
    s.update(parent=_i32(parent), prefix_len=_i32([100 + b for b in range(B)]))
    up = s["parent"].long().clamp(min=0)
    row = torch.gather(at, 1, up)   # a node was guessed from the distribution of its parent's depth
    if c["draft"]:
        s["draft_probs"] = torch.softmax(base / TEMPERATURE, -1)
        s["draft_row"] = row.int()
        cand = torch.stack([torch.multinomial(s["draft_probs"][b], T, replacement=True, generator=g)[row[b], torch.arange(T, device=DEV)] for b in range(B)])
    else:
        s["draft_probs"] = s["draft_row"] = None
        # the best tokens of the depth's guess, one each for a node's children
        best = torch.topk(base, min(16, V), dim=-1).indices
        rank = [[sum(parent[b][j] == parent[b][i] for j in range(1, i)) % 16 for i in range(T)] for b in range(B)]
        cand = torch.stack([best[b, row[b], _i32(rank[b]).long()] for b in range(B)])
    s["cand"] = torch.where(prompt, -1, cand).int()
    s["u"] = torch.rand(B, T, device=DEV, generator=g)
    s["noise"] = torch.empty(B, V, device=DEV).exponential_(generator=g).clamp_(min=1e-20)
    for k in ("accept_len", "next_token", "new_len"):
        s[k] = torch.empty(B, dtype=torch.int32, device=DEV)
    s["path"] = torch.empty(B, T, dtype=torch.int32, device=DEV)
    s["accept_prob"] = torch.empty(B, T, device=DEV)
    return s


# ------------------------------------------------------------------ plain forms

def _quantise(x):
    """fp32 [..., D] -> codes [..., D / 2], scales [..., D / 32]."""
    x = x.float()
    g = x.unflatten(-1, (-1, 32))
    top = torch.where(g == g, g.abs(), 0.0).amax(-1)
    up = (top / torch.full_like(top, 7.0)).view(torch.int32) + 0xFFFFF >> 20   # the next scale with three bits after the point
    b = (up - 107 * 8).clamp(0, 255)
    s = ((b + 856) << 20).view(torch.float32)
    q = torch.round(g / s[..., None])
    code = torch.where(q == q, q.clamp(-7, 7), 0.0).int() + 8
    code = code.reshape(*x.shape[:-1], -1, 4, 2).transpose(-1, -2).reshape(*x.shape[:-1], -1, 2)   # even channels first
    return (code[..., 0] | code[..., 1] << 4).to(torch.uint8), b.to(torch.uint8)


def _values(codes, scales):
    """codes [..., D / 2], scales [..., D / 32] -> fp32 [..., D]."""
    c = torch.stack([codes & 15, codes >> 4], -1).to(torch.float32)               # nibbles in order
    c = c.reshape(*codes.shape[:-1], -1, 2, 4).transpose(-1, -2).flatten(-3)      # channels in order
    s = ((scales.int() + 856) << 20).view(torch.float32)
    return ((c.unflatten(-1, (-1, 32)) - 8.0) * s[..., None]).flatten(-2)


def _rounded(x):
    """Operands of products are bf16; fp32 ones are rounded."""
    return x.to(torch.bfloat16).float()


def _visible(parent):
    """[B, T, T]: node j is i or an ancestor of i."""
    T = parent.shape[1]
    at = torch.arange(T, device=parent.device)
    see = ((parent[:, :, None] == at) | (at[:, None] == at)).float()
    for _ in range(max(1, (T - 1).bit_length())):
        see = ((see @ see) > 0).float()
    return see > 0


def _plain_attend(s):
    c = s["case"]
    L, B, H, G, D, T = (c[k] for k in ("L", "B", "H", "G", "D", "T"))
    P = c["P"]
    k = torch.cat([_values(s["k_cache"][:, :, :, :P], s["k_scale"][:, :, :, :P]), _rounded(s["k_tree"])], 3)
    x = _rounded(s["q"]).reshape(L, B, H, G * T, D) @ k.transpose(-1, -2) / math.sqrt(D)
    del k
    x = x.view(L, B, H, G, T, P + T)
    x[..., :P].masked_fill_((torch.arange(P, device=DEV) >= s["prefix_len"][:, None])[:, None, None, None], -math.inf)
    x[..., P:].masked_fill_(~_visible(s["parent"])[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    v = torch.cat([_values(s["v_cache"][:, :, :, :P], s["v_scale"][:, :, :, :P]), _rounded(s["v_tree"])], 3)
    out = (x.view(L, B, H, G * T, P + T) @ v).view(L, B, H, G, T, D) / l
    lse = (m + l.log()).view(L, B, H * G, T)
    return {"out": out.view(L, B, H * G, T, D).to(torch.bfloat16), "lse": lse, "status": torch.zeros_like(s["status"])}


def _plain_append(s):
    c = s["case"]
    n, S = c["n"], c["S"]
    b = torch.arange(c["B"], device=DEV)[:, None]
    slot = s["start"].long()[:, None] + torch.arange(n, device=DEV)   # [B, n]
    r = {"status": torch.zeros_like(s["status"])}
    for k in ("k", "v"):
        x = s[k + "_new"][:, :, :, :n]
        if s["rows"] is not None:
            rows = s["rows"][:, :n].long()
            x = torch.gather(s[k + "_new"], 3, rows[None, :, None, :, None].expand(c["L"], -1, c["H"], -1, c["D"]))
        codes, scales = _quantise(x)
        s[k + "_cache"].permute(1, 3, 0, 2, 4)[b, slot] = codes.permute(1, 3, 0, 2, 4)
        s[k + "_scale"].permute(1, 3, 0, 2, 4)[b, slot] = scales.permute(1, 3, 0, 2, 4)
        at = slot[None, :, None, :, None]
        back = [torch.gather(s[k + p], 3, at.expand(c["L"], -1, c["H"], -1, w)) for p, w in (("_cache", c["D"] // 2), ("_scale", c["D"] // 32))]
        r[k + "_back"] = _values(*back).to(torch.bfloat16)
    return r


def _plain_weigh(s):
    c = s["case"]
    L, B, H, G, D, T, S, n = (c[k] for k in ("L", "B", "H", "G", "D", "T", "S", "n"))
    at = s["path"][:, :n].long().clamp(min=0)
    pick = lambda x: torch.gather(x, 3, at[None, :, None, :, None].expand(L, -1, x.shape[2], -1, x.shape[4]))  # noqa: E731
    real = (torch.arange(n, device=DEV) < s["accept_len"][:, None])[:, None, None, :, None]   # [B, 1, 1, n, 1]
    q = pick(_rounded(s["q"])).view(L, B, H, G * n, D)
    lse = pick(s["lse"][..., None]).view(L, B, H, G, n, 1)
    k = s["k_cache"].float() if s["k_scale"] is None else _values(s["k_cache"], s["k_scale"])
    x = (q @ k.transpose(-1, -2)).view(L, B, H, G, n, S) / math.sqrt(D)
    old = torch.where(real, (x - lse).exp(), 0.0).sum((3, 4))
    x = (q @ pick(_rounded(s["k_tree"])).transpose(-1, -2)).view(L, B, H, G, n, n) / math.sqrt(D)
    new = torch.where(real & (torch.arange(n, device=DEV)[:, None] >= torch.arange(n, device=DEV)), (x - lse).exp(), 0.0).sum((3, 4))
    j = torch.arange(S, device=DEV) - s["prefix_len"][:, None]   # [B, S]: the row's place after the prefix
    new = torch.gather(new, 3, j.clamp(0, n - 1)[None, :, None].expand(L, -1, H, -1))
    j, m = j[:, None], s["accept_len"][:, None, None]
    s["weight"].copy_(torch.where(j < 0, s["weight"] + old, torch.where(j < m, new, s["weight"])))
    return {"weight": s["weight"]}


def _plain_evict(s):
    S, budget = s["weight"].shape[3], s["budget"]
    j, n = torch.arange(S, device=DEV), s["prefix_len"].long()[:, None, None]   # [B, 1, 1]
    w = torch.where((j < s["sink"]) | (j >= n - s["recent"]), math.inf, s["weight"])
    w = torch.where(j < n, w, -math.inf)
    kept = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]
    i = torch.arange(budget, device=DEV)
    kept = torch.sort(torch.where(i < n, kept, S), -1).values
    real, at = kept < S, kept.clamp(max=S - 1)
    r = {"kept": torch.where(real, kept, -1).int(), "new_len": s["prefix_len"].clamp(max=budget), "status": torch.zeros_like(s["status"])}
    for x, o in zip(s["planes"], s["out_planes"]):
        o.copy_(torch.where(real[..., None], torch.gather(x, 3, at[..., None].expand(-1, -1, -1, -1, x.shape[4])), o))
    s["out_weight"].copy_(torch.where(real, torch.gather(s["weight"], 3, at), s["out_weight"]))
    return dict(r, planes=s["out_planes"], weight=s["out_weight"])


def _plain_verify(s):
    # the walk is one node after another by its nature: node i is tested where its parent is
    # the last accepted node, what an earlier sibling's rejection leaves in hand
    B, T, V = s["logits"].shape
    b = torch.arange(B, device=DEV)
    probs = lambda x: torch.exp((x - x.amax(-1, keepdim=True)) / TEMPERATURE)  # noqa: E731
    left = probs(s["logits"][:, 0])
    z = left.sum(-1)
    cur = torch.zeros(B, dtype=torch.int64, device=DEV)
    length = torch.ones(B, dtype=torch.int64, device=DEV)
    path = torch.full((B, T), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    tested = torch.full((B, T), -1.0, device=DEV)
    for i in range(1, T):
        token = s["cand"][:, i].long()
        here = (s["parent"][:, i] == cur) & (token >= 0)
        t = token.clamp(min=0)
        p = left[b, t] / z
        if s["draft_probs"] is not None:
            q = s["draft_probs"][b, s["draft_row"][:, i].long()]
            p = torch.where(q[b, t] > 0, p / q[b, t], 0.0)
        p = p.clamp(max=1.0)
        tested[:, i] = torch.where(here, p, -1.0)
        good = here & (s["u"][:, i] < p)
        bad = here & ~good
        if s["draft_probs"] is not None:
            rest = (left / z[:, None] - q).clamp(min=0.0)
        else:
            rest = left.clone()
            rest[b, t] = 0.0
        left = torch.where(good[:, None], probs(s["logits"][:, i]), torch.where(bad[:, None], rest, left))
        z = left.sum(-1)
        path[b, length.clamp(max=T - 1)] = torch.where(good, i, path[b, length.clamp(max=T - 1)])
        length = length + good
        cur = torch.where(good, i, cur)
    # where rejections left nothing, the whole distribution
    left = torch.where((z > 0)[:, None], left, probs(s["logits"][b, cur]))
    return {"accept_len": length.int(), "path": path.int(), "next_token": torch.argmax(left / s["noise"], -1).int(),
            "new_len": (s["prefix_len"] + length).int(), "status": torch.zeros_like(s["status"]), "accept_prob": tested}


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "weigh": _plain_weigh, "evict": _plain_evict, "verify": _plain_verify}[kind](s)
    from paper_2405_18628_gb300 import ppd
    if kind == "attend":
        ppd.ppd_tree_attention_kv4(s["q"], s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"], s["k_tree"], s["v_tree"],
                                   s["prefix_len"], s["parent"], s["out"], s["status"], lse=s["lse"], workspace=s["workspace"])
        return {k: s[k] for k in ("out", "lse", "status")}
    if kind == "append":
        ppd.ppd_kv4_append(s["k_new"], s["v_new"], s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"], s["start"], s["n_new"],
                           s["status"], rows=s["rows"])
        for k in ("k", "v"):
            ppd.ppd_kv4_read(s[k + "_cache"], s[k + "_scale"], s["start"], s["n_new"], s[k + "_back"])
        return {k: s[k] for k in ("k_back", "v_back", "status")}
    if kind == "weigh":
        ppd.ppd_kv_weight_add(s["q"], s["lse"], s["k_cache"], s["k_tree"], s["path"], s["accept_len"], s["prefix_len"], s["weight"],
                              k_scale=s["k_scale"])
        return {"weight": s["weight"]}
    if kind == "evict":
        ppd.ppd_kv_evict(s["weight"], s["planes"], s["prefix_len"], s["budget"], s["sink"], s["recent"], s["kept"], s["new_len"],
                         s["status"], out_weight=s["out_weight"], out_planes=s["out_planes"])
        return dict({k: s[k] for k in ("kept", "new_len", "status")}, planes=s["out_planes"], weight=s["out_weight"])
    ppd.ppd_sample_accept(s["logits"], s["cand"], s["parent"], s["prefix_len"], s["case"]["S"], TEMPERATURE, s["u"], s["noise"],
                          s["accept_len"], s["path"], s["next_token"], s["new_len"], s["status"], draft_probs=s["draft_probs"],
                          draft_row=s["draft_row"], accept_prob=s["accept_prob"])
    return {k: s[k] for k in ("accept_len", "path", "next_token", "new_len", "status", "accept_prob")}


def work(case):
    """Each input read once, each output written once; of a cache the valid rows, of logits the
    rows of the nodes that are visited (about three a sequence) and the draft rows of a
    rejection each."""
    c = case
    L, B, H, G, D, T, n, V = (c[k] for k in ("L", "B", "H", "G", "D", "T", "n", "V"))
    eb = 2 if c["dtype"] == "bf16" else 4
    keys = L * H * sum(_lens(c))
    row4 = D // 2 + D // 32
    row = row4 if c["cache"] == "kv4" else 2 * D
    if c["kind"] == "attend":
        return {"bytes": keys * 2 * row4 + L * B * H * T * (2 * D * eb + G * (D * (eb + 2) + 4)),
                "flops": 4 * D * T * G * (keys + 6 * L * B * H)}
    if c["kind"] == "append":
        return {"bytes": 2 * L * B * H * n * (D * eb + 2 * row4 + 2 * D), "flops": 8 * L * B * H * n * D}
    if c["kind"] == "weigh":
        return {"bytes": keys * (row + 8) + L * B * H * n * D * (2 + 2 * G), "flops": 2 * D * n * G * keys}
    if c["kind"] == "evict":
        new = L * H * sum(min(x, c["budget"]) for x in _lens(c))
        return {"bytes": 4 * keys + new * (2 * 2 * row + 4 + 4), "flops": keys}
    rows = B * (3 + 1 + (2 if c["draft"] else 0))
    return {"bytes": 4 * rows * V + 24 * B * T, "flops": 4 * rows * V}


# ------------------------------------------------------------------ 64-bit results

def _scales64():
    return torch.tensor([(8 + b % 8) * 2.0 ** (b // 8 - 23) for b in range(256)], dtype=torch.float64, device=DEV)


def _row64(codes, scales):
    """The 64-bit values of rows [..., D / 2], [..., D / 32]: byte k of a word holds the
    channels (0, 2), (4, 6), (1, 3), (5, 7)."""
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=DEV)
    for k, (lo, hi) in enumerate(((0, 2), (4, 6), (1, 3), (5, 7))):
        out[..., lo::8] = (codes[..., k::4] % 16).double() - 8
        out[..., hi::8] = torch.div(codes[..., k::4], 16, rounding_mode="floor").double() - 8
    return out * _scales64()[scales.long()].repeat_interleave(32, -1)


def _ancestors64(parent):
    out = np.eye(len(parent), dtype=bool)
    for i in range(1, len(parent)):
        out[i] |= out[parent[i]]
    return torch.from_numpy(out).to(DEV)


def _exact_attend(c, s):
    f = lambda x: x.to(torch.bfloat16).double()  # noqa: E731
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:-1], dtype=torch.float64, device=DEV)
    G, T = c["G"], c["T"]
    for b, P in enumerate(_lens(c)):
        see = _ancestors64(s["parent"][b].tolist()).repeat(G, 1)
        for l in range(c["L"]):
            k, v = (torch.cat([_row64(s[x + "_cache"][l, b, :, :P], s[x + "_scale"][l, b, :, :P]), f(s[x + "_tree"][l, b])], 1) for x in "kv")
            x = f(s["q"][l, b]).view(c["H"], G * T, -1) @ k.transpose(1, 2) / math.sqrt(c["D"])
            x[:, :, P:].masked_fill_(~see, -math.inf)
            lse[l, b] = torch.logsumexp(x, -1).view(-1, T)
            out[l, b] = (torch.softmax(x, -1) @ v).view(-1, T, c["D"])
    return {"out": out, "lse": lse, "status": torch.zeros_like(s["status"])}


def _exact_append(c, s):
    r = {"status": torch.zeros_like(s["status"])}
    table = _scales64()
    for k in ("k", "v"):
        x = s[k + "_new"].double()
        if s["rows"] is None:
            x = x[:, :, :, :c["n"]]
        else:
            x = torch.stack([x[:, b][:, :, s["rows"][b, :c["n"]].long()] for b in range(c["B"])], 1)
        x = x.unflatten(-1, (-1, 32))
        scale = table[torch.searchsorted(table, x.abs().amax(-1) / 7).clamp(max=255)][..., None]
        r[k + "_back"] = (torch.round(x / scale).clamp(-7, 7) * scale).flatten(-2)
    return r


def _exact_weigh(c, s):
    w = s["weight"].double()
    G = c["G"]
    for b, P in enumerate(_lens(c)):
        path = [i for i in s["path"][b].tolist() if i >= 0]
        m, at = len(path), torch.tensor(path, device=DEV)
        for l in range(c["L"]):
            k = s["k_cache"][l, b, :, :P].double() if s["k_scale"] is None else _row64(s["k_cache"][l, b, :, :P], s["k_scale"][l, b, :, :P])
            k = torch.cat([k, s["k_tree"][l, b][:, at].double()], 1)
            x = s["q"][l, b][:, at].double().view(c["H"], G * m, -1) @ k.transpose(1, 2) / math.sqrt(c["D"])
            x = torch.exp(x - s["lse"][l, b][:, at].double().reshape(c["H"], G * m, 1))
            x[:, :, P:] *= torch.ones(m, m, dtype=torch.float64, device=DEV).tril().repeat(G, 1)
            w[l, b, :, :P] += x[:, :, :P].sum(1)
            w[l, b, :, P:P + m] = x[:, :, P:].sum(1)
    return {"weight": w}


def _exact_verify(c, s):
    tested = torch.full((c["B"], c["T"]), -1.0, dtype=torch.float64)
    for b in range(c["B"]):
        parent, cand, u = (s[k][b].tolist() for k in ("parent", "cand", "u"))
        row = lambda i: torch.softmax(s["logits"][b, i].double() / TEMPERATURE, -1)  # noqa: E731
        cur, p = 0, row(0)
        for i in range(1, c["T"]):
            if parent[i] != cur or cand[i] < 0:
                continue
            if s["draft_probs"] is None:
                a = float(p[cand[i]])
            else:
                q = s["draft_probs"][b, int(s["draft_row"][b, i])].double()
                a = min(1.0, float(p[cand[i]] / q[cand[i]])) if q[cand[i]] > 0 else 0.0
            tested[b, i] = a
            if u[i] < a:
                cur, p = i, row(i)
                continue
            if s["draft_probs"] is None:
                p[cand[i]] = 0
            else:
                p = (p - q).clamp(min=0)
            p = p / p.sum()
    return {"accept_len": None, "path": None, "next_token": None, "new_len": None, "status": None, "accept_prob": tested}


def exact(case, seed):
    if case["kind"] == "evict":
        return None   # rows are copied: nothing is computed
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "weigh": _exact_weigh, "verify": _exact_verify}[case["kind"]](case, s)
