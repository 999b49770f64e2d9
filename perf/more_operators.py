"""Operators of a decode step for many requests whose caches share one pool of pages:

  assign    pages for rows that requests gain, and back to the pool for rows that they lose:
            block tables, the stack of free pages and the slots of the new rows
  append    rows of K and V into their slots: accepted paths, or prompts of several lengths
  attend    the attention of token trees (or of single new tokens) over the requests' pages and
            their own ancestors, query heads sharing K/V heads
  logprobs  log probabilities of given tokens, with entropy, rank and the top alternatives

Sizes: L layers, B requests, H key/value heads, G query heads for each, head dim D, pages of
`page` rows, tables of M pages a request, cached rows P (the longest; the others down to half of
it), trees of T tokens, vocabulary V, n asked tokens a request, K alternatives.

A pool is [L, N, H, page, D], bf16, for K and for V; a page number is the same in every layer.  A
request's row j is row j % page of its page number j // page; its slot is page number * page + row.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TEMPERATURE = 0.8


def case(name, kind, L=1, B=1, H=1, G=1, D=128, P=64, T=1, page=16, n=1, V=0, K=0, dtype="bf16", **more):
    c = dict(kind=kind, L=L, B=B, H=H, G=G, D=D, P=P, T=T, page=page, n=n, V=V, K=K, dtype=dtype, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request's new token, one layer's call: latency is all there is
        case("attend_token_one", "attend", 1, 1, 8, 4, 128, 515, 1, 16, spare=0),
        # decoding of a large batch, one layer's call, tables twice as long as the longest request
        case("attend_token_batch", "attend", 1, 48, 8, 4, 128, 8192, 1, 16, spare=8192),
        # verification of 64-token trees with shared K/V heads, odd lengths
        case("attend_tree_gqa", "attend", 2, 6, 8, 4, 128, 5001, 64, 32, spare=0),
        # long contexts, small trees, fp32 projections, D = 64, large pages: the largest
        case("attend_long_f32", "attend", 4, 3, 16, 1, 64, 30001, 17, 128, dtype="f32", spare=2000),
        # a decode step of 64 requests: most gain a few rows, some end, some start
        case("assign_step", "assign", B=64, P=16384, page=16, kind_of="step"),
        # a wave of 512 requests: prompts come in, old requests go
        case("assign_prompts", "assign", B=512, P=4096, page=16, kind_of="prompts"),
        # accepted paths of up to six nodes enter every layer's pages
        case("append_paths", "append", 32, 8, 8, 1, 128, 200, 64, 16, n=6),
        # prompts of several odd lengths, kept in fp32, D = 64
        case("append_prompts_f32", "append", 8, 3, 16, 1, 64, 0, 1003, 64, n=1003, dtype="f32"),
        # the next token's alternatives of one request, an odd vocabulary
        case("logprobs_one", "logprobs", V=50257, K=5),
        # the tokens of accepted paths, padded to six a request
        case("logprobs_paths", "logprobs", B=8, T=64, n=6, V=32000, K=5, path=True),
        # every token of four pieces of prompt, bf16 logits of a large vocabulary
        case("logprobs_prompt", "logprobs", B=4, T=512, n=512, V=128256, K=20, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "assign", "append", "logprobs", "logprobs"])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    if kind == "assign":
        B = _log_int(rng, 1, 1024)
        return case(None, kind, B=B, P=_log_int(rng, 16, min(32768, 2000000 // B)), page=page, kind_of=rng.choice(["step", "prompts"]))
    if kind == "logprobs":
        V = rng.choice([1000, 32000, 32003, 50257, 128256, 151937, 256000])
        n = _log_int(rng, 1, 512)
        B = _log_int(rng, 1, max(1, min(128, int(2.6e8 / (V * n)))))
        path = n > 1 and rng.random() < 0.5
        return case(None, kind, B=B, T=min(512, n + rng.choice([0, 1, 40])) if path else n, n=n, V=V, K=rng.choice([0, 1, 5, 20, 32]),
                    dtype=rng.choice(["f32", "bf16"]), path=path)
    D = rng.choice([64, 128, 128])
    H = rng.choice([1, 2, 4, 8, 16, 32, 40])
    G = rng.choice([1, 2, 3, 4, 8]) if H <= 16 else 1
    B = 1 if rng.random() < 0.3 else _log_int(rng, 2, 128)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    # (layer, request, head, row) in all
    rows = 1.1e9 / (4 * D)
    if kind == "append":
        T = _log_int(rng, 1, 2000)
        n = T if T > 512 or rng.random() < 0.5 else _log_int(rng, 1, min(T, 12))
        rows /= 4
        B = max(1, min(B, int(rows / (H * (T + 64)))))
        L = max(1, min(_log_int(rng, 1, 32), int(rows / (B * H * (T + 64)))))
        return case(None, kind, L, B, H, 1, D, _log_int(rng, 1, 300), T, page, n=n, dtype=dtype)
    T = 1 if rng.random() < 0.4 else _log_int(rng, 2, 512)
    P, L, spare = _log_int(rng, 1, 65536), _log_int(rng, 1, 16), rng.choice([0, 0, 1, 500, 9000])
    while True:
        c = case(None, kind, L, B, H, G, D, P, T, page, dtype=dtype, spare=spare)
        w = work(c)
        if w["bytes"] <= 1.1e9 and w["flops"] <= 3e11:
            return c
        # fewer layers, then fewer requests, then fewer rows
        L, B, P = (max(1, L * 2 // 3), B, P) if L > 1 else (L, max(1, B * 2 // 3), P) if B > 1 else (L, B, P * 2 // 3)


# ------------------------------------------------------------------ inputs

def _lens(c):
    """Cached rows of each request: P, or down to half of it."""
    return [c["P"] - (b * 7919) % (c["P"] // 2 + 1) for b in range(c["B"])]


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _pages(rows, page):
    return (rows + page - 1) // page


def _tree(rng, T):
    """Parents of a tree: a quarter of its nodes (root included) are guesses at most six deep,
    chains of up to three prompt tokens fill the rest."""
    n = max(1, (T + 3) // 4)
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = rng.randrange(i)
        while depth[p] >= 6:
            p = rng.randrange(i)
        parent.append(p)
        depth.append(depth[p] + 1)
    anchor, left = 0, 0
    while len(parent) < T:
        parent.append(anchor % n if left == 0 else len(parent) - 1)
        anchor, left = (anchor + 1, 2) if left == 0 else (anchor, left - 1)
    return parent


def _table(rng, lens, page, M, N):
    """Tables of requests of these lengths over N pages in any order, -1 past their ends; the pages left."""
    need = [_pages(x, page) for x in lens]
    ids = np.random.default_rng(rng.randrange(1 << 30)).permutation(N).astype(np.int32)
    table = np.full((len(lens), M), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, ids[at:]


def prepare(case, seed):
    c = case
    L, B, H, G, D, T, page, n, V, K = (c[k] for k in ("L", "B", "H", "G", "D", "T", "page", "n", "V", "K"))
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 29)
    rng = random.Random(seed * 7919 + 11)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    normal = lambda *shape, dtype=dt: torch.randn(shape, dtype=dtype, device=DEV, generator=g)  # noqa: E731
    empty = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    s = dict(case=c, status=empty(torch.int32, B))
    if c["kind"] == "assign":
        old = [0] * B
        new = [0] * B
        for b in range(B):
            at = rng.randint(1, c["P"])
            if c["kind_of"] == "prompts":
                old[b], new[b] = (at, 0) if rng.random() < 0.2 else (0, at)
            elif rng.random() < 0.06:
                old[b], new[b] = (at, 0) if rng.random() < 0.5 else (0, min(at, 2000))
            else:
                old[b], new[b] = at, min(c["P"], at + rng.randint(1, 6))
        # a pool and a slot map that hold every request at its longest
        M, cap = _pages(c["P"], page), B * c["P"]
        N = B * M + 5
        table, free = _table(rng, old, page, M, N)
        stack = np.full(N, -1, np.int32)
        stack[:len(free)] = free
        s.update(old=_i32(old), new=_i32(new), table=torch.from_numpy(table).to(DEV), free=torch.from_numpy(stack).to(DEV), n_free=_i32([len(free)]),
                 status_back=empty(torch.int32, B))
        for k in ("n_mid", "n_back"):
            s[k] = empty(torch.int32, 1)
        for k in ("mid_len", "back_len"):
            s[k] = empty(torch.int32, B)
        for k in ("slots", "slots_back"):
            s[k] = torch.full((cap,), -1, dtype=torch.int32, device=DEV)
        for k in ("start", "start_back"):
            s[k] = empty(torch.int32, B + 1)
        return s
    if c["kind"] == "logprobs":
        s["logits"] = torch.empty(B, T, V, dtype=dt, device=DEV)
        for b in range(B):
            s["logits"][b] = 3.0 * torch.randn(T, V, device=DEV, generator=g)
        # tokens that the grammar of an answer forbids
        s["logits"][:, :, torch.randperm(V, device=DEV, generator=g)[:V // 16]] = -math.inf
        if c.get("path"):
            path = [sorted(rng.sample(range(T), rng.randint(1, n))) for _ in range(B)]
            s["rows"] = _i32([p + [-1] * (n - len(p)) for p in path])
        else:
            s["rows"] = None
        at = torch.arange(n, device=DEV).expand(B, n) if s["rows"] is None else s["rows"].long()
        # half are the best token, half any that is allowed
        best = torch.gather(s["logits"].argmax(-1), 1, at.clamp(min=0))
        some = torch.randint(0, V, (B, n), device=DEV, generator=g)
        free = s["logits"][0, 0][some] > -math.inf
        s["tokens"] = torch.where(at < 0, -1, torch.where(free & (torch.rand(B, n, device=DEV, generator=g) < 0.5), some, best)).int()
        s.update(logprob=empty(torch.float32, B, n), entropy=empty(torch.float32, B, n), rank=empty(torch.int32, B, n))
        s["top"] = (empty(torch.int32, B, n, K), empty(torch.float32, B, n, K)) if K else (None, None)
        return s
    if c["kind"] == "append":
        count = [rng.randint((n + 1) // 2, n) for _ in range(B)]
        start = [0 if n == T and T > 1 else x for x in _lens(c)]
        M = max(_pages(x + n, page) for x in start)
        N = B * M + 3
        table, _ = _table(rng, [x + k for x, k in zip(start, count)], page, M, N)
        slots = [int(table[b, j // page]) * page + j % page for b in range(B) for j in range(start[b], start[b] + count[b])]
        s.update(slots=_i32(slots), start=_i32(np.concatenate([[0], np.cumsum(count)])))
        s["rows"] = None if n == T else _i32([sorted(rng.sample(range(T), k)) + [-1] * (T - k) for k in count])
        s.update(k_new=normal(L, B, H, T, D), v_new=normal(L, B, H, T, D))
        s["k_pages"], s["v_pages"] = (torch.zeros(L, N, H, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return s
    lens = _lens(c)
    M = _pages(c["P"] + c["spare"], page)
    N = sum(_pages(x, page) for x in lens) + 2
    table, _ = _table(rng, lens, page, M, N)
    s.update(table=torch.from_numpy(table).to(DEV), prefix_len=_i32(lens), parent=_i32([_tree(rng, T) for _ in range(B)]))
    s["k_pages"], s["v_pages"] = (normal(L, N, H, page, D, dtype=torch.bfloat16) for _ in range(2))
    s.update(q=normal(L, B, H * G, T, D), k_tree=normal(L, B, H, T, D), v_tree=normal(L, B, H, T, D))
    s.update(out=empty(torch.bfloat16, L, B, H * G, T, D), lse=empty(torch.float32, L, B, H * G, T))
    # one scratch buffer serves a program's calls
    s["workspace"] = empty(torch.uint8, (64 << 20) + 2 * (s["q"].numel() + 2 * s["k_tree"].numel()))
    return s


# ------------------------------------------------------------------ plain forms

def _plain_assign_one(page, old, new, table, free, n_free, cap, slots):
    """Pages for rows [old, new) of each request, or back for rows [new, old): the tables and the
    stack in place.  All that is given back is pushed in order, then all that is needed is
    taken from the top, its order kept."""
    B, M = table.shape
    N = free.shape[0]
    held, want = (old + page - 1) // page, (new + page - 1) // page
    need, rows = (want - held).clamp(min=0), (new - old).clamp(min=0)
    j = torch.arange(M, device=DEV)
    back = (j >= want[:, None]) & (j < held[:, None])                                     # [B, M]
    given = back.sum()
    ok = ((torch.cumsum(need, 0) <= n_free + given) | (need == 0)) & ((torch.cumsum(rows, 0) <= cap) | (rows == 0))
    take = (j >= held[:, None]) & (j < want[:, None]) & ok[:, None]
    order = lambda m: torch.cumsum(m.flatten().int(), 0).view(B, M) - 1                    # noqa: E731
    stack = torch.cat([free, free.new_zeros(1)])
    stack[torch.where(back, n_free + order(back), N).flatten().long()] = table.flatten()
    left = n_free + given - take.sum()
    table.copy_(torch.where(take, stack[(left + order(take)).clamp(0, N).flatten().long()].view(B, M), table))
    free.copy_(torch.where(torch.arange(N, device=DEV) < left, stack[:N], free))
    start = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    start[1:] = torch.cumsum(torch.where(ok, rows, 0), 0)
    i = torch.arange(slots.shape[0], dtype=torch.int32, device=DEV)
    b = (torch.searchsorted(start, i, right=True) - 1).clamp(max=B - 1)
    at = (old[b] + i - start[b]).clamp(0, M * page - 1)
    slots.copy_(torch.where(i < start[B], table[b, (at // page).long()] * page + at % page, slots))
    return dict(length=torch.where(ok, new, old), n_free=left.int().view(1), start=start, status=torch.where(ok, 0, 4).int())


def _plain_assign(s):
    page, cap = s["case"]["page"], s["slots"].shape[0]
    f = _plain_assign_one(page, s["old"], s["new"], s["table"], s["free"], s["n_free"], cap, s["slots"])
    r = _plain_assign_one(page, f["length"], s["old"], s["table"], s["free"], f["n_free"], cap, s["slots_back"])
    return dict(table=s["table"], free=s["free"], slots=s["slots"], slots_back=s["slots_back"], there=f, back=r)


def _plain_append(s):
    c = s["case"]
    N = s["k_pages"].shape[1]
    B, page = c["B"], c["page"]
    i = torch.arange(s["slots"].shape[0], dtype=torch.int32, device=DEV)
    b = torch.searchsorted(s["start"], i, right=True) - 1
    j = (i - s["start"][b]).long()
    if s["rows"] is not None:
        j = s["rows"][b, j].long()
    slot = s["slots"].long()
    for k in ("k", "v"):
        new = s[k + "_new"].float().to(torch.bfloat16)
        s[k + "_pages"].permute(1, 3, 0, 2, 4)[slot // page, slot % page] = new.permute(1, 3, 0, 2, 4)[b, j]
    return dict(k=s["k_pages"], v=s["v_pages"], status=torch.zeros_like(s["status"]))


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
    B, H, G, D, T, P, page = (c[k] for k in ("B", "H", "G", "D", "T", "P", "page"))
    m = _pages(P, page)
    at = s["table"][:, :m].long().clamp(min=0)
    hidden = (torch.arange(m * page, device=DEV) >= s["prefix_len"][:, None])[:, None, None, None]
    unseen = ~_visible(s["parent"])[:, None, None]
    for l in range(c["L"]):
        k, v = (torch.cat([s[x + "_pages"][l][at].permute(0, 2, 1, 3, 4).reshape(B, H, m * page, D).float(), _rounded(s[x + "_tree"][l])], 2) for x in "kv")
        x = _rounded(s["q"][l]).reshape(B, H, G * T, D) @ k.transpose(-1, -2) / math.sqrt(D)
        x = x.view(B, H, G, T, m * page + T)
        x[..., :m * page].masked_fill_(hidden, -math.inf)
        x[..., m * page:].masked_fill_(unseen, -math.inf)
        top = x.amax(-1, keepdim=True)
        x = x.sub_(top).exp_()
        z = x.sum(-1, keepdim=True)
        s["out"][l] = ((x.view(B, H, G * T, -1) @ v).view(B, H, G, T, D) / z).view(B, H * G, T, D).to(torch.bfloat16)
        s["lse"][l] = (top + z.log()).view(B, H * G, T)
    return dict(out=s["out"], lse=s["lse"], status=torch.zeros_like(s["status"]))


def _plain_logprobs(s):
    c = s["case"]
    B, n, K = c["B"], c["n"], c["K"]
    x = s["logits"]
    live = torch.ones(B, n, dtype=torch.bool, device=DEV)
    if s["rows"] is not None:
        live = s["rows"] >= 0
        x = x[torch.arange(B, device=DEV)[:, None], s["rows"].long().clamp(min=0)]
    x = x.float()
    t = s["tokens"].long().clamp(min=0)[..., None]
    y = x / TEMPERATURE
    top = y.amax(-1, keepdim=True)
    e = torch.exp(y - top)
    z = e.sum(-1, keepdim=True)
    lse = top + z.log()
    entropy = (z.log() - (e * torch.where(e > 0, y - top, 0.0)).sum(-1, keepdim=True) / z)[..., 0]
    xt = torch.gather(x, 2, t)
    rank = ((x > xt) | ((x == xt) & (torch.arange(c["V"], device=DEV) < t))).sum(-1)
    logprob = (xt / TEMPERATURE - lse)[..., 0]
    r = dict(logprob=torch.where(live, logprob, 0.0), entropy=torch.where(live, entropy, 0.0), rank=torch.where(live, rank, -1).int(),
             status=torch.zeros_like(s["status"]))
    if K:
        ids, best = [], []
        x = x.clone() if x is s["logits"] else x
        for _ in range(K):
            i = x.argmax(-1, keepdim=True)      # the first of the largest
            best.append(torch.gather(x, 2, i) / TEMPERATURE - lse)
            ids.append(i)
            x.scatter_(2, i, -math.inf)
        r["top_tokens"] = torch.where(live[..., None], torch.cat(ids, -1), -1).int()
        r["top_logprobs"] = torch.where(live[..., None], torch.cat(best, -1), 0.0)
    return r


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"assign": _plain_assign, "append": _plain_append, "attend": _plain_attend, "logprobs": _plain_logprobs}[kind](s)
    from paper_2405_18628_gb300 import ppd
    if kind == "assign":
        # pages are reserved, then given back: the pool is as it was
        ppd.ppd_page_assign(s["old"], s["new"], s["case"]["page"], s["table"], s["free"], s["n_free"], s["n_mid"], s["mid_len"], s["slots"], s["start"],
                            s["status"])
        ppd.ppd_page_assign(s["mid_len"], s["old"], s["case"]["page"], s["table"], s["free"], s["n_mid"], s["n_back"], s["back_len"], s["slots_back"],
                            s["start_back"], s["status_back"])
        return dict(table=s["table"], free=s["free"], slots=s["slots"], slots_back=s["slots_back"],
                    there=dict(length=s["mid_len"], n_free=s["n_mid"], start=s["start"], status=s["status"]),
                    back=dict(length=s["back_len"], n_free=s["n_back"], start=s["start_back"], status=s["status_back"]))
    if kind == "append":
        ppd.ppd_page_append(s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["slots"], s["start"], s["status"], rows=s["rows"])
        return dict(k=s["k_pages"], v=s["v_pages"], status=s["status"])
    if kind == "attend":
        ppd.ppd_tree_attention_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["k_tree"], s["v_tree"], s["prefix_len"], s["parent"], s["out"],
                                     s["status"], lse=s["lse"], workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"], status=s["status"])
    ids, best = s["top"]
    ppd.ppd_token_logprobs(s["logits"], s["tokens"], TEMPERATURE, s["logprob"], s["entropy"], s["rank"], s["status"], rows=s["rows"], top_tokens=ids,
                           top_logprobs=best)
    r = dict(logprob=s["logprob"], entropy=s["entropy"], rank=s["rank"], status=s["status"])
    return dict(r, top_tokens=ids, top_logprobs=best) if ids is not None else r


def work(case):
    """Each input read once, each output written once; of pages the valid rows, of logits the asked
    rows (about half of a padded path's)."""
    c = case
    L, B, H, G, D, T, n, V, K, page = (c[k] for k in ("L", "B", "H", "G", "D", "T", "n", "V", "K", "page"))
    eb = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "assign":
        # a row's slot; a page's number out of the stack and into the table, there and back
        rows = B * (0.4 * c["P"] if c["kind_of"] == "prompts" else 4 + 0.03 * min(c["P"], 2000) / 2)
        return {"bytes": int(rows * 4 + 4 * rows / page * 4 + 2 * B * 20), "flops": int(4 * rows)}
    if c["kind"] == "append":
        return {"bytes": int(2 * L * B * H * 0.75 * n * D * (eb + 2)), "flops": int(2 * L * B * H * n * D)}
    if c["kind"] == "attend":
        keys = L * H * sum(_lens(c))
        return {"bytes": keys * 4 * D + 4 * sum(_pages(x, page) for x in _lens(c)) + L * B * H * T * (2 * D * eb + G * (D * (eb + 2) + 4)),
                "flops": 4 * D * T * G * (keys + 6 * L * B * H)}
    rows = B * ((n + 1) / 2 if c.get("path") else n)
    return {"bytes": int(rows * V * eb + B * n * (16 + 8 * K)), "flops": int(6 * rows * V)}


# ------------------------------------------------------------------ 64-bit results

def _ancestors64(parent):
    out = np.eye(len(parent), dtype=bool)
    for i in range(1, len(parent)):
        out[i] |= out[parent[i]]
    return torch.from_numpy(out).to(DEV)


def _exact_attend(c, s):
    f = lambda x: x.to(torch.bfloat16).double()  # noqa: E731
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:-1], dtype=torch.float64, device=DEV)
    H, G, T, D = (c[k] for k in ("H", "G", "T", "D"))
    for b, P in enumerate(_lens(c)):
        see = _ancestors64(s["parent"][b].tolist()).repeat(G, 1)
        ids = s["table"][b, :_pages(P, c["page"])].long()
        for l in range(c["L"]):
            k, v = (torch.cat([s[x + "_pages"][l].index_select(0, ids).transpose(0, 1).flatten(1, 2)[:, :P].double(), f(s[x + "_tree"][l, b])], 1) for x in "kv")
            for h in range(H):   # a head at a time: large trees over long caches fit the memory
                x = f(s["q"][l, b, h * G:(h + 1) * G]).view(G * T, D) @ k[h].T / math.sqrt(D)
                x[:, P:].masked_fill_(~see, -math.inf)
                lse[l, b, h * G:(h + 1) * G] = torch.logsumexp(x, -1).view(G, T)
                out[l, b, h * G:(h + 1) * G] = (torch.softmax(x, -1) @ v[h]).view(G, T, D)
    return dict(out=out, lse=lse, status=torch.zeros_like(s["status"]))


def _exact_append(c, s):
    """The rows as they were given, where their slots say."""
    r = dict(status=torch.zeros_like(s["status"]))
    first = s["start"].tolist()
    for x in "kv":
        pool = s[x + "_pages"].double()
        for b in range(c["B"]):
            slot = s["slots"][first[b]:first[b + 1]].long()
            rows = s[x + "_new"][:, b]
            rows = rows[:, :, :len(slot)] if s["rows"] is None else rows[:, :, s["rows"][b, :len(slot)].long()]
            for i, j in enumerate(slot.tolist()):
                pool[:, j // c["page"], :, j % c["page"]] = rows[:, :, i].double()
        r[x] = pool
    return r


def _exact_logprobs(c, s):
    B, n, K = c["B"], c["n"], c["K"]
    logprob, entropy = torch.zeros(B, n, dtype=torch.float64, device=DEV), torch.zeros(B, n, dtype=torch.float64, device=DEV)
    top = torch.zeros(B, n, K, dtype=torch.float64, device=DEV)
    for b in range(B):
        at = torch.arange(n, device=DEV) if s["rows"] is None else s["rows"][b].long()
        on = at >= 0
        p = torch.log_softmax(s["logits"][b, at[on]].double() / TEMPERATURE, -1)
        logprob[b, on] = p.gather(1, s["tokens"][b, on].long()[:, None])[:, 0]
        entropy[b, on] = -torch.where(p > -math.inf, p.exp() * p, 0.0).sum(-1)
        if K:
            top[b, on] = torch.topk(p, K, -1).values
    r = dict(logprob=logprob, entropy=entropy, rank=None, status=None)
    return dict(r, top_tokens=None, top_logprobs=top) if K else r


def exact(case, seed):
    if case["kind"] == "assign":
        return None   # page numbers: nothing is computed
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "logprobs": _exact_logprobs}[case["kind"]](case, s)
