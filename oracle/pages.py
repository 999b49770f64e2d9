"""Plain forms of the operators over a pool of pages: the definitions of include/ppd.h written
out, one sequence at a time, without the library's code."""
from __future__ import annotations

import math

import torch

from .operators import ancestors, bf16

OK, TREE, CAPACITY = 0, 3, 4


def pages_of(rows, page):
    return -(-rows // page)


def page_assign(old, new, page, table, stack, max_slots):
    """Lists of lengths, a table of lists, the stack as a list (its top last): table and stack are
    changed in place -> lengths, slots of each sequence (a list of lists), statuses."""
    limit = len(table[0]) * page
    fine = [0 <= o <= limit and 0 <= n <= limit for o, n in zip(old, new)]
    for b, (o, n) in enumerate(zip(old, new)):
        if fine[b]:
            stack += table[b][pages_of(n, page):max(pages_of(n, page), pages_of(o, page))]
    # who is served
    left, room, served = len(stack), max_slots, []
    for o, n, f in zip(old, new, fine):
        need, rows = (max(0, pages_of(n, page) - pages_of(o, page)), max(0, n - o)) if f else (0, 0)
        left, room = left - need, room - rows
        served.append(f and (need == 0 or left >= 0) and (rows == 0 or room >= 0))
    need = [max(0, pages_of(n, page) - pages_of(o, page)) if s else 0 for o, n, s in zip(old, new, served)]
    top = stack[len(stack) - sum(need):]
    del stack[len(stack) - sum(need):]
    slots = []
    for b, (o, n) in enumerate(zip(old, new)):
        for i in range(need[b]):
            table[b][pages_of(o, page) + i] = top.pop(0)
        slots.append([table[b][r // page] * page + r % page for r in range(o, n)] if served[b] else [])
    return [n if s else o for o, n, s in zip(old, new, served)], slots, [OK if s else CAPACITY for s in served]


def rows_of(pages, row_of_table, n):
    """The first n rows of a sequence: pages [n_pages,H,page,D] -> [H,n,D]."""
    n_pages, H, page, D = pages.shape
    ids = torch.tensor(row_of_table[:pages_of(n, page)], dtype=torch.long, device=pages.device)
    return pages[ids].transpose(0, 1).reshape(H, -1, D)[:, :n]


def attention(q, k_rows, v_rows, k_tree, v_tree, parent, scale=0.0):
    """One head's slice: q [G,T,D], rows [P,D], tree rows [T,D] -> out, lse, and sum p |v| and
    max_j scale sum |q k| (what roundings are measured against)."""
    G, T, D = q.shape
    P = k_rows.shape[0]
    scale = scale if scale > 0 else 1 / math.sqrt(D)
    k, v = torch.cat([k_rows.double(), bf16(k_tree)]), torch.cat([v_rows.double(), bf16(v_tree)])
    x = scale * (bf16(q) @ k.T)
    size = float((scale * (bf16(q).abs() @ torch.nan_to_num(k.abs()).T)).max())
    x[:, :, P:].masked_fill_(~ancestors(parent).to(x.device), -math.inf)
    p = torch.softmax(x, -1)
    return p @ v, torch.logsumexp(x, -1), p @ v.abs(), size


def logprobs(x, token, temperature):
    """One row of logits (float64 values) -> log probabilities of all tokens, entropy, rank of the
    token, and the ranking's order of all entries."""
    order = sorted(range(len(x)), key=lambda i: (not math.isnan(x[i]), -x[i] if not math.isnan(x[i]) else 0.0, i))
    rank = order.index(token) if token >= 0 else -1
    row = torch.tensor(x, dtype=torch.float64)
    if any(math.isnan(v) or v == math.inf for v in x) or max(x) == -math.inf:
        return torch.full((len(x),), math.nan, dtype=torch.float64), math.nan, rank, order
    lp = torch.log_softmax(row / temperature, -1)
    return lp, -float(torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum()), rank, order
