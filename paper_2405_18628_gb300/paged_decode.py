"""Decoding of many requests over one pool of pages, as a server's loop would run it: prompts come
in as places are free, every step verifies a token tree per request by exact matching, the accepted
rows enter pages that are taken as requests grow, log probabilities of the emitted tokens go back
with them, and requests that are done give their pages back.

    python -m paper_2405_18628_gb300.paged_decode --steps 32

runs the loop on seeded synthetic projections and logits in place of a model's (there is none here)
and prints what was emitted and what the pool holds.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import ppd
from . import workloads as W


class PagedRequests:
    """B places for requests over L layers: pools of n_pages pages of `page` rows, tables of max_pages pages, and
    the buffers of a step.  H K/V heads of G query heads each, trees of T tokens, a vocabulary of V, K alternatives
    for each emitted token; prompts of `prompt` rows at most.  A place is active from its prompt to finish().
    Projections are bf16 or fp32.
    Nothing here waits for the GPU: lengths, tables and the free pages stay on the device.  Where the pool
    is short, requests keep what they hold and assign_status says so (PPD_ERR_CAPACITY): finish() some and
    commit() or admit() again."""

    def __init__(self, L, B, H, G, T, D, V, n_pages, page, max_pages, prompt, K=5, device="cuda"):
        if min(prompt, T, B, n_pages, max_pages) < 1 or prompt > max_pages * page:
            raise ValueError(f"prompts of {prompt} rows in tables of {max_pages} pages of {page}")
        self.sizes = L, B, H, G, T, D, V, page, max_pages
        self.k, self.v = ppd.page_pool(L, n_pages, H, page, D, device), ppd.page_pool(L, n_pages, H, page, D, device)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        f32 = lambda *s: torch.zeros(s, device=device)  # noqa: E731
        self.table = torch.full((B, max_pages), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.n_free, self._n_free = torch.full((1,), n_pages, dtype=torch.int32, device=device), i32(1)
        self.length, self._length, self.wanted = i32(B), i32(B), i32(B)
        self.active = torch.zeros(B, dtype=torch.bool, device=device)
        self.slots, self.slot_start = i32(B * max(prompt, T)), i32(B + 1)
        self.out = torch.empty((L, B, H * G, T, D), dtype=torch.bfloat16, device=device)
        self.top1, self.path, self.accept_len, self.next_token = i32(B, T), i32(B, T), i32(B), i32(B)
        self.tokens, self.rank = i32(B, T), i32(B, T)
        self.logprob, self.entropy = f32(B, T), f32(B, T)
        self.top_tokens, self.top_logprobs = (i32(B, T, K), f32(B, T, K)) if K else (None, None)
        self.attend_status, self.accept_status, self.logprob_status = i32(L, B), i32(B), i32(B)
        self.assign_status, self.append_status = i32(B), i32(B)
        n = ppd.ppd_paged_attention_workspace_bytes(1, B, H, G, T, D, max_pages * page, ppd.PPD_F32)   # (no less than bf16 needs)
        self.workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def _assign(self, wanted):
        ppd.ppd_page_assign(self.length, wanted, self.sizes[7], self.table, self.free, self.n_free, self._n_free, self._length, self.slots, self.slot_start,
                            self.assign_status)
        self.length, self._length = self._length, self.length
        self.n_free, self._n_free = self._n_free, self.n_free

    def _append(self, k, v, rows=None):
        try:
            ppd.ppd_page_append(k, v, self.k, self.v, self.slots, self.slot_start, self.append_status, rows=rows)
        except Exception:
            self._assign(self._length.clone())   # lengths exchanged: nothing has changed
            raise

    def admit(self, k, v, count):
        """Prompts for free places: k and v [L,B,H,n,D] of every layer, count int32 [B] rows of each, n at most (0:
        none for this place, and for active ones).  A prompt that finds no pages leaves its place free."""
        count = torch.where(self.active, 0, count.clamp(0, k.shape[3]))
        self._assign(self.length + count)
        self._append(k, v)
        came = (count > 0) & (self.assign_status == 0)
        self.active |= came
        # what a place is to hold goes with its request: a new one has accepted nothing yet
        self.wanted.copy_(torch.where(came, self.length, self.wanted))

    def attend(self, layer, q, k_tree, v_tree, parent):
        """One layer's attention: q [B,H*G,T,D], k_tree and v_tree [B,H,T,D], bf16 or fp32 -> bf16 [B,H*G,T,D]."""
        at = slice(layer, layer + 1)
        ppd.ppd_tree_attention_paged(q[None], self.k[at], self.v[at], self.table, k_tree[None], v_tree[None], self.length, parent, self.out[at],
                                     self.attend_status[layer], workspace=self.workspace)
        return self.out[layer]

    def accept(self, logits, cand_tokens, parent):
        """The longest path that the model's top tokens confirm, by fp32 logits [B,T,V], the tree's tokens and parents,
        int32 [B,T] -> next_token [B]; path and accept_len say what was accepted, tokens [B,T] the emitted tokens
        (-1 past them), with their log probabilities, entropies, ranks and alternatives."""
        V, page, max_pages = self.sizes[6:]
        each = self.path.shape
        ppd._take(("logits", logits, torch.float32, (*each, V)), ("cand_tokens", cand_tokens, torch.int32, each), ("parent", parent, torch.int32, each))
        ppd.ppd_node_argmax_noalloc(logits, self.top1)
        ppd.ppd_accept_path(self.top1, cand_tokens, parent, self.length, V, page * max_pages, self.accept_len, self.path, self.next_token, self.wanted,
                            self.accept_status)
        # the token after path node j is what the row of node j emitted
        self.tokens.copy_(torch.where(self.path >= 0, self.top1.gather(1, self.path.long().clamp(min=0)), -1))
        ppd.ppd_token_logprobs(logits, self.tokens, 1.0, self.logprob, self.entropy, self.rank, self.logprob_status, rows=self.path,
                               top_tokens=self.top_tokens, top_logprobs=self.top_logprobs)
        return self.next_token

    def commit(self, k_tree, v_tree):
        """The accepted nodes' rows of every layer, k_tree and v_tree [L,B,H,T,D], enter the pages of active requests (of
        those that have accepted since they came and were not served yet)."""
        self._assign(torch.where(self.active, self.wanted, self.length))
        self._append(k_tree, v_tree, self.path)

    def finish(self, done):
        """Requests that are done, bool [B], give their pages back."""
        self._assign(torch.where(done, 0, self.length))
        self.active &= ~done
        self.wanted.masked_fill_(done, 0)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--pages", type=int, default=400)
    ap.add_argument("--tokens", type=int, default=40, help="emitted tokens after which a request is done")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    L, B, H, G, T, D, V, page, prompt = a.layers, a.batch, 8, 4, 32, 128, 32000, 16, 700
    g = torch.Generator(device="cuda")
    g.manual_seed(a.seed)
    rng = np.random.default_rng(a.seed)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device="cuda", generator=g)  # noqa: E731
    w = W.Workload("demo", L=1, B=1, H=1, D=64, P=0, T=T, V=1, n_cand=T // 4, max_depth=4, chains="fill3", match_rate=0.6)
    req = PagedRequests(L, B, H, G, T, D, V, a.pages, page, 64, prompt)
    since = torch.zeros(B, dtype=torch.int64, device="cuda")      # tokens of each request so far
    emitted, requests, refused, bad = 0, 0, 0, 0
    t0 = time.perf_counter()
    for step in range(a.steps):
        count = torch.tensor(rng.integers(20, prompt + 1, B), dtype=torch.int32, device="cuda")
        before = req.active.clone()
        req.admit(n(L, B, H, prompt, D), n(L, B, H, prompt, D), count)
        requests += int((req.active & ~before).sum())
        refused += int((req.assign_status != 0).sum())
        trees = [W.make_tree(np.random.Generator(np.random.PCG64(a.seed * 1000 + step * B + b)), w) for b in range(B)]
        parent = torch.tensor(np.stack([p for p, _ in trees]), dtype=torch.int32, device="cuda")
        is_prompt = torch.tensor(np.stack([p for _, p in trees]), device="cuda")
        # what a model's layers would give for the tree's tokens
        q, k_tree, v_tree = n(L, B, H * G, T, D), n(L, B, H, T, D), n(L, B, H, T, D)
        for layer in range(L):
            req.attend(layer, q[layer], k_tree[layer], v_tree[layer], parent)
        logits = 5 * torch.randn(B, T, V, device="cuda", generator=g)
        cand = torch.where(is_prompt, -1, logits.argmax(-1).gather(1, parent.long().clamp(min=0))).int()
        req.accept(logits, cand, parent)
        req.commit(k_tree, v_tree)
        grown = req.active & (req.assign_status == 0)
        refused += int((req.assign_status != 0).sum())
        gained = torch.where(grown, req.accept_len, 0)
        emitted += int(gained.sum())
        since += gained
        done = req.active & ((since >= a.tokens) | ~grown)
        req.finish(done)
        since.masked_fill_(done, 0)
        bad += sum(int(x.abs().sum()) for x in (req.attend_status, req.accept_status, req.append_status, req.logprob_status))
    torch.cuda.synchronize()
    held = int(((req.length + page - 1) // page).sum())
    print(f"{a.steps} steps: {requests} requests, {emitted} tokens; lengths {req.length.tolist()}, {held} pages held and {int(req.n_free)} free of {a.pages}; "
          f"{refused} times short of pages; {(time.perf_counter() - t0) / a.steps * 1e3:.2f} ms a step with its synthetic inputs")
    return 0 if not bad and held + int(req.n_free) == a.pages else 1


if __name__ == "__main__":
    raise SystemExit(main())
