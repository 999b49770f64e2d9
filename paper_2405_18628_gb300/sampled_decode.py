"""Sampled decoding over a long context, as a model's decode loop would run it: a 4-bit cache,
the tree's attention over it layer by layer, acceptance by sampling, the accepted rows and
their attention weight into the cache, and now and then the cache cut down to a budget.

    python -m paper_2405_18628_gb300.sampled_decode --steps 16

runs the loop on seeded synthetic projections and logits in place of a model's (there is
none here) and prints what was accepted and what the caches hold.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import ppd
from . import workloads as W


class LongContext:
    """The 4-bit caches of B sequences over L layers, the attention weight of every cached row,
    and the buffers of a step.  H K/V heads of G query heads each, trees of T tokens, a
    vocabulary of V.  A cache holds S_max rows per head (rounded up to eight) and is cut to `budget` rows (the first
    n_sink, the last n_recent, and the heaviest between) when a prompt does not fit, or a step of
    `most` accepted nodes (T where not given) might not fit any more.  Rows without weight yet
    (a prompt's, before a step) count as the lightest, the earlier ones first.
    Nothing here waits for the GPU but a prompt that might not fit: lengths stay on the device,
    and the host counts the most that they can be."""

    def __init__(self, L, B, H, G, T, D, V, S_max, budget, n_sink=4, n_recent=32, device="cuda", most=None):
        most = T if most is None else most
        if most < 1 or budget < 1 or budget + most > S_max:
            raise ValueError(f"a budget of {budget} rows and a step of {most} in caches of {S_max}")
        if n_sink < 0 or n_recent < 0 or n_sink + n_recent > budget:
            raise ValueError(f"{n_sink} first and {n_recent} last rows in a budget of {budget}")
        S_max = (S_max + 7) // 8 * 8           # a layer's scales, H S_max D / 32 bytes, start on 16 of them
        self.sizes = L, B, H, G, T, D, V, S_max
        self.budget, self.n_sink, self.n_recent, self.most = budget, n_sink, n_recent, most
        self.k, self.k_scale = ppd.kv4_cache(L, B, H, S_max, D, device)
        self.v, self.v_scale = ppd.kv4_cache(L, B, H, S_max, D, device)
        self.weight = torch.zeros((L, B, H, S_max), device=device)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        self.length, self.new_length = i32(B), i32(B)
        self.longest = 0                       # no sequence is longer (host)
        self.row = torch.arange(S_max, dtype=torch.int32, device=device)
        self.out = torch.empty((L, B, H * G, T, D), dtype=torch.bfloat16, device=device)
        self.lse = torch.empty((L, B, H * G, T), device=device)
        self.accept_len, self.next_token, self.path = i32(B), i32(B), i32(B, T)
        self.accept_prob = torch.empty((B, T), device=device)
        self.kept = i32(L, B, H, budget)
        self.attend_status, self.accept_status, self.append_status, self.evict_status = i32(L, B), i32(B), i32(B), i32(B)
        n = ppd.ppd_kv4_attention_workspace_bytes(1, B, H, G, T, D, S_max)
        self.workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def prompt(self, k, v):
        """A prompt's rows of every layer, k and v [L,B,H,n,D], enter the caches, without weight yet.
        One that does not fit, even after an eviction, is refused."""
        B, n, S_max = k.shape[1], k.shape[3], self.sizes[7]
        if self.longest + n > S_max:           # perhaps: what steps accepted decides (waits for the GPU)
            self.longest = int(self.length.max())
        if min(self.longest, self.budget) + n > S_max:
            raise ValueError(f"a prompt of {n} rows after {min(self.longest, self.budget)}: the caches hold {S_max}")
        if self.longest + n > S_max:
            self.evict()
        count = torch.full((B,), n, dtype=torch.int32, device=k.device)
        ppd.ppd_kv4_append(k, v, self.k, self.k_scale, self.v, self.v_scale, self.length, count, self.append_status)
        # an eviction leaves the weights of other rows past the new length: the prompt's start at 0
        self.weight.masked_fill_((self.row >= self.length[:, None])[:, None], 0.0)
        self.length += count
        self.longest += n
        if self.longest + self.most > S_max:
            self.evict()

    def attend(self, layer, q, k_tree, v_tree, parent):
        """One layer's attention: q [B,H*G,T,D], k_tree and v_tree [B,H,T,D] -> bf16 [B,H*G,T,D]."""
        at = slice(layer, layer + 1)
        ppd.ppd_tree_attention_kv4(q[None], self.k[at], self.k_scale[at], self.v[at], self.v_scale[at], k_tree[None], v_tree[None],
                                   self.length, parent, self.out[at], self.attend_status[layer], lse=self.lse[at],
                                   workspace=self.workspace)
        return self.out[layer]

    def accept(self, logits, cand_tokens, parent, temperature, u, noise, draft_probs=None, draft_row=None):
        """The drafted tokens against the target's probabilities -> next_token [B]; path and
        accept_len say what was accepted."""
        ppd.ppd_sample_accept(logits, cand_tokens, parent, self.length, self.sizes[7], temperature, u, noise, self.accept_len, self.path,
                              self.next_token, self.new_length, self.accept_status, draft_probs=draft_probs, draft_row=draft_row,
                              accept_prob=self.accept_prob)
        return self.next_token

    def commit(self, q, k_tree, v_tree, most=None):
        """The accepted nodes' attention weight and rows (of every layer: q [L,B,H*G,T,D], k_tree and
        v_tree [L,B,H,T,D]) enter the caches; `most`: nodes that this step and the next accept at most."""
        S_max = self.sizes[7]
        most = self.most if most is None else most
        ppd.ppd_kv_weight_add(q, self.lse, self.k, k_tree, self.path, self.accept_len, self.length, self.weight, k_scale=self.k_scale)
        ppd.ppd_kv4_append(k_tree, v_tree, self.k, self.k_scale, self.v, self.v_scale, self.length, self.accept_len, self.append_status,
                           rows=self.path)
        self.length, self.new_length = self.new_length, self.length
        self.longest += most
        if self.longest + most > S_max:
            self.evict()

    def evict(self):
        """Every head's cache down to the budget, in place."""
        ppd.ppd_kv_evict(self.weight, [self.k, self.k_scale, self.v, self.v_scale], self.length, self.budget, self.n_sink, self.n_recent,
                         self.kept, self.new_length, self.evict_status)
        self.length, self.new_length = self.new_length, self.length
        self.longest = min(self.longest, self.budget)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=900)
    ap.add_argument("--capacity", type=int, default=1024)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    L, B, H, G, T, D, V = a.layers, a.batch, 8, 4, 32, 128, 32000
    g = torch.Generator(device="cuda")
    g.manual_seed(a.seed)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device="cuda", generator=g)  # noqa: E731
    w = W.Workload("demo", L=1, B=1, H=1, D=64, P=0, T=T, V=1, n_cand=T // 4, max_depth=4, chains="fill3", match_rate=0.6)
    ctx = LongContext(L, B, H, G, T, D, V, a.capacity, a.capacity * 3 // 4, most=w.max_depth + 1)
    ctx.prompt(n(L, B, H, a.prompt, D), n(L, B, H, a.prompt, D))
    emitted = 0
    t0 = time.perf_counter()
    for step in range(a.steps):
        trees = [W.make_tree(np.random.Generator(np.random.PCG64(a.seed * 1000 + step * B + b)), w) for b in range(B)]
        parent = torch.tensor(np.stack([p for p, _ in trees]), dtype=torch.int32, device="cuda")
        prompt = torch.tensor(np.stack([p for _, p in trees]), device="cuda")
        # what a model's layers would give for the tree's tokens
        q, k_tree, v_tree = n(L, B, H * G, T, D), n(L, B, H, T, D), n(L, B, H, T, D)
        for layer in range(L):
            ctx.attend(layer, q[layer], k_tree[layer], v_tree[layer], parent)
        logits = 5 * torch.randn(B, T, V, device="cuda", generator=g)
        cand = torch.where(prompt, -1, logits.argmax(-1).gather(1, parent.long().clamp(min=0))).int()
        u, noise = torch.rand(B, T, device="cuda", generator=g), torch.empty(B, V, device="cuda").exponential_(generator=g).clamp_(min=1e-20)
        ctx.accept(logits, cand, parent, 0.7, u, noise)
        ctx.commit(q, k_tree, v_tree)
        emitted += int(ctx.accept_len.sum())
    torch.cuda.synchronize()
    bad = [int(x.abs().sum()) for x in (ctx.attend_status, ctx.accept_status, ctx.append_status, ctx.evict_status)]
    print(f"{a.steps} steps of {B} sequences: {emitted} tokens, {emitted / a.steps / B:.2f} a step; lengths {ctx.length.tolist()} of "
          f"{a.capacity}; statuses {bad}; {(time.perf_counter() - t0) / a.steps * 1e3:.2f} ms a step with its synthetic inputs")
    return 0 if not any(bad) else 1


if __name__ == "__main__":
    raise SystemExit(main())
