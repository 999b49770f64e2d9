"""The operators over pages together, as a server's loop runs them: rows, tables, attention and log
probabilities over several steps against plain lists and 64 bits."""
import numpy as np
import pytest
import torch

import oracle.pages as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,n_pages", [(4, 60), (3, 16)])
def test_steps_of_a_server(cuda_device, B, n_pages):
    """Prompts come and go; with few pages some requests are refused and keep what they have."""
    from paper_2405_18628_gb300 import paged_decode as S
    dev, L, H, G, T, D, V, page, M, prompt, K = cuda_device, 2, 2, 2, 10, 64, 300, 8, 12, 50, 3
    g = torch.Generator(device=dev)
    g.manual_seed(B)
    rng = np.random.default_rng(B)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
    req = S.PagedRequests(L, B, H, G, T, D, V, n_pages, page, M, prompt, K=K, device=dev)
    table, stack = [[-1] * M for _ in range(B)], list(range(n_pages))
    rows = [[] for _ in range(B)]              # what each request holds: (k, v) [L,H,D] a row
    active, refused = [False] * B, 0

    def assigned(wanted, new):
        """The plain pool after the same call; new[b]: the rows that b gains."""
        nonlocal refused
        length, _, status = O.page_assign([len(r) for r in rows], wanted, page, table, stack, req.slots.numel())
        assert req.length.tolist() == length and req.assign_status.tolist() == status
        for b in range(B):
            rows[b] = rows[b][:length[b]] + (new[b] if length[b] > len(rows[b]) else [])
            assert len(rows[b]) == length[b]
            assert req.table[b, :O.pages_of(length[b], page)].tolist() == table[b][:O.pages_of(length[b], page)]
        assert req.n_free.tolist() == [len(stack)] and req.free[:len(stack)].tolist() == stack
        refused += sum(s != 0 for s in status)
        return status

    for step in range(12):
        count = [0 if rng.random() < 0.2 else int(rng.integers(1, prompt + 1)) for _ in range(B)]
        kp, vp = n(L, B, H, prompt, D), n(L, B, H, prompt, D)
        req.admit(kp, vp, torch.tensor(count, dtype=torch.int32, device=dev))
        count = [0 if a else c for a, c in zip(active, count)]
        status = assigned([len(r) + c for r, c in zip(rows, count)], [[(kp[:, b, :, j], vp[:, b, :, j]) for j in range(count[b])] for b in range(B)])
        active = [a or (c > 0 and s == 0) for a, c, s in zip(active, count, status)]
        assert req.active.tolist() == active
        # a step of every place
        parent = [[-1] + [int(rng.integers(0, i)) for i in range(1, T)] for _ in range(B)]
        pt = torch.tensor(parent, dtype=torch.int32, device=dev)
        q, kt, vt = n(L, B, H * G, T, D), n(L, B, H, T, D), n(L, B, H, T, D)
        for l in range(L):
            req.attend(l, q[l], kt[l], vt[l], pt)
        logits = 4 * torch.randn(B, T, V, device=dev, generator=g)
        cand = torch.where(torch.rand(B, T, device=dev, generator=g) < 0.6, logits.argmax(-1).gather(1, pt.long().clamp(min=0)), 1).int()
        req.accept(logits, cand, pt)
        top = logits.argmax(-1).tolist()
        paths = [[x for x in p if x >= 0] for p in req.path.tolist()]
        for b in range(B):
            assert paths[b][0] == 0 and all(parent[b][y] == x and int(cand[b, y]) == top[b][x] for x, y in zip(paths[b], paths[b][1:]))
            for j, x in enumerate(paths[b]):
                lp, H_, rank, order = O.logprobs(logits[b, x].double().tolist(), top[b][x], 1.0)
                assert int(req.tokens[b, j]) == top[b][x] and int(req.rank[b, j]) == rank == 0
                assert abs(float(req.logprob[b, j]) - float(lp[top[b][x]])) <= 1e-5 and abs(float(req.entropy[b, j]) - H_) <= 2e-5
                assert req.top_tokens[b, j].tolist() == order[:K]
            assert (req.tokens[b, len(paths[b]):] == -1).all() and (req.logprob[b, len(paths[b]):] == 0).all()
            for l in range(L):
                k, v = (torch.stack([r[x][l] for r in rows[b]], 1) if rows[b] else kt.new_zeros(H, 0, D) for x in range(2))
                for h in range(H):
                    hs = slice(h * G, (h + 1) * G)
                    out, _, mass, size = O.attention(q[l, b, hs], k[h], v[h], kt[l, b, h], vt[l, b, h], parent[b])
                    assert ((req.out[l, b, hs].double() - out).abs() <= (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass + 1e-36).all()
        req.commit(kt, vt)
        status = assigned([len(r) + len(p) if a else len(r) for r, p, a in zip(rows, paths, active)],
                          [[(kt[:, b, :, x], vt[:, b, :, x]) for x in paths[b]] for b in range(B)])
        done = [a and (len(r) > 70 or s != 0 or rng.random() < 0.1) for a, r, s in zip(active, rows, status)]
        req.finish(torch.tensor(done, device=dev))
        assigned([0 if d else len(r) for d, r in zip(done, rows)], [[]] * B)
        active = [a and not d for a, d in zip(active, done)]
        # the rows are where the tables say
        for b in range(B):
            for x, pool in enumerate((req.k, req.v)):
                for l in range(L):
                    got = O.rows_of(pool[l], table[b], len(rows[b]))
                    want = torch.stack([r[x][l] for r in rows[b]], 1) if rows[b] else got
                    assert torch.equal(got, want)
        for st in (req.attend_status, req.accept_status, req.append_status, req.logprob_status):
            assert (st == 0).all()
    assert refused or n_pages == 60


def test_the_command(cuda_device, capsys):
    from paper_2405_18628_gb300 import paged_decode as S
    assert S.main(["--steps", "20", "--layers", "2"]) == 0
    assert S.main(["--steps", "10", "--layers", "1", "--pages", "90", "--batch", "6"]) == 0
    assert "free of 90" in capsys.readouterr().out


def test_sizes_that_do_not_fit_are_refused():
    from paper_2405_18628_gb300 import paged_decode as S
    for bad in (dict(prompt=129), dict(prompt=0), dict(n_pages=0)):
        with pytest.raises(ValueError, match="prompts of"):
            S.PagedRequests(**dict(dict(L=1, B=1, H=1, G=1, T=4, D=64, V=10, n_pages=9, page=16, max_pages=8, prompt=100), **bad), device="cpu")


class Plain:
    """Rows that each place holds and is to gain, beside a PagedRequests, with its calls in any order."""

    def __init__(self, dev, B, n_pages, seed, dtype=torch.bfloat16):
        from paper_2405_18628_gb300 import paged_decode as S
        self.g = torch.Generator(device=dev)
        self.g.manual_seed(seed)
        self.L, self.B, self.H, self.T, self.D, self.V, self.page, self.M, self.prompt = 2, B, 2, 10, 64, 50, 8, 12, 50
        self.req = S.PagedRequests(self.L, B, self.H, 2, self.T, self.D, self.V, n_pages, self.page, self.M, self.prompt, K=0, device=dev)
        self.dev, self.dtype = dev, dtype
        self.rows, self.pending, self.active = [[] for _ in range(B)], [[]] * B, [False] * B
        self.table, self.stack, self.tree = [[-1] * self.M for _ in range(B)], list(range(n_pages)), None

    def n(self, *s):
        return torch.randn(s, device=self.dev, generator=self.g).to(self.dtype)

    def assign(self, wanted, new):
        length, _, status = O.page_assign([len(r) for r in self.rows], wanted, self.page, self.table, self.stack, self.req.slots.numel())
        for b in range(self.B):
            self.rows[b] = self.rows[b][:length[b]] + (new[b] if length[b] > len(self.rows[b]) else [])
        assert self.req.assign_status.tolist() == status
        return status

    def admit(self, count):
        k, v = self.n(self.L, self.B, self.H, self.prompt, self.D), self.n(self.L, self.B, self.H, self.prompt, self.D)
        self.req.admit(k, v, torch.tensor(count, dtype=torch.int32, device=self.dev))
        count = [0 if a else c for a, c in zip(self.active, count)]
        status = self.assign([len(r) + c for r, c in zip(self.rows, count)], [[(k[:, b, :, j], v[:, b, :, j]) for j in range(count[b])] for b in range(self.B)])
        for b in range(self.B):
            if count[b] and status[b] == 0:
                self.active[b], self.pending[b] = True, []

    def accept(self, take):
        """Chains; take[b] rows of each are accepted (1 to T)."""
        parent = torch.arange(-1, self.T - 1, dtype=torch.int32, device=self.dev).repeat(self.B, 1)
        logits = torch.randn(self.B, self.T, self.V, device=self.dev, generator=self.g)
        cand = logits.argmax(-1).int().roll(1, 1)
        for b, t in enumerate(take):
            if t < self.T:
                cand[b, t] = -1
        self.tree = self.n(self.L, self.B, self.H, self.T, self.D), self.n(self.L, self.B, self.H, self.T, self.D)
        self.req.accept(logits, cand, parent)
        assert self.req.accept_len.tolist() == take
        self.pending = [[(self.tree[0][:, b, :, j], self.tree[1][:, b, :, j]) for j in range(t)] if a else [] for b, (t, a) in enumerate(zip(take, self.active))]

    def commit(self):
        self.req.commit(*self.tree)
        status = self.assign([len(r) + len(p) for r, p in zip(self.rows, self.pending)], self.pending)
        self.pending = [p if s else [] for p, s in zip(self.pending, status)]

    def finish(self, done):
        self.req.finish(torch.tensor(done, device=self.dev))
        self.assign([0 if d else len(r) for d, r in zip(done, self.rows)], [[]] * self.B)
        self.active = [a and not d for a, d in zip(self.active, done)]
        self.pending = [[] if d else p for d, p in zip(done, self.pending)]

    def check(self):
        req = self.req
        assert req.length.tolist() == [len(r) for r in self.rows] and req.active.tolist() == self.active
        assert req.n_free.tolist() == [len(self.stack)] and (req.append_status == 0).all()
        for b in range(self.B):
            held = O.pages_of(len(self.rows[b]), self.page)
            assert req.table[b, :held].tolist() == self.table[b][:held]
            for x, pool in enumerate((req.k, req.v)):
                for l in range(self.L):
                    got = O.rows_of(pool[l], self.table[b], len(self.rows[b]))
                    assert not self.rows[b] or torch.equal(got, torch.stack([r[x][l] for r in self.rows[b]], 1).to(torch.bfloat16))


@pytest.mark.parametrize("prompt", [5, 18, 30])
def test_a_commit_repeated_after_a_refusal(cuda_device, prompt):
    """Refused, some requests finished, another in the refused one's place, committed again: the new prompt
    stays as it is, whether shorter or longer than what the old request was to hold."""
    p = Plain(cuda_device, 3, 9, prompt)
    p.admit([24, 20, 8])
    p.accept([10, 3, 10])
    p.commit()                       # to 34, 23 and 18 rows: two pages are free, and the first takes them
    p.check()
    assert p.req.assign_status.tolist() == [0, 0, 4]
    p.finish([True, False, True])
    p.admit([0, 0, prompt])
    p.check()
    for _ in range(3):
        p.commit()
        p.check()
    assert p.req.length.tolist() == [0, 23, prompt]


def test_a_commit_without_an_acceptance(cuda_device):
    """Nothing was accepted yet: prompts stay as they are."""
    p = Plain(cuda_device, 3, 30, 1)
    p.tree = p.n(2, 3, 2, 10, 64), p.n(2, 3, 2, 10, 64)
    p.admit([20, 0, 7])
    p.commit()
    p.check()
    p.accept([3, 4, 5])              # of a place that is free: it gains nothing
    p.admit([0, 9, 0])
    p.commit()
    p.check()
    assert p.req.length.tolist() == [23, 9, 12]


@pytest.mark.parametrize("seed", range(6))
def test_calls_in_any_order(cuda_device, seed):
    rng = np.random.default_rng(seed)
    p = Plain(cuda_device, 4, 14 if seed % 2 else 40, seed)
    p.tree = p.n(2, 4, 2, 10, 64), p.n(2, 4, 2, 10, 64)
    for _ in range(60):
        what = rng.choice(["admit", "accept", "commit", "commit", "finish"])
        if what == "admit":
            p.admit([0 if rng.random() < 0.5 else int(rng.integers(1, p.prompt + 1)) for _ in range(4)])
        elif what == "accept" and max(len(r) for r in p.rows) <= p.M * p.page - p.T:
            p.accept([int(rng.integers(1, p.T + 1)) for _ in range(4)])
        elif what == "commit":
            p.commit()
        else:
            p.finish([bool(rng.random() < (0.9 if len(r) > 70 else 0.2)) for r in p.rows])
        p.check()


def test_fp32_projections(cuda_device):
    """Prompts, queries and tree rows in fp32, layer by layer."""
    p = Plain(cuda_device, 3, 30, 2, dtype=torch.float32)
    p.admit([20, 0, 50])
    p.accept([3, 1, 10])
    p.commit()
    p.check()
    parent = [[-1, 0, 0, 1, 1, 2, 5, 5, 0, 3]] * 3
    q, kt, vt = p.n(2, 3, 4, 10, 64), p.n(2, 3, 2, 10, 64), p.n(2, 3, 2, 10, 64)
    for l in range(2):
        p.req.attend(l, q[l], kt[l], vt[l], torch.tensor(parent, dtype=torch.int32, device=cuda_device))
        for b in range(3):
            k, v = (torch.stack([r[x][l] for r in p.rows[b]], 1).to(torch.bfloat16) if p.rows[b] else kt.new_zeros(2, 0, 64) for x in range(2))
            for h in range(2):
                hs = slice(2 * h, 2 * h + 2)
                out, _, mass, size = O.attention(q[l, b, hs], k[h], v[h], kt[l, b, h], vt[l, b, h], parent[b])
                assert ((p.req.out[l, b, hs].double() - out).abs() <= (2.0 ** -8 + 1e-4 + 2 * 64 * 2.0 ** -24 * size) * mass + 1e-36).all()
    assert (p.req.attend_status == 0).all()


def test_refused_rows_change_nothing(cuda_device):
    """Rows that cannot be appended: the call raises, and lengths, tables and the pool are as they were."""
    p = Plain(cuda_device, 3, 30, 3)
    p.admit([20, 0, 7])
    n, count = p.n, torch.tensor([0, 30, 0], dtype=torch.int32, device=cuda_device)
    good = n(2, 3, 2, 50, 64)
    off = torch.empty(good.numel() + 1, dtype=good.dtype, device=cuda_device)[1:].view(good.shape)
    for k, v in ((n(1, 3, 2, 50, 64), n(1, 3, 2, 50, 64)), (good, n(2, 3, 2, 49, 64)), (n(2, 3, 1, 50, 64), n(2, 3, 1, 50, 64)), (good.half(), good.half()),
                 (good, good.float()), (good.transpose(1, 2).contiguous().transpose(1, 2), good), (off, good), (good, good.cpu())):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            p.req.admit(k, v, count)
        p.check()
    p.accept([3, 1, 10])
    for k, v in ((n(2, 3, 2, 9, 64), n(2, 3, 2, 9, 64)), (n(2, 2, 2, 10, 64), n(2, 2, 2, 10, 64)), (p.tree[0], p.tree[1].float())):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            p.req.commit(k, v)
        p.check()
    p.commit()
    p.admit([0, 30, 0])
    p.check()
    assert p.req.length.tolist() == [23, 30, 17] and torch.equal(p.req.free[:p.req.n_free[0]].cpu(), torch.tensor(p.stack, dtype=torch.int32))
