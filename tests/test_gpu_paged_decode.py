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
