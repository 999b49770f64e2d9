"""Tree attention over pages against 64 bits.

Bounds, from the formula: an output is rounded to bf16 once, by at most 2^-8 |o| and so 2^-8 sum_j p_j
|v_j|; what the probabilities' two bf16 terms (2^-18) and the fp32 sums add is far below 1e-4 of that
sum; probabilities below fp32's normal numbers (2^-126) count as 0, which with a hundred keys of
that size is below 1e-36.  A score is a sum of D fp32 products, off by at most e = D 2^-24 of the sum of their
magnitudes: a probability by a factor of 1 +- 2 e (its own score's and the sum's), the
log-sum-exp by e, and 1e-5 for the exponentials and the logarithm."""
import numpy as np
import pytest
import torch

import oracle.pages as O

pytestmark = pytest.mark.gpu


def _i32(a, dev):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)


def _tree(kind, T, rng):
    if kind == "chain":
        return [i - 1 for i in range(T)]
    if kind == "star":
        return [-1] + [0] * (T - 1)
    return [-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, T)]


class Case:
    """Pools whose rows that no sequence holds are NaN, tables whose other entries name no page."""

    def __init__(self, dev, L, B, H, G, D, T, lens, page, spare=0, tree="random", dtype=torch.bfloat16, seed=0, size=1.0, shared=0):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        n = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
        self.dev, self.sizes, self.lens, self.dtype = dev, (L, B, H, G, D, T), lens, dtype
        need = [O.pages_of(x, page) for x in lens]
        M, N = max(1, max(need)) + spare, sum(need) + 3
        ids = rng.permutation(N)
        self.table = rng.choice([-1, N, 2 ** 31 - 1, -2 ** 31], (B, M)).astype(np.int64)
        at = 0
        self.k, self.v = (torch.full((L, N, H, page, D), float("nan"), dtype=torch.bfloat16, device=dev) for _ in range(2))
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
            if shared and b:                   # the first pages are the first sequence's
                both = min(shared, need[b], lens[0] // page)
                self.table[b, :both] = self.table[0, :both]
            for i in range(need[b]):
                rows = min(page, lens[b] - i * page)
                if shared and b and i < min(shared, lens[0] // page):
                    continue
                for p, s in ((self.k, size), (self.v, 1.0)):
                    p[:, self.table[b, i], :, :rows] = (n(L, H, rows, D) * s).to(torch.bfloat16)
        self.q, self.kt, self.vt = ((n(L, B, h, T, D) * f).to(dtype) for h, f in ((H * G, size), (H, size), (H, 1.0)))
        self.parent = [_tree(tree, T, rng) for _ in range(B)]
        self.out = torch.full((L, B, H * G, T, D), float("nan"), dtype=torch.bfloat16, device=dev)
        self.lse = torch.full((L, B, H * G, T), float("nan"), device=dev)
        self.status = _i32([77] * B, dev)
        self.args = [_i32(x, dev) for x in (self.table, self.lens, self.parent)]

    def workspace(self, ppd):
        L, B, H, G, D, T = self.sizes
        n = ppd.ppd_paged_attention_workspace_bytes(L, B, H, G, T, D, self.table.shape[1] * self.k.shape[3],
                                                    ppd.PPD_F32 if self.dtype == torch.float32 else ppd.PPD_BF16)
        return torch.full((max(n, 256),), 255, dtype=torch.uint8, device=self.dev)

    def run(self, ppd, workspace=True, lse=True, scale=0.0, stream=None, ws=None):
        table, lens, parent = self.args
        ws = ws if ws is not None else self.workspace(ppd) if workspace else None
        ppd.ppd_tree_attention_paged(self.q, self.k, self.v, table, self.kt, self.vt, lens, parent, self.out, self.status,
                                     lse=self.lse if lse else None, scale=scale, workspace=ws, stream=stream)

    def check(self, scale=0.0, lse=True, seqs=None, status=True):
        L, B, H, G, D, T = self.sizes
        for b in range(B) if seqs is None else seqs:
            for l in range(L):
                k, v = (O.rows_of(p[l], self.table[b].tolist(), self.lens[b]) for p in (self.k, self.v))
                for h in range(H):
                    hs = slice(h * G, (h + 1) * G)
                    out, want_lse, mass, size = O.attention(self.q[l, b, hs], k[h], v[h], self.kt[l, b, h], self.vt[l, b, h], self.parent[b], scale)
                    off = (self.out[l, b, hs].double() - out).abs() - (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass - 1e-36
                    assert float(off.max()) <= 0, (l, b, h, float(off.max()))
                    if lse:
                        e = (self.lse[l, b, hs].double() - want_lse).abs().max()
                        assert float(e) <= D * 2.0 ** -24 * size + 1e-5, (l, b, h, float(e))
        if status:
            assert (self.status == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 8), (2, 3), (7, 1), (16, 1), (5, 8), (31, 1), (32, 1), (33, 1), (64, 1), (16, 4), (17, 4), (65, 1),
                                 (64, 2), (64, 4), (13, 10), (100, 1), (128, 1), (129, 1), (200, 2), (150, 3), (285, 1), (512, 1), (1, 200)])
def test_trees_and_heads(cuda_device, D, T, G):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, D, T, [150, 77], 16, seed=T * 8 + G)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("D,T,G", [(64, 1, 4), (128, 20, 1), (128, 70, 1), (64, 40, 4)])
def test_pages_and_prefixes(cuda_device, page, D, T, G):
    """Lengths around pages' and tiles' ends."""
    from paper_2405_18628_gb300 import ppd
    lens = [0, 1, 7, 8, 9, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 383, 385, 513]
    c = Case(cuda_device, 1, len(lens), 2, G, D, T, lens, page, seed=page)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 8), (20, 1), (70, 1)])
@pytest.mark.parametrize("P", [0, 1, 15, 128, 1000, 4097])
def test_one_sequence(cuda_device, D, T, G, P):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 1, 3, G, D, T, [P], 16, seed=P)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("tree", ["chain", "star"])
@pytest.mark.parametrize("T", [3, 40, 64, 130, 512])
def test_tree_shapes(cuda_device, tree, T):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 1, 2, 2, 128, T, [45], 32, tree=tree, seed=T)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("L,B,H,G,D,T,page,spare", [
    (2, 5, 3, 1, 128, 9, 16, 0), (1, 9, 1, 4, 64, 1, 16, 50), (3, 2, 4, 1, 128, 64, 8, 0), (1, 3, 1, 1, 128, 1, 64, 400), (1, 4, 2, 3, 64, 96, 32, 0),
    (1, 2, 40, 1, 64, 64, 16, 0), (1, 20, 8, 4, 128, 1, 16, 0), (1, 21, 8, 2, 64, 33, 128, 3), (1, 7, 8, 4, 128, 64, 32, 0), (1, 80, 3, 2, 64, 1, 16, 0),
    (1, 70, 2, 4, 128, 40, 16, 1), (1, 8, 20, 3, 64, 100, 16, 0)])
def test_ragged_batches(cuda_device, workspace, L, B, H, G, D, T, page, spare):
    """Whole slices, clusters, shared tiles, pairs of query blocks; lengths from none on."""
    from paper_2405_18628_gb300 import ppd
    lens = [int(x) for x in np.linspace(0, 1500, B)]
    c = Case(cuda_device, L, B, H, G, D, T, lens, page, spare=spare, seed=B)
    c.run(ppd, workspace=workspace)
    c.check(seqs=range(B) if B < 30 else range(0, B, 9))


@pytest.mark.parametrize("B,H,G,T", [(1, 8, 4, 1), (1, 2, 1, 30), (2, 4, 4, 40), (3, 64, 1, 1)])
def test_long_caches(cuda_device, B, H, G, T):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, B, H, G, 128, T, [20011 - 6007 * b for b in range(B)], 16, seed=B + H)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("T,G,P", [(1, 4, 300), (20, 2, 300), (40, 3, 5000), (100, 1, 40)])
def test_fp32_operands(cuda_device, T, G, P):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 2, 2, 2, G, 64, T, [P, P // 3], 16, dtype=torch.float32, seed=T)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("size", [8.0, 40.0])
@pytest.mark.parametrize("T,G", [(1, 8), (64, 1), (48, 4)])
def test_peaked_scores_and_late_maxima(cuda_device, T, G, size):
    """Scores far apart, the largest near the end: the maximum moves, sums are rescaled."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, 128, T, [900, 2100], 16, seed=3, size=size ** 0.5)
    for b in range(2):
        i, r = (c.lens[b] - 9) // 16, (c.lens[b] - 9) % 16
        c.k[:, c.table[b, i], :, r] *= 3
    c.run(ppd)
    c.check()


def test_options(cuda_device):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 3, 2, 2, 64, 12, [100, 0, 333], 16, seed=4)
    c.run(ppd, lse=False, scale=0.3)
    c.check(scale=0.3, lse=False)
    assert torch.isnan(c.lse).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.out.fill_(float("nan"))
    torch.cuda.synchronize()
    c.run(ppd, stream=side)
    side.synchronize()
    c.check()


def test_shared_prefixes(cuda_device):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 2, 4, 2, 4, 128, 5, [200, 170, 90, 300], 16, seed=5, shared=8)
    assert (c.table[1, :8] == c.table[0, :8]).all()
    c.run(ppd)
    c.check()


def test_failed_sequences_leave_the_others(cuda_device):
    """A malformed tree, a prefix past the table, pages that are none: their statuses; the others' results."""
    from paper_2405_18628_gb300 import ppd
    for T, G in ((4, 2), (40, 3)):
        c = Case(cuda_device, 1, 7, 2, G, 64, T, [100, 100, 100, 100, 100, 100, 100], 16, seed=T)
        c.table[1, 3], c.table[2, 6], c.table[5, 0] = -1, c.k.shape[1], 2 ** 31 - 1
        table, lens, parent = c.args
        table.copy_(_i32(c.table, c.dev))
        lens[3], lens[4] = -1, c.table.shape[1] * 16 + 1
        parent[6, 2] = 2
        c.run(ppd)
        assert c.status.tolist() == [0, 4, 4, 4, 4, 4, 3]
        c.check(seqs=[0], status=False)


def test_two_graphs_with_one_workspace(cuda_device):
    """Steps of unlike sizes captured over the same scratch, replayed in turn; tables and lengths change in place."""
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    cases = [Case(dev, 1, 2, 4, 4, 128, 1, [9000, 5000], 16, seed=1), Case(dev, 1, 3, 2, 1, 64, 70, [700, 3000, 0], 32, seed=2)]
    ws = torch.full((max(c.workspace(ppd).numel() for c in cases),), 255, dtype=torch.uint8, device=dev)
    graphs = []
    side = torch.cuda.Stream()
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for _ in range(3):                 # a chain of programmatic launches
                c.run(ppd, ws=ws)
        graphs.append(g)
    for step in range(3):
        for c, g in zip(cases, graphs):
            c.out.fill_(float("nan"))
            if step == 2:                      # the first half of the last sequence's pages, shorter
                c.lens = [x // 2 for x in c.lens]
                c.args[1].copy_(_i32(c.lens, dev))
            g.replay()
            torch.cuda.synchronize()
            c.check()


def test_the_same_as_over_a_contiguous_cache(cuda_device):
    """Pages in order are a contiguous cache: the same tiles, sums and merges as ppd_tree_attention's, rounded once."""
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    for L, B, H, T, P in ((1, 2, 4, 30, 500), (1, 2, 4, 64, 1000), (4, 4, 12, 64, 300), (1, 2, 4, 100, 500)):
        g = torch.Generator(device=dev)
        g.manual_seed(T)
        n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
        page, M = 16, O.pages_of(P, 16)
        S = M * page
        kc, vc, q, kt, vt = n(L, B, H, S, 128), n(L, B, H, S, 128), n(L, B, H, T, 128), n(L, B, H, T, 128), n(L, B, H, T, 128)
        parent, lens = _i32([_tree("random", T, np.random.default_rng(T))] * B, dev), _i32([P, P - 77], dev).repeat(B // 2)
        want, status = torch.empty(L, B, H, T, 128, device=dev), _i32([0] * B, dev)
        wlse, lse = torch.empty(L, B, H, T, device=dev), torch.empty(L, B, H, T, device=dev)
        ppd.ppd_tree_attention(q, kc, vc, kt, vt, lens, parent, want, status, lse=wlse, workspace=ppd.workspace(L, B, H, T, 128, 1, S, device=dev))
        pools = [x.view(L, B, H, M, page, 128).permute(0, 1, 3, 2, 4, 5).reshape(L, B * M, H, page, 128).contiguous() for x in (kc, vc)]
        out = torch.empty(L, B, H, T, 128, dtype=torch.bfloat16, device=dev)
        ppd.ppd_tree_attention_paged(q, *pools, torch.arange(B * M, dtype=torch.int32, device=dev).view(B, M), kt, vt, lens, parent, out, status, lse=lse,
                                     workspace=torch.empty(max(256, ppd.ppd_paged_attention_workspace_bytes(L, B, H, 1, T, 128, S)), dtype=torch.uint8, device=dev))
        # (sums may be shared out otherwise: a relative 1e-4 covers fp32's, and a rounding of each side)
        assert ((out.float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4 * want.abs().amax(-1, keepdim=True)).all()
        assert float((lse - wlse).abs().max()) <= 2e-5


def test_pools_past_32_bits(cuda_device):
    """Pages whose elements are more than 2^32 from the pool's start: rows in, and attention over them."""
    from paper_2405_18628_gb300 import ppd
    dev, H, D, page, N, T = cuda_device, 4, 128, 128, 70000, 5
    g = torch.Generator(device=dev)
    g.manual_seed(8)
    n = lambda *s: torch.randn(s, dtype=torch.bfloat16, device=dev, generator=g)  # noqa: E731
    k, v = (torch.empty(1, N, H, page, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    assert k.numel() > 2 ** 32
    table = torch.tensor([[N - 1, 3, N - 2], [66000, N - 3, -1]], dtype=torch.int32, device=dev)
    lens = [300, 200]
    kn, vn = n(1, 2, H, 300, D), n(1, 2, H, 300, D)
    slots = [int(table[b, r // page]) * page + r % page for b in range(2) for r in range(lens[b])]
    status = _i32([77, 77], dev)
    ppd.ppd_page_append(kn, vn, k, v, _i32(slots, dev), _i32([0, 300, 500], dev), status)
    assert (status == 0).all()
    q, kt, vt = n(1, 2, 2 * H, T, D), n(1, 2, H, T, D), n(1, 2, H, T, D)
    parent = [[-1, 0, 1, 0, 3]] * 2
    out, lse = torch.empty(1, 2, 2 * H, T, D, dtype=torch.bfloat16, device=dev), torch.empty(1, 2, 2 * H, T, device=dev)
    ppd.ppd_tree_attention_paged(q, k, v, table, kt, vt, _i32(lens, dev), _i32(parent, dev), out, status, lse=lse)
    assert (status == 0).all()
    for b in range(2):
        for h in range(H):
            want, want_lse, mass, size = O.attention(q[0, b, 2 * h:2 * h + 2], kn[0, b, h, :lens[b]], vn[0, b, h, :lens[b]], kt[0, b, h], vt[0, b, h], parent[b])
            assert ((out[0, b, 2 * h:2 * h + 2].double() - want).abs() <= (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass + 1e-36).all()
            assert float((lse[0, b, 2 * h:2 * h + 2].double() - want_lse).abs().max()) <= D * 2.0 ** -24 * size + 1e-5


@pytest.mark.parametrize("B,lens", [(300, [0, 5, 40, 129]), (65, [700, 1])])
def test_many_requests(cuda_device, B, lens):
    """More requests than the plans for unequal lengths hold."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, B, 3, 2, 64, 3, [lens[b % len(lens)] for b in range(B)], 16, seed=B)
    c.run(ppd)
    c.check(seqs=range(0, B, 23))
    assert (c.status == 0).all()


@pytest.mark.parametrize("page", [8, 16, 128])
@pytest.mark.parametrize("T,G", [(1, 2), (8, 1), (9, 3), (57, 1), (64, 1)])
def test_trees_behind_the_last_rows(cuda_device, page, T, G):
    """The tree's keys share the last prefix tile where they fit behind its pages: lengths around where
    they do, one tile and several, whole slices and parts of them."""
    from paper_2405_18628_gb300 import ppd
    edge = (128 - T) // page * page
    lens = sorted({max(0, x + base) for base in (0, 128, 640) for x in (1, edge - 1, edge, edge + 1, edge - page, 127, 128)})
    for H, spare in ((1, 0), (40, 0), (2, 400)):
        c = Case(cuda_device, 1, len(lens), H, G, 128, T, lens, page, spare=spare, seed=T + page)
        c.run(ppd)
        c.check(seqs=range(0, len(lens), 1 if H < 3 else 7))


@pytest.mark.parametrize("D,T,G,lens", [(128, 70, 1, [130, 5]), (64, 40, 4, [300, 0]), (128, 1, 4, [77, 200]), (64, 300, 1, [20, 140])])
def test_outputs_on_16_bytes(cuda_device, D, T, G, lens):
    """Outputs that begin between two sectors of 32 bytes."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, D, T, lens, 16, seed=T)
    n = c.out.numel()
    flat = torch.full((n + 16,), 3.0, dtype=torch.bfloat16, device=cuda_device)
    c.out = flat[8:8 + n].view(c.out.shape)
    c.run(ppd)
    c.check()
    assert (flat[:8] == 3).all() and (flat[8 + n:] == 3).all()


@pytest.mark.parametrize("D,H,G,T,lens,spare", [(128, 2, 4, 1, [30011], 0), (64, 1, 1, 1, [40000], 0), (128, 1, 3, 5, [20001, 7], 0), (128, 2, 1, 1, [0, 9000, 33], 1500),
                                                (64, 1, 8, 1, [300], 3000), (128, 2, 1, 9, [15000], 0), (64, 2, 1, 33, [25000], 0)])
def test_few_rows_of_many_parts(cuda_device, D, H, G, T, lens, spare):
    """Long requests shared by all SMs: the merge's threads take parts each; tables that hold more than there is."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, len(lens), H, G, D, T, lens, 16, spare=spare, seed=T + G)
    c.run(ppd)
    c.check()
    first = c.out.clone()
    c.out.fill_(float("nan"))
    c.run(ppd)
    assert torch.equal(first.view(torch.int16), c.out.view(torch.int16))
