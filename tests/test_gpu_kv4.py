"""The 4-bit cache on the GPU: rows in and out bit for bit, the tree's attention over it
against 64 bits.

Bounds of the attention, from its formula: an output is rounded to bf16 once, by at most
2^-8 |o| and so 2^-8 sum_j p_j |v_j|; what the probabilities' two bf16 terms (2^-18) and the
fp32 sums add is far below 1e-4 of that sum; probabilities below fp32's normal numbers
(2^-126) count as 0, which with a hundred keys of that size is below 1e-36.
A score is a sum of D fp32 products, off by at most e = D 2^-24 of the sum of their magnitudes:
a probability by a factor of 1 +- 2 e (its own score's and the sum's), the log-sum-exp by e, and
1e-5 for the exponentials and the logarithm."""
import numpy as np
import pytest
import torch

import oracle.operators as O
from paper_2405_18628_gb300 import workloads as W

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
    """A 4-bit cache of random rows whose bytes beyond the prefixes are random too."""

    def __init__(self, dev, L, B, H, G, D, T, lens, S, tree="random", dtype=torch.bfloat16, seed=0, size=1.0):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        rng = np.random.default_rng(seed)
        n = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
        self.dev, self.sizes, self.lens = dev, (L, B, H, G, D, T, S), lens
        byte = lambda *s: torch.randint(0, 256, s, dtype=torch.uint8, device=dev, generator=g)  # noqa: E731
        self.kc, self.vc = byte(L, B, H, S, D // 2), byte(L, B, H, S, D // 2)
        self.ks, self.vs = byte(L, B, H, S, D // 32), byte(L, B, H, S, D // 32)
        for c, s in ((self.kc, self.ks), (self.vc, self.vs)):
            for b in range(B):
                if lens[b]:
                    c[:, b, :, :lens[b]], s[:, b, :, :lens[b]] = O.kv4_quantise(n(L, H, lens[b], D) * size)
        self.q, self.kt, self.vt = ((n(L, B, h, T, D) * f).to(dtype) for h, f in ((H * G, size), (H, size), (H, 1.0)))
        self.parent = [_tree(tree, T, rng) for _ in range(B)]
        self.out = torch.full((L, B, H * G, T, D), float("nan"), dtype=torch.bfloat16, device=dev)
        self.lse = torch.full((L, B, H * G, T), float("nan"), device=dev)
        self.status = torch.full((B,), 77, dtype=torch.int32, device=dev)

    def run(self, ppd, workspace=True, lse=True, scale=0.0, stream=None):
        L, B, H, G, D, T, S = self.sizes
        n = ppd.ppd_kv4_attention_workspace_bytes(L, B, H, G, T, D, S)
        ws = torch.full((max(n, 256),), 255, dtype=torch.uint8, device=self.dev) if workspace else None
        ppd.ppd_tree_attention_kv4(self.q, self.kc, self.ks, self.vc, self.vs, self.kt, self.vt, _i32(self.lens, self.dev),
                                   _i32(self.parent, self.dev), self.out, self.status, lse=self.lse if lse else None,
                                   scale=scale, workspace=ws, stream=stream)

    def check(self, scale=0.0, lse=True, slices=None):
        L, B, H, G, D, T, S = self.sizes
        for l in range(L):
            for b in range(B):
                P = self.lens[b]
                for h in range(H):
                    if slices is not None and (l, b, h) not in slices:
                        continue
                    k = O.kv4_values(self.kc[l, b, h, :P], self.ks[l, b, h, :P])
                    v = O.kv4_values(self.vc[l, b, h, :P], self.vs[l, b, h, :P])
                    hs = slice(h * G, (h + 1) * G)
                    out, want_lse, mass, size = O.attention_kv4(self.q[l, b, hs], k, v, self.kt[l, b, h], self.vt[l, b, h], P,
                                                                self.parent[b], scale)
                    off = (self.out[l, b, hs].double() - out).abs() - (2.0 ** -8 + 1e-4 + 2 * D * 2.0 ** -24 * size) * mass - 1e-36
                    assert float(off.max()) <= 0, (l, b, h, float(off.max()))
                    if lse:
                        e = (self.lse[l, b, hs].double() - want_lse).abs().max()
                        assert float(e) <= D * 2.0 ** -24 * size + 1e-5, (l, b, h, float(e))
        if slices is None:
            assert (self.status == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 8), (2, 3), (7, 1), (16, 1), (17, 1), (5, 8), (31, 1), (32, 1), (33, 1),
                                 (48, 1), (64, 1), (16, 4), (65, 1), (64, 2), (100, 1), (128, 1), (129, 1), (200, 2), (285, 1), (512, 1)])
def test_attention_tree_sizes(cuda_device, D, T, G):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, D, T, [150, 77], 211, seed=T * 8 + G)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 20, 70])
@pytest.mark.parametrize("P", [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 4097])
def test_attention_prefix_lengths(cuda_device, D, T, P):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 1, 3, 1, D, T, [P], max(1, P), seed=P)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("tree", ["chain", "star"])
@pytest.mark.parametrize("T", [3, 40, 64, 130, 512])
def test_attention_tree_shapes(cuda_device, tree, T):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 1, 2, 2, 128, T, [45], 64, tree=tree, seed=T)
    c.run(ppd)
    c.check()


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,B,H,G,T", [(2, 5, 3, 1, 9), (1, 9, 1, 4, 1), (3, 2, 4, 1, 64), (1, 3, 1, 1, 1), (1, 4, 2, 1, 96), (1, 2, 40, 1, 64)])
def test_attention_ragged_batches(cuda_device, workspace, D, L, B, H, G, T):
    from paper_2405_18628_gb300 import ppd
    lens = [int(x) for x in np.linspace(0, 3001, B)]
    c = Case(cuda_device, L, B, H, G, D, T, lens, 3011, seed=B)
    c.run(ppd, workspace=workspace)
    c.check()


@pytest.mark.parametrize("T", [1, 24, 64, 90])
def test_attention_fp32_operands_scale_and_peaked_scores(cuda_device, T):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, 2, 64, T, [300, 299], 301, dtype=torch.float32, seed=T, size=4.0)
    c.run(ppd, scale=0.5, lse=False)
    c.check(scale=0.5, lse=False)


@pytest.mark.parametrize("T", [1, 40, 80])
def test_attention_of_long_caches(cuda_device, T):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 1, 1, 2, 128, T, [100003], 100003, seed=T)
    c.run(ppd)
    c.check()


def test_attention_offsets_beyond_32_bits(cuda_device):
    """The last head's rows lie past 2^32 bytes of codes."""
    from paper_2405_18628_gb300 import ppd
    dev, H, S, D = cuda_device, 72, 1 << 20, 128
    for T in (1, 64, 70):
        c = Case(dev, 1, 1, 1, 1, D, T, [90], 90, seed=4)
        big = Case.__new__(Case)
        big.__dict__ = dict(c.__dict__)
        big.sizes = (1, 1, H, 1, D, T, S)
        for name, w in (("kc", 64), ("vc", 64), ("ks", 4), ("vs", 4)):
            t = torch.zeros((1, 1, H, S, w), dtype=torch.uint8, device=dev)
            t[0, 0, H - 1, :90] = getattr(c, name)[0, 0, 0]
            setattr(big, name, t)
        for name in ("q", "kt", "vt"):
            t = torch.zeros((1, 1, H, T, D), dtype=torch.bfloat16, device=dev)
            t[0, 0, H - 1] = getattr(c, name)[0, 0, 0]
            setattr(big, name, t)
        big.out = torch.empty((1, 1, H, T, D), dtype=torch.bfloat16, device=dev)
        big.lse = torch.empty((1, 1, H, T), device=dev)
        big.run(ppd)
        big.check(slices={(0, 0, H - 1)})
        del big


def test_attention_reports_malformed_trees_and_prefixes(cuda_device):
    from paper_2405_18628_gb300 import ppd
    for T in (12, 40, 100):
        c = Case(cuda_device, 2, 5, 2, 1, 64, T, [9, 9, 9, 9, 9], 20, seed=1)
        c.parent[1][3] = 3
        c.parent[2][0] = 0
        c.lens[3] = 21
        c.lens[4] = -1
        c.run(ppd)
        assert c.status.tolist() == [0, ppd.PPD_ERR_TREE, ppd.PPD_ERR_TREE, ppd.PPD_ERR_CAPACITY, ppd.PPD_ERR_CAPACITY]
        c.check(slices={(l, 0, h) for l in range(2) for h in range(2)})


def test_attention_on_another_stream_and_in_a_graph(cuda_device):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 4, 1, 128, 20, [700, 300], 720, seed=8)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.run(ppd)
    s.synchronize()
    c.check()
    L, B, H, G, D, T, S = c.sizes
    ws = torch.empty(max(256, ppd.ppd_kv4_attention_workspace_bytes(L, B, H, G, T, D, S)), dtype=torch.uint8, device=cuda_device)
    lens, parent = _i32(c.lens, cuda_device), _i32(c.parent, cuda_device)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            ppd.ppd_tree_attention_kv4(c.q, c.kc, c.ks, c.vc, c.vs, c.kt, c.vt, lens, parent, c.out, c.status, lse=c.lse, workspace=ws)
    for fresh in (1, 2):
        c.q.copy_(torch.randn(c.q.shape, device=cuda_device))
        c.out.zero_()
        g.replay()
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 7, 64, 700])
def test_append_and_read_bit_for_bit(cuda_device, D, dtype, T):
    from paper_2405_18628_gb300 import ppd
    dev, L, B, H, S = cuda_device, 2, 4, 3, 811
    g = torch.Generator(device=dev)
    g.manual_seed(T)
    x = [(torch.randn(L, B, H, T, D, device=dev, generator=g) * torch.exp(3 * torch.randn(H, 1, D, device=dev, generator=g))).to(dtype) for _ in "kv"]
    x[0][0, 0, 0, 0, :40] = 0                   # a group of zeros
    x[0][0, 1, 0, 0, 3] = float("nan")
    x[1][0, 1, 1, 0, 5] = float("inf")
    x[1][1, 1, 1, 0, 33] = -1e30
    x[1][1, 2, 1, 0, :32] = 1e-9
    for rows in (None, [sorted(np.random.default_rng(b).permutation(T)[:max(1, T // 2)].tolist()) for b in range(B)]):
        n = [T] * B if rows is None else [len(r) for r in rows]
        n[3] = 0
        start = [0, 5, S - n[2], 9]
        codes = [torch.randint(0, 256, (L, B, H, S, D // 2), dtype=torch.uint8, device=dev, generator=g) for _ in "kv"]
        scales = [torch.randint(0, 256, (L, B, H, S, D // 32), dtype=torch.uint8, device=dev, generator=g) for _ in "kv"]
        want = [(c.clone(), s.clone()) for c, s in zip(codes, scales)]
        status = torch.full((B,), 9, dtype=torch.int32, device=dev)
        at = None if rows is None else _i32([r + [-1] * (T - len(r)) for r in rows], dev)
        ppd.ppd_kv4_append(x[0], x[1], codes[0], scales[0], codes[1], scales[1], _i32(start, dev), _i32(n, dev), status, rows=at)
        for i in range(2):
            for b in range(B):
                src = x[i][:, b] if rows is None else x[i][:, b][:, :, rows[b]]
                if n[b]:
                    c, s = O.kv4_quantise(src[:, :, :n[b]])
                    want[i][0][:, b, :, start[b]:start[b] + n[b]], want[i][1][:, b, :, start[b]:start[b] + n[b]] = c, s
            assert torch.equal(codes[i], want[i][0]) and torch.equal(scales[i], want[i][1])
            for dt in (torch.bfloat16, torch.float32):
                N = max(n) + 3
                back = torch.full((L, B, H, N, D), float("nan"), dtype=dt, device=dev)
                ppd.ppd_kv4_read(codes[i], scales[i], _i32(start, dev), _i32(n, dev), back)
                for b in range(B):
                    v = O.kv4_values(codes[i][:, b, :, start[b]:start[b] + n[b]], scales[i][:, b, :, start[b]:start[b] + n[b]])
                    assert torch.equal(back[:, b, :, :n[b]].double(), v)
                    assert (back[:, b, :, n[b]:] == 0).all()
        assert status.tolist() == [0] * B


def test_append_refuses_sequences_that_do_not_fit(cuda_device):
    from paper_2405_18628_gb300 import ppd
    dev, B, T, S, D = cuda_device, 6, 4, 10, 64
    x = torch.ones(1, B, 1, T, D, device=dev)
    c, s = ppd.kv4_cache(1, B, 1, S, D, dev)
    c2, s2 = ppd.kv4_cache(1, B, 1, S, D, dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    ppd.ppd_kv4_append(x, x, c, s, c2, s2, _i32([0, 7, -1, 3, 3, 6], dev), _i32([4, 4, 1, 5, -1, 4], dev), status)
    E = ppd.PPD_ERR_CAPACITY
    assert status.tolist() == [0, E, E, E, E, 0]
    wrote = (s[0, :, 0].sum((1, 2)) > 0).tolist()
    assert wrote == [True, False, False, False, False, True]
    # row indices outside the new rows write nothing
    rows = _i32([[0, 9, -5, 1]] * B, dev)
    s.zero_()
    ppd.ppd_kv4_append(x, x, c, s, c2, s2, _i32([0] * B, dev), _i32([4] * B, dev), status, rows=rows)
    assert (s[0, 0, 0].sum(-1) > 0).tolist()[:5] == [True, False, False, True, False]


def test_read_of_rows_outside_the_cache_is_zero(cuda_device):
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    c, s = ppd.kv4_cache(1, 3, 1, 5, 64, dev)
    c.fill_(0xFF), s.fill_(160)
    out = torch.full((1, 3, 1, 4, 64), 9.0, device=dev)
    ppd.ppd_kv4_read(c, s, _i32([3, -1, 6], dev), _i32([4, 4, 4], dev), out)
    assert (out[0, 0, 0, :2] == 7).all() and (out[0, 0, 0, 2:] == 0).all() and (out[0, 1:] == 0).all()


def test_workloads_trees_run(cuda_device):
    """The library's own tree shapes, as the steps over a bf16 cache use them."""
    from paper_2405_18628_gb300 import ppd
    for name in ("tiny", "mobilellama"):
        w = W.WORKLOADS[name]
        c = Case(cuda_device, 1, 1, 4, 1, w.D, w.T, [w.P], w.S_max, seed=2)
        c.parent = [W.make_tree(np.random.default_rng(1), w)[0].tolist()]
        c.run(ppd)
        c.check()


@pytest.mark.parametrize("T", [1, 24, 90])
@pytest.mark.parametrize("workspace", [True, False])
def test_attention_into_its_queries(cuda_device, T, workspace):
    """The output may take the queries' place, and a call repeats itself bit for bit."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 2, 3, 2, 2, 128, T, [1500, 0, 333], 1501, seed=T)
    c.run(ppd, workspace=workspace)
    first, lse = c.out.clone(), c.lse.clone()
    c.run(ppd, workspace=workspace)
    assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    q = c.q.clone()
    c.out = c.q
    c.run(ppd, workspace=workspace)
    assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    c.q = q
    c.check()


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 8), (2, 8), (24, 1), (64, 1), (40, 2), (200, 1)])
def test_attention_of_maxima_that_come_late(cuda_device, T, G, D, dtype, workspace):
    """Keys that outweigh all before them by far, after many tiles: a prefix row, the root, and the last
    node (which only itself sees), for references that move when sums have been added up."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, D, T, [1000, 931], 1003, dtype=dtype, seed=T + G)
    c.q[..., :4] = c.q[..., :4].abs() + 1
    for b, row in ((0, 900), (1, 930)):
        k = torch.randn(2, D, device=cuda_device, generator=torch.Generator(device=cuda_device).manual_seed(b))
        k[:, :4] = 40.0
        c.kc[0, b, :, row], c.ks[0, b, :, row] = O.kv4_quantise(k)
    c.kt[0, :, :, 0, :4] = 80.0
    if T > 1:
        c.kt[0, :, :, T - 1, :4] = 160.0
    c.run(ppd, workspace=workspace)
    c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 8), (24, 1), (64, 1), (90, 1)])
def test_attention_fp32_operands_of_both_head_sizes(cuda_device, T, G, D):
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, 1, 2, 2, G, D, T, [300, 299], 301, dtype=torch.float32, seed=T, size=4.0)
    c.run(ppd, scale=0.5)
    c.check(scale=0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 7, 30, 64, 100])
@pytest.mark.parametrize("L,B,H", [(1, 4, 8), (2, 3, 1)])
def test_attention_of_capacities_far_above_the_lengths(cuda_device, L, B, H, T, D):
    """Parts of a slice's keys without any: planned by the capacity, which a program allocates once."""
    from paper_2405_18628_gb300 import ppd
    c = Case(cuda_device, L, B, H, 1, D, T, [500, 0, 33, 1][:B], 16384, seed=T)
    c.run(ppd)
    c.check()
