"""Pages assigned and rows appended on the GPU, bit for bit against plain lists."""
import numpy as np
import pytest
import torch

import oracle.pages as O

pytestmark = pytest.mark.gpu


def _i32(a, dev):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)


class Pool:
    """Tables and the stack of a pool on the GPU, beside the plain ones."""

    def __init__(self, dev, B, page, n_pages, max_pages, max_slots, rng, shift=0):
        self.dev, self.page, self.max_slots = dev, page, max_slots
        ids = rng.permutation(n_pages).tolist()
        self.table, self.stack, self.length = [[-1] * max_pages for _ in range(B)], list(ids), [0] * B
        self.d_table, self.d_stack = _i32(self.table, dev), _i32(ids, dev)
        self.d_free, self.d_len = _i32([n_pages], dev), _i32([0] * B, dev)
        self.buf = torch.full((max_slots + shift,), -5, dtype=torch.int32, device=dev)
        self.slots = self.buf[shift:]          # at any alignment
        self.start, self.status = _i32([-7] * (B + 1), dev), _i32([77] * B, dev)

    def assign(self, ppd, new, stream=None):
        B = len(new)
        self.slots.fill_(-5)
        old_stack, old_table, n_old = self.d_stack.clone(), self.d_table.clone(), len(self.stack)
        n_free, out_len = _i32([-1], self.dev), _i32([-1] * B, self.dev)
        ppd.ppd_page_assign(self.d_len, _i32(new, self.dev), self.page, self.d_table, self.d_stack, self.d_free, n_free, out_len, self.slots, self.start,
                            self.status, stream=stream)
        torch.cuda.synchronize()
        before = [list(t) for t in self.table]
        length, slots, status = O.page_assign(self.length, new, self.page, self.table, self.stack, self.max_slots)
        assert out_len.tolist() == length and self.status.tolist() == status
        assert self.start.tolist() == np.concatenate([[0], np.cumsum([len(s) for s in slots])]).tolist()
        flat = [x for s in slots for x in s]
        got = self.slots.tolist()
        assert got[:len(flat)] == flat and got[len(flat):] == [-5] * (self.max_slots - len(flat))
        assert n_free.tolist() == [len(self.stack)] and self.d_stack[:len(self.stack)].tolist() == self.stack
        # nothing but entries that were taken or pushed is written
        assert self.d_table.tolist() == self.table
        assert torch.equal(self.d_stack[max(n_old, len(self.stack)):], old_stack[max(n_old, len(self.stack)):])
        assert all(self.table[b][:O.pages_of(min(a, c), self.page)] == before[b][:O.pages_of(min(a, c), self.page)]
                   for b, (a, c) in enumerate(zip(self.length, length)) if a >= 0 and c >= 0)
        self.length, self.d_len, self.d_free = length, out_len, n_free
        held = [p for b, t in enumerate(self.table) for p in t[:O.pages_of(length[b], self.page)]]
        assert sorted(held + self.stack) == list(range(len(old_stack)))   # every page is somewhere, once
        return status


@pytest.mark.parametrize("each", [6, 3])
@pytest.mark.parametrize("page", [8, 16, 128])
@pytest.mark.parametrize("B", [1, 3, 70])
def test_requests_come_grow_and_go(cuda_device, B, page, each):
    """Pools of six pages a sequence, and of three, which run short."""
    from paper_2405_18628_gb300 import ppd
    rng = np.random.default_rng(B + page)
    pool = Pool(cuda_device, B, page, n_pages=B * each, max_pages=11, max_slots=B * 9 * page, rng=rng, shift=B % 2)
    short = 0
    for step in range(25):
        new = []
        for n in pool.length:
            r = rng.random()
            new.append(0 if r < 0.15 else min(11 * page, n + int(rng.integers(1, 6))) if r < 0.6 else int(rng.integers(0, 11 * page + 1)) if r < 0.95 else n)
        short += O.CAPACITY in pool.assign(ppd, new)
    assert short or each == 6
    pool.assign(ppd, [0] * B)


def test_a_call_and_its_reverse(cuda_device):
    """Lengths exchanged: tables and stack are as they were."""
    from paper_2405_18628_gb300 import ppd
    rng = np.random.default_rng(5)
    pool = Pool(cuda_device, 40, 16, 2000, 30, 30000, rng)
    first = rng.integers(0, 400, 40).tolist()
    pool.assign(ppd, first)
    held = [t[:O.pages_of(n, 16)] for t, n in zip(pool.table, first)]
    stack = list(pool.stack)
    assert O.CAPACITY not in pool.assign(ppd, rng.integers(0, 480, 40).tolist())
    pool.assign(ppd, first)
    assert pool.stack == stack and [t[:O.pages_of(n, 16)] for t, n in zip(pool.table, first)] == held


@pytest.mark.parametrize("B", [511, 512, 513, 1500, 8192])
def test_many_sequences(cuda_device, B):
    from paper_2405_18628_gb300 import ppd
    rng = np.random.default_rng(B)
    pool = Pool(cuda_device, B, 8, B * 2, 4, B * 20, rng)
    for _ in range(3):
        pool.assign(ppd, rng.integers(0, 33, B).tolist())


def test_shortages_and_lengths_outside(cuda_device):
    """First come, first served; who is refused keeps what it has; a sequence that shrinks, or gains rows
    of a page that it has, is served although an earlier one is not."""
    from paper_2405_18628_gb300 import ppd
    rng = np.random.default_rng(9)
    pool = Pool(cuda_device, 6, 16, 10, 8, 1000, rng)
    assert pool.assign(ppd, [20, 100, 33, 0, 1, 0]) == [0, 4, 0, 0, 0, 0][:1] + [0, 4, 0, 4, 0]      # 2 + 7 pages, then none is left but one
    assert pool.assign(ppd, [32, 100, 0, 40, 5, 0])[:1] == [0]
    for bad in ([-1, 100, 0, 0, 5, 3], [20, 129, 0, 0, 5, 3], [20, 2 ** 31 - 1, -2 ** 31, 0, 5, 3]):
        st = pool.assign(ppd, bad)
        assert [x for x, n in zip(st, bad) if not 0 <= n <= 128] == [O.CAPACITY] * sum(not 0 <= n <= 128 for n in bad)
    few = Pool(cuda_device, 3, 16, 100, 8, 50, rng)           # slots run out before pages
    assert few.assign(ppd, [30, 21, 20]) == [0, 4, 4]
    assert few.assign(ppd, [30, 21, 20]) == [0, 0, 0]


def test_one_graph_for_steps_of_any_size(cuda_device):
    """Captured once: lengths change in place."""
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    rng = np.random.default_rng(2)
    B, page, N, M = 5, 16, 60, 12
    ids = rng.permutation(N).tolist()
    table, stack, length = [[-1] * M for _ in range(B)], list(ids), [0] * B
    d = dict(old=_i32(length, dev), new=_i32(length, dev), table=_i32(table, dev), stack=_i32(ids, dev), n=_i32([N], dev), n2=_i32([0], dev),
             out=_i32(length, dev), slots=_i32([-5] * 700, dev), start=_i32([0] * (B + 1), dev), status=_i32([0] * B, dev))
    call = lambda: ppd.ppd_page_assign(d["old"], d["new"], page, d["table"], d["stack"], d["n"], d["n2"], d["out"], d["slots"], d["start"], d["status"])  # noqa: E731
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for step in range(8):
        new = rng.integers(0, M * page, B).tolist()
        d["new"].copy_(_i32(new, dev))
        graph.replay()
        length, slots, status = O.page_assign(length, new, page, table, stack, 700)
        assert d["out"].tolist() == length and d["status"].tolist() == status and d["table"].tolist() == table
        flat = [x for s in slots for x in s]
        assert d["slots"].tolist()[:len(flat)] == flat and d["stack"].tolist()[:len(stack)] == stack
        d["old"].copy_(d["out"])
        d["n"].copy_(d["n2"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,B,H,D,T,page,path", [(2, 3, 2, 64, 9, 16, True), (1, 1, 1, 128, 1, 8, False), (3, 4, 5, 128, 70, 32, True),
                                                 (2, 2, 3, 64, 131, 256, False), (1, 2, 2, 128, 600, 64, False), (1, 40, 2, 64, 64, 16, True)])
def test_append(cuda_device, dtype, L, B, H, D, T, page, path):
    from paper_2405_18628_gb300 import ppd
    dev, rng = cuda_device, np.random.default_rng(T + B)
    g = torch.Generator(device=dev)
    g.manual_seed(T)
    N = B * (T // page + 2)
    # halves between two bf16 numbers, and values beyond their range, among fp32 rows
    kn, vn = ((torch.randn(L, B, H, T, D, device=dev, generator=g) * 3).to(dtype) for _ in range(2))
    if dtype == torch.float32:
        kn[..., 0], kn[..., 1], kn[..., 2] = 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 3.4e38
        vn[..., 5] = float("nan")
    count = [0 if b == 1 else int(rng.integers(1, T + 1)) for b in range(B)]
    places = rng.permutation(N * page)
    slots, rows, at = [], np.full((B, T), -1), 0
    for b in range(B):
        slots.append(places[at:at + count[b]])
        at += count[b]
        rows[b, :count[b]] = np.sort(rng.permutation(T)[:count[b]])
    flat = np.concatenate(slots + [np.full(5, 3)])
    skipped = {}
    if count[0] > 2:
        flat[1] = -1                            # a slot outside the pool, and a row outside the tree
        skipped[0] = {1}
        if path:
            rows[0, 2] = T
            skipped[0] = {1, 2}
    start = np.concatenate([[0], np.cumsum(count)])
    pools = [torch.full((L, N, H, page, D), 9.0, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    want = [p.clone() for p in pools]
    status = _i32([77] * B, dev)
    ppd.ppd_page_append(kn, vn, *pools, _i32(flat, dev), _i32(start, dev), status, rows=_i32(rows, dev) if path else None)
    for w, x in zip(want, (kn, vn)):
        x = x.to(torch.bfloat16)
        for b in range(B):
            for j in range(count[b]):
                if j in skipped.get(b, ()):
                    continue
                s = int(slots[b][j])
                w[:, s // page, :, s % page] = x[:, b, :, int(rows[b, j]) if path else j]
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.int16), w.view(torch.int16)) or torch.equal(torch.nan_to_num(p.float(), 1234.5), torch.nan_to_num(w.float(), 1234.5))
    assert (status == 0).all()


def test_append_refuses_counts_that_do_not_fit(cuda_device):
    from paper_2405_18628_gb300 import ppd
    dev = cuda_device
    kn = torch.ones(1, 4, 1, 5, 64, dtype=torch.bfloat16, device=dev)
    pools = [torch.zeros(1, 8, 1, 8, 64, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    slots, status = torch.arange(20, dtype=torch.int32, device=dev), _i32([77] * 4, dev)
    ppd.ppd_page_append(kn, kn, *pools, slots, _i32([0, 6, 4, 9, 21], dev), status)    # six of five rows, fewer than none, fine, past the slots
    assert status.tolist() == [4, 4, 0, 4]
    filled = pools[0].view(64, 64)[:, 0].nonzero()[:, 0].tolist()
    assert filled == [4, 5, 6, 7, 8]
    ppd.ppd_page_append(kn, kn, *pools, slots, _i32([-1, 2, 2 ** 31 - 1, 9, 14], dev), status)
    assert status.tolist() == [4, 4, 4, 0]
