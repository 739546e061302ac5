"""vkv_pages_fork, vkv_pages_reserve and vkv_pages_compact against their definitions written out page by page."""
import random

import pytest
import torch

import paper_2609_03949_amd as vkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


class Model:
    """The state of a pool, on the CPU, and on the GPU beside it."""

    def __init__(self, lens, page, spare, seed=0, width=None, layers=2, sizes=(640, 3), pad=0):
        rng = random.Random(seed)
        self.page, self.B = page, len(lens)
        used = [-(-n // page) for n in lens]
        self.n = sum(used) + spare
        self.width = (max(used) + 2) if width is None else width
        order = list(range(self.n))
        rng.shuffle(order)
        self.table = [[order.pop() if j < u else -1 for j in range(self.width)] for u in used]
        self.lens = list(lens)
        self.refs = [0] * self.n
        for row in self.table:
            for e in row:
                if e >= 0:
                    self.refs[e] += 1
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.planes = [torch.randint(0, 256, (layers, self.n, page, s + pad), generator=g, device=DEV, dtype=torch.uint8) for s in sizes]
        self.want_planes = [p.clone() for p in self.planes]
        self.g_table = torch.tensor(self.table, dtype=torch.int32, device=DEV)
        self.g_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.g_refs = torch.tensor(self.refs, dtype=torch.int32, device=DEV)
        self.pool = vkv.Pool(self.g_table, self.g_lens, self.g_refs, page, self.planes)
        self.ws = torch.full((vkv.pool_workspace_size(self.pool),), 0xAB, dtype=torch.uint8, device=DEV)

    def check(self):
        torch.cuda.synchronize()
        assert self.g_table.tolist() == self.table
        assert self.g_lens.tolist() == self.lens
        assert self.g_refs.tolist() == self.refs
        for a, b in zip(self.planes, self.want_planes):
            assert torch.equal(a, b)

    def named(self, e):
        return 0 <= e < self.n

    def fork(self, ctx, source, **kw):
        vkv.pages_fork(ctx, self.pool, torch.tensor(source, dtype=torch.int32, device=DEV), self.ws, **kw)
        old, lens = [list(r) for r in self.table], list(self.lens)
        for b, s in enumerate(source):
            if s == b:
                continue
            row, n = [-1] * self.width, 0
            if 0 <= s < self.B:
                n = lens[s]
                for j in range(-(-n // self.page)):
                    row[j] = old[s][j] if self.named(old[s][j]) else -1
            self.table[b], self.lens[b] = row, n
        self.refs = [0] * self.n
        for row in self.table:
            for e in row:
                if self.named(e):
                    self.refs[e] += 1
        self.check()

    def reserve(self, ctx, want, **kw):
        missing = torch.full((self.B,), -9, dtype=torch.int32, device=DEV)
        vkv.pages_reserve(ctx, self.pool, torch.tensor(want, dtype=torch.int32, device=DEV), missing, self.ws, **kw)
        free, shared, lack = [p for p in range(self.n) if self.refs[p] == 0], list(self.refs), [0] * self.B
        before = [p.clone() for p in self.want_planes]
        for b, top in enumerate(want):
            n, top = self.lens[b], min(max(top, 0), self.width * self.page)
            if top <= n:
                continue
            first = n // self.page
            for j in range(first, -(-top // self.page)):
                e = self.table[b][j]
                if j == first and n % self.page:
                    if not self.named(e):
                        lack[b] += 1
                        continue
                    if shared[e] < 2:
                        continue
                elif self.named(e):
                    continue
                if not free:
                    lack[b] += 1
                    continue
                p = free.pop(0)
                if self.named(e):
                    self.refs[e] -= 1
                    for k, plane in enumerate(self.want_planes):
                        plane[:, p] = before[k][:, e]
                self.table[b][j] = p
                self.refs[p] += 1
        torch.cuda.synchronize()
        assert missing.tolist() == lack
        self.check()
        return lack

    def compact(self, ctx, **kw):
        used = torch.full((1,), -9, dtype=torch.int32, device=DEV)
        vkv.pages_compact(ctx, self.pool, used, self.ws, **kw)
        n = sum(r > 0 for r in self.refs)
        holes = [p for p in range(n) if self.refs[p] == 0]
        moved = {}
        for p in range(self.n - 1, n - 1, -1):
            if self.refs[p] > 0:
                moved[p] = holes[len(moved)]
        for p, q in moved.items():
            for plane in self.want_planes:
                plane[:, q] = plane[:, p]
            self.refs[q], self.refs[p] = self.refs[p], 0
        self.table = [[moved.get(e, e) for e in row] for row in self.table]
        torch.cuda.synchronize()
        assert used.tolist() == [n]
        self.check()

    def grow(self, by=1):
        """The rows that were asked for have come."""
        self.lens = [n + by for n in self.lens]
        self.g_lens += by


@pytest.mark.parametrize("page", [1, 2, 16, 64])
def test_beams_step_by_step(ctx, page):
    """Forks and growth as a decoding loop calls them, then the end of some, compaction, and new ones in their place."""
    m = Model([33, 33, 33, 33, 64, 65, 1, 0], page, spare=40 if page > 2 else 200, seed=page, width=-(-100 // page))
    rng = random.Random(page)
    for step in range(5):
        m.fork(ctx, [rng.randrange(4) for _ in range(4)] + [4, 5, 6, 7])
        lack = m.reserve(ctx, [n + 1 for n in m.lens])
        assert not any(lack)
        m.grow()
    m.fork(ctx, [0, -1, 2, 0, -7, 5, 99, 4])
    m.compact(ctx)
    m.reserve(ctx, [40] * 8)
    m.compact(ctx)


@pytest.mark.parametrize("seed", range(6))
def test_random_pools(ctx, seed):
    rng = random.Random(100 + seed)
    page, B = 1 << rng.randrange(6), rng.randrange(1, 40)
    m = Model([rng.randrange(0, 200) for _ in range(B)], page, spare=rng.randrange(0, 30), seed=seed, width=-(-256 // page),
              layers=rng.randrange(1, 4), sizes=rng.choice([(16,), (5, 640), (1, 2, 4, 160), ()]))
    for _ in range(4):
        m.fork(ctx, [rng.choice([b, rng.randrange(-2, B + 2)]) for b in range(B)])
        m.reserve(ctx, [n + rng.choice([0, 1, 1, 60, -3]) for n in m.lens])
        if rng.random() < 0.5:
            m.compact(ctx)


def test_pages_run_out(ctx):
    """The first sequences get theirs; the others' entries stay, also the shared page that could not be copied."""
    m = Model([10, 10, 10, 10], 4, spare=3, seed=1)
    m.fork(ctx, [0, 0, 0, 0])
    m.reserve(ctx, [11, 30, 11, 13])
    m.reserve(ctx, [1 << 30, -5, 11, 13])
    n = Model([10, 0, 10], 4, spare=1, seed=8)
    n.fork(ctx, [0, 0, 2])
    assert n.reserve(ctx, [11, 11, 20]) == [0, 1, 2]
    n.reserve(ctx, [20, 20, 20])


def test_absent_and_reserved_pages(ctx):
    """Entries that name no page stay so below the length; a fork takes no page beyond its source's length."""
    m = Model([10, 9], 4, spare=8, seed=2, width=5)
    m.reserve(ctx, [20, 12])
    for (b, j), e in {(0, 1): -1, (1, 2): 1 << 30}.items():
        m.refs[m.table[b][j]] -= 1
        m.table[b][j] = e
    m.g_refs.copy_(torch.tensor(m.refs, dtype=torch.int32))
    m.g_table.copy_(torch.tensor(m.table, dtype=torch.int32))
    m.reserve(ctx, [20, 20])
    m.fork(ctx, [1, 0])


def test_many_pages_and_sequences(ctx):
    """More than one block of pages is counted, small planes, many sequences."""
    m = Model([40 * (b % 7) for b in range(500)], 4, spare=1000, seed=3, layers=1, sizes=(4, 1))
    assert m.n > 2 * 4096
    m.fork(ctx, [b - b % 2 if b % 5 else -1 for b in range(500)])
    m.reserve(ctx, [n + 5 for n in m.lens])
    m.compact(ctx)


def test_one_of_everything(ctx):
    m = Model([0], 1, spare=1, seed=4, width=1, layers=1)
    m.compact(ctx)
    m.reserve(ctx, [1])
    m.grow()
    m.compact(ctx)
    m.fork(ctx, [-1])
    full = Model([8, 8], 4, spare=0, seed=5)
    full.compact(ctx)
    full.reserve(ctx, [9, 8])


def test_planes_with_gaps_and_layers_within_pages(ctx):
    """Pages of a larger buffer, layers that lie side by side within each page, 4- and 1-byte alignment."""
    m = Model([100, 50, 70], 16, spare=10, seed=6, layers=1, sizes=())
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    buf = torch.randint(0, 256, (m.n, 3, 1001), generator=g, device=DEV, dtype=torch.uint8)
    wide = torch.randint(0, 100, (2, m.n, 300), generator=g, device=DEV, dtype=torch.int32)
    planes = [buf[..., :17].transpose(0, 1), buf[..., 20:36].transpose(0, 1), wide[..., 1:258]]
    m.planes, m.want_planes = [buf, wide], [buf.clone(), wide.clone()]
    m.pool = vkv.Pool(m.g_table, m.g_lens, m.g_refs, 16, planes)
    copies = [m.want_planes[0][..., :17].transpose(0, 1), m.want_planes[0][..., 20:36].transpose(0, 1), m.want_planes[1][..., 1:258]]
    keep = m.want_planes
    m.want_planes = copies

    def check():
        torch.cuda.synchronize()
        assert m.g_table.tolist() == m.table and m.g_refs.tolist() == m.refs
        assert all(torch.equal(a, b) for a, b in zip(m.planes, keep))
    m.check = check
    m.fork(ctx, [0, 0, 2])
    m.reserve(ctx, [101, 101, 71])
    m.fork(ctx, [-1, 1, 2])
    m.compact(ctx)


def test_captured_replayed_and_on_another_stream(ctx):
    m = Model([30, 30, 30], 8, spare=60, seed=7, width=12)
    source = torch.tensor([1, 1, 0], dtype=torch.int32, device=DEV)
    want, missing = torch.tensor([31, 31, 31], dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    used = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vkv.pages_fork(ctx, m.pool, source, m.ws)
        vkv.pages_reserve(ctx, m.pool, want, missing, m.ws)
        vkv.pages_compact(ctx, m.pool, used, m.ws)
    twin = Model([30, 30, 30], 8, spare=60, seed=7, width=12)
    for k in range(4):
        g.replay()
        torch.cuda.synchronize()
        twin.fork(ctx, source.tolist())
        twin.reserve(ctx, want.tolist())
        twin.compact(ctx)
        assert torch.equal(m.g_table, twin.g_table) and torch.equal(m.g_refs, twin.g_refs) and torch.equal(m.g_lens, twin.g_lens)
        assert all(torch.equal(a, b) for a, b in zip(m.planes, twin.planes))
        for x in (m, twin):
            x.g_lens += 1
        twin.lens = [n + 1 for n in twin.lens]
        want += 1
        source.copy_(torch.tensor([[2, 1, 0], [0, 0, -1], [1, 1, 1], [0, 1, 2]][k], dtype=torch.int32))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    twin.fork(ctx, [0, 0, 0], stream=s)
    twin.reserve(ctx, [n + 9 for n in twin.lens], stream=s)
    twin.compact(ctx, stream=s)


@pytest.mark.parametrize("B,size", [(4, 2048), (4, 2049), (9, 5000)])
def test_large_pages(ctx, B, size):
    """Pages of many pieces, few enough bytes for one workgroup to copy (4 pages of 16 x 2048 bytes twice) and more."""
    m = Model([21] * B, 16, spare=3 * B, seed=B, layers=2, sizes=(size,))
    m.fork(ctx, [0] * (B - 1) + [B - 1])
    m.reserve(ctx, [22 + 16 * b for b in range(B)])
    m.compact(ctx)
