"""The operators of the 8-bit cache one after another, as a server calls them: pages for the new rows, rotary positions on queries and
keys, the rows' write, attention over them; between the steps beams fork, sequences end and begin, the pages are moved together.
Every step's rows and outputs are checked against what each sequence has been given, by its own history kept on the CPU.

A row that is read back is off by the rounding of its code, 2^-4 of its size or half of the format's last step, 2^-10 of
the scale 2^e; where a block's scale has grown, codes were rounded again, which moves only values below 2^-6 of the new scale, by
2^-10 of it, and the scales grow at least twofold: 2^-4 |x| + 2 2^-10 2^e in all.  Outputs are held against attention in 64 bits over
the rows as the cache holds them."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

from _attention import attention, check
from _paged8 import decode
from test_gpu_rope import frequencies, turned

pytestmark = pytest.mark.gpu
DEV, BF, I32 = "cuda", torch.bfloat16, torch.int32
SCALE = 1.0 / math.sqrt(192.0)


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


class Server:
    def __init__(self, B, H, page, block, n_pages, width, seed, inter):
        self.B, self.H, self.page, self.block, self.inter = B, H, page, block, inter
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.cache = torch.full((n_pages, page, 640), 0x7F, dtype=torch.uint8, device=DEV)
        self.scale = torch.full((n_pages, page // block), 255, dtype=torch.uint8, device=DEV)
        self.table = torch.full((B, width), -1, dtype=I32, device=DEV)
        self.kv_len = torch.zeros(B, dtype=I32, device=DEV)
        self.refs = torch.zeros(n_pages, dtype=I32, device=DEV)
        self.pool = vkv.Pool(self.table, self.kv_len, self.refs, page, [self.cache[None], self.scale[None]])
        self.pool_ws = torch.empty(vkv.pool_workspace_size(self.pool), dtype=torch.uint8, device=DEV)
        self.pages = vkv.Pages8(self.cache, self.scale, self.table, self.kv_len, width * page)
        self.rope = vkv.Rope(64, interleaved=inter, base=10000.0)
        self.freq = frequencies(64, 10000.0, vkv.VKV_ROPE_PLAIN, 1.0, 4096.0, 32.0, 1.0)
        self.missing = torch.empty(B, dtype=I32, device=DEV)
        self.rows = [(torch.empty(0, 512, dtype=torch.float64), torch.empty(0, 64, dtype=BF)) for _ in range(B)]   # given; turned

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV).to(BF)

    def step(self, ctx, q_lens):
        """q_lens new tokens a sequence, all checked."""
        n, H = sum(q_lens), self.H
        old = [r[0].shape[0] for r in self.rows]
        want = torch.tensor([o + q for o, q in zip(old, q_lens)], dtype=I32, device=DEV)
        vkv.pages_reserve(ctx, self.pool, want, self.missing, self.pool_ws)
        self.kv_len.copy_(want)
        pos = torch.cat([torch.arange(o, o + q, dtype=I32) for o, q in zip(old, q_lens)]).to(DEV)
        lat = (self.normal(n, 512).float() * torch.exp(self.normal(n, 1).float())).to(BF)
        branch, q_lat, q_rope = self.normal(n, 64), self.normal(n, H, 512), self.normal(n, H, 64)
        key, query = torch.empty_like(branch), q_rope.clone()
        vkv.rope_apply(ctx, self.rope, branch, pos, key)
        vkv.rope_apply(ctx, self.rope, query, pos, query)
        cu = torch.tensor([sum(q_lens[:b]) for b in range(self.B + 1)], dtype=I32, device=DEV)
        vkv.cache8_write(ctx, self.pages, lat, key, cu, max(q_lens))
        chunk = vkv.Chunk(q_lat, query, cu, max(q_lens))
        ws = torch.empty(max(vkv.chunk8_workspace_size(self.pages, chunk), 256), dtype=torch.uint8, device=DEV)
        out, lse = torch.empty(n, H, 512, dtype=BF, device=DEV), torch.empty(n, H, device=DEV)
        vkv.chunk8_attend(ctx, self.pages, chunk, ws, SCALE, out, lse)
        torch.cuda.synchronize()
        assert self.missing.tolist() == [0] * self.B
        for x, y in ((branch[:, None], key[:, None]), (q_rope, query)):
            w, tol = turned(x, pos, self.freq, 0, self.inter, 1.0, False)
            assert bool(((y.double().cpu() - w).abs() <= tol).all())
        at = 0
        for b, q in enumerate(q_lens):
            self.rows[b] = (torch.cat([self.rows[b][0], lat[at:at + q].double().cpu()]), torch.cat([self.rows[b][1], key[at:at + q].cpu()]))
            kv = self.read(b)
            if q == 0:
                continue
            seen = torch.arange(kv.shape[0])[None] <= (old[b] + torch.arange(q))[:, None]
            o, l, ot, lt = attention(torch.cat([q_lat[at:at + q], query[at:at + q]], 2).reshape(q * H, 576), kv, kv[:, :512],
                                     seen[:, None].expand(q, H, -1).reshape(q * H, -1), SCALE)
            check(f"lse of sequence {b}", lse[at:at + q].reshape(-1), l, lt)
            check(f"out of sequence {b}", out[at:at + q].reshape(-1, 512), o, ot)
            at += q
        self.settled()

    def read(self, b):
        """Sequence b's rows as the cache holds them, held against what it was given."""
        lat, branch = self.rows[b]
        u = torch.arange(lat.shape[0], device=DEV)
        p = self.table[b].long()[u // self.page]
        assert bool((p >= 0).all())
        raw, byte = self.cache[p, u % self.page], self.scale[p, u % self.page // self.block]
        got = decode(raw[:, :512], byte)
        tol = 2.0 ** -4 * lat.abs() + 2 * 2.0 ** -10 * torch.pow(2.0, byte.double().cpu() - 127)[:, None]
        assert bool(((got - lat).abs() <= tol).all())
        assert torch.equal(raw[:, 512:].contiguous().view(BF).cpu(), branch)
        return torch.cat([got, branch.double()], 1)

    def settled(self):
        """Lengths and reference counts agree with the histories and the table."""
        assert self.kv_len.tolist() == [r[0].shape[0] for r in self.rows]
        named = self.table[self.table >= 0].long()
        assert torch.equal(torch.bincount(named, minlength=len(self.refs)), self.refs.long())

    def fork(self, ctx, source):
        vkv.pages_fork(ctx, self.pool, torch.tensor(source, dtype=I32, device=DEV), self.pool_ws)
        none = (torch.empty(0, 512, dtype=torch.float64), torch.empty(0, 64, dtype=BF))
        self.rows = [self.rows[s] if s >= 0 else none for s in source]
        self.settled()

    def compact(self, ctx):
        used = torch.empty(1, dtype=I32, device=DEV)
        vkv.pages_compact(ctx, self.pool, used, self.pool_ws)
        n = int(used)
        assert bool((self.refs[:n] > 0).all()) and bool((self.refs[n:] == 0).all())
        self.settled()
        self.cache[n:] = 0x7F                 # what lies behind can be given back
        self.scale[n:] = 255


@pytest.mark.parametrize("H,page,block,inter", [(16, 16, 4, True), (128, 32, 16, False), (4, 4, 1, True), (64, 64, 64, False)])
def test_a_server(ctx, H, page, block, inter):
    s = Server(6, H, page, block, n_pages=6 * -(-140 // page), width=-(-160 // page), seed=H + page, inter=inter)
    s.step(ctx, [37, 5, 0, 64, 1, 0])                 # prompts
    for _ in range(2):
        s.step(ctx, [1, 1, 0, 1, 1, 0])
    s.fork(ctx, [0, 0, 0, 3, -1, 1])                  # two more answers to the first, one ends, one more of the second
    for _ in range(3):
        s.step(ctx, [1, 1, 1, 1, 0, 1])
    s.compact(ctx)
    s.step(ctx, [1, 0, 1, 2, 30, 1])                  # a prompt in the place that became free, a draft of two
    s.fork(ctx, [2, 1, 0, 3, 4, 4])                   # beams that change places
    s.compact(ctx)
    for _ in range(2):
        s.step(ctx, [1, 1, 1, 1, 1, 1])
    s.fork(ctx, [-1, 1, -1, -1, -1, -1])
    s.compact(ctx)
    s.step(ctx, [50, 1, 0, 0, 0, 20])
    assert bool((s.table[2:5] == -1).all())


def test_a_captured_step(ctx):
    """Decode steps replayed, with forks and compaction between them, against the same steps taken one call at a time."""
    B, H = 5, 16
    s = Server(B, H, 16, 16, n_pages=60, width=8, seed=3, inter=True)
    s.step(ctx, [30, 16, 47, 1, 100])
    lat, branch, q_lat, q_rope = s.normal(B, 512), s.normal(B, 64), s.normal(B, H, 512), s.normal(B, H, 64)
    key, query = torch.empty_like(branch), torch.empty_like(q_rope)
    want, pos = torch.empty(B, dtype=I32, device=DEV), torch.empty(B, dtype=I32, device=DEV)
    cu = torch.arange(B + 1, dtype=I32, device=DEV)
    chunk = vkv.Chunk(q_lat, query, cu, 1)
    ws = torch.empty(vkv.chunk8_workspace_size(s.pages, chunk), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(B, H, 512, dtype=BF, device=DEV), torch.empty(B, H, device=DEV)
    source, used = torch.arange(B, dtype=I32, device=DEV), torch.empty(1, dtype=I32, device=DEV)

    def step():
        vkv.pages_fork(ctx, s.pool, source, s.pool_ws)
        torch.add(s.kv_len, 1, out=want)
        vkv.pages_reserve(ctx, s.pool, want, s.missing, s.pool_ws)
        pos.copy_(s.kv_len)
        s.kv_len.copy_(want)
        vkv.rope_apply(ctx, s.rope, branch, pos, key)
        vkv.rope_apply(ctx, s.rope, q_rope, pos, query)
        vkv.cache8_write(ctx, s.pages, lat, key, cu, 1)
        vkv.chunk8_attend(ctx, s.pages, chunk, ws, SCALE, out, lse)
        vkv.pages_compact(ctx, s.pool, used, s.pool_ws)

    state = (s.cache, s.scale, s.table, s.kv_len, s.refs)
    start = [t.clone() for t in state]
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t, v in zip(state, start):
        t.copy_(v)
    for sources in ([0, 1, 2, 3, 4], [0, 1, 2, 2, 2], [4, 1, 0, -1, 2], [0, 1, 2, 3, 4], [1, 1, 1, 1, 1]):
        source.copy_(torch.tensor(sources, dtype=I32))
        for t in (lat, branch, q_lat, q_rope):
            t.copy_(s.normal(*t.shape))
        before = [t.clone() for t in state]
        step()
        eager = [t.clone() for t in (*state, out, lse, used, s.missing)]
        for t, v in zip(state, before):
            t.copy_(v)
        out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*state, out, lse, used, s.missing), eager))
        assert s.missing.tolist() == [0] * B and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("H", [4, 32, 64, 128])
def test_nothing_there(ctx, H):
    """No cache rows at all, no tokens at all: outputs of tokens that see nothing, and nothing else written."""
    u8 = torch.uint8
    cache, scale = torch.full((2, 16, 640), 9, dtype=u8, device=DEV), torch.full((2, 1), 9, dtype=u8, device=DEV)
    kv = torch.zeros(3, dtype=I32, device=DEV)
    cu = torch.tensor([0, 2, 2, 5], dtype=I32, device=DEV)
    q = torch.randn(5, H, 576, device=DEV).to(BF)
    for table, max_kv in ((torch.empty(3, 0, dtype=I32, device=DEV), 0), (torch.zeros(3, 1 << 14, dtype=I32, device=DEV), 1 << 18)):
        pages = vkv.Pages8(cache, scale, table, kv, max_kv)
        chunk = vkv.Chunk(q[..., :512], q[..., 512:], cu, 3)
        ws = torch.empty(max(vkv.chunk8_workspace_size(pages, chunk), 256), dtype=u8, device=DEV)
        out, lse = torch.full((5, H, 512), 7.0, dtype=BF, device=DEV), torch.full((5, H), 7.0, device=DEV)
        vkv.chunk8_attend(ctx, pages, chunk, ws, SCALE, out, lse)
        vkv.cache8_write(ctx, pages, q[:, 0, :512], q[:, 0, 512:], cu, 3)
        none = vkv.Chunk(q[:0, :, :512], q[:0, :, 512:], torch.zeros(4, dtype=I32, device=DEV), 3)
        vkv.chunk8_attend(ctx, pages, none, ws, SCALE, out[:0], lse[:0])
        vkv.cache8_write(ctx, pages, q[:0, 0, :512], q[:0, 0, 512:], torch.zeros(4, dtype=I32, device=DEV), 3)
        torch.cuda.synchronize()
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    x = torch.empty(0, H, 64, dtype=BF, device=DEV)
    vkv.rope_apply(ctx, vkv.Rope(64), x, torch.empty(0, dtype=I32, device=DEV), x)
    assert bool((cache == 9).all()) and bool((scale == 9).all())
