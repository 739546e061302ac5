"""vkv_chunk_attend against plain attention in 64 bits: contexts around the tiles of 32 rows, single tokens and
chunks, few and many rows (every split of the waves and of the work), pages of every kind, tokens that see
nothing, values that are not finite where a token does not look, strides, graphs, streams."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

from _attention import attention, check
from _paged import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 1.0 / math.sqrt(192.0)


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def handles(x):
    return vkv.Pages(x.cache, x.table, x.kv_len, x.max_kv), vkv.Chunk(x.q_lat, x.q_rope, x.cu, x.max_q)


def run(ctx, x, fill=7.0, stream=None):
    pages, chunk = handles(x)
    ws = torch.full((max(vkv.chunk_workspace_size(pages, chunk), 256),), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((x.n_tok, x.H, 512), fill, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((x.n_tok, x.H), fill, device=DEV)
    vkv.chunk_attend(ctx, pages, chunk, ws, SCALE, out, lse, stream)
    return out, lse


def compare(x, out, lse, rows=None, seen=None, only=None):
    at = 0
    for b, nq in enumerate(x.q_lens):
        if nq and (only is None or b in only):
            kv = x.rows(b).cpu() if rows is None else rows[b]
            vis = (x.seen(b) if seen is None else seen[b])[:, None, :].expand(nq, x.H, kv.shape[0]).reshape(nq * x.H, -1)
            q = x.q[at:at + nq].reshape(nq * x.H, 576)
            o, l, ot, lt = attention(q, kv, kv[:, :512], vis, SCALE)
            check(f"lse of sequence {b}", lse[at:at + nq].reshape(-1), l, lt)
            check(f"out of sequence {b}", out[at:at + nq].reshape(-1, 512), o, ot)
        at += nq


@pytest.mark.parametrize("H", [1, 16, 17, 40, 64, 65, 128])
def test_single_tokens(ctx, H):
    x = Case([1, 31, 32, 33, 64, 65, 0, 500], [1] * 8, H, seed=H)
    compare(x, *run(ctx, x))


@pytest.mark.parametrize("page", [1, 2, 32, 64, 512])
def test_pages(ctx, page):
    x = Case([300, 77, 1, 513], [1, 4, 1, 2], 16, page=page, seed=page)
    compare(x, *run(ctx, x))


@pytest.mark.parametrize("H,q_lens,kv_lens", [
    (16, [2, 1, 0, 3], [100, 40, 50, 3]),            # 32 rows and 48
    (8, [5, 16, 1], [5, 16, 1]),                     # a prompt: every token new
    (128, [3, 1, 2], [70, 33, 1000]),                # blocks of one token
    (3, [50, 7, 0, 90], [50, 100, 10, 89]),          # blocks that cut a token's heads; a first token that sees nothing
    (128, [4], [2]),                                 # tokens that see nothing
    (40, [9, 33], [0, 40]),                          # an empty cache
])
def test_chunks(ctx, H, q_lens, kv_lens):
    x = Case(kv_lens, q_lens, H, seed=H + len(q_lens))
    out, lse = run(ctx, x)
    compare(x, out, lse)
    at = 0
    for nq, kv in zip(q_lens, kv_lens):
        none = max(nq - kv, 0)
        assert bool((out[at:at + none] == 0).all()) and bool((lse[at:at + none] == -math.inf).all())
        at += nq


def test_long_context_is_split_and_joined(ctx):
    x = Case([20011, 3, 9000], [1, 1, 1], 16, page=64, seed=2)
    compare(x, *run(ctx, x))
    x = Case([12345], [3], 128, page=128, seed=3)
    compare(x, *run(ctx, x))


def test_many_units(ctx):
    """A bound on the chunk that gives more units than are cut into runs: a workgroup per unit."""
    q_lens = [1, 0, 3, 17, 130] + [1] * 28
    x = Case([200 + 7 * b for b in range(33)], q_lens, 8, seed=4, max_q=512)
    compare(x, *run(ctx, x), only=[0, 2, 3, 4, 20, 32])
    y = Case([200 + 7 * b for b in range(33)], q_lens, 8, seed=4)
    a, b = run(ctx, x), run(ctx, y)
    for s, e in zip(x.cu.tolist(), x.cu.tolist()[1:]):
        assert torch.allclose(a[1][s:e], b[1][s:e], rtol=1e-5, atol=1e-5)


def test_steep_scores(ctx):
    """Scores that rise along the context by far more than the reference maximum's slack, and equal rows."""
    x = Case([700], [2], 16, seed=5)
    f = torch.linspace(0.1, 14.0, 700, device=DEV)[:, None].to(torch.bfloat16)
    x.cache[x.where[0]] = x.rows(0) * f
    same = tuple(w[200:300] for w in x.where[0])
    x.cache[same] = x.rows(0)[200].expand(100, 576)
    compare(x, *run(ctx, x))


def test_absent_pages(ctx):
    """Rows on pages outside the cache do not exist, whatever the entry says; the rest is attended."""
    x = Case([300, 64, 40], [2, 1, 1], 16, page=16, seed=6)
    x.table[0, 3], x.table[0, 7], x.table[0, 18] = -1, 1 << 30, x.cache.shape[0]
    x.table[1, :] = -5
    seen = [x.seen(b).clone() for b in range(3)]
    for p in (3, 7, 18):
        seen[0][:, 16 * p:16 * p + 16] = False
    seen[1][:] = False
    out, lse = run(ctx, x)
    compare(x, out, lse, seen=seen)
    assert bool((out[2] == 0).all()) and bool((lse[2] == -math.inf).all())


def test_lengths_out_of_range_are_cut(ctx):
    x = Case([100, 50], [1, 1], 16, seed=7)
    x.kv_len.copy_(torch.tensor([1 << 30, -4], dtype=torch.int32))
    out, lse = run(ctx, x)
    compare(x, out, lse, only=[0])
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())


def test_chunk_past_its_bound_and_rows_behind(ctx):
    x = Case([90, 60], [10, 6], 5, seed=8, behind=4)
    out, lse = run(ctx, x, fill=3.0)
    compare(x, out, lse)
    assert bool((out[16:] == 3.0).all()) and bool((lse[16:] == 3.0).all())


@pytest.mark.parametrize("H,q_lens,kv_lens", [(16, [1, 40], [90, 100]), (128, [3, 20], [3000, 70])])
def test_what_a_token_does_not_see_does_not_reach_it(ctx, H, q_lens, kv_lens):
    """NaN and infinities in the rows of later tokens."""
    x = Case(kv_lens, q_lens, H, seed=9)
    clean = run(ctx, x)
    nq, n, at = q_lens[1], kv_lens[1], q_lens[0]
    pages, r = x.where[1]

    def put(tok, dim, value):       # into the cache row of the sequence's new token tok
        u = n - nq + tok
        x.cache[pages[u], r[u], dim] = value

    put(nq - 8, 5, math.inf), put(nq - 6, 6, math.nan), put(nq - 3, 540, math.nan)
    out, lse = run(ctx, x)
    a, b, c, e = at + nq - 8, at + nq - 6, at + nq - 3, at + nq
    assert torch.equal(out[:a], clean[0][:a]) and torch.equal(lse[:a], clean[1][:a])
    # a latent that is not finite makes the token's own score so too, with either sign
    assert not bool(torch.isfinite(out[a:e, :, 5]).any())
    assert bool(torch.isnan(out[b:e, :, 6]).all()) and bool(torch.isnan(out[c:e]).all()) and bool(torch.isnan(lse[c:e]).all())


def test_values_near_the_largest(ctx):
    """A latent dim that no query reads holds values near the type's largest, whose weighted mean is finite."""
    x = Case([60], [8], 16, seed=10)
    x.q_lat[..., 5] = 0
    x.q[..., 5] = 0
    pages, r = x.where[0]
    x.cache[pages[56], r[56], 5] = 3.0e38
    out, lse = run(ctx, x)
    compare(x, out, lse)
    for u in range(60):
        x.cache[pages[u], r[u], 5] = 3.0e38
    compare(x, *run(ctx, x))
    x = Case([9000], [1], 16, seed=10)      # the same where the parts of a context are joined
    x.q_lat[..., 5] = 0
    x.q[..., 5] = 0
    x.cache[x.where[0][0], x.where[0][1], 5] = 3.0e38
    compare(x, *run(ctx, x))


def test_strides(ctx):
    """Queries as parts of rows of 576 and more, pages and rows further apart than they are long, wider tables."""
    x = Case([100, 333], [3, 1], 16, seed=11)
    want = run(ctx, x)
    wide = torch.zeros(x.n_tok, x.H, 640, dtype=torch.bfloat16, device=DEV)
    wide[..., 8:520], wide[..., 576:640] = x.q_lat, x.q_rope
    x.q_lat, x.q_rope = wide[..., 8:520], wide[..., 576:640]
    n = x.cache.shape[0]
    big = torch.full((n, 17, 584), float("nan"), dtype=torch.bfloat16, device=DEV)
    big[:, 1:, 8:] = x.cache
    x.cache = big[:, 1:, 8:]
    table = torch.full((2, 50), -1, dtype=torch.int32, device=DEV)
    table[:, :x.table.shape[1]] = x.table
    x.table = table[:, :x.table.shape[1]]
    got = run(ctx, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_offsets_beyond_32_bits(ctx):
    """Pages more than 2^32 elements apart."""
    x = Case([40], [1], 16, page=8, seed=12, spare=0)
    want = run(ctx, x)
    n = x.cache.shape[0]
    step = (1 << 32) // (n - 1) // 8 * 8 + 8
    big = torch.empty(step * (n - 1) + 8 * 576, dtype=torch.bfloat16, device=DEV)
    far = big.as_strided((n, 8, 576), (step, 576, 1))
    far.copy_(x.cache)
    x.cache = far
    got = run(ctx, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_shared_pages(ctx):
    """Two sequences on the same pages, and a page twice in one table."""
    x = Case([64, 64], [1, 1], 16, seed=13)
    x.table[1] = x.table[0]
    x.where[1] = x.where[0]
    compare(x, *run(ctx, x))
    x.table[0, 2] = x.table[0, 1]
    out, lse = run(ctx, x)
    rows = x.rows(1).cpu()
    rows0 = rows.clone()
    rows0[32:48] = rows[16:32]
    compare(x, out, lse, rows=[rows0, rows])


def test_dense_cache(ctx):
    """The decode step's own cache [B, T, 576] as pages: the same as vkv_attend over all of its rows."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    B, T, H = 3, 256, 16
    cache = torch.randn(B, T, 576, generator=g, device=DEV).to(torch.bfloat16)
    ql = torch.randn(B, H, 512, generator=g, device=DEV).to(torch.bfloat16)
    qr = torch.randn(B, H, 64, generator=g, device=DEV).to(torch.bfloat16)
    pages = vkv.Pages.of_cache(cache, torch.full((B,), T, dtype=torch.int32, device=DEV), page=64)
    chunk = vkv.Chunk(ql, qr, torch.arange(B + 1, dtype=torch.int32, device=DEV), 1)
    ws = torch.empty(vkv.chunk_workspace_size(pages, chunk), dtype=torch.uint8, device=DEV)
    out = torch.empty(B, H, 512, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(B, H, device=DEV)
    vkv.chunk_attend(ctx, pages, chunk, ws, SCALE, out, lse)
    step = vkv.Step(cache, ql, qr, T, vkv.VKV_MODE_ROPE)
    w2 = vkv.alloc_workspace(step, 0)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    vkv.attend(ctx, step, w2, 0, None, None, None, 0, SCALE, out2, lse2)
    assert torch.allclose(lse, lse2, rtol=0, atol=1e-5)
    d = (out.double() - out2.double()).norm() / out2.double().norm()
    assert float(d) < 2 * 2.0 ** -8      # both are within a few roundings of the same values


def test_graph_stream_and_repeats(ctx):
    x = Case([900, 1, 333, 70], [1, 1, 3, 0], 40, seed=14, max_q=4, max_kv=1024)
    first = run(ctx, x)
    again = run(ctx, x)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = run(ctx, x)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, there))
    pages, chunk = handles(x)
    graphs = []
    for _ in range(2):      # two graphs, a workspace each
        ws = torch.empty(vkv.chunk_workspace_size(pages, chunk), dtype=torch.uint8, device=DEV)
        out, lse = torch.empty_like(first[0]), torch.empty_like(first[1])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            vkv.chunk_attend(ctx, pages, chunk, ws, SCALE, out, lse)
        graphs.append((g, ws, out, lse))
    for rep in range(3):    # other queries, other lengths
        gen = torch.Generator(device=DEV)
        gen.manual_seed(50 + rep)
        x.q_lat.copy_(torch.randn(x.q_lat.shape, generator=gen, device=DEV).to(torch.bfloat16))
        x.kv_len.copy_(torch.tensor([900 - 100 * rep, 1, 333 - rep, 70], dtype=torch.int32))
        for g, _, out, lse in graphs:
            out.zero_(), lse.zero_()
            g.replay()
        torch.cuda.synchronize()
        want = run(ctx, x)
        for _, _, out, lse in graphs:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), rep
