"""Calls whose work takes more workgroups than one grid dimension holds (2^32 work-items): very many sequences,
nearly all of them empty, against the same call with the others alone."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

pytestmark = pytest.mark.gpu
DEV, BF, I32 = "cuda", torch.bfloat16, torch.int32
SCALE = 1.0 / math.sqrt(192.0)
MANY = 65535


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def normal(*shape, seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(BF)


def test_prompt(ctx):
    """65535 sequences x 128 heads x 3 blocks of rows: 25 million workgroups of 256."""
    n, H = 500, 128
    q, k, v = normal(n, H, 64), normal(n, 1, 64, seed=2), normal(n, 1, 64, seed=3)
    cu = torch.full((MANY + 1,), 100, dtype=I32)
    cu[0], cu[MANY - 1], cu[MANY] = 0, 200, n
    got, want = [], []
    for offsets, to in ((cu, got), (torch.tensor([0, 100, 200, n], dtype=I32), want)):
        out, lse = torch.full((n, H, 64), 7.0, dtype=BF, device=DEV), torch.full((n, H), 7.0, device=DEV)
        vkv.prompt_attend(ctx, vkv.Prompt(q, k, v, offsets.to(DEV), 300), SCALE, out, lse)
        to += [out, lse]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_chunk(ctx):
    """65535 sequences x 130 blocks of rows: 8.5 million workgroups of 512."""
    H, page = 128, 64
    cache, q = normal(2, page, 576), normal(3, H, 576, seed=2)
    live = [70, MANY - 1]
    table, kv, cu = torch.full((MANY, 1), -1, dtype=I32), torch.zeros(MANY, dtype=I32), torch.zeros(MANY + 1, dtype=I32)
    table[live, 0], kv[live] = torch.tensor([1, 0], dtype=I32), torch.tensor([60, 33], dtype=I32)
    cu[71:], cu[MANY] = 2, 3
    few = (table[live], kv[live], torch.tensor([0, 2, 3], dtype=I32), 600)
    got, want = [], []
    for (t, n, c, max_q), to in (((table, kv, cu, 130), got), (few, want)):
        pages = vkv.Pages(cache, t.to(DEV), n.to(DEV), page)
        chunk = vkv.Chunk(q[..., :512], q[..., 512:], c.to(DEV), max_q)
        assert vkv.chunk_workspace_size(pages, chunk) == 0        # a workgroup per block of rows in both
        ws = torch.empty(256, dtype=torch.uint8, device=DEV)
        out, lse = torch.full((3, H, 512), 7.0, dtype=BF, device=DEV), torch.full((3, H), 7.0, device=DEV)
        vkv.chunk_attend(ctx, pages, chunk, ws, SCALE, out, lse)
        to += [out, lse]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool(torch.isfinite(want[1]).all())


def test_evict(ctx):
    """65535 sequences x 1025 groups of 8 slots: 67 million workgroups of 64."""
    K, page, rows = 8200, 64, 9000
    used = -(-rows // page)
    cache = normal(2 * used, page, 576)
    live = [5, MANY - 1]
    table = torch.full((MANY, used), -1, dtype=I32, device=DEV)
    table[live] = torch.arange(2 * used, dtype=I32, device=DEV).view(2, used)
    kv, count = torch.zeros(MANY, dtype=I32, device=DEV), torch.zeros(MANY, dtype=I32, device=DEV)
    kv[live] = rows
    g = torch.Generator()
    g.manual_seed(4)
    tier = torch.stack([torch.randperm(rows, generator=g)[:K].sort().values for _ in live]).to(I32).to(DEV)
    kept = torch.full((MANY, K), -1, dtype=I32, device=DEV)
    kept[live], count[live] = tier, K
    other = cache.clone()
    vkv.cache_evict(ctx, vkv.Pages(cache, table, kv, rows), kept, count)
    vkv.cache_evict(ctx, vkv.Pages(other, table[live].contiguous(), kv[live], rows), tier, count[live])
    assert torch.equal(cache, other)
    assert not torch.equal(cache, normal(2 * used, page, 576))
