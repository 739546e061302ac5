"""vkv_cache8_write at the end of a sequence's table: new rows from max_kv on have no place and are dropped, and the rows
that are there keep their bytes; what is written is what a call with the other tokens alone writes."""
import numpy as np
import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged8 import Case8
from test_gpu_write8 import rows

pytestmark = pytest.mark.gpu
DEV, I32 = "cuda", torch.int32


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def write(ctx, x, lens, lat, rope, q_lens, max_q=None):
    cu = torch.tensor([sum(q_lens[:b]) for b in range(len(q_lens) + 1)], dtype=I32, device=DEV)
    kv = torch.tensor(lens, dtype=I32, device=DEV)
    vkv.cache8_write(ctx, vkv.Pages8(x.cache, x.scale, x.table, kv, x.max_kv), lat, rope, cu, max(q_lens) if max_q is None else max_q)
    torch.cuda.synchronize()


def same(x, y):
    return torch.equal(x.cache, y.cache) and torch.equal(x.scale, y.scale)


@pytest.mark.parametrize("page,block", [(16, 16), (16, 4), (32, 2), (8, 1), (64, 64)])
@pytest.mark.parametrize("past", [1, 2, 40])
def test_single_tokens_past_the_table(ctx, page, block, past):
    """Sequences that have filled their tables: each further token, large enough to raise its block's scale, changes nothing."""
    make = lambda: Case8([96, 50, 96], [1, 1, 1], 1, page=page, block=block, seed=page + past, max_kv=96)
    x, y = make(), make()
    lat, rope = rows(3, past, 300.0)
    write(ctx, x, [96 + past, 50, 95 + past], lat, rope, [1, 1, 1])
    write(ctx, y, [0, 50, 0] if past > 1 else [0, 50, 96], lat, rope, [1, 1, 1])      # (a length of 0: its token has no row)
    assert same(x, y)


@pytest.mark.parametrize("page,block", [(16, 16), (16, 4), (32, 2), (8, 1), (64, 64)])
@pytest.mark.parametrize("nq,past,max_q", [(10, 3, 10), (10, 9, 10), (10, 10, 10), (10, 25, 10), (40, 5, 40), (40, 5, 36), (40, 5, 20), (130, 34, 130)])
def test_a_chunk_that_crosses_the_end(ctx, page, block, nq, past, max_q):
    """The first nq - past tokens are the rows up to max_kv (those below 0 dropped too); the others, which are larger, are nowhere
    and have no say in a scale."""
    make = lambda: Case8([96, 70], [nq, 2], 1, page=page, block=block, seed=nq + past, max_kv=96)
    x, y = make(), make()
    lat, rope = rows(nq + 2, nq)
    fit = max(nq - past, 0)
    lat[fit:nq] *= 64
    write(ctx, x, [96 + past, 70], lat, rope, [nq, 2], max_q)
    some = torch.cat([torch.arange(fit), torch.arange(nq, nq + 2)]).to(DEV)
    write(ctx, y, [96 if fit else 0, 70], lat[some], rope[some], [fit, 2], max_q)
    assert same(x, y)


def test_a_sequence_that_grows_past_its_table(ctx):
    """Pages asked for, rows written, as a server does that does not look at its bound: the rows up to it stay as they were."""
    page, width, B = 16, 3, 2
    cache = torch.full((8, page, 640), 0x7F, dtype=torch.uint8, device=DEV)
    scale = torch.full((8, 1), 255, dtype=torch.uint8, device=DEV)
    table, kv, refs = torch.full((B, width), -1, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV), torch.zeros(8, dtype=I32, device=DEV)
    pool = vkv.Pool(table, kv, refs, page, [cache[None], scale[None]])
    ws = torch.empty(vkv.pool_workspace_size(pool), dtype=torch.uint8, device=DEV)
    missing, cu = torch.empty(B, dtype=I32, device=DEV), torch.arange(B + 1, dtype=I32, device=DEV)
    pages = vkv.Pages8(cache, scale, table, kv, width * page)
    full = None
    for step in range(60):
        want = kv + 1
        vkv.pages_reserve(ctx, pool, want, missing, ws)
        kv.copy_(want)
        lat, rope = rows(B, step, 1.0 + step)
        vkv.cache8_write(ctx, pages, lat, rope, cu, 1)
        torch.cuda.synchronize()
        if step == 47:
            full = cache.clone(), scale.clone()       # 48 rows each: the tables are full
        if step > 47:
            assert torch.equal(cache, full[0]) and torch.equal(scale, full[1])
        assert np.all(refs.cpu().numpy() <= 1)


@pytest.mark.parametrize("block", [1, 2, 16])
def test_the_longest_chunk_beside_the_longest_sequence(ctx, block):
    """As many workgroups a sequence as 2^30 tokens take, for one whose block lies at the end of 2^30 rows too: block numbers
    whose rows pass 31 bits.  No page is there but the last one of the second sequence."""
    n, page = 1 << 30, 65536
    cache = torch.full((1, page, 640), 9, dtype=torch.uint8, device=DEV)
    scale = torch.full((1, page // block), 127, dtype=torch.uint8, device=DEV)
    table = torch.full((2, n // page), -1, dtype=I32, device=DEV)
    table[1, -1] = 0
    kv, cu = torch.tensor([n, n - 1], dtype=I32, device=DEV), torch.tensor([0, n, n + 1], dtype=I32, device=DEV)
    lat, rope = torch.ones(1, 512, dtype=torch.bfloat16, device=DEV), torch.ones(1, 64, dtype=torch.bfloat16, device=DEV)
    vkv.cache8_write(ctx, vkv.Pages8(cache, scale, table, kv, n), lat.expand(n + 1, 512), rope.expand(n + 1, 64), cu, n)
    torch.cuda.synchronize()
    older = block > 2                                 # in the new row's block: it keeps its scale, 1; else the new row's is 2^-8
    new, byte = cache[0, page - 2], scale[0, (page - 2) // block]
    assert bool((new[:512] == (0x38 if older else 0x78)).all()) and torch.equal(new[512:].view(torch.bfloat16), rope[0])
    assert int(byte) == (127 if older else 119)
    new.fill_(9)
    byte.fill_(127)
    assert bool((cache == 9).all()) and bool((scale == 127).all())
