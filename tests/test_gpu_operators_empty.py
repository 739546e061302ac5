"""The operators around the step on tensors without elements: no new tokens, no cache rows, no prompt."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged import Case

pytestmark = pytest.mark.gpu
DEV, BF, I32 = "cuda", torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def i32(*v):
    return torch.tensor(v, dtype=I32, device=DEV)


@pytest.mark.parametrize("max_q", [0, 1, 100])
def test_no_new_tokens(ctx, max_q):
    """The attention writes nothing, the weights are carried over (or start at 0), rows behind are left."""
    x = Case([70, 0, 33], [0, 0, 0], 16, seed=1, max_q=max_q)
    pages = vkv.Pages(x.cache, x.table, x.kv_len, x.max_kv)
    none = torch.empty(0, 16, 512, dtype=BF, device=DEV)
    chunk = vkv.Chunk(none, torch.empty(0, 16, 64, dtype=BF, device=DEV), x.cu, max_q)
    lse = torch.empty(0, 16, device=DEV)
    ws = torch.empty(max(vkv.chunk_workspace_size(pages, chunk), 256), dtype=torch.uint8, device=DEV)
    vkv.chunk_attend(ctx, pages, chunk, ws, 0.1, torch.empty_like(none), lse)
    n = vkv.weight_workspace_size(pages, chunk)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    prev = torch.rand(3, 72, device=DEV)
    for p in (prev, None):
        weight = torch.full((3, 72), -3.0, device=DEV)
        vkv.weight_accumulate(ctx, pages, chunk, lse, ws, 0.1, 0.5, p, weight)
        for b, rows in enumerate((70, 0, 33)):
            want = torch.zeros(rows, device=DEV) if p is None else prev[b, :rows]
            assert torch.equal(weight[b, :rows], want) and bool((weight[b, rows:] == -3.0).all())


def test_no_cache_rows(ctx):
    """Tokens over an empty cache see nothing; its tier is empty and nothing moves."""
    cache = torch.randn(4, 16, 576, device=DEV).to(BF)
    was = cache.clone()
    pages = vkv.Pages(cache, torch.empty(2, 0, dtype=I32, device=DEV), i32(0, 0), 0)
    q = torch.randn(3, 8, 576, device=DEV).to(BF)
    chunk = vkv.Chunk(q[..., :512], q[..., 512:], i32(0, 1, 3), 2)
    ws = torch.empty(vkv.chunk_workspace_size(pages, chunk), dtype=torch.uint8, device=DEV)
    out, lse = torch.full((3, 8, 512), 7.0, dtype=BF, device=DEV), torch.full((3, 8), 7.0, device=DEV)
    vkv.chunk_attend(ctx, pages, chunk, ws, 0.1, out, lse)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    weight = torch.empty(2, 0, device=DEV)
    vkv.weight_accumulate(ctx, pages, chunk, lse, None, 0.1, 0.5, None, weight)
    kept, count = torch.full((2, 5), 9, dtype=I32, device=DEV), torch.full((2,), 9, dtype=I32, device=DEV)
    vkv.weight_select(ctx, weight, pages.tensors[2], 0, 1, 2, kept, count)
    assert bool((kept == -1).all()) and bool((count == 0).all())
    origin, moved = torch.full((2, 5), 9, dtype=I32, device=DEV), torch.full((2, 5), 9.0, device=DEV)
    vkv.cache_evict(ctx, pages, kept, count, origin, weight, moved)
    assert bool((origin == -1).all()) and bool((moved == 0).all()) and torch.equal(cache, was)


def test_no_prompt(ctx):
    pr = vkv.Prompt(torch.empty(0, 4, 128, dtype=BF, device=DEV), torch.empty(0, 2, 128, dtype=BF, device=DEV),
                    torch.empty(0, 2, 128, dtype=BF, device=DEV), i32(0, 0), 0)
    vkv.prompt_attend(ctx, pr, 0.1, torch.empty(0, 4, 128, dtype=BF, device=DEV), torch.empty(0, 4, device=DEV))
