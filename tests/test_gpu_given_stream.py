"""The operators' `stream` argument: the call runs on that stream and on no other, with the same result."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged import Case
from test_gpu_chunk import SCALE, ctx     # noqa: F401 (the context's fixture)

pytestmark = pytest.mark.gpu
DEV, BF, I32 = "cuda", torch.bfloat16, torch.int32


def operators(ctx):     # noqa: F811
    """name -> (call(outputs, stream), fresh outputs)."""
    x = Case([900, 300, 70], [3, 1, 2], 40, seed=1)
    many = Case([700, 90], [30, 4], 16, seed=2)
    tier = Case([900, 300], [1, 1], 1, seed=3)
    prev, lse = torch.rand(3, 900, device=DEV), torch.randn(6, 40, device=DEV) + 6
    lse_many = torch.randn(34, 16, device=DEV) + 6
    kept = torch.stack([torch.randperm(300, device=DEV)[:64].sort().values for _ in range(2)]).to(I32)
    count = torch.full((2,), 64, dtype=I32, device=DEV)
    q, k, v = (torch.randn(300, h, 128, device=DEV).to(BF) for h in (8, 2, 2))
    prompt = vkv.Prompt(q, k, v, torch.tensor([0, 100, 300], dtype=I32, device=DEV), 200)

    def views(c):
        pages, chunk = vkv.Pages(c.cache, c.table, c.kv_len, c.max_kv), vkv.Chunk(c.q_lat, c.q_rope, c.cu, c.max_q)
        size = max(vkv.chunk_workspace_size(pages, chunk), vkv.weight_workspace_size(pages, chunk), 256)
        return pages, chunk, torch.empty(size, dtype=torch.uint8, device=DEV)

    p1, c1, w1 = views(x)
    p2, c2, w2 = views(many)
    full = lambda *s, dtype=torch.float32: torch.full(s, 7, dtype=dtype, device=DEV)
    cache = tier.cache.clone()

    def evict(o, s):
        vkv.cache_evict(ctx, vkv.Pages(o[0], tier.table, tier.kv_len, tier.max_kv), kept, count, o[1], None, None, s)

    return dict(
        prompt=(lambda o, s: vkv.prompt_attend(ctx, prompt, SCALE, o[0], o[1], s), lambda: [full(300, 8, 128, dtype=BF), full(300, 8)]),
        chunk=(lambda o, s: vkv.chunk_attend(ctx, p1, c1, w1, SCALE, o[0], o[1], s), lambda: [full(6, 40, 512, dtype=BF), full(6, 40)]),
        weights_few=(lambda o, s: vkv.weight_accumulate(ctx, p1, c1, lse, w1, SCALE, 0.5, prev, o[0], s), lambda: [full(3, 900)]),
        weights_many=(lambda o, s: vkv.weight_accumulate(ctx, p2, c2, lse_many, w2, SCALE, 0.5, None, o[0], s), lambda: [full(2, 700)]),
        select=(lambda o, s: vkv.weight_select(ctx, prev, x.kv_len, 900, 4, 16, o[0], o[1], s), lambda: [full(3, 50, dtype=I32), full(3, dtype=I32)]),
        evict=(evict, lambda: [cache.clone(), full(2, 64, dtype=I32)]))


def bits(t):
    return t.view(torch.int16) if t.dtype == BF else t


@pytest.mark.parametrize("name", ["prompt", "chunk", "weights_few", "weights_many", "select", "evict"])
def test_runs_on_the_given_stream(ctx, name):     # noqa: F811
    call, fresh = operators(ctx)[name]
    want, blank, got = fresh(), fresh(), fresh()
    call(want, None)
    given, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    # what is launched on a stream that is being captured is recorded and does not run; the current stream runs what it gets
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=given, capture_error_mode="relaxed"):
        with torch.cuda.stream(other):
            call(got, given)
    torch.cuda.synchronize()
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, blank))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want))
    assert not all(torch.equal(bits(a), bits(b)) for a, b in zip(got, blank))
    # and without a capture
    again = fresh()
    given.wait_stream(torch.cuda.current_stream())
    call(again, given)
    given.synchronize()
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(again, want))
