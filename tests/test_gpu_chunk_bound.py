"""Sequences with more new tokens than max_q: the first max_q of them are computed, each as a token of the whole chunk
(token i sees the rows up to kv_len - nq + i, nq all new tokens), and the chunk's rows are all of its tokens' rows."""
import math

import pytest
import torch

from _attention import attention, check
from _paged import Case
from test_gpu_chunk import SCALE, ctx, run      # noqa: F401 (the context's fixture)
from test_gpu_evict import accumulate, expected, true_lse

pytestmark = pytest.mark.gpu
DEV = "cuda"

CASES = [
    (16, [10, 1, 50], [100, 40, 60], 4),          # few rows
    (128, [3, 2, 40], [70, 33, 1000], 2),         # 256 rows of queries
    (128, [9, 3, 4], [600, 33, 3], 3),            # more: runs of blocks of cache rows
    (16, [700, 30], [900, 20], 20),               # new rows that no computed token sees, over several blocks
    (40, [300, 20], [290, 20], 10),               # tokens whose rows were never in the cache
    (8, [600] * 3, [2000, 600, 650], 512),        # a workgroup per block of rows
]


@pytest.mark.parametrize("H,q_lens,kv_lens,max_q", CASES)
def test_attention(ctx, H, q_lens, kv_lens, max_q):      # noqa: F811
    x = Case(kv_lens, q_lens, H, seed=H + max_q, max_q=max_q, page=32)
    out, lse = run(ctx, x)
    at = 0
    for b, nq in enumerate(q_lens):
        n = min(nq, max_q)
        kv, seen = x.rows(b).cpu(), x.seen(b)[:n, None, :].expand(n, H, kv_lens[b]).reshape(n * H, -1)
        o, l, ot, lt = attention(x.q[at:at + n].reshape(n * H, 576), kv, kv[:, :512], seen, SCALE)
        check(f"lse of sequence {b}", lse[at:at + n].reshape(-1), l, lt)
        check(f"out of sequence {b}", out[at:at + n].reshape(-1, 512), o, ot)
        assert bool((out[at + n:at + nq] == 7.0).all()) and bool((lse[at + n:at + nq] == 7.0).all())
        at += nq


@pytest.mark.parametrize("H,q_lens,kv_lens,max_q", CASES)
@pytest.mark.parametrize("decay", [0.0, 0.75])
def test_weights(ctx, H, q_lens, kv_lens, max_q, decay):      # noqa: F811
    x = Case(kv_lens, q_lens, H, seed=H + max_q, max_q=max_q, page=32)
    lse = true_lse(x)
    first, at = lse.clone(), 0
    for nq in q_lens:
        first[at + min(nq, max_q):at + nq] = -math.inf        # a query that draws nothing
        at += nq
    prev = torch.rand(len(kv_lens), x.max_kv, device=DEV)
    want, tol = expected(x, first, decay, prev)
    out = accumulate(ctx, x, lse, decay, prev, torch.full_like(prev, -3.0))
    for b, n in enumerate(kv_lens):
        check(f"weight of sequence {b}", out[b, :n], want[b], tol[b])
        assert bool((out[b, n:] == -3.0).all())
