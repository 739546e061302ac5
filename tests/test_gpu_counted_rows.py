"""Every row is counted once, wherever the work of a call is cut: with queries of 0 all scores are 0 and all softmax weights
equal, so sums are whole numbers that fp32 holds exactly, and a tile that is lost, repeated or masked wrongly at the
end of a run shows as itself.

Cache row u has a 1 in one dim, its tile's number modulo the dims, and 0 elsewhere.  A query that sees n rows then has
lse = log n and in dim d the share of its rows that lie in tiles of number d: their number times 1 / n, which is rounded
twice in fp32 (the reciprocal, the product) and once to bf16: off by at most 2^-8 (1 + 2^-20) of it.  lse is log2 n (1 ulp),
times ln 2 (rounded), rounded: 4 2^-24 of it.  A lost tile is at least a fifth of a dim's share, and its rows' share of
exp(lse)."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged import Case
from test_gpu_chunk import ctx, run     # noqa: F401 (the context's fixture)
from test_gpu_evict import accumulate

pytestmark = pytest.mark.gpu
DEV = "cuda"


def shares(n_seen, rows, tile, dims):
    """[len(n_seen), dims]: how many of a query's first n rows lie in tiles of number d modulo dims."""
    hot = torch.zeros(rows + 1, dims, dtype=torch.float64)
    u = torch.arange(rows)
    hot[u + 1, u // tile % dims] = 1.0
    return hot.cumsum(0)[n_seen]


def check(out, lse, n_seen, counts):
    n = n_seen.double()[:, None]
    want = torch.where(n > 0, counts / n.clamp(min=1), 0.0)
    assert bool(((out.double() - want).abs() <= want * 2.0 ** -8 * (1 + 2.0 ** -20)).all())
    log = torch.log(n_seen.double())                       # -inf: sees nothing
    some = n_seen > 0
    assert torch.equal(lse[~some].double(), log[~some])
    assert bool(((lse[some].double() - log[some]).abs() <= 4 * 2.0 ** -24 * log[some]).all())


CHUNKS = [
    (16, [20011], [1], None), (16, [20011, 3, 9000], [1, 1, 1], None), (1, [70001], [1], None), (8, [8192, 8193], [4, 2], None),
    (16, [15000], [4], None), (20, [9999, 31], [3, 2], None),                          # 33 to 64 rows of queries
    (128, [12345], [3], None), (128, [20011, 700, 0, 33, 5000], [1] * 5, None), (59, [2176] * 11, [21] * 11, None),
    (40, [3000, 1], [33, 2], None), (16, [500], [500], None), (128, [40], [60], None),
    (8, [200 + 7 * b for b in range(33)], [17] * 33, 512),                             # a workgroup per block of rows
]


@pytest.mark.parametrize("H,kv_lens,q_lens,max_q", CHUNKS)
def test_chunk(ctx, H, kv_lens, q_lens, max_q):     # noqa: F811
    x = Case(kv_lens, q_lens, H, page=64, seed=1, max_q=max_q)
    x.q_lat.zero_(), x.q_rope.zero_()
    for b, n in enumerate(kv_lens):
        u = torch.arange(n, device=DEV)
        rows = torch.zeros(n, 576, dtype=torch.bfloat16, device=DEV)
        rows[u, u // 32 % 512] = 1.0
        x.cache[x.where[b]] = rows
    out, lse = run(ctx, x)
    out, lse, at = out.cpu(), lse.cpu(), 0
    for n, nq in zip(kv_lens, q_lens):
        seen = (n - nq + 1 + torch.arange(nq)).clamp(min=0).repeat_interleave(H)
        check(out[at:at + nq].reshape(-1, 512), lse[at:at + nq].reshape(-1), seen, shares(seen, n, 32, 512))
        at += nq


@pytest.mark.parametrize("dims,lens,H,Hk", [((128, 64, 128), [5000, 1, 127, 129, 900], 4, 2), ((128, 0, 128), [2307, 64, 65], 16, 4),
                                            ((64, 0, 64), [3000, 17, 640], 8, 1)])
def test_prompt(ctx, dims, lens, H, Hk):     # noqa: F811
    dn, dr, dv = dims
    n = sum(lens)
    z = lambda *s: torch.randn(*s, device=DEV).to(torch.bfloat16)
    v = torch.zeros(n, Hk, dv, dtype=torch.bfloat16, device=DEV)
    at = 0
    for k in lens:
        u = torch.arange(k, device=DEV)
        v[at + u, :, u // 64 % dv] = 1.0
        at += k
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    pr = vkv.Prompt(torch.zeros(n, H, dn + dr, dtype=torch.bfloat16, device=DEV), z(n, Hk, dn), v, cu, max(lens),
                    k_rope=z(n, dr) if dr else None)
    out, lse = torch.empty(n, H, dv, dtype=torch.bfloat16, device=DEV), torch.empty(n, H, device=DEV)
    vkv.prompt_attend(ctx, pr, 0.1, out, lse)
    out, lse, at = out.cpu(), lse.cpu(), 0
    for k in lens:
        seen = torch.arange(1, k + 1)
        counts = shares(seen, k, 64, dv)
        for h in range(H):
            check(out[at:at + k, h], lse[at:at + k, h], seen, counts)
        at += k


@pytest.mark.parametrize("H,kv_lens,q_lens", [
    (16, [20011, 1, 0, 33], [1, 1, 1, 1]), (128, [32768, 5000], [1, 2]), (100, [4097], [2]),     # few queries: one and two streams
    (9, [14406, 14406], [41, 41]), (128, [700], [40]), (31, [17620, 300], [48, 300]), (1, [1000], [1000]), (64, [65536], [32]),
    (16, [257 + 31 * b for b in range(40)], [b for b in range(40)]),
])
def test_weights(ctx, H, kv_lens, q_lens):     # noqa: F811
    """With an lse of 0 a row's weight is the number of queries that see it."""
    x = Case(kv_lens, q_lens, H, page=64, seed=2)
    x.q_lat.zero_(), x.q_rope.zero_()
    weight = accumulate(ctx, x, torch.zeros(x.n_tok, H, device=DEV), 0.0, None, torch.full((len(kv_lens), x.max_kv), -3.0, device=DEV))
    for b, (n, nq) in enumerate(zip(kv_lens, q_lens)):
        want = H * torch.minimum(torch.full((n,), nq), n - torch.arange(n))          # row u: the tokens from u - (n - nq) on
        assert torch.equal(weight[b, :n].cpu(), want.float()) and bool((weight[b, n:] == -3.0).all())
