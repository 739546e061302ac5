"""vkv_cache_evict where rows or slots lie on pages that do not exist, and on tables that are no tier: what moves,
and what origin and the weights then say."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def evict(ctx, x, lists, K):
    """origin, weight_out, the weights and the rows of every sequence before the call."""
    B = len(lists)
    kept = torch.full((B, K), -1, dtype=torch.int32)
    for b, rows in enumerate(lists):
        kept[b, :len(rows)] = torch.tensor(rows, dtype=torch.int32)
    count = torch.tensor([len(r) for r in lists], dtype=torch.int32, device=DEV)
    before = [x.rows(b).clone() for b in range(B)]
    weight = torch.rand(B, x.max_kv, device=DEV)
    origin = torch.full((B, K), 55, dtype=torch.int32, device=DEV)
    out = torch.full((B, K), 55.0, device=DEV)
    vkv.cache_evict(ctx, vkv.Pages(x.cache, x.table, x.kv_len, x.max_kv), kept.to(DEV), count, origin, weight, out)
    return origin.cpu(), out.cpu(), weight.cpu(), before


def check(x, b, origin, out, weight, before, want, n):
    """Slot j holds row want[j] of the sequence (-1: what it held), with that row's weight (0)."""
    assert origin[b].tolist() == want + [-1] * (origin.shape[1] - len(want))
    for j, u in enumerate(want):
        assert float(out[b, j]) == (float(weight[b, u]) if u >= 0 else 0.0)
    assert bool((out[b, len(want):] == 0).all())
    after = x.rows(b)
    rows = [u if u >= 0 else j for j, u in enumerate(want)] + list(range(len(want), n))
    assert torch.equal(after.view(torch.int16), before[b].view(torch.int16)[torch.tensor(rows, device=DEV)])


@pytest.mark.parametrize("entry", [-1, 1 << 30])
def test_rows_on_absent_pages(ctx, entry):
    """Pages of 16 rows, 64 of them in three sequences: a source page, a slot page, and the page of kept rows that would stay."""
    x = Case([64, 64, 64, 64], [1] * 4, 1, page=16, seed=9)
    x.table[0, 3] = entry                   # rows 48..63
    x.table[1, 0] = entry                   # slots 0..15
    x.table[2, 1] = entry                   # rows and slots 16..31
    tiers = [[40, 41, 50, 63], [0, 3, 17, 20, 40], list(range(10, 20)) + list(range(30, 50)), [1, 33, 34]]
    origin, out, weight, before = evict(ctx, x, tiers, 32)
    check(x, 0, origin, out, weight, before, [40, 41, -1, -1], 64)
    check(x, 1, origin, out, weight, before, [-1] * 5, 64)
    # slots 0..29: 10..15 stay, 16..19 would; the holes 0..9 take 30, 31 (absent), 32..39, and 20..29 lie on the absent page
    check(x, 2, origin, out, weight, before, [-1, -1] + list(range(32, 40)) + list(range(10, 16)) + [-1] * 14, 64)
    check(x, 3, origin, out, weight, before, [33, 1, 34], 64)


def test_entries_that_are_not_ascending_do_not_move(ctx):
    """Descending and repeated entries, and rows that are none between rows that are."""
    x = Case([100] * 4, [1] * 4, 1, page=16, seed=10)
    tiers = [[99, 98, 97, 96], [5, 5, 70, 70], [60, 1 << 30, 70, 71], [0, 2, 50, 49, 51]]
    origin, out, weight, before = evict(ctx, x, tiers, 8)
    check(x, 0, origin, out, weight, before, [99, -1, -1, -1], 100)
    check(x, 1, origin, out, weight, before, [5, -1, 70, -1], 100)
    check(x, 2, origin, out, weight, before, [60, -1, -1, 71], 100)
    check(x, 3, origin, out, weight, before, [0, 50, 2, -1, 51], 100)
