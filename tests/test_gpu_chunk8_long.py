"""vkv_chunk8_attend over long contexts, against 64 bits with bounds that tell fp16 weights from coarser ones and a cache row from any
other (_long8.py): every split of the rows and of the work, runs that begin and end within contexts, pages of every kind."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from _long8 import SCALE, Exact, marked, spread
from _paged8 import Case8

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def attend(ctx, x, tiles, max_q=None):
    """tiles, max_q: what the call's bounds allow for; which kernel is taken goes by them."""
    max_kv = max(x.max_kv, 64 * tiles)
    table = torch.full((x.table.shape[0], -(-max_kv // x.page)), -1, dtype=torch.int32, device=DEV)
    table[:, :x.table.shape[1]] = x.table
    pages = vkv.Pages8(x.cache, x.scale, table, x.kv_len, max_kv)
    chunk = vkv.Chunk(x.q_lat, x.q_rope, x.cu, x.max_q if max_q is None else max_q)
    ws = torch.full((max(vkv.chunk8_workspace_size(pages, chunk), 256),), 0xFF, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(x.n_tok, x.H, 512, dtype=torch.bfloat16, device=DEV), torch.empty(x.n_tok, x.H, device=DEV)
    vkv.chunk8_attend(ctx, pages, chunk, ws, SCALE, out, lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("H,q,kv,page,block", [
    (16, [1, 1, 1], [20011, 700, 9000], 64, 16), (16, [1], [33000], 16, 16), (32, [1, 2], [12000, 801], 16, 4), (64, [1], [20011], 64, 16),
    (128, [3], [12345], 128, 32), (128, [1, 1], [7000, 16001], 8, 8), (5, [40], [6000], 1, 1), (24, [9], [9999], 64, 64)])
@pytest.mark.parametrize("own", [False, True], ids=["alike", "own"])
@pytest.mark.parametrize("kind", [marked, lambda x: x], ids=["marked", "random"])
def test_every_row_counts_once(ctx, H, q, kv, page, block, kind, own):
    x = kind(spread(Case8(kv, q, H, page=page, block=block, seed=H + len(q)), 1, own=own))
    exact = [Exact(x, b) for b in range(len(q))]
    for tiles, max_q in ((0, None), (3000, None), (9000, None), (0, 1 << 14)):      # units of 16 and more rows; of 128; one workgroup each
        out, lse = attend(ctx, x, -(-tiles // len(q)), max_q)
        at = 0
        for b, n in enumerate(q):
            exact[b].check(out[at:at + n].reshape(-1, 512), lse[at:at + n].reshape(-1))
            at += n
