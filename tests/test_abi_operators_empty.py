"""Calls of the paged operators that have nothing to do, as an empty tensor makes them: its address is NULL."""
import ctypes

import pytest

from test_abi_operators import CHUNK, EVICT, FAKE, PAGES, chunk, make, weights


@pytest.fixture(scope="module")
def vkv():
    import paper_2609_03949_amd as vkv
    vkv.load()
    return vkv


@pytest.fixture()
def ctx():
    return ctypes.create_string_buffer(1 << 14)


NO_TOKENS = dict(n_tok=0, q_lat=None, q_rope=None)
NO_ROWS = dict(max_kv=0, table=None, table_stride=0)


def test_no_tokens(vkv, ctx):
    assert chunk(vkv, ctx, NO_TOKENS, out=None, lse=None) == 0
    assert chunk(vkv, ctx, dict(NO_TOKENS, **NO_ROWS), out=None, lse=None) == 0
    assert weights(vkv, ctx, dict(NO_TOKENS, **NO_ROWS), lse=None, prev=None, weight=None, stride=0) == 0


def test_no_rows(vkv, ctx):
    assert weights(vkv, ctx, NO_ROWS) == 0
    assert weights(vkv, ctx, NO_ROWS, weight=None, prev=None, stride=0) == 0


@pytest.mark.parametrize("change", [dict(NO_TOKENS, max_q=0), NO_TOKENS, NO_ROWS, dict(NO_TOKENS, **NO_ROWS)])
def test_workspace_sizes(vkv, change):
    lib = vkv.load()
    pg = make(vkv._Pages, PAGES, **{k: v for k, v in change.items() if k in PAGES})
    ch = make(vkv._Chunk, CHUNK, **{k: v for k, v in change.items() if k in CHUNK})
    n = ctypes.c_size_t(1)
    assert lib.vkv_chunk_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n)) == 0
    assert lib.vkv_weight_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n)) == 0


def test_still_required_where_there_is_work(vkv, ctx):
    for bad in (dict(q_lat=None), dict(q_rope=None), dict(n_tok=0, cu=None), dict(table=None), dict(max_kv=0, kv_len=None),
                dict(max_kv=0, cache=None)):
        assert chunk(vkv, ctx, bad) == -1 and weights(vkv, ctx, bad) == -1
    assert chunk(vkv, ctx, NO_ROWS, out=None) == -1 and chunk(vkv, ctx, NO_ROWS, lse=None) == -1
    assert weights(vkv, ctx, {}, lse=None) == -1 and weights(vkv, ctx, NO_TOKENS, weight=None) == -1
    lib = vkv.load()
    pg = make(vkv._Pages, PAGES, **NO_ROWS)
    a = dict(EVICT, weight_out=None)
    assert lib.vkv_cache_evict(ctx, ctypes.byref(pg), a["kept"], a["count"], a["keep"], a["origin"], FAKE, 0, None, None) == -1
    assert lib.vkv_weight_select(ctx, None, 2, 1000, 1000, FAKE, 10, 0, 0, FAKE, FAKE, None) == -1


def test_bindings_take_empty_tensors(vkv):
    torch = pytest.importorskip("torch")
    bf, i32 = torch.bfloat16, torch.int32
    pg = vkv.Pages(torch.zeros(6, 16, 576, dtype=bf), torch.zeros(2, 0, dtype=i32), torch.zeros(2, dtype=i32), 0)
    for H in (1, 4):
        ch = vkv.Chunk(torch.zeros(0, H, 512, dtype=bf), torch.zeros(0, H, 64, dtype=bf), torch.zeros(3, dtype=i32), 1)
        assert vkv.chunk_workspace_size(pg, ch) > 0 and vkv.weight_workspace_size(pg, ch) == 0
