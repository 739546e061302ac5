"""Host-side checks of the prompt, chunk and eviction entry points (no GPU needed): what they refuse, with
which status, before they touch the device, and what they do not need a device for."""
import ctypes

import pytest

FAKE = 1 << 20          # aligned non-null host value; never dereferenced


@pytest.fixture(scope="module")
def vkv():
    import paper_2609_03949_amd as vkv
    vkv.load()
    return vkv


@pytest.fixture()
def ctx():
    """Zeroed memory in a context's place: a refused call only writes its error text there."""
    return ctypes.create_string_buffer(1 << 14)


def make(cls, base, **kw):
    s = cls()
    for k, v in {**base, **kw}.items():
        setattr(s, k, v)
    return s


PROMPT = dict(n_seq=2, n_tok=100, max_len=60, H=8, Hk=2, dn=128, dr=64, dv=128, q=FAKE, q_tok_stride=8 * 192,
              q_head_stride=192, k=FAKE, k_tok_stride=256, k_head_stride=128, k_rope=FAKE, k_rope_tok_stride=64, v=FAKE,
              v_tok_stride=256, v_head_stride=128, cu=FAKE)


def prompt(vkv, ctx, scale=0.1, out=FAKE, lse=FAKE, **kw):
    s = make(vkv._Prompt, PROMPT, **kw)
    return vkv.load().vkv_prompt_attend(ctx, ctypes.byref(s), scale, out, lse, None)


@pytest.mark.parametrize("change,code", [
    (dict(n_seq=0), -2), (dict(n_seq=65536), -2), (dict(H=0), -2), (dict(H=129, Hk=129), -2), (dict(Hk=3), -2), (dict(Hk=0), -2),
    (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(max_len=-1), -2),
    (dict(dn=96), -4), (dict(dr=32), -4), (dict(dv=64), -4), (dict(dn=64, dr=0), -4),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(cu=None), -1), (dict(out=None), -1), (dict(lse=None), -1),
    (dict(k_rope=None), -1), (dict(dr=0), -1),
    (dict(q=FAKE + 8), -3), (dict(k=FAKE + 2), -3), (dict(v=FAKE + 4), -3), (dict(k_rope=FAKE + 8), -3), (dict(out=FAKE + 8), -3),
    (dict(q_tok_stride=1540), -3), (dict(k_head_stride=-8), -3), (dict(k_rope_tok_stride=63), -3), (dict(v_tok_stride=4), -3),
    (dict(n_seq=65535, H=128, Hk=2, n_tok=(1 << 31) - 1, max_len=(1 << 31) - 1), -2),
])
def test_prompt_refusals(vkv, ctx, change, code):
    assert prompt(vkv, ctx, **change) == code
    assert vkv.load().vkv_last_error(ctx)


def test_prompt_without_work_needs_no_device(vkv, ctx):
    assert prompt(vkv, ctx, n_tok=0, q=None, k=None, v=None, out=None) == 0
    assert prompt(vkv, ctx, max_len=0) == 0
    assert vkv.load().vkv_prompt_attend(None, None, 0.1, None, None, None) == -1
    assert vkv.load().vkv_prompt_attend(ctx, None, 0.1, None, None, None) == -1


def test_prompt_binding_checks_its_tensors(vkv):
    torch = pytest.importorskip("torch")
    bf = torch.bfloat16
    q, k, v = torch.zeros(5, 4, 192, dtype=bf), torch.zeros(5, 2, 128, dtype=bf), torch.zeros(5, 2, 128, dtype=bf)
    kr, cu = torch.zeros(5, 64, dtype=bf), torch.tensor([0, 5], dtype=torch.int32)
    pr = vkv.Prompt(q, k, v, cu, 5, k_rope=kr)
    assert (pr.c.dn, pr.c.dr, pr.c.dv, pr.c.H, pr.c.Hk, pr.c.n_seq, pr.c.n_tok) == (128, 64, 128, 4, 2, 1, 5)
    for bad in (dict(q=q.float()), dict(q=q[:4]), dict(k=k[:4]), dict(v=v[:, :1]), dict(k_rope=None), dict(k_rope=kr[:3]),
                dict(cu=cu.long()), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(v=v.half())):
        with pytest.raises(ValueError):
            a = dict(dict(q=q, k=k, v=v, cu=cu, k_rope=kr), **bad)
            vkv.Prompt(a["q"], a["k"], a["v"], a["cu"], 5, k_rope=a["k_rope"])


PAGES = dict(B=3, max_kv=1000, n_pages=64, page=64, cache=FAKE, row_stride=576, page_stride=64 * 576, table=FAKE,
             table_stride=16, kv_len=FAKE)
CHUNK = dict(n_tok=7, H=16, max_q=4, q_lat=FAKE, q_lat_stride=512, q_rope=FAKE, q_rope_stride=64, cu=FAKE)
PAGES_BAD = [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(max_kv=-1), -2), (dict(max_kv=(1 << 30) + 1), -2), (dict(n_pages=0), -2),
    (dict(n_pages=1 << 31), -2), (dict(page=0), -4), (dict(page=48), -4), (dict(page=1 << 17), -4), (dict(page=-64), -4),
    (dict(cache=None), -1), (dict(table=None), -1), (dict(kv_len=None), -1), (dict(cache=FAKE + 8), -3), (dict(table=FAKE + 2), -3),
    (dict(kv_len=FAKE + 1), -3), (dict(row_stride=568), -3), (dict(row_stride=580), -3), (dict(page_stride=-8), -3),
    (dict(page_stride=4), -3), (dict(table_stride=15), -2), (dict(page_stride=1 << 35), -2), (dict(row_stride=1 << 35), -2),
]
CHUNK_BAD = [
    (dict(H=0), -2), (dict(H=129), -2), (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(max_q=-1), -2),
    (dict(max_q=1 << 27), -2), (dict(q_lat=None), -1), (dict(q_rope=None), -1), (dict(cu=None), -1), (dict(q_lat=FAKE + 8), -3),
    (dict(q_rope=FAKE + 2), -3), (dict(q_lat_stride=-8), -3), (dict(q_lat_stride=513), -3), (dict(q_rope_stride=68), -3),
]


def chunk(vkv, ctx, change, ws=FAKE, ws_bytes=None, scale=0.1, out=FAKE, lse=FAKE):
    lib = vkv.load()
    pg = make(vkv._Pages, PAGES, **{k: v for k, v in change.items() if k in PAGES})
    ch = make(vkv._Chunk, CHUNK, **{k: v for k, v in change.items() if k in CHUNK})
    n = ctypes.c_size_t(0)
    if ws_bytes is None:
        rc = lib.vkv_chunk_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n))
        if rc:
            return rc
        ws_bytes = n.value
    return lib.vkv_chunk_attend(ctx, ctypes.byref(pg), ctypes.byref(ch), ws, ws_bytes, scale, out, lse, None)


@pytest.mark.parametrize("change,code", PAGES_BAD + CHUNK_BAD)
def test_chunk_refusals(vkv, ctx, change, code):
    assert chunk(vkv, ctx, change) == code and vkv.load().vkv_last_error(None)
    assert chunk(vkv, ctx, change, ws_bytes=1 << 40) == code and vkv.load().vkv_last_error(ctx)


def test_chunk_call_refusals(vkv, ctx):
    assert chunk(vkv, ctx, {}, scale=0.0) == -1 and chunk(vkv, ctx, {}, scale=float("nan")) == -1
    assert chunk(vkv, ctx, {}, out=None) == -1 and chunk(vkv, ctx, {}, lse=None) == -1
    assert chunk(vkv, ctx, {}, out=FAKE + 8) == -3
    assert chunk(vkv, ctx, {}, ws=None) == -7 and chunk(vkv, ctx, {}, ws_bytes=100) == -7
    assert chunk(vkv, ctx, {}, ws=FAKE + 16) == -3
    lib = vkv.load()
    assert lib.vkv_chunk_attend(None, None, None, None, 0, 0.1, None, None, None) == -1
    assert lib.vkv_chunk_attend(ctx, None, None, None, 0, 0.1, None, None, None) == -1
    assert lib.vkv_chunk_workspace_size(None, None, None) == -1


def test_chunk_without_work_needs_no_device(vkv, ctx):
    assert chunk(vkv, ctx, dict(n_tok=0)) == 0
    assert chunk(vkv, ctx, dict(max_q=0)) == 0


def test_chunk_workspace_depends_on_the_bounds_alone(vkv):
    lib = vkv.load()

    def size(**kw):
        n = ctypes.c_size_t(0)
        pg = make(vkv._Pages, PAGES, **{k: v for k, v in kw.items() if k in PAGES})
        ch = make(vkv._Chunk, CHUNK, **{k: v for k, v in kw.items() if k in CHUNK})
        assert lib.vkv_chunk_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n)) == 0
        return n.value

    assert size(n_tok=1) == size(n_tok=1000) and size() % 256 == 0
    assert size(max_kv=1 << 20, table_stride=1 << 14, max_q=1, H=128) < 160 << 20
    assert size(B=65535, max_q=64, H=128) == 0        # a workgroup per block of rows: nothing to join


def test_pages_and_chunk_bindings_check_their_tensors(vkv):
    torch = pytest.importorskip("torch")
    bf, i32 = torch.bfloat16, torch.int32
    cache, table, kv = torch.zeros(6, 16, 576, dtype=bf), torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32)
    pg = vkv.Pages(cache, table, kv, 48)
    assert (pg.c.page, pg.c.n_pages, pg.c.page_stride, pg.c.row_stride, pg.c.table_stride) == (16, 6, 9216, 576, 3)
    for bad in (dict(cache=cache.float()), dict(cache=cache[..., :512]), dict(table=table.long()), dict(kv_len=kv[:1]),
                dict(max_kv=49), dict(table=table.t()), dict(kv_len=kv.long())):
        with pytest.raises(ValueError):
            vkv.Pages(**dict(dict(cache=cache, table=table, kv_len=kv, max_kv=48), **bad))
    dense = vkv.Pages.of_cache(torch.zeros(2, 96, 576, dtype=bf), kv, page=32)
    assert (dense.c.n_pages, dense.c.page, dense.max_kv) == (6, 32, 96)
    with pytest.raises(ValueError):
        vkv.Pages.of_cache(torch.zeros(2, 96, 576, dtype=bf), kv, page=64)
    q = torch.zeros(5, 4, 576, dtype=bf)
    cu = torch.tensor([0, 2, 5], dtype=i32)
    ch = vkv.Chunk(q[..., :512], q[..., 512:], cu, 3)
    assert (ch.c.q_lat_stride, ch.c.q_rope_stride, ch.c.n_tok, ch.c.H) == (576, 576, 5, 4)
    for bad in (dict(q_lat=q[..., :500]), dict(q_rope=q[:4, :, 512:]), dict(cu=cu.long()), dict(q_lat=q[..., :512].half()),
                dict(q_lat=torch.zeros(5, 8, 512, dtype=bf)[:, :4])):
        with pytest.raises(ValueError):
            vkv.Chunk(**dict(dict(q_lat=q[..., :512], q_rope=q[..., 512:], cu=cu, max_q=3), **bad))
    with pytest.raises(ValueError):
        vkv.chunk_workspace_size(pg, vkv.Chunk(q[..., :512], q[..., 512:], cu[:2], 3))


def weights(vkv, ctx, change, ws=FAKE, ws_bytes=1 << 40, scale=0.1, decay=0.9, lse=FAKE, prev=FAKE, weight=FAKE, stride=1000):
    pg = make(vkv._Pages, PAGES, **{k: v for k, v in change.items() if k in PAGES})
    ch = make(vkv._Chunk, CHUNK, **{k: v for k, v in change.items() if k in CHUNK})
    return vkv.load().vkv_weight_accumulate(ctx, ctypes.byref(pg), ctypes.byref(ch), lse, ws, ws_bytes, scale, decay, prev,
                                            weight, stride, None)


@pytest.mark.parametrize("change,code", PAGES_BAD + CHUNK_BAD)
def test_weight_refusals(vkv, ctx, change, code):
    assert weights(vkv, ctx, change) == code and vkv.load().vkv_last_error(ctx)
    n = ctypes.c_size_t(0)
    pg = make(vkv._Pages, PAGES, **{k: v for k, v in change.items() if k in PAGES})
    ch = make(vkv._Chunk, CHUNK, **{k: v for k, v in change.items() if k in CHUNK})
    assert vkv.load().vkv_weight_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n)) == code


def test_weight_call_refusals(vkv, ctx):
    assert weights(vkv, ctx, {}, scale=-1.0) == -1
    for decay in (-0.1, float("nan"), float("inf")):
        assert weights(vkv, ctx, {}, decay=decay) == -1
    assert weights(vkv, ctx, {}, lse=None) == -1 and weights(vkv, ctx, {}, weight=None) == -1
    assert weights(vkv, ctx, {}, stride=999) == -2
    many = dict(max_q=64, H=128)      # enough queries for parts, which need the workspace
    assert weights(vkv, ctx, many, ws=None) == -7 and weights(vkv, ctx, many, ws_bytes=64) == -7
    assert weights(vkv, ctx, many, ws=FAKE + 8) == -3
    assert weights(vkv, ctx, dict(max_kv=0), ws=None, ws_bytes=0) == 0
    assert vkv.load().vkv_weight_accumulate(None, None, None, None, None, 0, 0.1, 1.0, None, None, 0, None) == -1


SELECT = dict(weight=FAKE, B=2, max_kv=1000, weight_stride=1000, kv_len=FAKE, keep=100, nsink=4, recent=16, kept=FAKE, count=FAKE)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(max_kv=-1), -2), (dict(max_kv=(1 << 30) + 1, weight_stride=1 << 31), -2),
    (dict(weight_stride=999), -2), (dict(keep=0), -1), (dict(keep=(1 << 30) + 1), -1), (dict(nsink=-1), -1), (dict(recent=-1), -1),
    (dict(nsink=85), -1), (dict(nsink=1 << 62, recent=1 << 62), -1), (dict(weight=None), -1), (dict(kv_len=None), -1),
    (dict(kept=None), -1), (dict(count=None), -1),
])
def test_select_refusals(vkv, ctx, change, code):
    a = dict(SELECT, **change)
    assert vkv.load().vkv_weight_select(ctx, a["weight"], a["B"], a["max_kv"], a["weight_stride"], a["kv_len"], a["keep"],
                                        a["nsink"], a["recent"], a["kept"], a["count"], None) == code
    assert vkv.load().vkv_weight_select(None, None, 1, 1, 1, None, 1, 0, 0, None, None, None) == -1


EVICT = dict(kept=FAKE, count=FAKE, keep=100, origin=FAKE, weight=FAKE, weight_stride=1000, weight_out=FAKE)


@pytest.mark.parametrize("change,code", PAGES_BAD + [
    (dict(kept=None), -1), (dict(count=None), -1), (dict(keep=0), -1), (dict(keep=(1 << 30) + 1), -1), (dict(weight=None), -1),
    (dict(weight_out=None), -1), (dict(weight_stride=999), -2), (dict(B=65535, keep=1 << 30), -2),
])
def test_evict_refusals(vkv, ctx, change, code):
    pg = make(vkv._Pages, PAGES, **{k: v for k, v in change.items() if k in PAGES})
    a = dict(EVICT, **{k: v for k, v in change.items() if k in EVICT})
    assert vkv.load().vkv_cache_evict(ctx, ctypes.byref(pg), a["kept"], a["count"], a["keep"], a["origin"], a["weight"],
                                      a["weight_stride"], a["weight_out"], None) == code
    assert vkv.load().vkv_cache_evict(None, None, None, None, 1, None, None, 0, None, None) == -1


def test_misaligned_words_are_refused(vkv, ctx):
    """Offsets, lengths, statistics and tables that do not lie on a multiple of 4 bytes."""
    odd = FAKE + 2
    assert prompt(vkv, ctx, cu=odd) == -3 and prompt(vkv, ctx, lse=odd) == -3
    assert chunk(vkv, ctx, dict(cu=odd)) == -3 and chunk(vkv, ctx, {}, lse=odd) == -3
    assert chunk(vkv, ctx, dict(table=odd)) == -3 and chunk(vkv, ctx, dict(kv_len=odd)) == -3
    for k in ("lse", "prev", "weight"):
        assert weights(vkv, ctx, {}, **{k: odd}) == -3
    for k in ("weight", "kv_len", "kept", "count"):
        a = dict(SELECT, **{k: odd})
        assert vkv.load().vkv_weight_select(ctx, a["weight"], a["B"], a["max_kv"], a["weight_stride"], a["kv_len"], a["keep"],
                                            a["nsink"], a["recent"], a["kept"], a["count"], None) == -3
    pg = make(vkv._Pages, PAGES)
    for k in ("kept", "count", "origin", "weight", "weight_out"):
        a = dict(EVICT, **{k: odd})
        assert vkv.load().vkv_cache_evict(ctx, ctypes.byref(pg), a["kept"], a["count"], a["keep"], a["origin"], a["weight"],
                                          a["weight_stride"], a["weight_out"], None) == -3
