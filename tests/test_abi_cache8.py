"""Host-side checks of the rotary, 8-bit cache and page entry points (no GPU needed): what they refuse, with which status,
before they touch the device, what needs no device, and the frequencies, which are computed on the host."""
import ctypes
import math
import types

import pytest
import torch

import paper_2609_03949_amd as vkv

FAKE = 1 << 20          # aligned non-null host value; never dereferenced
BF, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


@pytest.fixture()
def ctx():
    """Zeroed memory in a context's place: a refused call only writes its error text there."""
    vkv.load()
    return ctypes.create_string_buffer(1 << 14)


def make(cls, defaults, **kw):
    s = cls()
    for k, v in {**defaults, **kw}.items():
        setattr(s, k, v)
    return s


def picked(base, change):
    return {k: v for k, v in change.items() if k in base}


# ------------------------------------------------------------------ rotary positions

ROPE = dict(dims=64, interleaved=0, scaling=0, base=1e4, factor=4.0, original=4096.0, fast=32.0, slow=1.0, magnitude=1.0)
CALL = dict(x=FAKE, n_tok=5, H=4, width=192, first=128, xts=4 * 192, xhs=192, pos=FAKE, back=0, out=2 * FAKE, ots=4 * 192, ohs=192)
INF, NAN = math.inf, math.nan
ROPE_BAD = [
    (dict(dims=0), -2), (dict(dims=63), -2), (dict(dims=258), -2), (dict(dims=-2), -2), (dict(scaling=-1), -1), (dict(scaling=4), -1),
    (dict(base=1.0), -1), (dict(base=NAN), -1), (dict(base=INF), -1), (dict(magnitude=0.0), -1), (dict(magnitude=NAN), -1),
    (dict(magnitude=1e39), -1), (dict(scaling=1, factor=0.0), -1), (dict(scaling=1, factor=-2.0), -1), (dict(scaling=2, factor=NAN), -1),
    (dict(scaling=3, factor=INF), -1), (dict(scaling=2, dims=2, first=0), -2), (dict(scaling=3, original=0.5), -1),
    (dict(scaling=3, original=NAN), -1), (dict(scaling=3, slow=-1.0), -1), (dict(scaling=3, fast=1.0), -1), (dict(scaling=3, fast=INF), -1),
    (dict(scaling=2, base=1e-300 + 2, factor=1e-300), -1),
]


def rope(ctx, **change):
    r, c = make(vkv._Rope, ROPE, **picked(ROPE, change)), {**CALL, **picked(CALL, change)}
    return vkv.load().vkv_rope_apply(ctx, ctypes.byref(r), c["x"], c["n_tok"], c["H"], c["width"], c["first"], c["xts"], c["xhs"],
                                     c["pos"], c["back"], c["out"], c["ots"], c["ohs"], None)


@pytest.mark.parametrize("change,code", ROPE_BAD + [
    (dict(H=0), -2), (dict(H=65536), -2), (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(n_tok=1 << 29), -2),
    (dict(width=1), -2), (dict(width=1 << 17), -2), (dict(first=-1), -2), (dict(first=129), -2), (dict(first=1 << 40), -2),
    (dict(x=None), -1), (dict(pos=None), -1), (dict(out=None), -1), (dict(x=FAKE + 1), -3), (dict(out=FAKE + 1), -3), (dict(pos=FAKE + 2), -3),
    (dict(xts=-8), -3), (dict(xhs=-1), -3), (dict(ots=-8), -3), (dict(ohs=-8), -3),
    (dict(ohs=191), -2), (dict(ots=0), -2), (dict(ots=700), -2), (dict(ohs=0), -2), (dict(ots=192, ohs=192), -2),
    (dict(out=FAKE, xts=0), -1), (dict(out=FAKE, xhs=0), -1),
])
def test_rope_refusals(ctx, change, code):
    assert rope(ctx, **change) == code
    assert vkv.load().vkv_last_error(ctx)


def test_rope_without_work_needs_no_device(ctx):
    assert rope(ctx, n_tok=0, x=None, pos=None, out=None) == 0
    assert vkv.load().vkv_rope_apply(None, None, None, 0, 1, 2, 0, 0, 0, None, 0, None, 0, 0, None) == -1
    assert vkv.load().vkv_rope_apply(ctx, None, None, 0, 1, 2, 0, 0, 0, None, 0, None, 0, 0, None) == -1


@pytest.mark.parametrize("change,code", ROPE_BAD)
def test_frequency_refusals(change, code):
    f = (ctypes.c_double * 128)(*[7.0] * 128)
    r = make(vkv._Rope, ROPE, **picked(ROPE, change))
    assert vkv.load().vkv_rope_frequencies(ctypes.byref(r), f) == code
    assert all(v == 7.0 for v in f) and vkv.load().vkv_last_error(None)
    assert vkv.load().vkv_rope_frequencies(ctypes.byref(make(vkv._Rope, ROPE)), None) == -1
    assert vkv.load().vkv_rope_frequencies(None, f) == -1


def test_frequencies():
    """Each term within a few roundings of fp64 (pow, a division, two products)."""
    close = lambda a, b: all(abs(x - y) <= 16 * 2.0 ** -53 * abs(y) for x, y in zip(a, b, strict=True))
    plain = [1e4 ** (-2 * i / 64) for i in range(32)]
    assert close(vkv.Rope(64).frequencies(), plain)
    assert close(vkv.Rope(64, scaling=vkv.VKV_ROPE_LINEAR, factor=8.0).frequencies(), [f / 8 for f in plain])
    base = 1e4 * 4.0 ** (64 / 62)
    assert close(vkv.Rope(64, scaling=vkv.VKV_ROPE_BASE, factor=4.0).frequencies(), [base ** (-2 * i / 64) for i in range(32)])
    parts = vkv.Rope(64, scaling=vkv.VKV_ROPE_PARTS, factor=40.0, original=4096, fast=32, slow=1).frequencies()
    turns = [4096 * f / (2 * math.pi) for f in plain]
    g = [min(max((n - 1) / 31, 0.0), 1.0) for n in turns]
    want = [f * ((1 - k) / 40 + k) for f, k in zip(plain, g)]
    assert all(abs(a - b) <= 64 * 2.0 ** -53 * abs(f) for a, b, f in zip(parts, want, plain))
    assert parts[0] == plain[0] and abs(parts[-1] - plain[-1] / 40) <= 16 * 2.0 ** -53 * parts[-1]
    with pytest.raises(vkv.VkvError):
        vkv.Rope(63)


# ------------------------------------------------------------------ the cache held in 8 bits

PAGES8 = dict(B=3, max_kv=1000, n_pages=64, page=64, block=16, cache=FAKE, row_stride=640, page_stride=64 * 640, scale=FAKE,
              scale_stride=4, table=FAKE, table_stride=16, kv_len=FAKE)
CHUNK = dict(n_tok=7, H=16, max_q=4, q_lat=FAKE, q_lat_stride=512, q_rope=FAKE, q_rope_stride=64, cu=FAKE)
PAGES8_BAD = [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(max_kv=-1), -2), (dict(max_kv=(1 << 30) + 1), -2), (dict(n_pages=0), -2),
    (dict(n_pages=1 << 31), -2), (dict(page=0), -4), (dict(page=48), -4), (dict(page=1 << 17), -4), (dict(block=0), -4),
    (dict(block=3), -4), (dict(block=128), -4), (dict(page=16, block=32, table_stride=63), -4), (dict(block=-16), -4),
    (dict(cache=None), -1), (dict(scale=None), -1), (dict(table=None), -1), (dict(kv_len=None), -1), (dict(cache=FAKE + 8), -3),
    (dict(table=FAKE + 2), -3), (dict(kv_len=FAKE + 1), -3), (dict(row_stride=624), -3), (dict(row_stride=648), -3),
    (dict(page_stride=-16), -3), (dict(page_stride=8), -3), (dict(row_stride=1 << 36), -2), (dict(page_stride=1 << 36), -2),
    (dict(scale_stride=3), -2), (dict(scale_stride=1 << 31), -2), (dict(table_stride=15), -2),
]
CHUNK_BAD = [
    (dict(H=0), -2), (dict(H=129), -2), (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(max_q=-1), -2),
    (dict(max_q=1 << 27), -2), (dict(q_lat=None), -1), (dict(q_rope=None), -1), (dict(cu=None), -1), (dict(q_lat=FAKE + 8), -3),
    (dict(q_rope=FAKE + 2), -3), (dict(q_lat_stride=-8), -3), (dict(q_lat_stride=513), -3), (dict(q_rope_stride=68), -3),
]
WRITE = dict(lat=FAKE, lat_stride=512, rope=FAKE, rope_stride=64, cu=FAKE, n_tok=7, max_q=4)


def chunk8(ctx, change, ws=FAKE, ws_bytes=None, scale=0.1, out=FAKE, lse=FAKE):
    lib = vkv.load()
    pg, ch = make(vkv._Pages8, PAGES8, **picked(PAGES8, change)), make(vkv._Chunk, CHUNK, **picked(CHUNK, change))
    n = ctypes.c_size_t(0)
    if ws_bytes is None:
        rc = lib.vkv_chunk8_workspace_size(ctypes.byref(pg), ctypes.byref(ch), ctypes.byref(n))
        if rc:
            return rc
        ws_bytes = n.value
    return lib.vkv_chunk8_attend(ctx, ctypes.byref(pg), ctypes.byref(ch), ws, ws_bytes, scale, out, lse, None)


def write(ctx, **change):
    pg, w = make(vkv._Pages8, PAGES8, **picked(PAGES8, change)), {**WRITE, **picked(WRITE, change)}
    return vkv.load().vkv_cache8_write(ctx, ctypes.byref(pg), w["lat"], w["lat_stride"], w["rope"], w["rope_stride"], w["cu"],
                                       w["n_tok"], w["max_q"], None)


@pytest.mark.parametrize("change,code", PAGES8_BAD + CHUNK_BAD)
def test_chunk8_refusals(ctx, change, code):
    assert chunk8(ctx, change) == code and vkv.load().vkv_last_error(None)
    assert chunk8(ctx, change, ws_bytes=1 << 40) == code and vkv.load().vkv_last_error(ctx)


def test_chunk8_call_refusals(ctx):
    for kw, code in ((dict(scale=0.0), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(out=None), -1),
                     (dict(lse=None), -1), (dict(out=FAKE + 8), -3), (dict(lse=FAKE + 2), -3), (dict(ws=None), -7),
                     (dict(ws=FAKE + 128), -3), (dict(ws_bytes=100), -7)):
        assert chunk8(ctx, {}, **kw) == code, kw
    lib = vkv.load()
    pg, ch = make(vkv._Pages8, PAGES8), make(vkv._Chunk, CHUNK)
    n = ctypes.c_size_t(0)
    assert lib.vkv_chunk8_workspace_size(ctypes.byref(pg), ctypes.byref(ch), None) == -1
    assert lib.vkv_chunk8_workspace_size(None, ctypes.byref(ch), ctypes.byref(n)) == -1
    assert lib.vkv_chunk8_workspace_size(ctypes.byref(pg), None, ctypes.byref(n)) == -1
    assert lib.vkv_chunk8_attend(None, ctypes.byref(pg), ctypes.byref(ch), FAKE, 1 << 40, 0.1, FAKE, FAKE, None) == -1
    # parts of at most 256 runs, two each, of the units' rows; none where units or tiles are too many to be counted
    def size(B, max_kv, H, max_q):
        a = make(vkv._Pages8, PAGES8, B=B, max_kv=max_kv, table_stride=1 << 24)
        assert lib.vkv_chunk8_workspace_size(ctypes.byref(a), ctypes.byref(make(vkv._Chunk, CHUNK, H=H, max_q=max_q)), ctypes.byref(n)) == 0
        return n.value
    for args, rows, runs in (((3, 1000, 16, 1), 16, 48), ((1, 1 << 20, 16, 1), 16, 256), ((4, 8192, 32, 1), 32, 256),
                             ((4, 32768, 128, 1), 64, 256), ((32, 32768, 128, 1), 128, 256)):
        assert 0 <= size(*args) - 2 * runs * rows * (512 + 2) * 4 < 20000, args
    assert size(1100, 1000, 16, 1) == 0 and size(100, 1 << 30, 64, 1) == 0 and size(0xFFFF, 1 << 30, 128, 1) == 0
    # nothing to attend from: no device needed
    assert chunk8(ctx, dict(n_tok=0, q_lat=None, q_rope=None), out=None, lse=None) == 0
    assert chunk8(ctx, dict(max_q=0)) == 0


@pytest.mark.parametrize("change,code", PAGES8_BAD + [
    (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(max_q=-1), -2), (dict(max_q=(1 << 30) + 1), -2), (dict(lat=None), -1),
    (dict(rope=None), -1), (dict(cu=None), -1), (dict(lat=FAKE + 8), -3), (dict(rope=FAKE + 2), -3), (dict(cu=FAKE + 2), -3),
    (dict(page_stride=0), -2), (dict(page_stride=63 * 640), -2), (dict(page_stride=640), -2), (dict(page_stride=640, row_stride=63 * 640), -2),
    (dict(page=1, block=1, table_stride=1000, page_stride=624), -2),
    (dict(lat_stride=-8), -3), (dict(lat_stride=513), -3), (dict(rope_stride=68), -3),
    (dict(B=65535, max_kv=1 << 30, table_stride=1 << 24, n_tok=(1 << 31) - 1, max_q=1 << 30), -2),
])
def test_write_refusals(ctx, change, code):
    assert write(ctx, **change) == code
    assert vkv.load().vkv_last_error(ctx)


def test_write_without_work_needs_no_device(ctx):
    assert write(ctx, n_tok=0, lat=None, rope=None) == 0
    assert write(ctx, max_q=0) == 0
    assert write(ctx, max_kv=0, table=None) == 0
    assert vkv.load().vkv_cache8_write(None, None, None, 0, None, 0, None, 0, 0, None) == -1
    assert vkv.load().vkv_cache8_write(ctx, None, None, 0, None, 0, None, 0, 0, None) == -1


# ------------------------------------------------------------------ the pages' life

POOL = dict(B=3, n_pages=64, width=16, page=64, n_planes=2, table=FAKE, table_stride=16, kv_len=FAKE, refs=FAKE)
PLANE = dict(base=FAKE, bytes=1000, page_stride=1024, layers=3, layer_stride=1 << 16)


def pool(change):
    s = make(vkv._Pool, POOL, **picked(POOL, change))
    for k in range(2):
        for name, v in {**PLANE, **(picked(PLANE, change) if k == 1 else {})}.items():
            setattr(s.plane[k], name, v)
    return s


POOL_BAD = [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(n_pages=0), -2), (dict(n_pages=1 << 31), -2), (dict(page=0), -4), (dict(page=24), -4),
    (dict(page=1 << 17), -4), (dict(width=0), -2), (dict(width=(1 << 24) + 1, table_stride=1 << 25), -2), (dict(table_stride=15), -2),
    (dict(table=None), -1), (dict(kv_len=None), -1), (dict(refs=None), -1), (dict(table=FAKE + 2), -3), (dict(kv_len=FAKE + 1), -3),
    (dict(refs=FAKE + 2), -3), (dict(n_planes=-1), -1), (dict(n_planes=5), -1),
    (dict(base=None), -1), (dict(bytes=0), -2), (dict(bytes=1 << 31), -2), (dict(layers=0), -2), (dict(layers=65536), -2),
    (dict(page_stride=999), -2), (dict(page_stride=-1024), -2), (dict(page_stride=1 << 31), -2), (dict(layer_stride=-1), -2),
    (dict(layer_stride=0), -2), (dict(layer_stride=1000), -2), (dict(layer_stride=63 * 1024 + 999), -2),
]


@pytest.mark.parametrize("change,code", POOL_BAD)
def test_pool_refusals(ctx, change, code):
    lib, s, n = vkv.load(), pool(change), ctypes.c_size_t(77)
    assert lib.vkv_pool_workspace_size(ctypes.byref(s), ctypes.byref(n)) == code and n.value == 77
    assert lib.vkv_pages_fork(ctx, ctypes.byref(s), FAKE, FAKE, 1 << 40, None) == code
    assert lib.vkv_pages_reserve(ctx, ctypes.byref(s), FAKE, FAKE, FAKE, 1 << 40, None) == code
    assert lib.vkv_pages_compact(ctx, ctypes.byref(s), FAKE, FAKE, 1 << 40, None) == code
    assert lib.vkv_last_error(ctx)


def test_pool_layouts_that_do_not_overlap():
    lib, n = vkv.load(), ctypes.c_size_t(0)
    for change in (dict(layer_stride=63 * 1024 + 1000), dict(layer_stride=1000, page_stride=4096),
                   dict(n_pages=1, page_stride=1000, layer_stride=1000), dict(layers=1, layer_stride=-5), dict(n_planes=0)):
        s = pool(change)
        assert lib.vkv_pool_workspace_size(ctypes.byref(s), ctypes.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0


def test_pool_call_refusals(ctx):
    lib, s, n = vkv.load(), pool({}), ctypes.c_size_t(0)
    assert lib.vkv_pool_workspace_size(ctypes.byref(s), ctypes.byref(n)) == 0
    b = ctypes.byref(s)
    for p, code in ((None, -1), (FAKE + 2, -3)):
        assert lib.vkv_pages_fork(ctx, b, p, FAKE, n.value, None) == code
        assert lib.vkv_pages_reserve(ctx, b, p, FAKE, FAKE, n.value, None) == code
        assert lib.vkv_pages_reserve(ctx, b, FAKE, p, FAKE, n.value, None) == code
        assert lib.vkv_pages_compact(ctx, b, p, FAKE, n.value, None) == code
    for ws, size, code in ((None, n.value, -7), (FAKE, n.value - 1, -7), (FAKE + 64, n.value, -3)):
        assert lib.vkv_pages_fork(ctx, b, FAKE, ws, size, None) == code
        assert lib.vkv_pages_reserve(ctx, b, FAKE, FAKE, ws, size, None) == code
        assert lib.vkv_pages_compact(ctx, b, FAKE, ws, size, None) == code
    assert lib.vkv_pages_fork(None, b, FAKE, FAKE, n.value, None) == -1
    assert lib.vkv_pages_compact(ctx, None, FAKE, FAKE, n.value, None) == -1
    assert lib.vkv_pool_workspace_size(b, None) == -1


# ------------------------------------------------------------------ the binding

def test_binding_checks_its_tensors():
    z = lambda *s, t=U8: torch.zeros(*s, dtype=t)
    cache, scale, table, kv = z(5, 16, 640), z(5, 4), z(2, 3, t=I32), z(2, t=I32)
    p = vkv.Pages8(cache, scale, table, kv, 48)
    assert (p.c.page, p.c.block, p.c.n_pages, p.c.row_stride, p.c.page_stride, p.c.scale_stride) == (16, 4, 5, 640, 10240, 4)
    good = dict(cache=cache, scale=scale, table=table, kv_len=kv, max_kv=48)
    for bad in (dict(cache=cache.view(torch.int8)), dict(cache=cache[..., :639]), dict(scale=z(4, 4)), dict(scale=z(5, 3)), dict(scale=z(5, 0)),
                dict(scale=z(5, 4, t=I32)), dict(table=table.long()), dict(kv_len=z(3, t=I32)), dict(max_kv=49),
                dict(table=z(1, 3, t=I32).expand(2, 3))):
        with pytest.raises(ValueError):
            vkv.Pages8(**{**good, **bad})
    refs, plane = z(6, t=I32), z(2, 6, 16, 640)
    s = vkv.Pool(table, kv, refs, 16, [plane, z(1, 6, 4)]).c
    assert (s.n_planes, s.plane[0].bytes, s.plane[0].page_stride, s.plane[0].layers, s.plane[0].layer_stride) == (2, 10240, 10240, 2, 61440)
    assert (s.plane[1].bytes, s.plane[1].layers, s.width, s.n_pages) == (4, 1, 3, 6)
    for bad in ([plane[:, :5]], [plane[0]], [plane.transpose(2, 3)], [plane] * 5, [plane[:0]]):
        with pytest.raises(ValueError):
            vkv.Pool(table, kv, refs, 16, bad)
    for bad in (dict(table=table.long()), dict(kv_len=z(3, t=I32)), dict(refs=refs.long())):
        with pytest.raises(ValueError):
            a = {**dict(table=table, kv_len=kv, refs=refs), **bad}
            vkv.Pool(a["table"], a["kv_len"], a["refs"], 16, [plane])


class Refused:
    """In libvkv's place: every call has been one too many."""

    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


def test_host_tensors_and_wrong_shapes_are_refused():
    c = types.SimpleNamespace(device=0, lib=Refused(), handle=None, check=lambda rc: None)
    z = lambda *s, t=BF: torch.zeros(*s, dtype=t)
    pages = vkv.Pages8(z(5, 16, 640, t=U8), z(5, 4, t=U8), z(2, 3, t=I32), z(2, t=I32), 48)
    chunk = vkv.Chunk(z(4, 3, 512), z(4, 3, 64), z(3, t=I32), 2)
    pool_ = vkv.Pool(z(2, 3, t=I32), z(2, t=I32), z(6, t=I32), 16, [z(1, 6, 4)])
    ws, x, pos, cu = z(1 << 12, t=U8), z(4, 3, 64), z(4, t=I32), z(3, t=I32)
    lat, rp, o, l, one, two = z(4, 512), z(4, 64), z(4, 3, 512), z(4, 3, t=torch.float32), z(1, t=I32), z(2, t=I32)
    r = vkv.Rope(64)
    for call in (lambda: vkv.rope_apply(c, r, x, pos, x), lambda: vkv.cache8_write(c, pages, lat, rp, cu, 2),
                 lambda: vkv.chunk8_attend(c, pages, chunk, ws, 0.1, o, l), lambda: vkv.pages_fork(c, pool_, two, ws),
                 lambda: vkv.pages_reserve(c, pool_, two, two, ws), lambda: vkv.pages_compact(c, pool_, one, ws)):
        with pytest.raises(ValueError, match="device"):
            call()
    for call in (lambda: vkv.rope_apply(c, r, x, pos[:3], x), lambda: vkv.rope_apply(c, r, x, pos, x[:, :2]),
                 lambda: vkv.rope_apply(c, r, x.float(), pos, x), lambda: vkv.rope_apply(c, r, x, pos.long(), x),
                 lambda: vkv.rope_apply(c, r, x[None], pos, x[None]), lambda: vkv.cache8_write(c, pages, lat[:, :511], rp, cu, 2),
                 lambda: vkv.cache8_write(c, pages, lat, rp[:3], cu, 2), lambda: vkv.cache8_write(c, pages, lat, rp, cu[:2], 2),
                 lambda: vkv.chunk8_attend(c, pages, chunk, ws, 0.1, o[:3], l), lambda: vkv.pages_fork(c, pool_, one, ws),
                 lambda: vkv.pages_reserve(c, pool_, two, one, ws), lambda: vkv.pages_compact(c, pool_, two, ws)):
        with pytest.raises(ValueError):
            call()
