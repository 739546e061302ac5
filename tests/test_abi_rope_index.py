"""Frequencies extended by parts with a ramp over the pair's index, against the formula (no GPU needed), and what is refused."""
import ctypes
import math

import pytest

import paper_2609_03949_amd as vkv

BY_INDEX = vkv.VKV_ROPE_PARTS | vkv.VKV_ROPE_BY_INDEX


def by_index(dims, base, factor, original, fast, slow):
    x = lambda n: dims * math.log(original / (n * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(x(fast)), 0), min(math.ceil(x(slow)), dims - 1)
    out = []
    for i in range(dims // 2):
        part = 0.0 if i <= lo else 1.0 if i >= hi else (i - lo) / (hi - lo)
        theta = base ** (-2 * i / dims)
        out.append(theta / factor * part + theta * (1 - part))
    return out


@pytest.mark.parametrize("args", [(64, 1e4, 40.0, 4096.0, 32.0, 1.0), (64, 1e4, 32.0, 4096.0, 32.0, 1.0), (128, 5e5, 8.0, 8192.0, 4.0, 1.0),
                                  (64, 1e4, 16.0, 2048.0, 32.0, 0.5), (64, 1e4, 40.0, 100.0, 32.0, 1.0), (32, 1e6, 2.5, 1e6, 8.0, 1e-3),
                                  (64, 1e4, 4.0, 1e6, 40.0, 39.9),
                                  (64, 1e4, 40.0, 1e9, 32.0, 1.0)])
def test_frequencies_by_index(args):
    """Each term within a few roundings of fp64 of what it is made of."""
    dims, base, factor, original, fast, slow = args
    got = vkv.Rope(dims, base, scaling=BY_INDEX, factor=factor, original=original, fast=fast, slow=slow).frequencies()
    want = by_index(*args)
    assert len(got) == dims // 2
    assert all(abs(a - b) <= 64 * 2.0 ** -53 * base ** (-2 * i / dims) for i, (a, b) in enumerate(zip(got, want)))


def test_the_two_ramps():
    """64 dims, base 10^4, 4096 positions times 40: equal outside pairs 11 to 22, up to 4.3 times apart between."""
    kw = dict(base=1e4, factor=40.0, original=4096.0, fast=32.0, slow=1.0)
    turns, index = (vkv.Rope(64, scaling=s, **kw).frequencies() for s in (vkv.VKV_ROPE_PARTS, BY_INDEX))
    plain = vkv.Rope(64).frequencies()
    assert turns[:11] == index[:11] == plain[:11]
    assert turns[23:] == index[23:] and all(abs(a - p / 40) <= 16 * 2.0 ** -53 * a for a, p in zip(index[23:], plain[23:]))
    assert abs(index[16] - 0.01 * (6 / 13 / 40 + 7 / 13)) <= 1e-17 and abs(turns[16] - 0.00199) < 1e-5
    assert abs(index[20] - 7.9e-4) < 2e-6 and 4.2 < max(b / a for a, b in zip(turns, index)) < 4.4


@pytest.mark.parametrize("change", [dict(scaling=8), dict(scaling=9), dict(scaling=10), dict(scaling=12), dict(scaling=11 + 16), dict(slow=0.0),
                                    dict(fast=1.0), dict(original=math.inf), dict(factor=0.0), dict(original=0.5),
                                    dict(original=1e12), dict(original=2.0, slow=31.0)])
def test_refused(change):
    r = vkv._Rope()
    for k, v in {**dict(dims=64, scaling=BY_INDEX, base=1e4, factor=40.0, original=4096.0, fast=32.0, slow=1.0, magnitude=1.0), **change}.items():
        setattr(r, k, v)
    f = (ctypes.c_double * 32)(*[7.0] * 32)
    assert vkv.load().vkv_rope_frequencies(ctypes.byref(r), f) == -1
    assert all(v == 7.0 for v in f) and vkv.load().vkv_last_error(None)
