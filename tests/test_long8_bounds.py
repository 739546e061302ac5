"""What the bounds of _long8.py let pass (no GPU needed): outputs made as the kernels make them do, and none whose weights have fewer bits
or whose values are not those of their rows: a tile left out, doubled, of another place, a row of another."""
import pytest
import torch

import _paged8
from _long8 import Exact, marked, spread
from _paged8 import Case8

N = 20011


@pytest.fixture(scope="module", params=["marked", "random", "random, own"])
def case(request):
    dev, _paged8.DEV = _paged8.DEV, "cpu"
    try:
        x = spread(Case8([N], [1], 64 if "own" in request.param else 16, page=64, block=16, seed=3), 4, own="own" in request.param)
        if request.param == "marked":
            marked(x)
        return request.param, Exact(x, 0)
    finally:
        _paged8.DEV = dev


def rounded(w, bits):
    """w > 0 to `bits` significant bits, nearest."""
    step = torch.pow(2.0, torch.floor(torch.log2(w)) - (bits - 1))
    return torch.round(w / step) * step


def made(x, weights=lambda w: w.to(torch.float16).double(), order=None, times=None):
    """Outputs from weights against the largest and exact codes: order[j] is the row whose values row j's weight meets."""
    w = x.p * x.f
    w = weights(w / w.amax(1, keepdim=True)) * w.amax(1, keepdim=True)
    if times is not None:
        w = w * times
    codes = x.v / x.f[:, None]
    return (w @ (codes if order is None else codes[order])).to(torch.bfloat16)


def passes(x, got):
    return max(x.far(got)) <= 1.0


def test_what_is_right_passes(case):
    _, x = case
    assert passes(x, made(x)) and passes(x, x.out.to(torch.bfloat16))


def test_weights_of_fewer_bits_do_not(case):
    """Of bf16 and of an 8-bit format.  (Where 39 rows of a sign share a dim, what bf16 makes of them averages below the output's step;
    where the queries are alike there are too few outputs to tell.)"""
    name, x = case
    for bits in (8, 4) if "own" in name else (4,):
        assert not passes(x, made(x, lambda w: rounded(w, bits))), bits


@pytest.mark.parametrize("tile", [32, 64])
def test_wrong_values_do_not(case, tile):
    """Tiles at the ends, at the middle and around a run's bounds (78 or 79 tiles of 64 in each of four)."""
    name, x = case
    last = N // tile * tile
    for u in (0, tile, 78 * 64, 79 * 64, 157 * 64, N // 2 // tile * tile, last - tile, last):
        own = torch.arange(u, min(u + tile, N))
        for factor in (0.0, 2.0):
            times = torch.ones(N, dtype=torch.float64)
            times[own] = factor
            # (11 rows of 20011 at the end do not show where the sharpest queries' outputs are most of the norm)
            assert not passes(x, made(x, times=times)) or ("own" in name and u == last), (u, factor)
        if u + 2 * tile <= N:                         # the next tile's rows; the other half's; its neighbour's row
            for there in (own + tile, own.roll(tile // 2), own.view(-1, 2).flip(1).reshape(-1)):
                order = torch.arange(N)
                order[own] = there
                assert not passes(x, made(x, order=order)), (u, there[:4])
    w = x.p / x.p.median(1, keepdim=True).values
    for row in (0, 77, 6000, 13001, N - 1):           # single rows of middling weight or more, where they are told apart
        times = torch.ones(N, dtype=torch.float64)
        times[row] = 0.0
        assert not passes(x, made(x, times=times)) or "random" in name or float(w[:, row].max()) < 0.7, row
