"""vkv_prompt_attend against plain attention in 64 bits: packed lengths around the tiles of 64 keys and
blocks of 128 rows, grouped heads, strided and broadcast inputs, values that are not finite in keys a
row does not see, tokens behind the last sequence, capture into a graph, another stream."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

from _attention import attention, check

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 1.0 / math.sqrt(192.0)
MLA, WIDE, NARROW = (128, 64, 128), (128, 0, 128), (64, 0, 64)


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def inputs(lens, H, Hk, dims, seed=0, behind=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dn, dr, dv = dims
    n = sum(lens) + behind
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    return dict(q=normal(g, n, H, dn + dr), k=normal(g, n, Hk, dn), v=normal(g, n, Hk, dv), cu=cu,
                max_len=max(lens), k_rope=normal(g, n, dr) if dr else None)


def run(ctx, x, fill=7.0, scale=SCALE, stream=None):
    pr = vkv.Prompt(**x)
    out = torch.full((pr.n_tok, pr.H, pr.dv), fill, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((pr.n_tok, pr.H), fill, device=DEV)
    vkv.prompt_attend(ctx, pr, scale, out, lse, stream)
    return out, lse


def compare(x, out, lse, heads=None, scale=SCALE):
    q, k, v, cu = x["q"].cpu(), x["k"].cpu(), x["v"].cpu(), x["cu"].tolist()
    H, Hk = q.shape[1], k.shape[1]
    for b, (s, e) in enumerate(zip(cu, cu[1:])):
        if e == s:
            continue
        seen = torch.ones(e - s, e - s, dtype=torch.bool).tril()
        for h in heads or range(H):
            kk = k[s:e, h // (H // Hk)]
            if x["k_rope"] is not None:
                kk = torch.cat([kk, x["k_rope"][s:e].cpu()], 1)
            o, l, ot, lt = attention(q[s:e, h], kk, v[s:e, h // (H // Hk)], seen, scale)
            check(f"lse of sequence {b} head {h}", lse[s:e, h], l, lt)
            check(f"out of sequence {b} head {h}", out[s:e, h], o, ot)


@pytest.mark.parametrize("dims", [MLA, WIDE, NARROW])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [31, 32, 33, 63, 64, 65], [127, 128, 129], [0, 5, 0, 300, 0], [513, 7, 190]])
def test_lengths(ctx, dims, lens):
    x = inputs(lens, 4, 2, dims, seed=sum(lens))
    out, lse = run(ctx, x)
    compare(x, out, lse)


@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 1), (6, 2), (8, 8), (16, 4), (40, 8), (128, 1)])
def test_heads(ctx, H, Hk):
    x = inputs([70, 200], H, Hk, MLA if H < 20 else WIDE, seed=H)
    out, lse = run(ctx, x)
    compare(x, out, lse, heads=sorted({0, 1 % H, H // 2, H - 1}))


def test_long_sequence(ctx):
    x = inputs([4001], 8, 2, MLA, seed=5)
    out, lse = run(ctx, x)
    compare(x, out, lse, heads=[0, 7])


def test_steep_scores(ctx):
    """Scores that rise along the sequence by far more than the reference maximum's slack, and ties."""
    x = inputs([400], 2, 1, WIDE, seed=9)
    x["k"] *= torch.linspace(0.1, 12.0, 400, device=DEV)[:, None, None].to(torch.bfloat16)
    x["k"][100:200] = x["k"][100]
    out, lse = run(ctx, x)
    compare(x, out, lse)


def test_strided_and_broadcast_inputs(ctx):
    """q, k and v as slices of one projection's output, odd row pitch; a key head shared by a stride of 0."""
    x = inputs([90, 41], 4, 4, WIDE, seed=3)
    n = 131
    both = torch.zeros(n, 4 * 128 * 3 + 8, dtype=torch.bfloat16, device=DEV)
    for i, name in enumerate(("q", "k", "v")):
        part = both[:, 512 * i + 8:512 * i + 520].view(n, 4, 128)
        part.copy_(x[name])
        x[name] = part
    out, lse = run(ctx, x)
    compare(x, out, lse)
    x["k"], x["v"] = x["k"][:, :1].expand(n, 4, 128), x["v"][:, 2:3].expand(n, 4, 128)
    out, lse = run(ctx, x)
    compare(x, out, lse)


def test_offsets_beyond_32_bits(ctx):
    """Keys and values whose last rows lie more than 2^32 elements behind the first."""
    x = inputs([35], 2, 1, NARROW, seed=4)
    big = torch.empty(34 * (1 << 27) + 64, dtype=torch.bfloat16, device=DEV)
    for name in ("k", "v"):
        part = big.as_strided((35, 1, 64), (1 << 27, 64, 1))
        part.copy_(x[name])
        got = run(ctx, dict(x, **{name: part}))
        compare(x, *got)


@pytest.mark.parametrize("dims", [MLA, NARROW])
def test_what_a_row_does_not_see_does_not_reach_it(ctx, dims):
    """NaN and infinities in keys and values of later tokens, of other sequences and behind the last one."""
    x = inputs([150, 97], 2, 1, dims, seed=6, behind=9)
    clean = [t.clone() for t in run(ctx, x)]
    x["v"][100, 0, 5], x["v"][120, 0, 6], x["v"][130, 0, 7] = math.inf, -math.inf, math.nan
    x["k"][140] = math.nan
    x["v"][247:], x["k"][247:] = math.nan, math.inf
    out, lse = run(ctx, x)
    assert torch.equal(out[:100], clean[0][:100]) and torch.equal(lse[:140], clean[1][:140])
    assert torch.equal(out[150:247], clean[0][150:247]) and torch.equal(lse[150:247], clean[1][150:247])
    assert bool((out[100:140, :, 5] == math.inf).all()) and bool((out[120:140, :, 6] == -math.inf).all())
    assert bool(torch.isnan(out[130:140, :, 7]).all()) and bool(torch.isnan(out[140:150]).all())
    assert bool(torch.isnan(lse[140:150]).all())
    other = [d for d in range(dims[2]) if d not in (5, 6, 7)]
    assert torch.equal(out[100:140, :, other], clean[0][100:140, :, other])
    assert bool((out[247:] == 7.0).all()) and bool((lse[247:] == 7.0).all())


def test_values_near_the_largest(ctx):
    """Values near the type's largest, whose weighted mean is finite."""
    x = inputs([200], 2, 1, WIDE, seed=12)
    x["v"][..., 3] = 3.0e38
    x["v"][50, :, 4] = -3.0e38
    compare(x, *run(ctx, x))


def test_rows_behind_are_left(ctx):
    x = inputs([20, 44], 3, 3, NARROW, behind=30)
    out, lse = run(ctx, x, fill=3.0)
    compare(x, out, lse)
    assert bool((out[64:] == 3.0).all()) and bool((lse[64:] == 3.0).all())
    out, lse = run(ctx, dict(x, max_len=40), fill=3.0)      # the last four tokens of the longer one are cut off
    assert bool((out[60:] == 3.0).all()) and bool((lse[60:] == 3.0).all())
    y = dict(x, cu=torch.tensor([0, 20, 60], dtype=torch.int32, device=DEV))
    compare(y, out, lse)


def test_offsets_out_of_range_are_cut(ctx):
    """Offsets below 0 and above n_tok are taken as the bounds; a descending pair is an empty sequence."""
    x = inputs([50], 2, 2, NARROW, seed=8)
    out, lse = run(ctx, dict(x, cu=torch.tensor([-5, 30, 20, 1 << 30], dtype=torch.int32, device=DEV)))
    y = dict(x, cu=torch.tensor([0, 30], dtype=torch.int32, device=DEV))
    # rows 20..29 belong to the first and the third sequence here, so only the others are compared
    first = run(ctx, y)
    assert torch.equal(out[:20], first[0][:20]) and torch.equal(lse[:20], first[1][:20])
    last = run(ctx, dict(x, cu=torch.tensor([20, 50], dtype=torch.int32, device=DEV)))
    assert torch.equal(out[30:], last[0][30:]) and torch.equal(lse[30:], last[1][30:])


def test_repeats_graph_and_stream(ctx):
    """The same bits again, on another stream, and from a graph replayed on new inputs."""
    x = inputs([300, 77, 1], 8, 2, MLA, seed=11)
    first = run(ctx, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = run(ctx, x)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, there))
    given = run(ctx, x, stream=s)
    torch.cuda.synchronize()
    assert given[0].shape == first[0].shape
    pr = vkv.Prompt(**x)
    out, lse = torch.empty_like(first[0]), torch.empty_like(first[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vkv.prompt_attend(ctx, pr, SCALE, out, lse)
    for rep in range(3):
        y = inputs([300, 77, 1], 8, 2, MLA, seed=20 + rep)
        for name in ("q", "k", "v", "k_rope"):
            x[name].copy_(y[name])
        out.zero_(), lse.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = run(ctx, y)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), rep
