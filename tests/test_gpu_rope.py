"""vkv_rope_apply against the formula in 64 bits.

For a pair (a, b), with c, s cosine and sine: the angle's fp64 product p f is off by 2^-53 |p f| relative to the definition's, and its
reduction and the frequency by a few of the same; sine and cosine in fp32 (argument rounded: 2 pi 2^-25 at most; the function a few
2^-24) times the magnitude: 8 2^-24 + 2^-50 |p f| m in all; two products and one sum in fp32: 3 2^-24; then half a step of bf16."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.finfo(torch.bfloat16).eps / 2, torch.finfo(torch.float32).eps / 2


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


def frequencies(dims, base, scaling, factor, original, fast, slow):
    out = []
    for i in range(dims // 2):
        if scaling == vkv.VKV_ROPE_BASE:
            f = (base * factor ** (dims / (dims - 2))) ** (-2 * i / dims)
        else:
            f = base ** (-2 * i / dims)
        if scaling == vkv.VKV_ROPE_LINEAR:
            f /= factor
        if scaling == vkv.VKV_ROPE_PARTS:
            turns = original * f / (2 * math.pi)
            g = 0.0 if turns <= slow else 1.0 if turns >= fast else (turns - slow) / (fast - slow)
            f = f * (1 - g) / factor + f * g
        out.append(f)
    return out


def turned(x, pos, freq, first, inter, magnitude, back):
    """The result in fp64 and the bound on its error, on the CPU."""
    out = x.double().cpu()
    tol = torch.zeros_like(out)
    dims = 2 * len(freq)
    t = pos.double().cpu()[:, None] * torch.tensor(freq, dtype=torch.float64)[None, :]
    c, s = magnitude * torch.cos(t), magnitude * torch.sin(t)
    if back:
        s = -s
    c, s, far = c[:, None], s[:, None], (magnitude * t.abs())[:, None]
    one = torch.arange(first, first + dims, 2) if inter else torch.arange(first, first + dims // 2)
    two = one + 1 if inter else one + dims // 2
    a, b = out[..., one].clone(), out[..., two].clone()
    out[..., one], out[..., two] = a * c - b * s, b * c + a * s
    size = a.abs() + b.abs()
    err = size * (magnitude * (8 + 3) * F32 + 2.0 ** -50 * far) + 1e-36
    for d in (one, two):
        tol[..., d] = (BF * out[..., d].abs() + (1 + BF) * err)
    return out, tol


def check(ctx, rope, args, x, pos, first=0, back=False, out=None, inter=False, magnitude=1.0, **kw):
    want, tol = turned(x, pos, frequencies(*args), first, inter, magnitude, back)
    out = torch.full_like(x, 9.0) if out is None else out
    vkv.rope_apply(ctx, rope, x, pos, out, first=first, transposed=back, **kw)
    torch.cuda.synchronize()
    d = (out.double().cpu() - want).abs()
    assert bool((d <= tol).all()), f"{float((d / tol.clamp(min=1e-300)).max()):.3g} of the bound"
    return out


def data(n, H, D, top, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(n, H, D, generator=g, device=DEV).to(torch.bfloat16)
    return x, torch.randint(0, top, (n,), generator=g, device=DEV, dtype=torch.int32)


MODES = [(vkv.VKV_ROPE_PLAIN, 1.0), (vkv.VKV_ROPE_LINEAR, 8.0), (vkv.VKV_ROPE_BASE, 4.0), (vkv.VKV_ROPE_PARTS, 32.0)]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("scaling,factor", MODES)
@pytest.mark.parametrize("back", [False, True])
def test_modes(ctx, inter, scaling, factor, back):
    m = 1.0 if scaling != vkv.VKV_ROPE_PARTS else 1.3
    rope = vkv.Rope(64, 10000.0, inter, scaling, factor, 4096, 32.0, 1.0, m)
    x, pos = data(37, 5, 192, 1 << 20, scaling)
    pos[:4] = torch.tensor([0, 1, -5, 2 ** 31 - 1], dtype=torch.int32)
    check(ctx, rope, (64, 10000.0, scaling, factor, 4096, 32.0, 1.0), x, pos, 128, back, inter=inter, magnitude=m)


@pytest.mark.parametrize("n,H,D,first,dims", [
    (1, 1, 2, 0, 2), (1, 1, 64, 0, 64), (1, 128, 64, 0, 64), (3, 128, 576, 512, 64), (5, 1, 64, 0, 64), (2, 3, 30, 1, 26),
    (7, 2, 256, 0, 256), (1500, 2, 128, 0, 128), (9, 4, 100, 4, 48), (4, 33, 96, 16, 16), (2, 2, 24, 8, 8), (1, 300, 18, 2, 16)])
@pytest.mark.parametrize("inter", [False, True])
def test_sizes(ctx, n, H, D, first, dims, inter):
    x, pos = data(n, H, D, 5000, n + D)
    check(ctx, vkv.Rope(dims, 5e5, inter), (dims, 5e5, 0, 1.0, 0, 0, 0), x, pos, first, inter=inter)


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_leaves_the_other_dims(ctx, inter):
    x, pos = data(20, 6, 576, 9000, 3)
    before = x.clone()
    rope = vkv.Rope(64, 10000.0, inter)
    want, tol = turned(x, pos, frequencies(64, 10000.0, 0, 1.0, 0, 0, 0), 512, inter, 1.0, False)
    part = x[..., 512:]                                 # rows of 64 at a stride of 576, in place
    vkv.rope_apply(ctx, rope, part, pos, part)
    torch.cuda.synchronize()
    assert torch.equal(x[..., :512], before[..., :512])
    assert bool(((x.double().cpu() - want).abs() <= tol).all())
    x.copy_(before)
    vkv.rope_apply(ctx, rope, x, pos, x, first=512)
    torch.cuda.synchronize()
    assert torch.equal(x[..., :512], before[..., :512]) and bool(((x.double().cpu() - want).abs() <= tol).all())


def test_strides_and_broadcast_rows(ctx):
    x, pos = data(6, 4, 64, 900, 4)
    rope, args = vkv.Rope(64), (64, 10000.0, 0, 1.0, 0, 0, 0)
    out = torch.zeros(4, 6, 80, dtype=torch.bfloat16, device=DEV)
    check(ctx, rope, args, x, pos, out=out.transpose(0, 1)[..., 8:72])     # heads first, rows apart
    assert bool((out[..., :8] == 0).all()) and bool((out[..., 72:] == 0).all())
    check(ctx, rope, args, x[:, :1].expand(6, 4, 64), pos)
    check(ctx, rope, args, x[:1].expand(6, 4, 64), pos)
    odd = torch.zeros(6, 4, 65, dtype=torch.bfloat16, device=DEV)[..., 1:]      # addresses of 2 bytes
    check(ctx, rope, args, x, pos, out=odd)
    flat = x[:, 0].contiguous()
    check(ctx, rope, args, flat[:, None], pos)
    got = torch.empty_like(flat)
    vkv.rope_apply(ctx, rope, flat, pos, got)
    assert torch.equal(got, check(ctx, rope, args, flat[:, None], pos)[:, 0])


def test_the_transposed_map_is_the_gradient(ctx):
    """<R x, y> = <x, R^T y> for the map R, by differences of a linear map: each side a sum of n bf16-rounded terms."""
    rope = vkv.Rope(32, 10000.0, True, vkv.VKV_ROPE_PARTS, 8.0, 2048, 16.0, 2.0, 1.2)
    x, pos = data(11, 3, 48, 40000, 5)
    y, _ = data(11, 3, 48, 1, 6)
    a, b = torch.empty_like(x), torch.empty_like(x)
    vkv.rope_apply(ctx, rope, x, pos, a, first=8)
    vkv.rope_apply(ctx, rope, y, pos, b, first=8, transposed=True)
    left, right = a.double() * y.double(), x.double() * b.double()
    size = float(left.abs().sum() + right.abs().sum())
    assert abs(float(left.sum() - right.sum())) <= (BF + 64 * F32) * size


@pytest.mark.parametrize("inter", [False, True])
def test_the_gradient_against_differences(ctx, inter):
    """d(y . R x) / dx_j = y . (R(x + e_j) - R x), exactly so for a linear map: with x = 0 the columns of R, each rounded to bf16
    once (two entries of a column), against the gradient, rounded once."""
    D, at = 24, 12345
    rope = vkv.Rope(16, 500.0, inter, magnitude=0.9)
    one = torch.eye(D, dtype=torch.bfloat16, device=DEV)
    pos = torch.full((D,), at, dtype=torch.int32, device=DEV)
    cols, y = torch.empty_like(one), data(1, 1, D, 4, 8)[0][:, 0]
    vkv.rope_apply(ctx, rope, one, pos, cols, first=4)
    grad = torch.empty_like(y)
    vkv.rope_apply(ctx, rope, y, pos[:1], grad, first=4, transposed=True)
    want = cols.double() @ y[0].double()
    size = cols.double().abs() @ y[0].double().abs()
    assert bool(((grad[0].double() - want).abs() <= (2 * BF + 16 * F32) * size).all())


def test_not_finite_values_stay_in_their_pairs(ctx):
    x, pos = data(4, 2, 64, 100, 7)
    clean = torch.empty_like(x)
    rope = vkv.Rope(64)
    vkv.rope_apply(ctx, rope, x, pos, clean)
    x[1, 0, 3], x[2, 1, 40] = math.nan, math.inf
    out = torch.empty_like(x)
    vkv.rope_apply(ctx, rope, x, pos, out)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, 0, 3] = hit[1, 0, 35] = hit[2, 1, 40] = hit[2, 1, 8] = True
    assert torch.equal(out[~hit], clean[~hit]) and not bool(out[hit].isfinite().any())


def test_captured_and_on_another_stream(ctx):
    x, pos = data(8, 16, 64, 5000, 8)
    rope = vkv.Rope(64, interleaved=True)
    out = torch.empty_like(x)
    vkv.rope_apply(ctx, rope, x, pos, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vkv.rope_apply(ctx, rope, x, pos, out)
    for k in range(3):
        a, p = data(8, 16, 64, 5000, 20 + k)
        x.copy_(a)
        pos.copy_(p)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = torch.empty_like(x)
        vkv.rope_apply(ctx, rope, x, pos, want)
        assert torch.equal(got, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(ctx, rope, (64, 10000.0, 0, 1.0, 0, 0, 0), x, pos, inter=True, stream=s)


def test_very_many_tokens(ctx):
    """67 million tokens, four a workgroup: more workgroups of 256 than one grid dimension holds; offsets past 32 bits."""
    rope = vkv.Rope(256)
    n = (1 << 26) + 77
    x = torch.zeros(n, 256, dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    at = torch.tensor([0, 1, 12345, n // 2, (1 << 23) - 1, 1 << 23, n - 2, n - 1], device=DEV)
    some = data(8, 1, 256, 4, 99)[0][:, 0]
    x[at] = some
    vkv.rope_apply(ctx, rope, x, pos, x)
    torch.cuda.synchronize()
    want, tol = turned(some[:, None], pos[at], frequencies(256, 10000.0, vkv.VKV_ROPE_PLAIN, 1.0, 4096.0, 32.0, 1.0), 0, False, 1.0, False)
    assert bool(((x[at][:, None].double().cpu() - want).abs() <= tol).all())
    x[at] = 0
    assert not any(bool(part.any()) for part in x.split(1 << 24))
