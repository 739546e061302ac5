"""vkv_chunk8_attend where one row outweighs each of up to 2^24 others by 2^18 to 2^33: light one by one, what they add together
has to reach the outputs, as it does the sums.  (Tables that name a few pages over and over, so that the context costs nothing.)

A weight is rounded to fp16, half a step of 2^-11 of it, or by 2^-25 at the most below fp16's normal numbers, where the reference has
made the largest weight of the segment 2^first, and first is such that the rows of one lose 2^-11 of that together.  (Segments without
the heavy row have references of their own, 2^-18 of its weight and less.)  So beside the output's own half step of bf16, the weights'
roundings in fp32 (2^-12 of one: 2^-24 of a score of up to 24 and what follows) and the sums' (n terms, none of them negative, each
added once, with the products of 32 rows summed before: (n + n/32) 2^-23 of the result for the output and for the sum of the
weights, as in _attention.py; n those of a run, and the runs, where there are some), an output is off by 2^-11 of the heavy row's weight times the largest magnitude in its dim.  In 256 runs a segment has 2^16 of 2^24 rows; with a bound on the new
tokens that gives too many units, a workgroup takes a whole context."""
import math

import pytest
import torch

import paper_2609_03949_amd as vkv

from _paged8 import decode

pytestmark = pytest.mark.gpu
DEV, BF, I32 = "cuda", torch.bfloat16, torch.int32
SCALE = 1.0 / math.sqrt(192.0)


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("log,heavy,max_q", [(12, 0, 1), (16, 65535, 1), (20, 700000, 1), (24, 5, 1), (16, 0, 1 << 14), (20, 0, 1 << 14),
                                             (20, 700000, 1 << 14), (22, 99, 1 << 14)])
@pytest.mark.parametrize("H", [16, 32, 64, 128])
@pytest.mark.parametrize("byte", [127, 120])
def test_rows_that_are_light_one_by_one(ctx, log, heavy, max_q, H, byte):
    n, page, some = 1 << log, 64, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(log + H)
    rows = torch.randn(some, page, 640, generator=g, device=DEV)
    cache = torch.empty(some, page, 640, dtype=torch.uint8, device=DEV)
    codes = (64 + 32 * rows[..., :512]).clamp(8, 448)          # positive: nothing cancels
    codes[0, heavy % page, 256:] = 0                            # half of the dims have light rows alone
    cache[..., :512] = codes.to(torch.float8_e4m3fn).view(torch.uint8)
    branch = torch.zeros(some, page, 64, dtype=BF, device=DEV)
    branch[0, heavy % page, 0] = math.log(2.0) / SCALE
    cache[..., 512:] = branch.view(torch.uint8)
    scale = torch.full((some, page // 16), byte, dtype=torch.uint8, device=DEV)
    scale[0, heavy % page // 16] = 127
    table = (1 + torch.arange(n // page, device=DEV) % (some - 1)).to(I32)
    table[heavy // page] = 0
    k = 18 + torch.arange(H, device=DEV) % 16                   # a head's light rows weigh 2^-k
    q_lat, q_rope = torch.zeros(1, H, 512, dtype=BF, device=DEV), torch.zeros(1, H, 64, dtype=BF, device=DEV)
    q_rope[0, :, 0] = k.to(BF)
    pages = vkv.Pages8(cache, scale, table[None], torch.tensor([n], dtype=I32, device=DEV), n)
    chunk = vkv.Chunk(q_lat, q_rope, torch.tensor([0, 1], dtype=I32, device=DEV), max_q)
    ws = torch.empty(max(vkv.chunk8_workspace_size(pages, chunk), 256), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(1, H, 512, dtype=BF, device=DEV), torch.empty(1, H, device=DEV)
    vkv.chunk8_attend(ctx, pages, chunk, ws, SCALE, out, lse)
    torch.cuda.synchronize()
    times = torch.bincount(table.long(), minlength=some).double().cpu()[:, None].expand(some, page).reshape(-1)
    v = decode(cache[..., :512], scale.repeat_interleave(16, 1)).reshape(-1, 512)
    f = torch.pow(2.0, scale.cpu().double() - 127).repeat_interleave(16, 1).reshape(-1)
    s = SCALE * (k.double().cpu()[:, None] * branch.double().cpu()[..., 0].reshape(1, -1))
    w = torch.exp(s - s.amax(1, keepdim=True))                  # [H, rows]; of the largest: 1
    total = (w * times).sum(1, keepdim=True)
    want = (w * times) @ v / total
    floor = 2.0 ** -11 * (w * f).amax(1, keepdim=True) * (v / f[:, None]).amax(0) / total
    terms = n if max_q > 1 else n // 256 + 512                  # of one sum; in runs, of one run's, and 256 runs
    sums = (terms + terms / 32) * 2.0 ** -23
    tol = (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -12 + sums) * want + floor
    d = (out[0].double().cpu() - want).abs() / tol
    assert float(d.max()) <= 1.0, f"{float(d.max()):.3g} of the bound, head {int(d.amax(1).argmax())}"
    l = torch.log(total[:, 0]) + s.amax(1)
    assert bool(((lse[0].double().cpu() - l).abs() <= 2.0 ** -12 * (1 + l.abs()) + sums).all())
