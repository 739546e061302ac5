"""vkv_rope_apply with frequencies extended by parts over the pair's index, against the formula in 64 bits, forward and as a
gradient takes it."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from test_abi_rope_index import BY_INDEX, by_index
from test_gpu_rope import data, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("D,first", [(64, 0), (576, 512), (70, 3)])
def test_by_index(ctx, inter, back, D, first):
    x, pos = data(41, 5, D, 163840, D)
    rope = vkv.Rope(64, 10000.0, inter, BY_INDEX, 40.0, 4096, 32.0, 1.0, 1.2)
    out = torch.full_like(x, 9.0)
    vkv.rope_apply(ctx, rope, x, pos, out, first=first, transposed=back)
    torch.cuda.synchronize()
    want, tol = turned(x, pos, by_index(64, 10000.0, 40.0, 4096.0, 32.0, 1.0), first, inter, 1.2, back)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
