"""vkv_weight_select where the sampled bracket of a long sequence ends between the negative weights and 0."""
import pytest
import torch

import paper_2609_03949_amd as vkv

from test_gpu_evict import check_tier, sampled_rows

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = vkv.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("n", [16400, 20000, 40000])
@pytest.mark.parametrize("share", [0.4, 0.45, 0.475, 0.5, 0.55, 0.65])
def test_bracket_that_ends_below_zero(ctx, n, share):
    """The smallest sampled weight is -1.9999999, whose distance to 0 in the order of the keys is a power of two, so a bin of
    the bracket's histogram ends right below 0; that bin holds tiny negative weights, the next one zeros of both signs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    w = torch.zeros(2, n, device=DEV)
    r, x = torch.rand(2, n, generator=g, device=DEV), torch.rand(2, n, generator=g, device=DEV)
    w[r < 0.05] = -0.0
    w[(r >= 0.05) & (r < 0.2)] = -1e-40
    w = torch.where((r >= 0.3) & (r < 0.6), 0.01 + 0.9 * x, w)
    w = torch.where(r >= 0.6, -x, w)
    at = sampled_rows(n).to(DEV)
    w[:, at[5]] = -torch.tensor(0x3FFFFFFF, dtype=torch.int32).view(torch.float32).item()
    w[1] = torch.where(w[1] == -1e-40, torch.zeros_like(w[1]), w[1])     # no weight between the last negative bin and 0
    check_tier(ctx, w, [n, n], int(n * share), 0, 0)
