"""Plain attention in 64 bits for the tests of the prompt and chunk operators, with bounds on how
far a result computed with bf16 operands and fp32 sums may be from it.

For one query, s_j the scores, p_j the softmax weights, v_jd the values:
  - a score is a sum of D exact products, accumulated in fp32: off by at most
    e = 2 (D + D/32) 2^-23 scale sum_d |q_d k_jd| (at most D + D/32 roundings, factor 2 of slack),
    and the exponent's argument by 4 2^-23 (|s_j| + max |s|) more (two roundings of each);
  - a relative weight exp(s_j) / sum exp(s) is then off by a factor within 2 e plus the roundings
    of the sum (n 2^-24 at most) and of exp2 and the division (16 2^-24);
  - the weight of the product with v is rounded to bf16: half a step, 2^-8 relative;
  - the sum over j in fp32: (n + n/32) 2^-23 of sum_j p_j |v_jd|;
  - the output is rounded to bf16: 2^-8 |o_d|.
"""
import math

import torch

BF, F32 = torch.finfo(torch.bfloat16).eps / 2, torch.finfo(torch.float32).eps / 2


def attention(q, k, v, seen, scale):
    """q [m, D], k [n, D], v [n, dv] (any type), seen [m, n] bool -> out, lse and their bounds, fp64 on the CPU.
    Rows that see nothing: out 0, lse -inf."""
    q, k, v, seen = q.double().cpu(), k.double().cpu(), v.double().cpu(), seen.cpu()
    m, n, D = q.shape[0], k.shape[0], q.shape[1]
    s = torch.where(seen, scale * (q @ k.T), torch.full((m, n), -math.inf, dtype=torch.float64))
    lse = torch.logsumexp(s, 1) if n else torch.full((m,), -math.inf, dtype=torch.float64)
    some = seen.any(1)
    p = torch.where(seen, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
    out = p @ v
    size = torch.where(seen, scale * (q.abs() @ k.abs().T), 0.0).amax(1) if n else torch.zeros(m, dtype=torch.float64)
    far = torch.where(seen, s.abs(), 0.0).amax(1) if n else torch.zeros(m, dtype=torch.float64)
    e = 2 * (D + D / 32) * 2 * F32 * size + 4 * 2 * F32 * 2 * far
    weight = 2 * e + (n + 16) * F32
    out_tol = BF * out.abs() + (BF + weight * (1 + BF) + (n + n / 32) * 2 * F32)[:, None] * (p @ v.abs()) + 1e-30
    lse_tol = e + (n + 16) * F32 + 4 * 2 * F32 * torch.where(some, lse, 0.0).abs() + 1e-30
    return out, lse, out_tol, lse_tol


def check(name, got, want, tol):
    """Every element within its bound; what is not finite equal in kind."""
    got, want = got.double().cpu(), want.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    other = ~fine & ~torch.isnan(want)
    assert torch.equal(got[other], want[other]), f"{name}: infinities differ"
    d = torch.where(fine, (got - want).abs() / tol, 0.0)
    assert d.numel() == 0 or float(d.max()) <= 1.0, f"{name}: {float(d.max()):.3g} of the bound at {int(d.argmax())}"
