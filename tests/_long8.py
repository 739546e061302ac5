"""Long contexts in 8 bits whose outputs tell every cache row from the others, and bounds on them that count a weight's rounding to
fp16 and no more.

Scores come from the first dim of the branch alone, but for 2^-12 of them: so the bound on a score's error, which goes by the sum of
the magnitudes of its products, is as small as its error.  For one query, p_j the softmax weights, v_jd the values, f_j a row's power of
two, n rows:
  - a score s_j, with e = 2 (576 + 18) 2^-23 size + 8 2^-23 |s| of error (as in _attention.py), gives p_j within 2 e + (n + 16) 2^-24;
  - p_j f_j is rounded to fp16: half a step of 2^-11 of it, or 2^-25 of the largest of them;
  - the sum over j in fp32: (n + n/32) 2^-23 of sum_j p_j |v_jd|;
  - the output is rounded to bf16: half a step.
These count every rounding at its most and of one sign.  The norm of the outputs' error is held against what the roundings make
together where they are even and independent:
  - a half step of bf16 is an even error of mean square z = step^2 / 12, whose square has 0.9 of that as deviation: the sum of them is
    below sum z + 6 * 0.9 sqrt(c sum z^2), where the outputs of c queries with the same scores have the same errors;
  - an output takes (2^-11 p_j v_jd)^2 / 3 of the weights' roundings, or (2^-25 of the largest p_j f_j v_jd / f_j)^2 below fp16's normal
    numbers (no row here is so light that it is lost), and (4 e p_j v_jd)^2 of the scores', where e has the square root of 594 in place of it;
  - the sums' roundings grow with the square root of n, and each is 2^-24 of a partial sum, which for rows in no order is within
    |o_d| + 4 sqrt(sum_j (p_j v_jd)^2): 2 sqrt(n) 2^-24 of that.
"""
import math

import torch

import _paged8

SCALE = 1.0 / math.sqrt(192.0)
BF, F16, F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


def spread(x, seed, nats=1.5, own=False):
    """Queries and branches of case x so that scores are nats * normal; the values have next to no say in them.  own: a
    query has a factor of its own, 0.5 to 2, as far as bf16 has some."""
    g = torch.Generator(device=_paged8.DEV)
    g.manual_seed(seed)
    x.q[..., :512] *= 2.0 ** -12
    x.q[..., 512:] = 0
    x.q[..., 512] = 1.0
    if own:
        n = x.n_tok * x.H
        x.q[..., 512] = torch.pow(2.0, -1 + 2 * torch.arange(n, device=_paged8.DEV) / n).view(x.n_tok, x.H).to(torch.bfloat16)
    x.q_lat, x.q_rope = x.q[..., :512].contiguous(), x.q[..., 512:].contiguous()
    for p, r in x.where:
        branch = torch.zeros(len(p), 64, dtype=torch.bfloat16, device=_paged8.DEV)
        branch[:, 0] = (nats / SCALE * torch.randn(len(p), generator=g, device=_paged8.DEV)).to(torch.bfloat16)
        x.cache[p, r, 512:] = branch.view(torch.uint8)
    return x


def marked(x):
    """Row j has the one value 64 to 120, in dim 37 j mod 512: the rows of 512 in a row lie in dims of their own."""
    for p, r in x.where:
        j = torch.arange(len(p), device=_paged8.DEV)
        code = torch.zeros(len(p), 512, device=_paged8.DEV)
        code[j, 37 * j % 512] = 64.0 + 8 * (j % 8)
        x.cache[p, r, :512] = code.to(torch.float8_e4m3fn).view(torch.uint8)
    return x


class Exact:
    """Sequence b's outputs in 64 bits, [tokens * heads, 512], and their bounds."""

    def __init__(self, x, b):
        nq, at = x.q_lens[b], sum(x.q_lens[:b])
        kv, self.f = x.rows(b), x.scales(b)
        n = kv.shape[0]
        q = x.q[at:at + nq].reshape(nq * x.H, 576).double().cpu()
        self.vis = x.seen(b)[:, None, :].expand(nq, x.H, n).reshape(nq * x.H, n)
        self.s = torch.where(self.vis, SCALE * (q @ kv.T), -math.inf)
        self.lse = torch.logsumexp(self.s, 1)
        self.p, self.v = torch.exp(self.s - self.lse[:, None]), kv[:, :512]
        self.out = self.p @ self.v
        size, far = SCALE * (q.abs() @ kv.abs().T).amax(1), torch.where(self.vis, self.s.abs(), 0.0).amax(1)
        self.e = 2 * (576 + 18) * 2 * F32 * size + 8 * 2 * F32 * far
        self.some = self.p @ self.v.abs()
        rest = 2 * self.e + (n + 16) * F32 + (n + n / 32) * 2 * F32
        light = 2.0 ** -25 * (self.p * self.f).amax(1, keepdim=True) * (self.vis.double() @ (self.v.abs() / self.f[:, None]))
        fixed = rest[:, None] * self.some + light
        self.tol = BF * self.out.abs() + F16 * self.some * (1 + BF) + fixed + 1e-30
        step = torch.pow(2.0, torch.floor(torch.log2(self.out.abs().clamp(min=1e-30))) - 7)
        z = step ** 2 / 12
        even = z.sum() + 5.4 * torch.sqrt(q.shape[0] / len(torch.unique(q[:, 512])) * (z ** 2).sum())
        each = 4 * (2 * math.sqrt(594) * 2 * F32 * size + 8 * 2 * F32 * far)
        square = self.p ** 2 @ self.v ** 2
        low = (2.0 ** -25 * (self.p * self.f).amax(1, keepdim=True)) ** 2 * (self.vis.double() @ (self.v / self.f[:, None]) ** 2)
        sums = 2 * math.sqrt(n) * F32 * (self.out.abs() + 4 * torch.sqrt(square))
        self.norm = float(torch.sqrt(even + ((F16 ** 2 / 3 + each[:, None] ** 2) * square + low).sum()) + torch.linalg.norm(sums))

    def far(self, got):
        """The largest error as a part of its bound, and the norm's."""
        d = got.double().cpu() - self.out
        return float((d.abs() / self.tol).max()), float(torch.linalg.norm(d)) / self.norm

    def check(self, got, lse):
        each, norm = self.far(got)
        assert each <= 1.0 and norm <= 1.0, f"{each:.3g} of the bound on each output, {norm:.3g} of the norm's"
        tol = self.e + (self.p.shape[1] + 16) * F32 + 8 * F32 * self.lse.abs()
        assert bool(((lse.double().cpu() - self.lse).abs() <= tol).all())
