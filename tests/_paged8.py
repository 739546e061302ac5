"""Seeded paged caches held in 8 bits, and what their codes stand for, for the tests of the operators that read and write them."""
import numpy as np
import torch

DEV = "cuda"
# the 127 magnitudes of the 8-bit format, by code: 4 exponent bits of bias 7, 3 fraction bits
VALUES = np.array([(c % 8) * 2.0 ** -9 if c < 8 else (1 + (c % 8) / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])
BYTE_MIN, BYTE_MAX, TOP = 63, 191, 448.0


def decode(codes, byte):
    """codes uint8 [..., n], byte [...] -> fp64 (NaN codes: NaN); bytes outside [63, 191] count as the nearest bound."""
    c, s = codes.cpu().numpy(), np.clip(byte.cpu().numpy().astype(np.int64), BYTE_MIN, BYTE_MAX)
    table = np.concatenate([VALUES, [np.nan]])
    v = table[c & 0x7F] * np.where(c & 0x80, -1.0, 1.0)
    return torch.from_numpy(v * 2.0 ** (s - 127.0)[..., None])


def encode(x):
    """fp64 values within +-448 (or NaN) -> codes, nearest, halfway to the even code."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(VALUES, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    down = (a - VALUES[lo] < VALUES[hi] - a) | ((a - VALUES[lo] == VALUES[hi] - a) & (lo % 2 == 0))
    c = np.where(np.isnan(x), 127, np.where(down, lo, hi)).astype(np.uint8)
    return c | np.where(np.signbit(x) & ~np.isnan(x), 128, 0).astype(np.uint8)


def least_byte(x):
    """The scale byte of the values x (fp64): the least with every finite one up to 448 * 2^64 within 448 times it."""
    a = np.abs(x[np.isfinite(x)]) if x.size else x
    a = a[a <= TOP * 2.0 ** 64]
    top, s = (a.max() if a.size else 0.0), BYTE_MIN
    while s < BYTE_MAX and top > TOP * 2.0 ** (s - 127):
        s += 1
    return s


def same_codes(a, b):
    """Codes that stand for the same values (of NaN and of zero there are two each)."""
    a, b = np.asarray(a), np.asarray(b)
    nan = ((a & 0x7F) == 0x7F) & ((b & 0x7F) == 0x7F)
    zero = ((a & 0x7F) == 0) & ((b & 0x7F) == 0)
    return bool(((a == b) | nan | zero).all())


class Case8:
    """kv_lens rows and q_lens new tokens per sequence; pages in random order; the rows behind a sequence's
    end and the spare pages hold NaN."""

    def __init__(self, kv_lens, q_lens, H, page=16, block=16, seed=0, max_q=None, max_kv=None, behind=0, spare=2,
                 spread=1.0, pad=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.kv_lens, self.q_lens, self.H, self.page, self.block = list(kv_lens), list(q_lens), H, page, block
        B = len(self.kv_lens)
        used = [-(-n // page) for n in self.kv_lens]
        total = sum(used) + spare
        order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        self.max_kv = max(max(self.kv_lens), 0) if max_kv is None else max_kv
        self.table = torch.full((B, max(-(-self.max_kv // page), 1)), -1, dtype=torch.int32, device=DEV)
        self.whole = torch.full((total, page, 640 + pad), 0x7F, dtype=torch.uint8, device=DEV)
        self.cache = self.whole[..., :640]
        self.cache[..., 512:].copy_(torch.full((total, page, 64), float("nan"), dtype=torch.bfloat16, device=DEV).view(torch.uint8))
        # normal codes under scales of different size
        e = torch.randn(total, page // block, generator=g, device=DEV) * spread
        self.scale = (121 + e.round()).clamp(0, 255).to(torch.uint8)
        at, self.where = 0, []
        for b, (n, k) in enumerate(zip(used, self.kv_lens)):
            self.table[b, :n] = order[at:at + n]
            u = torch.arange(k, device=DEV)
            pages = order[at:at + n].long()[u // page] if k else u
            self.where.append((pages, u % page))
            x = (64 * torch.randn(k, 512, generator=g, device=DEV)).clamp(-448, 448)
            self.cache[pages, u % page, :512] = x.to(torch.float8_e4m3fn).view(torch.uint8)
            r = torch.randn(k, 64, generator=g, device=DEV).to(torch.bfloat16)
            self.cache[pages, u % page, 512:] = r.view(torch.uint8)
            at += n
        self.kv_len = torch.tensor(self.kv_lens, dtype=torch.int32, device=DEV)
        n = sum(self.q_lens) + behind
        self.n_tok, self.max_q = n, max(self.q_lens) if max_q is None else max_q
        self.cu = torch.tensor([sum(self.q_lens[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV)
        self.q = torch.randn(n, H, 576, generator=g, device=DEV).to(torch.bfloat16)
        self.q_lat, self.q_rope = self.q[..., :512].contiguous(), self.q[..., 512:].contiguous()

    def rows(self, b):
        """Sequence b's cache rows [kv, 576], fp64 on the CPU."""
        p, r = self.where[b]
        raw = self.cache[p, r]
        lat = decode(raw[:, :512], self.scale[p, r // self.block])
        return torch.cat([lat, raw[:, 512:].contiguous().view(torch.bfloat16).double().cpu()], 1)

    def scales(self, b):
        """The power of two of each of sequence b's rows, fp64 on the CPU."""
        p, r = self.where[b]
        return torch.pow(2.0, self.scale[p, r // self.block].cpu().double().clamp(BYTE_MIN, BYTE_MAX) - 127)

    def seen(self, b):
        """[nq, kv]: which rows each new token sees."""
        n, nq = self.kv_lens[b], self.q_lens[b]
        return torch.arange(n)[None, :] <= (n - nq + torch.arange(nq))[:, None]
