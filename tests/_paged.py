"""Seeded paged caches and chunks of queries for the tests of the operators that read them."""
import torch

DEV = "cuda"


class Case:
    """kv_lens rows and q_lens new tokens per sequence; pages in random order, the rows behind a
    sequence's end and the spare pages hold NaN."""

    def __init__(self, kv_lens, q_lens, H, page=16, seed=0, max_q=None, max_kv=None, behind=0, spare=2):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.kv_lens, self.q_lens, self.H, self.page = list(kv_lens), list(q_lens), H, page
        B = len(self.kv_lens)
        used = [-(-n // page) for n in self.kv_lens]
        total = sum(used) + spare
        order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        self.max_kv = max(max(self.kv_lens), 0) if max_kv is None else max_kv
        self.table = torch.full((B, max(-(-self.max_kv // page), 1)), -1, dtype=torch.int32, device=DEV)
        self.cache = torch.full((total, page, 576), float("nan"), dtype=torch.bfloat16, device=DEV)
        at, self.where = 0, []
        for b, (n, k) in enumerate(zip(used, self.kv_lens)):
            self.table[b, :n] = order[at:at + n]
            u = torch.arange(k, device=DEV)
            pages = order[at:at + n].long()[u // page] if k else u
            self.where.append((pages, u % page))
            self.cache[pages, u % page] = torch.randn(k, 576, generator=g, device=DEV).to(torch.bfloat16)
            at += n
        self.kv_len = torch.tensor(self.kv_lens, dtype=torch.int32, device=DEV)
        n = sum(self.q_lens) + behind
        self.n_tok, self.max_q = n, max(self.q_lens) if max_q is None else max_q
        self.cu = torch.tensor([sum(self.q_lens[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV)
        self.q = torch.randn(n, H, 576, generator=g, device=DEV).to(torch.bfloat16)
        self.q_lat, self.q_rope = self.q[..., :512].contiguous(), self.q[..., 512:].contiguous()

    def rows(self, b):
        """Sequence b's cache rows [kv, 576]."""
        return self.cache[self.where[b]]

    def seen(self, b):
        """[nq, kv]: which rows each new token sees."""
        n, nq = self.kv_lens[b], self.q_lens[b]
        return torch.arange(n)[None, :] <= (n - nq + torch.arange(nq))[:, None]
