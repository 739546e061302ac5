"""The operators around the decode step, as cases that can be timed and checked.

Prompt attention (`prompt`), attention of a chunk of new tokens over a paged latent cache (`chunk`),
and eviction by accumulated attention weight: the weights (`weights`), the tier they give
(`select`) and the move of its rows to the front of the paged cache (`evict`).  `own` says whether
`run` calls libvkv or computes the operator in its plain form, in 32 bits with elementary torch
operations.  `exact` is the definition in 64 bits, sequence by sequence.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
SCALE = 1.0 / math.sqrt(192.0)
D_LAT, D_ROPE, D_ROW = 512, 64, 576
_kept = {}             # what a program keeps for the process: its libvkv context


def listed():
    return [
        # one long document prefilled by a tensor-parallel shard of 16 heads, expanded MLA heads
        dict(name="prompt_16k_mla", kind="prompt", B=1, H=16, Hk=16, L=16384, low=16384, dn=128, dr=64, dv=128),
        # a serving batch of ordinary prompts of different lengths, grouped heads
        dict(name="prompt_2k_grouped", kind="prompt", B=16, H=32, Hk=8, L=2048, low=17, dn=128, dr=0, dv=128),
        # a few short prompts, narrow heads: the launch is what counts
        dict(name="prompt_short", kind="prompt", B=4, H=16, Hk=4, L=129, low=1, dn=64, dr=0, dv=64),
        # single-token decode of one sequence on a shard of 16 heads
        dict(name="chunk_8k_decode", kind="chunk", B=1, H=16, T=8192, low=8192, nq=1, page=16),
        # decode of a full batch at full head count, contexts of different lengths
        dict(name="chunk_32k_decode", kind="chunk", B=32, H=128, T=32768, low=20011, nq=1, page=64),
        # chunked prefill: the next 512 tokens of three requests
        dict(name="chunk_16k_prefill", kind="chunk", B=3, H=128, T=16384, low=9001, nq=512, page=64),
        # observation window of the last 32 tokens over long contexts, as weights before an eviction
        dict(name="weights_64k_window", kind="weights", B=4, H=64, T=65536, low=50021, nq=32, page=64),
        # the weights' update after a decode step
        dict(name="weights_32k_decode", kind="weights", B=16, H=128, T=32768, low=32768, nq=1, page=128),
        # tier of one sequence of ordinary length
        dict(name="select_8k", kind="select", B=1, T=8192, low=8192, keep=1024, sinks=4, recent=128),
        # tiers of a batch of long contexts
        dict(name="select_128k", kind="select", B=32, T=131072, low=99991, keep=4096, sinks=4, recent=512),
        # one sequence cut to an eighth
        dict(name="evict_8k", kind="evict", B=1, T=8192, low=8192, keep=1024, page=16),
        # a batch of contexts cut to a thirty-second
        dict(name="evict_32k", kind="evict", B=16, T=32768, low=30011, keep=1024, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "chunk", "chunk", "chunk", "weights", "select", "evict"])
    if kind == "prompt":
        dn, dr, dv = rng.choice([(128, 64, 128), (128, 0, 128), (64, 0, 64)])
        Hk = _log(rng, 1, 16)
        H = Hk * rng.choice([1, 2, 4, 8])
        L = _log(rng, 32, 16384)
        L = min(L, int(16384 * math.sqrt(16 / H)))
        B = max(1, min(_log(rng, 1, 32), 16 * 16384 * 16384 // (H * L * L)))
        return dict(kind=kind, B=B, H=H, Hk=Hk, L=L, low=rng.randint(1, L), dn=dn, dr=dr, dv=dv)
    T = _log(rng, 2048, 131072)
    if kind in ("chunk", "weights"):
        H, nq = _log(rng, 4, 128), rng.choice([1, 1, _log(rng, 2, 512)])
        T = min(T, 65536)
        B = max(1, min(_log(rng, 1, 32), 8 * 65536 // T))
        nq = max(1, min(nq, 3 * 512 * 128 * 11264 // (B * H * T)))
        return dict(kind=kind, B=B, H=H, T=T, low=rng.randint(max(nq, T // 2), T), nq=nq, page=1 << rng.randint(4, 8))
    B = max(1, min(_log(rng, 1, 32), (32 * 131072 if kind == "select" else 16 * 32768) // T))
    keep = max(64, T // _log(rng, 4, 64))
    c = dict(kind=kind, B=B, T=T, low=rng.randint(T // 2, T), keep=keep)
    return dict(c, sinks=4, recent=rng.randint(0, 512) % (keep - 4)) if kind == "select" else dict(c, page=1 << rng.randint(4, 8))


def _lens(B, top, low):
    """B lengths in [low, top], the first one the longest."""
    return [top] + [low + int((top - low + 1) * ((b * 0.6180339887498949) % 1.0)) for b in range(1, B)]


def _kv_lens(case):
    return _lens(case["B"], case["T"], case["low"])


def _q_lens(case):
    """New tokens of each sequence: the chunk's size, and less of it in every third sequence."""
    return [case["nq"] if b % 3 != 2 else (case["nq"] + 1) // 2 for b in range(case["B"])]


def _starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def _pairs(case):
    """(query, row) pairs that the causal mask leaves, over all sequences."""
    if case["kind"] == "prompt":
        return sum(n * (n + 1) // 2 for n in _lens(case["B"], case["L"], case["low"]))
    return sum(q * k - q * (q - 1) // 2 for q, k in zip(_q_lens(case), _kv_lens(case)))


def work(case):
    kind, B = case["kind"], case["B"]
    if kind == "prompt":
        n = sum(_lens(B, case["L"], case["low"]))
        H, Hk, dn, dr, dv = (case[x] for x in ("H", "Hk", "dn", "dr", "dv"))
        return {"bytes": n * (2 * H * (dn + dr + dv) + 2 * Hk * (dn + dv) + 2 * dr + 4 * H),
                "flops": 2 * H * (dn + dr + dv) * _pairs(case)}
    rows = sum(_kv_lens(case))
    if kind in ("chunk", "weights"):
        q, H = sum(_q_lens(case)), case["H"]
        if kind == "chunk":
            return {"bytes": 2 * D_ROW * (rows + q * H) + q * H * (2 * D_LAT + 4),
                    "flops": 2 * (D_ROW + D_LAT) * H * _pairs(case)}
        return {"bytes": 2 * D_ROW * (rows + q * H) + 4 * q * H + 8 * rows, "flops": 2 * D_ROW * H * _pairs(case)}
    K = case["keep"]
    if kind == "select":
        return {"bytes": 4 * rows + 4 * B * K, "flops": 0}
    moved = sum(K - K * K // n for n in _kv_lens(case) if n > K)     # kept rows lie evenly over the context
    return {"bytes": 2 * 2 * D_ROW * moved + 16 * B * K, "flops": 0}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _pages(g, case, s):
    """A paged cache whose pages lie in any order, and the sequences' tables."""
    page, lens = case["page"], _kv_lens(case)
    width = -(-max(lens) // page)
    used = [-(-n // page) for n in lens]
    total = sum(used) + 3
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    s["cache"] = _normal(g, total, page, D_ROW)
    s["table"], s["kv_len"], s["max_kv"] = table, _i32(lens), max(lens)


def _weights(g, B, T):
    """Accumulated weights as they come out: heavy-tailed, many of them nearly nothing, some equal."""
    w = torch.exp(2.0 * torch.randn(B, T, generator=g, device=DEV)) / T
    return torch.where(torch.rand(B, T, generator=g, device=DEV) < 0.05, torch.zeros_like(w), w)


def prepare(case, seed):
    g = _generator(seed)
    kind, B = case["kind"], case["B"]
    s = {"case": dict(case)}
    if kind == "prompt":
        lens = _lens(B, case["L"], case["low"])
        n = sum(lens)
        s["lens"], s["cu"], s["max_len"] = lens, _i32(_starts(lens)), max(lens)
        s["q"] = _normal(g, n, case["H"], case["dn"] + case["dr"])
        s["k"] = _normal(g, n, case["Hk"], case["dn"])
        s["k_rope"] = _normal(g, n, case["dr"]) if case["dr"] else None
        s["v"] = _normal(g, n, case["Hk"], case["dv"])
        return s
    if kind in ("chunk", "weights"):
        _pages(g, case, s)
        lens = _q_lens(case)
        n = sum(lens)
        s["lens"], s["cu"], s["max_q"] = lens, _i32(_starts(lens)), max(lens)
        s["q_lat"], s["q_rope"] = _normal(g, n, case["H"], D_LAT), _normal(g, n, case["H"], D_ROPE)
        if kind == "weights":
            s["prev"] = _weights(g, B, case["T"])
            # the attention call of the same step leaves the lse; here one of that size is drawn
            s["lse"] = math.log(case["T"]) + 1.5 + 0.05 * torch.randn(n, case["H"], generator=g, device=DEV)
        return s
    if kind == "select":
        s["kv_len"], s["weight"] = _i32(_kv_lens(case)), _weights(g, B, case["T"])
        return s
    _pages(g, case, s)
    K = case["keep"]
    s["prev"] = _weights(g, B, case["T"])
    # a tier as the selection leaves it: rows anywhere in the context, ascending, -1 past the count
    u = torch.rand(B, case["T"], generator=g, device=DEV)
    u = torch.where(torch.arange(case["T"], device=DEV)[None, :] < s["kv_len"][:, None], u, torch.full_like(u, -1.0))
    kept = u.topk(K, dim=1).indices.sort(dim=1).values
    s["count"] = torch.clamp(s["kv_len"], max=K)
    kept = torch.where(kept < s["kv_len"][:, None], kept, torch.full_like(kept, 1 << 30)).sort(dim=1).values
    s["kept"] = torch.where(kept < (1 << 30), kept, torch.full_like(kept, -1)).to(torch.int32)
    return s


# ------------------------------------------------------------------ the plain forms

def _padded(x, cu, n_max):
    """Packed rows [n, ...] -> [B, n_max, ...] in 32 bits (rows past a sequence's end repeat one of the tensor's)."""
    at = cu[:-1, None].long() + torch.arange(n_max, device=DEV)[None, :]
    return x[at.clamp(max=x.shape[0] - 1)].float()


def _packed(x, cu, n):
    """[B, n_max, ...] -> the packed rows [n, ...]."""
    tok = torch.arange(n, device=DEV)
    b = (tok[:, None] >= cu[None, 1:].long()).sum(1)
    return x[b, tok - cu.long()[b]]


def _softmax_parts(s, visible):
    """exp(s - max), its sum and the log-sum-exp of each row of s, in place; rows that see nothing have sum 0 and lse -inf."""
    s.masked_fill_(~visible, -math.inf)
    m = s.amax(-1, keepdim=True)
    s.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = s.sum(-1, keepdim=True)
    return s, total, (m + torch.log(total)).squeeze(-1)


def _plain_prompt(s):
    c, n, L = s["case"], s["q"].shape[0], s["max_len"]
    H, Hk, dn = c["H"], c["Hk"], c["dn"]
    q = _padded(s["q"], s["cu"], L).permute(0, 2, 1, 3).reshape(c["B"], Hk, H // Hk * L, -1)
    k = _padded(s["k"], s["cu"], L).permute(0, 2, 3, 1)
    x = torch.matmul(q[..., :dn], k)
    if c["dr"]:
        x += torch.matmul(q[..., dn:], _padded(s["k_rope"], s["cu"], L).transpose(1, 2)[:, None])
    x = x.mul_(SCALE).view(c["B"], Hk, H // Hk, L, L)
    visible = torch.ones(L, L, dtype=torch.bool, device=DEV).tril()
    p, total, lse = _softmax_parts(x, visible)
    v = _padded(s["v"], s["cu"], L).permute(0, 2, 1, 3)
    o = torch.matmul(p.view(c["B"], Hk, H // Hk * L, L), v).view(c["B"], H, L, -1) / total.view(c["B"], H, L, 1)
    out = _packed(o.permute(0, 2, 1, 3), s["cu"], n).to(torch.bfloat16)
    return {"out": out, "lse": _packed(lse.reshape(c["B"], H, L).permute(0, 2, 1), s["cu"], n)}


def _cached_rows(s):
    """The sequences' cache rows [B, max_kv, 576] in 32 bits."""
    page = s["cache"].shape[1]
    u = torch.arange(s["max_kv"], device=DEV)
    at = s["table"].long()[:, u // page].clamp(min=0) * page + u % page
    return s["cache"].view(-1, D_ROW)[at].float()


def _chunk_scores(s):
    """(scores [B, max_q, H, max_kv], which of them the mask leaves, the cache rows)."""
    c, Q, T = s["case"], s["max_q"], s["max_kv"]
    kv = _cached_rows(s)
    q = torch.cat([_padded(s["q_lat"], s["cu"], Q), _padded(s["q_rope"], s["cu"], Q)], -1)
    x = torch.bmm(q.view(c["B"], Q * c["H"], D_ROW), kv.transpose(1, 2)).mul_(SCALE)
    nq = (s["cu"][1:] - s["cu"][:-1]).long()
    i = torch.arange(Q, device=DEV)
    last = s["kv_len"].long()[:, None] - nq[:, None] + i[None, :]
    visible = torch.arange(T, device=DEV)[None, None, :] <= last[:, :, None]
    visible &= (i[None, :] < nq[:, None])[:, :, None]
    return x.view(c["B"], Q, c["H"], T), visible[:, :, None, :], kv


def _plain_chunk(s):
    c, Q, n = s["case"], s["max_q"], s["q_lat"].shape[0]
    x, visible, kv = _chunk_scores(s)
    p, total, lse = _softmax_parts(x, visible)
    o = torch.bmm(p.view(c["B"], Q * c["H"], -1), kv[..., :D_LAT]).view(c["B"], Q, c["H"], D_LAT)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return {"out": _packed(o, s["cu"], n).to(torch.bfloat16), "lse": _packed(lse, s["cu"], n)}


def _plain_weights(s):
    c, Q, T = s["case"], s["max_q"], s["max_kv"]
    x, visible, _ = _chunk_scores(s)
    lse = _padded(s["lse"], s["cu"], Q)
    p = x.sub_(lse[..., None]).masked_fill_(~visible, -math.inf).exp_()
    u = torch.arange(T, device=DEV)[None, :]
    n, nq = s["kv_len"].long()[:, None], (s["cu"][1:] - s["cu"][:-1]).long()[:, None]
    prev = torch.where(u < n - nq, s["prev"], torch.zeros_like(s["prev"]))
    return {"weight": torch.where(u < n, 0.9 * prev + p.sum((1, 2)), s["prev"])}


def _plain_select(s):
    c, w = s["case"], s["weight"]
    T, K = c["T"], c["keep"]
    u, n = torch.arange(T, device=DEV)[None, :], s["kv_len"].long()[:, None]
    # what is kept in any case comes first, what is no row last
    w = torch.where((u < c["sinks"]) | (u >= n - c["recent"]), torch.full_like(w, math.inf), w)
    w = torch.where(u < n, w, torch.full_like(w, -math.inf))
    first = torch.sort(w, dim=1, descending=True, stable=True).indices[:, :K]
    kept = torch.where(first < n, first, torch.full_like(first, T)).sort(dim=1).values
    return {"kept": torch.where(kept < T, kept, torch.full_like(kept, -1)).to(torch.int32),
            "count": torch.clamp(s["kv_len"], max=K)}


def _plain_evict(s):
    c, kept = s["case"], s["kept"].long()
    B, K, page = c["B"], c["keep"], s["cache"].shape[1]
    slot = torch.arange(K, device=DEV)[None, :].expand(B, K)
    live = slot < s["count"].long()[:, None]
    stays = torch.zeros(B, K + 1, dtype=torch.bool, device=DEV)
    stays.scatter_(1, torch.where(live & (kept < K), kept, torch.full_like(kept, K)), True)
    stays = stays[:, :K]
    # the r-th slot that holds no kept row takes the r-th kept row from K on
    rank = torch.cumsum((live & ~stays).long(), 1) - 1
    below = (live & (kept < K)).sum(1, keepdim=True)
    source = torch.where(stays | ~live, slot, kept.gather(1, (below + rank).clamp(0, K - 1)))
    table, rows = s["table"].long(), s["cache"].view(-1, D_ROW)
    b, j = (live & ~stays).nonzero(as_tuple=True)
    u = source[b, j]
    rows[table[b, j // page] * page + j % page] = rows[table[b, u // page] * page + u % page]
    return {"cache": s["cache"], "origin": torch.where(live, source, torch.full_like(source, -1)).to(torch.int32),
            "weight": torch.where(live, s["prev"].gather(1, source), torch.zeros(B, K, device=DEV))}


# ------------------------------------------------------------------ libvkv's calls

def _plan(s):
    """What a program keeps from pass to pass: the context, the descriptions of its tensors, workspace and outputs."""
    import paper_2609_03949_amd as vkv
    if "ctx" not in _kept:
        _kept["ctx"] = vkv.Context(0)
    c, kind, p = s["case"], s["case"]["kind"], {}
    if kind == "prompt":
        p["prompt"] = vkv.Prompt(s["q"], s["k"], s["v"], s["cu"], s["max_len"], k_rope=s["k_rope"])
        p["out"] = torch.empty(s["q"].shape[0], c["H"], c["dv"], dtype=torch.bfloat16, device=DEV)
        p["lse"] = torch.empty(s["q"].shape[0], c["H"], device=DEV)
    if kind in ("chunk", "weights", "evict"):
        p["pages"] = vkv.Pages(s["cache"], s["table"], s["kv_len"], s["max_kv"])
    if kind in ("chunk", "weights"):
        p["chunk"] = vkv.Chunk(s["q_lat"], s["q_rope"], s["cu"], s["max_q"])
    if kind == "chunk":
        n = s["q_lat"].shape[0]
        p["ws"] = torch.empty(vkv.chunk_workspace_size(p["pages"], p["chunk"]), dtype=torch.uint8, device=DEV)
        p["out"] = torch.empty(n, c["H"], D_LAT, dtype=torch.bfloat16, device=DEV)
        p["lse"] = torch.empty(n, c["H"], device=DEV)
    if kind == "weights":
        p["ws"] = torch.empty(vkv.weight_workspace_size(p["pages"], p["chunk"]), dtype=torch.uint8, device=DEV)
        p["weight"] = s["prev"].clone()
    if kind in ("select", "evict"):
        K = c["keep"]
        p["kept"] = torch.empty(c["B"], K, dtype=torch.int32, device=DEV)
        p["count"] = torch.empty(c["B"], dtype=torch.int32, device=DEV)
        p["origin"] = torch.empty(c["B"], K, dtype=torch.int32, device=DEV)
        p["weight"] = torch.zeros(c["B"], K, device=DEV)
    return p


def _own(s):
    import paper_2609_03949_amd as vkv
    if "plan" not in s:
        s["plan"] = _plan(s)
    c, p, ctx = s["case"], s["plan"], _kept["ctx"]
    kind = c["kind"]
    if kind == "prompt":
        vkv.prompt_attend(ctx, p["prompt"], SCALE, p["out"], p["lse"])
        return {"out": p["out"], "lse": p["lse"]}
    if kind == "chunk":
        vkv.chunk_attend(ctx, p["pages"], p["chunk"], p["ws"], SCALE, p["out"], p["lse"])
        return {"out": p["out"], "lse": p["lse"]}
    if kind == "weights":
        vkv.weight_accumulate(ctx, p["pages"], p["chunk"], s["lse"], p["ws"], SCALE, 0.9, s["prev"], p["weight"])
        return {"weight": p["weight"]}
    if kind == "select":
        vkv.weight_select(ctx, s["weight"], s["kv_len"], c["T"], c["sinks"], c["recent"], p["kept"], p["count"])
        return {"kept": p["kept"], "count": p["count"]}
    vkv.cache_evict(ctx, p["pages"], s["kept"], s["count"], p["origin"], s["prev"], p["weight"])
    return {"cache": s["cache"], "origin": p["origin"], "weight": p["weight"]}


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "chunk": _plain_chunk, "weights": _plain_weights, "select": _plain_select,
            "evict": _plain_evict}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ the definition in 64 bits

def _rows_of(s, b, n):
    page = s["cache"].shape[1]
    return s["cache"][s["table"][b, :-(-n // page)].long()].reshape(-1, D_ROW)[:n].double()


def _exact_prompt(s):
    c = s["case"]
    out = torch.empty(s["q"].shape[0], c["H"], c["dv"], dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[0], c["H"], dtype=torch.float64, device=DEV)
    at = 0
    for n in s["lens"]:
        for h in range(c["H"]):
            g = h * c["Hk"] // c["H"]
            k = s["k"][at:at + n, g].double()
            if c["dr"]:
                k = torch.cat([k, s["k_rope"][at:at + n].double()], 1)
            for i in range(0, n, 4096):
                e = min(n, i + 4096)
                x = (s["q"][at + i:at + e, h].double() @ k[:e].T.contiguous()) * SCALE
                ahead = torch.arange(e, device=DEV)[None, :] > torch.arange(i, e, device=DEV)[:, None]
                x = x.masked_fill(ahead, -math.inf)
                lse[at + i:at + e, h] = torch.logsumexp(x, 1)
                out[at + i:at + e, h] = torch.exp(x - lse[at + i:at + e, h, None]) @ s["v"][at:at + e, g].double()
        at += n
    return {"out": out, "lse": lse}


def _exact_chunk(s, weights):
    c, H = s["case"], s["case"]["H"]
    n_tok = s["q_lat"].shape[0]
    out = torch.zeros(n_tok, H, D_LAT, dtype=torch.float64, device=DEV)
    lse = torch.zeros(n_tok, H, dtype=torch.float64, device=DEV)
    weight = s["prev"].double() if weights else None
    at = 0
    for b, (nq, n) in enumerate(zip(s["lens"], _kv_lens(c))):
        rows = _rows_of(s, b, n)
        if weights and nq:
            weight[b, :n - nq] *= 0.9
            weight[b, n - nq:n] = 0.0
        for i in range(0, nq, 32):
            e = min(nq, i + 32)
            q = torch.cat([s["q_lat"][at + i:at + e], s["q_rope"][at + i:at + e]], 2).double()
            x = (q.reshape(-1, D_ROW) @ rows.T.contiguous()).view(e - i, H, n) * SCALE
            seen = torch.arange(n, device=DEV)[None, :] <= (n - nq + torch.arange(i, e, device=DEV))[:, None]
            x = x.masked_fill(~seen[:, None, :], -math.inf)
            if weights:
                weight[b, :n] += torch.exp(x - s["lse"][at + i:at + e, :, None].double()).sum((0, 1))
                continue
            z = torch.logsumexp(x, 2)
            lse[at + i:at + e] = z
            out[at + i:at + e] = (torch.exp(x - z[..., None]).view(-1, n) @ rows[:, :D_LAT]).view(e - i, H, D_LAT)
        at += nq
    return {"weight": weight} if weights else {"out": out, "lse": lse}


def _exact_select(s):
    c = s["case"]
    kept = torch.full((c["B"], c["keep"]), -1, dtype=torch.int64)
    weight = s["weight"].cpu()
    for b, n in enumerate(_kv_lens(c)):
        if n <= c["keep"]:
            rows = list(range(n))
        else:
            always = [u for u in range(n) if u < c["sinks"] or u >= n - c["recent"]]
            others = weight[b, c["sinks"]:n - c["recent"]].numpy()
            order = np.lexsort((np.arange(len(others)), -others))[:c["keep"] - len(always)]
            rows = sorted(always + (order + c["sinks"]).tolist())
        kept[b, :len(rows)] = torch.tensor(rows)
    return {"kept": kept, "count": torch.tensor([min(n, c["keep"]) for n in _kv_lens(c)])}


def _exact_evict(s):
    c, K, page = s["case"], s["case"]["keep"], s["cache"].shape[1]
    cache = s["cache"].clone()
    origin = torch.full((c["B"], K), -1, dtype=torch.int64)
    weight = torch.zeros(c["B"], K, dtype=torch.float64)
    kept, count, table, prev = s["kept"].tolist(), s["count"].tolist(), s["table"].cpu(), s["prev"].cpu().double()
    for b in range(c["B"]):
        rows = kept[b][:count[b]]
        inside = {u for u in rows if u < count[b]}
        outside = iter(u for u in rows if u >= count[b])
        at = [j if j in inside else next(outside) for j in range(count[b])]
        u = torch.tensor(at)
        origin[b, :count[b]], weight[b, :count[b]] = u, prev[b, u]
        j = torch.arange(count[b])
        to, src = table[b, j // page].long(), table[b, u // page].long()
        cache[to.to(DEV), (j % page).to(DEV)] = s["cache"][src.to(DEV), (u % page).to(DEV)]
    return {"cache": cache.double(), "origin": origin, "weight": weight}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "prompt":
        return _exact_prompt(s)
    if kind in ("chunk", "weights"):
        return _exact_chunk(s, kind == "weights")
    return _exact_select(s) if kind == "select" else _exact_evict(s)
