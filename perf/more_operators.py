"""The 8-bit latent cache from its filling to its pages' life, as cases that can be timed and checked.

Rotary positions (`rope`), the write of new rows into a paged cache held in 8 bits (`write`), attention of
new tokens over it (`chunk8`), and its pages: sequences that become forks of others and take pages for their
next rows (`beams`), and used pages moved to the front (`compact`).  `own` says whether `run` calls
libvkv or computes the operator in its plain form, in 32 bits with elementary torch operations.  `exact` is
the definition in 64 bits, sequence by sequence.

A cache row is 640 bytes: 512 codes (8-bit floating point, 4 exponent and 3 fraction bits) and 64 bf16.
`block` consecutive rows of a page share the scale 2^(byte - 127) of their codes.
"""
import math

import torch

own = False

DEV = "cuda:0"
SCALE = 1.0 / math.sqrt(192.0)
D_LAT, D_ROPE, D_ROW, D_BYTES = 512, 64, 576, 640
TOP, BYTE_MIN, BYTE_MAX = 448.0, 63, 191
_kept = {}             # what a program keeps for the process: its libvkv context


def listed():
    return [
        # the branch queries of one decode step, far into long contexts; the launch is what counts
        dict(name="rope_decode", kind="rope", n=32, H=128, D=64, first=0, dims=64, inter=True, mode="parts", factor=32.0, T=131072, back=False),
        # the gradients of a prompt's queries on a shard of 16 heads, the last 64 of 192 dims rotated; an odd count of tokens
        dict(name="rope_16k_grad", kind="rope", n=16387, H=16, D=192, first=128, dims=64, inter=False, mode="base", factor=4.0, T=32768, back=True),
        # one new row of every sequence of a full batch
        dict(name="write_decode", kind="write", B=32, T=32768, low=20011, nq=1, page=64, block=16),
        # the rows of a chunk of prompts of different lengths
        dict(name="write_prefill", kind="write", B=4, T=16384, low=9001, nq=8192, page=64, block=16),
        # single-token decode of one sequence on a shard of 16 heads
        dict(name="chunk8_8k_decode", kind="chunk8", B=1, H=16, T=8192, low=8192, nq=1, page=16, block=16),
        # decode of a batch of long contexts on a shard of 16 heads
        dict(name="chunk8_64k_decode", kind="chunk8", B=16, H=16, T=65536, low=50021, nq=1, page=64, block=16),
        # decode of a full batch at full head count, contexts of different lengths
        dict(name="chunk8_32k_decode", kind="chunk8", B=32, H=128, T=32768, low=20011, nq=1, page=64, block=32),
        # chunked prefill: the next 512 tokens of three requests
        dict(name="chunk8_16k_prefill", kind="chunk8", B=3, H=128, T=16384, low=9001, nq=512, page=64, block=16),
        # four beams of one request change places before their next token
        dict(name="beams_2k", kind="beams", B=4, width=4, T=2048, low=1999, page=64, block=16, layers=1),
        # beams of a batch of requests, several layers on one table
        dict(name="beams_8k", kind="beams", B=64, width=4, T=8192, low=5003, page=64, block=16, layers=4),
        # a small pool of one layer: the launches are what counts
        dict(name="compact_2k", kind="compact", B=4, T=2048, low=1001, page=16, block=16, layers=1),
        # a pool with holes after many requests have ended
        dict(name="compact_16k", kind="compact", B=16, T=16384, low=3001, page=64, block=16, layers=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "write", "write", "chunk8", "chunk8", "chunk8", "beams", "compact"])
    if kind == "rope":
        dims = 2 * rng.randint(8, 64)
        first = rng.choice([0, 0, 64, 128])
        D = first + dims + rng.choice([0, 0, 64, 2 * rng.randint(1, 32)])
        H = _log(rng, 1, 128)
        n = _log(rng, 1, 16384)
        n = max(1, min(n, 16384 * 16 * 192 // (H * D)))
        return dict(kind=kind, n=n, H=H, D=D, first=first, dims=dims, inter=rng.random() < 0.5,
                    mode=rng.choice(["plain", "linear", "base", "parts"]), factor=rng.choice([1.5, 4.0, 32.0]),
                    T=_log(rng, 2048, 1 << 20), back=rng.random() < 0.3)
    page = 1 << rng.randint(4, 8)
    block = 1 << rng.randint(0, min(6, page.bit_length() - 1))
    if kind == "write":
        T = _log(rng, 2048, 65536)
        nq = rng.choice([1, 1, _log(rng, 2, T)])
        B = max(1, min(_log(rng, 1, 32), 32 * 32768 // T))
        nq = min(nq, max(1, 32768 // B))
        return dict(kind=kind, B=B, T=T, low=rng.randint(max(nq, T // 2), T), nq=nq, page=page, block=block)
    if kind == "chunk8":
        T = _log(rng, 2048, 65536)
        H, nq = _log(rng, 4, 128), rng.choice([1, 1, _log(rng, 2, 512)])
        B = max(1, min(_log(rng, 1, 32), 8 * 65536 // T))
        nq = max(1, min(nq, 3 * 512 * 128 * 11264 // (B * H * T)))
        return dict(kind=kind, B=B, H=H, T=T, low=rng.randint(max(nq, T // 2), T), nq=nq, page=page, block=block)
    layers = rng.choice([1, 2, 4])
    T = _log(rng, 1024, 16384)
    T = max(T, page)
    if kind == "beams":
        width = rng.choice([2, 3, 4, 8])
        requests = max(1, min(_log(rng, 1, 16), 16 * 8192 * 8 // (T * layers)))
        return dict(kind=kind, B=width * requests, width=width, T=T, low=rng.randint(T // 2, T), page=page, block=block, layers=layers)
    B = max(2, min(_log(rng, 2, 32), 16 * 16384 * 4 // (T * layers)))
    return dict(kind=kind, B=B, T=T, low=rng.randint(max(T // 8, 1), T), page=page, block=block, layers=layers)


def _lens(B, top, low):
    """B lengths in [low, top], the first one the longest."""
    return [top] + [low + int((top - low + 1) * ((b * 0.6180339887498949) % 1.0)) for b in range(1, B)]


def _kv_lens(case):
    if case["kind"] == "beams":      # the beams of a request are equally long
        lens = _lens(case["B"] // case["width"], case["T"], case["low"])
        return [n for n in lens for _ in range(case["width"])]
    return _lens(case["B"], case["T"], case["low"])


def _q_lens(case):
    """New tokens of each sequence: the chunk's size, and less of it in every third sequence."""
    return [case["nq"] if b % 3 != 2 else (case["nq"] + 1) // 2 for b in range(case["B"])]


def _starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def _page_bytes(case):
    return case["page"] * D_BYTES + case["page"] // case["block"]


def _beam_sources(case):
    """Which beam of its request each sequence goes on from: the first one survives most often."""
    w = case["width"]
    return [b - b % w + (b * b // w + b // 3) % w * (b % 2) for b in range(case["B"])]


def work(case):
    kind = case["kind"]
    if kind == "rope":
        return {"bytes": 4 * case["n"] * case["H"] * case["D"] + 4 * case["n"], "flops": 3 * case["n"] * case["H"] * case["dims"]}
    if kind == "write":
        n = sum(_q_lens(case))
        return {"bytes": n * (2 * D_ROW + D_BYTES) + n // case["block"], "flops": 2 * n * D_LAT}
    if kind == "chunk8":
        lens, new, H = _kv_lens(case), _q_lens(case), case["H"]
        rows, q = sum(lens), sum(new)
        pairs = sum(q_ * k - q_ * (q_ - 1) // 2 for q_, k in zip(new, lens))
        return {"bytes": D_BYTES * rows + -(-rows // case["block"]) + q * H * (2 * D_ROW + 2 * D_LAT + 4),
                "flops": 2 * (D_ROW + D_LAT) * H * pairs}
    lens, page = _kv_lens(case), case["page"]
    used = [-(-n // page) for n in lens]
    if kind == "beams":
        src = _beam_sources(case)
        moved = [b for b in range(case["B"]) if src[b] != b]
        holders = [src.count(s) for s in range(case["B"])]
        # every sequence that shares a last page that is not full copies it
        copies = sum(1 for b in range(case["B"]) if holders[src[b]] > 1 and lens[b] % page)
        return {"bytes": 2 * copies * case["layers"] * _page_bytes(case) + 8 * sum(used[b] for b in moved) + 8 * len(lens), "flops": 0}
    live = sum(used[0::2])
    pages = sum(used) + 3
    moved = live - live * live // pages          # used pages lie evenly over the pool
    return {"bytes": 2 * moved * case["layers"] * _page_bytes(case) + 4 * pages + 8 * moved, "flops": 0}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _latents(g, n):
    """Latent rows whose sizes differ from token to token."""
    x = torch.randn(n, D_LAT, generator=g, device=DEV)
    return (x * torch.exp(0.5 * torch.randn(n, 1, generator=g, device=DEV))).to(torch.bfloat16)


def _scale_bytes(amax):
    """The scale of each largest magnitude: 2^(byte - 127) is the least power with amax <= 448 * 2^(byte - 127)."""
    m, e = torch.frexp(amax.float())
    byte = torch.where(m <= 0.875, e - 9, e - 8) + 127
    return torch.where(amax > 0, byte, torch.zeros_like(byte)).clamp(BYTE_MIN, BYTE_MAX).to(torch.int32)


def _power(byte):
    return torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.to(torch.int32) - 127)


def _coded(x, byte):
    """Codes of x (32 bits) under the scales of byte, as bytes."""
    return (x / _power(byte)).to(torch.float8_e4m3fn).view(torch.uint8)


def _valued(codes, byte):
    return codes.view(torch.float8_e4m3fn).float() * _power(byte)


def _pages(g, case, s):
    """A paged 8-bit cache whose pages lie in any order, and the sequences' tables."""
    page, block, lens = case["page"], case["block"], _kv_lens(case)
    width = -(-max(lens) // page)
    used = [-(-n // page) for n in lens]
    total = sum(used) + 3
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device=DEV)
    s["cache"] = torch.zeros(total, page, D_BYTES, dtype=torch.uint8, device=DEV)
    s["scale"] = torch.full((total, page // block), 127, dtype=torch.uint8, device=DEV)
    at = 0
    for b, n in enumerate(used):
        where = order[at:at + n]
        table[b, :n] = where
        at += n
        x = _latents(g, n * page).float().view(n, page // block, block, D_LAT)
        byte = _scale_bytes(x.abs().amax((2, 3)))
        s["cache"][where.long(), :, :D_LAT] = _coded(x, byte[..., None, None]).view(n, page, D_LAT)
        s["cache"][where.long(), :, D_LAT:] = _normal(g, n, page, D_ROPE).view(torch.uint8)
        s["scale"][where.long()] = byte.to(torch.uint8)
    s["table"], s["kv_len"], s["max_kv"] = table, _i32(lens), max(lens)


def _pool(g, case, s):
    """A pool of pages of several layers: what lies in it does not matter to those who move it."""
    page, B, lens = case["page"], case["B"], _kv_lens(case)
    used = [-(-n // page) for n in lens]
    spare = 2 * B + 8 if case["kind"] == "beams" else 3
    total = sum(used) + spare
    width = -(-(max(lens) + 1) // page)
    s["cache"] = torch.randint(0, 256, (case["layers"], total, page, D_BYTES), generator=g, device=DEV, dtype=torch.uint8)
    s["scale"] = torch.randint(BYTE_MIN, BYTE_MAX + 1, (case["layers"], total, page // case["block"]), generator=g, device=DEV, dtype=torch.uint8)
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    s["refs"] = torch.zeros(total, dtype=torch.int32, device=DEV)
    live = range(B) if case["kind"] == "beams" else range(0, B, 2)    # of a pool with holes every second sequence has ended
    at = [0]
    for n in used:
        at.append(at[-1] + n)
    for b in live:
        s["table"][b, :used[b]] = order[at[b]:at[b + 1]]
        s["refs"][order[at[b]:at[b + 1]].long()] = 1
    s["kv_len"] = _i32([n if b in live else 0 for b, n in enumerate(lens)])


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    s = {"case": dict(case)}
    if kind == "rope":
        s["x"] = _normal(g, case["n"], case["H"], case["D"])
        s["pos"] = torch.randint(0, case["T"], (case["n"],), generator=g, device=DEV, dtype=torch.int32)
        return s
    if kind in ("write", "chunk8"):
        _pages(g, case, s)
        lens = _q_lens(case)
        n = sum(lens)
        s["lens"], s["cu"], s["max_q"] = lens, _i32(_starts(lens)), max(lens)
        if kind == "write":
            s["lat"], s["rope"] = _latents(g, n), _normal(g, n, D_ROPE)
        else:
            s["q_lat"], s["q_rope"] = _normal(g, n, case["H"], D_LAT), _normal(g, n, case["H"], D_ROPE)
        return s
    _pool(g, case, s)
    if kind == "beams":
        s["from"] = _i32(_beam_sources(case))
        s["want"] = s["kv_len"] + 1
    else:
        # the pool as it was found: a pass begins with it
        s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
    return s


# ------------------------------------------------------------------ the plain forms

def _frequencies(c):
    i = torch.arange(c["dims"] // 2, dtype=torch.float64, device=DEV)
    base = 10000.0
    if c["mode"] == "base":
        base *= c["factor"] ** (c["dims"] / (c["dims"] - 2.0))
    f = torch.exp(-2.0 * i / c["dims"] * math.log(base))
    if c["mode"] == "linear":
        f = f / c["factor"]
    if c["mode"] == "parts":      # turns over 4096 positions: at most 1 stretched, from 32 on as they were
        keep = ((4096.0 * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * ((1.0 - keep) / c["factor"] + keep)
    return f


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["mode"] == "parts" else 1.0


def _plain_rope(s):
    c = s["case"]
    at, dims = c["first"], c["dims"]
    angle = s["pos"].double()[:, None] * _frequencies(c)[None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if c["back"]:
        sin = -sin
    out = s["x"].clone()
    x = s["x"][..., at:at + dims].float()
    y = torch.empty_like(x)
    one, two = (slice(0, None, 2), slice(1, None, 2)) if c["inter"] else (slice(0, dims // 2), slice(dims // 2, None))
    m = _magnitude(c)
    y[..., one] = m * (x[..., one] * cos - x[..., two] * sin)
    y[..., two] = m * (x[..., two] * cos + x[..., one] * sin)
    out[..., at:at + dims] = y.to(torch.bfloat16)
    return {"out": out}


def _plain_write(s):
    page, R = s["cache"].shape[1], s["case"]["block"]
    cu, n = s["cu"].long(), s["lat"].shape[0]
    tok = torch.arange(n, device=DEV)
    b = (tok[:, None] >= cu[None, 1:]).sum(1)
    first = s["kv_len"].long() - (cu[1:] - cu[:-1])       # the row of each sequence's first new token
    u = first[b] + tok - cu[b]
    # the blocks that hold new rows: (sequence, block of the sequence), each once
    width = s["table"].shape[1] * (page // R)
    which = torch.unique(b * width + u // R)
    wb, wu = which // width, which % width * R
    rows = wu[:, None] + torch.arange(R, device=DEV)[None, :]
    new = (rows >= first[wb][:, None]) & (rows < s["kv_len"].long()[wb][:, None])
    old = rows < first[wb][:, None]
    source = (cu[wb][:, None] + rows - first[wb][:, None]).clamp(0, n - 1)
    p = s["table"][wb, wu // page].long()
    j = wu % page // R
    x = torch.where(new[..., None], s["lat"][source].float(), torch.zeros((), device=DEV))
    before = torch.where(old.any(1), s["scale"][p, j].to(torch.int32), torch.full_like(j, BYTE_MIN, dtype=torch.int32))
    byte = torch.maximum(_scale_bytes(x.abs().amax((1, 2))), before)
    in_page = rows % page
    codes = s["cache"][p[:, None], in_page, :D_LAT]
    again = _coded(_valued(codes, before[:, None, None]), byte[:, None, None])
    codes = torch.where(new[..., None], _coded(x, byte[:, None, None]), torch.where(old[..., None], again, codes))
    rope = torch.where(new[..., None], s["rope"].view(torch.uint8)[source], s["cache"][p[:, None], in_page, D_LAT:])
    s["cache"][p[:, None], in_page] = torch.cat([codes, rope], -1)
    s["scale"][p, j] = byte.to(torch.uint8)
    return _written(s)


def _written(s):
    return {"codes": s["cache"][..., :D_LAT].view(torch.float8_e4m3fn), "rope": s["cache"][..., D_LAT:].view(torch.bfloat16),
            "scale": s["scale"]}


def _padded(x, cu, n_max):
    """Packed rows [n, ...] -> [B, n_max, ...] in 32 bits (rows past a sequence's end repeat one of the tensor's)."""
    at = cu[:-1, None].long() + torch.arange(n_max, device=DEV)[None, :]
    return x[at.clamp(max=x.shape[0] - 1)].float()


def _packed(x, cu, n):
    """[B, n_max, ...] -> the packed rows [n, ...]."""
    tok = torch.arange(n, device=DEV)
    b = (tok[:, None] >= cu[None, 1:].long()).sum(1)
    return x[b, tok - cu.long()[b]]


def _plain_chunk8(s):
    c, Q, T, page = s["case"], s["max_q"], s["max_kv"], s["cache"].shape[1]
    B, H, n = c["B"], c["H"], s["q_lat"].shape[0]
    u = torch.arange(T, device=DEV)
    p = s["table"].long()[:, u // page].clamp(min=0)
    rows = s["cache"][p, u % page]
    byte = s["scale"][p, u % page // c["block"]]
    lat = _valued(rows[..., :D_LAT].contiguous(), byte[..., None])
    kv = torch.cat([lat, rows[..., D_LAT:].contiguous().view(torch.bfloat16).float()], -1)
    q = torch.cat([_padded(s["q_lat"], s["cu"], Q), _padded(s["q_rope"], s["cu"], Q)], -1)
    x = torch.bmm(q.view(B, Q * H, D_ROW), kv.transpose(1, 2)).mul_(SCALE).view(B, Q, H, T)
    nq = (s["cu"][1:] - s["cu"][:-1]).long()
    i = torch.arange(Q, device=DEV)
    last = s["kv_len"].long()[:, None] - nq[:, None] + i[None, :]
    visible = (u[None, None, :] <= last[:, :, None]) & (i[None, :] < nq[:, None])[:, :, None]
    x.masked_fill_(~visible[:, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.bmm(x.view(B, Q * H, T), lat).view(B, Q, H, D_LAT)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (m + torch.log(total)).squeeze(-1)
    return {"out": _packed(o, s["cu"], n).to(torch.bfloat16), "lse": _packed(lse, s["cu"], n)}


def _state(s, **more):
    return {"cache": s["cache"], "scale": s["scale"], "table": s["table"], "refs": s["refs"], "kv_len": s["kv_len"], **more}


def _plain_beams(s):
    table, refs, page = s["table"], s["refs"], s["cache"].shape[2]
    B, width = table.shape
    src, j = s["from"].long(), torch.arange(width, device=DEV)[None, :]
    stays = (src == torch.arange(B, device=DEV))[:, None]
    used = -(-s["kv_len"].long()[src] // page)
    now = torch.where(stays, table, torch.where(j < used[:, None], table[src], torch.full_like(table, -1)))
    spare = torch.zeros(refs.shape[0] + 1, dtype=torch.int32, device=DEV)      # the last place counts entries that name no page
    count = spare.index_add(0, torch.where(now >= 0, now, torch.full_like(now, refs.shape[0])).view(-1).long(),
                            torch.ones(B * width, dtype=torch.int32, device=DEV))[:-1]
    s["kv_len"].copy_(s["kv_len"][src])
    # pages for the next rows: lowest free page first, sequence by sequence, a shared last page's copy first
    at = s["kv_len"].long() // page
    last = now.gather(1, at[:, None].clamp(max=width - 1))[:, 0].long()
    copied = (s["kv_len"] % page != 0) & (s["want"] > s["kv_len"]) & (last >= 0) & (count[last.clamp(min=0)] > 1)
    more = (j >= at[:, None]) & (j < (-(-s["want"].long() // page))[:, None]) & (now < 0)
    need = more | ((j == at[:, None]) & copied[:, None])
    rank = torch.cumsum(need.view(-1).long(), 0).view(B, width) - 1
    free = (count == 0).nonzero()[:, 0]
    got = need & (rank < free.shape[0])
    page_of = free[rank.clamp(0, max(free.shape[0] - 1, 0))].to(torch.int32)
    to = page_of.gather(1, at[:, None].clamp(max=width - 1))[:, 0]
    mine = copied & got.gather(1, at[:, None].clamp(max=width - 1))[:, 0]
    old, fresh = last[mine], to[mine].long()
    s["cache"][:, fresh] = s["cache"][:, old]
    s["scale"][:, fresh] = s["scale"][:, old]
    one = torch.ones_like(old, dtype=torch.int32)
    count = count.index_add(0, old, -one)
    now = torch.where(got, page_of, now)
    count = count.index_add(0, now[got].long(), torch.ones_like(now[got]))
    table.copy_(now)
    refs.copy_(count)
    return _state(s, missing=(need & ~got).sum(1).to(torch.int32))


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    refs, table = s["refs"], s["table"]
    n = refs.shape[0]
    live = refs > 0
    used = live.sum()
    p = torch.arange(n, device=DEV)
    # the highest used page goes to the lowest free one
    source = (live & (p >= used)).nonzero()[:, 0].flip(0)
    hole = (~live & (p < used)).nonzero()[:, 0]
    s["cache"][:, hole] = s["cache"][:, source]
    s["scale"][:, hole] = s["scale"][:, source]
    to = p.clone()
    to[source] = hole
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table))
    refs[hole] = refs[source]
    refs[source] = 0
    return _state(s, used=used.to(torch.int32).view(1))


# ------------------------------------------------------------------ libvkv's calls

def _plan(s):
    """What a program keeps from pass to pass: the context, the descriptions of its tensors, workspace and outputs."""
    import paper_2609_03949_amd as vkv
    if "ctx" not in _kept:
        _kept["ctx"] = vkv.Context(0)
    c, kind, p = s["case"], s["case"]["kind"], {}
    if kind == "rope":
        scaling = {"plain": vkv.VKV_ROPE_PLAIN, "linear": vkv.VKV_ROPE_LINEAR, "base": vkv.VKV_ROPE_BASE,
                   "parts": vkv.VKV_ROPE_PARTS}[c["mode"]]
        p["rope"] = vkv.Rope(c["dims"], base=10000.0, interleaved=c["inter"], scaling=scaling, factor=c["factor"],
                             original=4096, fast=32.0, slow=1.0, magnitude=_magnitude(c))
        p["out"] = torch.empty_like(s["x"])
        return p
    if kind in ("write", "chunk8"):
        p["pages"] = vkv.Pages8(s["cache"], s["scale"], s["table"], s["kv_len"], s["max_kv"])
    if kind == "chunk8":
        n = s["q_lat"].shape[0]
        p["chunk"] = vkv.Chunk(s["q_lat"], s["q_rope"], s["cu"], s["max_q"])
        p["ws"] = torch.empty(vkv.chunk8_workspace_size(p["pages"], p["chunk"]), dtype=torch.uint8, device=DEV)
        p["out"] = torch.empty(n, c["H"], D_LAT, dtype=torch.bfloat16, device=DEV)
        p["lse"] = torch.empty(n, c["H"], device=DEV)
    if kind in ("beams", "compact"):
        p["pool"] = vkv.Pool(s["table"], s["kv_len"], s["refs"], c["page"], [s["cache"], s["scale"]])
        p["ws"] = torch.empty(vkv.pool_workspace_size(p["pool"]), dtype=torch.uint8, device=DEV)
        p["missing"] = torch.empty(c["B"], dtype=torch.int32, device=DEV)
        p["used"] = torch.empty(1, dtype=torch.int32, device=DEV)
    return p


def _own(s):
    import paper_2609_03949_amd as vkv
    if "plan" not in s:
        s["plan"] = _plan(s)
    c, p, ctx = s["case"], s["plan"], _kept["ctx"]
    kind = c["kind"]
    if kind == "rope":
        vkv.rope_apply(ctx, p["rope"], s["x"], s["pos"], p["out"], first=c["first"], transposed=c["back"])
        return {"out": p["out"]}
    if kind == "write":
        vkv.cache8_write(ctx, p["pages"], s["lat"], s["rope"], s["cu"], s["max_q"])
        return _written(s)
    if kind == "chunk8":
        vkv.chunk8_attend(ctx, p["pages"], p["chunk"], p["ws"], SCALE, p["out"], p["lse"])
        return {"out": p["out"], "lse": p["lse"]}
    if kind == "beams":
        vkv.pages_fork(ctx, p["pool"], s["from"], p["ws"])
        vkv.pages_reserve(ctx, p["pool"], s["want"], p["missing"], p["ws"])
        return _state(s, missing=p["missing"])
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    vkv.pages_compact(ctx, p["pool"], p["used"], p["ws"])
    return _state(s, used=p["used"])


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "write": _plain_write, "chunk8": _plain_chunk8, "beams": _plain_beams,
            "compact": _plain_compact}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_rope(s):
    c, half = s["case"], s["case"]["dims"] // 2
    out, pos = s["x"].double(), s["pos"].double()
    for i in range(half):
        base = 10000.0 if c["mode"] != "base" else 10000.0 * math.pow(c["factor"], c["dims"] / (c["dims"] - 2))
        f = math.pow(base, -2.0 * i / c["dims"])
        if c["mode"] == "linear":
            f /= c["factor"]
        if c["mode"] == "parts":
            turns = 4096.0 * f / (2.0 * math.pi)
            keep = 0.0 if turns < 1.0 else 1.0 if turns > 32.0 else (turns - 1.0) / 31.0
            f = (1.0 - keep) * f / c["factor"] + keep * f
        a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
        turn = torch.polar(torch.full_like(pos, _magnitude(c)), -pos * f if c["back"] else pos * f)[:, None]
        z = torch.complex(s["x"][..., c["first"] + a].double(), s["x"][..., c["first"] + b].double()) * turn
        out[..., c["first"] + a], out[..., c["first"] + b] = z.real, z.imag
    return {"out": out}


_E4M3 = sorted(v for e in range(16) for f in range(8)
               for v in [f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)] if v <= TOP)


def _nearest(x):
    """The nearest 8-bit value of each element (64 bits), halfway ones to the value of even code."""
    values = torch.tensor(_E4M3, dtype=torch.float64, device=DEV)
    hi = torch.searchsorted(values, x.abs()).clamp(max=len(_E4M3) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = x.abs() - values[lo], values[hi] - x.abs()
    down = (below < above) | ((below == above) & (lo % 2 == 0))
    return torch.copysign(torch.where(down, values[lo], values[hi]), x)


def _exact_write(s):
    c, page, R = s["case"], s["case"]["page"], s["case"]["block"]
    codes = s["cache"][..., :D_LAT].contiguous().view(torch.float8_e4m3fn).double()
    rope = s["cache"][..., D_LAT:].contiguous().view(torch.bfloat16).double()
    scale, table = s["scale"].to(torch.int64).cpu(), s["table"].cpu().tolist()
    at = 0
    for b, (nq, n) in enumerate(zip(s["lens"], _kv_lens(c))):
        x = s["lat"][at:at + nq].double()
        tops = x.abs().amax(1).cpu().tolist()
        u = n - nq
        while u < n:
            start, end = u - u % R, min(u - u % R + R, n)
            p, r = table[b][u // page], start % page
            top, byte = max(tops[u - (n - nq):end - (n - nq)]), BYTE_MIN
            while byte < BYTE_MAX and top > TOP * 2.0 ** (byte - 127):
                byte += 1
            if u > start:
                old = int(scale[p, r // R])
                if old < byte:
                    codes[p, r:r + u - start] = _nearest(codes[p, r:r + u - start] * 2.0 ** (old - byte))
                byte = max(byte, old)
            scale[p, r // R] = byte
            i = u - (n - nq)
            codes[p, u % page:u % page + end - u] = _nearest(x[i:i + end - u] * 2.0 ** (127 - byte))
            rope[p, u % page:u % page + end - u] = s["rope"][at + i:at + i + end - u].double()
            u = end
        at += nq
    return {"codes": codes, "rope": rope, "scale": scale}


def _exact_chunk8(s):
    c, H, page = s["case"], s["case"]["H"], s["case"]["page"]
    n_tok = s["q_lat"].shape[0]
    out = torch.zeros(n_tok, H, D_LAT, dtype=torch.float64, device=DEV)
    lse = torch.zeros(n_tok, H, dtype=torch.float64, device=DEV)
    at = 0
    for b, (nq, n) in enumerate(zip(s["lens"], _kv_lens(c))):
        p = s["table"][b, :-(-n // page)].long()
        raw = s["cache"][p]
        power = torch.pow(2.0, s["scale"][p].double() - 127.0).repeat_interleave(c["block"], 1)[..., None]
        lat = (raw[..., :D_LAT].contiguous().view(torch.float8_e4m3fn).double() * power).reshape(-1, D_LAT)[:n]
        rope = raw[..., D_LAT:].contiguous().view(torch.bfloat16).double().reshape(-1, D_ROPE)[:n]
        rows = torch.cat([lat, rope], 1).T.contiguous()
        for i in range(0, nq, 32):
            e = min(nq, i + 32)
            q = torch.cat([s["q_lat"][at + i:at + e], s["q_rope"][at + i:at + e]], 2).double()
            x = (q.reshape(-1, D_ROW) @ rows).view(e - i, H, n) * SCALE
            seen = torch.arange(n, device=DEV)[None, :] <= (n - nq + torch.arange(i, e, device=DEV))[:, None]
            x = x.masked_fill(~seen[:, None, :], -math.inf)
            z = torch.logsumexp(x, 2)
            lse[at + i:at + e] = z
            out[at + i:at + e] = (torch.exp(x - z[..., None]).view(-1, n) @ lat).view(e - i, H, D_LAT)
        at += nq
    return {"out": out, "lse": lse}


def _exact_beams(s):
    c, page = s["case"], s["case"]["page"]
    table, refs, lens = s["table"].cpu().tolist(), s["refs"].cpu().tolist(), s["kv_len"].cpu().tolist()
    src, want = s["from"].cpu().tolist(), s["want"].cpu().tolist()
    now, longer = [], []
    for b in range(c["B"]):
        held = -(-lens[src[b]] // page)
        now.append(list(table[b]) if src[b] == b else table[src[b]][:held] + [-1] * (len(table[b]) - held))
        longer.append(lens[src[b]])
    refs = [0] * len(refs)
    for row in now:
        for p in row:
            if p >= 0:
                refs[p] += 1
    free, shared = iter([p for p, r in enumerate(refs) if r == 0]), list(refs)
    pairs, missing = [], [0] * c["B"]
    for b in range(c["B"]):
        n = longer[b]
        for j in range(n // page, -(-want[b] // page)):
            held = now[b][j]
            if held >= 0 and not (j == n // page and n % page and shared[held] > 1):
                continue
            p = next(free, -1)
            if p < 0:
                missing[b] += 1
                continue
            if held >= 0:
                pairs.append((held, p))
                refs[held] -= 1
            now[b][j] = p
            refs[p] += 1
    cache, scale = s["cache"].clone(), s["scale"].clone()
    for a, p in pairs:
        cache[:, p], scale[:, p] = s["cache"][:, a], s["scale"][:, a]
    return {"cache": cache, "scale": scale, "table": torch.tensor(now), "refs": torch.tensor(refs),
            "kv_len": torch.tensor(longer), "missing": torch.tensor(missing)}


def _exact_compact(s):
    refs = s["refs"].cpu().tolist()
    used = sum(r > 0 for r in refs)
    holes = [p for p in range(used) if refs[p] == 0]
    to = {}
    for p in range(len(refs) - 1, used - 1, -1):
        if refs[p] > 0:
            to[p] = holes[len(to)]
    cache, scale = s["cache"].clone(), s["scale"].clone()
    for p, q in to.items():
        cache[:, q], scale[:, q] = s["cache"][:, p], s["scale"][:, p]
        refs[q], refs[p] = refs[p], 0
    table = [[to.get(p, p) for p in row] for row in s["table"].cpu().tolist()]
    return {"cache": cache, "scale": scale, "table": torch.tensor(table), "refs": torch.tensor(refs),
            "kv_len": s["kv_len"].cpu(), "used": torch.tensor([used])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "write": _exact_write, "chunk8": _exact_chunk8, "beams": _exact_beams,
            "compact": _exact_compact}[case["kind"]](s)
