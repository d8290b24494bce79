"""The operators of a paged K/V cache held in 4 bits, as cases that can be prepared, run in a plain form or on the library, and timed.

Four kinds of case:

``append``
    The K/V rows of a ragged batch of prompts are quantised into their pages, and the same tokens are read back as rows of the
    model's type.
``read``
    A range of every row's slots comes back as dense rows.
``decode``
    One new token's queries for every row of a batch attend over the row's slots.  With ``fresh`` the token's K/V rows are
    written into the row's last slot first, as a step does that has not appended them by itself, and are read back after it.
``attend``
    The queries of a ragged batch of prompts, or parts of prompts, whose rows are in the pages already attend over the row's
    slots up to their own.

A cached row is head_dim signed 4-bit numbers, -7 to 7, held as number + 8, the even element in the lower half of its byte, and a
scale for every 32 of them: 8 bits without a sign, 5 of exponent (bias 15) and 3 of mantissa, at most 480.  The scale is the one
nearest to the block's largest magnitude / 7, a number the nearest to element / scale (ties to even both).  The scales of a
slot's K row and V row stand together.  Pages are taken in random order, as in a cache that has served for a while.  ``lens`` is a
rule of the case, everything else of the seed.
"""
from __future__ import annotations

import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 32  # elements that share a scale


def _case(name, kind, rows, context, hq, hkv, dim, page, dtype, layout="hnd", even=False, padded=False, fresh=False, new=0):
    c = dict(kind=kind, rows=rows, context=context, hq=hq, hkv=hkv, dim=dim, page=page, dtype=dtype, layout=layout, even=even,
             padded=padded, fresh=fresh, new=new)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's short turn on its way into the pages
        _case("append_turn", "append", 1, 41, 8, 2, 128, 16, "bf16"),
        # prompts of a batch on their way into the pages
        _case("append_prompts", "append", 5, 16384, 32, 8, 128, 16, "bf16", padded=True),
        # a short row handed to a program that wants it dense, token-major pages of an odd size
        _case("read_700", "read", 1, 700, 16, 4, 64, 7, "fp16", layout="nhd"),
        # the prefixes of a batch, as a prompt's attention outside of the library reads them
        _case("read_prefixes", "read", 4, 32768, 32, 8, 128, 16, "bf16"),
        # one user's next token at the start of an answer, a narrow layer: latency alone
        _case("decode_300", "decode", 1, 300, 8, 2, 128, 16, "bf16"),
        # one user's next token behind a long document: the cache's length is split over the GPU
        _case("decode_128k", "decode", 1, 131072, 32, 8, 128, 64, "bf16"),
        # the benchmark's batched decode, over its whole contexts
        _case("decode_16x24k", "decode", 16, 24576, 32, 8, 128, 16, "bf16", even=True),
        # a serving batch of ragged rows, half-width heads, some of its slots empty, rows written by the step itself
        _case("decode_64", "decode", 64, 8000, 32, 8, 64, 32, "fp16", padded=True, fresh=True),
        # every query head with a KV head of its own, wide heads, token-major pages of an odd size
        _case("decode_mha", "decode", 3, 10007, 8, 8, 256, 7, "fp16", layout="nhd", fresh=True),
        # drafted tokens of a batch on their way through the model together
        _case("attend_drafts", "attend", 16, 8000, 32, 8, 128, 16, "bf16", new=5),
        # the benchmark's streamed chunk, over everything in front of it
        _case("attend_chunk", "attend", 1, 24576, 32, 8, 128, 16, "bf16", new=512),
        # whole prompts of a batch
        _case("attend_prompts", "attend", 3, 16384, 32, 8, 128, 64, "fp16", new=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """Another case of the listed ones' ranges."""
    kind = rng.choice(["append", "read", "decode", "decode", "decode", "attend", "attend"])
    hq, hkv = rng.choice([(8, 2), (8, 8), (16, 4), (16, 8), (32, 8), (32, 8), (64, 8), (6, 2), (32, 2), (12, 12)])
    dim = rng.choice([64, 128, 128, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([1, 7, 16, 16, 32, 64, 100, 128])
    layout = rng.choice(["hnd", "nhd"])
    # slots of all rows, so that a case costs no more than the largest listed one, in its plain form too
    room = (1 << 18) * 1024 // (max(hkv, hq // 4) * dim)
    context = _log_int(rng, 40, min(131072, room))
    rows = _log_int(rng, 1, max(1, min(64, room // context)))
    new = 0
    if kind == "attend":
        # (pairs of tokens and slots, at all heads, within those of the listed prompts)
        most = (1 << 39) // (hq * dim * context * rows)
        new = _log_int(rng, 1, max(1, min(context, most)))
    return _case("", kind, rows, context, hq, hkv, dim, page, dtype, layout, rng.random() < 0.3, rng.random() < 0.3,
                 kind == "decode" and rng.random() < 0.4, new)


def _lens(case):
    """Slots of every row: the first has all of `context`, ragged ones spread over their logarithm, padded ones are empty."""
    rng = random.Random(case["rows"] * 65537 + case["context"])
    lens = [case["context"] if case["even"] or i == 0 else _log_int(rng, max(1, case["context"] / 30), case["context"])
            for i in range(case["rows"])]
    if case["padded"]:
        lens = [0 if i % 5 == 4 else n for i, n in enumerate(lens)]
    return lens


def _tokens(case):
    """(first slot, tokens) of every row that a case writes, reads or attends for."""
    got = []
    for i, n in enumerate(_lens(case)):
        if case["kind"] == "attend":
            m = min(n, case["new"])
            got.append((n - m, m))
        elif case["kind"] == "decode":
            got.append((n - 1, 1) if n else (0, 0))
        elif case["kind"] == "read":
            got.append((n // 9, n - n // 9))  # (what lies in front was read before)
        else:
            got.append((0, n))
    return got


class State:
    pass


# ---- the format, in elementary operations ---------------------------------------------------------------------------


def _scale_of(byte):
    """fp32 scales that stand in the bytes: those are the upper half of a half-precision number without its sign."""
    return (byte.to(torch.int16) << 7).view(torch.float16).float()


def _quantise(x):
    """x [..., dim] -> (bytes [..., dim / 2], scales' bytes [..., dim / 32])."""
    # (64 bits: quotients next to a midpoint)
    y = x.double().unflatten(-1, (-1, BLOCK))
    s = y.abs().amax(-1) / 7.0
    step = torch.exp2(torch.floor(torch.log2(s.clamp(min=2.0 ** -14))) - 3)
    s = (torch.round(s / step) * step).clamp(max=480.0)
    n = torch.round(y / torch.where(s > 0, s, 1.0)[..., None]).clamp(-7, 7) * (s > 0)[..., None]
    n = (n + 8).to(torch.uint8).flatten(-2)
    return n[..., 0::2] | (n[..., 1::2] << 4), (s.to(torch.float16).view(torch.int16) >> 7).to(torch.uint8)


def _values(code, scale):
    """fp32 values of bytes [..., dim / 2] and scales' bytes [..., dim / 32]."""
    n = torch.stack([code & 15, code >> 4], -1).flatten(-2).float() - 8.0
    return (n.unflatten(-1, (-1, BLOCK)) * _scale_of(scale)[..., None]).flatten(-2)


# ---- states ---------------------------------------------------------------------------------------------------------


def _draw_rows(gen, shape, dtype, device, mean=None, spread=1.0):
    x = torch.randn(shape, generator=gen, device=device, dtype=torch.float32) * spread
    return (x if mean is None else x + mean).to(dtype)


def _prepare(case, seed, library):
    s = State()
    s.case = case
    dev = s.device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    hq, hkv, dim, page, kind = case["hq"], case["hkv"], case["dim"], case["page"], case["kind"]
    rows, dtype = case["rows"], TYPES[case["dtype"]]
    held = _lens(case)
    need = [-(-n // page) for n in held]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev)
    # entries behind a row's last page name a page that is nobody's
    table = order[-1].to(torch.int32).repeat(rows, max(need)).contiguous()
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n].to(torch.int32)
        at += n
    s.table = table
    s.lens = torch.tensor(held, dtype=torch.int32, device=dev)
    shape = (hkv, page) if case["layout"] == "hnd" else (page, hkv)
    s.k, s.v = (torch.zeros((1, n_pages) + shape + (dim // 2,), dtype=torch.uint8, device=dev) for _ in range(2))
    if case["layout"] == "nhd":
        s.k, s.v = s.k.transpose(2, 3), s.v.transpose(2, 3)
    s.scales = torch.zeros((1, n_pages, hkv, page, 2, dim // BLOCK), dtype=torch.uint8, device=dev)
    # keys around a mean per KV head with some wide channels, as a trained model's are; the cached rows are what an append left
    mean = _draw_rows(gen, (hkv, 1, dim), torch.float32, dev) * torch.exp(0.5 * _draw_rows(gen, (hkv, 1, dim), torch.float32, dev))
    few = max(1, (1 << 26) // (hkv * page * dim))
    if kind != "append":
        for lo in range(0, n_pages, few):
            for i, (pages, m) in enumerate(((s.k, mean), (s.v, None))):
                part = pages[0, lo:lo + few]
                x = _draw_rows(gen, part.shape[:-1] + (dim,), torch.float32, dev, m)
                code, scale = _quantise(x.to(dtype))
                part.copy_(code)
                s.scales[0, lo:lo + few, :, :, i] = scale
    took = _tokens(case)
    s.total = sum(n for _, n in took)
    s.starts = torch.tensor([sum(n for _, n in took[:i]) for i in range(rows + 1)], dtype=torch.int32, device=dev)
    s.first = torch.tensor([f for f, _ in took], dtype=torch.int32, device=dev)
    if kind == "append" or case["fresh"]:
        n = s.total if kind == "append" else rows
        s.new_k = _draw_rows(gen, (n, hkv, dim), dtype, dev, mean[:, 0])
        s.new_v = _draw_rows(gen, (n, hkv, dim), dtype, dev)
    if kind in ("append", "read") or case["fresh"]:
        s.back_k, s.back_v = (torch.zeros((s.total, hkv, dim), dtype=dtype, device=dev) for _ in range(2))
    if kind in ("decode", "attend"):
        # queries that lean on the mean of their KV head: logits with a spread of some units
        n = rows if kind == "decode" else s.total
        s.q = _draw_rows(gen, (n, hq, dim), dtype, dev, 0.3 * mean[:, 0].repeat_interleave(hq // hkv, 0), 1.3)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((n, hq), dtype=torch.float32, device=dev)
    if library:
        from paper_2412_04757_b200 import binding

        s.cache = binding.LtriPaged(s.k, s.v, n_q_heads=hq, dtype=dtype, max_rows=rows, block_scales=s.scales,
                                    max_tokens=s.total if kind == "attend" else 0)
    return s


def prepare(case, seed):
    return _prepare(case, seed, own)


# ---- plain forms ----------------------------------------------------------------------------------------------------


def _places(s):
    """(page, place) of every token that the case writes or reads, in their order."""
    i = torch.arange(s.total, device=s.device)
    row = torch.searchsorted(s.starts[1:].contiguous(), i.to(torch.int32), right=True)
    slot = s.first[row] + i - s.starts[row]
    return s.table[row, slot // s.case["page"]].long(), slot % s.case["page"]


def _plain_write(s, page, place, k, v):
    for i, (pages, new) in enumerate(((s.k, k), (s.v, v))):
        code, scale = _quantise(new)
        pages[0][page, :, place] = code
        s.scales[0][page, :, place, i] = scale


def _plain_read(s):
    page, place = _places(s)
    for i, (pages, back) in enumerate(((s.k, s.back_k), (s.v, s.back_v))):
        back.copy_(_values(pages[0][page, :, place], s.scales[0][page, :, place, i]))


def _held(s, r, n):
    """K, V in fp32 of row r's first n slots, [Hkv][n][dim]."""
    t = torch.arange(n, device=s.device)
    page, place = s.table[r].long()[t // s.case["page"]], t % s.case["page"]
    return [_values(pages[0][page, :, place], s.scales[0][page, :, place, i]).transpose(0, 1)
            for i, pages in enumerate((s.k, s.v))]


def _plain_attend(s):
    """Every token's queries over its row's slots up to its own; of a decode, one token a row."""
    case, hkv, dim = s.case, s.case["hkv"], s.case["dim"]
    G = case["hq"] // hkv
    decode = case["kind"] == "decode"
    if decode:
        s.out.zero_()
        s.lse.fill_(float("-inf"))
    at = 0
    for r, (n, (first, m)) in enumerate(zip(_lens(case), _tokens(case))):
        if not m:
            continue
        at = r if decode else at
        K, V = _held(s, r, n)
        few = max(1, (1 << 28) // (case["hq"] * n))
        for lo in range(0, m, few):
            hi = min(m, lo + few)
            seen = first + hi
            q = s.q[at + lo:at + hi].float().view(hi - lo, hkv, G, dim).permute(1, 2, 0, 3).reshape(hkv, -1, dim)
            x = torch.matmul(q, K[:, :seen].transpose(1, 2)).mul_(dim ** -0.5).view(hkv, G, hi - lo, seen)
            if hi - lo > 1:
                limit = first + lo + torch.arange(hi - lo, device=s.device)
                x.masked_fill_(torch.arange(seen, device=s.device) > limit[:, None], float("-inf"))
            top = x.amax(-1, keepdim=True)
            x.sub_(top).exp_()
            total = x.sum(-1, keepdim=True)
            o = torch.matmul(x.view(hkv, -1, seen), V[:, :seen]).view(hkv, G, hi - lo, dim) / total
            s.out[at + lo:at + hi] = o.permute(2, 0, 1, 3).reshape(hi - lo, -1, dim).to(s.out.dtype)
            s.lse[at + lo:at + hi] = (top + torch.log(total))[..., 0].permute(2, 0, 1).reshape(hi - lo, -1)
        at += m


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    case, kind = s.case, s.case["kind"]
    got = {}
    if kind == "append":
        if own:
            s.cache.ltri_paged_append(0, s.table, s.lens, s.starts, s.new_k, s.new_v)
        else:
            _plain_write(s, *_places(s), s.new_k, s.new_v)
    elif kind == "decode":
        if own:
            s.cache.ltri_paged_decode(0, s.table, s.lens, s.q, s.new_k if case["fresh"] else None,
                                      s.new_v if case["fresh"] else None, out=s.out, lse=s.lse)
        else:
            if case["fresh"]:
                on = s.lens > 0
                _plain_write(s, *_places(s), s.new_k[on], s.new_v[on])
            _plain_attend(s)
        got = {"out": s.out, "lse": s.lse}
    elif kind == "attend":
        if own:
            s.cache.ltri_paged_attend(0, s.table, s.lens, s.starts, s.q, out=s.out, lse=s.lse)
        else:
            _plain_attend(s)
        got = {"out": s.out, "lse": s.lse}
    if kind in ("append", "read") or case["fresh"]:
        if own:
            s.cache.ltri_paged_read(0, s.table, s.lens, s.starts, s.back_k, s.back_v, first=s.first)
        else:
            _plain_read(s)
        got["k"], got["v"] = s.back_k, s.back_v
    return got


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    hq, hkv, dim, kind = case["hq"], case["hkv"], case["dim"], case["kind"]
    held = hkv * (dim + 2 * dim // BLOCK)  # bytes of a slot's K and V
    dense = 2 * hkv * dim * 2
    byt = flo = 0.0
    for n, (first, m) in zip(_lens(case), _tokens(case)):
        if kind == "append":
            byt += m * (dense + held + dense)  # the rows read back are those just written
        elif kind == "read":
            byt += m * (held + dense)
        elif n:
            byt += n * held + m * (2 * hq * dim * 2 + 4 * hq)
            byt += (2 * dense + held) if case["fresh"] else 0
            flo += 4.0 * hq * dim * (m * first + m * (m + 1) / 2)
    return {"bytes": byt, "flops": flo}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _scales64(device):
    """Every scale there is, ascending: the byte's number is the position."""
    b = torch.arange(0xC0, device=device)
    e, f = b // 8, (b % 8).double()
    return torch.where(e == 0, f * 2.0 ** -17, (8 + f) * torch.exp2(e.double() - 18))


def _nearest(x, grid):
    """Number of the entry of an ascending grid nearest to every x; of two as near, the even one."""
    hi = torch.searchsorted(grid, x.contiguous()).clamp(1, len(grid) - 1)
    lo = hi - 1
    d = (grid[hi] - x) - (x - grid[lo])
    return torch.where((d < 0) | ((d == 0) & (hi % 2 == 0)), hi, lo)


def _exact_rows(x):
    """The values that rows [..., dim] are held as, in 64 bits, a piece at a time."""
    grid = _scales64(x.device)
    got = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    flat, to = x.reshape(-1, BLOCK), got.view(-1, BLOCK)
    for lo in range(0, flat.shape[0], 1 << 21):
        y = flat[lo:lo + (1 << 21)].double()
        s = grid[_nearest(y.abs().max(-1).values / 7, grid)][:, None]
        n = _half_even(y / s.clamp(min=2.0 ** -30)).clamp(-7, 7)
        to[lo:lo + (1 << 21)] = torch.where(s > 0, n * s, 0.0)
    return got


def _half_even(y):
    """The whole number nearest to every y, of two as near the even one."""
    down = torch.floor(y)
    d = y - down
    up = (d > 0.5) | ((d == 0.5) & (torch.remainder(down, 2) == 1))
    return down + up.double()


def _exact_held(s, which, r, n):
    """K (0) or V (1) of row r's first n slots in 64 bits, [Hkv][n][dim]."""
    pages, P = (s.k, s.v)[which][0], s.case["page"]
    grid = torch.cat([_scales64(s.device), torch.full((0x40,), float("nan"), dtype=torch.float64, device=s.device)])
    number = torch.arange(16, device=s.device).double() - 8
    got = []
    for p in s.table[r, :-(-n // P)].tolist():
        byte = pages[p].long()
        two = torch.stack([number[byte % 16], number[byte // 16]], -1).reshape(byte.shape[:-1] + (s.case["dim"],))
        scale = grid[s.scales[0, p, :, :, which].long()].repeat_interleave(BLOCK, -1)
        got.append(two * scale)
    return torch.cat(got, 1)[:, :n]


def exact(case, seed):
    if sum(-(-n // case["page"]) for n in _lens(case)) > 30000:
        return None
    s = _prepare(case, seed, False)
    kind, hkv, dim = case["kind"], case["hkv"], case["dim"]
    G = case["hq"] // hkv
    if kind == "append":
        return {"k": _exact_rows(s.new_k), "v": _exact_rows(s.new_v)}
    rows = list(zip(_lens(case), _tokens(case)))
    got = {}
    if kind == "read":
        for which, name in ((0, "k"), (1, "v")):
            got[name] = torch.cat([_exact_held(s, which, r, n)[:, f:f + m].transpose(0, 1) for r, (n, (f, m)) in enumerate(rows)
                                   if m])
        return got
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=s.device)
    lse = torch.full(s.lse.shape, float("-inf"), dtype=torch.float64, device=s.device)
    fresh = [_exact_rows(x) for x in (s.new_k, s.new_v)] if case["fresh"] else None
    at = 0
    for r, (n, (first, m)) in enumerate(rows):
        if not m:
            continue
        base = r if kind == "decode" else at
        K, V = _exact_held(s, 0, r, n), _exact_held(s, 1, r, n)
        if fresh:
            K[:, n - 1], V[:, n - 1] = fresh[0][r], fresh[1][r]
        few = max(1, (1 << 27) // n)
        for h in range(case["hq"]):
            for lo in range(0, m, few):
                hi = min(m, lo + few)
                x = s.q[base + lo:base + hi, h].double() @ K[h // G].T / dim ** 0.5
                own_slot = first + torch.arange(lo, hi, device=s.device)
                x = torch.where(torch.arange(n, device=s.device) <= own_slot[:, None], x, float("-inf"))
                lse[base + lo:base + hi, h] = torch.logsumexp(x, -1)
                out[base + lo:base + hi, h] = torch.softmax(x, -1) @ V[h // G]
        at += m
    got = {"out": out, "lse": lse}
    if fresh:
        # (a batch's empty rows have no token)
        on = torch.tensor([n > 0 for n, _ in rows], device=s.device)
        got["k"], got["v"] = fresh[0][on], fresh[1][on]
    return got
