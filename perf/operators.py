"""The operators over a caller's paged K/V cache, as cases that can be prepared, run in a plain form or on the library, and timed.

Four kinds of case:

``decode``
    One new token for every row of a batch: its K/V rows are written into the row's last slot and its queries attend over
    the row's slots, layer by layer.  With ``weights`` every slot also accumulates the attention it gets.
``append``
    The K/V rows of a ragged batch of prompts are written into their pages.
``evict``
    Rows that hold more than ``budget`` slots are cut to it: the first ``sink`` and the newest ``recent`` positions stay, and the
    slots of the largest accumulated weights.  The pass first puts back the weights and positions that the eviction moves
    (8 bytes a slot), so that every pass finds the same rows.
``step``
    What a bounded cache does for every token: ``decode`` with weights for each layer, then one eviction for all layers.
    The rows are at their budget, so every pass appends a slot and evicts one.

Pages are taken in random order, as in a cache that has served for a while.  ``lens`` is a rule of the case, everything else of
the seed.  A cache of type ``e4m3`` holds its rows in 8 bits with a scale per KV head; any other holds the queries' type.
"""
from __future__ import annotations

import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _case(name, kind, rows, context, hq, hkv, dim, page, dtype, cache=None, layers=1, layout="hnd", even=False, padded=False,
          weights=False, budget=0, sink=0, recent=0):
    c = dict(kind=kind, rows=rows, context=context, hq=hq, hkv=hkv, dim=dim, page=page, dtype=dtype, cache=cache or dtype,
             layers=layers, layout=layout, even=even, padded=padded, weights=weights, budget=budget, sink=sink, recent=recent)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token at the start of an answer, a narrow layer: latency alone
        _case("decode_300", "decode", 1, 300, 8, 2, 128, 16, "bf16"),
        # a small chat batch of ragged rows, two of its slots empty, half-width heads
        _case("decode_chat", "decode", 10, 1700, 32, 8, 64, 16, "fp16", padded=True),
        # one user's next token behind a long document: the cache's length is split over the GPU
        _case("decode_128k", "decode", 1, 131072, 32, 8, 128, 64, "bf16"),
        # the benchmark's batched decode, over its whole contexts
        _case("decode_16x24k", "decode", 16, 24576, 32, 8, 128, 16, "bf16", even=True),
        # a serving batch of ragged rows on 8-bit pages
        _case("decode_64_e4m3", "decode", 64, 8000, 32, 8, 128, 32, "bf16", cache="e4m3"),
        # every query head with a KV head of its own, wide heads, token-major pages of an odd size
        _case("decode_mha", "decode", 3, 10007, 8, 8, 256, 7, "fp16", layout="nhd"),
        # a batch whose slots accumulate their attention
        _case("decode_weights", "decode", 16, 5000, 32, 8, 128, 16, "bf16", weights=True),
        # prompts of a batch on their way into the pages
        _case("append_prompts", "append", 5, 16384, 32, 8, 128, 16, "bf16", padded=True),
        # short prompts into 8-bit pages, with weights and positions
        _case("append_e4m3", "append", 9, 500, 16, 4, 128, 32, "fp16", cache="e4m3", layout="nhd", weights=True),
        # a short row cut in half
        _case("evict_2k", "evict", 1, 2000, 8, 2, 64, 16, "fp16", weights=True, budget=1000, sink=16, recent=200),
        # prompts cut to a window of 4096 and the heaviest slots besides, all layers at once; two rows are short enough to stay
        _case("evict_prompts", "evict", 4, 32768, 32, 8, 128, 16, "bf16", layers=4, weights=True, budget=5120, sink=64,
              recent=4096),
        # a token of a batch that lives within its budget
        _case("step_budget", "step", 16, 4096, 32, 8, 128, 16, "bf16", layers=2, even=True, weights=True, budget=4096, sink=64,
              recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """Another case of the listed ones' ranges."""
    kind = rng.choice(["decode", "decode", "decode", "append", "evict", "step"])
    hq, hkv = rng.choice([(8, 2), (8, 8), (16, 4), (16, 8), (32, 8), (32, 8), (64, 8), (6, 2), (32, 2), (12, 12)])
    dim = rng.choice([64, 128, 128, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    cache = rng.choice([dtype, dtype, "e4m3"])
    page = rng.choice([1, 7, 16, 16, 32, 64, 100, 128])
    layout = rng.choice(["hnd", "nhd"])
    # slots of all rows and layers, so that a case costs no more than the largest listed one, in its plain form too
    room = (1 << 18) * 1024 // (max(hkv, hq // 4) * dim)
    layers = rng.choice([1, 1, 2, 4]) if kind in ("evict", "step") else 1
    context = _log_int(rng, 40, min(131072, room // layers))
    rows = _log_int(rng, 1, max(1, min(64, room // layers // context)))
    even, padded = rng.random() < 0.3, rng.random() < 0.3
    weights = kind in ("evict", "step") or rng.random() < 0.3
    budget = sink = recent = 0
    if kind in ("evict", "step"):
        budget = context if kind == "step" else max(8, int(context * rng.uniform(0.05, 0.9)))
        sink = rng.randint(0, min(64, budget // 4))
        recent = rng.randint(1, budget // 2)
        even, padded = even or kind == "step", padded and kind == "evict"
    return _case("", kind, rows, context, hq, hkv, dim, page, dtype, cache, layers, layout, even, padded, weights, budget, sink,
                 recent)


def _lens(case):
    """Slots of every row: the first has all of `context`, ragged ones spread over their logarithm, padded ones are empty."""
    rng = random.Random(case["rows"] * 65537 + case["context"])
    lens = [case["context"] if case["even"] or i == 0 else _log_int(rng, max(1, case["context"] / 30), case["context"])
            for i in range(case["rows"])]
    if case["padded"]:
        lens = [0 if i % 5 == 4 else n for i, n in enumerate(lens)]
    return lens


class State:
    pass


def _pages(case, n_pages, device):
    """Zeroed pages [layers][n_pages][Hkv][page][dim], in the order of the case's layout."""
    h, p = case["hkv"], case["page"]
    shape = (h, p) if case["layout"] == "hnd" else (p, h)
    t = torch.zeros((case["layers"], n_pages) + shape + (case["dim"],), dtype=torch.uint8 if case["cache"] == "e4m3"
                    else TYPES[case["cache"]], device=device)
    t = t if case["layout"] == "hnd" else t.transpose(2, 3)
    return t.view(TYPES["e4m3"]) if case["cache"] == "e4m3" else t


def _draw_rows(gen, shape, dtype, device, mean=None, spread=1.0):
    x = torch.randn(shape, generator=gen, device=device, dtype=torch.float32) * spread
    return (x if mean is None else x + mean).to(dtype)


def _prepare(case, seed, library):
    s = State()
    s.case = case
    dev = s.device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    L, hkv, dim, page = case["layers"], case["hkv"], case["dim"], case["page"]
    dtype = TYPES[case["dtype"]]
    held = _lens(case)
    extra = 1 if case["kind"] == "step" else 0  # the slot that a step appends and its eviction takes back
    need = [-(-(n + extra) // page) for n in held]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev)
    # entries behind a row's last page name a page that is nobody's
    table = order[-1].to(torch.int32).repeat(case["rows"], max(need)).contiguous()
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n].to(torch.int32)
        at += n
    s.table = table
    s.lens = torch.tensor([n + extra for n in held], dtype=torch.int32, device=dev)
    s.k, s.v = _pages(case, n_pages, dev), _pages(case, n_pages, dev)
    s.k_scale = s.v_scale = None
    if case["cache"] == "e4m3":
        s.k_scale = 0.012 + 0.01 * torch.rand(hkv, generator=gen, device=dev)
        s.v_scale = 0.012 + 0.01 * torch.rand(hkv, generator=gen, device=dev)
    # keys around a mean per layer and KV head, as a trained model's are; the cached rows are what an append left there
    mean = _draw_rows(gen, (L, 1, hkv, 1, dim), torch.float32, dev)
    for l in range(L):
        for pages, scale, m in ((s.k, s.k_scale, mean[l]), (s.v, s.v_scale, None)):
            for lo in range(0, n_pages, max(1, (1 << 27) // (hkv * page * dim))):
                part = pages[l, lo:lo + max(1, (1 << 27) // (hkv * page * dim))]
                x = _draw_rows(gen, part.shape, torch.float32, dev, m)
                part.copy_(_to_cache(case, x.to(dtype).float(), None if scale is None else scale[:, None, None]))
    s.weights = s.positions = None
    if case["weights"]:
        s.weights = torch.exp(1.5 * torch.randn((L, n_pages, hkv, page), generator=gen, device=dev))
        s.positions = torch.zeros((L, n_pages, hkv, page), dtype=torch.int32, device=dev)
        for r, n in enumerate(need):
            pos = torch.arange(n * page, dtype=torch.int32, device=dev).view(n, 1, page)
            s.positions[:, table[r, :n].long()] = pos.expand(n, hkv, page)
    rows = case["rows"]
    if case["kind"] in ("decode", "step"):
        # queries that lean on the mean of their KV head: logits with a spread of some units
        group = case["hq"] // hkv
        lean = mean[:, 0, :, 0].repeat_interleave(group, 1)
        s.q = [_draw_rows(gen, (rows, case["hq"], dim), dtype, dev, 0.3 * lean[l], 1.3) for l in range(L)]
        s.new_k = [_draw_rows(gen, (rows, hkv, dim), dtype, dev, mean[l, 0, :, 0]) for l in range(L)]
        s.new_v = [_draw_rows(gen, (rows, hkv, dim), dtype, dev) for l in range(L)]
        s.out = [torch.empty_like(q) for q in s.q]
        s.lse = [torch.empty((rows, case["hq"]), dtype=torch.float32, device=dev) for _ in range(L)]
        s.row_pos = (s.lens - 1).clone()
    if case["kind"] == "append":
        total = sum(held)
        s.starts = torch.tensor([sum(held[:i]) for i in range(rows + 1)], dtype=torch.int32, device=dev)
        s.new_k = _draw_rows(gen, (total, hkv, dim), dtype, dev, mean[0, :, :, 0])
        s.new_v = _draw_rows(gen, (total, hkv, dim), dtype, dev)
        s.row_pos = torch.zeros(rows, dtype=torch.int32, device=dev)
        s.new_w = torch.rand((total, hkv), generator=gen, device=dev) if case["weights"] else None
    if case["kind"] in ("evict", "step"):
        s.new_lens = torch.zeros_like(s.lens)
    if case["kind"] == "evict":
        s.weights0, s.positions0 = s.weights.clone(), s.positions.clone()
    if library:
        from paper_2412_04757_b200 import binding

        s.cache = binding.LtriPaged(s.k, s.v, n_q_heads=case["hq"], dtype=dtype, max_rows=rows,
                                    k_scale=s.k_scale, v_scale=s.v_scale, weights=s.weights, positions=s.positions)
    return s


def prepare(case, seed):
    return _prepare(case, seed, own)


# ---- plain forms ----------------------------------------------------------------------------------------------------


def _to_cache(case, x, scale):
    """fp32 rows as the cache holds them; `scale` is already shaped like the KV heads of x."""
    if scale is None:
        return x.to(TYPES[case["cache"]])
    return (x / scale).clamp(-448.0, 448.0).to(TYPES["e4m3"])


def _bits(t):
    """8-bit pages as whole numbers: indexing takes those."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _write_slots(pages, page, off, on, rows):
    """pages[page[i], :, off[i]] = rows[i] where on[i]."""
    pages, rows = _bits(pages), _bits(rows)
    old = pages[page, :, off]
    pages[page, :, off] = torch.where(on.view(-1, *[1] * (rows.dim() - 1)), rows, old)


def _plain_decode(s, l):
    case, P, hkv, dim = s.case, s.case["page"], s.case["hkv"], s.case["dim"]
    rows, G = case["rows"], case["hq"] // hkv
    # the new rows into their slots
    at = (s.lens - 1).clamp(min=0).long()
    on = s.lens > 0
    page = s.table.gather(1, (at // P)[:, None])[:, 0].long()
    for pages, new, scale in ((s.k[l], s.new_k[l], s.k_scale), (s.v[l], s.new_v[l], s.v_scale)):
        _write_slots(pages, page, at % P, on, _to_cache(case, new.float(), None if scale is None else scale[:, None]))
    # attention over each row's slots, all rows padded to the longest
    t = torch.arange(s.table.shape[1] * P, device=s.device)
    pg, off = s.table.long()[:, t // P], t % P
    seen = t[None] < s.lens[:, None]

    def held(pages, scale):
        x = _bits(pages)[pg, :, off].view(pages.dtype).float()
        x = torch.where(seen[:, :, None, None], x, 0.0)
        return (x if scale is None else x * scale[:, None]).transpose(1, 2)

    q = s.q[l].float().view(rows, hkv, G, dim)
    x = torch.matmul(q, held(s.k[l], s.k_scale).transpose(2, 3)) * dim ** -0.5
    x = torch.where(seen[:, None, None], x, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == float("-inf"), 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    s.out[l].copy_(torch.matmul(p, held(s.v[l], s.v_scale)).view(rows, -1, dim))
    s.lse[l].copy_((torch.where(total == 0, 0.0, top) + torch.log(total)).view(rows, -1))
    if s.weights is not None:
        w, pos = s.weights[l], s.positions[l]
        _write_slots(pos, page, at % P, on, s.row_pos[:, None].expand(rows, hkv))
        _write_slots(w, page, at % P, on, torch.zeros((rows, hkv), device=s.device))
        # (slots behind a row's end, whatever page the table names there, add a probability of zero)
        w.transpose(1, 2).index_put_((pg, off.expand_as(pg)), p.sum(2).transpose(1, 2), accumulate=True)


def _plain_append(s):
    case, P = s.case, s.case["page"]
    i = torch.arange(s.new_k.shape[0], device=s.device)
    row = torch.searchsorted(s.starts[1:].contiguous(), i.to(torch.int32), right=True)
    nth = i - s.starts[row]
    at = s.lens[row] - (s.starts[row + 1] - s.starts[row]) + nth
    page, off = s.table[row, at // P].long(), at % P
    for pages, new, scale in ((s.k[0], s.new_k, s.k_scale), (s.v[0], s.new_v, s.v_scale)):
        _bits(pages)[page, :, off] = _bits(_to_cache(case, new.float(), None if scale is None else scale[:, None]))
    if s.weights is not None:
        s.weights[0][page, :, off] = s.new_w
        s.positions[0][page, :, off] = (s.row_pos[row] + nth)[:, None].to(torch.int32).expand(-1, case["hkv"])


def _plain_evict(s):
    case, P, B = s.case, s.case["page"], s.case["budget"]
    T = s.table.shape[1] * P
    t = torch.arange(T, device=s.device)
    pg, off = s.table.long()[:, t // P], (t % P).expand(case["rows"], T)

    def slots(state):  # [layers][rows][Hkv][T]
        return state[:, pg, :, off].permute(2, 0, 3, 1)

    w, pos = slots(s.weights), slots(s.positions)
    live = (t[None] < s.lens[:, None])[None, :, None]
    newest = torch.where(live, pos, -1).amax(-1, keepdim=True)
    w = torch.where(torch.isnan(w), float("-inf"), w)
    stays = (pos < case["sink"]) | (pos > newest - case["recent"])
    # ranks: the slots that stay, then by weight, then those behind the row's end; equal ones by slot
    by_weight = torch.sort(w, dim=-1, descending=True, stable=True).indices
    group = torch.where(live, torch.where(stays, 0, 1), 2).gather(-1, by_weight)
    order = by_weight.gather(-1, torch.sort(group, dim=-1, stable=True).indices)
    kept = torch.zeros_like(live.expand_as(w)).scatter(-1, order[..., :B], True) & live
    cut = (s.lens > B)[None, :, None, None]
    mover, hole = kept & (t >= B) & cut, ~kept & (t < B) & cut
    src = torch.sort((~mover).to(torch.int8), dim=-1, stable=True).indices[..., :B]
    dst = torch.sort((~hole).to(torch.int8), dim=-1, stable=True).indices[..., :B]
    count = mover.sum(-1, keepdim=True)
    # entries of the lists behind the last move repeat the first one; where there is none, slot 0 is written to itself
    moves = torch.arange(src.shape[-1], device=s.device) < count
    src, dst = (torch.where(moves, x, torch.where(count > 0, x[..., :1], 0)) for x in (src, dst))
    r = torch.arange(case["rows"], device=s.device)[None, :, None, None]
    h = torch.arange(case["hkv"], device=s.device)[None, None, :, None]
    l = torch.arange(case["layers"], device=s.device)[:, None, None, None]
    table = s.table.long()
    for state in (_bits(s.k), _bits(s.v), s.weights, s.positions):
        state[l, table[r, dst // P], h, dst % P] = state[l, table[r, src // P], h, src % P]
    s.new_lens.copy_(s.lens.clamp(max=B))


# ---- one pass -------------------------------------------------------------------------------------------------------


def _updated(s):
    got = {"k": s.k, "v": s.v}
    if s.weights is not None:
        got["weights"], got["positions"] = s.weights, s.positions
    return got


def run(s):
    case = s.case
    kind = case["kind"]
    if kind == "append":
        if own:
            s.cache.ltri_paged_append(0, s.table, s.lens, s.starts, s.new_k, s.new_v, row_pos=s.row_pos, weights=s.new_w)
        else:
            _plain_append(s)
        return _updated(s)
    got = {}
    if kind in ("decode", "step"):
        for l in range(case["layers"]):
            if own:
                s.cache.ltri_paged_decode(l, s.table, s.lens, s.q[l], s.new_k[l], s.new_v[l], row_pos=s.row_pos, out=s.out[l],
                                          lse=s.lse[l])
            else:
                _plain_decode(s, l)
        got = {"out": s.out, "lse": s.lse}
    if kind == "evict":
        s.weights.copy_(s.weights0)
        s.positions.copy_(s.positions0)
    if kind in ("evict", "step"):
        if own:
            s.cache.ltri_paged_evict(0, case["layers"], s.table, s.lens, s.new_lens, case["budget"], case["sink"],
                                     case["recent"])
        else:
            _plain_evict(s)
        got["new_lens"] = s.new_lens
    if kind == "step":
        s.row_pos.add_(1)
    got.update(_updated(s))
    return got


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    lens = _lens(case)
    hq, hkv, dim, L, kind = case["hq"], case["hkv"], case["dim"], case["layers"], case["kind"]
    es = 1 if case["cache"] == "e4m3" else 2
    state = 8 if case["weights"] else 0  # a weight and a position
    byt = flo = 0.0
    if kind == "append":
        byt = sum(lens) * hkv * (2 * dim * (2 + es) + state + (4 if state else 0))
        return {"bytes": byt, "flops": 0.0}
    if kind in ("decode", "step"):
        for n in lens:
            n += kind == "step"
            if n:
                byt += (n - 1) * hkv * 2 * dim * es + 2 * (2 * hq + 2 * hkv) * dim + 2 * hkv * dim * es + 4 * hq
                byt += n * hkv * state  # every weight read and written
                flo += 4.0 * n * hq * dim
    if kind in ("evict", "step"):
        B, fixed = case["budget"], case["sink"] + case["recent"]
        for n in lens:
            n += kind == "step"
            if n > B:
                # the slots kept from behind the budget: the newest, and the heavy ones spread evenly
                late = min(case["recent"], n - B)
                moved = late + (B - fixed) * max(0, n - B - late) / max(1, n - fixed)
                byt += hkv * (8.0 * n + moved * 2 * (2 * dim * es + 8))
    return {"bytes": byt * L, "flops": flo * L}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _e4m3_nearest(x):
    """The e4m3 value nearest to every x (ties to the even one), both in 64 bits."""
    # 8 exponents' binades of 8 steps each from 2^-6, below it steps of 2^-9
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(a / step) * step, x)


def _exact_row(s, l, r, n):
    """K, V in 64 bits of row r's first n slots, [Hkv][n][dim]."""
    P = s.case["page"]
    got = []
    for pages, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
        x = torch.cat([pages[l, p].to(torch.float64) for p in s.table[r, :-(-n // P)].tolist()], 1)[:, :n]
        got.append(x if scale is None else x * scale.double()[:, None, None])
    return got


def _exact_decode(s, l, lens, got):
    case, hkv, dim = s.case, s.case["hkv"], s.case["dim"]
    G = case["hq"] // hkv
    out = torch.zeros((case["rows"], case["hq"], dim), dtype=torch.float64, device=s.device)
    lse = torch.full((case["rows"], case["hq"]), float("-inf"), dtype=torch.float64, device=s.device)
    weights = None if s.weights is None else s.weights[l].double()
    for r, n in enumerate(lens):
        if not n:
            continue
        K, V = _exact_row(s, l, r, n)
        for x, new, scale in ((K, s.new_k, s.k_scale), (V, s.new_v, s.v_scale)):
            row = new[l][r].double()
            x[:, n - 1] = row if scale is None else _e4m3_nearest(row / scale.double()[:, None]) * scale.double()[:, None]
        per_slot = []
        for h in range(hkv):
            x = (s.q[l][r, h * G:(h + 1) * G].double() @ K[h].T) / dim ** 0.5
            lse[r, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            p = torch.softmax(x, -1)
            out[r, h * G:(h + 1) * G] = p @ V[h]
            per_slot.append(p.sum(0))
        if weights is not None:
            P = case["page"]
            page = s.table[r, :-(-n // P)].long()
            idx = torch.arange(n, device=s.device)
            at = (page[idx // P], idx % P)
            w = weights.transpose(1, 2)
            w[at[0][-1], at[1][-1]] = 0.0
            w[at] = w[at] + torch.stack(per_slot, -1)
    got["out"].append(out)
    got["lse"].append(lse)
    got["weights"].append(weights)


def _exact_evict(case, table, lens, weights, positions, k, v):
    """Slot by slot of every unit, on the host's order: (weights, positions, k, v) after the eviction, new tensors."""
    P, B = case["page"], case["budget"]
    weights, positions = weights.clone(), positions.clone()
    k, v = k.clone(), v.clone()
    pages = table.tolist()
    for l in range(case["layers"]):
        for r, n in enumerate(lens):
            if n <= B:
                continue
            page = torch.tensor(pages[r], device=k.device)
            idx = torch.arange(n, device=k.device)
            pg, off = page[idx // P], idx % P
            for h in range(case["hkv"]):
                w, pos = weights[l, pg, h, off], positions[l, pg, h, off]
                top = int(pos.max())
                score = w.double().clone()
                score[(pos < case["sink"]) | (pos > top - case["recent"])] = float("inf")
                kept = set(sorted(range(n), key=lambda j, x=score.tolist(): (-x[j], j))[:B])
                src = torch.tensor([j for j in range(B, n) if j in kept], dtype=torch.long, device=k.device)
                dst = torch.tensor([j for j in range(B) if j not in kept], dtype=torch.long, device=k.device)
                for x in (_bits(k), _bits(v), weights, positions):
                    x[l, pg[dst], h, off[dst]] = x[l, pg[src], h, off[src]]
    return weights, positions, k, v


def exact(case, seed):
    s = _prepare(case, seed, False)
    kind, lens = case["kind"], _lens(case)
    if kind == "append":
        k, v = s.k[0].double(), s.v[0].double()
        w = None if s.weights is None else s.weights[0].double()
        first = 0
        for r, n in enumerate(lens):
            idx = torch.arange(n, device=s.device)
            page, off = s.table[r].long()[idx // case["page"]], idx % case["page"]
            for x, new, scale in ((k, s.new_k, s.k_scale), (v, s.new_v, s.v_scale)):
                rows = new[first:first + n].double()
                x[page, :, off] = rows if scale is None else _e4m3_nearest(rows / scale.double()[:, None])
            if w is not None:
                w[page, :, off] = s.new_w[first:first + n].double()
            first += n
        got = {"k": k[None], "v": v[None]}
        if w is not None:
            got["weights"], got["positions"] = w[None], None
        return got
    got = {"out": [], "lse": [], "weights": []}
    if kind == "decode":
        _exact_decode(s, 0, lens, got)
        got["weights"] = got["weights"][0]
        got["weights"] = None if got["weights"] is None else got["weights"][None]
        return {**got, "k": None, "v": None}
    if kind == "step":
        for l in range(case["layers"]):
            _exact_decode(s, l, [n + 1 for n in lens], got)
        return {"out": got["out"], "lse": got["lse"], "k": None, "v": None, "weights": None, "positions": None, "new_lens": None}
    if sum(lens) * case["layers"] * case["hkv"] > 4_000_000:
        return None
    w, pos, k, v = _exact_evict(case, s.table, lens, s.weights, s.positions, s.k, s.v)
    return {"k": k.double(), "v": v.double(), "weights": w.double(), "positions": None, "new_lens": None}
