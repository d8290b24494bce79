"""Attention of several new tokens per row over the paged cache on the GPU against its definition in 64 bits.

Tolerances are worst-case bounds of the arithmetic, per element, as for single tokens: a logit is off by d, at most (D + 8) units of
2^-23 of c sum_i |q_i K_i|; probabilities by exp(2 d), 2^-21 of exp2 and (n + 16) 2^-23 of a sum that truncates; they meet V as two
terms of 8 bits or more each, 2^-17, or, where bf16 outputs come of 8-bit or 4-bit pages, as one half, 2^-11, and halves end 2^-35
below the row's largest; the output is rounded once."""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_int4_reference as i4
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
KINDS = ["bf16", "fp16", "e4m3-bf16", "e4m3-fp16", "int4-bf16", "int4-fp16"]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(kind, lens, hq, hkv, dim, page, **kw):
    dtype = FP16 if kind.endswith("fp16") else BF16
    if kind.startswith("int4"):
        return i4.Cache(lens, hq, hkv, dim, page, dtype, **kw)
    return ref.Cache(lens, hq, hkv, dim, page, dtype, kind.startswith("e4m3"), **kw)


def starts_of(news, first=0):
    return [first + sum(news[:i]) for i in range(len(news) + 1)]


def check(c, l, q, out, lse, news, starts, scale=None, absent=()):
    """Every token's outputs against its row's slots as they are (absent: slots of row 0 without a page)."""
    scale = c.dim ** -0.5 if scale is None else scale
    half, tiny = ref.HALF_STEP[c.dtype], torch.finfo(c.dtype).smallest_normal * torch.finfo(c.dtype).eps
    errors, sizes = 0.0, 0.0
    term = 2.0 ** -11 if c.dtype == BF16 and c.k.element_size() == 1 else 2.0 ** -17
    for r, (n, m) in enumerate(zip(c.lens_cpu, news)):
        if not m:
            continue
        K, V = (x.cuda() for x in c.row(l, r, n))
        x = q[starts[r]:starts[r] + m].double()
        seen = torch.arange(n, device="cuda") <= (n - m + torch.arange(m, device="cuda"))[:, None]
        if r == 0 and len(absent):
            seen[:, list(absent)] = False
            K, V = K.clone(), V.clone()
            K[list(absent)], V[list(absent)] = 0.0, 0.0
        for h in range(c.hq):
            k, v, qh = K[:, h // c.G], V[:, h // c.G], x[:, h]
            logits = torch.where(seen, qh @ k.T * scale, -math.inf)
            p = torch.softmax(logits, -1)
            want, want_lse = p @ v, torch.logsumexp(logits, -1)
            d = (qh.abs() @ k.abs().T).amax(-1) * scale * (c.dim + 8) * 2.0 ** -23
            sums = (n + 16) * 2.0 ** -23 + 2.0 ** -21
            rel = torch.expm1(2 * d) + sums
            tol = (rel + term)[:, None] * (p @ v.abs()) + ((1 + rel) * p.amax(-1) * 2.0 ** -35)[:, None] * v.abs().sum(0)
            got, got_lse = out[starts[r]:starts[r] + m, h].double(), lse[starts[r]:starts[r] + m, h].double()
            bad = (got - want).abs() - (want.abs() * half + tol * (1 + half) + tiny)
            where = bad.isnan() | (bad > 0)
            assert not where.any(), (f"row {r} of {n}, head {h}: {int(where.sum())} of {where.numel()} elements, first at "
                                     f"{where.nonzero()[0].tolist()}: {got[where][:4].tolist()}, not {want[where][:4].tolist()}")
            bad = (got_lse - want_lse).abs() - (d + sums + want_lse.abs() * 2.0 ** -22)
            assert (bad <= 0).all(), f"row {r} of {n}, head {h}: lse off by {float((got_lse - want_lse).abs().max())}"
            errors, sizes = errors + float((got - want).square().sum()), sizes + float(want.square().sum())
    # all together: half a step, and what is off at random besides far below it where logits are a few units
    if scale == c.dim ** -0.5 and sizes and float(q.float().abs().max()) < 10:
        assert errors ** 0.5 <= (half + 2.0 ** -16 + term) * sizes ** 0.5


def attend(c, news, lp=None, q=None, l=0, q_scale=1.0, scale=None, first=0, behind=0):
    total = sum(news) + first + behind
    lp = lp or c.handle(max_tokens=max(1, total), **({} if scale is None else dict(softmax_scale=scale)))
    q = c.randn(total, c.hq, c.dim, scale=q_scale) if q is None else q
    starts = starts_of(news, first)
    lse = torch.full((total, c.hq), 7.0, device="cuda")
    out = torch.full_like(q, 5.0) if q.is_contiguous() else None
    out = lp.ltri_paged_attend(l, c.table, c.lens(), ints(starts), q, out=out, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for side in (slice(0, first), slice(total - behind, total)):
        assert (out[side] == 5.0).all() and (lse[side] == 7.0).all()
    check(c, l, q, out, lse, news, starts, scale)
    return out, lse


# lengths and tokens at which tiles, blocks of queries and pages begin and end
EDGES = [(1, 1), (0, 0), (5, 5), (130, 130), (300, 7), (129, 1), (64, 64), (40, 0), (257, 100), (128, 128), (65, 2), (200, 65)]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout,page", [("hnd", 16), ("nhd", 7), ("both", 1)])
def test_attend_at_the_edges(dim, kind, layout, page):
    c = make(kind, [n for n, _ in EDGES], 8, 2, dim, page, layout=layout, layers=2, seed=dim + page)
    c.fill()
    before = c.snapshot()
    attend(c, [m for _, m in EDGES], l=1, first=3, behind=2)
    assert all(torch.equal(x, before[name]) for name, x in c.snapshot().items())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (16, 1), (32, 2), (24, 1), (64, 1), (9, 1)])
@pytest.mark.parametrize("kind,dim", [("int4-bf16", 128), ("bf16", 64), ("int4-fp16", 256)])
def test_attend_of_every_group_size(hq, hkv, kind, dim):
    c = make(kind, [200, 0, 17, 1, 90], hq, hkv, dim, 16, seed=hq)
    c.fill()
    attend(c, [61, 0, 17, 1, 2])


@pytest.mark.parametrize("kind,rows,n,m,hq,hkv,dim", [
    ("int4-bf16", 1, 20011, 3, 8, 2, 128), ("int4-bf16", 1, 9001, 700, 8, 2, 128), ("int4-fp16", 3, 7000, 40, 8, 8, 64),
    ("int4-bf16", 2, 5000, 300, 6, 2, 256), ("bf16", 1, 12000, 500, 4, 1, 128), ("fp16", 40, 1200, 33, 8, 4, 128),
    ("e4m3-bf16", 2, 6000, 1000, 4, 1, 64), ("bf16", 16, 3000, 5, 32, 8, 128), ("int4-bf16", 1, 3000, 3000, 16, 4, 128),
    ("bf16", 1, 2500, 2500, 4, 1, 256), ("int4-bf16", 300, 60, 9, 4, 2, 64)])
def test_attend_split_over_ctas(kind, rows, n, m, hq, hkv, dim):
    lens = [max(1, n - 977 * i % n) if i % 7 != 5 else 0 for i in range(rows)]
    news = [min(x, max(0, m - i % 3)) for i, x in enumerate(lens)]
    c = make(kind, lens, hq, hkv, dim, 64, seed=rows)
    c.fill()
    lp = c.handle(max_tokens=sum(news))
    q = c.randn(sum(news), hq, dim)
    first = [x.clone() for x in attend(c, news, lp, q)]
    # the same inputs, the same bits
    for _ in range(3):
        again = attend(c, news, lp, q)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


@pytest.mark.parametrize("kind,dim", [("int4-bf16", 64), ("int4-bf16", 128), ("bf16", 128), ("e4m3-fp16", 64), ("int4-fp16", 256)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (12, 12), (32, 2)])
def test_attend_of_few_and_many_tokens_together(kind, dim, hq, hkv):
    # units of one tile of query rows and of two in turn, whole and in parts, of every number of tiles up to a dozen
    news = [1, 70, 5, 8, 300, 2, 9, 130, 3, 16, 1, 40, 7]
    lens = [511, 700, 512, 513, 1200, 640, 641, 1300, 1500, 90, 1409, 600, 769]
    c = make(kind, lens, hq, hkv, dim, 32, seed=dim + hq)
    c.fill()
    lp = c.handle(max_tokens=sum(news))
    q = c.randn(sum(news), hq, dim)
    first = [x.clone() for x in attend(c, news, lp, q)]
    again = attend(c, news, lp, q)
    assert all(torch.equal(x, y) for x, y in zip(first, again))


@pytest.mark.parametrize("kind,dim", [("fp16", 64), ("int4-fp16", 128), ("e4m3-fp16", 256)])
def test_sums_of_many_slots_do_not_fall_behind(kind, dim):
    # The tensor cores' sums are cut off towards zero: k additions take k / 2 times 2^-24 of a sum that grows evenly (half of the
    # last place, which is 2^-23 of it at the most), and as much again where products lose their own last places beside the sum.
    # Two for each 16 slots of up to 2^13: 2^-14 on the average, which values of one sign show.  The outputs' roundings do not
    # average out, since all outputs lie within a few of their steps of 1: they are known from the exact values, and taken out.
    n, m, hq, hkv = 100000, 600, 16, 4
    c = make(kind, [n], hq, hkv, dim, 128, seed=dim)
    pg, off = c.places(0, n)
    K, V = torch.randn(n, hkv, dim, generator=c.g), torch.rand(n, hkv, dim, generator=c.g) + 0.5
    if kind.startswith("int4"):
        c.store(0, pg, off, 0, K)
        c.store(0, pg, off, 1, V)
    else:
        ref.put(c.k[0], pg, off, K.to(c.k.dtype))
        ref.put(c.v[0], pg, off, V.to(c.v.dtype))
    lp, q = c.handle(max_tokens=m), c.randn(m, hq, dim, scale=0.5)
    lse = torch.empty(m, hq, device="cuda")
    out = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, m]), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    K, V = (x.cuda() for x in c.row(0, 0, n))
    seen = torch.arange(n, device="cuda") <= (n - m + torch.arange(m, device="cuda"))[:, None]
    for h in (0, 7, 13):
        logits = torch.where(seen, q[:, h].double() @ K[:, h // 4].T * dim ** -0.5, -math.inf)
        want = torch.softmax(logits, -1) @ V[:, h // 4]
        assert abs(float(((out[:, h].double() - want.to(c.dtype).double()) / want).mean())) <= 2.0 ** -14
        assert (lse[:, h].double() - torch.logsumexp(logits, -1)).abs().max() <= 1e-4


def test_parts_of_more_slots_than_a_bf16_sum_takes():
    # 40 units of 300000 slots: the CTAs' parts have some 80000, which O adds up in stretches of 2^16 at most
    n, m = 300000, 600
    c = make("bf16", [n], 16, 4, 64, 128, seed=33)
    pg, off = c.places(0, n)
    g = torch.Generator(device="cuda").manual_seed(34)
    for pages in (c.k, c.v):
        ref.put(pages[0], pg, off, torch.randn(n, 4, 64, generator=g, device="cuda").to(BF16).cpu())
    lp, q = c.handle(max_tokens=m), c.randn(m, 16, 64, scale=3.0)
    lse = torch.empty(m, 16, device="cuda")
    out = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, m]), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    K, V = (x.cuda() for x in c.row(0, 0, n))
    which = torch.arange(0, m, 12, device="cuda")
    seen = torch.arange(n, device="cuda") <= (n - m + which)[:, None]
    for h in (0, 6, 13):
        k, v, qh = K[:, h // 4], V[:, h // 4], q[which, h].double()
        logits = torch.where(seen, qh @ k.T / 8, -math.inf)
        p = torch.softmax(logits, -1)
        want = p @ v
        # (as above; the sums of a stretch lose 2^-11 of what they add up)
        d = (qh.abs() @ k.abs().T).amax(-1) / 8 * (64 + 8) * 2.0 ** -23
        tol = (torch.expm1(2 * d) + 2.0 ** -21 + 2.0 ** -17 + 2.0 ** -10)[:, None] * (p @ v.abs())
        assert ((out[which, h].double() - want).abs() <= want.abs() * 2.0 ** -8 + tol).all()
        assert ((lse[which, h].double() - torch.logsumexp(logits, -1)).abs() <= d + 1e-4).all()


@pytest.mark.parametrize("q_scale", [1.0, 4.0])
def test_long_units_within_one_cta(q_scale):
    # (more units than CTAs, each longer than what O adds up at a time)
    c = make("fp16", [10100] * 10, 16, 16, 64, 128, seed=31)
    c.fill()
    attend(c, [2, 1, 0, 2, 3, 1, 1, 2, 1, 5], q_scale=q_scale)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q_scale,scale", [(30.0, 0.05), (2.0 ** -9, 40.0)])
def test_attend_of_large_and_small_queries(kind, q_scale, scale):
    c = make(kind, [77, 500], 8, 2, 128, 16, seed=4)
    c.fill()
    attend(c, [40, 20], q_scale=q_scale, scale=float(torch.tensor(scale)))


@pytest.mark.parametrize("q_scale", [2.0 ** 60, 2.0 ** -60])
@pytest.mark.parametrize("kind", ["bf16", "e4m3-bf16", "int4-bf16"])
def test_attend_of_queries_of_any_magnitude(kind, q_scale):
    c = make(kind, [77, 300], 8, 2, 128, 16, seed=6)
    c.fill()
    attend(c, [3, 100], q_scale=q_scale, scale=float(torch.tensor(0.088 / q_scale)))


@pytest.mark.parametrize("kind", ["bf16", "int4-bf16", "int4-fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_where_every_tile_raises_the_reference(kind, dim):
    # logits that grow along the row, 15 a tile of 64 slots: the sums so far are rescaled in every tile, by 2^-20 and more
    n = 700
    c = make(kind, [n], 4, 2, dim, 16, seed=dim)
    c.fill(0.05)
    pg, off = c.places(0, n)
    K = torch.randn(n, 2, dim, generator=c.g) * 0.05
    K[:, :, 0] = torch.arange(n)[:, None] / 64 * 0.25
    if kind.startswith("int4"):
        c.store(0, pg, off, 0, K)
    else:
        ref.put(c.k[0], pg, off, K.to(c.k.dtype))
    q = c.randn(300, 4, dim)
    q[:, :, 0] = 60.0
    attend(c, [300], q=q, scale=1.0)


def test_attend_writes_over_dense_queries_and_reads_strided_ones():
    c = make("int4-bf16", [150, 400], 8, 2, 128, 16, seed=12)
    c.fill()
    news = [90, 130]
    lp, wide = c.handle(max_tokens=220), c.randn(220, 12, 128)
    out, _ = attend(c, news, lp, wide[:, :8])
    dense = wide[:, :8].contiguous()
    assert torch.equal(lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 90, 220]), dense, out=dense), out)


def test_attend_agrees_with_single_tokens():
    for kind in KINDS:
        c = make(kind, [300, 1, 0, 77], 8, 2, 128, 16, seed=13)
        c.fill()
        lp = c.handle(max_tokens=3)
        q = c.randn(4, 8, 128)
        some = q[[0, 1, 3]].contiguous()
        lse, lse1 = torch.empty(3, 8, device="cuda"), torch.empty(4, 8, device="cuda")
        out = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 1, 2, 2, 3]), some, lse=lse)
        one = lp.ltri_paged_decode(0, c.table, c.lens(), q, lse=lse1)[[0, 1, 3]]
        assert ((out.float() - one.float()).abs() <= one.float().abs() * 2 * ref.HALF_STEP[c.dtype] + 1e-3).all()
        assert ((lse - lse1[[0, 1, 3]]).abs() < 1e-4).all()


def test_bad_pages_are_absent_and_recorded():
    for kind in ("bf16", "e4m3-fp16", "int4-bf16"):
        for dim in (128, 256):
            c = make(kind, [150, 60], 4, 2, dim, 16, seed=11)
            c.fill()
            lp, q = c.handle(max_tokens=80), c.randn(80, 4, dim)
            table = c.table.clone()
            table[0, 1], table[0, 7] = c.n_pages, -1
            lse = torch.empty(80, 4, device="cuda")
            out = lp.ltri_paged_attend(0, table, c.lens(), ints([0, 60, 80]), q, lse=lse)
            assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE and lp.ltri_paged_sync_status() == binding.LTRI_OK
            check(c, 0, q, out, lse, [60, 20], [0, 60, 80], absent=[*range(16, 32), *range(112, 128)])


def test_a_row_without_any_page_and_more_tokens_than_slots():
    c = make("int4-bf16", [40, 30, 20], 4, 2, 64, 16, seed=15)
    c.fill()
    lp, q = c.handle(max_tokens=100), c.randn(100, 4, 64)
    table = c.table.clone()
    table[1] = -1
    lens = c.lens()
    lens[2] = 10 ** 6
    lse, out = torch.full((100, 4), 3.0, device="cuda"), torch.full_like(q, 2.0)
    lp.ltri_paged_attend(0, table, lens, ints([0, 50, 70, 90]), q, out=out, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE
    # ten tokens in front of the row's first slot, a row of absent slots, a row of a bad length
    for rows in (slice(0, 10), slice(50, 90)):
        assert (out[rows] == 0).all() and (lse[rows] == -math.inf).all()
    assert (out[90:] == 2.0).all() and (lse[90:] == 3.0).all()
    check(c, 0, q[10:], out[10:], lse[10:], [40, 0, 0], [0, 40, 40, 40])


@pytest.mark.parametrize("kind,dim", [("bf16", 256), ("int4-bf16", 64)])
def test_attend_of_thousands_of_rows(kind, dim):
    # (more rows, and at head_dim 256 more blocks of queries, than the threads that lay them out)
    rows = 2300
    lens = [(i * 7) % 12 for i in range(rows)]
    news = [min(n, i % 5) for i, n in enumerate(lens)]
    c = make(kind, lens, 2, 1, dim, 4, seed=22)
    c.fill()
    lp, total = c.handle(max_tokens=sum(news)), sum(news)
    q, lse = c.randn(total, 2, dim), torch.empty(total, 2, device="cuda")
    starts = starts_of(news)
    out = lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    some = [*range(0, 40), *range(1000, 1060), *range(2040, 2060), *range(2260, 2300)]
    check(c, 0, q, out, lse, [m if r in set(some) else 0 for r, m in enumerate(news)], starts)
    assert out.isfinite().all() and lse.isfinite().all()


def test_attend_of_rows_without_a_token():
    c = make("int4-bf16", [40, 0, 20], 4, 2, 128, 16, seed=23)
    c.fill()
    lp, q = c.handle(max_tokens=9), c.randn(9, 4, 128)
    out, lse = torch.full_like(q, 2.0), torch.full((9, 4), 3.0, device="cuda")
    lp.ltri_paged_attend(0, c.table, c.lens(), ints([4, 4, 4, 4]), q, out=out, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert (out == 2.0).all() and (lse == 3.0).all()


@pytest.mark.parametrize("kind", KINDS)
def test_infinities_and_nan_in_keys_that_are_not_seen(kind):
    # token i sees the slots up to its own: those of the later ones hold what their logits make NaN and infinite
    c = make(kind, [300], 4, 2, 128, 16, seed=24)
    c.fill()
    lp, q = c.handle(max_tokens=200), c.randn(200, 4, 128)
    lse = torch.empty(200, 4, device="cuda")
    want = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 200]), q, lse=lse).clone()
    pg, off = c.places(0, 300)
    for slot, bad in ((230, math.inf), (231, -math.inf), (260, math.nan)):
        row = torch.zeros(1, 2, 128)
        row[:, :, 7] = bad
        if kind.startswith("int4"):
            row = torch.where(row == 0, row, math.nan)  # (infinities are clamped in 4 bits)
            c.store(0, pg[slot:slot + 1], off[slot:slot + 1], 0, row)
        else:
            ref.put(c.k[0], pg[slot:slot + 1], off[slot:slot + 1], row.to(c.k.dtype))
    got = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 200]), q)
    assert torch.equal(got[:130], want[:130]) and not got[160:].isfinite().any()


def test_attend_beyond_32_bits():
    # pages 2 MiB apart (a view of one page in 1024 of a larger tensor): the last ones lie 5 GiB behind the first
    for kind in ("bf16", "int4"):
        pages, P, hkv = 2600, 128, 2
        row = 64 if kind == "bf16" else 32  # elements of the tensor
        dtype = BF16 if kind == "bf16" else torch.uint8
        step = (1 << 21) // (2 if kind == "bf16" else 1)
        bases = [torch.zeros(pages, step, dtype=dtype, device="cuda") for _ in range(2)]
        k, v = (b.as_strided((1, pages, hkv, P, row), (0, step, row, row * hkv, 1), 0) for b in bases)
        sc = {} if kind == "bf16" else dict(block_scales=torch.zeros(1, pages, hkv, P, 2, 2, dtype=torch.uint8, device="cuda"))
        lp = binding.LtriPaged(k, v, 4, dtype=BF16, max_rows=1, max_tokens=70, **sc)
        table, lens, starts = ints([[0, pages - 1]]), ints([2 * P]), ints([0, 70])
        g = torch.Generator().manual_seed(3)
        x, y = (torch.randn(70, hkv, 64, generator=g).to(BF16) for _ in range(2))
        q = torch.randn(70, 4, 64, generator=g).to(BF16)
        lp.ltri_paged_append(0, table, lens, starts, x.cuda(), y.cuda())
        out = lp.ltri_paged_attend(0, table, lens, starts, q.cuda())
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        K, V = ((r.double() if kind == "bf16" else i4.quantise(r)[2]).repeat_interleave(2, 1) for r in (x, y))
        # (all other slots hold zeros: logits of 0, values of 0)
        logits = torch.einsum("ihd,jhd->hij", q.double(), K) / 8
        p = torch.where(torch.ones(70, 70).tril().bool(), logits.exp(), 0.0)
        want = torch.einsum("hij,jhd->ihd", p, V) / (p.sum(-1) + 2 * P - 70).T[:, :, None]
        size = torch.einsum("hij,jhd->ihd", p, V.abs()) / (p.sum(-1) + 2 * P - 70).T[:, :, None]
        assert ((out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -10 + 1e-6).all()


@pytest.mark.parametrize("starts", [[0, 30, 20, 60], [5, 5, 90, 90], [-4, 10, 20, 30], [0, 2 ** 31 - 1, 20, 30], [60, 60, 0, 60]])
def test_starts_that_are_none_are_recorded_and_stay_in_bounds(starts):
    c = make("bf16", [40, 30, 20], 4, 2, 64, 16, seed=16)
    c.fill()
    lp, q = c.handle(max_tokens=60), c.randn(62, 4, 64)
    out = torch.full_like(q, 2.0)
    lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q[:60], out=out[:60])
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE
    assert (out[60:] == 2.0).all()
    torch.cuda.synchronize()


def test_what_lies_behind_a_row_is_not_read():
    # (the caches of these tests hold NaN in every slot that nobody has written; here also in the last tile's pages)
    for kind in ("bf16", "int4-bf16"):
        c = make(kind, [129, 3], 4, 2, 128, 64, room=60, seed=17)
        c.fill()
        out, lse = attend(c, [129, 3])
        assert out.isfinite().all() and lse.isfinite().all()


def test_prompts_in_parts_eager_and_captured():
    def serve(graph):
        c = make("int4-bf16", [0, 0, 0], 8, 2, 128, 16, room=400, seed=21)
        parts = [[100, 0, 33], [1, 130, 60], [150, 7, 0], [40, 1, 1]]
        most = max(sum(p) for p in parts)
        lp = c.handle(max_tokens=most)
        dev, starts = ints([0, 0, 0]), ints([0, 0, 0, 0])
        q, k, v = c.randn(most, 8, 128), c.randn(most, 2, 128), c.randn(most, 2, 128)
        out, lse = torch.zeros_like(q), torch.zeros(most, 8, device="cuda")

        def step():
            lp.ltri_paged_append(0, c.table, dev, starts, k, v)
            lp.ltri_paged_attend(0, c.table, dev, starts, q, out=out, lse=lse)

        captured, lens, got = torch.cuda.CUDAGraph(), [0, 0, 0], []
        if graph:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(captured, stream=side):
                step()
        for p in parts:
            for t in (q, k, v):
                t.copy_(c.randn(*t.shape))
            lens = [a + b for a, b in zip(lens, p)]
            dev.copy_(ints(lens))
            starts.copy_(ints(starts_of(p)))
            captured.replay() if graph else step()
            assert lp.ltri_paged_sync_status() == binding.LTRI_OK
            c.lens_cpu = lens
            if not graph:
                check(c, 0, q, out, lse, p, starts_of(p))
            got += [ref.bits(out).clone(), ref.bits(lse).clone()]
        return got + [x for x in c.snapshot().values()]

    assert all(torch.equal(x, y) for x, y in zip(serve(False), serve(True)))


def test_two_handles_on_two_streams_at_once():
    cs = [make("int4-bf16", [3000, 500], 8, 2, 128, 16, seed=s) for s in (1, 2)]
    lps, qs, want = [], [], []
    for c in cs:
        c.fill()
        lps.append(c.handle(max_tokens=400))
        qs.append(c.randn(400, 8, 128))
    starts, lens = ints([0, 300, 400]), cs[0].lens()
    for c, lp, q in zip(cs, lps, qs):
        want.append(lp.ltri_paged_attend(0, c.table, lens, starts, q).clone())
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [lp.ltri_paged_attend(0, c.table, lens, starts, q, stream=s) for c, lp, q, s in zip(cs, lps, qs, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_are_refused_before_anything_is_launched():
    c = make("int4-bf16", [20, 30], 4, 2, 64, 16, seed=1)
    c.fill()
    lp, lens, starts = c.handle(max_tokens=8), c.lens(), ints([0, 4, 8])
    launches = lp.ltri_paged_launch_count()
    q = c.randn(8, 4, 64)
    out, lse = torch.empty_like(q), torch.empty(8, 4, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    raw, cols = binding.load(), c.table.shape[1]
    ws, room = lp._attend
    assert raw.ltri_paged_attend_workspace_bytes(lp._h, 8) == room
    assert [raw.ltri_paged_attend_workspace_bytes(lp._h, n) for n in (0, -1, (1 << 24) + 1)] == [0, 0, 0]

    def rc(layer=0, n=2, starts=p(starts), tokens=8, q=p(q), stride=0, out=p(out), lse=p(lse), ws=ws, room=room):
        return raw.ltri_paged_attend(lp._h, layer, p(c.table), cols, cols, p(lens), n, starts, tokens, q, stride, out, lse, ws, room,
                                     None)

    for kw in (dict(layer=-1), dict(layer=1), dict(n=0), dict(starts=None), dict(starts=p(starts) + 2), dict(tokens=-1),
               dict(q=None), dict(q=p(q) + 8), dict(stride=64), dict(stride=260), dict(out=None), dict(out=p(out) + 4),
               dict(lse=p(lse) + 1), dict(ws=None), dict(ws=ws + 16), dict(out=p(q) + 512), dict(out=p(q), stride=512)):
        assert rc(**kw) == binding.LTRI_EINVAL, kw
    assert rc(n=3) == binding.LTRI_ECAPACITY and rc(tokens=(1 << 24) + 1) == binding.LTRI_ECAPACITY
    assert rc(room=room - 1) == binding.LTRI_ECAPACITY and rc(tokens=0) == binding.LTRI_OK
    for kw in (dict(q=q.half()), dict(q=q[:, :2]), dict(q=q.cpu()), dict(out=out[:4]), dict(lse=lse[:4]), dict(starts=starts[:2])):
        with pytest.raises(ValueError):
            lp.ltri_paged_attend(**{**dict(layer=0, table=c.table, lens=lens, starts=starts, q=q), **kw})
    with pytest.raises(binding.LtriError):  # a handle without room for it
        c.handle().ltri_paged_attend(0, c.table, lens, starts, q)
    torch.cuda.synchronize()
    assert lp.ltri_paged_launch_count() == launches
