"""The paged cache's operators over 4-bit pages on the GPU against their definition in 64 bits."""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_int4_reference as i4
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
# lengths at which tiles, pages and shares of the work begin and end
EDGES = [1, 0, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- appending and reading back ----


def hard_rows(dtype, n, hkv, dim, g):
    """Rows whose blocks lie at the format's edges: midpoints of numbers and of scales, the smallest and largest scales, zeros."""
    x = torch.randn(n, hkv, dim, generator=g) * torch.exp2(torch.randint(-20, 12, (n, hkv, dim // 32), generator=g).float()
                                                           ).repeat_interleave(32, -1)
    b = x.view(n, hkv, dim // 32, 32)
    s = (8 + torch.randint(0, 8, (n, hkv, dim // 32), generator=g)) * torch.exp2(
        torch.randint(-20, 6, (n, hkv, dim // 32), generator=g).float())
    ties = s[..., None] * torch.randint(-14, 15, b.shape, generator=g) / 2
    ties[..., 0] = 7 * s
    pick = torch.randint(0, 6, (n, hkv, dim // 32), generator=g)
    b[pick == 0] = ties[pick == 0]
    b[pick == 1] = 0.0
    # the largest magnitude a midpoint of two scales times 7
    mid = b.clone().clamp(-1, 1) * s[..., None]
    mid[..., 5] = 7 * (s + torch.exp2(torch.floor(torch.log2(s)) - 4))
    b[pick == 2] = mid[pick == 2]
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("layout,page,dim,hkv", [("hnd", 16, 128, 3), ("nhd", 3, 64, 1), ("both", 64, 256, 2), ("nhd", 16, 64, 5)])
@pytest.mark.parametrize("weighted", [False, True])
def test_append_and_read_back(dtype, layout, page, dim, hkv, weighted):
    lens, news = [40, 0, 7, 100, 1, 33], [40, 0, 5, 64, 1, 0]
    c = i4.Cache(lens, hkv, hkv, dim, page, dtype, layout=layout, layers=2, weighted=weighted, seed=page + dim)
    lp, total = c.handle(), sum(news)
    starts = [2 + sum(news[:i]) for i in range(len(news) + 1)]  # (two tokens in front that are nobody's, three behind)
    k, v = (hard_rows(dtype, total + 5, hkv, dim, c.g) for _ in range(2))
    before = c.snapshot()
    w = torch.rand(total + 5, hkv, generator=c.g).cuda() if weighted else None
    pos = ints([5, 6, 7, 8, 9, 10])
    lp.ltri_paged_append(1, c.table, c.lens(), ints(starts), k.cuda(), v.cuda(), row_pos=pos, weights=w)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    after, want = c.snapshot(), {n: x.clone() for n, x in before.items()}
    values = [torch.zeros(total + 5, hkv, dim).double() for _ in range(2)]
    for r, (n, m) in enumerate(zip(lens, news)):
        pg, off = (x[n - m:] for x in c.places(r, n))
        for which, (name, x) in enumerate((("k", k), ("v", v))):
            code, scale, value = i4.quantise(x[starts[r]:starts[r + 1]])
            want[name][1][pg, :, off] = code.cuda()
            want["sc"][1][pg, :, off, which] = scale.cuda()
            values[which][starts[r]:starts[r + 1]] = value
        if weighted:
            ref.put(want["w"][1], pg, off, ref.bits(w[starts[r]:starts[r + 1]]))
            ref.put(want["pos"][1], pg, off, (5 + r + torch.arange(m, dtype=torch.int32))[:, None].expand(m, hkv))
    for name in want:
        assert torch.equal(after[name], want[name]), name
    # the same tokens back, the others' rows as they were
    for both in ((True, True), (True, False), (False, True)):
        back = [torch.full((total + 5, hkv, dim), 3.0, dtype=dtype, device="cuda") if b else None for b in both]
        lp.ltri_paged_read(1, c.table, c.lens(), ints(starts), *back)
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        for got, value in zip(back, values):
            if got is not None:
                assert torch.equal(got[2:-3].cpu().double(), value[2:-3])
                assert (got[:2] == 3.0).all() and (got[-3:] == 3.0).all()


def test_append_of_strided_rows():
    c = i4.Cache([50, 9], 3, 3, 128, 16, BF16, seed=5)
    lp = c.handle()
    both = c.randn(59, 2, 3, 128)  # (K and V side by side)
    lp.ltri_paged_append(0, c.table, c.lens(), ints([0, 50, 59]), both[:, 0], both[:, 1])
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    back = torch.empty_like(both)
    lp.ltri_paged_read(0, c.table, c.lens(), ints([0, 50, 59]), back[:, 0], back[:, 1])
    for which in (0, 1):
        assert torch.equal(back[:, which].cpu().double(), i4.quantise(both[:, which].contiguous().cpu())[2])


def test_append_of_infinities_and_nan():
    c = i4.Cache([6], 1, 1, 64, 4, BF16, seed=3)
    lp = c.handle()
    x = torch.randn(6, 1, 64, generator=c.g)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 5], x[3, 0, 0], x[4, 0, 63] = math.inf, -math.inf, math.nan, 3e38, -math.nan
    x = x.to(BF16)
    lp.ltri_paged_append(0, c.table, c.lens(), ints([0, 6]), x.cuda(), x.cuda())
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    pg, off = c.places(0, 6)
    code, scale, value = i4.quantise(x)
    for which, pages in ((0, c.k), (1, c.v)):
        bad = scale == i4.NAN
        assert torch.equal(c.sc[0][pg, :, off, which].cpu(), scale) and bad.sum() == 2
        same = (pages[0][pg, :, off].cpu() == code).unflatten(-1, (-1, 16)).all(-1)
        assert (same | bad).all()
    back = torch.zeros(6, 1, 64, dtype=BF16, device="cuda")
    lp.ltri_paged_read(0, c.table, c.lens(), ints([0, 6]), back)
    assert torch.equal(back.cpu().double().nan_to_num(77.0), value.nan_to_num(77.0))
    # a logit that is not a number reaches the outputs
    out = lp.ltri_paged_decode(0, c.table, c.lens(), c.randn(1, 1, 64))
    assert out.isnan().all()


@pytest.mark.parametrize("dtype,kind", [(BF16, "plain"), (FP16, "plain"), (BF16, "e4m3"), (FP16, "e4m3"), (BF16, "int4"), (FP16, "int4")])
@pytest.mark.parametrize("layout,page,dim,hkv", [("hnd", 16, 128, 8), ("nhd", 7, 64, 1), ("both", 1, 256, 3)])
def test_read_of_ranges(dtype, kind, layout, page, dim, hkv):
    lens = [90, 0, 3, 200, 17]
    c = (i4.Cache if kind == "int4" else ref.Cache)(lens, hkv, hkv, dim, page, dtype, layout=layout, layers=2, seed=dim,
                                                   **({} if kind == "int4" else dict(e4m3=kind == "e4m3")))
    c.fill()
    lp = c.handle()
    first, count = [10, 0, 2, 0, 0], [61, 0, 1, 200, 0]
    starts = [sum(count[:i]) for i in range(6)]
    both = torch.full((sum(count) + 2, 2, hkv, dim), 9.0, dtype=dtype, device="cuda")  # (K and V side by side)
    lp.ltri_paged_read(1, c.table, c.lens(), ints(starts), both[:, 0], both[:, 1], first=ints(first))
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for r, n in enumerate(lens):
        if not count[r]:
            continue
        for which, want in enumerate(c.row(1, r, n)):
            got = both[starts[r]:starts[r + 1], which].cpu()
            # (element * scale is fp32's product, then rounded)
            want = want.float().to(dtype) if kind == "e4m3" else want.to(dtype)
            assert torch.equal(got, want[first[r]:first[r] + count[r]])
    assert (both[sum(count):] == 9.0).all()


def test_read_of_many_rows_and_of_slots_that_are_not_there():
    rows = 700
    lens = [(i * 37) % 23 for i in range(rows)]
    c = i4.Cache(lens, 2, 2, 64, 5, FP16, seed=8)
    c.fill()
    lp = c.handle()
    starts = [sum(lens[:i]) for i in range(rows + 1)]
    k = torch.empty(starts[-1], 2, 64, dtype=FP16, device="cuda")
    lp.ltri_paged_read(0, c.table, c.lens(), ints(starts), k)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    want = torch.cat([c.row(0, r, n)[0] for r, n in enumerate(lens) if n])
    assert torch.equal(k.cpu().double(), want)
    # more than the row has, in front of its first slot and behind its last; a page that is none
    table = c.table.clone()
    table[4, 1] = c.n_pages
    lens = c.lens()
    n4 = int(lens[4])
    got = torch.full((30, 2, 64), 5.0, dtype=FP16, device="cuda")
    starts = ints([0, 0, 0, 0, 0, 30] + [30] * (rows - 5))
    lp.ltri_paged_read(0, table, lens, starts, None, got, first=ints([0, 0, 0, 0, -3] + [0] * (rows - 5)))
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE and lp.ltri_paged_sync_status() == binding.LTRI_OK
    V = c.row(0, 4, n4)[1]
    want = torch.zeros(30, 2, 64).double()
    for i in range(30):
        if 0 <= i - 3 < n4 and not 5 <= i - 3 < 10:
            want[i] = V[i - 3]
    assert torch.equal(got.cpu().double(), want)


# ---- single tokens ----


def decode(c, lp, l=0, new=True, row_pos=None, decay=1.0, scale=None, q=None, q_scale=1.0):
    n = len(c.lens_cpu)
    q = c.randn(n, c.hq, c.dim, scale=q_scale) if q is None else q
    k, v = (c.randn(n, c.hkv, c.dim), c.randn(n, c.hkv, c.dim)) if new else (None, None)
    before = None if c.w is None else c.w.clone()
    s = torch.full((n, c.hq), 7.0, device="cuda")
    out = lp.ltri_paged_decode(l, c.table, c.lens(), q, k, v, row_pos=row_pos, lse=s)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for r, m in enumerate(c.lens_cpu if new else []):
        if m == 0:
            continue
        pg, off = c.places(r, m)
        for which, (pages, x) in enumerate(((c.k, k), (c.v, v))):
            code, byte, _ = i4.quantise(x[r].cpu())
            assert torch.equal(pages[l][pg[-1], :, off[-1]].cpu(), code)
            assert torch.equal(c.sc[l][pg[-1], :, off[-1], which].cpu(), byte)
        if c.w is not None:
            assert (c.pos[l, pg[-1], :, off[-1]] == (m - 1 if row_pos is None else int(row_pos[r]))).all()
    i4.check_decode(c, l, q, out, s, c.lens_cpu, before, decay, new, scale)
    return out


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("layout,page", [("hnd", 16), ("nhd", 7), ("both", 1), ("hnd", 48)])
def test_decode_at_the_edges(dim, dtype, layout, page):
    c = i4.Cache(EDGES, 8, 2, dim, page, dtype, layout=layout, seed=dim + page)
    c.fill()
    before = c.snapshot()
    decode(c, c.handle())
    # nothing but the new slots has changed
    after = c.snapshot()
    for name in before:
        x, y = before[name].clone(), after[name].clone()
        for r, n in enumerate(c.lens_cpu):
            if n:
                pg, off = c.places(r, n)
                x[0, pg[-1], :, off[-1]] = 0
                y[0, pg[-1], :, off[-1]] = 0
        assert torch.equal(x, y), name


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (16, 1), (32, 2), (24, 1), (64, 1), (9, 1)])
@pytest.mark.parametrize("weighted", [False, True])
def test_decode_of_every_group_size(hq, hkv, weighted):
    c = i4.Cache([200, 0, 17, 1], hq, hkv, 128, 16, BF16, weighted=weighted, seed=hq)
    c.fill()
    decode(c, c.handle())


@pytest.mark.parametrize("dim,dtype,hq", [(64, BF16, 12), (128, FP16, 12), (256, BF16, 12), (256, FP16, 48), (64, FP16, 48)])
@pytest.mark.parametrize("decay", [1.0, 0.5])
def test_decode_accumulates_weights(dim, dtype, hq, decay):
    c = i4.Cache(EDGES, hq, 3, dim, 5, dtype, layers=2, layout="nhd", weighted=True, seed=3)
    c.fill()
    lp = c.handle(weight_decay=decay)
    decode(c, lp, 1, row_pos=ints(list(range(100, 100 + len(EDGES)))), decay=decay)
    decode(c, lp, 1, new=False, decay=decay)


@pytest.mark.parametrize("rows,n,hq,hkv,dim", [(1, 40000, 8, 2, 128), (1, 9001, 32, 8, 64), (1, 20011, 4, 1, 256),
                                               (40, 1200, 8, 4, 128), (3, 7000, 8, 8, 128), (2, 9000, 32, 2, 64),
                                               (2, 9000, 40, 1, 256)])
@pytest.mark.parametrize("weighted", [False, True])
def test_decode_split_over_the_length(rows, n, hq, hkv, dim, weighted):
    lens = [max(1, n - 977 * i) if i % 7 != 5 else 0 for i in range(rows)]
    c = i4.Cache(lens, hq, hkv, dim, 64, BF16, weighted=weighted, seed=rows)
    c.fill()
    lp = c.handle()
    decode(c, lp)
    q = c.randn(rows, hq, dim)
    first = lp.ltri_paged_decode(0, c.table, c.lens(), q).clone()
    assert torch.equal(first, lp.ltri_paged_decode(0, c.table, c.lens(), q))


@pytest.mark.parametrize("lens,hq,hkv,dim", [([1, 0, 100, 512, 511], 8, 2, 128), ([513, 3], 16, 16, 64),
                                             ([64] * 7 + [0, 33], 32, 8, 256), ([257, 255, 5], 8, 2, 256),
                                             ([100] * 19, 8, 8, 128), ([0, 0, 0], 4, 2, 64)])
def test_decode_of_units_around_a_ctas_size(lens, hq, hkv, dim):
    c = i4.Cache(lens, hq, hkv, dim, 16, BF16, seed=len(lens) + dim)
    c.fill()
    decode(c, c.handle())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("q_scale,scale", [(2.0 ** -9, 40.0), (30.0, 0.05), (2.0 ** -13, 600.0)])
def test_decode_of_small_and_large_queries(dtype, q_scale, scale):
    c = i4.Cache([77, 400], 8, 2, 128, 16, dtype, seed=4)
    c.fill()
    decode(c, c.handle(softmax_scale=scale), q_scale=q_scale, scale=scale)


@pytest.mark.parametrize("q_scale", [2.0 ** 60, 2.0 ** -60, 2.0 ** -126, 2.0 ** 100])
def test_decode_of_queries_of_any_magnitude(q_scale):
    # the softmax's scale makes up for the queries': the logits are those of ordinary ones
    c = i4.Cache([77, 300], 8, 2, 128, 16, BF16, seed=6)
    c.fill()
    scale = 0.088 / q_scale if q_scale > 2.0 ** -100 else 0.088 * 2.0 ** 120
    decode(c, c.handle(softmax_scale=scale), q_scale=q_scale, scale=float(torch.tensor(scale)))


@pytest.mark.parametrize("magnitude", [1e-4, 300.0])
def test_decode_over_scales_at_the_ends_of_their_range(magnitude):
    c = i4.Cache([77, 300], 8, 2, 64, 16, FP16, seed=9)
    c.fill(magnitude)
    decode(c, c.handle(softmax_scale=1e-3 / magnitude), new=False, scale=float(torch.tensor(1e-3 / magnitude)))


@pytest.mark.parametrize("small", [2.0 ** -9, 7 * 2.0 ** -9])
def test_small_values_survive_among_large_ones_that_cancel(small):
    # All probabilities are equal.  1024 slots of V = 448, 2048 of the small one and 1024 of -448.  16 times 7 * 2^-9 are exact
    # beside the large ones' sum (1024 * 448 < 2^19, in steps of 2^-5), and with them all sums of tiles: what is left is exact.
    # 2^-9 is held as 63 * 2^-15, and a tile's sum of it is rounded to those steps: 2^-6 off at most in each of the 64 additions of
    # 32 slots at the least, which the 4096 slots' mean divides.
    n, hkv, rows = 4096, 8, torch.cuda.get_device_properties(0).multi_processor_count
    for dim, hq in ((64, 8), (128, 128), (256, 8)):
        c = i4.Cache([n], hq, hkv, dim, 16, BF16, seed=dim)
        pg, off = c.places(0, n)
        v = torch.full((n, hkv, dim), small)
        v[:1024], v[-1024:] = 448.0, -448.0
        c.store(0, pg, off, 0, torch.zeros(n, hkv, dim))
        got = c.store(0, pg, off, 1, v)
        assert torch.equal(got[:1024], v[:1024].double())
        mean = float(got[2000, 0, 0]) / 2
        lp = c.handle(max_rows=rows)
        lens = ints([n] * rows)
        out = lp.ltri_paged_decode(0, c.table.repeat(rows, 1), lens, c.randn(rows, hq, dim))
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        off_by = float((out.double() - mean).abs().max())
        assert off_by == 0.0 if small > 2.0 ** -8 else off_by <= 64 * 2.0 ** -6 / n + mean * 2.0 ** -8


def test_bad_pages_and_lengths_are_recorded_and_touch_nothing_else():
    c = i4.Cache([40, 40, 40], 4, 2, 128, 16, BF16, weighted=True, seed=11)
    c.fill()
    lp, q = c.handle(), c.randn(3, 4, 128)
    table, lens = c.table.clone(), c.lens()
    table[0, 1] = c.n_pages  # sixteen slots of row 0 are absent
    table[1, 2] = -1         # so are the last ones of row 1, its new token's among them
    lens[2] = 100000
    before = c.snapshot()
    k, v = c.randn(3, 2, 128), c.randn(3, 2, 128)
    out = lp.ltri_paged_decode(0, table, lens, q, k, v)
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE and lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert (out[2] == 0).all()
    K, V = c.row(0, 0, 40)
    there = [j for j in range(40) if not 16 <= j < 32]
    o, _, _, tol, _, _ = i4.attend(q[0].cpu().double(), K[there], V[there], c.steps(0, 0, 40)[there], 128 ** -0.5)
    assert ((out[0].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2 * tol).all()
    K, V = c.row(0, 1, 40)
    o, _, _, tol, _, _ = i4.attend(q[1].cpu().double(), K[:32], V[:32], c.steps(0, 1, 40)[:32], 128 ** -0.5)
    assert ((out[1].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2 * tol).all()
    pg, off = c.places(0, 40)
    for name, x in c.snapshot().items():
        if name in ("k", "v", "sc"):
            x[0, pg[-1], :, off[-1]] = 0
            before[name][0, pg[-1], :, off[-1]] = 0
            assert torch.equal(x, before[name]), name


def test_strided_queries_over_their_own_outputs():
    c = i4.Cache([50, 9], 8, 2, 64, 16, FP16, seed=12)
    c.fill()
    lp, wide = c.handle(), c.randn(2, 12, 64)
    q = wide[:, :8]
    out = lp.ltri_paged_decode(0, c.table, c.lens(), q, wide[:, 8:10], wide[:, 10:])
    i4.check_decode(c, 0, q, out, None, c.lens_cpu)
    dense = c.randn(2, 8, 64)
    want = lp.ltri_paged_decode(0, c.table, c.lens(), dense).clone()
    assert torch.equal(lp.ltri_paged_decode(0, c.table, c.lens(), dense, out=dense), want)


# ---- eviction, and all of it together ----


@pytest.mark.parametrize("dim,layout,page", [(64, "hnd", 16), (128, "nhd", 3), (256, "both", 64)])
@pytest.mark.parametrize("n,budget", [(300, 128), (300, 299), (5000, 1700)])
def test_evict_moves_scales_with_their_rows(dim, layout, page, n, budget):
    lens = [n, 0, budget, n - 7]
    c = i4.Cache(lens, 4, 2, dim, page, BF16, layers=2, layout=layout, weighted=True, seed=n + dim)
    c.fill()
    lp, new = c.handle(), ints([0] * 4)
    want, lens = i4.evict(c, lens, budget, 4, 40, range(2))
    lp.ltri_paged_evict(0, 2, c.table, c.lens(), new, budget, 4, 40)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK and new.tolist() == lens
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


def serve(graph):
    """Prompts, an eviction, then steps within a budget, the steps as one captured graph or call by call (then every call is
    checked), their rows read back.  Returns everything at the end."""
    c = i4.Cache([50, 0, 33], 8, 2, 128, 16, BF16, layers=2, weighted=True, room=4, seed=21)
    lp = c.handle(weight_decay=0.9)
    lens, budget = c.lens_cpu, 40
    dev, used = c.lens(), ints([1, 0, 1])
    w = torch.rand(83, 2, generator=c.g).cuda()
    for l in range(2):
        lp.ltri_paged_append(l, c.table, dev, ints([0, 50, 50, 83]), c.randn(83, 2, 128), c.randn(83, 2, 128), weights=w)
    want, lens = i4.evict(c, lens, budget, 4, 10, range(2))
    lp.ltri_paged_evict(0, 2, c.table, dev, dev, budget, 4, 10)
    row_pos = ints([50, 0, 33])
    q, kv = [c.randn(3, 8, 128) for _ in range(2)], [c.randn(3, 4, 128) for _ in range(2)]
    out, lse = [torch.zeros_like(t) for t in q], [torch.zeros(3, 8, device="cuda") for _ in range(2)]
    back = torch.zeros(80, 2, 128, dtype=BF16, device="cuda")
    all_rows = ints([0, 40, 40, 73])

    def decode_layer(l):
        lp.ltri_paged_decode(l, c.table, dev, q[l], kv[l][:, :2], kv[l][:, 2:], row_pos=row_pos, out=out[l], lse=lse[l])

    def evict():
        lp.ltri_paged_evict(0, 2, c.table, dev, dev, budget, 4, 10)

    captured = torch.cuda.CUDAGraph()
    if graph:
        before, side = c.snapshot(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(captured, stream=side):
            dev.add_(used)
            decode_layer(0)
            decode_layer(1)
            evict()
            lp.ltri_paged_read(1, c.table, dev, all_rows, None, back, first=ints_zero)
            row_pos.add_(used)
        assert all(torch.equal(x, before[n]) for n, x in c.snapshot().items())  # (capturing runs nothing)
    for _ in range(9):
        for l in range(2):
            q[l].copy_(c.randn(3, 8, 128))
            kv[l].copy_(c.randn(3, 4, 128))
        if graph:
            captured.replay()
            torch.cuda.synchronize()
            continue
        lens = [n + 1 if n else 0 for n in lens]
        dev.add_(used)
        old = c.w.clone()
        for l in range(2):
            decode_layer(l)
            i4.check_decode(c, l, q[l], out[l], lse[l], lens, old, 0.9, True)
        want, lens = i4.evict(c, lens, budget, 4, 10, range(2))
        evict()
        assert dev.tolist() == lens
        for name, t in c.snapshot().items():
            assert torch.equal(t, want[name]), name
        lp.ltri_paged_read(1, c.table, dev, all_rows, None, back, first=ints_zero)
        assert torch.equal(back[:40].cpu().double(), c.row(1, 0, 40)[1])
        row_pos.add_(used)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    return {**c.snapshot(), "out": ref.bits(out[1]), "lse": ref.bits(lse[1]), "lens": dev.clone(), "back": ref.bits(back)}


def test_prompts_then_steps_within_a_budget_eager_and_captured():
    global ints_zero
    ints_zero = ints([0, 0, 0])
    eager, replayed = serve(False), serve(True)
    for name in eager:
        assert torch.equal(eager[name], replayed[name]), name


def test_offsets_beyond_32_bits():
    # pages 2 MiB apart (a view of one page in 1024 of a larger tensor): the last ones lie 5 GiB behind the first; scales of
    # 2600 pages of 8192 slots and 8 heads take 2.5 GiB
    pages, P, hkv = 2600, 8192, 8
    base = torch.zeros(pages, 1 << 21, dtype=torch.uint8, device="cuda")
    k, v = (base.as_strided((1, pages, hkv, P, 32), (0, 1 << 21, 32, 32 * hkv, 1), at) for at in (0, 0))
    v = torch.zeros_like(base).as_strided((1, pages, hkv, P, 32), (0, 1 << 21, 32, 32 * hkv, 1), 0)
    sc = torch.zeros(1, pages, hkv, P, 2, 2, dtype=torch.uint8, device="cuda")
    lp = binding.LtriPaged(k, v, hkv, dtype=BF16, max_rows=1, block_scales=sc)
    table, lens = ints([[0, pages - 1]]), ints([2 * P])
    g = torch.Generator().manual_seed(2)
    x, y = (torch.randn(41, hkv, 64, generator=g).to(BF16) for _ in range(2))
    lp.ltri_paged_append(0, table, lens, ints([0, 41]), x.cuda(), y.cuda())
    for pages_, rows, which in ((k, x, 0), (v, y, 1)):
        code, scale, value = i4.quantise(rows)
        assert torch.equal(pages_[0, pages - 1, :, P - 41:].transpose(0, 1).cpu(), code)
        assert torch.equal(sc[0, pages - 1, :, P - 41:, which].transpose(0, 1).cpu(), scale)
        back = torch.empty(41, hkv, 64, dtype=BF16, device="cuda")
        lp.ltri_paged_read(0, table, lens, ints([0, 41]), *((back, None) if which == 0 else (None, back)))
        assert torch.equal(back.cpu().double(), value)
    # (all other slots hold zeros: logits of 0, values of 0)
    q = torch.zeros(1, hkv, 64, dtype=BF16, device="cuda")
    q[:] = 0.25
    out = lp.ltri_paged_decode(0, table, lens, q)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    K, V = (i4.quantise(r)[2] for r in (x, y))
    p = torch.exp((K * 0.25).sum(-1) / 8)
    want = (p[:, :, None] * V).sum(0) / (p.sum(0) + 2 * P - 41)[:, None]
    assert ((out[0].cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + 1e-6).all()


def test_calls_are_refused_before_anything_is_launched():
    c = i4.Cache([20, 30], 4, 2, 64, 16, BF16, seed=1)
    c.fill()
    lp, lens = c.handle(), c.lens()
    before, launches = c.snapshot(), lp.ltri_paged_launch_count()
    k, starts = c.randn(2, 2, 64), ints([0, 1, 2])
    p = lambda t: t.data_ptr()  # noqa: E731
    raw, cols = binding.load(), c.table.shape[1]

    def read_rc(layer=0, n=2, starts=p(starts), first=None, tokens=2, k=p(k), v=None, stride=0):
        return raw.ltri_paged_read(lp._h, layer, p(c.table), cols, cols, p(lens), n, starts, first, tokens, k, v, stride, None)

    for kw in (dict(layer=-1), dict(layer=1), dict(n=0), dict(starts=None), dict(starts=p(starts) + 1), dict(first=p(lens) + 2),
               dict(tokens=-1), dict(k=None), dict(k=p(k) + 8), dict(v=p(k) + 2), dict(stride=64), dict(stride=132)):
        assert read_rc(**kw) == binding.LTRI_EINVAL, kw
    assert read_rc(n=3) == binding.LTRI_ECAPACITY and read_rc(tokens=1 << 31) == binding.LTRI_ECAPACITY
    assert read_rc(tokens=0) == binding.LTRI_OK
    for kw in (dict(k=k.half()), dict(k=k.cpu()), dict(k=None), dict(starts=starts[:2]), dict(first=starts), dict(k=k[:, :1]),
               dict(v=c.randn(2, 4, 64)[:, :2])):
        with pytest.raises(ValueError):
            lp.ltri_paged_read(**{**dict(layer=0, table=c.table, lens=lens, starts=starts, k=k), **kw})
    with pytest.raises(binding.LtriError):  # nothing to evict by
        lp.ltri_paged_evict(0, 1, c.table, lens, lens, 8, 0, 0)
    torch.cuda.synchronize()
    assert lp.ltri_paged_launch_count() == launches
    for name, t in c.snapshot().items():
        assert torch.equal(t, before[name]), name
    for kw in (dict(block_scales=c.sc[:, :, :, :, :1]), dict(block_scales=c.sc.float()), dict(block_scales=None),
               dict(block_scales=c.sc.cpu()), dict(dtype=None), dict(k_scale=torch.ones(2, device="cuda"))):
        with pytest.raises(ValueError):
            binding.LtriPaged(c.k, c.v, 4, **{**dict(dtype=BF16, block_scales=c.sc), **kw})
    with pytest.raises(ValueError):
        binding.LtriPaged(c.k.view(torch.int8), c.v.view(torch.int8), 4, dtype=BF16, block_scales=c.sc)
