"""The paged cache's operators on the GPU against their definition in 64 bits."""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
# lengths at which tiles, pages and shares of the work begin and end
EDGES = [1, 0, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300]


def decode(c, lp, l=0, new=True, row_pos=None, decay=1.0, scale=None, q=None, lse=True, q_scale=1.0):
    n = len(c.lens_cpu)
    q = c.randn(n, c.hq, c.dim, scale=q_scale) if q is None else q
    k, v = (c.randn(n, c.hkv, c.dim), c.randn(n, c.hkv, c.dim)) if new else (None, None)
    before = None if c.w is None else c.w.clone()
    s = torch.full((n, c.hq), 7.0, device="cuda") if lse else None
    out = lp.ltri_paged_decode(l, c.table, c.lens(), q, k, v, row_pos=row_pos, lse=s)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    if new:
        for r, m in enumerate(c.lens_cpu):
            if m == 0:
                continue
            pg, off = c.places(r, m)
            for pages, x, scl in ((c.k, k, c.ks), (c.v, v, c.vs)):
                got, want = ref.take(pages[l], pg[-1:], off[-1:])[0], x[r]
                if scl is None:
                    assert torch.equal(got, want)
                else:
                    assert torch.equal(got.cpu().double(), ref.quantise(want.cpu(), scl.cpu()))
            if c.w is not None:
                want = m - 1 if row_pos is None else int(row_pos[r])
                assert (c.pos[l, pg[-1], :, off[-1]] == want).all()
    ref.check_decode(c, l, q, out, s, c.lens_cpu, before, decay, new, scale)
    return out


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,e4m3", [(BF16, False), (FP16, False), (BF16, True), (FP16, True)])
@pytest.mark.parametrize("layout,page", [("hnd", 16), ("nhd", 7), ("both", 1)])
def test_decode_at_the_edges(dim, dtype, e4m3, layout, page):
    c = ref.Cache(EDGES, 8, 2, dim, page, dtype, e4m3, layout=layout, seed=dim + page)
    c.fill()
    before = c.snapshot()
    lp = c.handle()
    decode(c, lp)
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
    c = ref.Cache([200, 0, 17, 1], hq, hkv, 128, 16, BF16, weighted=weighted, seed=hq)
    c.fill()
    decode(c, c.handle())


@pytest.mark.parametrize("dim,dtype,e4m3", [(64, BF16, True), (128, FP16, False), (256, BF16, False), (128, FP16, True)])
@pytest.mark.parametrize("decay", [1.0, 0.5, 0.0])
def test_decode_accumulates_weights(dim, dtype, e4m3, decay):
    c = ref.Cache(EDGES, 12, 3, dim, 5, dtype, e4m3, layers=2, layout="nhd", weighted=True, seed=3)
    c.fill()
    lp = c.handle(weight_decay=decay)
    pos = torch.arange(100, 100 + len(EDGES), dtype=torch.int32, device="cuda")
    other = [t.clone() for t in (c.w[0], c.pos[0])]
    decode(c, lp, 1, row_pos=pos, decay=decay)
    decode(c, lp, 1, new=False, decay=decay)
    assert torch.equal(ref.bits(c.w[0]), ref.bits(other[0])) and torch.equal(c.pos[0], other[1])


@pytest.mark.parametrize("rows,n,hq,hkv", [(1, 40000, 8, 2), (1, 9001, 32, 8), (1, 20011, 4, 1), (40, 1200, 8, 4),
                                           (3, 7000, 8, 8)])
@pytest.mark.parametrize("weighted", [False, True])
def test_decode_split_over_the_length(rows, n, hq, hkv, weighted):
    lens = [max(1, n - 977 * i) if i % 7 != 5 else 0 for i in range(rows)]
    c = ref.Cache(lens, hq, hkv, 128, 64, BF16, weighted=weighted, seed=rows)
    c.fill()
    lp = c.handle()
    out = decode(c, lp)
    # the same inputs, the same bits
    q = c.randn(rows, hq, 128)
    first = lp.ltri_paged_decode(0, c.table, c.lens(), q).clone()
    assert torch.equal(first, lp.ltri_paged_decode(0, c.table, c.lens(), q)) and out.shape == first.shape


@pytest.mark.parametrize("lens,hq,hkv,dim", [([1, 0, 100, 128, 127], 8, 2, 128), ([256, 3], 16, 16, 64),
                                             ([64] * 7 + [0, 33], 32, 8, 256), ([129, 5], 8, 2, 128),
                                             ([100] * 19, 8, 8, 128), ([0, 0, 0], 4, 2, 64)])
@pytest.mark.parametrize("weighted", [False, True])
def test_decode_of_units_around_a_ctas_size(lens, hq, hkv, dim, weighted):
    # units with a CTA of their own, and batches that just miss that: a slot more than the CTA's tiles, a CTA too few
    c = ref.Cache(lens, hq, hkv, dim, 16, BF16, weighted=weighted, seed=len(lens) + dim)
    c.fill()
    decode(c, c.handle())


@pytest.mark.parametrize("rows,hkv,e4m3", [(70, 1, False), (70, 3, True), (33, 2, True)])
def test_decode_of_many_ragged_rows(rows, hkv, e4m3):
    # more rows than a warp has lanes, several units to a warp's run, runs that end inside units and inside tiles
    lens = [(i * 37) % 401 if i % 9 else 0 for i in range(rows)]
    c = ref.Cache(lens, 2 * hkv, hkv, 64, 5, FP16, e4m3, weighted=True, layout="nhd", seed=rows)
    c.fill()
    decode(c, c.handle())


@pytest.mark.parametrize("dtype,e4m3", [(BF16, False), (FP16, False), (BF16, True)])
def test_decode_of_large_logits(dtype, e4m3):
    # one slot takes all, at the beginning, in the middle and at the end, and its neighbours come within a few units
    c = ref.Cache([700, 700, 700, 2], 4, 1, 128, 16, dtype, e4m3, seed=9)
    c.fill(0.1)
    q = c.randn(4, 4, 128)
    for r, hot in ((0, 0), (1, 350), (2, 699), (3, 0)):
        pg, off = c.places(r, c.lens_cpu[r])
        row = (q[r, 0].float() * 20).clamp(-400, 400)
        ref.put(c.k[0], pg[hot:hot + 1], off[hot:hot + 1], row[None, None].to(c.k.dtype))
    decode(c, c.handle(), new=False, q=q)


@pytest.mark.parametrize("dtype,e4m3,scale", [(BF16, False, 2.0 ** 60), (BF16, False, 2.0 ** -60), (BF16, True, 2.0 ** 60),
                                              (BF16, True, 2.0 ** -60), (FP16, False, 2.0 ** 10), (FP16, True, 2.0 ** -10)])
def test_decode_of_queries_of_any_magnitude(dtype, e4m3, scale):
    # queries at the ends of their type's range, brought back by the softmax scale
    c = ref.Cache([300, 40], 8, 2, 64, 16, dtype, e4m3, seed=4)
    c.fill()
    decode(c, c.handle(softmax_scale=0.125 / scale), scale=0.125 / scale, q=c.randn(2, 8, 64, scale=scale))


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_decode_of_a_diffuse_tail_behind_one_heavy_slot(dtype):
    # one slot of weight 1/2 and 2^15 of about 2^-16 each: what a half-precision probability would lose is the tail
    n = (1 << 15) + 1
    c = ref.Cache([n], 1, 1, 64, 64, dtype, seed=5)
    pg, off = c.places(0, n)
    k = torch.zeros(n, 1, 64)
    k[0, 0, 0] = 15 * math.log(2.0) * 8 / 8
    ref.put(c.k[0], pg, off, k.to(dtype))
    v = torch.ones(n, 1, 64)
    v[0] = 0.0
    ref.put(c.v[0], pg, off, v.to(dtype))
    q = torch.zeros(1, 1, 64)
    q[0, 0, 0] = 8.0
    decode(c, c.handle(), new=False, q=q.to(dtype).cuda())


def test_decode_reads_strided_rows_and_writes_over_its_queries():
    c = ref.Cache([33, 0, 90], 8, 2, 64, 16, BF16, seed=6)
    c.fill()
    lp = c.handle()
    fused = c.randn(3, 12, 64)
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    want = lp.ltri_paged_decode(0, c.table, c.lens(), q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(want, lp.ltri_paged_decode(0, c.table, c.lens(), q, k, v))
    wide = torch.zeros(3, c.table.shape[1] + 5, dtype=torch.int32, device="cuda")
    wide[:, :-5] = c.table
    assert torch.equal(want, lp.ltri_paged_decode(0, wide[:, :-5], c.lens(), q, k, v))
    dense = q.contiguous()
    assert lp.ltri_paged_decode(0, c.table, c.lens(), dense, k, v, out=dense) is dense and torch.equal(dense, want)


def test_rows_may_share_pages_that_nobody_writes():
    c = ref.Cache([100, 100], 4, 2, 128, 16, FP16, seed=8)
    c.fill()
    c.table_cpu[1] = c.table_cpu[0]
    c.table = c.table_cpu.cuda()
    c.lens_cpu = [100, 61]
    decode(c, c.handle(), new=False)


@pytest.mark.parametrize("weighted,e4m3", [(False, False), (True, False), (True, True)])
def test_bad_pages_and_lengths_are_recorded_and_touch_nothing_else(weighted, e4m3):
    c = ref.Cache([40, 40, 40, 40, 40], 4, 2, 64, 16, BF16, e4m3, weighted=weighted, seed=11)
    c.fill()
    lp = c.handle()
    q, k, v = c.randn(5, 4, 64), c.randn(5, 2, 64), c.randn(5, 2, 64)
    good = lp.ltri_paged_decode(0, c.table, c.lens(), q, k, v).clone()
    before = c.snapshot()
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    table, lens = c.table.clone(), c.lens()
    table[0, 1] = -1           # sixteen slots in the middle are absent
    table[1, 2] = c.n_pages    # the last ones, the new one among them
    lens[2], lens[3] = -1, 49  # no length; more than the table holds
    bad = v.clone()
    bad[1] = math.nan          # (what an absent slot would have held does not matter)
    out = lp.ltri_paged_decode(0, table, lens, q, k, bad)
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE and lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert (out[2] == 0).all() and (out[3] == 0).all() and torch.equal(out[4], good[4])
    after = c.snapshot()
    for name in ("k", "v"):
        assert torch.equal(before[name], after[name])
    for r, keep in ((0, list(range(16)) + list(range(32, 40))), (1, list(range(32)))):
        K, V = c.row(0, r, 40)
        o, _, _, tol, _, _ = ref.attend(q[r].cpu().double(), K[keep], V[keep], 0.125)
        assert ((out[r].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2 * tol).all()
    starts = torch.tensor([0, 1, 2, 3, 4, 45], dtype=torch.int32, device="cuda")  # the last row has 41 tokens for 40 slots
    x = c.randn(45, 2, 64)
    before = c.snapshot()
    lp.ltri_paged_append(0, table, lens, starts, x, x)
    assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE
    after = c.snapshot()
    for r, tokens in ((4, x[5:]), (0, x[:1])):
        pg, off = c.places(r, 40)
        got = ref.take(c.k[0], pg, off)[-len(tokens):]
        if e4m3:
            assert torch.equal(got.cpu().double(), ref.quantise(tokens.cpu(), c.ks.cpu()))
        else:
            assert torch.equal(got, tokens)
    for r in (1, 2, 3):
        pg, _ = c.places(r, 40)
        assert torch.equal(before["k"][0, pg], after["k"][0, pg])
    # starts that do not ascend: whose a token is is then undefined, but nothing outside the rows is written
    before = c.snapshot()
    starts = torch.tensor([0, 30, 10, 45, 20, 45], dtype=torch.int32, device="cuda")
    lp.ltri_paged_append(0, c.table, c.lens(), starts, x, x)
    assert lp.ltri_paged_sync_status() in (binding.LTRI_OK, binding.LTRI_EDEVICE)
    owned = torch.zeros(c.n_pages, 16, dtype=torch.bool, device="cuda")
    for r in range(5):
        owned[c.places(r, 40)] = True
    for name, y in c.snapshot().items():
        assert torch.equal(before[name][0].transpose(1, 2)[~owned], y[0].transpose(1, 2)[~owned]), name
    if weighted:
        c.fill()
        lens[4] = 40
        new = torch.full((5,), -3, dtype=torch.int32, device="cuda")
        want, _ = ref.evict(c, [0, 0, 0, 0, 40], 24, 2, 4, [0])
        lp.ltri_paged_evict(0, 1, table, lens, new, 24, 2, 4)
        assert lp.ltri_paged_sync_status() == binding.LTRI_EDEVICE
        assert new.tolist() == [24, 24, 0, 0, 24]
        pg, _ = c.places(4, 40)
        for name, x in c.snapshot().items():
            assert torch.equal(x[0, pg], want[name][0, pg]), name


@pytest.mark.parametrize("dtype,e4m3", [(BF16, False), (FP16, True), (BF16, True)])
@pytest.mark.parametrize("layout,page,weighted", [("hnd", 16, True), ("nhd", 3, False), ("both", 64, True)])
def test_append_of_ragged_prompts(dtype, e4m3, layout, page, weighted):
    lens = [40, 0, 1, 130, 16, 9]
    new = [40, 0, 1, 70, 0, 5]  # the others' slots are held already
    c = ref.Cache(lens, 6, 3, 128, page, dtype, e4m3, layers=2, layout=layout, weighted=weighted, seed=page)
    before = c.snapshot()
    lp = c.handle()
    lead, total = 2, sum(new)
    starts = [lead]
    for m in new:
        starts.append(starts[-1] + m)
    fused = c.randn(lead + total + 3, 2 * 3, 128, scale=2.0)
    if e4m3:  # beyond the largest value, halfway between two, infinite and not a number
        scale = c.ks.cpu().float()
        odd = torch.tensor([1e4, -1e4, math.inf, -math.inf, 0.0, -0.0, 1e-5, 448.0 * float(scale[0]), 17.0 * float(scale[0])])
        fused[lead, 0, :len(odd)] = odd.to(dtype).cuda()
    k, v = fused[:, :3], fused[:, 3:]
    w = torch.rand(lead + total + 3, 3, generator=c.g).cuda()
    pos = torch.tensor([5, 6, 7, 8, 9, 10], dtype=torch.int32, device="cuda")
    dev_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    lp.ltri_paged_append(1, c.table, c.lens(), dev_starts, k, v, row_pos=pos, weights=w)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    after = c.snapshot()
    for name in before:
        assert torch.equal(before[name][0], after[name][0])  # the other layer
    written = torch.zeros(c.n_pages, page, dtype=torch.bool, device="cuda")
    for r, m in enumerate(new):
        if not m:
            continue
        pg, off = (x[lens[r] - m:] for x in c.places(r, lens[r]))
        written[pg, off] = True
        tok = slice(starts[r], starts[r] + m)
        for pages, x, s in ((c.k, k, c.ks), (c.v, v, c.vs)):
            got = ref.take(pages[1], pg, off)
            if s is None:
                assert torch.equal(got, x[tok])
            else:
                want = ref.quantise(x[tok].cpu(), s.cpu())
                assert torch.equal(got.cpu().double(), want)
        if weighted:
            assert torch.equal(ref.take(c.w[1], pg, off), w[tok])
            want = pos[r] + torch.arange(m, device="cuda", dtype=torch.int32)
            assert (ref.take(c.pos[1], pg, off) == want[:, None]).all()
    for name in before:
        x, y = before[name][1].transpose(1, 2), after[name][1].transpose(1, 2)
        assert torch.equal(x[~written], y[~written]), name
    if weighted:  # without positions and weights: slots' numbers and zeros
        lp.ltri_paged_append(0, c.table, c.lens(), dev_starts, k, v)
        pg, off = c.places(3, 130)
        assert (c.pos[0, pg[60:], :, off[60:]] == torch.arange(60, 130, device="cuda")[:, None]).all()
        assert (c.w[0, pg[60:], :, off[60:]] == 0).all()


def test_append_of_nothing_and_a_nan():
    c = ref.Cache([3], 2, 1, 64, 16, BF16, True, seed=1)
    lp = c.handle()
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    lp.ltri_paged_append(0, c.table, c.lens(), none, c.randn(0, 1, 64), c.randn(0, 1, 64))
    x = c.randn(3, 1, 64)
    x[1, 0, 5] = math.nan
    lp.ltri_paged_append(0, c.table, c.lens(), torch.tensor([0, 3], dtype=torch.int32, device="cuda"), x, x)
    pg, off = c.places(0, 3)
    got = ref.take(c.k[0], pg, off).float()
    assert torch.isnan(got[1, 0, 5]) and int(torch.isnan(got).sum()) == 1


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_append_rounds_every_quotient_to_the_nearest_8_bit_value(dtype):
    # every finite 16-bit value against scales that make quotients ties, near ties, tiny and huge, and reciprocals that are
    # not normal numbers
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(dtype)
    bits = torch.where(torch.isfinite(bits.float()), bits, 1.0).view(-1, 64)
    scales = [1.0, 0.5, 1 / 3, 0.0123, 2.0 ** -9, 17 / 16, 2.0 ** 100, 2.0 ** 127, 2.0 ** -120, 1.1754944e-38, 1e-40, 3e38]
    n = bits.shape[0]
    c = ref.Cache([n], len(scales), len(scales), 64, 64, dtype, True, seed=1)
    c.ks = c.vs = torch.tensor(scales, device="cuda")
    lp = c.handle()
    x = bits[:, None].expand(n, len(scales), 64).contiguous().cuda()
    lp.ltri_paged_append(0, c.table, c.lens(), torch.tensor([0, n], dtype=torch.int32, device="cuda"), x, x)
    pg, off = c.places(0, n)
    got = ref.take(c.k[0], pg, off).cpu().double()
    assert torch.equal(got, ref.quantise(x.cpu(), c.ks.cpu()))


def weights_of(kind, c, shape):
    w = torch.rand(shape, generator=c.g)
    if kind == "ties":
        w = torch.randint(0, 3, shape, generator=c.g).float() - 1.0
        w = torch.where(w == 0, torch.where(torch.rand(shape, generator=c.g) < 0.5, 0.0, -0.0), w)
    if kind == "equal":
        w = torch.full(shape, 0.25)
    if kind == "odd":
        u = torch.rand(shape, generator=c.g)
        w = torch.where(u < 0.1, math.nan, torch.where(u < 0.2, math.inf, torch.where(u < 0.3, -math.inf, w * 1e-40)))
    if kind == "wide":
        w = torch.exp(60 * torch.rand(shape, generator=c.g) - 30)
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd", "wide"])
@pytest.mark.parametrize("budget,n_sink,recent", [(1, 0, 0), (1, 0, 1), (40, 4, 16), (40, 8, 32), (128, 0, 0), (300, 16, 100)])
def test_evict_keeps_what_the_definition_keeps(kind, budget, n_sink, recent):
    lens = [300, 0, 1, 40, 41, 129, 1100, 128, 39]
    c = ref.Cache(lens, 4, 2, 64, 16 if kind == "plain" else 5, FP16, layers=3, weighted=True, layout="nhd", seed=budget)
    c.fill()
    for r, n in enumerate(lens):
        for l in range(3):
            pg, off = c.places(r, n)
            ref.put(c.w[l], pg, off, weights_of(kind, c, (n, 2)))
            # slots that an earlier eviction has filled out of order
            order = torch.stack([torch.randperm(n, generator=c.g) for _ in range(2)], 1).to(torch.int32)
            ref.put(c.pos[l], pg, off, order + 1000 if l == 2 else order)
    want, new = ref.evict(c, lens, budget, n_sink, recent, [1, 2])
    lp = c.handle()
    got = c.lens() if kind == "ties" else torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    lp.ltri_paged_evict(1, 2, c.table, got if kind == "ties" else c.lens(), got, budget, n_sink, recent)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert got.tolist() == new
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


@pytest.mark.parametrize("n,budget,e4m3,dim,hkv", [(9000, 4100, False, 128, 2), (20000, 64, True, 64, 1),
                                                 (4097, 4096, True, 256, 4),
                                                   (70000, 60000, False, 64, 1), (230000, 90000, True, 64, 1)])
def test_evict_of_long_rows(n, budget, e4m3, dim, hkv):
    c = ref.Cache([n, n // 2], hkv, hkv, dim, 16, BF16, e4m3, weighted=True, seed=n)
    c.fill()
    want, new = ref.evict(c, c.lens_cpu, budget, 16, budget // 3, [0])
    lp = c.handle()
    got = torch.zeros(2, dtype=torch.int32, device="cuda")
    lp.ltri_paged_evict(0, 1, c.table, c.lens(), got, budget, 16, budget // 3)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert got.tolist() == new
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


def serve(e4m3, graph):
    """Prompts, an eviction, then steps within a budget, the steps as one captured graph or call by call (then every call is
    checked).  Returns everything at the end."""
    c = ref.Cache([50, 0, 33], 8, 2, 128, 16, BF16, e4m3, layers=2, weighted=True, room=4, seed=21)
    lp = c.handle(weight_decay=0.9)
    lens, budget = c.lens_cpu, 40
    starts = torch.tensor([0, 50, 50, 83], dtype=torch.int32, device="cuda")
    dev, used = c.lens(), torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    w = torch.rand(83, 2, generator=c.g).cuda()
    for l in range(2):
        lp.ltri_paged_append(l, c.table, dev, starts, c.randn(83, 2, 128), c.randn(83, 2, 128), weights=w)

    def evict():
        lp.ltri_paged_evict(0, 2, c.table, dev, dev, budget, 4, 10)

    def check_evict(want, lens):
        assert dev.tolist() == lens
        for name, t in c.snapshot().items():
            assert torch.equal(t, want[name]), name

    want, lens = ref.evict(c, lens, budget, 4, 10, range(2))
    evict()
    check_evict(want, lens)
    row_pos = torch.tensor([50, 0, 33], dtype=torch.int32, device="cuda")
    q, kv = [c.randn(3, 8, 128) for _ in range(2)], [c.randn(3, 4, 128) for _ in range(2)]
    out, lse = [torch.zeros_like(t) for t in q], [torch.zeros(3, 8, device="cuda") for _ in range(2)]

    def decode_layer(l):
        lp.ltri_paged_decode(l, c.table, dev, q[l], kv[l][:, :2], kv[l][:, 2:], row_pos=row_pos, out=out[l], lse=lse[l])

    captured = torch.cuda.CUDAGraph()
    if graph:
        before, side = c.snapshot(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(captured, stream=side):
            dev.add_(used)
            decode_layer(0)
            decode_layer(1)
            evict()
            row_pos.add_(used)
        assert all(torch.equal(x, before[n]) for n, x in c.snapshot().items())  # (capturing runs nothing)
    for _ in range(12):
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
            ref.check_decode(c, l, q[l], out[l], lse[l], lens, old, 0.9, True)
        want, lens = ref.evict(c, lens, budget, 4, 10, range(2))
        evict()
        check_evict(want, lens)
        row_pos.add_(used)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    return {**c.snapshot(), "out": ref.bits(out[1]), "lse": ref.bits(lse[1]), "lens": dev.clone()}


@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_then_steps_within_a_budget_eager_and_captured(e4m3):
    eager, replayed = serve(e4m3, False), serve(e4m3, True)
    for name in eager:
        assert torch.equal(eager[name], replayed[name]), name


def test_handles_on_two_streams_at_once_and_a_stream_of_ones_own():
    cs = [ref.Cache([3000, 500], 8, 2, 128, 16, BF16, weighted=True, seed=s) for s in (1, 2)]
    lps, qs, want = [], [], []
    for c in cs:
        c.fill()
        lps.append(c.handle())
        qs.append(c.randn(2, 8, 128))
    start = [c.w.clone() for c in cs]
    for c, lp, q in zip(cs, lps, qs):
        want.append((lp.ltri_paged_decode(0, c.table, c.lens(), q).clone(), c.w.clone()))
    lens = [c.lens() for c in cs]
    for c, w in zip(cs, start):
        c.w.copy_(w)
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got = [lp.ltri_paged_decode(0, c.table, n, q, stream=s) for c, lp, q, s, n in zip(cs, lps, qs, streams, lens)]
    torch.cuda.synchronize()
    for c, g, (o, w), w0 in zip(cs, got, want, start):
        assert torch.equal(g, o)
        pg, off = c.places(0, 3000)
        once, many = ref.take(w[0] - w0[0], pg, off), ref.take(c.w[0] - w0[0], pg, off)
        assert torch.allclose(many, 20 * once, rtol=1e-3, atol=1e-4)
    s = streams[0]
    with torch.cuda.stream(s):
        g = lps[0].ltri_paged_decode(0, cs[0].table, lens[0], qs[0])
    s.synchronize()
    assert torch.equal(g, want[0][0])


def test_offsets_beyond_32_bits():
    # pages 4 MiB apart (a view of one page in 64 of a larger tensor): the last ones lie 5 GiB behind the first
    base = torch.zeros(1300, 1 << 21, dtype=BF16, device="cuda")
    k, v = (base.as_strided((1, 1300, 2, 16, 64), (0, 1 << 21, 1024, 64, 1), at) for at in (0, 4096))
    lp = binding.LtriPaged(k, v, 4, max_rows=1)
    table = torch.tensor([[1299, 0, 700]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([41], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(2)
    x, y = (torch.randn(41, 2, 64, generator=g).to(BF16).cuda() for _ in range(2))
    lp.ltri_paged_append(0, table, lens, torch.tensor([0, 41], dtype=torch.int32, device="cuda"), x, y)
    q = torch.randn(1, 4, 64, generator=g).to(BF16).cuda()
    out = lp.ltri_paged_decode(0, table, lens, q)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert torch.equal(k[0, 1299, :, 5], x[5]) and torch.equal(v[0, 700, :, 8], y[40])
    o, _, _, tol, _, _ = ref.attend(q[0].cpu().double(), x.cpu().double(), y.cpu().double(), 0.125)
    assert ((out[0].cpu().double() - o).abs() <= o.abs() * 2.0 ** -8 + 2 * tol).all()


def test_the_longest_row_and_tables_for_longer_ones():
    # 32767 times the same page of 65536 slots: the softmax is that of one page, its log-sum larger by log(32767)
    c = ref.Cache([65536], 1, 1, 64, 65536, BF16, seed=5)
    c.fill()
    lp = c.handle()
    q = c.randn(1, 1, 64)
    one = torch.empty(1, 1, device="cuda")
    out1 = lp.ltri_paged_decode(0, c.table, c.lens(), q, lse=one)
    table = c.table[:, :1].repeat(1, 32767).contiguous()
    lens = torch.full((1,), 32767 * 65536, dtype=torch.int32, device="cuda")
    many = torch.empty(1, 1, device="cuda")
    out = lp.ltri_paged_decode(0, table, lens, q, lse=many)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    # a warp adds up 2^27 / 1184 < 113400 tiles one after the other; a tile's sum may lose 2^-23 of what is there, its two
    # products with V as much each, and the output is the quotient, rounded
    slack, most = 113400 * 2.0 ** -23, float(c.v[0, int(c.table_cpu[0, 0])].float().abs().max())
    assert abs(float(many) - float(one) - math.log(32767)) < slack
    assert float((out.float() - out1.float()).abs().max()) < (3 * slack + 2.0 ** -8) * most
    # a table that could hold one slot more, and one of the largest row that 31 bits count, whatever the lengths are
    for cols, page in ((32768, 65536), (2 ** 31 - 2 ** 16 + 1, 1), (2 ** 31 - 1, 1)):
        d = ref.Cache([1], 1, 1, 64, page, BF16, seed=5)
        h, n = d.handle(), d.lens()
        rc = binding.load().ltri_paged_decode(h._h, 0, d.table.data_ptr(), cols, cols, n.data_ptr(), 1, q.data_ptr(), 0, None,
                                              None, 0, None, out.data_ptr(), None, None)
        assert rc == binding.LTRI_ECAPACITY and h.ltri_paged_launch_count() == 0


def test_calls_are_refused_before_anything_is_launched():
    c = ref.Cache([20, 30], 4, 2, 64, 16, BF16, weighted=True, seed=1)
    c.fill()
    lp = c.handle()
    before, launches = c.snapshot(), lp.ltri_paged_launch_count()
    q, k, lens = c.randn(2, 4, 64), c.randn(2, 2, 64), c.lens()
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    out, raw, h, s = torch.empty_like(q), binding.load(), lp._h, None
    cols = c.table.shape[1]
    rows = (p(c.table), cols, cols, p(lens))

    def decode_rc(layer=0, rows=rows, n=2, q=p(q), qs=0, k=p(k), v=p(k), ks=0, pos=None, out=p(out), lse=None):
        return raw.ltri_paged_decode(h, layer, *rows, n, q, qs, k, v, ks, pos, out, lse, s)

    def append_rc(layer=0, n=2, starts=p(starts), tokens=2, k=p(k), stride=0, pos=None, w=None):
        return raw.ltri_paged_append(h, layer, *rows, n, starts, tokens, k, k, stride, pos, w, s)

    def evict_rc(begin=0, count=1, new=p(lens), n=2, budget=8, sink=0, recent=0):
        return raw.ltri_paged_evict(h, begin, count, *rows, new, n, budget, sink, recent, s)

    for kw in (dict(layer=-1), dict(layer=1), dict(n=0), dict(q=None), dict(q=p(q) + 2), dict(qs=4), dict(qs=257), dict(k=None),
               dict(v=None), dict(v=p(k) + 8), dict(ks=64), dict(ks=132), dict(pos=p(lens) + 1), dict(out=None),
               dict(out=p(out) + 8),
               dict(lse=p(out) + 2), dict(rows=(None, cols, cols, p(lens))), dict(rows=(p(c.table), 0, cols, p(lens))),
               dict(rows=(p(c.table), cols, cols - 1, p(lens))), dict(rows=(p(c.table), cols, cols, None)),
               dict(rows=(p(c.table), cols, -4, p(lens)))):
        assert decode_rc(**kw) == binding.LTRI_EINVAL, kw
    assert decode_rc(n=3) == binding.LTRI_ECAPACITY
    # more tiles than 32 bits count (the table's columns say how many there may be)
    assert decode_rc(rows=(p(c.table), 1 << 30, 1 << 30, p(lens))) == binding.LTRI_ECAPACITY
    for kw in (dict(layer=1), dict(starts=None), dict(tokens=-1), dict(k=None), dict(k=p(k) + 2), dict(stride=64),
               dict(stride=129),
               dict(n=0), dict(w=p(lens) + 2)):
        assert append_rc(**kw) == binding.LTRI_EINVAL, kw
    assert append_rc(n=3) == binding.LTRI_ECAPACITY and append_rc(tokens=1 << 31) == binding.LTRI_ECAPACITY
    for kw in (dict(begin=-1), dict(begin=1), dict(count=0), dict(count=2), dict(new=None), dict(budget=0), dict(sink=-1),
               dict(recent=-1), dict(sink=4, recent=5), dict(n=0), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert evict_rc(**kw) == binding.LTRI_EINVAL, kw
    for kw in (dict(table=c.table.long()), dict(table=c.table.cpu()), dict(lens=lens[:1]), dict(q=q.half()), dict(q=q[:1]),
               dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(v=None), dict(k=k[:, :1]), dict(out=q.float()),
               dict(lse=torch.empty(2, 4)), dict(row_pos=lens.long())):
        with pytest.raises(ValueError):
            lp.ltri_paged_decode(**{**dict(layer=0, table=c.table, lens=lens, q=q, k=k, v=k), **kw})
    with pytest.raises(ValueError):
        lp.ltri_paged_append(0, c.table, lens, starts[:2], k, k)
    with pytest.raises(binding.LtriError):
        lp.ltri_paged_evict(0, 1, c.table, lens, lens, 4, 3, 3)
    torch.cuda.synchronize()
    assert lp.ltri_paged_launch_count() == launches
    for name, t in c.snapshot().items():
        assert torch.equal(t, before[name]), name
    plain = ref.Cache([20], 4, 2, 64, 16, BF16)
    with pytest.raises(binding.LtriError):  # nothing to evict by
        plain.handle().ltri_paged_evict(0, 1, plain.table, plain.lens(), plain.lens(), 8, 0, 0)
    with pytest.raises(ValueError):
        binding.LtriPaged(c.k, c.v.half(), 4)
    with pytest.raises(ValueError):
        binding.LtriPaged(c.k, c.v, 4, weights=c.w)
    with pytest.raises(binding.LtriError):
        binding.LtriPaged(c.k, c.v, 3)
