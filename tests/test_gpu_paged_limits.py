"""The paged cache's operators where the first tests of them do not reach: calls at the borders of what the header allows."""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("n,budget", [(300, 100), (230000, 90000)])
def test_rows_that_share_evicted_pages_are_undefined_but_in_bounds(n, budget):
    # shared memory holds the shorter rows' keys, the longer ones' are read again while the other row moves its slots
    c = ref.Cache([n, n - 11, 50], 1, 1, 64, 16, BF16, True, weighted=True, seed=n)
    c.fill()
    shared = c.table_cpu[0].clone()
    own = torch.zeros(c.n_pages, dtype=torch.bool)
    own[shared.long()[:-(-n // 16)]] = True
    table = torch.stack([shared, shared, c.table_cpu[2]]).cuda()
    lp, before = c.handle(), c.snapshot()
    for _ in range(3):
        got = torch.zeros(3, dtype=torch.int32, device="cuda")
        lp.ltri_paged_evict(0, 1, table, c.lens(), got, budget, 16, 20)
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        assert got.tolist() == [budget, budget, 50]
    for name, x in c.snapshot().items():
        assert torch.equal(x[0][~own.cuda()], before[name][0][~own.cuda()]), name
    # and the handle is as it was: rows of their own afterwards are cut as the definition says
    c.fill()
    want, new = ref.evict(c, c.lens_cpu, budget, 16, 20, [0])
    lp.ltri_paged_evict(0, 1, c.table, c.lens(), got, budget, 16, 20)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK and got.tolist() == new
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


def test_new_lengths_over_other_rows_lengths_are_refused():
    c = ref.Cache([40, 30, 20], 2, 1, 64, 16, FP16, weighted=True, room=4, seed=2)
    c.fill()
    lp, before = c.handle(), c.snapshot()
    both = torch.tensor([40, 30, 20, 7, 7, 7, 7], dtype=torch.int32, device="cuda")
    for lens, new in ((both[:3], both[1:4]), (both[:3], both[2:5]), (both[1:4], both[:3]), (both[2:5], both[:3])):
        with pytest.raises(binding.LtriError) as e:
            lp.ltri_paged_evict(0, 1, c.table, lens, new, 8, 1, 1)
        assert e.value.code == binding.LTRI_EINVAL
    torch.cuda.synchronize()
    assert lp.ltri_paged_launch_count() == 0 and both.tolist() == [40, 30, 20, 7, 7, 7, 7]
    for name, x in c.snapshot().items():
        assert torch.equal(x, before[name]), name
    want, _ = ref.evict(c, [40, 30, 20], 8, 1, 1, [0])
    lp.ltri_paged_evict(0, 1, c.table, both[:3], both[3:6], 8, 1, 1)  # side by side
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK and both.tolist() == [40, 30, 20, 8, 8, 8, 7]
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


def test_a_handle_made_on_another_stream_while_the_current_one_is_busy():
    c = ref.Cache([3000, 500, 70], 8, 2, 128, 16, BF16, weighted=True, seed=3)
    c.fill()
    q, start, lens = c.randn(3, 8, 128), c.w.clone(), c.lens()
    lp = c.handle()
    want = lp.ltri_paged_decode(0, c.table, lens, q).clone()
    nbytes = lp.workspace.numel()
    weights = c.w.clone()
    c.w.copy_(start)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    del lp
    # a block of the workspace's size, freed while its stream still has writes to it before it
    block = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda._sleep(200_000_000)
    block.fill_(1)
    del block
    lp = c.handle(stream=side)
    torch.cuda.synchronize()
    got = lp.ltri_paged_decode(0, c.table, lens, q)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert torch.equal(got, want) and torch.equal(ref.bits(c.w), ref.bits(weights))
    new = torch.zeros_like(lens)
    lp.ltri_paged_evict(0, 1, c.table, lens, new, 100, 4, 10)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK and new.tolist() == [100, 100, 70]


def check_step(c, lens, q, decay=1.0, **kw):
    """One decode call over the cache as it is, compared with the definition."""
    before, lse = None if c.w is None else c.w.clone(), torch.full(q.shape[:2], 7.0, device="cuda")
    lp = c.handle(**kw)
    out = lp.ltri_paged_decode(0, c.table, c.lens(), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    ref.check_decode(c, 0, q, out, lse, lens, before, decay)
    return out, lse


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("k_scale,q_scale", [(1e-40, 1.0), (2.0 ** -126 / 448, 1.0), (0.02, 2.0 ** -124), (3e-39, 2.0 ** -60),
                                             (2.0 ** 100, 2.0 ** -124), (1e-40, 2.0 ** 125)])
def test_logits_whose_factor_lies_below_fp32s_range(dim, k_scale, q_scale):
    # scale * k_scale * the queries' power of two: the logits are what they are, and slots behind a row's end stay outside
    c = ref.Cache([1, 17, 40, 300, 33, 64], 4, 2, dim, 16, BF16, True, weighted=True, seed=dim)
    c.fill()
    c.ks = torch.full_like(c.ks, k_scale)
    q = (torch.randn(6, 4, dim, generator=c.g).clamp(-3.5, 3.5) * q_scale).to(BF16).cuda()
    check_step(c, c.lens_cpu, q)


@pytest.mark.parametrize("v_scale", [1e-40, 2.0 ** -126 / 448, 1e-38, 2.0 ** 110])
@pytest.mark.parametrize("n", [1, 8, 100, 5000])
def test_values_whose_scale_is_at_the_ends_of_fp32s_range(n, v_scale):
    # outputs that are normal numbers of their type, from scales that are not: all slots' logits are zero, V is 320 or 384, so
    # that nothing cancels.  n = 5000: parts of several CTAs are joined.
    c = ref.Cache([n], 2, 1, 64, 16, BF16, True, seed=n)
    pg, off = c.places(0, n)
    v = torch.where(torch.rand(n, 1, 64, generator=c.g) < 0.5, 320.0, 384.0)
    ref.put(c.k[0], pg, off, torch.ones(n, 1, 64).to(ref.E4M3))
    ref.put(c.v[0], pg, off, v.to(ref.E4M3))
    c.vs = torch.full_like(c.vs, v_scale)
    check_step(c, [n], torch.zeros(1, 2, 64, dtype=BF16, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("hq,hkv", [(4, 2), (3, 1)])
def test_rows_whose_logits_are_all_minus_infinity(dtype, hq, hkv):
    # the softmax of nothing, as of an empty row: out 0, lse -infinity, and the slots get no weight; rows beside are as they were
    lens = [20, 3000, 40]
    c = ref.Cache(lens, hq, hkv, 64, 16, dtype, weighted=True, seed=hq)
    c.fill()
    for r in (0, 1):
        pg, off = c.places(r, lens[r])
        k = torch.randn(lens[r], hkv, 64, generator=c.g)
        k[..., 0] = -math.inf
        ref.put(c.k[0], pg, off, k.to(dtype))
    q = c.randn(3, hq, 64)
    q[:, :, 0] = 1.0
    before, lse = c.w.clone(), torch.zeros(3, hq, device="cuda")
    lp = c.handle(weight_decay=0.5)
    out = lp.ltri_paged_decode(0, c.table, c.lens(), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for r in (0, 1):
        pg, off = c.places(r, lens[r])
        assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
        assert torch.equal(ref.take(c.w[0], pg, off), 0.5 * ref.take(before[0], pg, off))
    c.lens_cpu = [0, 0, 40]
    ref.check_decode(c, 0, torch.cat([q[:2] * 0, q[2:]]), out, lse, c.lens_cpu, before, 0.5)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,hq", [(BF16, 8), (BF16, 16), (FP16, 8)])
def test_probabilities_meet_v_with_all_their_bits(dim, dtype, hq):
    # Three slots: one of logit 0 and V = 0, and two of logits -a and -a - 2^-14 or so with V = 1 and -1, which leave some
    # 2^-16 of probabilities of 0.5 to 1.  What an output may be off: two products make a logit, below 1 in log2 units, which
    # is off by 2^-22 (their sum, scale * log2(e)) and a rounding of 2^-24 of its distance to the maximum; exp2 by 2^-22; so p by
    # 2^-21.  A product of a term of p (up to three) with V may lose 2^-23 of what it is added to.
    rows = 64
    c = ref.Cache([3] * rows, hq, 1, dim, 16, dtype, seed=dim)
    q = torch.zeros(rows, hq, dim)
    q[..., 0] = 4.0 + 4.0 * torch.rand(rows, hq, generator=c.g)
    q[..., 1] = 2.0 ** -12 * (1 + torch.rand(rows, hq, generator=c.g))
    q = q.to(dtype)
    for r in range(rows):
        k, v = torch.zeros(3, 1, dim), torch.zeros(3, 1, dim)
        k[1:, 0, 0] = -0.1 - 0.5 * torch.rand(1, generator=c.g)
        k[2, 0, 1] = -4.0
        v[1], v[2] = 1.0, -1.0
        pg, off = c.places(r, 3)
        ref.put(c.k[0], pg, off, k.to(dtype))
        ref.put(c.v[0], pg, off, v.to(dtype))
    lp = c.handle(softmax_scale=0.125)
    out = lp.ltri_paged_decode(0, c.table, c.lens(), q.cuda()).cpu().double()
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for r in range(rows):
        K, V = c.row(0, r, 3)
        for h in range(hq):
            x = K[:, 0] @ q[r, h].double() * 0.125
            assert float(x.abs().max()) * 1.4427 < 1
            p = torch.exp(x)
            want, most = (p[1] - p[2]) / p.sum(), float(p[1] / p.sum())
            # (fp16 outputs of 2^-16 are subnormal: half their spacing of 2^-24)
            bound = 2 * most * 2.0 ** -21 + 3 * most * 2.0 ** -23 + max(abs(float(want)) * ref.HALF_STEP[dtype], 2.0 ** -25)
            assert float((out[r, h] - want).abs().max()) <= bound, (r, h)


@pytest.mark.parametrize("page,hkv", [(1, 1), (1, 2), (16, 1)])
def test_pages_with_axes_of_one_entry_at_any_stride(page, hkv):
    c = ref.Cache([40, 1, 17], 2 * hkv, hkv, 64, page, BF16, seed=page + hkv)
    c.fill()
    new = [1, c.k.stride(1), 3 if hkv == 1 else c.k.stride(2), 5 if page == 1 else c.k.stride(3), 1]
    c.k, c.v = c.k.as_strided(c.k.shape, new), c.v.as_strided(c.v.shape, new)
    q = c.randn(3, 2 * hkv, 64)
    check_step(c, c.lens_cpu, q)
    x, starts = c.randn(3, hkv, 64), torch.tensor([0, 1, 1, 3], dtype=torch.int32, device="cuda")
    lp = c.handle()
    lp.ltri_paged_append(0, c.table, c.lens(), starts, x, x)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    pg, off = c.places(2, 17)
    assert torch.equal(ref.take(c.k[0], pg[-2:], off[-2:]), x[1:]) and torch.equal(ref.take(c.v[0], pg[-2:], off[-2:]), x[1:])


def test_every_part_of_the_longest_row_is_in_its_output():
    # 32767 pages of 65536 slots, of four in memory that have the same keys: the first, one in the middle and the last one have
    # V of 2^15 in 16 elements each, the others none there, and all have 1 in the rest
    P, cols, dim = 65536, 32767, 64
    c = ref.Cache([4 * P], 1, 1, dim, P, BF16, seed=5)
    pages = c.table_cpu[0].long()
    k = torch.randn(P, 1, dim, generator=c.g).to(BF16)
    where = torch.arange(P, device="cuda")
    for i, page in enumerate(pages):
        v = torch.zeros(P, 1, dim)
        v[..., 48:] = 1.0
        if i > 0:
            v[..., 16 * (i - 1):16 * i] = 2.0 ** 15
        pg = torch.full((P,), int(page), device="cuda")
        ref.put(c.k[0], pg, where, k)
        ref.put(c.v[0], pg, where, v.to(BF16))
    table = torch.full((1, cols), int(pages[0]), dtype=torch.int32)
    table[0, 0], table[0, cols // 2], table[0, -1] = pages[1], pages[2], pages[3]
    lens = torch.full((1,), cols * P, dtype=torch.int32, device="cuda")
    q, lse = c.randn(1, 1, dim), torch.empty(1, 1, device="cuda")
    lp = c.handle()
    out = lp.ltri_paged_decode(0, table.cuda(), lens, q, lse=lse)[0, 0].cpu().double()
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    x = k[:, 0].double() @ q[0, 0].cpu().double() * dim ** -0.5
    d = float((k[:, 0].double().abs() @ q[0, 0].cpu().double().abs()).max()) * dim ** -0.5 * (dim + 8) * 2.0 ** -23
    # a warp adds up 2^27 / 1184 < 113400 tiles one after the other, for the sum of the probabilities two slots of each, rounded;
    # a product of one of three terms with V may lose 2^-23 of what it is added to, on 4096 tiles of a page or on all
    total, page, row = 2 * 113400 * 2.0 ** -24, 3 * 4096 * 2.0 ** -23, 3 * 113400 * 2.0 ** -23
    assert abs(float(lse) - float(torch.logsumexp(x, 0)) - math.log(cols)) < total + 2 * d
    want = torch.full((dim,), 2.0 ** 15 / cols, dtype=torch.float64)
    want[48:] = 1.0
    bound = torch.full((dim,), total + page, dtype=torch.float64)
    bound[48:] = total + row
    assert ((out / want - 1).abs() <= bound + 2 * d + 2.0 ** -8).all(), out


def test_outputs_over_other_rows_queries_are_refused():
    c = ref.Cache([40, 30, 20], 4, 2, 64, 16, FP16, seed=2)
    c.fill()
    lp, lens = c.handle(), c.lens()
    buf = c.randn(40 * 64).view(-1)
    at = lambda first, stride: buf[first * 64:].as_strided((3, 4, 64), (stride * 64, 64, 1))  # noqa: E731  (heads)
    want = lp.ltri_paged_decode(0, c.table, lens, at(0, 6).contiguous())
    launches, before = lp.ltri_paged_launch_count(), buf.clone()
    # (queries' first head and stride, outputs' first head): one over the other, over a row of it, over itself with gaps
    for first, stride, o in ((0, 4, 1), (4, 4, 0), (0, 6, 0), (0, 6, 15), (5, 6, 0), (0, 12, 4), (12, 4, 1)):
        with pytest.raises(binding.LtriError) as e:
            lp.ltri_paged_decode(0, c.table, lens, at(first, stride), out=at(o, 4))
        assert e.value.code == binding.LTRI_EINVAL
    torch.cuda.synchronize()
    assert lp.ltri_paged_launch_count() == launches and torch.equal(buf, before)
    # beside them, behind them, and between two rows that are far apart
    wide = torch.zeros(40 * 64, dtype=FP16, device="cuda")
    for first, stride, o in ((0, 6, 16), (12, 6, 0), (0, 16, 4)):
        x = wide[first * 64:].as_strided((3, 4, 64), (stride * 64, 64, 1))
        x.copy_(at(0, 6))
        got = lp.ltri_paged_decode(0, c.table, lens, x, out=wide[o * 64:].as_strided((3, 4, 64), (256, 64, 1)))
        assert torch.equal(got, want), (first, stride, o)
    x = at(0, 4)
    x.copy_(at(0, 6).contiguous())
    assert torch.equal(lp.ltri_paged_decode(0, c.table, lens, x, out=x), want)


@pytest.mark.parametrize("hq,hkv,dim,dtype,e4m3", [(64, 1, 128, BF16, False), (48, 2, 256, BF16, True), (40, 1, 64, FP16, False),
                                                   (34, 2, 256, FP16, False)])
@pytest.mark.parametrize("weighted", [False, True])
def test_wide_groups_split_over_many_ctas(hq, hkv, dim, dtype, e4m3, weighted):
    lens = [5000, 17, 0, 900]
    c = ref.Cache(lens, hq, hkv, dim, 16, dtype, e4m3, weighted=weighted, seed=hq)
    c.fill()
    check_step(c, lens, c.randn(4, hq, dim))


@pytest.mark.parametrize("rows,kind", [(1500, "short"), (300, "ragged")])
def test_batches_of_many_rows(rows, kind):
    g = torch.Generator().manual_seed(rows)
    top = 20 if kind == "short" else 600
    lens = [0 if i % 7 == 3 else int(torch.randint(1, top, (1,), generator=g)) for i in range(rows)]
    c = ref.Cache(lens, 4, 2, 64, 16, BF16, weighted=True, seed=rows)
    c.fill()
    lp = c.handle()
    q, before, lse = c.randn(rows, 4, 64), c.w.clone(), torch.zeros(rows, 4, device="cuda")
    out = lp.ltri_paged_decode(0, c.table, c.lens(), q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    ref.check_decode(c, 0, q, out, lse, lens, before)
    want, new = ref.evict(c, lens, 10, 2, 3, [0])
    got = c.lens()
    lp.ltri_paged_evict(0, 1, c.table, got, got, 10, 2, 3)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK and got.tolist() == new
    for name, x in c.snapshot().items():
        assert torch.equal(x, want[name]), name


def test_a_capture_whose_steps_come_from_two_streams():
    # a side stream prepares the new token's rows while the main one evicts; both are followed by the attention
    c = ref.Cache([50, 33], 8, 2, 64, 16, BF16, weighted=True, room=1, seed=4)
    c.fill()
    lp, dev, one = c.handle(), c.lens(), torch.ones(2, dtype=torch.int32, device="cuda")
    q, x, kv = c.randn(2, 8, 64), c.randn(2, 4, 64), torch.zeros(2, 4, 64, dtype=BF16, device="cuda")
    out = torch.zeros_like(q)
    graph, main, side = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        with torch.cuda.stream(side):
            kv.copy_(x)
        lp.ltri_paged_evict(0, 1, c.table, dev, dev, 40, 4, 8)
        dev.add_(one)
        main.wait_stream(side)
        lp.ltri_paged_decode(0, c.table, dev, q, kv[:, :2], kv[:, 2:], out=out)
    for step in range(3):
        x.copy_(c.randn(2, 4, 64))
        want, lens = ref.evict(c, dev.tolist(), 40, 4, 8, [0])
        w = want["w"].view(torch.float32)
        graph.replay()
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        lens = [n + 1 for n in lens]
        assert dev.tolist() == lens
        ref.check_decode(c, 0, q, out, None, lens, w, 1.0, True)
        pg, off = c.places(0, lens[0])
        assert torch.equal(ref.take(c.k[0], pg[-1:], off[-1:])[0], x[0, :2])


@pytest.mark.parametrize("dim,hq", [(64, 8), (128, 8), (256, 8), (64, 128), (128, 128), (256, 128)])
@pytest.mark.parametrize("dtype,e4m3", [(BF16, False), (FP16, False), (BF16, True)])
def test_small_values_survive_among_large_ones_that_cancel(dim, hq, dtype, e4m3):
    # All probabilities are equal.  1024 slots of V = B, 2048 of 2^-9 and 1024 of -B: a block of 16 of the small ones, 2^-5, is
    # exact beside the large ones' sum (1024 B < 2^19), and so are all sums of blocks, whoever adds them: what is left is
    # 2048 * 2^-9 of 4096 slots.  As many units as the GPU has warps at work, so that runs are whole rows.
    n, hkv, rows = 4096, 8, torch.cuda.get_device_properties(0).multi_processor_count
    c = ref.Cache([n], hq, hkv, dim, 16, dtype, e4m3, seed=dim)
    pg, off = c.places(0, n)
    v = torch.full((n, hkv, dim), 2.0 ** -9)
    v[:1024], v[-1024:] = (448.0, -448.0) if e4m3 else (128.0, -128.0)
    ref.put(c.k[0], pg, off, torch.zeros(n, hkv, dim).to(c.k.dtype))
    ref.put(c.v[0], pg, off, v.to(c.v.dtype))
    if e4m3:
        c.vs = torch.ones_like(c.vs)
    lp = c.handle(max_rows=rows)
    q, lse = c.randn(rows, hq, dim), torch.empty(rows, hq, device="cuda")
    lens = torch.full((rows,), n, dtype=torch.int32, device="cuda")
    out = lp.ltri_paged_decode(0, c.table.repeat(rows, 1), lens, q, lse=lse)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert (out == 2.0 ** -10).all() and float((lse - 12 * math.log(2.0)).abs().max()) < 2.0 ** -20
