"""V rows that are not finite, in slots that some of a call's tokens see and others do not: a token's outputs depend on its own slots
alone.  (Keys: test_gpu_paged_attend.py.)"""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests.test_gpu_paged_attend import KINDS, ints, make, starts_of

pytestmark = pytest.mark.gpu


def spoil(c, r, slot, head, el, bad):
    """Element `el` of a slot's V row is `bad` (8 bits: NaN; 4 bits: its block's scale is).  Returns the elements that it spoils."""
    page, off = int(c.table_cpu[r, slot // c.page]), slot % c.page
    if c.v.dtype == torch.uint8:
        c.sc[0, page, head, off, 1, el // 32] = 0xFC
        return slice(el // 32 * 32, el // 32 * 32 + 32)
    if c.v.dtype == torch.float8_e4m3fn:
        c.v.view(torch.uint8)[0, page, head, off, el] = 0xFF
    else:
        c.v[0, page, head, off, el] = bad
    return slice(el, el + 1)


def check(kind, lens, news, hq, hkv, dim, page, spots, layout="hnd"):
    """spots: (row, slot, KV head, element, value)"""
    c = make(kind, lens, hq, hkv, dim, page, layout=layout, seed=7)
    c.fill()
    total, starts = sum(news), starts_of(news)
    lp, q = c.handle(max_tokens=total), c.randn(total, hq, dim)
    lse, lse1 = torch.empty(total, hq, device="cuda"), torch.empty(total, hq, device="cuda")
    want = lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, lse=lse)
    nan = torch.zeros(want.shape, dtype=torch.bool, device="cuda")
    for r, slot, head, el, bad in spots:
        els = spoil(c, r, slot, head, el, bad)
        first = max(0, slot - (lens[r] - news[r]))  # of the row's tokens that sees the slot
        nan[starts[r] + first:starts[r + 1], head * c.G:(head + 1) * c.G, els] = True
    got = lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, lse=lse1)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    assert torch.equal(lse, lse1)
    assert nan.any() and not nan.all()
    assert not got[nan].isfinite().any()
    wrong = (got != want) & ~nan
    assert not wrong.any(), f"{int(wrong.sum())} of {wrong.numel()}, first at {wrong.nonzero()[0].tolist()}"


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", KINDS)
def test_values_that_a_token_does_not_see(kind, dim):
    # tokens 100 to 299 of a row, and a whole prompt: the first, middle and last slots of units, tiles and pages
    check(kind, [300, 257, 40], [200, 257, 1], 4, 2, dim, 16,
          [(0, 101, 0, 3, math.nan), (0, 180, 1, dim - 1, math.inf), (0, 299, 0, dim // 2, -math.inf), (1, 0, 0, 5, math.nan),
           (1, 63, 0, 40, math.inf), (1, 64, 1, 32, math.nan), (1, 128, 0, 41, math.nan), (1, 256, 1, 0, math.nan),
           (2, 7, 1, 9, math.nan)])


@pytest.mark.parametrize("kind", KINDS)
def test_drafted_tokens_behind_a_bad_one(kind):
    # five drafted tokens of 24 rows, of which the second or the last has a V row of NaN
    lens = [100 + 61 * i for i in range(24)]
    check(kind, lens, [5] * 24, 32, 8, 128, 7, [(r, lens[r] - (4 if r % 2 else 1), r % 8, 17 * r % 128, math.nan)
                                               for r in range(0, 24, 3)], layout="nhd")


@pytest.mark.parametrize("kind,dim,hq,hkv", [("bf16", 128, 8, 2), ("fp16", 64, 6, 1), ("int4-bf16", 256, 4, 2), ("e4m3-fp16", 128, 2, 2),
                                             ("int4-fp16", 128, 64, 1)])
def test_values_not_seen_in_rows_split_over_ctas(kind, dim, hq, hkv):
    n, m = 30011, 700
    check(kind, [n], [m], hq, hkv, dim, 64, [(0, n - m + k, k % hkv, 13 * k % dim, math.nan) for k in (1, 250, 255, 256, 511, 640, 699)])


@pytest.mark.parametrize("kind", ["fp16", "bf16", "int4-bf16"])
def test_values_not_seen_in_long_units_of_one_cta(kind):
    # (more units than CTAs, each longer than what O adds up at a time)
    lens = [10100 - 3 * r for r in range(10)]
    check(kind, lens, [9] * 10, 16, 16, 64, 128, [(r, lens[r] - 1 - r % 9, (3 * r) % 16, 5 * r, math.nan) for r in range(10)])


@pytest.mark.parametrize("kind", ["bf16", "e4m3-bf16", "int4-fp16"])
def test_values_that_all_tokens_see_spoil_their_element_alone(kind):
    check(kind, [500, 90], [130, 20], 8, 2, 128, 16, [(0, 10, 0, 3, math.nan), (0, 369, 1, 77, math.nan), (1, 0, 1, 127, math.nan)])
