"""Waits of attention over a paged cache that run out: the call ends, says so once, and the next one is as ever."""
import pytest
import torch

from paper_2412_04757_b200 import binding
from tests.test_gpu_paged_attend import ints, make, starts_of

pytestmark = pytest.mark.gpu

LIMIT = 200_000  # SM cycles: a tenth of a millisecond


@pytest.mark.parametrize("held", [1, 2, 3])
@pytest.mark.parametrize("kind,dim,hq,hkv", [("bf16", 128, 8, 2), ("e4m3-bf16", 64, 4, 4), ("int4-fp16", 256, 4, 1),
                                             ("int4-bf16", 128, 32, 2)])
def test_a_wait_that_runs_out_ends_the_call(kind, dim, hq, hkv, held):
    # whole units and parts of them, rows of few tokens and of many
    lens, news = [700, 3, 0, 2600, 130], [300, 3, 0, 5, 130]
    c = make(kind, lens, hq, hkv, dim, 16, seed=dim)
    c.fill()
    total, starts = sum(news) + 3, starts_of(news, 2)
    lp, q = c.handle(max_tokens=total), c.randn(total, hq, dim)
    before = c.snapshot()
    out, lse = torch.full_like(q, 5.0), torch.full((total, hq), 7.0, device="cuda")
    want = [x.clone() for x in (lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, out=out, lse=lse), lse)]
    for _ in range(2):
        lp.ltri_paged_debug_wait(LIMIT, held)
        lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, out=out, lse=lse)
        assert lp.ltri_paged_sync_status() == binding.LTRI_ETIMEOUT and lp.ltri_paged_sync_status() == binding.LTRI_OK
        assert (out[:2] == 5.0).all() and (out[-1:] == 5.0).all() and (lse[:2] == 7.0).all() and (lse[-1:] == 7.0).all()
        lp.ltri_paged_debug_wait()
        lp.ltri_paged_attend(0, c.table, c.lens(), ints(starts), q, out=out, lse=lse)
        assert lp.ltri_paged_sync_status() == binding.LTRI_OK
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert all(torch.equal(x, before[name]) for name, x in c.snapshot().items())


def test_a_short_limit_alone_changes_nothing():
    c = make("int4-bf16", [3000, 40], 8, 2, 128, 16, seed=5)
    c.fill()
    lp, q = c.handle(max_tokens=240), c.randn(240, 8, 128)
    want = lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 200, 240]), q).clone()
    lp.ltri_paged_debug_wait(100_000_000)
    assert torch.equal(lp.ltri_paged_attend(0, c.table, c.lens(), ints([0, 200, 240]), q), want)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK


def test_limits_out_of_range_are_refused():
    lp = make("bf16", [4], 1, 1, 64, 4, seed=1).handle()
    for limit, held in ((-1, 0), (10 ** 8 + 1, 0), (1000, -1), (1000, 4), (0, 1)):
        with pytest.raises(binding.LtriError):
            lp.ltri_paged_debug_wait(limit, held)
    assert lp.lib.ltri_paged_debug_wait(None, 0, 0) == binding.LTRI_EINVAL
