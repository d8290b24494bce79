"""Reading 8-bit pages back rounds element * scale once.  The product of a 4-bit and a 24-bit significand has up to 28 bits; where
fp32's rounding of it lies on a midpoint of two values of the model's type, a second rounding may go the wrong way."""
import math

import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_reference as ref

BF16, FP16 = torch.bfloat16, torch.float16


def rounded(x, dtype):
    """64-bit values to the nearest of `dtype`, ties to even, infinite beyond the largest."""
    bits, low = (8, -126) if dtype == BF16 else (11, -14)
    e = (torch.frexp(x)[1] - 1).clamp(min=low)
    step = torch.ldexp(torch.ones_like(x), e - (bits - 1))
    y = torch.round(x / step) * step
    return torch.where(y.abs() > torch.finfo(dtype).max, torch.copysign(torch.full_like(y, math.inf), y), y)


def hard_scales(dtype, n, seed):
    """(element, scale) pairs whose product in fp32 is a midpoint of `dtype`'s values and whose exact product is not."""
    g = torch.Generator().manual_seed(seed)
    bits, low, high = (8, -134, 120) if dtype == BF16 else (11, -25, 14)
    out = []
    while len(out) < n:
        e = int(torch.randint(low, high + 1, (1,), generator=g))
        e = [e, low + 3, high, 0][int(torch.randint(0, 4, (1,), generator=g))]
        at = max(e, -126 if dtype == BF16 else -14)  # (subnormals have the smallest normals' spacing)
        step = 2.0 ** (at - (bits - 1))
        mid = (math.floor(2.0 ** e * (1 + float(torch.rand(1, generator=g))) / step) + 0.5) * step
        x = float(torch.tensor([3.0, 5.0, 7.0, 11.0, 13.0, 0.9375, 1.375, 240.0, 416.0])[torch.randint(0, 9, (1,), generator=g)])
        s = torch.tensor(mid / x, dtype=torch.float32)
        for s in (s, torch.nextafter(s, torch.tensor(0.0)), torch.nextafter(s, torch.tensor(math.inf))):
            exact = x * float(s)
            if float(torch.tensor(x) * s) == mid and exact != mid and len(out) < n:
                out.append((x * (-1 if len(out) % 3 == 0 else 1), float(s)))
    return out


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_such_products_tell_one_rounding_from_two(dtype):
    pairs = hard_scales(dtype, 128, 1)
    exact = torch.tensor([x * s for x, s in pairs], dtype=torch.float64)
    twice = torch.tensor([x for x, _ in pairs]) * torch.tensor([s for _, s in pairs])
    assert (rounded(exact, dtype) != twice.to(dtype).double()).sum() >= 32
    # what the helper gives for values of every kind is what a single rounding from fp32 gives
    some = torch.randn(10000, dtype=torch.float32) * torch.exp2(torch.randint(-140, 128, (10000,)).float())
    assert torch.equal(rounded(some.double(), dtype), some.to(dtype).double())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_read_rounds_once(dtype):
    hkv, n = 64, 9
    pairs = [hard_scales(dtype, hkv, seed) for seed in (1, 2)]
    c = ref.Cache([n], hkv, hkv, 64, 4, dtype, e4m3=True, seed=3)
    pg, off = c.places(0, n)
    for pages, scale, pair in ((c.k, c.ks, pairs[0]), (c.v, c.vs, pairs[1])):
        scale.copy_(torch.tensor([s for _, s in pair]))
        rows = torch.randn(n, hkv, 64, generator=c.g).to(ref.E4M3)
        rows[:, :, ::2] = torch.tensor([x for x, _ in pair]).to(ref.E4M3)[None, :, None]
        ref.put(pages[0], pg, off, rows)
    lp = c.handle()
    got = [torch.empty(n, hkv, 64, dtype=dtype, device="cuda") for _ in range(2)]
    lp.ltri_paged_read(0, c.table, c.lens(), torch.tensor([0, n], dtype=torch.int32, device="cuda"), *got)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    for x, want in zip(got, c.row(0, 0, n)):
        assert torch.equal(x.cpu().double(), rounded(want, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_read_of_every_element(dtype):
    # all 256 bytes at scales over fp32's whole range: zeros keep their sign, NaN stays NaN, what is too large is infinite
    hkv, n = 16, 4
    c = ref.Cache([n], hkv, hkv, 64, 4, dtype, e4m3=True, seed=4)
    scales = torch.exp2(torch.linspace(-149, 120, hkv)) * torch.linspace(1, 1.99, hkv)
    every = torch.arange(256, dtype=torch.uint8).view(n, 1, 64).expand(n, hkv, 64).contiguous().view(ref.E4M3)
    pg, off = c.places(0, n)
    for pages, s in ((c.k, c.ks), (c.v, c.vs)):
        s.copy_(scales)
        ref.put(pages[0], pg, off, every)
    lp = c.handle()
    got = torch.empty(n, hkv, 64, dtype=dtype, device="cuda")
    lp.ltri_paged_read(0, c.table, c.lens(), torch.tensor([0, n], dtype=torch.int32, device="cuda"), got)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    want = every.double() * c.ks.cpu().double()[None, :, None]
    nan = want.isnan()
    got = got.cpu().double()
    assert torch.equal(got.isnan(), nan)
    assert torch.equal(got[~nan], rounded(want[~nan], dtype))
    assert torch.equal(torch.signbit(got[~nan]), torch.signbit(want[~nan]))
