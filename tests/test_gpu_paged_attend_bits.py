"""What attention of several new tokens per row keeps of its probabilities and sums, against the definition in 64 bits."""
import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import attend, ints, make

pytestmark = pytest.mark.gpu


def store(c, r, n, K, V):
    """K, V [n][Hkv][dim] into row r's slots, as the pages hold them."""
    pg, off = c.places(r, n)
    for which, (pages, x, s) in enumerate(((c.k, K, c.ks), (c.v, V, c.vs))):
        if pages.dtype == torch.uint8:
            c.store(0, pg, off, which, x)
        else:
            ref.put(pages[0], pg, off, (x if s is None else x / s.cpu()[:, None]).to(pages.dtype))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind,hq", [("e4m3-bf16", 8), ("e4m3-fp16", 8), ("int4-bf16", 8), ("int4-bf16", 16), ("int4-fp16", 8),
                                     ("fp16", 8), ("bf16", 8), ("bf16", 16)])
def test_probabilities_meet_v_with_all_their_bits(dim, kind, hq):
    # As for single tokens: three slots, one of logit 0 and V = 0, and two of logits -a and -a - 2^-14 or so with V = 1 and -1, which
    # leave some 2^-16 of probabilities of 0.5 to 1.  What an output may be off: two products make a logit, below 1 in log2
    # units, which is off by 2^-22 (their sum, scale * log2(e)) and a rounding of its distance to the reference, which is 2^-24
    # below 1, or 2^-20 where halves have their largest probability at 2^10 (half of the last place below 16 is 2^-21, times ln 2
    # less); exp2 by 2^-22; so p by 2^-21, or 2^-19.  Two terms of 11 bits hold p to 2^-22, two of 8 bits (over bf16 pages) to
    # 2^-16 by what is documented.  A product of a term of p with V may lose 2^-23 of what it is added to.
    rows = 64
    c = make(kind, [3] * rows, hq, 1, dim, 16, seed=dim)
    if c.ks is not None:
        c.ks.fill_(0.25)
        c.vs.fill_(0.25)
    q = torch.zeros(rows, hq, dim)
    q[..., 0] = 4.0 + 4.0 * torch.rand(rows, hq, generator=c.g)
    q[..., 40] = 2.0 ** -12 * (1 + torch.rand(rows, hq, generator=c.g))
    q = q.to(c.dtype)
    for r in range(rows):
        k, v = torch.zeros(3, 1, dim), torch.zeros(3, 1, dim)
        k[1:, 0, 0] = -0.1 - 0.5 * torch.rand(1, generator=c.g)
        k[2, 0, 40] = -4.0
        v[1], v[2] = 1.0, -1.0
        store(c, r, 3, k, v)
    lp = c.handle(softmax_scale=0.125, max_tokens=rows)
    out = lp.ltri_paged_attend(0, c.table, c.lens(), ints(list(range(rows + 1))), q.cuda()).cpu().double()
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    off = 2.0 ** -21 + 2.0 ** -16 if kind == "bf16" else 2.0 ** -19 + 2.0 ** -22
    for r in range(rows):
        K, V = c.row(0, r, 3)
        for h in range(hq):
            x = K[:, 0] @ q[r, h].double() * 0.125
            assert float(x.abs().max()) * 1.4427 < 1
            p = torch.exp(x) / torch.exp(x).sum()
            want, most = p @ V[:, 0], float(p[1:].max() * V.abs().max())
            # (fp16 outputs of 2^-16 are subnormal: half their spacing of 2^-24)
            bound = 2 * most * (off + 2.0 ** -23)
            bound = bound + (want.abs() * ref.HALF_STEP[c.dtype]).clamp(min=2.0 ** -25)
            assert ((out[r, h] - want).abs() <= bound).all(), (r, h)


@pytest.mark.parametrize("power", [110, -110])
def test_values_of_the_stated_range(power):
    # 300 slots of |V| up to 6 times 2^110: 16 times their sum is 2^125, 4 * 10^37
    c = make("bf16", [300, 40], 8, 2, 128, 16, seed=9)
    c.fill()
    c.v.mul_(2.0 ** power)
    attend(c, [130, 40])


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("e4m3-bf16", 128), ("int4-bf16", 64), ("fp16", 64)])
def test_sums_that_rise_and_fall(kind, dim):
    # 148 rows over the same 2^16 slots, all but the last of which hold values of one sign and those 64 times as large ones of the
    # other: sums rise along the row, and what the additions have cut off (towards zero) stays when the last slots have brought them
    # back to where outputs and their roundings are small.  Documented is 2^-14 of a sum of one sign: of the rise, half of the
    # values' sum without their signs, and as much again for the fall.
    n, m, rows = 1 << 16, 64, 148
    c = make(kind, [n], 4, 1, dim, 128, seed=dim)
    if c.ks is not None:
        c.ks.fill_(0.25)
        c.vs.fill_(0.25)
    K, V = torch.randn(n, 1, dim, generator=c.g), torch.rand(n, 1, dim, generator=c.g) + 0.5
    V[n - m - 1024:n - m] = -64 + V[:1024]
    store(c, 0, n, K, V)
    lp, q = c.handle(max_rows=rows, max_tokens=rows * m), c.randn(rows * m, 4, dim, scale=0.25)
    starts = ints([m * r for r in range(rows + 1)])
    out = lp.ltri_paged_attend(0, c.table.repeat(rows, 1), ints([n] * rows), starts, q)
    assert lp.ltri_paged_sync_status() == binding.LTRI_OK
    K, V = (x[:, 0].cuda() for x in c.row(0, 0, n))
    seen = torch.arange(n, device="cuda") <= (n - m + torch.arange(m, device="cuda"))[:, None]
    for r in (0, 70, 147):
        for h in range(4):
            logits = torch.where(seen, q[m * r:m * r + m, h].double() @ K.T * dim ** -0.5, -float("inf"))
            p = torch.softmax(logits, -1)
            want, size = p @ V, p @ V.abs()
            off = (out[m * r:m * r + m, h].double() - want).abs() - want.abs() * ref.HALF_STEP[c.dtype]
            assert float(off.mean()) <= 2.0 ** -14 * float(size.mean()), (r, h, float(off.mean() / size.mean()))
