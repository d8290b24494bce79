"""What attention of several new tokens per row keeps of its probabilities and sums, against the definition in 64 bits."""
import pytest
import torch

from paper_2412_04757_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import BF16, FP16, ints, make

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
                                     ("fp16", 8)])
def test_probabilities_meet_v_with_all_their_bits(dim, kind, hq):
    # As for single tokens: three slots, one of logit 0 and V = 0, and two of logits -a and -a - 2^-14 or so with V = 1 and -1, which
    # leave some 2^-16 of probabilities of 0.5 to 1.  What an output may be off: two products make a logit, below 1 in log2
    # units, which is off by 2^-22 (their sum, scale * log2(e)) and a rounding of its distance to the reference, which is 2^-24
    # below 1, or 2^-20 where halves have their largest probability at 2^10 (half of the last place below 16 is 2^-21, times ln 2
    # less); exp2 by 2^-22; so p by 2^-21, or 2^-19.  Two terms of 11 bits hold p to 2^-22, three of 8 bits to 2^-24.  A product
    # of a term of p (up to three) with V may lose 2^-23 of what it is added to.
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
    far = kind != "bf16"
    for r in range(rows):
        K, V = c.row(0, r, 3)
        for h in range(hq):
            x = K[:, 0] @ q[r, h].double() * 0.125
            assert float(x.abs().max()) * 1.4427 < 1
            p = torch.exp(x) / torch.exp(x).sum()
            want, most = p @ V[:, 0], float(p[1:].max() * V.abs().max())
            # (fp16 outputs of 2^-16 are subnormal: half their spacing of 2^-24)
            bound = 2 * most * ((2.0 ** -19 + 2.0 ** -22 if far else 2.0 ** -21 + 2.0 ** -24) + 1.5 * 2.0 ** -23)
            bound = bound + (want.abs() * ref.HALF_STEP[c.dtype]).clamp(min=2.0 ** -25)
            assert ((out[r, h] - want).abs() <= bound).all(), (r, h)
