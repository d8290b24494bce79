"""4-bit pages for the tests: their format in 64 bits, and how far attention over them may be off.

What differs from 8-bit pages in the arithmetic: a logit's products are numbers from 0 to 15 with the queries, and 8 times the
queries' sum is taken away, so that an fp32 sum of a block of 32 elements goes through terms of up to (15 + 8) |q_i| s where
attention in 64 bits has |q_i| |n_i| s.  Queries enter as halves scaled to their largest element, half of which may fall 2^-36 of it
short.  Values meet the probabilities exactly.

Numbers of 0 are frequent, so that an element may be left to slots of small probabilities alone.  A probability enters as two halves
with the row's largest at 2^10 or above: its second term is off by half the smallest half, 2^-25, which is 2^-35 of the largest,
times |v| of every slot."""
import math

import torch

from tests import paged_reference as ref

NAN = 0xFC
BLOCK = 32


def scales64():
    """All scales, by their byte."""
    got = [(b & 7) * 2.0 ** -17 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 18) for b in range(0xC0)]
    return torch.tensor(got + [math.nan] * 0x40, dtype=torch.float64)


def quantise(x):
    """Rows [..., dim] (CPU) -> (bytes, scales' bytes, values), from the definition."""
    y = x.double().unflatten(-1, (-1, BLOCK))
    bad = y.isnan().any(-1)
    y = torch.where(bad[..., None], 0.0, y)
    grid = scales64()[:0xC0]
    t = (y.abs().amax(-1) / 7).clamp(max=480.0)
    hi = torch.searchsorted(grid, t.contiguous()).clamp(1, 0xBF)
    d = (grid[hi] - t) - (t - grid[hi - 1])
    byte = torch.where((d < 0) | ((d == 0) & (hi % 2 == 0)), hi, hi - 1)
    s = grid[byte]
    z = (y / torch.where(s > 0, s, 1.0)[..., None]).clamp(-7.0, 7.0)  # (infinities)
    n = torch.where((s > 0)[..., None], torch.round(z), 0.0)
    code = (n + 8).to(torch.uint8).flatten(-2)
    value = torch.where(bad[..., None], math.nan, n * s[..., None]).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(bad, NAN, byte).to(torch.uint8), value


def values(code, scale):
    """Bytes [..., dim / 2], scales' bytes [..., dim / 32] (CPU) -> values in 64 bits."""
    n = torch.stack([code & 15, code >> 4], -1).flatten(-2).double() - 8
    return (n.unflatten(-1, (-1, BLOCK)) * scales64()[scale.long()][..., None]).flatten(-2)


class Cache(ref.Cache):
    """As the base class, of 4 bits: slots that nobody has written hold NaN scales."""

    def __init__(self, lens, hq, hkv, dim, page, dtype, layout="hnd", **kw):
        super().__init__(lens, hq, hkv, 64, page, dtype, layout=layout, **kw)
        self.dim, n, p, h, d, L = dim, self.n_pages, page, hkv, dim // 2, self.layers
        if layout == "hnd":
            self.k, self.v = (torch.full((L, n, h, p, d), 0xF0, dtype=torch.uint8, device=self.device) for _ in range(2))
        elif layout == "nhd":
            self.k, self.v = (torch.full((L, n, p, h, d), 0x0F, dtype=torch.uint8, device=self.device).transpose(2, 3)
                              for _ in range(2))
        else:  # K and V of a page side by side in one tensor, layers inside the page, rows apart from each other
            both = torch.full((n, L, 2, p, h, d + 16), 0xF0, dtype=torch.uint8, device=self.device)
            self.k, self.v = (both[:, :, i, :, :, :d].permute(1, 0, 3, 2, 4) for i in (0, 1))
        self.sc = torch.full((L, n, h, p, 2, dim // BLOCK), NAN, dtype=torch.uint8, device=self.device)

    def handle(self, **kw):
        from paper_2412_04757_b200 import binding

        kw.setdefault("max_rows", len(self.lens_cpu))
        return binding.LtriPaged(self.k, self.v, self.hq, dtype=self.dtype, weights=self.w, positions=self.pos,
                                 block_scales=self.sc, **kw)

    def store(self, l, pg, off, which, rows):
        """The rows [n][Hkv][dim] into their places, quantised; returns their values."""
        code, scale, value = quantise(rows.cpu())
        (self.k, self.v)[which][l][pg, :, off] = code.to(self.device)
        self.sc[l][pg, :, off, which] = scale.to(self.device)
        return value

    def fill(self, scale=1.0):
        for l in range(self.layers):
            for r, n in enumerate(self.lens_cpu):
                if not n:
                    continue
                pg, off = self.places(r, n)
                for which in (0, 1):
                    self.store(l, pg, off, which, torch.randn(n, self.hkv, self.dim, generator=self.g) * scale)
                if self.w is not None:
                    ref.put(self.w[l], pg, off, torch.exp(torch.randn(n, self.hkv, generator=self.g)))
                    ref.put(self.pos[l], pg, off, torch.arange(n, dtype=torch.int32)[:, None].expand(n, self.hkv))

    def row(self, l, r, n, scaled=True):
        pg, off = self.places(r, n)
        return [values(pages[l][pg, :, off].cpu(), self.sc[l][pg, :, off, which].cpu())
                for which, pages in ((0, self.k), (1, self.v))]

    def steps(self, l, r, n):
        """The scales of K, one an element, [n][Hkv][dim]."""
        pg, off = self.places(r, n)
        return scales64()[self.sc[l][pg, :, off, 0].cpu().long()].repeat_interleave(BLOCK, -1)

    def snapshot(self):
        return {**super().snapshot(), "sc": self.sc.clone()}


def attend(q, K, V, steps, scale):
    """As the base module's, with this format's bounds."""
    out, lse, per, _, _, _ = ref.attend(q, K, V, scale)
    n, hkv, dim = K.shape
    G = q.shape[0] // hkv
    tol_out, tol_lse, tol_per = torch.zeros_like(q), torch.zeros(q.shape[0]).double(), torch.zeros(n, hkv).double()
    for h in range(q.shape[0]):
        k, v, s, a = K[:, h // G], V[:, h // G], steps[:, h // G], q[h].abs()
        d = float((s @ a).max()) * 23 * scale * (dim + 8) * 2.0 ** -23
        d += float((k.abs().sum(1)).max()) * float(a.max()) * 2.0 ** -36 * scale
        p = torch.softmax(k @ q[h] * scale, 0)
        sums = (n + 16) * 2.0 ** -24 + 2.0 ** -21
        rel = math.expm1(2 * d) + sums
        tol_out[h] = (rel + 2.0 ** -17) * (p @ v.abs()) + (1 + rel) * float(p.max()) * 2.0 ** -35 * v.abs().sum(0)
        tol_lse[h] = d + sums + abs(float(lse[h])) * 2.0 ** -22
        tol_per[:, h // G] += p * rel + 2.0 ** -120
    return out, lse, per, tol_out, tol_lse, tol_per


def check_decode(c, l, q, out, lse, lens, before_w=None, decay=1.0, new=False, scale=None):
    """Outputs, lse and weights of one decode call against the cache as the call left its rows."""
    scale = c.dim ** -0.5 if scale is None else scale
    half, tiny = ref.HALF_STEP[c.dtype], torch.finfo(c.dtype).smallest_normal * torch.finfo(c.dtype).eps
    errors, sizes = 0.0, 0.0
    for r, n in enumerate(lens):
        o, s = out[r].cpu().double(), None if lse is None else lse[r].cpu().double()
        if n == 0:
            assert (o == 0).all() and (s is None or (s == -math.inf).all()), f"row {r} is empty"
            continue
        K, V = c.row(l, r, n)
        ro, rl, per, to, tl, tp = attend(q[r].cpu().double(), K, V, c.steps(l, r, n), scale)
        err = (o - ro).abs() - (ro.abs() * half + to * (1 + half) + tiny)
        assert err.max() <= 0, f"row {r} of {n}: out off by {float((o - ro).abs().max())}, {float(err.max())} beyond the bound"
        errors, sizes = errors + float((o - ro).square().sum()), sizes + float(ro.square().sum())
        if s is not None:
            assert ((s - rl).abs() <= tl).all(), f"row {r}: lse off by {float((s - rl).abs().max())}"
        if before_w is not None:
            pg, off = c.places(r, n)
            old = ref.take(before_w[l], pg, off).cpu().double() * decay
            if new:
                old[n - 1] = 0.0
            got = ref.take(c.w[l], pg, off).cpu().double()
            want = old + per
            bound = tp + want.abs() * 2.0 ** -22 * (1 + 64 / 4)  # (up to 64 heads' terms and the old weight, each rounded)
            assert ((got - want).abs() <= bound).all(), f"row {r}: weights off by {float((got - want).abs().max())}"
    # All outputs together: a rounding is off by half a step at most, and what is off at random besides is far below it where
    # logits are a few units (2^-16: 40 times fp32's steps over a hundred products)
    if scale == c.dim ** -0.5 and sizes and float(q.float().abs().max()) < 10:
        assert errors ** 0.5 <= (half + 2.0 ** -16) * sizes ** 0.5


def evict(c, lens, budget, n_sink, recent, layers):
    """Applies an eviction to copies of the cache's tensors: their bits, and the new lengths."""
    got, new = ref.evict(c, lens, budget, n_sink, recent, layers)
    for l in layers:
        for r, n in enumerate(lens):
            if n <= budget:
                continue
            pg, off = c.places(r, n)
            for h in range(c.hkv):
                src, dst = ref.evict_unit(c.w[l, pg, h, off].tolist(), c.pos[l, pg, h, off].tolist(), budget, n_sink, recent)
                got["sc"][l, pg[dst], h, off[dst]] = got["sc"][l, pg[src], h, off[src]]
    return got, new
