"""The paged cache's operators in 64 bits, slot by slot, and how far a kernel may be off them.

Tolerances are worst-case bounds of the arithmetic, per element:

* A logit x = c * sum_i q_i k_i is summed in fp32 from exact products: its error is at most (D + 8) units of 2^-23 of
  A = c * sum_i |q_i k_i| (one rounding, of up to 2^-23 where a sum truncates, per addition; the factor c; the
  subtraction of the running maximum).  Probabilities are then off by a factor of at most exp(2 d), d that error's maximum
  over the row, together with the error of exp2 (2^-21) and of a sum of n terms, (n + 16) 2^-24.
* Probabilities that meet V enter as two terms of 8 significant bits or more each: off by 2^-17 relative.
* The output is rounded once, half a step of its type, and a value below the type's smallest normal by half its spacing.
"""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E4M3 = torch.float8_e4m3fn


class Cache:
    """Pages of every layout with NaN in every slot nobody has written, and the batch's table."""

    def __init__(self, lens, hq, hkv, dim, page, dtype, e4m3=False, layers=1, layout="hnd", weighted=False, room=0, seed=0,
                 device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.g, self.hq, self.hkv, self.dim, self.page, self.dtype, self.layers = g, hq, hkv, dim, page, dtype, layers
        self.G, self.device = hq // hkv, device
        need = [-(-(n + room) // page) for n in lens]
        self.n_pages = sum(need) + 3
        order = torch.randperm(self.n_pages, generator=g)
        cols = max(need + [1])
        table = torch.full((len(lens), cols), -7, dtype=torch.int32)  # entries that nobody may read
        at = 0
        for r, k in enumerate(need):
            table[r, :k] = order[at:at + k]
            at += k
        self.table_cpu, self.table = table, table.to(device)
        self.lens_cpu = list(lens)
        held = E4M3 if e4m3 else dtype
        n, p, h, d = self.n_pages, page, hkv, dim
        if layout == "hnd":
            make = lambda: torch.full((layers, n, h, p, d), float("nan")).to(held).to(device)  # noqa: E731
            self.k, self.v = make(), make()
        elif layout == "nhd":
            make = lambda: torch.full((layers, n, p, h, d), float("nan")).to(held).to(device).transpose(2, 3)  # noqa: E731
            self.k, self.v = make(), make()
        else:  # K and V of a page side by side in one tensor, layers inside the page, rows apart from each other
            both = torch.full((n, layers, 2, p, h, d + 16), float("nan")).to(held).to(device)
            self.k, self.v = (both[:, :, i, :, :, :d].permute(1, 0, 3, 2, 4) for i in (0, 1))
        self.ks = self.vs = None
        if e4m3:
            self.ks = (0.01 + 0.02 * torch.rand(hkv, generator=g)).to(device)
            self.vs = (0.01 + 0.02 * torch.rand(hkv, generator=g)).to(device)
        self.w = self.pos = None
        if weighted:
            self.w = torch.full((layers, n, h, p), float("nan")).to(device)
            self.pos = torch.full((layers, n, h, p), -5, dtype=torch.int32).to(device)

    def handle(self, **kw):
        from paper_2412_04757_b200 import binding

        kw.setdefault("max_rows", len(self.lens_cpu))
        return binding.LtriPaged(self.k, self.v, self.hq, dtype=self.dtype, k_scale=self.ks, v_scale=self.vs, weights=self.w,
                                 positions=self.pos, **kw)

    def lens(self):
        return torch.tensor(self.lens_cpu, dtype=torch.int32, device=self.device)

    def randn(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.g) * scale).to(self.dtype).to(self.device)

    def places(self, r, n):
        """(pages, places) of row r's first n slots."""
        j = torch.arange(n)
        return self.table_cpu[r].long()[j // self.page].to(self.device), (j % self.page).to(self.device)

    def fill(self, scale=1.0):
        """Rows, weights and positions for every slot in use."""
        for l in range(self.layers):
            for r, n in enumerate(self.lens_cpu):
                if not n:
                    continue
                pg, off = self.places(r, n)
                for pages in (self.k, self.v):
                    put(pages[l], pg, off, (torch.randn(n, self.hkv, self.dim, generator=self.g) * scale).to(pages.dtype))
                if self.w is not None:
                    put(self.w[l], pg, off, torch.exp(torch.randn(n, self.hkv, generator=self.g)))
                    put(self.pos[l], pg, off, torch.arange(n, dtype=torch.int32)[:, None].expand(n, self.hkv))

    def row(self, l, r, n, scaled=True):
        """K, V [n][Hkv][dim] in 64 bits (CPU)."""
        pg, off = self.places(r, n)
        got = []
        for pages, s in ((self.k, self.ks), (self.v, self.vs)):
            x = take(pages[l], pg, off).cpu().double()
            got.append(x if s is None or not scaled else x * s.cpu().double()[:, None])
        return got

    def snapshot(self):
        return {name: bits(t).clone() for name, t in (("k", self.k), ("v", self.v), ("w", self.w), ("pos", self.pos))
                if t is not None}


def bits(t):
    """A tensor as whole numbers: NaN equals itself there."""
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def _index(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def put(pages, pg, off, rows):
    _index(pages)[pg, :, off] = _index(rows.to(pages.device))


def take(pages, pg, off):
    return _index(pages)[pg, :, off].view(pages.dtype)


def quantise(x, scale):
    """The nearest e4m3 value to x / scale, ties to even, in 64 bits; x [..., Hkv, dim], scale [Hkv].  The quotient is
    fp32's."""
    y = (x.float() / scale.float()[:, None]).double()
    a = y.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(a / step) * step, y)


def attend(q, K, V, scale):
    """q [Hq][dim], K, V [n][Hkv][dim], all 64 bits -> out, lse, per-slot sums [n][Hkv] and the bounds of each."""
    n, hkv, dim = K.shape
    G = q.shape[0] // hkv
    out, lse = torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    per, tol_per = torch.zeros(n, hkv).double(), torch.zeros(n, hkv).double()
    tol_out, tol_lse = torch.zeros_like(q), torch.zeros(q.shape[0]).double()
    for h in range(q.shape[0]):
        k, v = K[:, h // G], V[:, h // G]
        x = k @ q[h] * scale
        d = float((k.abs() @ q[h].abs()).max()) * scale * (dim + 8) * 2.0 ** -23
        lse[h] = torch.logsumexp(x, 0)
        p = torch.softmax(x, 0)
        out[h] = p @ v
        sums = (n + 16) * 2.0 ** -24 + 2.0 ** -21
        rel = math.expm1(2 * d) + sums
        tol_out[h] = (rel + 2.0 ** -17) * (p @ v.abs())
        tol_lse[h] = d + sums + abs(float(lse[h])) * 2.0 ** -22
        per[:, h // G] += p
        tol_per[:, h // G] += p * rel + 2.0 ** -120
    return out, lse, per, tol_out, tol_lse, tol_per


def check_decode(c, l, q, out, lse, lens, before_w=None, decay=1.0, new=False, scale=None):
    """Outputs, lse and weights of one decode call against the cache as the call left its rows."""
    scale = c.dim ** -0.5 if scale is None else scale
    half, tiny = HALF_STEP[c.dtype], torch.finfo(c.dtype).smallest_normal * torch.finfo(c.dtype).eps
    for r, n in enumerate(lens):
        o, s = out[r].cpu().double(), None if lse is None else lse[r].cpu().double()
        if n == 0:
            assert (o == 0).all() and (s is None or (s == -math.inf).all()), f"row {r} is empty"
            continue
        K, V = c.row(l, r, n)
        ro, rl, per, to, tl, tp = attend(q[r].cpu().double(), K, V, scale)
        err = (o - ro).abs() - (ro.abs() * half + to * (1 + half) + tiny)
        assert err.max() <= 0, f"row {r} of {n}: out off by {float((o - ro).abs().max())}, {float(err.max())} beyond the bound"
        if s is not None:
            assert ((s - rl).abs() <= tl).all(), f"row {r}: lse off by {float((s - rl).abs().max())}"
        if before_w is not None:
            pg, off = c.places(r, n)
            old = take(before_w[l], pg, off).cpu().double() * decay
            if new:
                old[n - 1] = 0.0
            got = take(c.w[l], pg, off).cpu().double()
            ref = old + per
            bound = tp + ref.abs() * 2.0 ** -22 * (1 + 64 / 4)  # (up to 64 heads' terms and the old weight, each rounded)
            assert ((got - ref).abs() <= bound).all(), f"row {r}: weights off by {float((got - ref).abs().max())}"


def evict_unit(w, pos, budget, n_sink, recent):
    """(sources, destinations) of one unit's moves; w, pos: lists of its slots."""
    newest = max(pos)
    nan = [-math.inf if x != x else x for x in w]
    stays = [p < n_sink or p > newest - recent for p in pos]
    order = sorted(range(len(w)), key=lambda j: (not stays[j], 0.0 if stays[j] else -nan[j], j))
    kept = set(order[:budget])
    return [j for j in range(budget, len(w)) if j in kept], [j for j in range(budget) if j not in kept]


def evict(c, lens, budget, n_sink, recent, layers):
    """Applies an eviction to copies of the cache's tensors: their bits, and the new lengths."""
    got = c.snapshot()
    full = {"k": c.k, "v": c.v, "w": c.w, "pos": c.pos}
    for l in layers:
        for r, n in enumerate(lens):
            if n <= budget:
                continue
            pg, off = c.places(r, n)
            for h in range(c.hkv):
                w, pos = c.w[l, pg, h, off].tolist(), c.pos[l, pg, h, off].tolist()
                src, dst = evict_unit(w, pos, budget, n_sink, recent)
                for name in full:
                    x = got[name]
                    x[l, pg[dst], h, off[dst]] = x[l, pg[src], h, off[src]]
    return got, [min(n, budget) for n in lens]
