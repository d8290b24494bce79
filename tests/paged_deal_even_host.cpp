// Runs the dealing of 4-bit rows' tiles on the host: CTAs' runs of equal length, and a CTA's warps with their shares of it.
#define main other_main
#include "paged_deal_host.cpp"
#undef main

static Run deal_even(const PagedCache& c, const PagedRows& r, int blocks, int runs, int before, int warps) {
  Run got[32];
  std::vector<std::thread> lanes;
  for (int i = 0; i < 32; ++i)
    lanes.emplace_back([&, i] {
      threadIdx.x = i;
      t_looks = 0;
      Run x{};
      x.per = pd_deal<TILE, true>(x.u, x.total, x.lone, runs, before, warps, c, r, blocks);
      got[i] = x;
    });
  for (auto& t : lanes) t.join();
  for (int i = 1; i < 32; ++i)
    if (got[i].total != got[0].total || got[i].per != got[0].per || got[i].u.row != got[0].u.row || got[i].u.tile != got[0].u.tile)
      return puts("lanes differ"), exit(5), got[0];
  return got[0];
}

int main() {
  for (int warps : {1, 4, 8, 12})
    for (int n = 0; n < 60; ++n)
      for (int w = 0; w < warps; ++w)
        for (int at = pd_share(n, w, warps); at < pd_share(n, w + 1, warps); ++at)
          if (pd_sharer(n, at, warps) != w || pd_share(n, w + 1, warps) - pd_share(n, w, warps) > n / warps + 1) return puts("shares"), 1;
  std::mt19937 rng(2);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int trial = 0; trial < 30; ++trial) {
    const int n = trial < 10 ? pick(1, 8) : pick(1, 200), most = trial % 3 ? 400 : 40, blocks = pick(1, 2), W = trial % 2 ? 4 : 3;
    const PagedCache c{pick(1, 3)};
    std::vector<int> lens(n);
    for (int& x : lens) x = pick(0, 4) ? pick(1, most) : 0;
    const PagedRows r{&lens, &lens, 0, n};
    std::vector<PdCursor> want;
    for (int row = 0; row < n; ++row)
      for (int h = 0; h < c.Hkv; ++h)
        for (int b = 0; b < blocks; ++b)
          for (int t = 0; t * TILE < lens[row]; ++t) want.push_back({row, h, b, t, (lens[row] + TILE - 1) / TILE, lens[row]});
    const int ctas = pick(1, 12);
    size_t at = 0;
    for (int before = 0; before < ctas * W; ++before) {
      Run x = deal_even(c, r, blocks, ctas * W, before, W);
      const int c0 = before / W * x.per, w = before % W, t0 = c0 + pd_share(x.per, w, W), t1 = c0 + pd_share(x.per, w + 1, W);
      if (x.lone ? x.per != W : x.per != (int)(want.size() + ctas - 1) / ctas) return puts("a run's length"), 1;
      t_looks = 0;
      const int mine = t0 >= x.total ? 0 : max(0, min(t1 - t0, x.lone ? x.u.tiles - x.u.tile : x.total - t0));
      for (int i = 0; i < mine; ++i, ++at) {
        if (at >= want.size()) return puts("too many tiles"), 1;
        const PdCursor &a = x.u, &b = want[at];
        if (a.row != b.row || a.head != b.head || a.block != b.block || a.tile != b.tile || a.tiles != b.tiles || a.n != b.n)
          return printf("trial %d, tile %zu: row %d, tile %d\n", trial, at, a.row, a.tile), 1;
        pd_advance<TILE>(x.u, c, r, blocks);
      }
    }
    if (at != want.size()) return puts("too few tiles"), 1;
  }
  return g_status;
}
