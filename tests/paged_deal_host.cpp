// Runs the dealing of the paged attention's tiles on the host: 32 threads are a warp, and its collectives meet at a barrier.
// Arguments: lines | shorter.  Exits with 0 if all is as it should be.
#include <unistd.h>

#include <algorithm>
#include <barrier>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>
#include <thread>
#include <vector>

#define __device__
#define __forceinline__ inline

using std::max;
using std::min;

static std::barrier<> g_meet(32);
static int g_x[32];
static thread_local struct { unsigned x; } threadIdx;

template <typename F>
static int together(int x, F pick) {
  g_x[threadIdx.x] = x;
  g_meet.arrive_and_wait();
  const int y = pick(g_x);
  g_meet.arrive_and_wait();
  return y;
}
static int __shfl_sync(unsigned, int x, int from) { return together(x, [&](int* a) { return a[from & 31]; }); }
static int __shfl_up_sync(unsigned, int x, int d) {
  const int lane = threadIdx.x;
  return together(x, [&](int* a) { return lane >= d ? a[lane - d] : x; });
}
static int __reduce_add_sync(unsigned, int x) {
  return together(x, [](int* a) { int s = 0; for (int i = 0; i < 32; ++i) s += a[i]; return s; });
}
static int __reduce_max_sync(unsigned, int x) { return together(x, [](int* a) { return *std::max_element(a, a + 32); }); }
static unsigned __ballot_sync(unsigned, bool x) {
  return (unsigned)together(x, [](int* a) {
    unsigned m = 0;
    for (int i = 0; i < 32; ++i) m |= (unsigned)(a[i] != 0) << i;
    return (int)m;
  });
}
static int __popc(unsigned x) { return __builtin_popcount(x); }
static int __ffs(unsigned x) { return __builtin_ffs((int)x); }
static int __fns(unsigned mask, unsigned, int nth) {
  for (int i = 0; i < 32; ++i)
    if ((mask >> i & 1) && --nth == 0) return i;
  return -1;
}

namespace ltri {
struct PagedCache {
  int Hkv;
};
struct PagedRows {
  const std::vector<int>* lens;
  const std::vector<int>* later;  // the lengths from a lane's `change`th look on
  int change, n;
};
static thread_local int t_looks;
static int g_status;
static int paged_len(const PagedCache&, const PagedRows& r, int row) {
  if (row < 0 || row >= r.n) {
    printf("length of row %d of %d\n", row, r.n);
    fflush(stdout);
    _exit(4);
  }
  if (t_looks > 1000000) {
    puts("endless");
    fflush(stdout);
    _exit(3);
  }
  return (t_looks++ < r.change ? *r.lens : *r.later)[row];
}
static void paged_status(const PagedCache&, int) { g_status = 1; }
}  // namespace ltri

#include "../paper_2412_04757_b200/csrc/paged_deal.cuh"

using namespace ltri;

constexpr int TILE = 16;

struct Run {
  PdCursor u;
  int total, per;
  bool lone;
};

// pd_deal by a warp whose lanes must agree.
static Run deal(const PagedCache& c, const PagedRows& r, int blocks, int runs, int before, int warps) {
  Run got[32];
  std::vector<std::thread> lanes;
  for (int i = 0; i < 32; ++i)
    lanes.emplace_back([&, i] {
      threadIdx.x = i;
      t_looks = 0;
      Run x{};
      x.per = pd_deal<TILE>(x.u, x.total, x.lone, runs, before, warps, c, r, blocks);
      got[i] = x;
    });
  for (auto& t : lanes) t.join();
  for (int i = 1; i < 32; ++i)
    if (got[i].total != got[0].total || got[i].per != got[0].per || got[i].u.row != got[0].u.row ||
        got[i].u.tile != got[0].u.tile) {
      puts("lanes differ");
      exit(5);
    }
  return got[0];
}

static int lines() {
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int trial = 0; trial < 30; ++trial) {
    const int n = trial < 10 ? pick(1, 8) : pick(1, 200), most = trial % 3 ? 400 : 40, blocks = pick(1, 2), W = 4;
    const PagedCache c{pick(1, 3)};
    std::vector<int> lens(n);
    for (int& x : lens) x = pick(0, 4) ? pick(1, most) : 0;
    const PagedRows r{&lens, &lens, 0, n};
    std::vector<PdCursor> want;
    for (int row = 0; row < n; ++row)
      for (int h = 0; h < c.Hkv; ++h)
        for (int b = 0; b < blocks; ++b)
          for (int t = 0; t * TILE < lens[row]; ++t) want.push_back({row, h, b, t, (lens[row] + TILE - 1) / TILE, lens[row]});
    const int runs = W * pick(1, 12);
    size_t at = 0;
    for (int before = 0; before < runs; ++before) {
      Run x = deal(c, r, blocks, runs, before, trial % 2 ? W : 0);
      const int t0 = before * x.per;
      t_looks = 0;
      const int mine = t0 >= x.total ? 0 : max(0, min(x.per, x.lone ? x.u.tiles - x.u.tile : x.total - t0));
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

// Rows that become shorter between the two times that their lengths are read: every call of the dealing comes to an end, says
// so, and no cursor leaves the rows.
static int shorter() {
  const int n = 200, blocks = 1, runs = 40;
  const PagedCache c{2};
  const std::vector<int> lens(n, 100), later(n, 16);
  for (int look : {7, 6, 4, 2}) {  // (a lane looks six or seven times in the first pass)
    int recorded = 0;
    for (int before = 0; before < runs; ++before) {
      g_status = 0;
      const PagedRows r{&lens, &later, look, n};
      Run x = deal(c, r, blocks, runs, before, 0);
      t_looks = look;  // (from here on the rows are short)
      const int t0 = before * x.per, mine = t0 >= x.total ? 0 : min(x.per, x.total - t0);
      for (int i = 0; i < mine; ++i) {
        if (x.u.row < 0 || x.u.row >= n || x.u.head >= c.Hkv || x.u.tile < 0) return puts("a cursor behind the rows"), 1;
        pd_advance<TILE>(x.u, c, r, blocks);
      }
      recorded += g_status;
    }
    if (look >= 6 && recorded == 0) return puts("nothing recorded"), 1;
  }
  return 0;
}

int main(int, char** argv) { return std::string(argv[1]) == "lines" ? lines() : shorter(); }
