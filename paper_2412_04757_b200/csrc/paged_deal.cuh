// How the tiles of a batch's rows are dealt to warps: the line of all (row, KV head, block of heads) units' tiles, and cursors
// that walk along it.  Of the device it uses a warp's collectives, paged_len and paged_status only, so that a test can bring
// its own and run it on the host.
#pragma once

#ifdef __CUDACC__
#include "paged.cuh"
#endif

namespace ltri {

// A place in the line of tiles.
struct PdCursor {
  int row, head, block, tile, tiles, n;
};

template <int TILE>
__device__ __forceinline__ void pd_advance(PdCursor& u, const PagedCache& c, const PagedRows& r, int blocks) {
  if (++u.tile < u.tiles) return;
  u.tile = 0;
  if (++u.block < blocks) return;
  u.block = 0;
  if (++u.head < c.Hkv) return;
  u.head = 0;
  do {
    // (behind the last row: a tile of it without a slot)
    u.n = u.row + 1 < r.n ? paged_len(c, r, ++u.row) : -1;
    u.tiles = u.n < 0 ? 1 : (u.n + TILE - 1) / TILE;
  } while (u.tiles == 0);
  u.n = max(u.n, 0);
}

// A CTA's run of n tiles dealt evenly to its warps, the first n % warps of which have one more: where warp w's begin, and whose tile
// `at` is.
__device__ __forceinline__ int pd_share(int n, int w, int warps) { return w * (n / warps) + min(w, n % warps); }
__device__ __forceinline__ int pd_sharer(int n, int at, int warps) {
  const int each = n / warps, more = n % warps;
  return at < more * (each + 1) ? at / (each + 1) : more + (at - more * (each + 1)) / max(each, 1);
}

// All lanes of a warp: the tiles of the whole call, and the cursor of tile `runs_before` * per, where per is every run's length
// (returned) when `runs` of them cover the line.  EVEN: per is a CTA's run, and its `warps` warps have their shares of it, so that
// SMs differ by a tile where they would differ by one a warp.
// Where every unit can have a CTA of its own and a warp no more than one of its tiles, it begins with one, as if all were as
// long as the CTAs' runs (`lone`; the cursor may then lie behind the unit's end): no two CTAs share a unit, and the join at
// the end, two trips through L2, is spared.  (8 query heads, 2 KV heads, 100 slots: 7.1 us, 9.5 dealt evenly; with up to three
// tiles a warp, 300 slots: 9.0 and 8.6.)
template <int TILE, bool EVEN = false>
__device__ __forceinline__ int pd_deal(PdCursor& u, int& total, bool& lone, int runs, int runs_before, int warps,
                                       const PagedCache& c, const PagedRows& r, int blocks) {
  const int lane = threadIdx.x & 31, per_row = c.Hkv * blocks;
  lone = false;
  auto scan = [&](int x) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    return x;
  };
  // the first 64 rows are asked for at once, and kept
  const int n0 = lane < r.n ? paged_len(c, r, lane) : 0, n1 = lane + 32 < r.n ? paged_len(c, r, lane + 32) : 0;
  if (r.n <= 32) {
    const unsigned rows = __ballot_sync(0xffffffffu, n0 > 0);
    const int units = __popc(rows) * per_row;
    if (warps > 0 && __reduce_max_sync(0xffffffffu, n0) <= warps * TILE && units * warps <= runs) {
      const int unit = (unsigned)runs_before / (unsigned)warps;
      total = units * warps;
      lone = true;
      const int one = EVEN ? warps : 1;
      if (unit >= units) return one;
      const int nth = unit / per_row, in_row = unit - nth * per_row;
      u.row = __fns(rows, 0, nth + 1);
      u.n = __shfl_sync(0xffffffffu, n0, u.row);
      u.tiles = (u.n + TILE - 1) / TILE;
      u.tile = runs_before - unit * warps;
      u.head = in_row / blocks;
      u.block = in_row - u.head * blocks;
      return one;
    }
  }
  const int inc0 = scan((n0 + TILE - 1) / TILE * per_row);
  total = __shfl_sync(0xffffffffu, inc0, 31);
  if (r.n > 32) total += __reduce_add_sync(0xffffffffu, (n1 + TILE - 1) / TILE * per_row);
  for (int base = 64; base < r.n; base += 32) {
    const int row = base + lane;
    total += __reduce_add_sync(0xffffffffu, row < r.n ? (paged_len(c, r, row) + TILE - 1) / TILE * per_row : 0);
  }
  if (EVEN) runs /= warps;
  const int per = (int)((unsigned)(total + runs - 1) / (unsigned)runs);
  int left = EVEN ? runs_before / warps * per + pd_share(per, runs_before % warps, warps) : runs_before * per;
  if (left >= total) return per;
  for (int base = 0; base < r.n; base += 32) {
    const int row = base + lane;
    const int n = base == 0 ? n0 : base == 32 ? n1 : row < r.n ? paged_len(c, r, row) : 0;
    const int inc = base == 0 ? inc0 : scan((n + TILE - 1) / TILE * per_row);
    const unsigned in = __ballot_sync(0xffffffffu, left < inc);
    if (in) {
      const int at = __ffs(in) - 1;
      u.row = base + at;
      u.n = __shfl_sync(0xffffffffu, n, at);
      u.tiles = (u.n + TILE - 1) / TILE;
      left -= __shfl_sync(0xffffffffu, inc, at) - u.tiles * per_row;
      const int unit = (int)((unsigned)left / (unsigned)u.tiles);
      u.tile = left - unit * u.tiles;
      u.head = blocks == 1 ? unit : unit / blocks;
      u.block = unit - u.head * blocks;
      return per;
    }
    left -= __shfl_sync(0xffffffffu, inc, 31);
  }
  // the rows have become shorter since they were added up (somebody writes to the lengths that this call reads): no run
  paged_status(c, 0);
  total = 0;
  return per;
}

}  // namespace ltri
