// Eviction from a caller-owned paged cache by accumulated attention weight.
//
// Per (layer, row, KV head) of n > budget slots: the budget-th largest key is found, where a key is a weight as an ordered
// integer and protected positions have the largest; slots below it are holes if they lie in front of the budget, slots above
// it move if they lie behind, the i-th into the i-th hole.  Sources and destinations are disjoint, so the moves need no order,
// and a full budget that has grown by one token costs one row, not a shifted cache.
//
// A cluster owns a unit; its CTAs hold a stretch of the slots each, as keys in shared memory.  Where one slot leaves, as in a
// step that has appended one, it is the lowest key's, and the last slot moves there.  Otherwise a histogram of 2048 bins over
// the range that the keys really have, summed through distributed shared memory, leaves some ten keys around the cut (weights
// of a few powers of two); they are ranked against each other.  Where many are left (equal ones above all), up to two more
// histograms go through the bin's range instead.
//
// Keys that shared memory does not hold are read again by every sweep.  Where rows share pages that are evicted, or somebody
// else writes to them, the sweeps then differ: which slots stay is undefined, but bins, candidates and lists are bounded, and
// every CTA of a cluster takes the same way through the barriers.
//
// Bound: latency where few slots leave, HBM where many rows move (read once, written once).  Measured: one slot of each of 256
// units of 4097 slots, 8 to 14 us within a step; 64 of 128 units, of 29369 to 32768 slots, cut to 5120, 108 us, 30 of them for
// the keys and lists, the rest for 5000 moves a unit at 4.5 TB/s (read and written), which neither more rows on the way nor
// rows side by side raise.  The launch is shaped by the table's columns, since lengths are not read on the host: with a table
// for 131072 slots instead of 4112 the step of two layers takes 240 us instead of 135, the cut of 32768 slots 224 instead of 111.
#include <cooperative_groups.h>
#include <limits.h>

#include "paged.cuh"

namespace ltri {

namespace cg = cooperative_groups;

constexpr int kEvThreads = 512;  // two CTAs an SM: one's rows move while another's keys are counted
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBinBits = 11, kEvBins = 1 << kEvBinBits;
constexpr int kEvMaxCluster = 8;    // (of sixteen CTAs too few run at once: 32 units of 32768 slots took 139 us instead of 79)
constexpr int kEvMaxSlots = 27136;  // keys and positions that a CTA can hold (212 KB); those of longer stretches are read again
constexpr int kEvSlots = 1024, kEvLong = 8192;  // slots of a CTA: above the first a unit gets more CTAs where SMs are idle,
                                                // above the second anyway
constexpr int kEvBatch = 9;         // slots of a thread whose weights and positions are on their way
constexpr int kEvCand = kEvThreads;       // keys around the cut that are ranked against each other
constexpr int kEvGroup = 4;         // moves that a warp takes side by side
constexpr int kEvMoves = 2;         // 16-byte chunks that a lane has on their way

// Order of a slot: larger is kept first.  Protected positions come before every weight, NaN counts as -infinity, and the
// two zeros are equal.
__device__ __forceinline__ unsigned ev_key(float w, bool stays) {
  if (stays) return 0xffffffffu;
  if (w != w) w = -INFINITY;
  const unsigned u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive prefix sum of x over the CTA; s: kEvWarps ints.
__device__ __forceinline__ int ev_scan(int x, int* s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) s[warp] = x;
  __syncthreads();
  const int before = __reduce_add_sync(0xffffffffu, lane < warp ? s[lane] : 0);  // (at most 32 warps)
  __syncthreads();
  return before + x;
}

__global__ void __launch_bounds__(kEvThreads, 2)
    k_paged_evict(PagedCache c, PagedRows r, int layer_begin, int layers, int* new_lens, int budget, int n_sink, int recent,
                  int held) {
  extern __shared__ unsigned s_key[];  // [held], and behind them
  int* s_pos = reinterpret_cast<int*>(s_key) + held;   // [held]: positions; then every warp's movers and holes
  int* s_list = reinterpret_cast<int*>(s_key);         // at last the CTA's, movers from the front and holes from the back
  __shared__ __align__(16) unsigned s_hist[kEvBins];
  __shared__ unsigned s_cand[kEvCand], s_all[kEvCand];
  __shared__ int s_scan[kEvWarps], s_hole[kEvWarps], s_mover[kEvWarps];
  __shared__ int s_n, s_newest, s_stay, s_bin, s_above, s_in, s_eq, s_holes, s_movers, s_cands;
  __shared__ unsigned s_lo, s_hi, s_cut;
  __shared__ unsigned long long s_least;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = cluster.num_blocks(), rank = cluster.block_rank();
  const int unit = blockIdx.x / C, head = unit % c.Hkv, row = unit / c.Hkv % r.n, layer = layer_begin + unit / c.Hkv / r.n;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  chain_wait();
  if (tid == 0) {
    s_n = paged_len(c, r, row);
    s_newest = INT_MIN;
    s_stay = s_cands = 0;
    s_lo = 0xffffffffu;
    s_hi = 0u;
    s_least = ~0ull;
  }
  __syncthreads();
  const int n = s_n;
  // the lengths may be replaced in place: by the last CTA of the row to have read its
  if (tid == 32 && paged_arrive(&c.seen[row]) == layers * c.Hkv * C - 1) {
    c.seen[row] = 0;
    new_lens[row] = min(n, budget);
  }
  // A cluster goes on if all of it has read the same length: should somebody write to the lengths meanwhile, no CTA may be gone
  // while another one asks for its shared memory.
  if (n <= budget) {
    if (C > 1) {
      cluster.sync();
      cluster.sync();
    }
    return;
  }

  const int chunk = (n + C - 1) / C, begin = rank * chunk, end = min(n, begin + chunk);
  bool bad = false;  // a page that is none
  auto page_of = [&](int nth) {
    const int page = r.table[row * r.table_stride + nth];
    if ((unsigned)page < (unsigned)c.n_pages) return page;
    bad = true;
    return -1;
  };
  const size_t word0 = paged_word(c, layer, 0, head, 0);
  const unsigned page_words = (unsigned)c.Hkv * c.P;
  auto word = [&](int slot) -> long long {  // -1: no page
    const int nth = paged_nth(c, slot), page = page_of(nth);
    return page < 0 ? -1 : (long long)(word0 + (unsigned long long)page_words * (unsigned)page) + (slot - nth * c.P);
  };
  // The CTA's sum, least or largest value over the cluster: lane i asks CTA i.
  auto ask = [&](int* x, int none) { return lane < C ? *cluster.map_shared_rank(x, lane) : none; };
  // ---- where one slot leaves, the last one's rows are on their way to its place from the beginning ----
  const bool single = n - budget == 1, carries = single && rank == 0 && warp == kEvWarps - 1;
  const int chunks = c.row_bytes / 16;  // 4, 8, 16 or 32 of 16 bytes: a move is 2 * chunks
  uint4 carried[2];
  float carried_w = 0.f;
  int carried_pos = 0, carried_page = -1;
  if (carries) {
    const int nth = paged_nth(c, n - 1), place = n - 1 - nth * c.P;
    carried_page = page_of(nth);
    if (carried_page >= 0) {
      const size_t from = paged_row(c, layer, carried_page, head, place);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int ch = k * 32 + lane;
        if (ch < 2 * chunks)
          carried[k] = __ldcg(reinterpret_cast<const uint4*>((ch >= chunks ? c.v + (ch - chunks) * 16 : c.k + ch * 16) + from));
      }
      const size_t at = paged_word(c, layer, carried_page, head, place);
      carried_w = c.w[at];
      carried_pos = c.pos[at];
    }
  }
  // ---- keys: a thread's slots in batches whose loads are all on their way at once; the newest position comes out of them ----
  const bool all_held = chunk <= held;
  int newest = INT_MIN;
  for (int j0 = begin + tid; j0 < end; j0 += kEvBatch * kEvThreads) {
    long long at[kEvBatch];
#pragma unroll
    for (int b = 0; b < kEvBatch; ++b) at[b] = j0 + b * kEvThreads < end ? word(j0 + b * kEvThreads) : -1;
    int pos[kEvBatch];
    float w[kEvBatch];
#pragma unroll
    for (int b = 0; b < kEvBatch; ++b) {
      pos[b] = at[b] >= 0 ? c.pos[at[b]] : INT_MIN;
      w[b] = at[b] >= 0 ? c.w[at[b]] : 0.f;
    }
#pragma unroll
    for (int b = 0; b < kEvBatch; ++b) {
      const int j = j0 + b * kEvThreads;
      newest = max(newest, pos[b]);
      if (j < end && j - begin < held) {
        s_key[j - begin] = at[b] < 0 ? 0u : ev_key(w[b], pos[b] < n_sink);
        s_pos[j - begin] = pos[b];
      }
    }
  }
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (lane == 0) atomicMax(&s_newest, newest);
  cluster.sync();
  const bool agreed = __all_sync(0xffffffffu, ask(&s_n, n) == n);
  newest = __reduce_max_sync(0xffffffffu, ask(&s_newest, INT_MIN));
  const long long first_recent = (long long)newest - recent;
  auto key = [&](int slot) {
    if (slot - begin < held) return s_key[slot - begin];
    const long long at = word(slot);
    if (at < 0) return 0u;
    const int pos = c.pos[at];
    return ev_key(c.w[at], pos < n_sink || pos > first_recent);
  };
  unsigned lo = 0xffffffffu, hi = 0u;
  int stay = 0;
  unsigned long long least = ~0ull;  // the lowest key, and of its slots the highest
  for (int j = begin + tid; j < end; j += kEvThreads) {
    unsigned x = key(j);
    // (a slot without a page has position INT_MIN here: where no position is larger, it is not protected either)
    if (j - begin < held && s_pos[j - begin] > first_recent && s_pos[j - begin] != INT_MIN) s_key[j - begin] = x = 0xffffffffu;
    if (x == 0xffffffffu) ++stay;
    else lo = min(lo, x), hi = max(hi, x);
    least = min(least, (unsigned long long)x << 32 | (unsigned)(0x7fffffff - j));
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  stay = __reduce_add_sync(0xffffffffu, stay);
  if (single) {
#pragma unroll
    for (int d = 16; d; d >>= 1) least = min(least, __shfl_xor_sync(0xffffffffu, least, d));
    if (lane == 0) atomicMin(&s_least, least);
  }
  if (lane == 0) {
    atomicMin(&s_lo, lo);
    atomicMax(&s_hi, hi);
    atomicAdd(&s_stay, stay);
  }
  cluster.sync();
  if (!agreed) {
    paged_status(c, row);
    return;
  }
  int count = 0;                     // moves
  int m_incl = 0, h_incl = 0;        // lane i: movers and holes up to CTA i
  if (single) {
    least = lane < C ? *cluster.map_shared_rank(&s_least, lane) : ~0ull;
#pragma unroll
    for (int d = 16; d; d >>= 1) least = min(least, __shfl_xor_sync(0xffffffffu, least, d));
    const int gap = 0x7fffffff - (int)(unsigned)least;
    if (carries && carried_page >= 0 && gap < n - 1) {
      const int nth = paged_nth(c, gap), place = gap - nth * c.P, page = page_of(nth);
      if (page >= 0) {
        const size_t to = paged_row(c, layer, page, head, place);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int ch = k * 32 + lane;
          if (ch < 2 * chunks)
            __stcg(reinterpret_cast<uint4*>((ch >= chunks ? c.v + (ch - chunks) * 16 : c.k + ch * 16) + to), carried[k]);
        }
        if (lane == 0) {
          const size_t at = paged_word(c, layer, page, head, place);
          c.w[at] = carried_w;
          c.pos[at] = carried_pos;
        }
      }
    }
  } else {
  {
    const unsigned l = lane < C ? *cluster.map_shared_rank(&s_lo, lane) : 0xffffffffu;
    const unsigned h = lane < C ? *cluster.map_shared_rank(&s_hi, lane) : 0u;
    const int st = ask(&s_stay, 0);
    lo = __reduce_min_sync(0xffffffffu, l);
    hi = __reduce_max_sync(0xffffffffu, h);
    stay = __reduce_add_sync(0xffffffffu, st);
  }
  // ---- the budget-th largest key: `ties` slots of key `cut` stay, the lowest ones, of `equal` that there are ----
  unsigned cut = 0xffffffffu;
  int ties = budget, equal = stay;
  if (stay < budget) {
    int need = budget - stay;
    while (true) {
      const int shift = max(0, 32 - __clz(hi - lo) - kEvBinBits);
      for (int i = tid; i < kEvBins; i += kEvThreads) s_hist[i] = 0;
      __syncthreads();
      for (int j = begin + tid; j < begin + (chunk + 31) / 32 * 32; j += kEvThreads) {  // (whole warps)
        const unsigned x = j < end ? key(j) : 0xffffffffu;
        const bool in = x >= lo && x <= hi && x != 0xffffffffu;
        const unsigned bin = in ? (x - lo) >> shift : 0u;
        // many equal keys, as a cache that nobody has attended to yet has, meet in one bin: one addition for the warp
        const unsigned who = __ballot_sync(0xffffffffu, in);
        if (who == 0) continue;
        const unsigned first = __shfl_sync(0xffffffffu, bin, __ffs(who) - 1);
        if (__all_sync(0xffffffffu, !in || bin == first)) {
          if (lane == 0) atomicAdd(&s_hist[first], __popc(who));
        } else if (in) {
          atomicAdd(&s_hist[bin], 1u);
        }
      }
      cluster.sync();
      // bins from the top, four a thread
      static_assert(kEvBins == 4 * kEvThreads, "a thread has four bins");
      int sum[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kEvMaxCluster; ++i) {
        if (i >= C) break;
        const uint4 x = reinterpret_cast<const uint4*>(cluster.map_shared_rank(s_hist, i))[kEvThreads - 1 - tid];
        sum[0] += x.w;
        sum[1] += x.z;
        sum[2] += x.y;
        sum[3] += x.x;
      }
      const int to = ev_scan(sum[0] + sum[1] + sum[2] + sum[3], s_scan);
      int from = to - sum[0] - sum[1] - sum[2] - sum[3];
      const bool lowest = tid == kEvThreads - 1;  // (has what no bin holds)
      if (from < need && (need <= to || lowest)) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if ((from < need && need <= from + sum[b]) || (lowest && b == 3)) {
            s_bin = kEvBins - 1 - 4 * tid - b;
            s_above = from;
            s_in = sum[b];
            break;
          }
          from += sum[b];
        }
      }
      cluster.sync();  // (and nobody reads the histograms any more)
      need -= s_above;
      lo += (unsigned)s_bin << shift;
      equal = s_in;
      cut = lo;
      ties = need;
      if (shift == 0) break;
      hi = min(hi, lo + ((1u << shift) - 1));
      if (equal > kEvCand) continue;
      // few keys left: every CTA gets all of them (in whatever order) and ranks them
      for (int j = begin + tid; j < end; j += kEvThreads) {
        const unsigned x = key(j);
        if (x >= lo && x <= hi && x != 0xffffffffu) {
          const int at = atomicAdd(&s_cands, 1);
          if (at < kEvCand) s_cand[at] = x;
        }
      }
      static_assert(kEvCand == kEvThreads, "a thread has a candidate");
      s_all[tid] = 0u;
      cluster.sync();
      if (tid == 0) s_cut = lo, s_above = 0, s_in = equal;
      if (warp < C) {
        const int count = min(ask(&s_cands, 0), kEvCand), before = __reduce_add_sync(0xffffffffu, lane < warp ? count : 0);
        const unsigned* from = cluster.map_shared_rank(s_cand, warp);
        const int theirs = min(__shfl_sync(0xffffffffu, count, warp), kEvCand - before);
        for (int i = lane; i < theirs; i += 32) s_all[before + i] = from[i];
      }
      __syncthreads();
      if (tid < equal) {
        const unsigned x = s_all[tid];
        int above = 0, same = 0;
        for (int i = 0; i < equal; ++i) {
          above += s_all[i] > x;
          same += s_all[i] == x;
        }
        if (above < need && need <= above + same) {  // (threads of equal keys write the same)
          s_cut = x;
          s_above = above;
          s_in = same;
        }
      }
      __syncthreads();
      cut = s_cut;
      ties = need - s_above;
      equal = s_in;
      break;
    }
  }
  // ---- holes and movers: a warp has a stretch of whole groups of 32 slots ----
  const int seg = (chunk + kEvThreads - 1) / kEvThreads * 32;
  const int w0 = min(end, begin + warp * seg), w1 = min(end, w0 + seg);
  int eq0 = 0;  // slots of the cut's key in front of this warp's
  if (ties < equal) {
    int eq = 0;
    for (int j = w0 + lane; j < w1; j += 32) eq += key(j) == cut;
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) s_scan[warp] = eq;
    __syncthreads();
    eq0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_scan[lane] : 0);
    if (tid == 0) s_eq = 0;
    __syncthreads();
    if (lane == 0) atomicAdd(&s_eq, eq);
    cluster.sync();
    const int others = ask(&s_eq, 0);
    eq0 += __reduce_add_sync(0xffffffffu, lane < rank ? others : 0);
  }
  // Lists.  In shared memory a warp's come first, movers from the front of its stretch and holes from its back, then the CTA's;
  // of longer stretches, in a second sweep, the i-th hole goes to the word of slot budget + i, the i-th mover to slot i's.
  int hole0 = 0, mover0 = 0;
  auto sweep = [&](bool to_words) {
    int eq = eq0;
    const unsigned before = (1u << lane) - 1;
    for (int base = w0; base < w1; base += 32) {
      const int j = base + lane;
      const bool in = j < w1;
      const unsigned x = in ? key(j) : 0u;
      bool kept = in && x >= cut;
      if (ties < equal) {
        const unsigned same = __ballot_sync(0xffffffffu, in && x == cut);
        if (x == cut && eq + __popc(same & before) >= ties) kept = false;
        eq += __popc(same);
      }
      const bool hole = in && j < budget && !kept, mover = j >= budget && kept;
      const unsigned holes = __ballot_sync(0xffffffffu, hole), movers = __ballot_sync(0xffffffffu, mover);
      const int h = hole0 + __popc(holes & before), m = mover0 + __popc(movers & before);
      if (hole || mover) {
        if (all_held) {
          s_pos[hole ? w1 - 1 - h - begin : w0 + m - begin] = j;
        } else if (to_words) {
          const long long at = !hole ? word(m) : h < n - budget ? word(budget + h) : -1;
          if (at >= 0) c.list[at] = j;
        }
      }
      hole0 += __popc(holes);
      mover0 += __popc(movers);
    }
  };
  sweep(false);
  const int my_holes = hole0, my_movers = mover0;
  if (lane == 0) s_hole[warp] = hole0, s_mover[warp] = mover0;
  __syncthreads();
  hole0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_hole[lane] : 0);
  mover0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_mover[lane] : 0);
  if (warp == 0) {
    const int h = __reduce_add_sync(0xffffffffu, lane < kEvWarps ? s_hole[lane] : 0);
    const int m = __reduce_add_sync(0xffffffffu, lane < kEvWarps ? s_mover[lane] : 0);
    if (lane == 0) s_holes = h, s_movers = m;
  }
  if (all_held) {
    for (int i = lane; i < my_movers; i += 32) s_list[mover0 + i] = s_pos[w0 - begin + i];
    for (int i = lane; i < my_holes; i += 32) s_list[held - 1 - hole0 - i] = s_pos[w1 - 1 - begin - i];
  }
  cluster.sync();
  m_incl = ask(&s_movers, 0);
  h_incl = ask(&s_holes, 0);
  count = __reduce_add_sync(0xffffffffu, m_incl);
#pragma unroll
  for (int d = 1; d < kEvMaxCluster; d <<= 1) {
    const int m = __shfl_up_sync(0xffffffffu, m_incl, d), h = __shfl_up_sync(0xffffffffu, h_incl, d);
    if (lane >= d) m_incl += m, h_incl += h;
  }
  if (!all_held) {
    const int m = __shfl_sync(0xffffffffu, m_incl, max(0, rank - 1)), h = __shfl_sync(0xffffffffu, h_incl, max(0, rank - 1));
    if (rank > 0) mover0 += m, hole0 += h;
    sweep(true);
    cluster.sync();
  }
  }
  if (bad) paged_status(c, row);
  // Entry i of the cluster's lists of movers or holes: in CTA k, the number of CTAs whose last entry lies in front of it.
  auto entry = [&](int incl, int i, bool of_holes) {
    int k = 0;
    for (int q = 0; q < C - 1; ++q) k += __shfl_sync(0xffffffffu, incl, q) <= i;
    const int before = __shfl_sync(0xffffffffu, incl, max(0, k - 1)) * (k > 0);
    const int* list = cluster.map_shared_rank(s_list, k);
    return i < count ? list[of_holes ? held - 1 - (i - before) : i - before] : -1;
  };
  // ---- moves: a lane finds out about one, then the warp copies them, K and V rows as 2 * row_bytes / 16 chunks a move ----
  const int stride = kEvWarps * C * kEvGroup;
  const int rounds = (2 * chunks + 31) / 32;
  const int together = 32 / min(32, 2 * chunks), mine = lane / min(32, 2 * chunks);  // moves that the lanes share at a time
  for (int base = (rank * kEvWarps + warp) * kEvGroup; base < count; base += 32 / kEvGroup * stride) {
    const int i = base + lane / kEvGroup * stride + lane % kEvGroup;
    long long from = -1, to = -1, wt = -1;
    float w = 0.f;
    int pos = 0;
    int src = -1, dst = -1;
    if (all_held) {
      src = entry(m_incl, i, false);
      dst = entry(h_incl, i, true);
    }
    if (i < count) {
      if (!all_held) {
        const long long a0 = word(i), a1 = word(budget + i);
        src = a0 < 0 ? -1 : __ldcg(&c.list[a0]);
        dst = a1 < 0 ? -1 : __ldcg(&c.list[a1]);
      }
      if ((unsigned)src < (unsigned)n && (unsigned)dst < (unsigned)n) {
        const int sn = paged_nth(c, src), dn = paged_nth(c, dst), sp = page_of(sn), dp = page_of(dn);
        if (sp >= 0 && dp >= 0) {
          from = (long long)paged_row(c, layer, sp, head, src - sn * c.P);
          to = (long long)paged_row(c, layer, dp, head, dst - dn * c.P);
          const size_t wf = paged_word(c, layer, sp, head, src - sn * c.P);
          wt = (long long)paged_word(c, layer, dp, head, dst - dn * c.P);
          w = c.w[wf];
          pos = c.pos[wf];
        }
      }
    }
    const int moves = __popc(__ballot_sync(0xffffffffu, i < count));  // (of the first lanes)
    for (int round = 0; round < rounds; ++round) {
      const int ch = (round * 32 + lane) & (2 * chunks - 1);
      unsigned char* pages = ch >= chunks ? c.v + (ch - chunks) * 16 : c.k + ch * 16;
      for (int m = 0; m < moves; m += kEvMoves * together) {
        uint4 x[kEvMoves];
#pragma unroll
        for (int b = 0; b < kEvMoves; ++b) {
          const int mv = m + b * together + mine;
          const long long f = shfl_ll(from, min(31, mv));
          if (f >= 0 && mv < moves) x[b] = __ldcg(reinterpret_cast<const uint4*>(pages + f));
        }
#pragma unroll
        for (int b = 0; b < kEvMoves; ++b) {
          const int mv = m + b * together + mine;
          const long long g = shfl_ll(to, min(31, mv));
          if (g >= 0 && mv < moves) __stcg(reinterpret_cast<uint4*>(pages + g), x[b]);
        }
      }
    }
    if (wt >= 0) {
      c.w[wt] = w;
      c.pos[wt] = pos;
    }
  }
  cluster.sync();  // no CTA leaves while its shared memory is read
}

cudaError_t prepare_paged_evict() {
  return allow_smem(k_paged_evict, kEvMaxSlots * 8);
}

// Largest cluster size that the device runs (a power of two).
int paged_evict_cluster() {
  for (int cl = kEvMaxCluster; cl > 1; cl >>= 1)
    if (active_clusters(k_paged_evict, cl, kEvThreads, kEvMaxSlots * 8) > 0) return cl;
  return 1;
}

cudaError_t launch_paged_evict(const PagedCache& c, const PagedRows& r, int layer_begin, int layer_count, int* new_lens,
                               int budget, int n_sink, int recent, cudaStream_t s) {
  const long long units = (long long)c.Hkv * r.n * layer_count;
  // Two CTAs for every SM, none with less than kEvSlots to do, and none with more than kEvLong: rows within their budget leave
  // at once, and a batch has few long ones (128 units, half of them of 32768 slots: 144 us in clusters of two, 112 in fours)
  int cl = 1;
  auto slots = [&] { return (r.cap + cl - 1) / cl; };
  while (cl < c.evict_cluster && slots() > kEvSlots && (units * cl <= c.sms || slots() > kEvLong)) cl *= 2;
  const int held = min(slots(), kEvMaxSlots);
  return launch_chained_cluster(k_paged_evict, dim3((unsigned)(units * cl)), dim3(kEvThreads), cl, held * 8, s, c, r,
                                layer_begin, layer_count, new_lens, budget, n_sink, recent, held);
}

}  // namespace ltri
