// Eviction from a caller-owned paged cache by accumulated attention weight.
//
// Per (layer, row, KV head) of n > budget slots: the budget-th largest key is found, where a key is a weight as an ordered
// integer and protected positions have the largest; slots below it are holes if they lie in front of the budget, slots above it
// move if they lie behind, the i-th into the i-th hole.  Sources and destinations are disjoint, so the moves need no order, and a
// full budget that has grown by one token costs one row, not a shifted cache.
//
// A cluster owns a unit; its CTAs hold a stretch of the slots each, as keys in shared memory.  A histogram of 2048 bins over the
// range that the keys really have, summed through distributed shared memory, leaves some ten keys around the cut (weights
// of a few powers of two); they are ranked against each other.  Where many are left (equal ones above all), up to two more
// histograms go through the bin's range instead.
//
// Bound: latency where few slots leave, HBM where many rows move (read once, written once).
#include <cooperative_groups.h>
#include <limits.h>

#include "paged.cuh"

namespace ltri {

namespace cg = cooperative_groups;

constexpr int kEvThreads = 512;  // two CTAs an SM: one's rows move while another's keys are counted
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvBinBits = 11, kEvBins = 1 << kEvBinBits;
constexpr int kEvMaxCluster = 16;
constexpr int kEvMaxSlots = 24576;  // keys that a CTA can hold (96 KB); those of longer stretches are made again for every pass
constexpr int kEvSlots = 4096;      // of a CTA, at least, before a unit gets more CTAs
constexpr int kEvCand = kEvThreads;       // keys around the cut that are ranked against each other
constexpr int kEvMoves = 8;         // 16-byte chunks that a lane has on their way

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
  extern __shared__ unsigned s_key[];  // [held]
  __shared__ __align__(16) unsigned s_hist[kEvBins];
  __shared__ unsigned s_cand[kEvCand], s_all[kEvCand];
  __shared__ int s_scan[kEvWarps], s_hole[kEvWarps], s_mover[kEvWarps];
  __shared__ int s_n, s_newest, s_stay, s_bin, s_above, s_in, s_eq, s_holes, s_movers, s_cands;
  __shared__ unsigned s_lo, s_hi, s_cut;
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
  }
  __syncthreads();
  const int n = s_n;
  // the lengths may be replaced in place: by the last CTA of the row to have read its
  if (tid == 32 && paged_arrive(&c.seen[row]) == layers * c.Hkv * C - 1) {
    c.seen[row] = 0;
    new_lens[row] = min(n, budget);
  }
  if (n <= budget) return;

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
  // ---- keys: a thread's slots in batches whose loads are all on their way at once ----
  int newest = INT_MIN;
  for (int j0 = begin + tid; j0 < end; j0 += 8 * kEvThreads) {
    long long at[8];
#pragma unroll
    for (int b = 0; b < 8; ++b) at[b] = j0 + b * kEvThreads < end ? word(j0 + b * kEvThreads) : -1;
    int pos[8];
#pragma unroll
    for (int b = 0; b < 8; ++b) pos[b] = at[b] >= 0 ? c.pos[at[b]] : INT_MIN;
#pragma unroll
    for (int b = 0; b < 8; ++b) newest = max(newest, pos[b]);
  }
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (lane == 0) atomicMax(&s_newest, newest);
  cluster.sync();
  newest = __reduce_max_sync(0xffffffffu, ask(&s_newest, INT_MIN));
  const long long first_recent = (long long)newest - recent;
  auto key_at = [&](long long at, int pos, float w) { return at < 0 ? 0u : ev_key(w, pos < n_sink || pos > first_recent); };
  auto key = [&](int slot) {
    if (slot - begin < held) return s_key[slot - begin];
    const long long at = word(slot);
    return at < 0 ? 0u : key_at(at, c.pos[at], c.w[at]);
  };
  unsigned lo = 0xffffffffu, hi = 0u;
  int stay = 0;
  for (int j0 = begin + tid; j0 < end; j0 += 4 * kEvThreads) {
    long long at[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) at[b] = j0 + b * kEvThreads < end ? word(j0 + b * kEvThreads) : -1;
    int pos[4];
    float w[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      pos[b] = at[b] >= 0 ? c.pos[at[b]] : 0;
      w[b] = at[b] >= 0 ? c.w[at[b]] : 0.f;
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int j = j0 + b * kEvThreads;
      if (j >= end) break;
      const unsigned x = key_at(at[b], pos[b], w[b]);
      if (j - begin < held) s_key[j - begin] = x;
      if (x == 0xffffffffu) ++stay;
      else lo = min(lo, x), hi = max(hi, x);
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  stay = __reduce_add_sync(0xffffffffu, stay);
  if (lane == 0) {
    atomicMin(&s_lo, lo);
    atomicMax(&s_hi, hi);
    atomicAdd(&s_stay, stay);
  }
  cluster.sync();
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
      if (from < need && need <= to) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (from < need && need <= from + sum[b]) {
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
        if (x >= lo && x <= hi && x != 0xffffffffu) s_cand[atomicAdd(&s_cands, 1)] = x;
      }
      cluster.sync();
      if (warp < C) {
        const int count = ask(&s_cands, 0), before = __reduce_add_sync(0xffffffffu, lane < warp ? count : 0);
        const unsigned* from = cluster.map_shared_rank(s_cand, warp);
        const int theirs = __shfl_sync(0xffffffffu, count, warp);
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
  int hole0 = 0, mover0 = 0;
  // lists: the i-th hole in the word of slot budget + i, the i-th mover in the word of slot i
  auto sweep = [&](bool emit) {
    int eq = eq0;
    const unsigned before = (1u << lane) - 1;
    for (int base = w0; base < w1; base += 4 * 32) {
      unsigned x[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) x[b] = base + b * 32 + lane < w1 ? key(base + b * 32 + lane) : 0u;
      int rank_in[4];  // of a hole, or of a mover behind all holes; -1: neither
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int j = base + b * 32 + lane;
        const bool in = j < w1;
        const unsigned same = __ballot_sync(0xffffffffu, in && x[b] == cut);
        const bool kept = in && (x[b] > cut || (x[b] == cut && eq + __popc(same & before) < ties));
        eq += __popc(same);
        const bool hole = in && j < budget && !kept, mover = j >= budget && kept;
        const unsigned holes = __ballot_sync(0xffffffffu, hole), movers = __ballot_sync(0xffffffffu, mover);
        rank_in[b] = hole ? budget + hole0 + __popc(holes & before) : mover ? mover0 + __popc(movers & before) : -1;
        hole0 += __popc(holes);
        mover0 += __popc(movers);
      }
      if (!emit) continue;
      long long at[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) at[b] = rank_in[b] >= 0 ? word(rank_in[b]) : -1;
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (at[b] >= 0) c.list[at[b]] = base + b * 32 + lane;
    }
  };
  sweep(false);
  if (lane == 0) s_hole[warp] = hole0, s_mover[warp] = mover0;
  __syncthreads();
  hole0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_hole[lane] : 0);
  mover0 = __reduce_add_sync(0xffffffffu, lane < warp ? s_mover[lane] : 0);
  if (warp == 0) {
    const int h = __reduce_add_sync(0xffffffffu, lane < kEvWarps ? s_hole[lane] : 0);
    const int m = __reduce_add_sync(0xffffffffu, lane < kEvWarps ? s_mover[lane] : 0);
    if (lane == 0) s_holes = h, s_movers = m;
  }
  cluster.sync();
  int count;
  {
    const int m = ask(&s_movers, 0), h = ask(&s_holes, 0);
    count = __reduce_add_sync(0xffffffffu, m);
    mover0 += __reduce_add_sync(0xffffffffu, lane < rank ? m : 0);
    hole0 += __reduce_add_sync(0xffffffffu, lane < rank ? h : 0);
  }
  sweep(true);
  cluster.sync();  // the lists are complete, and no CTA's shared memory is read from here on
  if (bad) paged_status(c, row);
  // ---- moves: a lane finds out about one, then the warp copies them, K and V rows as 2 * row_bytes / 16 chunks a move ----
  const int warps = kEvWarps * C, each = (count + warps - 1) / warps, m0 = (rank * kEvWarps + warp) * each;
  const int m1 = min(count, m0 + each);
  const int chunks = c.row_bytes / 16, shift = 32 - __clz(chunks);  // 2 * chunks = 1 << shift
  for (int base = m0; base < m1; base += 32) {
    const int i = base + lane;
    long long from = -1, to = -1;
    if (i < m1) {
      const long long a0 = word(i), a1 = word(budget + i);
      const int src = a0 < 0 ? -1 : __ldcg(&c.list[a0]), dst = a1 < 0 ? -1 : __ldcg(&c.list[a1]);
      if (src >= 0 && dst >= 0) {
        const int sn = paged_nth(c, src), dn = paged_nth(c, dst), sp = page_of(sn), dp = page_of(dn);
        if (sp >= 0 && dp >= 0) {
          from = (long long)paged_row(c, layer, sp, head, src - sn * c.P);
          to = (long long)paged_row(c, layer, dp, head, dst - dn * c.P);
          const size_t wf = paged_word(c, layer, sp, head, src - sn * c.P), wt = paged_word(c, layer, dp, head, dst - dn * c.P);
          const float w = c.w[wf];
          const int pos = c.pos[wf];
          c.w[wt] = w;
          c.pos[wt] = pos;
        }
      }
    }
    const int items = min(32, m1 - base) << shift;
    for (int t0 = 0; t0 < items; t0 += 32 * kEvMoves) {
      uint4 x[kEvMoves];
      unsigned char* dst[kEvMoves];
#pragma unroll
      for (int b = 0; b < kEvMoves; ++b) {
        const int item = t0 + b * 32 + lane, mv = min(item >> shift, 31), ch = item & (2 * chunks - 1);
        const long long f = shfl_ll(from, mv), g = shfl_ll(to, mv);
        const bool is_v = ch >= chunks;
        unsigned char* pages = (is_v ? c.v : c.k) + (is_v ? ch - chunks : ch) * 16;
        dst[b] = item < items && f >= 0 ? pages + g : nullptr;
        if (dst[b]) x[b] = __ldcs(reinterpret_cast<const uint4*>(pages + f));
      }
#pragma unroll
      for (int b = 0; b < kEvMoves; ++b)
        if (dst[b]) __stcs(reinterpret_cast<uint4*>(dst[b]), x[b]);
    }
  }
}

cudaError_t prepare_paged_evict() {
  const cudaError_t e = cudaFuncSetAttribute(k_paged_evict, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  return first_error(e, allow_smem(k_paged_evict, kEvMaxSlots * (int)sizeof(unsigned)));
}

// Largest cluster size that the device runs (a power of two).
int paged_evict_cluster() {
  for (int cl = kEvMaxCluster; cl > 1; cl >>= 1)
    if (active_clusters(k_paged_evict, cl, kEvThreads, kEvMaxSlots * (int)sizeof(unsigned)) > 0) return cl;
  return 1;
}

cudaError_t launch_paged_evict(const PagedCache& c, const PagedRows& r, int layer_begin, int layer_count, int* new_lens,
                               int budget, int n_sink, int recent, cudaStream_t s) {
  const long long units = (long long)c.Hkv * r.n * layer_count;
  // Two CTAs for every SM and again as many, since rows within their budget leave at once; none with less than kEvSlots to do
  int cl = 1;
  while (cl < c.evict_cluster && units * cl < 2 * c.sms && (r.cap + cl - 1) / cl > kEvSlots) cl *= 2;
  const int held = min((r.cap + cl - 1) / cl, kEvMaxSlots);
  return launch_chained_cluster(k_paged_evict, dim3((unsigned)(units * cl)), dim3(kEvThreads), cl, held * sizeof(unsigned), s, c, r,
                                layer_begin, layer_count, new_lens, budget, n_sink, recent, held);
}

}  // namespace ltri
