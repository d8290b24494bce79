// Attention of several new tokens per row (prompts, parts of prompts, drafted tokens) over a caller-owned paged cache that holds
// their K/V rows already: token i of a row's m sees the row's slots 0 .. lens - m + i.
//
// out_i = sum_j 2^(x_ij - L_i) V_j with x_ij = c q_i.K_j in log2 units and L_i = log2 sum_j 2^(x_ij); one pass over the slots with a
// running reference, as over a single token.  A query row is a (token, head of the KV head's group), so that a tile of K and V
// serves the whole group.
//
// Bound: the tensor cores where there are many tokens (two products of 2 D flops a pair of token and slot), so both run on
// tcgen05.mma: S = Q K^T from shared memory, O += P V with P in TMEM.  P enters as two 16-bit terms, the second what the first has
// left over: the outputs then carry the rounding of their type once, and the tensor pipe has three products to do instead of
// two.  Rows of 8 and 4 bits become halves on their way into shared memory, exactly; queries over them become halves too, each row
// scaled by a power of two.  With few tokens it is the cache's bytes and the CTAs' latency.
//
// Work: units are (row, KV head, block of query rows), as long as the tiles of slots that their last token sees.  A small kernel
// puts all units' tiles into one line, of which every CTA (one per SM) takes an equal run, across units if need be; the partial sums
// of units that CTAs share are joined by a third kernel, in the order of the line.
//
// Roles of a CTA's 17 warps: 0-3 and 4-7 softmax of the two tiles of 128 query rows (a thread a row; it also loads the row's
// queries and writes its outputs), 8-15 bring K and V tiles into shared memory, 16 issues the products.  TMEM: S0, S1, O0, O1 of
// 128 columns each; P replaces S in its columns.  head_dim 256: one tile of query rows, whose O takes 256 columns, and two S of 64
// columns in turn.
#include "paged_int4.cuh"
#include "tc_util.cuh"

namespace ltri {

using namespace tc;

enum { kPaBf16 = 0, kPaFp16 = 1, kPaE4m3 = 2, kPaInt4 = 3 };  // what the pages hold

template <int KIND, int D>
struct PaShape {
  static constexpr int kRow = KIND == kPaInt4 ? D / 2 : KIND == kPaE4m3 ? D : 2 * D;  // bytes of a cached row
  static constexpr int kQt = D == 256 ? 1 : 2;          // tiles of 128 query rows
  static constexpr int kSb = D == 256 ? 2 : 1;          // S of each
  static constexpr int kRows = 128 * kQt;               // query rows of a unit
  static constexpr int kTile = D == 256 ? 64 : 128;     // slots
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr int kMat = kTile * D * 2;            // bytes of a tile of K, or of V, in shared memory
  static constexpr int kQBytes = 128 * D * 2;           // of a tile of queries
  static constexpr int kSmem = kQt * kQBytes + kStages * 2 * kMat + 1024;
};

constexpr int kPaLoaders = 8;  // warps
constexpr int kPaThreads = 32 * (8 + kPaLoaders + 1);
// Upper bound of any single wait, in SM cycles (about ten seconds: a CTA's longest run of tiles lies far below)
constexpr long long kPaWaitLimit = 10 * kWaitLimitCycles;
constexpr float kPaNone = -3.0e38f;  // reference of sums that nothing has entered yet: below every logit, and finite

// A block of a row's query rows, and the first of its KV heads' tiles in the line (they follow each other).
struct __align__(32) PaEntry {
  int row, block;
  int start, m;      // the row's first token in q, its tokens
  int base;          // slots in front of the row's tokens (negative: tokens that have none)
  int tiles;         // of each KV head, one at least
  long long before;
};
struct PaPlan {
  long long total;   // tiles
  int entries;
  int pad;
};

struct PaWork {
  PaPlan* plan;
  PaEntry* entry;
  int max_entries;
  int* row_first;    // [n_rows + 1]: entries in front of a row's
  float* part;       // [CTAs][2]: partial sums, O as [tile][D / 4][128][4], then references and sums of the rows
};

template <int KIND, int D>
__host__ __device__ constexpr size_t pa_part_floats() {
  return (size_t)PaShape<KIND, D>::kRows * (D + 2);
}

__device__ __forceinline__ float pa_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Slots that the last token of a block sees.
__device__ __forceinline__ int pa_limit(const PaEntry& e, int G, int rows) {
  const int last = min(e.m * G, (e.block + 1) * rows) - 1;
  return max(0, e.base + min(last / G + 1, e.m));
}

// ---- the line of tiles ----
constexpr int kPlThreads = 1024;
__global__ void __launch_bounds__(kPlThreads)
    k_paged_attend_plan(PagedCache c, PagedRows r, const int* starts, long long n_tokens, PaWork wk, int rows, int tile) {
  __shared__ long long s_sum[32];
  __shared__ long long s_total;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_wait();
  // Sum of all threads in front of this one, and of all of them.
  auto scan = [&](long long x, long long& all) {
    long long inc = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = shfl_up_ll(inc, d);
      if (lane >= d) inc += y;
    }
    __syncthreads();
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    if (warp == 0) {
      const long long mine = s_sum[lane];
      long long w = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = shfl_up_ll(w, d);
        if (lane >= d) w += y;
      }
      s_sum[lane] = w - mine;
      if (lane == 31) s_total = w;
    }
    __syncthreads();
    all = s_total;
    return s_sum[warp] + inc - x;
  };
  // tokens of a row, none where the starts do not ascend within q
  auto tokens = [&](int row, int& start) {
    start = starts[row];
    const int end = starts[row + 1];
    if (start >= 0 && end >= start && end <= n_tokens) return end - start;
    paged_status(c, row);
    return 0;
  };
  long long entries = 0;
  for (int base = 0; base < r.n; base += kPlThreads) {
    const int row = base + tid;
    int start, n = 0;
    if (row < r.n) n = (tokens(row, start) * c.G + rows - 1) / rows;
    long long all;
    const long long at = entries + scan(n, all);
    if (row < r.n) wk.row_first[row] = (int)min(at, (long long)wk.max_entries);
    entries += all;
  }
  // (more than there is room for: the starts do not ascend)
  if (entries > wk.max_entries) {
    if (tid == 0) paged_status(c, 0);
    entries = wk.max_entries;
  }
  if (tid == 0) wk.row_first[r.n] = (int)entries;
  __threadfence_block();
  __syncthreads();
  long long total = 0;
  for (int base = 0; base < entries; base += kPlThreads) {
    const int at = base + tid;
    PaEntry e;
    long long n = 0;
    if (at < entries) {
      int lo = 0, hi = r.n - 1;  // the last row whose entries begin at or in front of this one
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (wk.row_first[mid] <= at) lo = mid;
        else hi = mid - 1;
      }
      e.row = lo;
      e.block = at - wk.row_first[lo];
      e.m = tokens(lo, e.start);
      e.base = paged_len(c, r, lo) - e.m;
      if (e.base < 0 && e.block == 0) paged_status(c, lo);
      e.tiles = max(1, (pa_limit(e, c.G, rows) + tile - 1) / tile);
      n = (long long)e.tiles * c.Hkv;
    }
    long long all;
    e.before = total + scan(n, all);
    if (at < entries) wk.entry[at] = e;
    total += all;
  }
  if (tid == 0) {
    wk.plan->total = total;
    wk.plan->entries = (int)entries;
  }
}

// A CTA's run of the line, part of a unit after the other.
struct PaWalk {
  PaEntry e;
  int at, head;       // entry, KV head
  int begin, end;     // tiles of the unit
  long long left;     // of the run, this part's included
};
__device__ __forceinline__ void pa_part(PaWalk& w) { w.end = (int)min((long long)w.e.tiles, w.begin + w.left); }
// The next part; false at the run's end.
__device__ __forceinline__ bool pa_next(PaWalk& w, const PaWork& wk, int heads) {
  w.left -= w.end - w.begin;
  if (w.left <= 0) return false;
  w.begin = 0;
  if (++w.head == heads) {
    w.head = 0;
    w.e = wk.entry[++w.at];
  }
  pa_part(w);
  return true;
}
// One warp: the entry of a tile (below the line's total).
__device__ __forceinline__ int pa_find(const PaWork& wk, int entries, long long tile) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = entries;  // the last one of lo .. lo + n - 1 that begins at or in front of the tile
  while (n > 1) {
    const int step = (n + 31) / 32, at = lane * step;
    const bool in = at < n && wk.entry[lo + at].before <= tile;
    const int which = __popc(__ballot_sync(0xffffffffu, in)) - 1;
    lo += which * step;
    n = min(step, n - which * step);
  }
  return lo;
}

// Two terms of `type` that add up to two fp32 values.
__device__ __forceinline__ void pa_terms(int type, float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = paged_pack(type, a, b);
  const float2 back = paged_unpack(type, hi);
  lo = paged_pack(type, a - back.x, b - back.y);
}

// Sixteen bytes of a cached row as 16-bit elements, in the order that the products take them (see pa_element).
template <int KIND>
struct PaChunk {
  static constexpr int kOut = KIND == kPaInt4 ? 4 : KIND == kPaE4m3 ? 2 : 1;  // chunks of 16 bytes
};

// Which element of each eight stands at place i of a 16-byte chunk: numbers of 4 bits come out of a word in pairs of i and i + 4.
template <int KIND>
__device__ __forceinline__ constexpr int pa_element(int i) {
  return KIND == kPaInt4 ? (i & 1) * 4 + i / 2 : i;
}

// Eight elements of a dense row in that order.
template <int KIND>
__device__ __forceinline__ uint4 pa_order(const uint4& x) {
  if (KIND != kPaInt4) return x;
  return make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                    __byte_perm(x.y, x.w, 0x7632));
}
// And back.
template <int KIND>
__device__ __forceinline__ uint4 pa_reorder(const uint4& x) {
  if (KIND != kPaInt4) return x;
  return make_uint4(__byte_perm(x.x, x.y, 0x5410), __byte_perm(x.z, x.w, 0x5410), __byte_perm(x.x, x.y, 0x7632),
                    __byte_perm(x.z, x.w, 0x7632));
}

__device__ __forceinline__ void pa_store(uint32_t to, const uint4& x) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}

// A row's elements [32 cg, 32 cg + 32) of `type` from values in the products' order, scaled.
template <int KIND>
__device__ __forceinline__ void pa_put32(int type, unsigned char* to, const float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 x = make_uint4(paged_pack(type, v[8 * i], v[8 * i + 1]), paged_pack(type, v[8 * i + 2], v[8 * i + 3]),
                               paged_pack(type, v[8 * i + 4], v[8 * i + 5]), paged_pack(type, v[8 * i + 6], v[8 * i + 7]));
    *reinterpret_cast<uint4*>(to + i * 16) = pa_reorder<KIND>(x);
  }
}

template <int KIND>
__device__ __forceinline__ float pa_v_scale(const PagedCache& c, int head) {
  return KIND == kPaInt4 ? kI4Back : KIND == kPaE4m3 ? c.vs[head] : 1.f;
}

template <int KIND, int D>
__global__ void __launch_bounds__(kPaThreads, 1)
    k_paged_attend(PagedCache c, int layer, const int* table, long long table_stride, PagedQueries a, PaWork wk) {
  using Sh = PaShape<KIND, D>;
  constexpr int QT = Sh::kQt, SB = Sh::kSb, TILE = Sh::kTile, S = Sh::kStages, ROWS = Sh::kRows;
  constexpr int kType = KIND == kPaBf16 ? LTRI_TYPE_BF16 : LTRI_TYPE_FP16;  // of the products
  // as for single tokens: halves have their largest probability at 2^kOff, and a reference moves only when a logit exceeds it
  // by kGrow
  constexpr float kOff = KIND == kPaBf16 ? 0.f : 10.f, kGrow = 4.f;
  extern __shared__ unsigned char smem_raw[];
  enum {
    B_KFULL = 0, B_VFULL = S, B_KEMPTY = 2 * S, B_VEMPTY = 3 * S, B_QFULL = 4 * S, B_SREADY = B_QFULL + QT,
    B_PREADY = B_SREADY + QT * SB, B_OFREE = B_PREADY + QT * SB, B_ODONE = B_OFREE + QT, B_PVDONE = B_ODONE + QT,
    B_DRAIN = B_PVDONE + 1, B_COUNT = B_DRAIN + 1
  };
  __shared__ __align__(8) unsigned long long bars[B_COUNT];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ PaWalk s_walk;
  // by tile: slots that have a page, a bit each.  (Eight tiles: when the K of tile j is written, that of j - S has met its
  // queries, and so the softmax of j - S - 1 and those in front of it have ended.)
  __shared__ __align__(16) unsigned short s_there[8][kPaLoaders];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = (smem_addr(smem_raw) + 1023u) & ~1023u, sQ = sbase, sKV = sbase + QT * Sh::kQBytes;
  auto bar = [&](int i) { return smem_addr(&bars[i]); };
  volatile int* abortp = &s_abort;
  auto wait = [&](int i, int parity) { return mbar_wait(bar(i), parity & 1, abortp, kPaWaitLimit); };
  auto arrive = [&](int i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(i));
  };

  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < S; ++i) {
      mbar_init(bar(B_KFULL + i), kPaLoaders);
      mbar_init(bar(B_VFULL + i), kPaLoaders);
      mbar_init(bar(B_KEMPTY + i), 1);
      mbar_init(bar(B_VEMPTY + i), 1);
    }
    for (int q = 0; q < QT; ++q) {
      mbar_init(bar(B_QFULL + q), 4);
      mbar_init(bar(B_OFREE + q), 4);
      mbar_init(bar(B_ODONE + q), 1);
      for (int b = 0; b < SB; ++b) {
        mbar_init(bar(B_SREADY + q * SB + b), 1);
        mbar_init(bar(B_PREADY + q * SB + b), 4);
      }
    }
    mbar_init(bar(B_PVDONE), 1);
    mbar_init(bar(B_DRAIN), 1);
    fence_mbar_init();
  }
  if (warp == 16) tmem_alloc(smem_addr(&s_tmem), 512);
  chain_wait();
  // the CTA's run
  const long long total = wk.plan->total;
  const long long per = (total + gridDim.x - 1) / gridDim.x, c0 = blockIdx.x * per;
  const bool works = c0 < total;
  if (warp == 0 && works) {
    const int at = pa_find(wk, wk.plan->entries, c0);
    if (lane == 0) {
      PaWalk w;
      w.e = wk.entry[at];
      w.at = at;
      w.head = (int)((c0 - w.e.before) / w.e.tiles);
      w.begin = (int)((c0 - w.e.before) % w.e.tiles);
      w.left = min(per, total - c0);
      pa_part(w);
      s_walk = w;
    }
  }
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = s_tmem;
  // query rows of a part's unit
  auto rows_of = [&](const PaEntry& e) { return min(ROWS, e.m * c.G - e.block * ROWS); };

  if (works && warp >= 8 && warp < 16) {
    // ------------------------------------------------------------------ K and V tiles
    constexpr int RC = Sh::kRow / 16, CL = RC < 4 ? RC : 4, SL = 32 / CL;  // lanes: SL slots, CL chunks of 16 bytes of each
    constexpr int PASSES = TILE / kPaLoaders / SL, KC = RC / CL;           // of slots, of chunks
    static_assert(PASSES >= 1 && PASSES * SL * kPaLoaders == TILE, "");
    constexpr int OUT = PaChunk<KIND>::kOut;
    const int lw = warp - 8, sub = lane % SL, ch0 = lane / SL;
    const unsigned char* pages_k = c.k + layer * c.ls;
    const long long vk = c.v - c.k;
    PaWalk wp = s_walk, wd = s_walk;  // of the page numbers that are asked for, of the rows that are
    int tp = wp.begin, td = wd.begin;
    bool more_p = true, more_d = true;
    auto step = [&](PaWalk& w, int& t, bool& more) {
      if (++t >= w.end) {
        more = pa_next(w, wk, c.Hkv);
        t = w.begin;
      }
    };
    int page[PASSES], page_next[PASSES];
    auto ask_pages = [&](int (&to)[PASSES]) {
      const int limit = pa_limit(wp.e, c.G, ROWS);
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int slot = tp * TILE + lw * (TILE / kPaLoaders) + p * SL + sub;
        to[p] = more_p && slot < limit ? table[wp.e.row * table_stride + paged_nth(c, slot)] : -1;
      }
      if (more_p) step(wp, tp, more_p);
    };
    // rows of a tile as they lie in the cache, and 4-bit rows' scales
    uint4 raw[2][PASSES][KC];
    unsigned scale[2][PASSES][KC];
    long long off[PASSES];
    int there;  // slots of the warp with a page, of the tile whose rows are on their way
    size_t word[PASSES];
    auto locate = [&]() {
      const int limit = pa_limit(wd.e, c.G, ROWS);
      there = 0;
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int slot = td * TILE + lw * (TILE / kPaLoaders) + p * SL + sub;
        const bool in = more_d && slot < limit, has = in && (unsigned)page[p] < (unsigned)c.n_pages;
        if (in && !has) paged_status(c, wd.e.row);
        const int place = slot - paged_nth(c, slot) * c.P;
        off[p] = has ? (long long)paged_row(c, 0, page[p], wd.head, place) : -1;
        if (KIND == kPaInt4) word[p] = has ? paged_word(c, layer, page[p], wd.head, place) : 0;
        const unsigned b = __ballot_sync(0xffffffffu, has || !in);  // (slots behind the limit are masked by their number)
        there |= (int)(b & ((1ull << SL) - 1)) << (p * SL);
      }
    };
    auto ask_rows = [&](int of_v) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          raw[of_v][p][k] = make_uint4(0u, 0u, 0u, 0u);
          scale[of_v][p][k] = 0u;
          if (off[p] < 0) continue;
          const int ch = ch0 + k * CL;
          raw[of_v][p][k] = *reinterpret_cast<const uint4*>(pages_k + (of_v ? vk : 0) + off[p] + ch * 16);
          if (KIND == kPaInt4) scale[of_v][p][k] = c.sc[(word[p] * 2 + of_v) * (D / kI4Block) + ch];
        }
    };
    auto write_rows = [&](int of_v, uint32_t mat) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const int row = lw * (TILE / kPaLoaders) + p * SL + sub, ch = ch0 + k * CL;
          const uint4& x = raw[of_v][p][k];
          const uint32_t in[4] = {x.x, x.y, x.z, x.w};
          I4Scale f;
          if (KIND == kPaInt4) f = i4_factors(scale[of_v][p][k] * 0x00800080u);
#pragma unroll
          for (int o = 0; o < OUT; ++o) {
            uint4 y = x;
            if (KIND == kPaInt4) {
              uint32_t v[4];
              i4_values(v, in[o], f);
              y = make_uint4(v[0], v[1], v[2], v[3]);
            }
            if (KIND == kPaE4m3) {
              uint32_t v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(in[2 * o + i / 2] >> (16 * (i & 1)));
                const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
                v[i] = (uint32_t)h.x | (uint32_t)h.y << 16;
              }
              y = make_uint4(v[0], v[1], v[2], v[3]);
            }
            const int oc = ch * OUT + o;  // 16-byte chunk of the dense row
            pa_store(mat + (oc >> 3) * (TILE * 128) + row * 128 + (((oc & 7) ^ (row & 7)) << 4), y);
          }
        }
      fence_async_smem();
    };
    ask_pages(page);
    locate();
    ask_rows(0);
    ask_rows(1);
    int there_now = there;
    ask_pages(page_next);
    bool ok = true;
    for (int jt = 0; more_d; ++jt) {
      const int st = jt % S;
      const uint32_t mat = sKV + st * 2 * Sh::kMat;
      step(wd, td, more_d);  // now of the next tile
#pragma unroll
      for (int p = 0; p < PASSES; ++p) page[p] = page_next[p];
      ask_pages(page_next);
      if (jt >= S) ok = wait(B_KEMPTY + st, jt / S - 1);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane == 0) s_there[jt & 7][lw] = (unsigned short)there_now;
      write_rows(0, mat);
      arrive(B_KFULL + st);
      locate();
      if (more_d) ask_rows(0);
      there_now = there;
      if (jt >= S) ok = wait(B_VEMPTY + st, jt / S - 1);
      if (!__all_sync(0xffffffffu, ok)) break;
      write_rows(1, mat + Sh::kMat);
      arrive(B_VFULL + st);
      if (more_d) ask_rows(1);
    }
  } else if (works && warp == 16) {
    // ------------------------------------------------------------------ products
    if (lane == 0) {
      constexpr uint32_t kFmt = kType == LTRI_TYPE_BF16 ? 1u : 0u;
      constexpr uint32_t kF = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (8u << 24);  // fp32 sums, both operands' type, M = 128
      constexpr uint32_t idesc_qk = kF | (uint32_t)(TILE >> 3) << 17, idesc_pv = kF | 1u << 16 | (uint32_t)(D >> 3) << 17;
      const uint64_t dQ = make_desc(sQ, 16, 1024), dK = make_desc(sKV, 16, 1024), dV = make_desc(sKV + Sh::kMat, TILE * 128, 1024);
      constexpr uint32_t kO = 256;  // first column of O
      auto s_col = [&](int q, int b) { return tmem + (SB == 2 ? b * TILE : q * 128); };
      auto issue_qk = [&](int q, int b, int st) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t half = ks >> 2, in = (ks & 3) * 32;
          mma_ss(s_col(q, b), dQ + ((q * Sh::kQBytes + half * 16384 + in) >> 4),
                 dK + ((uint32_t)(st * 2 * Sh::kMat + half * (TILE * 128) + in) >> 4), idesc_qk, ks > 0);
        }
        mma_commit(bar(B_SREADY + q * SB + b));
      };
      // P of 32 slots: 16 columns of first terms, 16 of second ones
      auto issue_pv = [&](int q, int b, int st, bool acc) {
#pragma unroll
        for (int ks = 0; ks < TILE / 16; ++ks) {
          const uint64_t db = dV + ((uint32_t)(st * 2 * Sh::kMat + ks * 2048) >> 4);
          const uint32_t pa = s_col(q, b) + (ks >> 1) * 32 + (ks & 1) * 8;
          mma_ts(tmem + kO + q * D, pa + 16, db, idesc_pv, acc || ks > 0);
          mma_ts(tmem + kO + q * D, pa, db, idesc_pv, true);
        }
      };
      PaWalk w = s_walk;
      int jt = 0, n[QT] = {}, units[QT] = {};  // tiles; of each tile of queries: tiles, parts
      bool ok = true;
      do {
        const int nq = QT == 2 && rows_of(w.e) > 128 ? 2 : 1, T = w.end - w.begin;
        for (int q = 0; ok && q < nq; ++q) ok = wait(B_QFULL + q, units[q]);
        if (ok) ok = wait(B_KFULL + jt % S, jt / S);
        if (!ok) break;
        fence_after_sync();
#pragma unroll
        for (int q = 0; q < QT; ++q)
          if (q < nq) issue_qk(q, n[q] % SB, jt % S);
        mma_commit(bar(B_KEMPTY + jt % S));
        for (int j = 0; ok && j < T; ++j, ++jt) {
          const int st = jt % S, nst = (jt + 1) % S;
          const bool next = j + 1 < T;
          if (SB == 2 && next) {
            ok = wait(B_KFULL + nst, (jt + 1) / S);
            if (!ok) break;
            fence_after_sync();
            issue_qk(0, (n[0] + 1) % SB, nst);
            mma_commit(bar(B_KEMPTY + nst));
          }
          ok = wait(B_VFULL + st, jt / S);
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            if (!ok || q >= nq) continue;
            ok = wait(B_PREADY + q * SB + n[q] % SB, n[q] / SB);
            // the first product of a part overwrites O: the one before it must have been read
            if (ok && j == 0 && units[q] > 0) ok = wait(B_OFREE + q, units[q] - 1);
            if (!ok) continue;
            fence_after_sync();
            issue_pv(q, n[q] % SB, st, j > 0);
            if (SB == 2) mma_commit(bar(B_PVDONE));
            if (SB == 1 && next) {
              if (q == 0) ok = wait(B_KFULL + nst, (jt + 1) / S);
              if (!ok) continue;
              fence_after_sync();
              issue_qk(q, 0, nst);
            }
            if (!next) mma_commit(bar(B_ODONE + q));
            ++n[q];
          }
          if (!ok) break;
          mma_commit(bar(B_VEMPTY + st));
          if (SB == 1 && next) mma_commit(bar(B_KEMPTY + nst));
        }
        for (int q = 0; q < nq; ++q) ++units[q];
      } while (ok && pa_next(w, wk, c.Hkv));
      // nothing of this CTA's is under way when it gives its TMEM back
      mma_commit(bar(B_DRAIN));
      const long long t0 = clock64();
      while (!mbar_try_suspend(bar(B_DRAIN), 0, 2000u) && clock64() - t0 < kPaWaitLimit) {
      }
    }
    __syncwarp();
  } else if (works && warp < 4 * QT) {
    // ------------------------------------------------------------------ softmax, queries and outputs: a thread a row
    const int q = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tO = tmem + lanes + 256 + q * D;
    PaWalk w = s_walk;
    int n = 0, unit = 0, jt = 0;  // tiles and parts of this tile of queries; the CTA's tiles
    bool ok = true, more = true;
    float back = 1.f;
    // the row's queries of part w into shared memory (free: all products with the last ones have been seen to end)
    auto load_queries = [&]() {
      const int rho = w.e.block * ROWS + q * 128 + r;
      const bool in = rho < w.e.m * c.G;
      const int tok = w.e.start + rho / c.G, h = w.head * c.G + rho % c.G;
      const unsigned char* from = a.q + (in ? tok * a.q_stride + (size_t)h * (D * 2) : 0);
      const uint32_t to = sQ + q * Sh::kQBytes + r * 128;
      back = 1.f;
      float u0 = 1.f, u1 = 1.f;
      if (KIND >= kPaE4m3 && c.type == LTRI_TYPE_BF16) {
        // bf16 queries as halves: a power of two brings the row's largest element to [2^14, 2^15)
        uint32_t most = 0;
        if (in) {
#pragma unroll 8
          for (int i = 0; i < D / 8; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(from + i * 16);
            most = __vmaxu2(most, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu),
                                           __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
          }
        }
        most = max(most & 0xffffu, most >> 16);
        const int ex = (int)(most >> 7);  // biased exponent
        const int up = ex == 0 || ex == 255 ? 0 : 127 + 14 - ex;
        // (2^up may lie outside fp32's range: two factors)
        u0 = __int_as_float((127 + up / 2) << 23), u1 = __int_as_float((127 + up - up / 2) << 23);
        back = __int_as_float((127 - up / 2) << 23) * __int_as_float((127 - up + up / 2) << 23);
      }
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        uint4 x = in ? *reinterpret_cast<const uint4*>(from + i * 16) : make_uint4(0u, 0u, 0u, 0u);
        if (KIND >= kPaE4m3 && c.type == LTRI_TYPE_BF16) {
          auto half = [&](uint32_t y) {
            const float2 f = paged_unpack(LTRI_TYPE_BF16, y);
            return paged_pack(LTRI_TYPE_FP16, f.x * u0 * u1, f.y * u0 * u1);
          };
          x = make_uint4(half(x.x), half(x.y), half(x.z), half(x.w));
        }
        pa_store(to + (i >> 3) * 16384 + (((i & 7) ^ (r & 7)) << 4), pa_order<KIND>(x));
      }
      fence_async_smem();
      arrive(B_QFULL + q);
    };
    // (a tile of queries without a row in the unit takes no part in it)
    auto skip = [&]() {
      while (more && rows_of(w.e) <= q * 128) {
        jt += w.end - w.begin;
        more = pa_next(w, wk, c.Hkv);
      }
    };
    skip();
    if (more) load_queries();
    while (more && ok) {
      const PaWalk now = w;
      const int rho = now.e.block * ROWS + q * 128 + r;
      const bool row_ok = rho < now.e.m * c.G;
      const int own = row_ok ? now.e.base + rho / c.G + 1 : 0;  // slots that the row sees
      float sc = c.scale;
      if (KIND == kPaInt4) sc = (float)((double)c.scale * back * kI4Back);
      if (KIND == kPaE4m3) sc = (float)((double)c.scale * c.ks[now.head] * back);
      if (KIND >= kPaE4m3 && sc < 0x1p-126f) sc = 0x1p-126f;  // (as for single tokens)
      float ref = kPaNone, sum = 0.f;
      for (int t = now.begin; t < now.end; ++t, ++n, ++jt) {
        const int b = n % SB;
        const uint32_t tS = tmem + lanes + (SB == 2 ? b * TILE : q * 128);
        ok = wait(B_SREADY + q * SB + b, n / SB);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        fence_after_sync();
        // columns that the row sees, as a number of the first ones, and where pages are missing, a bit each
        const int lim = own - t * TILE;
        const uint4 words = *reinterpret_cast<const uint4*>(s_there[jt & 7]);  // (16 slots a half-word, 8 where tiles are of 64)
        const uint32_t there[4] = {TILE == 128 ? words.x : __byte_perm(words.x, words.y, 0x6420),
                                   TILE == 128 ? words.y : __byte_perm(words.z, words.w, 0x6420), words.z, words.w};
        bool holes = false;
#pragma unroll
        for (int i = 0; i < TILE / 32; ++i) holes |= there[i] != 0xffffffffu;
        const bool masked = __any_sync(0xffffffffu, lim < TILE) || holes;
        auto mask = [&](uint32_t (&v)[32], int i) {
          const int l = lim - i * 32;
          const uint32_t m = (l >= 32 ? 0xffffffffu : l <= 0 ? 0u : (1u << l) - 1u) & there[i];
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!(m >> e & 1u)) v[e] = 0xff800000u;
        };
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < TILE / 32; ++i) {
          uint32_t v[32];
          tmem_ld32(tS + i * 32, v);
          tmem_ld_wait();
          if (masked) mask(v, i);
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 32; ++e) m4[e & 3] = fmaxf(m4[e & 3], __uint_as_float(v[e]));
          most = fmaxf(most, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])));
        }
        const float top = most * sc;
        const bool grow = top > ref + (kOff + kGrow);
        if (__any_sync(0xffffffffu, grow)) {
          const float to = grow ? fmaxf(ref, top - kOff) : ref, by = pa_exp2(ref - to);
          ref = to;
          sum *= by;
          if (t > now.begin) {
            if (SB == 2 && !wait(B_PVDONE, n - 1)) ok = false;
            fence_after_sync();
#pragma unroll 1
            for (int i = 0; i < D / 32; ++i) {
              uint32_t v[32];
              tmem_ld32(tO + i * 32, v);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * by);
              tmem_st32(tO + i * 32, v);
            }
            tmem_st_wait();
          }
        }
        float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < TILE / 32; ++i) {
          uint32_t v[32];
          tmem_ld32(tS + i * 32, v);
          tmem_ld_wait();
          if (masked) mask(v, i);
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p0 = pa_exp2(fmaf(__uint_as_float(v[2 * e]), sc, -ref));
            const float p1 = pa_exp2(fmaf(__uint_as_float(v[2 * e + 1]), sc, -ref));
            s4[e & 3] += p0 + p1;
            pa_terms(kType, p0, p1, hi[e], lo[e]);
          }
          tmem_st16(tS + i * 32, hi);
          tmem_st16(tS + i * 32 + 16, lo);
        }
        sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
        tmem_st_wait();
        fence_before_sync();
        arrive(B_PREADY + q * SB + b);
      }
      if (!ok) break;
      // the next part's queries while this one's last products run
      more = pa_next(w, wk, c.Hkv);
      skip();
      if (more) load_queries();
      ok = wait(B_ODONE + q, unit);
      if (!__all_sync(0xffffffffu, ok)) break;
      fence_after_sync();
      const bool whole = now.begin == 0 && now.end == now.e.tiles;
      const float by = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum, vs = whole ? pa_v_scale<KIND>(c, now.head) : 1.f;
      const int tok = now.e.start + rho / c.G, h = now.head * c.G + rho % c.G;
      float* part = wk.part + (size_t)(2 * blockIdx.x + (now.begin == 0 ? 1 : 0)) * pa_part_floats<KIND, D>();
#pragma unroll 1
      for (int i = 0; i < D / 32; ++i) {
        uint32_t v[32];
        tmem_ld32(tO + i * 32, v);
        tmem_ld_wait();
        float z[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) z[e] = __uint_as_float(v[e]) * by * vs;
        if (!row_ok) continue;
        if (whole) {
          pa_put32<KIND>(c.type, a.out + ((size_t)tok * c.Hq + h) * (D * 2) + i * 64, z);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<float4*>(part + ((size_t)(q * (D / 4) + i * 8 + e) * 128 + r) * 4) =
                make_float4(z[4 * e], z[4 * e + 1], z[4 * e + 2], z[4 * e + 3]);
        }
      }
      fence_before_sync();
      arrive(B_OFREE + q);
      if (row_ok) {
        if (whole && a.lse)
          a.lse[(size_t)tok * c.Hq + h] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
        if (!whole) *reinterpret_cast<float2*>(part + (size_t)ROWS * D + (q * 128 + r) * 2) = make_float2(ref, sum);
      }
      ++unit;
    }
  }
  __syncthreads();
  if (tid == 0 && s_abort && atomicCAS(&c.status[0], 0, (int)LTRI_ETIMEOUT) == 0) c.status[1] = blockIdx.x;
  if (warp == 16) tmem_dealloc(tmem, 512);
}

// Joins the parts of a unit that begins in CTA x's run and does not end there: 128 query rows of it, 32 elements a thread.
template <int KIND, int D>
__global__ void __launch_bounds__(128) k_paged_attend_join(PagedCache c, PagedQueries a, PaWork wk, int ctas) {
  using Sh = PaShape<KIND, D>;
  chain_wait();
  const long long total = wk.plan->total, per = (total + ctas - 1) / ctas;
  const long long c0 = blockIdx.x * per, c1 = c0 + per;
  if (c1 >= total) return;
  __shared__ int s_at;
  if (threadIdx.x < 32) {
    const int at = pa_find(wk, wk.plan->entries, c1 - 1);
    if (threadIdx.x == 0) s_at = at;
  }
  __syncthreads();
  const PaEntry e = wk.entry[s_at];
  const int head = (int)((c1 - 1 - e.before) / e.tiles);
  const long long begin = e.before + (long long)head * e.tiles, end = begin + e.tiles;
  if (begin < c0 || end == c1) return;
  const int parts = (int)((end - 1) / per - blockIdx.x) + 1;
  const int q = blockIdx.y, r = threadIdx.x, i = blockIdx.z;
  const int rho = e.block * Sh::kRows + q * 128 + r;
  if (rho >= e.m * c.G) return;
  const size_t stride = pa_part_floats<KIND, D>();
  const float* first = wk.part + (size_t)(2 * blockIdx.x + 1) * stride;
  auto part = [&](int k) { return k == 0 ? first : wk.part + (size_t)(2 * (blockIdx.x + k)) * stride; };
  float ref = kPaNone, sum = 0.f, z[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) z[k] = 0.f;
  for (int k = 0; k < parts; ++k) {
    const float2 m = *reinterpret_cast<const float2*>(part(k) + (size_t)Sh::kRows * D + (q * 128 + r) * 2);
    const float to = fmaxf(ref, m.x), f0 = pa_exp2(ref - to), f1 = pa_exp2(m.x - to);
    ref = to;
    sum = sum * f0 + m.y * f1;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float4 y = *reinterpret_cast<const float4*>(part(k) + ((size_t)(q * (D / 4) + i * 8 + x) * 128 + r) * 4);
      z[4 * x] = z[4 * x] * f0 + y.x * f1;
      z[4 * x + 1] = z[4 * x + 1] * f0 + y.y * f1;
      z[4 * x + 2] = z[4 * x + 2] * f0 + y.z * f1;
      z[4 * x + 3] = z[4 * x + 3] * f0 + y.w * f1;
    }
  }
  const float by = sum == 0.f ? 0.f : 1.f / sum, vs = pa_v_scale<KIND>(c, head);
#pragma unroll
  for (int k = 0; k < 32; ++k) z[k] = z[k] * by * vs;
  const int tok = e.start + rho / c.G, h = head * c.G + rho % c.G;
  pa_put32<KIND>(c.type, a.out + ((size_t)tok * c.Hq + h) * (D * 2) + i * 64, z);
  if (a.lse && i == 0) a.lse[(size_t)tok * c.Hq + h] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
}

namespace {

template <int KIND, int D>
cudaError_t prepare_one() {
  return allow_smem(k_paged_attend<KIND, D>, PaShape<KIND, D>::kSmem);
}
template <int KIND>
cudaError_t prepare_kind() {
  return first_error(prepare_one<KIND, 64>(), first_error(prepare_one<KIND, 128>(), prepare_one<KIND, 256>()));
}

template <int KIND, int D>
cudaError_t launch_one(const PagedCache& c, const PagedRows& r, int layer, const PagedQueries& a, const PaWork& wk, cudaStream_t s) {
  using Sh = PaShape<KIND, D>;
  cudaError_t e = launch_chained(k_paged_attend_plan, dim3(1), dim3(kPlThreads), 0, s, c, r, a.starts, a.n_tokens, wk, Sh::kRows,
                                 Sh::kTile);
  if (e != cudaSuccess) return e;
  e = launch_chained(k_paged_attend<KIND, D>, dim3(c.sms), dim3(kPaThreads), Sh::kSmem, s, c, layer, r.table, r.table_stride, a, wk);
  if (e != cudaSuccess) return e;
  return launch_chained(k_paged_attend_join<KIND, D>, dim3(c.sms, Sh::kQt, D / 32), dim3(128), 0, s, c, a, wk, c.sms);
}
template <int KIND>
cudaError_t launch_kind(const PagedCache& c, const PagedRows& r, int layer, const PagedQueries& a, const PaWork& wk, cudaStream_t s) {
  if (c.D == 64) return launch_one<KIND, 64>(c, r, layer, a, wk, s);
  if (c.D == 128) return launch_one<KIND, 128>(c, r, layer, a, wk, s);
  return launch_one<KIND, 256>(c, r, layer, a, wk, s);
}

int rows_of_unit(int D) { return D == 256 ? 128 : 256; }
long long entries_of(const PagedCache& c, long long n_tokens, long long n_rows) {
  return n_tokens * c.G / rows_of_unit(c.D) + n_rows;
}

// Carves the workspace; returns its size.
size_t layout(const PagedCache& c, long long n_tokens, long long n_rows, PaWork* wk, unsigned char* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* at = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  const long long entries = entries_of(c, n_tokens, n_rows);
  unsigned char *plan = take(sizeof(PaPlan)), *entry = take(entries * sizeof(PaEntry)), *rows = take((n_rows + 1) * sizeof(int));
  unsigned char* part = take((size_t)c.sms * 2 * rows_of_unit(c.D) * (c.D + 2) * sizeof(float));
  if (wk) *wk = PaWork{reinterpret_cast<PaPlan*>(plan), reinterpret_cast<PaEntry*>(entry), (int)entries,
                       reinterpret_cast<int*>(rows), reinterpret_cast<float*>(part)};
  return off;
}

}  // namespace

cudaError_t prepare_paged_attend() {
  return first_error(first_error(prepare_kind<kPaBf16>(), prepare_kind<kPaFp16>()),
                     first_error(prepare_kind<kPaE4m3>(), prepare_kind<kPaInt4>()));
}

size_t paged_attend_workspace(const PagedCache& c, long long n_tokens, long long n_rows) {
  return layout(c, n_tokens, n_rows, nullptr, nullptr);
}

cudaError_t launch_paged_attend(const PagedCache& c, const PagedRows& r, int layer, const PagedQueries& a, unsigned char* workspace,
                                cudaStream_t s) {
  PaWork wk;
  layout(c, a.n_tokens, r.n, &wk, workspace);
  if (c.cache_type == LTRI_TYPE_INT4) return launch_kind<kPaInt4>(c, r, layer, a, wk, s);
  if (c.cache_type == LTRI_TYPE_E4M3) return launch_kind<kPaE4m3>(c, r, layer, a, wk, s);
  if (c.type == LTRI_TYPE_BF16) return launch_kind<kPaBf16>(c, r, layer, a, wk, s);
  return launch_kind<kPaFp16>(c, r, layer, a, wk, s);
}

}  // namespace ltri
