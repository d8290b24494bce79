// Attention of several new tokens per row (prompts, parts of prompts, drafted tokens) over a caller-owned paged cache that holds
// their K/V rows already: token i of a row's m sees the row's slots 0 .. lens - m + i.
//
// out_i = sum_j 2^(x_ij - L_i) V_j with x_ij = c q_i.K_j in log2 units and L_i = log2 sum_j 2^(x_ij); one pass over the slots with a
// running reference, as over a single token.  A query row is a (token, head of the KV head's group), so that a tile of K and V
// serves the whole group.
//
// Bound: the tensor cores where there are many tokens (two products of 2 D flops a pair of token and slot), so both run on
// tcgen05.mma: S = Q K^T from shared memory, O += P V with P in TMEM.  P enters as two 16-bit terms, the second what the first has
// left over, so that the outputs carry the rounding of their type once, also where values cancel, and drafted tokens have what single
// ones have.  (One half's 11 bits would spare bf16 outputs a third of the tensor work, 226 us instead of 258 for 512 tokens over
// 24576 slots; of two probabilities 2^-14 apart whose V are 1 and -1 it leaves nothing.  Over bf16 pages two terms are 16 bits, and
// three would be fp32's: their 96 columns leave TMEM no room for a second S, without which the same call takes 469 us instead of
// 264, and at head_dim 256, where there is room, 647 instead of 545.)  Rows of 8 and 4 bits become halves on their way into
// shared memory, exactly; queries over them become halves too, each row scaled by a power of two.  With few tokens it is the
// cache's bytes and the CTAs' latency.
//
// A probability of 0 times a value that is not finite is NaN, which a later token's V row must not make of an earlier one's outputs.
// So the V rows of the call's own tokens are looked through beforehand, beside the dealing of the work (their bytes once more: calls are
// 0 to 2% longer; looking at every row as it comes into shared memory: prompts 8%).  Where any is not finite, such elements enter the
// products as 0 in slots that some of a unit's tokens do not see, and outputs of tokens that do see them become NaN as they are written.
//
// Work: units are (row, KV head, block of query rows), as long as the tiles of slots that their last token sees.  A small kernel
// puts all units' tiles into one line, of which every CTA (one per SM) takes an equal run, across units if need be; the partial sums
// of units that CTAs share are joined by a third kernel, in the order of the line.
//
// Roles of a CTA's 28 warps: 0-7 and 8-15 softmax of the two tiles of 128 query rows (16 rows a warp, four lanes a row; they also load
// the queries and write the outputs, two threads a row), 16-19 bring K tiles into shared memory, 20-23 V tiles, 24 and 25 issue the
// products.  TMEM: two S of 64 columns in turn for each tile of query rows, in whose columns P replaces S, then the two O.  head_dim
// 256: one tile of query rows.
//
// Measured over 4-bit pages, 32 query and 8 KV heads of 128: 512 tokens over 24576 slots 249 to 261 us in a short series of calls,
// 279 to 285 in a long one, which the power limit slows (715 TFLOP/s; 122 us at the rate of large matrix products), three prompts of up
// to 16384 tokens in fp16 4.2 ms, and 4.7 in a long series, 16 ragged rows of up to 8000 slots with five tokens each 57 to 59 us.
#include "paged_int4.cuh"
#include "tc_util.cuh"

namespace ltri {

using namespace tc;

enum { kPaBf16 = 0, kPaFp16 = 1, kPaE4m3 = 2, kPaInt4 = 3 };  // what the pages hold

template <int KIND, int D>
struct PaShape {
  static constexpr int kRow = KIND == kPaInt4 ? D / 2 : KIND == kPaE4m3 ? D : 2 * D;  // bytes of a cached row
  static constexpr int kQt = D == 256 ? 1 : 2;          // tiles of 128 query rows
  static constexpr int kSb = 2;                         // S of each, of 64 slots
  static constexpr int kRows = 128 * kQt;               // query rows of a unit
  static constexpr int kTile = D == 256 ? 64 : 128;     // slots
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr int kMat = kTile * D * 2;            // bytes of a tile of K, or of V, in shared memory
  static constexpr int kQBytes = 128 * D * 2;           // of a tile of queries
  static constexpr int kSmem = kQt * kQBytes + kStages * 2 * kMat + 1024;
};

constexpr int kPaSoftmax = 16, kPaLoaders = 8;  // warps
constexpr int kPaIssuer = kPaSoftmax + kPaLoaders;  // this warp
constexpr int kPaThreads = 32 * (kPaIssuer + 4);
// Registers a thread: of the launch (prepare_kernel sees that it has them), and of the roles, which add up to them.  (All
// 72, which the softmax's loop has not enough of: with one term of the probabilities 512 tokens over 24576 slots 234 us, with these
// 225; five drafted tokens of 16 rows 62 and 58; 96, 40 and 40, or 88, 64 and 24: no faster.)
constexpr int kPaRegs = 72, kPaSoftmaxRegs = 88, kPaLoadRegs = 56, kPaIssueRegs = 40;
static_assert(kPaSoftmax * kPaSoftmaxRegs + kPaLoaders * kPaLoadRegs + 4 * kPaIssueRegs <= kPaThreads / 32 * kPaRegs,
              "more would wait for ever");
// Upper bound of the wait for a CTA's last products, in SM cycles, whatever the handle's limit: TMEM is theirs until they end.
constexpr long long kPaDrainLimit = 10 * kWaitLimitCycles;
constexpr float kPaNone = -3.0e38f;  // reference of sums that nothing has entered yet: below every logit, and finite

// A block of a row's query rows, and the first of its KV heads' places in the line (they follow each other).
struct __align__(32) PaEntry {
  int row, block;
  int start, m;      // the row's first token in q, its tokens
  int base;          // slots in front of the row's tokens (negative: tokens that have none)
  int tiles;         // of each KV head, one at least
  long long before;
};
struct PaPlan {
  long long total;   // places
  int entries;
  int pad;
};

struct PaWork {
  PaPlan* plan;
  PaEntry* entry;
  int max_entries;
  int* row_first;    // [n_rows + 1]: entries in front of a row's
  int* spoilt;       // [scans]: whether a CTA has found tokens' V rows that are not finite
  int scans;
  float* part;       // [CTAs][2]: partial sums, O as [tile][D / 4][128][4], then references and sums of the rows
};

template <int KIND, int D>
__host__ __device__ constexpr size_t pa_part_floats() {
  return (size_t)PaShape<KIND, D>::kRows * (D + 2);
}

// mbar_wait with all but the first try out of line
static __device__ __noinline__ bool pa_wait_long(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
  return mbar_wait(bar, parity, abort_flag, limit);
}
__device__ __forceinline__ bool pa_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
  return mbar_try(bar, parity) || pa_wait_long(bar, parity, abort_flag, limit);
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

// What a unit costs besides its tiles (queries to be loaded, outputs to be written, while the products wait), as tiles: it takes so
// many more places in the line.  Four where more than 128 query rows are left of the row's, so that both tiles of query rows have some,
// or the unit is full at head_dim 256, where a tile has half the slots; else two.  (None: the CTAs with the shortest units were
// through 1.3 times as late as the others.  Of 16 ragged rows of five tokens, with 2 58 us; 1 or 3 60, 4 62; of three prompts of up to
// 16384 tokens, with 4 4.0 to 4.2 ms in a stream of calls; 1 4.9, 2 4.4, 3 4.1 to 4.2: both measured with one term of the
// probabilities.  Head_dim 256, prompts of 8192 and 3001 tokens: 2.07 ms, with 2 for all units 2.49.)
__device__ __forceinline__ int pa_extra(const PaEntry& e, int G, int rows) { return e.m * G - e.block * rows > 128 ? 4 : 2; }

// Elements of `type` that are not finite, their exponents all ones: the upper bits of those halves of x, after one more in the last
// place of the exponent.
__device__ __forceinline__ uint32_t pa_not_finite(int type, uint32_t x) {
  return (type == LTRI_TYPE_BF16 ? (x & 0x7f807f80u) + 0x00800080u : (x & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
}
// They become 0.
__device__ __forceinline__ uint32_t pa_finite(int type, uint32_t x) { return x & ~((pa_not_finite(type, x) >> 15) * 0xffffu); }

// ---- V rows of the call's own tokens that are not finite: a token a warp ----
__device__ __forceinline__ bool pa_scan(const PagedCache& c, const PagedRows& r, int layer, const int* starts, long long n_tokens,
                                        long long first, long long step) {
  // (a lane has 16 bytes of a row, of 4-bit rows the scale of a block)
  const int lane = threadIdx.x & 31, of_row = c.cache_type == LTRI_TYPE_INT4 ? c.D / 32 : c.row_bytes / 16;
  bool bad = false;
  for (long long tok = first; tok < n_tokens; tok += step) {
    int lo = 0, hi = r.n;  // the last row that starts at or in front of the token
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (starts[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    if (lo >= r.n || starts[lo] > tok || starts[lo] < 0) continue;
    const int n = r.lens[lo], end = starts[lo + 1];
    const long long slot = (long long)n - end + tok;
    if (tok >= end || end > n_tokens || (unsigned)n > (unsigned)r.cap || slot < 0) continue;
    const int nth = paged_nth(c, (int)slot), page = r.table[lo * r.table_stride + nth], place = (int)slot - nth * c.P;
    if ((unsigned)page >= (unsigned)c.n_pages) continue;
    for (int i = lane; i < c.Hkv * of_row; i += 32) {
      const int head = i / of_row, in = i % of_row;
      if (c.cache_type == LTRI_TYPE_INT4) {
        bad |= (c.sc[paged_word(c, layer, page, head, place) * (c.D / 16) + c.D / 32 + in] & 0xf8) == 0xf8;
      } else {
        const uint4 x = *reinterpret_cast<const uint4*>(c.v + paged_row(c, layer, page, head, place) + in * 16);
        if (c.cache_type == LTRI_TYPE_E4M3) {
          auto nan = [](uint32_t y) { return ((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
          bad |= (nan(x.x) | nan(x.y) | nan(x.z) | nan(x.w)) != 0u;
        } else {
          bad |= (pa_not_finite(c.type, x.x) | pa_not_finite(c.type, x.y) | pa_not_finite(c.type, x.z) | pa_not_finite(c.type, x.w)) != 0u;
        }
      }
    }
  }
  return bad;
}

// ---- the line of tiles ----
constexpr int kPlThreads = 1024;
__global__ void __launch_bounds__(kPlThreads)
    k_paged_attend_plan(PagedCache c, PagedRows r, int layer, const int* starts, long long n_tokens, PaWork wk, int rows, int tile) {
  __shared__ long long s_sum[32];
  __shared__ long long s_total;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_wait();
  if (blockIdx.x > 0) {
    const long long warps = kPlThreads / 32, mine = blockIdx.x - 1;
    const bool bad = pa_scan(c, r, layer, starts, n_tokens, mine * warps + warp, wk.scans * warps);
    const int any = __syncthreads_or(bad);
    if (tid == 0) wk.spoilt[mine] = any;
    return;
  }
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
      n = (long long)(e.tiles + pa_extra(e, c.G, rows)) * c.Hkv;
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

// A place in a CTA's run of the line: a part of a unit after the other, in stretches of up to `most` tiles, and their tiles.
struct PaPlace {
  int at, head;           // entry, KV head
  int row, start;         // of the batch; the row's first token in q
  int rows, rho;          // query rows of the row, and the unit's first
  int base, limit;        // slots in front of the row's tokens, and those that the unit's last token sees
  int tiles, extra;       // of the unit; its places in front of them
  int first, stop;        // the part's first tile, and behind it
  int tile, end;          // the place; behind the stretch
  long long left;         // places of the run behind the part
};
__device__ __forceinline__ void pa_entry(PaPlace& w, const PaEntry& e, int G, int rows) {
  w.row = e.row;
  w.start = e.start;
  w.rows = e.m * G;
  w.rho = e.block * rows;
  w.base = e.base;
  w.limit = pa_limit(e, G, rows);
  w.tiles = e.tiles;
  w.extra = pa_extra(e, G, rows);
}
// The unit's part in the run, whose next place is the unit's number `at`; false if it has none (the run ends in front of the first
// tile).
__device__ __forceinline__ bool pa_part(PaPlace& w, int at, int most) {
  const int n = (int)min((long long)(w.tiles + w.extra - at), w.left);
  w.left -= n;
  w.first = w.tile = max(0, at - w.extra);
  w.stop = max(0, at + n - w.extra);
  w.end = min(w.stop, w.tile + most);
  return w.tile < w.end;
}
// The next stretch; false at the run's end.
__device__ __forceinline__ bool pa_next(PaPlace& w, const PaWork& wk, int heads, int G, int rows, int most) {
  if (w.end < w.stop) {
    w.tile = w.end;
    w.end = min(w.stop, w.tile + most);
    return true;
  }
  if (w.left <= 0) return false;
  if (++w.head == heads) {
    w.head = 0;
    pa_entry(w, wk.entry[++w.at], G, rows);
  }
  return pa_part(w, 0, most);
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

// Pairs of fp32 values, one instruction for both.
__device__ __forceinline__ unsigned long long pa_pair(float a, float b) {
  unsigned long long x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ float2 pa_split(unsigned long long x) {
  float2 y;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(y.x), "=f"(y.y) : "l"(x));
  return y;
}
__device__ __forceinline__ unsigned long long pa_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long pa_add2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// Two terms of `type` that add up to a pair of fp32 values.
__device__ __forceinline__ void pa_terms(int type, unsigned long long p, uint32_t& hi, uint32_t& lo) {
  const float2 f = pa_split(p);
  hi = paged_pack(type, f.x, f.y);
  const float2 back = paged_unpack(type, hi);
  const float2 rest = pa_split(pa_fma2(pa_pair(back.x, back.y), pa_pair(-1.f, -1.f), p));
  lo = paged_pack(type, rest.x, rest.y);
}
// A barrier of 256 threads: whether it is so for any of them.
__device__ __forceinline__ bool pa_any(int id, bool so) {
  uint32_t any;
  asm volatile(
      "{\n.reg .pred p, r;\nsetp.ne.b32 p, %1, 0;\nbar.red.or.pred r, %2, 256, p;\nselp.u32 %0, 1, 0, r;\n}\n"
      : "=r"(any)
      : "r"((uint32_t)so), "r"(id)
      : "memory");
  return any != 0;
}
// The products' instructions, for a warp that runs together: one of its lanes issues, and the operands are the warp's.  (A single
// lane in a branch of its own: 512 tokens over 24576 slots take 248 us, 241 so.)
__device__ __forceinline__ void pa_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void pa_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void pa_commit(uint32_t bar) {
  asm volatile(
      "{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar)
      : "memory");
}
// TMEM in the layout of mma.sync's accumulators: a warp has 16 rows, its lane t rows t / 4 and t / 4 + 8; of every eight columns
// t % 4 * 2 and the next one (r[4 i], r[4 i + 1]; r[4 i + 2], r[4 i + 3]), of every four columns of pairs t % 4 (r[2 i]; r[2 i + 1]).
__device__ __forceinline__ void pa_ld64(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void pa_ld32(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void pa_st32(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void pa_st_pairs(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// A bulk of 16 bytes on its way into shared memory, or zeros.
__device__ __forceinline__ void pa_request(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// Sixteen bytes of a cached row as 16-bit elements, in the order that the products take them (see pa_order).
template <int KIND>
struct PaChunk {
  static constexpr int kOut = KIND == kPaInt4 ? 4 : KIND == kPaE4m3 ? 2 : 1;  // chunks of 16 bytes
};

// Eight elements of a dense row in that order: numbers of 4 bits come out of a word in pairs of element i and i + 4.
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

// Of 32 elements those that are not finite in any of a row's slots [slot, end), a bit each.  (Out of line, and seldom called.)  `at`:
// the elements of page 0's first place, or, of 4-bit rows, the byte of their scale; `ps` and `ts` its strides.
template <int KIND>
static __device__ __noinline__ uint32_t pa_spoilt(const unsigned char* at, long long ps, long long ts, const int* pages, int n_pages,
                                                  int P, unsigned p_mul, int p_shift, int slot, int end) {
  uint32_t bits = 0u;
#pragma unroll 1
  for (; slot < end; ++slot) {
    const int nth = (int)(((unsigned long long)(unsigned)slot * p_mul) >> p_shift), page = pages[nth];
    if ((unsigned)page >= (unsigned)n_pages) continue;
    const unsigned char* x = at + (unsigned)page * ps + (unsigned)(slot - nth * P) * ts;
    if (KIND == kPaInt4) {
      if ((*x & 0xf8) == 0xf8) return 0xffffffffu;
    } else if (KIND == kPaE4m3) {
#pragma unroll 1
      for (int i = 0; i < 32; ++i) bits |= (uint32_t)((x[i] & 0x7f) == 0x7f) << i;
    } else {
      constexpr unsigned kMost = KIND == kPaBf16 ? 0x7f80u : 0x7c00u;
#pragma unroll 1
      for (int i = 0; i < 32; ++i) bits |= (uint32_t)((reinterpret_cast<const unsigned short*>(x)[i] & kMost) == kMost) << i;
    }
  }
  return bits;
}

template <int KIND>
__device__ __forceinline__ float pa_v_scale(const PagedCache& c, int head) {
  return KIND == kPaInt4 ? kI4Back : KIND == kPaE4m3 ? c.vs[head] : 1.f;
}

template <int KIND, int D>
__global__ void __launch_bounds__(kPaThreads, 1)
    k_paged_attend(PagedCache c, int layer, const int* table, long long table_stride, PagedQueries a, PaWork wk) {
  using Sh = PaShape<KIND, D>;
  constexpr int QT = Sh::kQt, SB = Sh::kSb, TILE = Sh::kTile, S = Sh::kStages, ROWS = Sh::kRows, SUBS = TILE / 64;
  constexpr int kType = KIND == kPaBf16 ? LTRI_TYPE_BF16 : LTRI_TYPE_FP16;  // of the products
  // as for single tokens: halves have their largest probability at 2^kOff, and a reference moves only when a logit exceeds it
  // by kGrow
  constexpr float kOff = KIND == kPaBf16 ? 0.f : 10.f, kGrow = 4.f;
  // Tiles that O adds up before its sums go elsewhere.  (The tensor cores cut off what an accumulator has no bits for, towards zero.
  // Measured over values of one sign: 2^13 slots take 2^-14 of the sum, an eighth of fp16 outputs' half step, 2^16 2^-11.  For as
  // long as a CTA's part is, fp16 outputs over 108152 slots of 12 heads were off by 1.2 times what their rounding is, and bf16 ones
  // that values of both signs leave small by more than theirs.)
  constexpr int kMost = (1 << 13) / TILE;
  extern __shared__ unsigned char smem_raw[];
  enum {
    B_KFULL = 0, B_VFULL = S, B_KEMPTY = 2 * S, B_VEMPTY = 3 * S, B_QFULL = 4 * S, B_SREADY = B_QFULL + QT,
    B_PREADY = B_SREADY + QT * SB, B_OFREE = B_PREADY + QT * SB, B_ODONE = B_OFREE + QT, B_PVDONE = B_ODONE + QT,
    B_DRAIN = B_PVDONE + QT, B_COUNT = B_DRAIN + 1
  };
  __shared__ __align__(8) unsigned long long bars[B_COUNT];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ PaPlace s_place;
  // by tile: slots that have a page, a bit each.  (Eight tiles: when the K of tile j is written, that of j - S has met its
  // queries, which takes that the softmax of j - S - 1 and those in front of it have ended.)
  __shared__ __align__(16) uint32_t s_there[8][4];
  // of a tile of queries' rows: references and sums, what their queries were divided by, and the largest elements of those' halves
  __shared__ float s_ref[QT][128], s_sum[QT][128], s_back[QT][128];
  __shared__ uint32_t s_most[QT][2][128];
  // where the softmax's warps are, while their loops run, which want the registers
  __shared__ PaPlace s_where[kPaSoftmax];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = (smem_addr(smem_raw) + 1023u) & ~1023u, sQ = sbase, sKV = sbase + QT * Sh::kQBytes;
  auto bar = [&](int i) { return smem_addr(&bars[i]); };
  volatile int* abortp = &s_abort;
  auto wait = [&](int i, int parity) { return mbar_wait(bar(i), parity & 1, abortp, c.wait_limit); };
  auto arrive = [&](int i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(i));
  };

  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < S; ++i) {
      mbar_init(bar(B_KFULL + i), kPaLoaders / 2);
      mbar_init(bar(B_VFULL + i), kPaLoaders / 2);
      mbar_init(bar(B_KEMPTY + i), QT);
      mbar_init(bar(B_VEMPTY + i), QT);
    }
    for (int q = 0; q < QT; ++q) {
      mbar_init(bar(B_QFULL + q), 8);
      mbar_init(bar(B_OFREE + q), 8);
      mbar_init(bar(B_ODONE + q), 1);
      mbar_init(bar(B_PVDONE + q), 1);
      for (int b = 0; b < SB; ++b) {
        mbar_init(bar(B_SREADY + q * SB + b), 1);
        mbar_init(bar(B_PREADY + q * SB + b), 8);
      }
    }
    mbar_init(bar(B_DRAIN), QT);
    fence_mbar_init();
  }
  if (warp == kPaIssuer) tmem_alloc(smem_addr(&s_tmem), 512);
  chain_wait();
  // the CTA's run
  const long long total = wk.plan->total;
  const long long per = (total + gridDim.x - 1) / gridDim.x, c0 = blockIdx.x * per;
  __shared__ bool s_works, s_spoilt;
  if (warp == 1) {
    int bad = 0;
    for (int i = lane; i < wk.scans; i += 32) bad |= wk.spoilt[i];
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) s_spoilt = bad != 0;
  }
  if (tid == 0 && c0 >= total) s_works = false;
  if (warp == 0 && c0 < total) {
    const int at = pa_find(wk, wk.plan->entries, c0);
    if (lane == 0) {
      const PaEntry e = wk.entry[at];
      PaPlace w;
      pa_entry(w, e, c.G, ROWS);
      w.at = at;
      w.head = (int)((c0 - e.before) / (e.tiles + w.extra));
      w.left = min(per, total - c0);
      s_works = pa_part(w, (int)((c0 - e.before) % (e.tiles + w.extra)), kMost);
      s_place = w;
    }
  }
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = s_tmem;
  const bool works = s_works;
  auto next_part = [&](PaPlace& w) { return pa_next(w, wk, c.Hkv, c.G, ROWS, kMost); };

  if (warp >= kPaSoftmax && warp < kPaIssuer) {
    // ------------------------------------------------------------------ K and V tiles
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPaLoadRegs));
    // Four warps bring K and four V, so that what a tile costs them (page numbers, addresses, the wait for its stage) passes twice
    // at a time.
    constexpr int RC = Sh::kRow / 16, CL = RC < 4 ? RC : 4, SL = 32 / CL;  // lanes: SL slots, CL chunks of 16 bytes of each
    constexpr int MINE = TILE / 4, PASSES = MINE / SL, KC = RC / CL;       // slots of a warp; passes of slots, of chunks
    static_assert(PASSES >= 1 && PASSES * SL == MINE && SL % 8 == 0 && (MINE == 32 || MINE == 16), "a warp's slots");
    constexpr bool kCopy = KIND == kPaBf16 || KIND == kPaFp16;  // rows go into shared memory as they are
    const bool of_v = warp - kPaSoftmax >= 4;
    const int lw = warp & 3, sub = lane % SL, ch0 = lane / SL, full = of_v ? B_VFULL : B_KFULL;
    const unsigned char* pages = (of_v ? c.v : c.k) + layer * c.ls;
    bool more_p = works, more_d = works && !(c.held >> of_v & 1);
    PaPlace wd = s_place, wp = s_place;  // of the rows that are asked for, of the page numbers
    // A lane finds out about one of the warp's slots, and the others ask it.  (Every lane about those whose rows it loads: 3000 of
    // 9300 cycles a tile.)
    int page, page_next;
    const int mine = lw * MINE + lane % MINE;
    const int* pages_row = table + wp.row * table_stride;
    auto ask_page = [&]() {
      const int slot = wp.tile * TILE + mine;
      const int x = more_p && slot < wp.limit ? pages_row[paged_nth(c, slot)] : -1;
      if (++wp.tile == wp.end && more_p) {
        more_p = next_part(wp);
        pages_row = table + wp.row * table_stride;
      }
      return x;
    };
    const unsigned char* head_row = pages + wd.head * c.hs;
    long long off = -1;
    uint32_t there = 0;  // slots with a page, of the tile whose rows are asked for
    constexpr int SW = D <= 128 ? 1 : 2;
    uint32_t scales[SW];  // of a 4-bit row (64 elements: K's and V's in one word); 0 where there is no slot
    auto locate = [&]() {
      const int slot = wd.tile * TILE + mine;
      const bool in = more_d && slot < wd.limit, has = in && (unsigned)page < (unsigned)c.n_pages;
      if (in && !has) paged_status(c, wd.row);
      const int place = slot - paged_nth(c, slot) * c.P;
      off = has ? (unsigned)page * c.ps + (unsigned)place * c.ts : -1;
      if constexpr (KIND == kPaInt4) {
        const size_t word = has ? paged_word(c, layer, page, wd.head, place) : 0;
        const uint32_t* sc = reinterpret_cast<const uint32_t*>(c.sc) + (D == 64 ? word : (word * 2 + of_v) * SW);
#pragma unroll
        for (int i = 0; i < SW; ++i) scales[i] = has ? sc[i] : 0u;
      }
      there = __ballot_sync(0xffffffffu, has || !in);  // (slots behind the limit are masked by their number)
    };
    uint4 raw[kCopy ? 1 : PASSES][kCopy ? 1 : KC];
    auto ask_rows = [&]() {
      if constexpr (!kCopy) {
        // (numbers of 4 bits without a slot: a scale of 0 makes zeros of whatever they are, so that those of page 0 will do)
        const unsigned char* from0 = head_row + ch0 * 16;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          const long long o = shfl_ll(KIND == kPaInt4 ? max(off, 0ll) : off, p * SL + sub);
          const uint4* from = reinterpret_cast<const uint4*>(from0 + o);
#pragma unroll
          for (int k = 0; k < KC; ++k)
            raw[p][k] = KIND != kPaInt4 && o < 0 ? make_uint4(0u, 0u, 0u, 0u) : from[k * CL];
        }
      }
    };
    // Where chunk i of those behind a lane's first one goes in a row of the tile: the swizzle's bits of the two do not meet (a lane's
    // first chunk is a multiple of OUT, and those of other lanes lie a multiple of CL * OUT, 4 at least, further on).
    constexpr int OUT = PaChunk<KIND>::kOut;
    const int row0 = lw * MINE + sub, oc0 = ch0 * OUT;
    const uint32_t lane_at = (oc0 >> 3) * (TILE * 128) + row0 * 128 + (((oc0 & 7) ^ (row0 & 7)) << 4);
    auto place_of = [&](uint32_t mat, int p, int i) {  // (SL is a multiple of 8)
      return ((mat + lane_at) ^ ((i & 7) << 4)) + (i >> 3) * (TILE * 128) + p * (SL * 128);
    };
    auto copy_rows = [&](uint32_t mat) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const long long o = shfl_ll(off, p * SL + sub);
        const unsigned char* from = head_row + max(o, 0ll) + ch0 * 16;
#pragma unroll
        for (int k = 0; k < KC; ++k) pa_request(place_of(mat, p, k * CL), from + k * CL * 16, o >= 0);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // Elements of this lane's that are not finite, in slots that not all of the unit's tokens see, become 0.  (Slow: seldom called.)
    auto clean = [&](uint32_t mat, int from) {
#pragma unroll 1
      for (int i = 0; i < PASSES * KC * OUT; ++i) {
        const int p = i / (KC * OUT), k = i % (KC * OUT);
        if (row0 + p * SL < from) continue;
        const uint32_t at = place_of(mat, p, k / OUT * (CL * OUT) + k % OUT);
        uint4 x;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
        pa_store(at, make_uint4(pa_finite(kType, x.x), pa_finite(kType, x.y), pa_finite(kType, x.z), pa_finite(kType, x.w)));
      }
    };
    auto seen_by_all = [&](const PaPlace& w) { return w.base + w.rho / c.G + 1 - w.tile * TILE; };
    const bool cleans = of_v && s_spoilt;
    auto write_rows = [&](uint32_t mat) {
      if constexpr (!kCopy) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            const uint4& x = raw[p][k];
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            I4Scale f;
            if constexpr (KIND == kPaInt4) {
              const uint32_t w = __shfl_sync(0xffffffffu, scales[k * CL / 4], p * SL + sub);
              f = i4_factors((w >> (8 * ((D == 64 && of_v ? 2 : 0) + ch0)) & 0xffu) * 0x00800080u);
            }
#pragma unroll
            for (int o = 0; o < OUT; ++o) {
              uint32_t v[4];
              if constexpr (KIND == kPaInt4) {
                i4_values(v, in[o], f);
              } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(in[(2 * o + i / 2) & 3] >> (16 * (i & 1)));
                  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
                  v[i] = (uint32_t)h.x | (uint32_t)h.y << 16;
                }
              }
              pa_store(place_of(mat, p, k * CL * OUT + o), make_uint4(v[0], v[1], v[2], v[3]));
            }
          }
      }
    };
    if (works) {
      page = ask_page();
      locate();
      ask_rows();
      page_next = ask_page();
    }
    int jt = 0;
    while (more_d) {
      const int st = jt % S;
      const uint32_t mat = sKV + st * 2 * Sh::kMat + (of_v ? Sh::kMat : 0);
      // the stage is free again
      const bool ok = jt < S || wait((of_v ? B_VEMPTY : B_KEMPTY) + st, jt / S - 1);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (!of_v && lane == 0) {
        if (MINE == 32) s_there[jt & 7][lw] = there;
        else reinterpret_cast<unsigned short*>(s_there[jt & 7])[lw] = (unsigned short)there;
      }
      if (kCopy) {
        copy_rows(mat);
        if (cleans) {
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          clean(mat, seen_by_all(wd));
        }
        if (jt > 0) {  // the tile before has arrived
          asm volatile("cp.async.wait_group 1;" ::: "memory");
          fence_async_smem();
          arrive(full + (jt - 1) % S);
        }
      } else {
        write_rows(mat);
        if (cleans) clean(mat, seen_by_all(wd));
        fence_async_smem();
        arrive(full + st);
      }
      if (++wd.tile == wd.end) {  // now of the next tile
        more_d = next_part(wd);
        head_row = pages + wd.head * c.hs;
      }
      page = page_next;
      page_next = ask_page();
      locate();
      if (more_d) ask_rows();
      ++jt;
    }
    if (kCopy && works) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      fence_async_smem();
      if (jt > 0) arrive(full + (jt - 1) % S);
    }
  } else if (warp >= kPaIssuer) {
    // ------------------------------------------------------------------ products
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPaIssueRegs));
    // A warp for each tile of query rows: S(q) of the next tile of slots follows O(q) += P(q) V of this one, and the other
    // tile's products run while this one's softmax does.
    if (works && warp < kPaIssuer + QT) {
      constexpr uint32_t kFmt = kType == LTRI_TYPE_BF16 ? 1u : 0u;
      constexpr uint32_t kF = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (8u << 24);  // fp32 sums, both operands' type, M = 128
      constexpr uint32_t idesc_qk = kF | (uint32_t)(64 >> 3) << 17, idesc_pv = kF | 1u << 16 | (uint32_t)(D >> 3) << 17;
      const int q = __shfl_sync(0xffffffffu, warp, 0) - kPaIssuer;
      const uint64_t dQ = make_desc(sQ + q * Sh::kQBytes, 16, 1024), dK = make_desc(sKV, 16, 1024);
      const uint64_t dV = make_desc(sKV + Sh::kMat, TILE * 128, 1024);
      const uint32_t tS = tmem + q * 128, tO = tmem + 256 + q * D;
      const uint32_t bars0 = bar(0), q_bars = bars0 + 8 * q, s_bars = bars0 + 8 * (q * SB);
      // 64 slots of the tile in stage st
      auto issue_qk = [&](int b, int st, int sub) {
        const uint64_t db = dK + (uint32_t)(st * (2 * Sh::kMat >> 4) + sub * (64 * 128 >> 4));
        const uint32_t d = tS + b * 64;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t half = ks >> 2, in = (ks & 3) * 32;
          pa_mma_ss(d, dQ + ((half * 16384 + in) >> 4), db + ((half * (TILE * 128) + in) >> 4), idesc_qk, ks > 0);
        }
        pa_commit(s_bars + 8 * B_SREADY + 8 * b);
      };
      // P: 32 columns of first terms, 32 of second ones
      auto issue_pv = [&](int b, int st, int sub, bool acc) {
        const uint32_t pa = tS + b * 64;
        const uint64_t db = dV + (uint32_t)(st * (2 * Sh::kMat >> 4) + sub * (64 * 128 >> 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pa_mma_ts(tO, pa + 32 + i * 8, db + (i * 16 * 128 >> 4), idesc_pv, acc || i > 0);
          pa_mma_ts(tO, pa + i * 8, db + (i * 16 * 128 >> 4), idesc_pv, true);
        }
      };
      auto wait_at = [&](uint32_t at, uint32_t parity) { return __all_sync(0xffffffffu, pa_wait(at, parity, abortp, c.wait_limit)) != 0; };
      PaPlace w = s_place;
      uint32_t st = 0, turn = 0;           // the stage and its parity
      uint32_t s_turn = 0, unit_turn = 0;  // a bit for each S: the parity of S and P; that of the parts of units
      int b = 0;                           // the S in turn
      bool ok = true, had = false;         // had: a part before this one
      do {
        int left = w.end - w.tile;
        if (q == 1 && w.rows - w.rho <= 128) {
          // none of this tile's rows: its leave to the stages alone
          for (; ok && left > 0; --left) {
            ok = wait_at(bars0 + 8 * B_KFULL + 8 * st, turn);
            if (lane == 0) mbar_arrive(bars0 + 8 * B_KEMPTY + 8 * st);
            ok = ok && wait_at(bars0 + 8 * B_VFULL + 8 * st, turn);
            if (lane == 0) mbar_arrive(bars0 + 8 * B_VEMPTY + 8 * st);
            if (++st == S) st = 0, turn ^= 1;
          }
          continue;
        }
        ok = wait_at(q_bars + 8 * B_QFULL, unit_turn) && wait_at(bars0 + 8 * B_KFULL + 8 * st, turn);
        if (!ok) break;
        fence_after_sync();
        issue_qk(b, st, 0);
        if (SUBS == 1) pa_commit(bars0 + 8 * B_KEMPTY + 8 * st);
        bool first = true;
        int sub = 0;
        left *= SUBS;
#pragma unroll 1
        for (; left > 0; --left) {
          // S of the next 64 slots, while this one's softmax runs
          const bool last = sub + 1 == SUBS;  // of the tile
          const uint32_t nst = !last ? st : st + 1 == S ? 0 : st + 1, nturn = turn ^ (last && nst == 0);
          const int nsub = last ? 0 : sub + 1;
          if (left > 1) {
            if (last) {
              ok = wait_at(bars0 + 8 * B_KFULL + 8 * nst, nturn);
              if (!ok) break;
              fence_after_sync();
            }
            issue_qk(b ^ 1, nst, nsub);
            if (nsub + 1 == SUBS) pa_commit(bars0 + 8 * B_KEMPTY + 8 * nst);
          }
          ok = (sub > 0 || wait_at(bars0 + 8 * B_VFULL + 8 * st, turn)) && wait_at(s_bars + 8 * B_PREADY + 8 * b, s_turn >> b & 1);
          // the first product of a part of a unit overwrites O: the one before it must have been read
          if (first && had) ok = ok && wait_at(q_bars + 8 * B_OFREE, unit_turn ^ 1);
          if (!ok) break;
          fence_after_sync();
          issue_pv(b, st, sub, !first);
          if (last) pa_commit(bars0 + 8 * B_VEMPTY + 8 * st);
          pa_commit(q_bars + 8 * B_PVDONE);
          if (left == 1) pa_commit(q_bars + 8 * B_ODONE);
          s_turn ^= 1u << b;
          first = false;
          st = nst;
          turn = nturn;
          sub = nsub;
          b ^= 1;
        }
        unit_turn ^= 1;
        had = true;
      } while (ok && next_part(w));
      // nothing of this CTA's is under way when it gives its TMEM back
      pa_commit(bar(B_DRAIN));
      const long long t0 = clock64();
      while (!mbar_try_suspend(bar(B_DRAIN), 0, 2000u) && clock64() - t0 < kPaDrainLimit) {
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax, queries and outputs
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPaSoftmaxRegs));
    // A warp has 16 rows of S, four lanes each, so that a softmax needs no other warp.  Queries and outputs go by rows of a lane, two
    // threads each, with half of the elements.  Whatever goes wrong, all 256 threads of a tile of queries meet at the same barriers.
    if (works && warp < 8 * QT) {
      const int q = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
      const int row16 = (warp & 3) * 32 + half * 16 + (lane >> 2);
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, lanes16 = lanes + ((uint32_t)(half * 16) << 16);
      const uint32_t tO = tmem + lanes + 256 + q * D + half * (D / 2);
      PaPlace w = s_place;
      int n = 0, unit = 0, jt = 0;  // tiles and parts of this tile of queries; the CTA's tiles
      bool ok = true, more = true;
      // the row's queries of part w into shared memory (free: all products with the last ones have been seen to end)
      auto load_queries = [&]() {
        const int rho = w.rho + q * 128 + r;
        const bool in = rho < w.rows;
        const int tok = w.start + rho / c.G, h = w.head * c.G + rho % c.G;
        const unsigned char* from = a.q + (in ? tok * a.q_stride + (size_t)h * (D * 2) : 0);
        const uint32_t to = sQ + q * Sh::kQBytes + r * 128;
        // (eight chunks of 16 bytes at a time on their way)
        constexpr int GROUP = D / 16 < 8 ? D / 16 : 8, GROUPS = D / 16 / GROUP;
        uint4 x[GROUP];
        auto load = [&](int g) {
#pragma unroll
          for (int k = 0; k < GROUP; ++k)
            x[k] = in ? *reinterpret_cast<const uint4*>(from + (half * (D / 16) + g * GROUP + k) * 16) : make_uint4(0u, 0u, 0u, 0u);
        };
        load(0);
        float u0 = 1.f, u1 = 1.f;
        constexpr bool kHalves = KIND >= kPaE4m3;
        if (kHalves && c.type == LTRI_TYPE_BF16) {
          // bf16 queries as halves: a power of two brings the row's largest element to [2^14, 2^15)
          uint32_t most = 0;
#pragma unroll 1
          for (int g = 0; g < GROUPS; ++g) {
            if (g) load(g);
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
              most = __vmaxu2(most, __vmaxu2(__vmaxu2(x[k].x & 0x7fff7fffu, x[k].y & 0x7fff7fffu),
                                             __vmaxu2(x[k].z & 0x7fff7fffu, x[k].w & 0x7fff7fffu)));
          }
          if (GROUPS > 1) load(0);
          s_most[q][half][r] = max(most & 0xffffu, most >> 16);
          pa_any(1 + q, false);
          const int ex = (int)(max(s_most[q][0][r], s_most[q][1][r]) >> 7);  // biased exponent
          const int up = ex == 0 || ex == 255 ? 0 : 127 + 14 - ex;
          // (2^up may lie outside fp32's range: two factors)
          u0 = __int_as_float((127 + up / 2) << 23), u1 = __int_as_float((127 + up - up / 2) << 23);
          if (half == 0) s_back[q][r] = __int_as_float((127 - up / 2) << 23) * __int_as_float((127 - up + up / 2) << 23);
        }
#pragma unroll 1
        for (int g = 0; g < GROUPS; ++g) {
          if (g) load(g);
#pragma unroll
          for (int k = 0; k < GROUP; ++k) {
            const int i = half * (D / 16) + g * GROUP + k;
            if (kHalves && c.type == LTRI_TYPE_BF16) {
              auto as_half = [&](uint32_t y) {
                const float2 f = paged_unpack(LTRI_TYPE_BF16, y);
                return paged_pack(LTRI_TYPE_FP16, f.x * u0 * u1, f.y * u0 * u1);
              };
              x[k] = make_uint4(as_half(x[k].x), as_half(x[k].y), as_half(x[k].z), as_half(x[k].w));
            }
            pa_store(to + (i >> 3) * 16384 + (((i & 7) ^ (r & 7)) << 4), pa_order<KIND>(x[k]));
          }
        }
        fence_async_smem();
        arrive(B_QFULL + q);
      };
      // (a tile of queries without a row in the unit takes no part in it)
      auto skip = [&]() {
        while (more && w.rows - w.rho <= q * 128) {
          jt += w.end - w.tile;
          more = next_part(w);
        }
      };
      skip();
      if (more) load_queries();
      float old_top = kPaNone, old_sum = 0.f;  // of the part's stretches so far
      while (more) {
        const int begin = w.tile, end = w.end;
        if (lane == 0) s_where[warp] = w;
        pa_any(1 + q, false);  // (s_back is there, and s_sum and s_ref of the part before have been read)
        // this lane's two rows: slots that they see, logits' factors, references and sums
        int own[2];
        unsigned long long sc2[2], ref2[2], sum2[2];
        float sc[2], ref[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = w.rho + q * 128 + row16 + 8 * i;
          own[i] = at < w.rows ? w.base + at / c.G + 1 : 0;
          sc[i] = c.scale;
          if (KIND >= kPaE4m3) {
            const float back = c.type == LTRI_TYPE_BF16 ? s_back[q][row16 + 8 * i] : 1.f;
            const float f = (float)((double)c.scale * (KIND == kPaE4m3 ? c.ks[w.head] : kI4Back) * back);
            sc[i] = f < 0x1p-126f ? 0x1p-126f : f;  // (as for single tokens)
          }
          ref[i] = kPaNone;
          sc2[i] = pa_pair(sc[i], sc[i]);
          ref2[i] = pa_pair(-ref[i], -ref[i]);
          sum2[i] = 0ull;
        }
#pragma unroll 1
        for (int s = begin * SUBS; s < end * SUBS; ++s, ++n) {  // 64 slots
          const int b = n & 1;
          const uint32_t tS = tmem + lanes16 + q * 128 + b * 64;
          ok = ok && __all_sync(0xffffffffu, wait(B_SREADY + q * SB + b, n >> 1));
          if (!ok) continue;
          fence_after_sync();
          uint32_t v[32];
          pa_ld64(tS, v);
          // columns that a row sees, and those that have a page, a bit each
          const uint32_t* there = s_there[(jt + s / SUBS - begin) & 7] + s % SUBS * 2;
          const uint32_t t0 = there[0], t1 = there[1];
          const int l0 = own[0] - s * 64, l1 = own[1] - s * 64;
          tmem_ld_wait();
          if (__any_sync(0xffffffffu, min(l0, l1) < 64 || (t0 & t1) != 0xffffffffu)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int l = i ? l1 : l0;
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int lk = l - k * 32;
                const uint32_t m = ((lk >= 32 ? 0xffffffffu : lk <= 0 ? 0u : (1u << lk) - 1u) & (k ? t1 : t0)) >> (lane & 3) * 2;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (!(m >> (e / 2 * 8 + (e & 1)) & 1u)) v[16 * k + e / 2 * 4 + 2 * i + (e & 1)] = 0xff800000u;
              }
            }
          }
          float top[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float m2[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              m2[e & 1] = fmaxf(m2[e & 1], fmaxf(__uint_as_float(v[4 * e + 2 * i]), __uint_as_float(v[4 * e + 2 * i + 1])));
            top[i] = fmaxf(m2[0], m2[1]) * sc[i];
          }
          if (__any_sync(0xffffffffu, top[0] > ref[0] + (kOff + kGrow) || top[1] > ref[1] + (kOff + kGrow))) {
            float by[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
              top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
              const float to = top[i] > ref[i] + (kOff + kGrow) ? fmaxf(ref[i], top[i] - kOff) : ref[i];
              by[i] = pa_exp2(ref[i] - to);
              ref[i] = to;
              ref2[i] = pa_pair(-to, -to);
              const float2 x = pa_split(sum2[i]);
              sum2[i] = pa_pair(x.x * by[i], x.y * by[i]);
            }
            if (s > begin * SUBS) {
              // (the products with V of the slots before are seen to end; if they are not, so is the CTA's end)
              ok = __all_sync(0xffffffffu, wait(B_PVDONE + q, n - 1));
              fence_after_sync();
#pragma unroll 1
              for (int i = 0; i < D / 32; ++i) {
                uint32_t o[16];
                pa_ld32(tmem + lanes16 + 256 + q * D + i * 32, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by[e >> 1 & 1]);
                pa_st32(tmem + lanes16 + 256 + q * D + i * 32, o);
              }
              tmem_st_wait();
            }
          }
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {  // columns e / 2 * 8 + ..., of row e & 1
            const int i = e & 1;
            const float2 x = pa_split(pa_fma2(pa_pair(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), sc2[i], ref2[i]));
            const unsigned long long p = pa_pair(pa_exp2(x.x), pa_exp2(x.y));
            sum2[i] = pa_add2(sum2[i], p);
            pa_terms(kType, p, hi[e], lo[e]);
          }
          pa_st_pairs(tS, hi);
          pa_st_pairs(tS + 32, lo);
          tmem_st_wait();
          fence_before_sync();
          arrive(B_PREADY + q * SB + b);
        }
        jt += end - begin;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 x = pa_split(sum2[i]);
          float all = x.x + x.y;
          all += __shfl_xor_sync(0xffffffffu, all, 1);
          all += __shfl_xor_sync(0xffffffffu, all, 2);
          if ((lane & 3) == 0) {
            s_sum[q][row16 + 8 * i] = all;
            s_ref[q][row16 + 8 * i] = ref[i];
          }
        }
        __syncwarp();
        w = s_where[warp];
        const int rho = w.rho + q * 128 + r, head = w.head, first = w.first;
        const bool row_ok = rho < w.rows, final = end == w.stop, whole = final && first == 0 && end == w.tiles;
        const size_t to_row = (size_t)(w.start + rho / c.G) * c.Hq + head * c.G + rho % c.G;
        // the next part's queries while this one's last products run
        more = next_part(w);
        skip();
        if (!final) arrive(B_QFULL + q);
        else if (more) load_queries();
        ok = ok && wait(B_ODONE + q, unit);
        if (pa_any(1 + q, !ok)) break;
        float sum = s_sum[q][r], top = s_ref[q][r], now = 1.f, old = 0.f;
        if (begin > first) {
          const float to = fmaxf(top, old_top);
          now = pa_exp2(top - to), old = pa_exp2(old_top - to);
          sum = sum * now + old_sum * old;
          top = to;
        }
        old_top = top, old_sum = sum;
        fence_after_sync();
        const float by = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum, vs = whole ? pa_v_scale<KIND>(c, head) : 1.f;
        float* part = wk.part + (size_t)(2 * blockIdx.x + (first == 0 ? 1 : 0)) * pa_part_floats<KIND, D>();
#pragma unroll 1
        for (int k = 0; k < D / 64; ++k) {
          const int i = half * (D / 64) + k;
          uint32_t v[32];
          __syncwarp();  // (lanes without a row have gone ahead)
          tmem_ld32(tO + k * 32, v);
          tmem_ld_wait();
          float z[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) z[e] = __uint_as_float(v[e]);
          if (!row_ok) continue;
          if (begin > first) {  // (a thread's own stores)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 y = *reinterpret_cast<const float4*>(part + ((size_t)(q * (D / 4) + i * 8 + e) * 128 + r) * 4);
              z[4 * e] = z[4 * e] * now + y.x * old;
              z[4 * e + 1] = z[4 * e + 1] * now + y.y * old;
              z[4 * e + 2] = z[4 * e + 2] * now + y.z * old;
              z[4 * e + 3] = z[4 * e + 3] * now + y.w * old;
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) z[e] = z[e] * by * vs;
          if (whole) {
            pa_put32<KIND>(c.type, a.out + to_row * (D * 2) + i * 64, z);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              *reinterpret_cast<float4*>(part + ((size_t)(q * (D / 4) + i * 8 + e) * 128 + r) * 4) =
                  make_float4(z[4 * e], z[4 * e + 1], z[4 * e + 2], z[4 * e + 3]);
          }
        }
        fence_before_sync();
        arrive(B_OFREE + q);
        if (s_spoilt && row_ok) {  // (by the slots that this row sees; s_where still has the stretch's place)
          const PaPlace& u = s_where[warp];
          const int from = max(u.base + u.rho / c.G + 1, u.tile * TILE), end = min(u.base + (u.rho + q * 128 + r) / c.G + 1, u.end * TILE);
#pragma unroll 1
          for (int i = half * (D / 64); i < (half + 1) * (D / 64); ++i) {
            const unsigned char* at = KIND == kPaInt4 ? c.sc + paged_word(c, layer, 0, u.head, 0) * (D / 16) + D / 32 + i
                                                      : c.v + layer * c.ls + u.head * c.hs + i * (Sh::kRow * 32 / D);
            const long long ps = KIND == kPaInt4 ? (long long)c.Hkv * c.P * (D / 16) : c.ps;
            const uint32_t bad = pa_spoilt<KIND>(at, ps, KIND == kPaInt4 ? D / 16 : c.ts, table + u.row * table_stride, c.n_pages, c.P,
                                                 c.p_mul, c.p_shift, from, end);
#pragma unroll 1
            for (int e = 0; e < 32; ++e) {
              if (!(bad >> e & 1u)) continue;
              if (whole) reinterpret_cast<unsigned short*>(a.out)[to_row * D + i * 32 + e] = 0x7fffu;  // (NaN of both types)
              else part[((size_t)(q * (D / 4) + i * 8 + e / 4) * 128 + r) * 4 + e % 4] = __int_as_float(0x7fffffff);
            }
          }
        }
        __syncwarp();  // (s_where)
        if (row_ok && half == 0) {
          if (whole && a.lse)
            a.lse[to_row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
          if (final && !whole) *reinterpret_cast<float2*>(part + (size_t)ROWS * D + (q * 128 + r) * 2) = make_float2(top, sum);
        }
        ++unit;
      }
    }
  }
  __syncthreads();
  if (tid == 0 && s_abort && atomicCAS(&c.status[0], 0, (int)LTRI_ETIMEOUT) == 0) c.status[1] = blockIdx.x;
  if (warp == kPaIssuer) tmem_dealloc(tmem, 512);
}

// Joins the parts of a unit whose first tile is in CTA x's run and whose last is not: 128 query rows of it, 32 elements a thread.
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
  const int extra = pa_extra(e, c.G, Sh::kRows), places = e.tiles + extra, head = (int)((c1 - 1 - e.before) / places);
  const long long begin = e.before + (long long)head * places + extra, end = begin + e.tiles;
  if (begin < c0 || begin >= c1 || end == c1) return;
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

template <typename F>
cudaError_t prepare_kernel(F* fn, int smem) {
  cudaFuncAttributes a;
  cudaError_t e = cudaFuncGetAttributes(&a, fn);
  // the roles' registers come out of the launch's
  if (e == cudaSuccess && a.numRegs < kPaRegs) e = cudaErrorInvalidConfiguration;
  return first_error(e, allow_smem(fn, smem));
}
template <int KIND>
cudaError_t prepare_kind(int D) {
  if (D == 64) return prepare_kernel(k_paged_attend<KIND, 64>, PaShape<KIND, 64>::kSmem);
  if (D == 128) return prepare_kernel(k_paged_attend<KIND, 128>, PaShape<KIND, 128>::kSmem);
  return prepare_kernel(k_paged_attend<KIND, 256>, PaShape<KIND, 256>::kSmem);
}

template <int KIND, int D>
cudaError_t launch_one(const PagedCache& c, const PagedRows& r, int layer, const PagedQueries& a, const PaWork& wk, cudaStream_t s) {
  using Sh = PaShape<KIND, D>;
  cudaError_t e = launch_chained(k_paged_attend_plan, dim3(1 + wk.scans), dim3(kPlThreads), 0, s, c, r, layer, a.starts, a.n_tokens,
                                 wk, Sh::kRows, Sh::kTile);
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

// CTAs that look through the tokens' V rows: a token a warp, as long as there are SMs.
int scans_of(const PagedCache& c, long long n_tokens) {
  const long long warps = kPlThreads / 32, most = c.sms > 1 ? c.sms - 1 : 1;
  return (int)((n_tokens + warps - 1) / warps < most ? (n_tokens + warps - 1) / warps : most);
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
  const int scans = scans_of(c, n_tokens);
  unsigned char* spoilt = take(scans * sizeof(int));
  unsigned char* part = take((size_t)c.sms * 2 * rows_of_unit(c.D) * (c.D + 2) * sizeof(float));
  if (wk) *wk = PaWork{reinterpret_cast<PaPlan*>(plan), reinterpret_cast<PaEntry*>(entry), (int)entries,
                       reinterpret_cast<int*>(rows), reinterpret_cast<int*>(spoilt), scans, reinterpret_cast<float*>(part)};
  return off;
}

}  // namespace

cudaError_t prepare_paged_attend(const PagedCache& c) {
  if (c.cache_type == LTRI_TYPE_INT4) return prepare_kind<kPaInt4>(c.D);
  if (c.cache_type == LTRI_TYPE_E4M3) return prepare_kind<kPaE4m3>(c.D);
  return c.type == LTRI_TYPE_BF16 ? prepare_kind<kPaBf16>(c.D) : prepare_kind<kPaFp16>(c.D);
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
