// Attention of one new token per row over a caller-owned paged cache, split over the cache's length and joined.
//
// x_j = c q.K_j, out = sum_j 2^(x_j - L) V_j with c in log2 units and L = log2 sum_j 2^(x_j): one pass over K and V with a
// running reference m, sums of 2^(x_j - m) and of 2^(x_j - m) V_j, which parts of a row join by rescaling to the larger m.
//
// Bound: HBM (a KV head's rows are read once for up to 16 of its query heads: 2 G flop a byte in 16 bits; more heads are blocks
// of 16 with a unit each, which read the rows again).  So the work is the rows' tiles, and it is dealt evenly: the tiles of all
// (row, KV head, block) units stand in one line, of which every warp takes an equal run, across units if need be, and a CTA (one
// per SM) its warps' runs.  Ragged batches and single long rows fill the GPU alike, and no count of splits has to be chosen.  A
// unit within one warp's run is written by the warp; of a unit that several warps share, the sums are joined when their CTA has
// finished its run, and of one that several CTAs share, the last CTA to finish joins the others' sums, always in the order of
// the line.
//
// A warp has a ring of its own that cp.async fills several tiles ahead, across units.  (One bulk copy a row instead: 341 us for
// 16 rows of 24576 slots, 254 so; a row's copy costs the copy unit some 15 cycles however short it is.)  A row's 16-byte chunks
// are permuted by its number, so that eight rows' equal chunks fall into different banks.  (Rows 16 bytes further apart than
// they are long, which needs no permutation: 279 us, the writes then straddle lines.)
//
// Both products run on mma.sync with the slots (or head_dim) as the 16 rows and the heads of the KV group as the 8 columns:
// S^T = K Q^T, O^T = V^T P^T, so that up to eight heads fill the instruction exactly.  (Memory is the bound and the tensor pipe
// 19% busy: tcgen05, with 64 rows at least and accumulators to fetch, has nothing to gain.)
//
// Measured (nine B200s, copy rate 6454 GB/s): 16 rows of 24576 slots, 32 query and 8 KV heads of 128 in bf16, 239 to 261 us on
// all but one (270), 6.2 to 6.7 TB/s; one row of 131072, 88 to 94 us, 5.7 to 6.1 TB/s.  What a call costs beyond its bytes is 10
// to 15 us: two dependent lookups before the first row (lengths, pages), and after the last one the joins; 300 slots of one row
// take 8.6 to 9.5 us.  32 query heads of one KV head, 16 rows of 24576 slots: 76 to 83 us, 64 of them 138 to 167, at a floor of 31.
//
// 4-bit rows: a quarter of the bytes for the same products, and numbers to be unpacked, so that instructions are the bound (some 410 of
// a warp for 16 slots of 128; half of the issue slots are taken).  K's numbers enter the products as they stand, as the smallest
// halves, and their scales are applied to the sums of 32 elements; V's become values by one multiply-add for two.  The same 16
// rows 132 to 134 us (66 at the copy rate), the row of 131072 57 to 58.5 (22), 300 slots 9.5 to 9.8.
#include "mma_util.cuh"
#include "paged_deal.cuh"
#include "paged_int4.cuh"

namespace ltri {

enum { kPdBf16 = 0, kPdFp16 = 1, kPdE4m3 = 2, kPdInt4 = 3 };  // what the pages hold

template <int KIND, int D, int NT>
struct PdShape {
  static constexpr int kRow = KIND == kPdInt4 ? D / 2 : KIND == kPdE4m3 ? D : 2 * D;  // bytes of a cached row
  static constexpr int kScales = KIND == kPdInt4 ? D / 16 : 0;  // bytes of a slot's scales, K's and V's
  // 4-bit rows take the instructions of the other kinds for a quarter of 16-bit rows' bytes: twelve warps where their registers
  // allow it.
  static constexpr bool kWide = KIND == kPdInt4 && (NT == 2 || D == 256);
  // Blocks of 16 slots in a tile: 8 KB of rows or more, since what a tile costs besides its rows (cursors, page numbers, the
  // reference) took 8-bit rows in tiles of 16 slots to 1.4 times the instructions.
  static constexpr int kMt = KIND == kPdInt4 ? (D == 256 ? 2 : 4) : kRow >= 256 ? 1 : 256 / kRow;
  static constexpr int kTile = 16 * kMt;                        // slots
  static constexpr int kStage = kTile * (2 * kRow + kScales);   // K rows, V rows, scales
  static constexpr int kTable = KIND == kPdInt4 ? 8 * D : 0;    // factors of V's values of 32 slots, of a warp: 256 bytes for 32 elements
  static constexpr int kWarps = kRow == 512 ? 4 : KIND == kPdInt4 && !kWide ? 12 : 8;  // of a CTA, one CTA an SM
  static constexpr int kRoom = (232448 - (KIND == kPdInt4 ? 1024 : 2048)) / kWarps - kTable;  // of a warp
  static constexpr int kFit = (kRoom + (KIND == kPdInt4 ? 4 * kTile : 0)) / (kStage + 8 * kTile);
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kAhead = kStages - 1;                    // tiles that rows are on their way of
  static constexpr int kPages = 2 * kStages - (KIND == kPdInt4 ? 1 : 0);  // tiles whose page numbers are known or on their way
  static constexpr int kRing = kStages * kStage;                // of a warp
  static constexpr int kSmem = kWarps * (kRing + kPages * kTile * 4 + kTable);
  static_assert(kStages >= (KIND == kPdInt4 ? 2 : 3), "tiles on their way and one in use");
};

// Parts of a unit, up to which the warp that hands in the last of them joins them; more of them take a whole CTA, behind a
// barrier.  (Always the CTA: 64 ragged rows in 8 bits 61.8 us, 59.5 so.  Up to 3 parts: 10 ragged rows of 1700 slots at
// most 10.9 us, 10.1 to 10.5 so.  Up to 12 or 24: two rows of 4000 slots 14.1 us, 12.0 so.)
constexpr int kPdFew = 6;

// Reference of sums that nothing has entered yet: below every logit, and finite.
constexpr float kPdNone = -3.0e38f;

struct PdWork {
  int heads;            // of a block: 8 or 16
  int blocks;           // of a KV head's query heads
  float* part;          // [CTAs][2] partial sums of CTAs
  float* lead;          // [CTAs][warps] partial sums of warps whose run begins inside a unit and outlasts it
  int stride;           // floats of one: 16 references, 16 sums, then the accumulators
  int* count;           // [rows * Hkv * blocks]: CTAs that have written their part
  float* logits;        // [n_pages][Hkv][P][G rounded up to even], with weights
  float* lse2;          // [rows][Hq], with weights
};

__device__ __forceinline__ float pd_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pd_transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_fp16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int KIND>
__device__ __forceinline__ void pd_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (KIND == kPdBf16) mma_bf16(c, a, b0, b1);
  else mma_fp16(c, a, b0, b1);
}
// d = a b + c, where c is not d's registers: zeros and what a sum begins with need no moves
__device__ __forceinline__ void pd_mma_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1,
                                            float c2, float c3) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void pd_add2(float& a, float& b, float c, float d) {
  asm("{\n.reg .b64 x, y;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nadd.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}\n"
      : "+f"(a), "+f"(b)
      : "f"(c), "f"(d));
}
// Two e4m3 values, the lower or the upper ones of x, as two halves.
__device__ __forceinline__ uint32_t pd_halves_lo(uint32_t x) {
  uint32_t y;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pd_halves_hi(uint32_t x) {
  uint32_t y;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}\n" : "=r"(y) : "r"(x));
  return y;
}

// What a row's number does to the number of a chunk in it, for rows of CHUNKS chunks.
template <int CHUNKS>
__device__ __forceinline__ constexpr int pd_swizzle(int row) {
  return CHUNKS >= 8 ? row & 7 : CHUNKS == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
}

// BYTES bytes on their way, or zeros.
template <int BYTES>
__device__ __forceinline__ void pd_request(uint32_t to, const void* from, bool there) {
  const int n = there ? BYTES : 0;
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to), "l"(from), "r"(n));
  else if (BYTES == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;\n" ::"r"(to), "l"(from), "r"(n));
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(to), "l"(from), "r"(n));
}

// A unit that a warp's run, or a CTA's, leaves unfinished.
struct PdOpen {
  int begin;                    // in the line
  int row, head, block, tiles;  // tiles 0: none
};

template <int KIND, int D, int NT>
__global__ void __launch_bounds__(PdShape<KIND, D, NT>::kWarps * 32, 1)
    k_paged_decode(PagedCache c, PagedRows r, int layer, PagedStep a, PdWork wk) {
  using Sh = PdShape<KIND, D, NT>;
  constexpr int W = Sh::kWarps, TILE = Sh::kTile, MT = Sh::kMt, S = Sh::kStages, DT = D / 16, H = 8 * NT;
  constexpr int kSlices = NT * DT / W > 0 ? NT * DT / W : 1;  // 16-row slices of the sums that a warp joins
  // Probabilities carry a factor 2^kOff that cancels in out and lse.  A half has 2^-24 as its smallest step: with the largest
  // probability at 2^10 a slot's contribution is still seen 2^-35 below it, so that 2^20 of them cannot lose 2^-14 of a sum.
  // The reference moves only when a logit exceeds it by kGrow, which bounds the probabilities by 2^(kOff + kGrow).
  constexpr float kOff = KIND == kPdBf16 ? 0.f : 10.f, kGrow = 4.f;
  // Probabilities meet V as that many terms of the products' type: fp32's 24 bits over bf16 rows, 22 over the others (with two
  // terms over bf16 rows, 16 bits, values that cancel show it).
  constexpr int kTerms = KIND == kPdBf16 ? 3 : 2;
  extern __shared__ __align__(1024) unsigned char dsm[];
  __shared__ PdOpen s_open[W];
  __shared__ PdOpen s_part[2];
  __shared__ int s_last[2];
  chain_wait();
  // The weights kernel waits for this one's end, but may start: beside this one's CTAs where they leave it registers (head_dim
  // 64 and up to eight heads in 16 bits), else on SMs whose CTA is through.
  if (c.w) chain_release();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  unsigned char* ring = dsm + warp * Sh::kRing;
  int* s_pages = reinterpret_cast<int*>(dsm + W * Sh::kRing) + warp * Sh::kPages * TILE;
  const uint32_t ring_s = smem_u32(ring), pages_s = smem_u32(s_pages);
  // Blocks of 16 slots within a page are requested from one address, stepping; others a row at a time, from addresses that the
  // lanes exchange.  (All by single rows: 16 rows of 24576 slots of 128 in bf16 263 to 274 us, one row of 131072 95 to 97, by
  // steps 242 to 248 and 89 to 91; 64 ragged rows in 8 bits 4 us more.)
  const bool one_page = c.P % 16 == 0;

  PdCursor cu;
  int total;
  bool lone;  // the CTA has one unit, and all of it
  // 4-bit rows, where an SM's instructions are the bound: its warps' runs may differ by a tile.  (Equal ones: 16 rows of 24576 slots
  // of 128 141 us, 134 so; one row of 131072 62.6 and 58.5; 64 ragged rows of 64 41.6 and 39.5; 300 slots 0.2 us less.)
  constexpr bool kEven = KIND == kPdInt4;
  const int per = pd_deal<TILE, kEven>(cu, total, lone, gridDim.x * W, blockIdx.x * W + warp, W, c, r, wk.blocks);
  const int run = kEven ? per : W * per;
  const int c0 = blockIdx.x * run, c1 = min(c0 + run, total);  // the CTA's run
  const int t0 = c0 + (kEven ? pd_share(per, warp, W) : warp * per);
  const int most = kEven ? c0 + pd_share(per, warp + 1, W) - t0 : per;
  const int mine = t0 >= total ? 0 : max(0, min(most, lone ? cu.tiles - cu.tile : total - t0));
  if (lane == 0) {
    s_open[warp].tiles = 0;
    if (warp == 0) s_part[0].tiles = s_part[1].tiles = 0;
  }

  // Page numbers of a tile's slots on their way into entry `st` (-1 behind the row's end).
  auto request_pages = [&](const PdCursor& u, int st) {
#pragma unroll
    for (int j = lane; j < TILE; j += 32) {
      const int slot = u.tile * TILE + j;
      if (slot < u.n) cp_async4(pages_s + (st * TILE + j) * 4, r.table + u.row * r.table_stride + paged_nth(c, slot));
      else s_pages[st * TILE + j] = -1;
    }
  };
  // Rows of a tile on their way: this lane takes chunk `in` of rows lane_row, lane_row + kStep, ...
  constexpr int RC = Sh::kRow / 16, kStep = 32 / RC;
  const int in = lane % RC, lane_row = lane / RC;
  const size_t lane_at = lane_row * c.ts + in * 16, step = kStep * c.ts;
  const uint32_t lane_s = ring_s + lane_row * Sh::kRow + ((in ^ pd_swizzle<RC>(lane_row)) << 4);
  const long long vk = c.v - c.k;
  auto issue = [&](const PdCursor& u, const int* s_page, int st) {
    if constexpr (KIND == kPdInt4) {
      // A lane finds out about the slots `lane`, lane + 32 ..., and asks for their scales; the lanes that ask for their rows ask it.
      // Slots that are not there have scales of zero, which make zeros of whatever their numbers are: those of page 0 will do, as
      // will for the new token's slot, which is written over, what its page holds.
      long long off[(TILE + 31) / 32];
#pragma unroll
      for (int j = 0; j < (TILE + 31) / 32; ++j) {
        if (j * 32 + lane >= TILE) break;
        const int slot = u.tile * TILE + j * 32 + lane, page = s_page[j * 32 + lane];
        const bool has = (unsigned)page < (unsigned)c.n_pages;
        if (!has && slot < u.n) paged_status(c, u.row);
        const unsigned place = has ? slot - paged_nth(c, slot) * c.P : 0u, at_page = has ? page : 0;
        off[j] = at_page * c.ps + place * c.ts;
        const size_t word = (size_t)at_page * (unsigned)(c.Hkv * c.P) + place + paged_word(c, layer, 0, u.head, 0);
        pd_request<Sh::kScales>(ring_s + st * Sh::kStage + 2 * TILE * Sh::kRow + (j * 32 + lane) * Sh::kScales,
                                c.sc + word * Sh::kScales, has);
      }
      const unsigned char* head = c.k + paged_row(c, layer, 0, u.head, 0) + in * 16;
      const uint32_t sk = lane_s + st * Sh::kStage;
#pragma unroll
      for (int i = 0; i < TILE / kStep; ++i) {
        const unsigned char* from = head + shfl_ll(off[i * kStep / 32], (i * kStep + lane_row) & 31);
        const uint32_t to = (sk ^ (pd_swizzle<RC>(i * kStep % 16) << 4)) + i * (kStep * Sh::kRow);
        cp_async16(to, from, 16);
        cp_async16(to + TILE * Sh::kRow, from + vk, 16);
      }
      return;
    }
    // the new token's row comes from the caller (in 8 bits: later, when the tile is used), rows without a slot are zeros:
    // their probability of zero meets their values
    const int fresh = a.k && u.n - 1 - u.tile * TILE < TILE ? u.n - 1 - u.tile * TILE : -1;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int base = u.tile * TILE + m * 16, slot = base + (lane & 15);
      const int page = s_page[m * 16 + (lane & 15)];
      const bool in_page = (unsigned)page < (unsigned)c.n_pages;
      const uint32_t sk = lane_s + st * Sh::kStage + m * 16 * Sh::kRow;
      // (kStep is a power of two above lane_row: their bits, and their swizzles, combine by xor)
      auto to = [&](int i) { return (sk ^ (pd_swizzle<RC>(i * kStep) << 4)) + i * (kStep * Sh::kRow); };
      if (one_page && base + 16 <= u.n && (unsigned)(fresh - m * 16) >= 16u && __all_sync(0xffffffffu, in_page)) {
        const unsigned char* from = c.k + paged_row(c, layer, page, u.head, base - paged_nth(c, base) * c.P) + lane_at;
#pragma unroll
        for (int i = 0; i < RC / 2; ++i) {
          cp_async16(to(i), from, 16);
          cp_async16(to(i) + TILE * Sh::kRow, from + vk, 16);
          from += step;
        }
      } else {
        if (!in_page && slot < u.n) paged_status(c, u.row);
        const long long off = in_page ? (long long)paged_row(c, layer, page, u.head, slot - paged_nth(c, slot) * c.P) : -1;
#pragma unroll
        for (int i = 0; i < RC / 2; ++i) {
          const long long o = shfl_ll(off, i * kStep + lane_row);
          if (m * 16 + i * kStep + lane_row == fresh) continue;
          const unsigned char* from = c.k + (o < 0 ? 0 : o + in * 16);
          cp_async16(to(i), from, o < 0 ? 0 : 16);
          cp_async16(to(i) + TILE * Sh::kRow, from + vk, o < 0 ? 0 : 16);
        }
      }
    }
    if (KIND != kPdE4m3 && fresh >= 0 && lane < RC) {
      const int bytes = (unsigned)s_page[fresh] < (unsigned)c.n_pages ? 16 : 0;
      const size_t at = u.row * a.kv_stride + (size_t)u.head * (2 * D) + lane * 16;
      const uint32_t to = ring_s + st * Sh::kStage + fresh * Sh::kRow + ((lane ^ pd_swizzle<RC>(fresh)) << 4);
      cp_async16(to, a.k + at, bytes);
      cp_async16(to + TILE * Sh::kRow, a.v + at, bytes);
    }
  };
  // The queries of a unit as the products' columns (head g of each block), and the scales of its KV head.  Behind the requests
  // of rows that fill the memory's queues a load takes 3000 cycles, so where there are registers the next unit's are asked for
  // when the first of its rows are.
  constexpr bool kEarly = NT * D <= 128 && KIND != kPdInt4;
  struct Queries {
    uint32_t b[NT][DT][2];
    float ks, vs;
  };
  Queries q, q_next;
  int next_at = -(1 << 30);  // the tile of the run that q_next's unit begins with
  auto load_queries = [&](Queries& x, const PdCursor& u) {
    x.ks = c.ks ? c.ks[u.head] : 1.f;
    x.vs = KIND == kPdInt4 ? kI4Back : c.vs ? c.vs[u.head] : 1.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int in_group = u.block * H + nt * 8 + g;
      const unsigned char* qr = a.q + u.row * a.q_stride + ((size_t)u.head * c.G + in_group) * D * 2;
      if constexpr (KIND == kPdInt4) {
        // (a lane's eight neighbours of 32 elements, as the numbers' bits lie in a word: 0 and 4, 1 and 5; 2 and 6, 3 and 7)
#pragma unroll
        for (int i = 0; i < DT; i += 2) {
          const uint4 e = in_group < c.G ? *reinterpret_cast<const uint4*>(qr + (i * 16 + q4 * 8) * 2) : make_uint4(0u, 0u, 0u, 0u);
          x.b[nt][i][0] = __byte_perm(e.x, e.z, 0x5410);
          x.b[nt][i][1] = __byte_perm(e.x, e.z, 0x7632);
          x.b[nt][i + 1][0] = __byte_perm(e.y, e.w, 0x5410);
          x.b[nt][i + 1][1] = __byte_perm(e.y, e.w, 0x7632);
        }
      } else {
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          // (8-bit rows: a 16-byte chunk is one step of 16, of which a lane holds four neighbours)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int el = KIND == kPdE4m3 ? i * 16 + q4 * 4 + 2 * j : i * 16 + q4 * 2 + 8 * j;
            x.b[nt][i][j] = in_group < c.G ? *reinterpret_cast<const uint32_t*>(qr + el * 2) : 0u;
          }
        }
      }
    }
  };
  float sc[NT][2];  // logits' factors of this lane's heads
  // 4-bit rows: what 8 more in every number adds to the sums of a block's products, for this lane's heads, with its sign turned
  float bias[NT][KIND == kPdInt4 ? D / kI4Block : 1][2];
  auto scale_queries = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float back = 1.f;
      if constexpr (KIND == kPdInt4) {
        // As over 8-bit rows, a power of two brings the row's largest element to [2^14, 2^15), and halves do the rest.  The
        // numbers enter as the smallest halves, n * 2^-24, and every other pair of them 2^4 larger, which is taken from its
        // queries: what falls below the halves' range is 2^-35 of the largest.
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 f = paged_unpack(c.type, q.b[nt][i][j]);
            most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int ex = (int)(__float_as_uint(most) >> 23);  // biased exponent
        const int up = ex == 0 || ex == 255 ? 0 : 127 + 14 - ex;
        // (2^up may lie outside fp32's range: two factors)
        const float u0 = __int_as_float((127 + up / 2) << 23), u1 = __int_as_float((127 + up - up / 2) << 23);
#pragma unroll
        for (int b = 0; b < D / kI4Block; ++b) {
          float all = 0.f;
#pragma unroll
          for (int i = 2 * b; i < 2 * b + 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float2 f = paged_unpack(c.type, q.b[nt][i][j]);
              const float by = j ? u1 * 0x1p-4f : u1;
              const uint32_t h = paged_pack(LTRI_TYPE_FP16, f.x * u0 * by, f.y * u0 * by);
              q.b[nt][i][j] = h;
              const float2 z = paged_unpack(LTRI_TYPE_FP16, h);
              all += (z.x + z.y) * (j ? 16.f : 1.f);
            }
          all += __shfl_xor_sync(0xffffffffu, all, 1);
          all += __shfl_xor_sync(0xffffffffu, all, 2);
#pragma unroll
          for (int e = 0; e < 2; ++e) bias[nt][b][e] = -0x1p-21f * __shfl_sync(0xffffffffu, all, (2 * q4 + e) * 4);
        }
        back = 0x1p24f * __int_as_float((127 - up / 2) << 23) * __int_as_float((127 - up + up / 2) << 23);
      }
      if (KIND == kPdE4m3 && c.type == LTRI_TYPE_BF16) {
        // bf16 queries as halves: a power of two brings the row's largest element to [2^14, 2^15); what then falls below
        // the halves' range is 2^-39 of it
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) most = max(most, max(q.b[nt][i][j] & 0x7fffu, (q.b[nt][i][j] >> 16) & 0x7fffu));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int ex = (int)(most >> 7);  // biased exponent
        const int up = ex == 0 || ex == 255 ? 0 : 127 + 14 - ex;
        // (2^up may lie outside fp32's range: two factors)
        const float u0 = __int_as_float((127 + up / 2) << 23), u1 = __int_as_float((127 + up - up / 2) << 23);
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 f = paged_unpack(LTRI_TYPE_BF16, q.b[nt][i][j]);
            q.b[nt][i][j] = paged_pack(LTRI_TYPE_FP16, f.x * u0 * u1, f.y * u0 * u1);
          }
        back = __int_as_float((127 - up / 2) << 23) * __int_as_float((127 - up + up / 2) << 23);
      }
      // (the queries lie with head g, the logits with heads 2 q4 and 2 q4 + 1)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float b = __shfl_sync(0xffffffffu, back, (2 * q4 + e) * 4);
        sc[nt][e] = c.scale;
        if (KIND != kPdE4m3 && KIND != kPdInt4) continue;
        // The three factors' product may lie in fp32's range where that of two does not.  Never zero: the logits of slots that
        // are not there are -infinity times this, and at the smallest normal number products q.K, here below 2^36, are nothing.
        const float f = (float)((double)c.scale * q.ks * b);
        sc[nt][e] = f < 0x1p-126f ? 0x1p-126f : f;
      }
    }
  };
  // A slice of 16 elements of the eight heads of block nt, normalised, to the output.
  auto put_slice = [&](const PdCursor& u, int nt, int i, const float (&z)[4]) {
    const uint32_t y0 = pd_transpose(paged_pack(c.type, z[0], z[1])), y1 = pd_transpose(paged_pack(c.type, z[2], z[3]));
    const int in_group = u.block * H + nt * 8 + g;
    if (in_group >= c.G) return;
    if constexpr (KIND == kPdInt4) {  // element i % 4 of the groups of four 2 q4 and 2 q4 + 1 of 32, and of the next 32
      unsigned char* to = a.out + (((size_t)u.row * c.Hq + (size_t)u.head * c.G + in_group) * D + i / 4 * 64 + q4 * 8 + i % 4) * 2;
      *reinterpret_cast<unsigned short*>(to) = (unsigned short)y0;
      *reinterpret_cast<unsigned short*>(to + 8) = (unsigned short)(y0 >> 16);
      *reinterpret_cast<unsigned short*>(to + 64) = (unsigned short)y1;
      *reinterpret_cast<unsigned short*>(to + 72) = (unsigned short)(y1 >> 16);
      return;
    }
    unsigned char* to = a.out + (((size_t)u.row * c.Hq + (size_t)u.head * c.G + in_group) * D + i * 16) * 2;
    if (KIND == kPdE4m3) {  // elements 4 q4, + 2 and 4 q4 + 1, + 3
      *reinterpret_cast<uint2*>(to + q4 * 8) = make_uint2(__byte_perm(y0, y1, 0x5410), __byte_perm(y0, y1, 0x7632));
    } else {
      *reinterpret_cast<uint32_t*>(to + q4 * 4) = y0;
      *reinterpret_cast<uint32_t*>(to + 16 + q4 * 4) = y1;
    }
  };
  // The log-sum of head 2 q4 + e of block nt.
  auto put_lse = [&](const PdCursor& u, int nt, int e, float top, float sum) {
    const int in_group = u.block * H + nt * 8 + 2 * q4 + e;
    if (g != 0 || in_group >= c.G) return;
    const size_t at = (size_t)u.row * c.Hq + (size_t)u.head * c.G + in_group;
    const float l2 = sum == 0.f ? -INFINITY : top + log2f(sum);
    if (a.lse) a.lse[at] = l2 * 0.69314718055994531f;
    if (c.w) wk.lse2[at] = sum == 0.f ? INFINITY : l2;  // (logits of -infinity alone: 2^(x - L) is to be 0)
  };
  // (one after the other: the quotient of a small scale and a large sum may lie below fp32's range where the output does not)
  auto one_over = [](float sum) { return sum == 0.f ? 0.f : 1.f / sum; };
  auto scaled = [](float x, float by, float vs) { return KIND == kPdE4m3 || KIND == kPdInt4 ? x * by * vs : x * by; };

  float O[NT][DT][4], ref[NT][2], sum[NT][2];
  // A unit's heads, all of whose sums this warp has.
  auto put_unit = [&](const PdCursor& u) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float by[2] = {one_over(sum[nt][0]), one_over(sum[nt][1])};
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const float z[4] = {scaled(O[nt][i][0], by[0], q.vs), scaled(O[nt][i][1], by[1], q.vs), scaled(O[nt][i][2], by[0], q.vs),
                            scaled(O[nt][i][3], by[1], q.vs)};
        put_slice(u, nt, i, z);
      }
      put_lse(u, nt, 0, ref[nt][0], sum[nt][0]);
      put_lse(u, nt, 1, ref[nt][1], sum[nt][1]);
    }
  };
  // This warp's sums to memory.
  auto set_aside = [&](float* to) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (g == 0) {
        *reinterpret_cast<float2*>(to + nt * 8 + 2 * q4) = make_float2(ref[nt][0], ref[nt][1]);
        *reinterpret_cast<float2*>(to + 16 + nt * 8 + 2 * q4) = make_float2(sum[nt][0], sum[nt][1]);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i)
        reinterpret_cast<float4*>(to + 32)[(nt * DT + i) * 32 + lane] =
            make_float4(O[nt][i][0], O[nt][i][1], O[nt][i][2], O[nt][i][3]);
    }
  };
  // Adds a piece of the same unit to this warp's sums.
  auto add = [&](const float* from) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float2 m = *reinterpret_cast<const float2*>(from + nt * 8 + 2 * q4);
      const float2 s = *reinterpret_cast<const float2*>(from + 16 + nt * 8 + 2 * q4);
      const float t0 = fmaxf(ref[nt][0], m.x), t1 = fmaxf(ref[nt][1], m.y);
      const float a0 = pd_exp2(ref[nt][0] - t0), a1 = pd_exp2(ref[nt][1] - t1);
      const float b0 = pd_exp2(m.x - t0), b1 = pd_exp2(m.y - t1);
      ref[nt][0] = t0;
      ref[nt][1] = t1;
      sum[nt][0] = sum[nt][0] * a0 + s.x * b0;
      sum[nt][1] = sum[nt][1] * a1 + s.y * b1;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const float4 z = reinterpret_cast<const float4*>(from + 32)[(nt * DT + i) * 32 + lane];
        O[nt][i][0] = O[nt][i][0] * a0 + z.x * b0;
        O[nt][i][1] = O[nt][i][1] * a1 + z.y * b1;
        O[nt][i][2] = O[nt][i][2] * a0 + z.z * b0;
        O[nt][i][3] = O[nt][i][3] * a1 + z.w * b1;
      }
    }
  };
  // A tile of 4-bit rows, 32 slots after the other: all of their work is little code, which the warps' turns keep in the instruction
  // caches, and few registers, which lets more warps hide its latencies.  (16 slots at a time: 16 rows of 24576 slots of 128
  // 145 us, 141 so.)
  unsigned char* table4 = dsm + W * (Sh::kRing + Sh::kPages * TILE * 4) + warp * Sh::kTable;
  auto int4_tile = [&](int stage_at, int page_at, int slot0) {
    constexpr int B = D / kI4Block;
    const unsigned char* s_sc = ring + stage_at * Sh::kStage + 2 * TILE * Sh::kRow;
    const uint32_t sk = ring_s + stage_at * Sh::kStage, sv = sk + TILE * Sh::kRow;
    const int row = lane & 15;  // K's and V's matrices: 8 slots, 8 more; 32 elements, 32 more
    const uint32_t at = row * Sh::kRow + ((lane >> 4 ^ pd_swizzle<RC>(row)) << 4);
    I4Scale* tv = reinterpret_cast<I4Scale*>(table4);  // [B][16 pairs of slots]
#pragma unroll 1
    for (int m0 = 0; m0 < MT; m0 += 2) {
      if (slot0 + m0 * 16 >= cu.n) break;
      __syncwarp();
#pragma unroll
      for (int i = lane; i < 16 * B; i += 32) {
        const unsigned char* v = s_sc + (m0 * 16 + i % 16 * 2) * Sh::kScales + Sh::kScales / 2 + i / 16;
        tv[i] = i4_factors(v[0] << 7 | v[Sh::kScales] << 23);
      }
      // S^T = sum over the blocks of 32 elements of scale * (numbers Q^T): a product's accumulator begins with what makes up for the
      // numbers' offset
      float x[2][NT][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[m][nt][0] = x[m][nt][1] = x[m][nt][2] = x[m][nt][3] = 0.f;
        const unsigned char* sc_k = s_sc + ((m0 + m) * 16 + g) * Sh::kScales;
#pragma unroll
        for (int b2 = 0; b2 < B; b2 += 2) {
          uint32_t w[4];
          ldsm_x4(w, ((sk + at) ^ (b2 << 4)) + (m0 + m) * 16 * Sh::kRow);
          // (64 elements a row: two scales beside V's, in one word)
          const uint32_t s_lo = *reinterpret_cast<const uint32_t*>(sc_k + b2 / 4 * 4);
          const uint32_t s_hi = *reinterpret_cast<const uint32_t*>(sc_k + 8 * Sh::kScales + b2 / 4 * 4);
          const float2 lo = i4_scales_f32(s_lo, b2 % 4, s_lo, b2 % 4 + 1), hi = i4_scales_f32(s_hi, b2 % 4, s_hi, b2 % 4 + 1);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int b = b2 + j;
            const uint32_t w0 = w[2 * j], w1 = w[2 * j + 1], u0 = w0 >> 8, u1 = w1 >> 8;
            const uint32_t f0[4] = {w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u};
            const uint32_t f1[4] = {u0 & 0x000f000fu, u1 & 0x000f000fu, u0 & 0x00f000f0u, u1 & 0x00f000f0u};
            const float s0 = j ? lo.y : lo.x, s1 = j ? hi.y : hi.x;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float z[4];
              pd_mma_from(z, f0, q.b[nt][2 * b][0], q.b[nt][2 * b][1], bias[nt][b][0], bias[nt][b][1], bias[nt][b][0], bias[nt][b][1]);
              pd_mma<KIND>(z, f1, q.b[nt][2 * b + 1][0], q.b[nt][2 * b + 1][1]);
              x[m][nt][0] = fmaf(s0, z[0], x[m][nt][0]);
              x[m][nt][1] = fmaf(s0, z[1], x[m][nt][1]);
              x[m][nt][2] = fmaf(s1, z[2], x[m][nt][2]);
              x[m][nt][3] = fmaf(s1, z[3], x[m][nt][3]);
            }
          }
        }
      }
      // lane: slots g and g + 8 of a block (x[..][..][0..1], x[..][..][2..3]), heads 2 q4 and 2 q4 + 1
      const int* s_page = s_pages + page_at * TILE + m0 * 16;
      if (!__all_sync(0xffffffffu, (unsigned)s_page[lane] < (unsigned)c.n_pages)) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bool there = (unsigned)s_page[m * 16 + g + 8 * e] < (unsigned)c.n_pages;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if (!there) x[m][nt][2 * e] = x[m][nt][2 * e + 1] = -INFINITY;
          }
      }
      if (c.w) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int page = s_page[m * 16 + g + 8 * e];
            if ((unsigned)page >= (unsigned)c.n_pages) continue;
            const int slot = slot0 + (m0 + m) * 16 + g + 8 * e, place = slot - paged_nth(c, slot) * c.P;
            const size_t word = ((size_t)page * c.Hkv + cu.head) * c.P + place;
            float* to = wk.logits + word * paged_even(c.G);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const int in_group = cu.block * H + nt * 8 + 2 * q4;
              const float2 y = make_float2(x[m][nt][2 * e] * sc[nt][0], x[m][nt][2 * e + 1] * sc[nt][1]);
              if (in_group < c.G) *reinterpret_cast<float2*>(to + in_group) = y;
            }
          }
      }
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[nt][e] = fmaxf(fmaxf(x[0][nt][e], x[0][nt][e + 2]), fmaxf(x[1][nt][e], x[1][nt][e + 2])) * sc[nt][e];
          grow |= top[nt][e] > ref[nt][e] + (kOff + kGrow);
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top[nt][e] = fmaxf(top[nt][e], __shfl_xor_sync(0xffffffffu, top[nt][e], d));
            const float to = fmaxf(ref[nt][e], top[nt][e] - kOff), by = pd_exp2(ref[nt][e] - to);
            ref[nt][e] = to;
            sum[nt][e] *= by;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
              O[nt][i][e] *= by;
              O[nt][i][e + 2] *= by;
            }
          }
      }
      uint32_t term[2][2][NT][2];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = pd_exp2(fmaf(x[m][nt][e], sc[nt][e & 1], -ref[nt][e & 1]));
            sum[nt][e & 1] += p[e];
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t h = paged_pack(LTRI_TYPE_FP16, p[2 * e], p[2 * e + 1]);
            const float2 back = paged_unpack(LTRI_TYPE_FP16, h);
            term[0][m][nt][e] = pd_transpose(h);
            term[1][m][nt][e] = pd_transpose(paged_pack(LTRI_TYPE_FP16, p[2 * e] - back.x, p[2 * e + 1] - back.y));
          }
        }
      __syncwarp();
      // O^T += V^T P^T.  A 16-byte chunk's 8 groups of four neighbours are the 8 rows of a transposed matrix: row g has elements 4g
      // to 4g + 3 of slots 2 q4 and 2 q4 + 1 (b[0], b[2]: of 32 elements and the next 32) or of slots 8 further (b[1], b[3]).
      // The products of the 32 slots are added up by themselves (see below).
#pragma unroll
      for (int i = 0; i < DT; i += 4) {
        float z[4][NT][4];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          uint32_t b[4], v4[4][4];
          ldsm_x4_t(b, ((sv + at) ^ (i << 3)) + (m0 + m) * 16 * Sh::kRow);
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 2; ++j) i4_values(v4[2 * j + e], b[2 * j + e], tv[(i / 2 + j) * 16 + m * 8 + e * 4 + q4]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t f[4] = {v4[0][j], v4[2][j], v4[1][j], v4[3][j]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              if (m == 0) pd_mma_from(z[j][nt], f, term[1][m][nt][0], term[1][m][nt][1], 0.f, 0.f, 0.f, 0.f);
              else pd_mma<KIND>(z[j][nt], f, term[1][m][nt][0], term[1][m][nt][1]);
              pd_mma<KIND>(z[j][nt], f, term[0][m][nt][0], term[0][m][nt][1]);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            pd_add2(O[nt][i + j][0], O[nt][i + j][1], z[j][nt][0], z[j][nt][1]);
            pd_add2(O[nt][i + j][2], O[nt][i + j][3], z[j][nt][2], z[j][nt][3]);
          }
      }
    }
  };
  // This CTA's part of a unit that other CTAs share is complete in this warp's sums: into the workspace with it.  Of a unit of
  // few parts the last to hand in its own adds up all of them (in their order, so that it does not matter who it is) and
  // returns true; units of many are left to the whole CTA.
  const unsigned cta_run = max(1, run);
  auto parts_of = [&](const PdOpen& o) {  // (never behind the grid's, whatever the lengths have become meanwhile)
    return (int)(min((unsigned)(o.begin + o.tiles - 1) / cta_run, gridDim.x - 1) - (unsigned)o.begin / cta_run) + 1;
  };
  auto hand_in = [&](const PdOpen& o, bool begins) {
    const unsigned first = (unsigned)o.begin / cta_run;
    const int parts = parts_of(o);
    set_aside(wk.part + (size_t)(2 * blockIdx.x + (begins ? 1 : 0)) * wk.stride);
    if (parts > kPdFew) {
      if (lane == 0) s_part[begins ? 1 : 0] = o;
      return false;
    }
    int last = 0;
    __syncwarp();
    if (lane == 0) {
      int* count = wk.count + ((size_t)o.row * c.Hkv + o.head) * wk.blocks + o.block;
      last = paged_arrive(count) == parts - 1;
      if (last) *count = 0;
    }
    if (!__shfl_sync(0xffffffffu, last, 0)) return false;
    __syncwarp();  // (what lane 0 has acquired, for the others: the shuffle orders no memory)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      ref[nt][0] = ref[nt][1] = kPdNone;
      sum[nt][0] = sum[nt][1] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) O[nt][i][0] = O[nt][i][1] = O[nt][i][2] = O[nt][i][3] = 0.f;
    }
#pragma unroll 1
    for (int i = 0; i < parts; ++i) add(wk.part + (size_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * wk.stride);
    return true;
  };
  bool whole = false;   // the unit has begun in this run
  // Rounds: in round `at` tile `at` is used, the rows of tile at + kAhead are requested and the page numbers of tile
  // at + 2 kAhead.  A round's requests are one group, complete when the round kAhead later begins; only the first tiles' page
  // numbers are waited for at once, with the first queries on their way.
  PdCursor ci = cu, cp = cu;
  int stage_at = 0, page_at = 0;            // of tile `at`
  int stage_in = 0, page_in = 0, page_rq = 0;  // of the tiles that are requested
  auto next = [](int x, int n) { return x + 1 == n ? 0 : x + 1; };
  auto ahead = [&](int at) {
    if (at >= -Sh::kAhead && at + Sh::kAhead < mine) {
      if (kEarly && ci.tile == 0 && at > -Sh::kAhead && next_at <= at) {
        next_at = at + Sh::kAhead;
        load_queries(q_next, ci);
      }
      issue(ci, s_pages + page_in * TILE, stage_in);
      stage_in = next(stage_in, S);
      page_in = next(page_in, Sh::kPages);
      pd_advance<TILE>(ci, c, r, wk.blocks);
    }
    if (at + 2 * Sh::kAhead < mine) {
      request_pages(cp, page_rq);
      page_rq = next(page_rq, Sh::kPages);
      pd_advance<TILE>(cp, c, r, wk.blocks);
    }
  };
#pragma unroll 1
  for (int at = mine > 0 ? -2 * Sh::kAhead : 0; at < mine; ++at) {
    if (at == -Sh::kAhead) {
      cp_async_wait<0>();
      __syncwarp();
    }
    if (at >= 0) {
      if (at == 0 || cu.tile == 0) {  // a unit begins
        whole = cu.tile == 0;
        if (kEarly && at > 0 && next_at == at) q = q_next;
        scale_queries();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          ref[nt][0] = ref[nt][1] = kPdNone;
          sum[nt][0] = sum[nt][1] = 0.f;
#pragma unroll
          for (int i = 0; i < DT; ++i) O[nt][i][0] = O[nt][i][1] = O[nt][i][2] = O[nt][i][3] = 0.f;
        }
      }
      const int slot0 = cu.tile * TILE;
      const int fresh = a.k && cu.n - 1 - slot0 < TILE ? cu.n - 1 - slot0 : -1;
      uint4 kx = make_uint4(0u, 0u, 0u, 0u), vx = kx;
      if ((KIND == kPdE4m3 || KIND == kPdInt4) && fresh >= 0 && lane < D / 8) {
        const size_t at_new = cu.row * a.kv_stride + ((size_t)cu.head * D + lane * 8) * 2;
        kx = *reinterpret_cast<const uint4*>(a.k + at_new);
        vx = *reinterpret_cast<const uint4*>(a.v + at_new);
      }
      cp_async_wait<S - 2>();
      __syncwarp();
      // (4-bit rows have few stages: the next tile's are on their way while this one is used)
      if (KIND == kPdInt4) ahead(at);
      unsigned char* stage = ring + stage_at * Sh::kStage;
      const uint32_t sk = ring_s + stage_at * Sh::kStage, sv = sk + TILE * Sh::kRow;
      const int* s_page = s_pages + page_at * TILE;
      if (fresh >= 0) {  // the new token's row into its page, if it has one
        const int page = s_page[fresh], place = cu.n - 1 - paged_nth(c, cu.n - 1) * c.P, sw = pd_swizzle<RC>(fresh);
        const bool has = (unsigned)page < (unsigned)c.n_pages, writes = has && cu.block == 0;
        const size_t to = paged_row(c, layer, has ? page : 0, cu.head, place);
        unsigned char* in = stage + fresh * Sh::kRow;
        if (lane < D / 8) {
          if constexpr (KIND == kPdInt4) {  // and into the tile
            uint32_t kn = 0u, vn = 0u;
            unsigned ks = 0u, vs = 0u;
            if (has) {
              kn = i4_quantise(c.type, kx, ks);
              vn = i4_quantise(c.type, vx, vs);
            }
            in += ((lane / 4 ^ sw) << 4) + (lane & 3) * 4;
            *reinterpret_cast<uint32_t*>(in) = kn;
            *reinterpret_cast<uint32_t*>(in + TILE * Sh::kRow) = vn;
            unsigned char* s_sc = stage + 2 * TILE * Sh::kRow + fresh * Sh::kScales;
            if ((lane & 3) == 0) {
              s_sc[lane / 4] = (unsigned char)ks;
              s_sc[D / 32 + lane / 4] = (unsigned char)vs;
            }
            if (writes) {
              *reinterpret_cast<uint32_t*>(c.k + to + lane * 4) = kn;
              *reinterpret_cast<uint32_t*>(c.v + to + lane * 4) = vn;
              unsigned char* g_sc = c.sc + paged_word(c, layer, page, cu.head, place) * Sh::kScales;
              if ((lane & 3) == 0) {
                g_sc[lane / 4] = (unsigned char)ks;
                g_sc[D / 32 + lane / 4] = (unsigned char)vs;
              }
            }
          } else if (KIND == kPdE4m3) {  // and into the tile
            uint2 ky = make_uint2(0u, 0u), vy = ky;
            if (has) {
              ky = paged_quantise(c.type, kx, c.ks[cu.head]);
              vy = paged_quantise(c.type, vx, c.vs[cu.head]);
            }
            in += ((lane / 2 ^ sw) << 4) + (lane & 1) * 8;
            *reinterpret_cast<uint2*>(in) = ky;
            *reinterpret_cast<uint2*>(in + TILE * Sh::kRow) = vy;
            if (writes) {
              *reinterpret_cast<uint2*>(c.k + to + lane * 8) = ky;
              *reinterpret_cast<uint2*>(c.v + to + lane * 8) = vy;
            }
          } else if (writes) {
            in += (lane ^ sw) << 4;
            *reinterpret_cast<uint4*>(c.k + to + lane * 16) = *reinterpret_cast<const uint4*>(in);
            *reinterpret_cast<uint4*>(c.v + to + lane * 16) = *reinterpret_cast<const uint4*>(in + TILE * Sh::kRow);
          }
        }
        if (c.w && writes && lane == 0)
          c.pos[paged_word(c, layer, page, cu.head, place)] = a.row_pos ? a.row_pos[cu.row] : cu.n - 1;
        __syncwarp();
      }
      if constexpr (KIND == kPdInt4) {
        int4_tile(stage_at, page_at, slot0);
      } else {
      float x[MT][NT][4];
      // (a tile lies on a multiple of its rows' length: the chunk's bits of an address can be set by xor)
      const uint32_t k_at = sk + (lane & 15) * Sh::kRow + ((lane >> 4 ^ pd_swizzle<RC>(lane & 15)) << 4);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[m][nt][0] = x[m][nt][1] = x[m][nt][2] = x[m][nt][3] = 0.f;
        if (KIND == kPdE4m3) {
#pragma unroll
          for (int i = 0; i < DT; i += 2) {
            uint32_t b[4];
            ldsm_x4(b, (k_at ^ (i << 4)) + m * 16 * Sh::kRow);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t f[4] = {pd_halves_lo(b[2 * j]), pd_halves_lo(b[2 * j + 1]), pd_halves_hi(b[2 * j]),
                                     pd_halves_hi(b[2 * j + 1])};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) pd_mma<KIND>(x[m][nt], f, q.b[nt][i + j][0], q.b[nt][i + j][1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            uint32_t f[4];
            ldsm_x4(f, (k_at ^ (i << 5)) + m * 16 * Sh::kRow);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) pd_mma<KIND>(x[m][nt], f, q.b[nt][i][0], q.b[nt][i][1]);
          }
        }
      }
      // lane: slots g and g + 8 of a block (x[..][..][0..1], x[..][..][2..3]), heads 2 q4 and 2 q4 + 1
      bool every = true;  // slot of the tile is there
#pragma unroll
      for (int j = lane; j < TILE; j += 32) every &= (unsigned)s_page[j] < (unsigned)c.n_pages;
      if (!__all_sync(0xffffffffu, every)) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bool there = (unsigned)s_page[m * 16 + g + 8 * e] < (unsigned)c.n_pages;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              // (the factors are positive; an infinite logit of a slot that is not there stays below every reference)
              if (!there) x[m][nt][2 * e] = x[m][nt][2 * e + 1] = -INFINITY;
            }
          }
      }
      if (c.w) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int page = s_page[m * 16 + g + 8 * e];
            if ((unsigned)page >= (unsigned)c.n_pages) continue;
            const int slot = slot0 + m * 16 + g + 8 * e, place = slot - paged_nth(c, slot) * c.P;
            const size_t word = ((size_t)page * c.Hkv + cu.head) * c.P + place;
            float* to = wk.logits + word * paged_even(c.G);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const int in_group = cu.block * H + nt * 8 + 2 * q4;
              const float2 y = make_float2(x[m][nt][2 * e] * sc[nt][0], x[m][nt][2 * e + 1] * sc[nt][1]);
              if (in_group < c.G) *reinterpret_cast<float2*>(to + in_group) = y;
            }
          }
      }
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float most = fmaxf(x[0][nt][e], x[0][nt][e + 2]);
#pragma unroll
          for (int m = 1; m < MT; ++m) most = fmaxf(most, fmaxf(x[m][nt][e], x[m][nt][e + 2]));
          top[nt][e] = most * sc[nt][e];
          grow |= top[nt][e] > ref[nt][e] + (kOff + kGrow);
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top[nt][e] = fmaxf(top[nt][e], __shfl_xor_sync(0xffffffffu, top[nt][e], d));
            const float to = fmaxf(ref[nt][e], top[nt][e] - kOff), by = pd_exp2(ref[nt][e] - to);
            ref[nt][e] = to;
            sum[nt][e] *= by;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
              O[nt][i][e] *= by;
              O[nt][i][e + 2] *= by;
            }
          }
      }
      // probabilities as a sum of terms of the products' type, as V^T P^T takes them
      uint32_t term[kTerms][MT][NT][2];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = pd_exp2(fmaf(x[m][nt][e], sc[nt][e & 1], -ref[nt][e & 1]));
            sum[nt][e & 1] += p[e];
          }
          constexpr int T = KIND == kPdBf16 ? LTRI_TYPE_BF16 : LTRI_TYPE_FP16;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int t = 0; t < kTerms; ++t) {
              const uint32_t h = paged_pack(T, p[2 * e], p[2 * e + 1]);
              term[t][m][nt][e] = pd_transpose(h);
              const float2 back = paged_unpack(T, h);
              p[2 * e] -= back.x;
              p[2 * e + 1] -= back.y;
            }
          }
        }
      // A tile's products are added up by themselves, a block's smallest term first, and their sum to the other tiles'.  (The
      // tensor cores cut off what an accumulator has no bits for, always towards zero: with O as the accumulator small values
      // beside large ones were lost, and outputs over bf16 pages differed twice as much from fp32 arithmetic's.  64 ragged rows in
      // 8 bits 61.5 us, with O 59.8; rows of 256 in 16 bits 35.8 and 34.7; the others no slower.)
      const int v_row = KIND == kPdE4m3 ? lane & 15 : (lane & 7) + (lane >> 4) * 8;
      const int v_ch = KIND == kPdE4m3 ? lane >> 4 : (lane >> 3) & 1;
      const uint32_t v_at = sv + v_row * Sh::kRow + ((v_ch ^ pd_swizzle<RC>(v_row)) << 4);
      constexpr int kAtOnce = KIND == kPdE4m3 ? 2 : 1;  // slices of 16 elements
#pragma unroll
      for (int i = 0; i < DT; i += kAtOnce) {
        float z[kAtOnce][NT][4];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) z[j][nt][0] = z[j][nt][1] = z[j][nt][2] = z[j][nt][3] = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          uint32_t b[4];
          ldsm_x4_t(b, (v_at ^ (i << (KIND == kPdE4m3 ? 4 : 5))) + m * 16 * Sh::kRow);
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j) {
            uint32_t f[4] = {b[0], b[1], b[2], b[3]};
            if (KIND == kPdE4m3) {
              // a 16-byte chunk's 8 pairs of neighbours are the 8 rows of a transposed matrix: row g has elements 2g and 2g + 1
              // of slots 2 q4 and 2 q4 + 1
#pragma unroll
              for (int e = 0; e < 2; ++e) {  // (with e, 8 slots further)
                const uint32_t y = __byte_perm(b[2 * j + e], 0u, 0x3120);
                f[2 * e] = pd_halves_lo(y);
                f[2 * e + 1] = pd_halves_hi(y);
              }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int t = kTerms - 1; t >= 0; --t) pd_mma<KIND>(z[j][nt], f, term[t][m][nt][0], term[t][m][nt][1]);
          }
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) O[nt][i + j][e] += z[j][nt][e];
      }
      }
      __syncwarp();
      stage_at = next(stage_at, S);
      page_at = next(page_at, Sh::kPages);
      const bool ends = cu.tile + 1 == cu.tiles;
      if (ends || at + 1 == mine) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], d);
        // A unit that reaches back behind the run and ends here is set aside for the warp that has its first piece, or, if
        // that is another CTA's, handed in; one that outlasts the run stays in the registers, and in the ring, which is empty
        // then.
        const PdOpen o{t0 + at - cu.tile, cu.row, cu.head, cu.block, cu.tiles};
        bool complete = whole && ends;
        if (!ends) {
          if (lane == 0) s_open[warp] = o;
          set_aside(reinterpret_cast<float*>(ring));
        } else if (!whole && warp > 0) {
          set_aside(wk.lead + ((size_t)blockIdx.x * W + warp) * wk.stride);
        } else if (!whole) {
          complete = hand_in(o, false);
        }
        if (complete) put_unit(cu);
      }
      pd_advance<TILE>(cu, c, r, wk.blocks);
    }
    if (KIND != kPdInt4 || at < 0) ahead(at);
    cp_async_commit();
    const bool begins = at >= 0 && at + 1 < mine && cu.tile == 0;
    if (at == -Sh::kAhead - 1 || (begins && !(kEarly && next_at == at + 1))) load_queries(q, cu);
  }

  // ---- units that the CTA's warps share: the warp that has a unit's first piece in this CTA adds the others to its own ----
  __syncthreads();
  {
    const PdOpen o = s_open[warp];
    if (o.tiles != 0 && (warp == 0 || o.begin >= t0)) {
      const int end = o.begin + o.tiles;
      const bool begins = o.begin >= c0, ends = end <= c1;
      const int upto = min(end, c1) - 1 - c0, last = kEven ? pd_sharer(per, upto, W) : (int)((unsigned)upto / (unsigned)per);  // warp
#pragma unroll 1
      for (int w = warp + 1; w <= last; ++w)
        add(ends && w == last ? wk.lead + ((size_t)blockIdx.x * W + w) * wk.stride
                              : reinterpret_cast<const float*>(dsm + w * Sh::kRing));
      PdCursor u;
      u.row = o.row;
      u.head = o.head;
      u.block = o.block;
      if ((begins && ends) || hand_in(o, begins)) put_unit(u);
    }
  }
  // ---- units of many CTAs: whoever comes last to one joins its parts, a slice a warp ----
  __syncthreads();
  if (threadIdx.x < 2) {
    const PdOpen o = s_part[threadIdx.x];
    int last = 0;
    if (o.tiles != 0) {
      const int ctas = parts_of(o);
      int* count = wk.count + ((size_t)o.row * c.Hkv + o.head) * wk.blocks + o.block;
      // (the other threads' stores are ordered in front of it by the barrier; with __threadfence on either side 3000 cycles)
      last = paged_arrive(count) == ctas - 1;
      if (last) *count = 0;
    }
    s_last[threadIdx.x] = last;
  }
  __syncthreads();
#pragma unroll 1
  for (int w = 0; w < 2; ++w) {
    if (!s_last[w]) continue;
    const PdOpen o = s_part[w];
    // part 0, and parts 1 to n - 1 at equal distances
    const unsigned first = (unsigned)o.begin / cta_run;
    const int pieces = parts_of(o);
    const size_t stride = 2 * wk.stride;
    const float *base = wk.part + first * stride, *p0 = base + wk.stride;
    // their sums, brought to the largest reference: the heads' in top and tot, the warp's slices' in got
    float top[NT][2], tot[NT][2];
    float4 got[kSlices];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = kPdNone, tot[nt][0] = tot[nt][1] = 0.f;
#pragma unroll
    for (int k = 0; k < kSlices; ++k) got[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kBatch = kSlices <= 4 ? 4 : 2;  // (more make the passage longer, which costs as much as they save)
#pragma unroll 1
    for (int i0 = 0; i0 < pieces; i0 += kBatch) {
      float2 m[kBatch][NT], s[kBatch][NT];
      float4 z[kBatch][kSlices];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int i = i0 + b;
        const float* p = i == 0 ? p0 : base + min(i, pieces - 1) * stride;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          m[b][nt] = *reinterpret_cast<const float2*>(p + nt * 8 + 2 * q4);
          s[b][nt] = *reinterpret_cast<const float2*>(p + 16 + nt * 8 + 2 * q4);
          if (i >= pieces) m[b][nt] = make_float2(kPdNone, kPdNone), s[b][nt] = make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < kSlices; ++k)
          z[b][k] = reinterpret_cast<const float4*>(p + 32)[min(k * W + warp, NT * DT - 1) * 32 + lane];
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float to = top[nt][e];
#pragma unroll
          for (int b = 0; b < kBatch; ++b) to = fmaxf(to, e ? m[b][nt].y : m[b][nt].x);
          const float by = pd_exp2(top[nt][e] - to);
          top[nt][e] = to;
          tot[nt][e] *= by;
          float f[kBatch];
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            f[b] = pd_exp2((e ? m[b][nt].y : m[b][nt].x) - to);
            tot[nt][e] += f[b] * (e ? s[b][nt].y : s[b][nt].x);
          }
#pragma unroll
          for (int k = 0; k < kSlices; ++k) {
            if ((k * W + warp) / DT != nt) continue;
            float& g0 = e ? got[k].y : got[k].x;
            float& g1 = e ? got[k].w : got[k].z;
            g0 *= by;
            g1 *= by;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              if (i0 + b >= pieces) continue;  // (a repeated piece's sums may be infinite)
              g0 += f[b] * (e ? z[b][k].y : z[b][k].x);
              g1 += f[b] * (e ? z[b][k].w : z[b][k].z);
            }
          }
        }
      }
    }
    PdCursor u;
    u.row = o.row;
    u.head = o.head;
    u.block = o.block;
    const float vs = KIND == kPdInt4 ? kI4Back : c.vs ? c.vs[o.head] : 1.f;
#pragma unroll
    for (int k = 0; k < kSlices; ++k) {
      if (k * W + warp >= NT * DT) continue;
      const bool upper = NT == 2 && (k * W + warp) / DT == 1;
      const float b0 = one_over(upper ? tot[NT - 1][0] : tot[0][0]), b1 = one_over(upper ? tot[NT - 1][1] : tot[0][1]);
      const float z[4] = {scaled(got[k].x, b0, vs), scaled(got[k].y, b1, vs), scaled(got[k].z, b0, vs), scaled(got[k].w, b1, vs)};
      put_slice(u, upper ? 1 : 0, (k * W + warp) % DT, z);
    }
    if (warp == 0)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        put_lse(u, nt, 0, top[nt][0], tot[nt][0]);
        put_lse(u, nt, 1, top[nt][1], tot[nt][1]);
      }
  }
  // empty rows
  for (int row = blockIdx.x; row < r.n; row += gridDim.x) {
    if (paged_len(c, r, row) != 0) continue;
    for (int i = threadIdx.x; i < c.Hq * D / 8; i += W * 32)
      reinterpret_cast<uint4*>(a.out)[(size_t)row * (c.Hq * D / 8) + i] = make_uint4(0u, 0u, 0u, 0u);
    if (a.lse)
      for (int i = threadIdx.x; i < c.Hq; i += W * 32) a.lse[(size_t)row * c.Hq + i] = -INFINITY;
  }
}

// weights[j] = decay * weights[j] + sum over the group's heads of 2^(x_j - L), from the logits that the attention left in L2.
// Bound: latency (page number, then logits and weight), so a slot's page and weight are asked for ahead of its logits, the
// first ones before the attention kernel is through.  (32 bytes a slot whatever the group, and nothing ahead: 10.8 us for 16
// rows of 4097 slots and 8 KV heads, 9.5 so; eight CTAs an SM instead of four: a step of two layers 3 us longer.)
constexpr int kPwThreads = 256, kPwCtas = 4;
__global__ void __launch_bounds__(kPwThreads, kPwCtas)
    k_paged_weights(PagedCache c, PagedRows r, int layer, PdWork wk, bool fresh) {
  // (the lengths are older than the attention kernel, which had waited for its predecessor when it released this one; so are
  // the weights, but for the new token's slot, which starts from 0)
  PdCursor u;
  int total;
  bool lone;
  const int per = pd_deal<kPwThreads>(u, total, lone, gridDim.x, blockIdx.x, 0, c, r, 1), t0 = blockIdx.x * per;
  const int t1 = min(t0 + per, total);
  float* weights = c.w + (size_t)layer * c.n_pages * c.Hkv * c.P;
  size_t word = 0;
  float old = 0.f;
  int page = -1;
  auto ask = [&]() {
    const int slot = u.tile * kPwThreads + threadIdx.x, nth = paged_nth(c, slot);
    page = slot < u.n ? paged_page(c, r, u.row, nth) : -1;
    word = ((size_t)max(page, 0) * c.Hkv + u.head) * c.P + (slot - nth * c.P);
    old = page < 0 || (fresh && slot == u.n - 1) ? 0.f : weights[word];
  };
  if (t0 < t1) ask();
  chain_wait();
  for (int t = t0; t < t1; ++t) {
    if (t > t0) ask();
    if (page >= 0) {
      const float2* x = reinterpret_cast<const float2*>(wk.logits + word * paged_even(c.G));
      const float* l2 = wk.lse2 + (size_t)u.row * c.Hq + (size_t)u.head * c.G;
      float p = 0.f;
      int h = 0;
#pragma unroll 4
      for (; h + 1 < c.G; h += 2) {
        const float2 y = x[h / 2];
        p += pd_exp2(y.x - l2[h]);
        p += pd_exp2(y.y - l2[h + 1]);
      }
      if (h < c.G) p += pd_exp2(x[h / 2].x - l2[h]);
      weights[word] = old * c.decay + p;
    }
    pd_advance<kPwThreads>(u, c, r, 1);
  }
}

namespace {

template <int KIND, int D, int NT>
cudaError_t prepare_one() {
  return allow_smem(k_paged_decode<KIND, D, NT>, PdShape<KIND, D, NT>::kSmem);
}
template <int KIND, int D>
cudaError_t prepare_dim() {
  return first_error(prepare_one<KIND, D, 1>(), prepare_one<KIND, D, 2>());
}
template <int KIND>
cudaError_t prepare_kind(int D) {
  return D == 64 ? prepare_dim<KIND, 64>() : D == 128 ? prepare_dim<KIND, 128>() : prepare_dim<KIND, 256>();
}

template <int KIND, int D, int NT>
cudaError_t launch_one(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, const PdWork& w,
                       cudaStream_t s) {
  using Sh = PdShape<KIND, D, NT>;
  static_assert(Sh::kWarps <= kPagedWarps, "the workspace has partial sums of that many warps");
  return launch_chained(k_paged_decode<KIND, D, NT>, dim3(c.sms), dim3(Sh::kWarps * 32), Sh::kSmem, s, c, r, layer, a, w);
}
template <int KIND, int D>
cudaError_t launch_dim(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, const PdWork& w,
                       cudaStream_t s) {
  return w.heads == 8 ? launch_one<KIND, D, 1>(c, r, layer, a, w, s) : launch_one<KIND, D, 2>(c, r, layer, a, w, s);
}
template <int KIND>
cudaError_t launch_kind(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, const PdWork& w,
                        cudaStream_t s) {
  if (c.D == 64) return launch_dim<KIND, 64>(c, r, layer, a, w, s);
  if (c.D == 128) return launch_dim<KIND, 128>(c, r, layer, a, w, s);
  return launch_dim<KIND, 256>(c, r, layer, a, w, s);
}

}  // namespace

cudaError_t prepare_paged(const PagedCache& c) {
  if (c.cache_type == LTRI_TYPE_INT4) return prepare_kind<kPdInt4>(c.D);
  if (c.cache_type == LTRI_TYPE_E4M3) return prepare_kind<kPdE4m3>(c.D);
  return c.type == LTRI_TYPE_BF16 ? prepare_kind<kPdBf16>(c.D) : prepare_kind<kPdFp16>(c.D);
}

PagedBlocks paged_blocks(int group) {
  PagedBlocks b;
  b.heads = group <= 8 ? 8 : 16;
  b.count = (group + b.heads - 1) / b.heads;
  return b;
}
size_t paged_part_floats(int group, int head_dim) { return 32 + (size_t)paged_blocks(group).heads * head_dim; }

int paged_decode_kernels(const PagedCache& c) { return c.w ? 2 : 1; }

cudaError_t launch_paged_decode(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, cudaStream_t s) {
  const PagedBlocks b = paged_blocks(c.G);
  const PdWork w{b.heads, b.count, c.part, c.lead, (int)paged_part_floats(c.G, c.D), c.count, c.logits, c.lse2};
  cudaError_t e;
  if (c.cache_type == LTRI_TYPE_INT4) e = launch_kind<kPdInt4>(c, r, layer, a, w, s);
  else if (c.cache_type == LTRI_TYPE_E4M3) e = launch_kind<kPdE4m3>(c, r, layer, a, w, s);
  else if (c.type == LTRI_TYPE_BF16) e = launch_kind<kPdBf16>(c, r, layer, a, w, s);
  else e = launch_kind<kPdFp16>(c, r, layer, a, w, s);
  if (e != cudaSuccess || !c.w) return e;
  return launch_chained(k_paged_weights, dim3(c.sms * kPwCtas), dim3(kPwThreads), 0, s, c, r, layer, w, a.k != nullptr);
}

}  // namespace ltri
