// Attention of one new token per row over a caller-owned paged cache, split over the cache's length and joined.
//
// x_j = c q.K_j, out = sum_j 2^(x_j - L) V_j with c in log2 units and L = log2 sum_j 2^(x_j): one pass over K and V with a running
// reference m, sums of 2^(x_j - m) and of 2^(x_j - m) V_j, which parts of a row join by rescaling to the larger m.
//
// Bound: HBM (a KV head's rows are read once for all of its query heads: 2 G flop a byte in 16 bits).  So the work is the rows'
// tiles, and it is dealt evenly: the tiles of all (row, KV head) units stand in one line, of which every CTA (one per SM) takes an
// equal run, across units if need be.  Ragged batches and single long rows fill the GPU alike, and no count of splits has to
// be chosen.  A unit within one run is written by its CTA; of a unit that several CTAs share, the last one to finish joins the
// partial sums, in the order of the runs.
//
// A warp has 16 slots of a tile and a ring of its own that cp.async fills several tiles ahead, across units; warps meet
// only at the end of a unit.  Both products run on mma.sync with the slots (or head_dim) as the 16 rows and the heads of
// the KV group as the 8 columns: S^T = K Q^T, O^T = V^T P^T, so that up to eight heads fill the instruction exactly.  (tcgen05 takes
// 64 rows at least, and its operands come through descriptors of whole tiles, which pages of any size are not.)
#include "mma_util.cuh"
#include "paged.cuh"

namespace ltri {

enum { kPdBf16 = 0, kPdFp16 = 1, kPdE4m3 = 2 };  // what the pages hold

template <int KIND, int D>
struct PdShape {
  static constexpr int kRow = KIND == kPdE4m3 ? D : 2 * D;      // bytes of a cached row
  static constexpr int kChunks = kRow / 16;
  static constexpr int kWarps = D == 256 ? 4 : 8;
  static constexpr int kTile = kWarps * 16;                     // slots of a CTA's tile
  static constexpr int kRaw = 32 * kRow;                        // a stage: 16 K rows, 16 V rows, the new token's
  static constexpr int kStage = kRaw + 4 * D + 64;              // K and V rows as they come, 16 page numbers
  static constexpr int kMerge = kWarps / 2 * 8 * D * 4;         // half the warps' sums of eight heads
  static constexpr int kFit = (232448 - 1024 - kMerge - 2048) / (kWarps * kStage);
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kSmem = kWarps * kStages * kStage + kMerge;
  static_assert(kStages >= 3, "two tiles on their way and one in use");
};

struct PdWork {
  int heads;            // of a block: 8 or 16
  int blocks;           // of a KV head's query heads
  float* part;          // [CTAs][2] partial sums: 16 references, 16 sums, then the accumulators
  int part_stride;      // floats
  int* count;           // [rows * Hkv * blocks]: CTAs that have written their part
  float* logits;        // [n_pages][Hkv][P][blocks * heads], with weights
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
// Two e4m3 values in the lower half of x as two halves.
__device__ __forceinline__ uint32_t pd_halves(uint32_t x) {
  uint32_t y;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(y) : "r"(x));
  return y;
}

// Byte of 16-byte chunk `ch` of row `row` in a tile of rows of CHUNKS chunks: eight rows' equal chunks lie in different banks.
template <int CHUNKS>
__device__ __forceinline__ uint32_t pd_at(int row, int ch) {
  const int x = CHUNKS >= 8 ? row & 7 : (row >> 1) & 3;
  return row * (CHUNKS * 16) + ((ch ^ x) << 4);
}

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
    u.n = ++u.row < r.n ? paged_len(c, r, u.row) : 1;
    u.tiles = (u.n + TILE - 1) / TILE;
  } while (u.tiles == 0);
}

// All lanes of a warp: tiles of the whole call, and the cursor of tile CTA * per where per is every CTA's run.  Returns per.
template <int TILE>
__device__ __forceinline__ long long pd_deal(PdCursor& u, long long& total, const PagedCache& c, const PagedRows& r, int blocks) {
  const int lane = threadIdx.x & 31;
  const long long per_row = (long long)c.Hkv * blocks;
  total = 0;
  long long first = 0;  // of the first 32 rows, kept
  for (int base = 0; base < r.n; base += 32) {
    const int row = base + lane;
    long long t = row < r.n ? (paged_len(c, r, row) + TILE - 1) / TILE * per_row : 0;
    if (base == 0) first = t;
#pragma unroll
    for (int d = 16; d; d >>= 1) t += shfl_xor_ll(t, d);
    total += t;
  }
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  long long left = blockIdx.x * per;
  if (left >= total) return per;
  for (int base = 0; base < r.n; base += 32) {
    const int row = base + lane;
    const long long t = base == 0 ? first : row < r.n ? (paged_len(c, r, row) + TILE - 1) / TILE * per_row : 0;
    long long inc = t;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = shfl_up_ll(inc, d);
      if (lane >= d) inc += y;
    }
    const unsigned in = __ballot_sync(0xffffffffu, left < inc);
    if (in) {
      const int at = __ffs(in) - 1;
      const long long begin = shfl_ll(inc - t, at);
      u.row = base + at;
      u.n = paged_len(c, r, u.row);
      u.tiles = (u.n + TILE - 1) / TILE;
      left -= begin;
      const long long unit = left / u.tiles;
      u.tile = (int)(left - unit * u.tiles);
      u.head = (int)(unit / blocks);
      u.block = (int)(unit - (long long)u.head * blocks);
      return per;
    }
    left -= shfl_ll(inc, 31);
  }
  return per;
}

template <int KIND, int D, int NT>
__global__ void __launch_bounds__(PdShape<KIND, D>::kWarps * 32, 1)
    k_paged_decode(PagedCache c, PagedRows r, int layer, PagedStep a, PdWork wk) {
  using Sh = PdShape<KIND, D>;
  constexpr int W = Sh::kWarps, TILE = Sh::kTile, S = Sh::kStages, RC = Sh::kChunks, DT = D / 16, H = 8 * NT;
  constexpr int kSlices = NT * DT / W > 0 ? NT * DT / W : 1;  // 16-row slices of the sums that a warp finishes
  // Probabilities carry a factor 2^kOff that cancels in out and lse.  A half has 2^-24 as its smallest step: with the largest
  // probability at 2^10 a slot's contribution is still seen 2^-35 below it, so that 2^20 of them cannot lose 2^-14 of a sum.
  // The reference moves only when a logit exceeds it by kGrow, which bounds the probabilities by 2^(kOff + kGrow).
  constexpr float kOff = KIND == kPdBf16 ? 0.f : 10.f, kGrow = 4.f;
  extern __shared__ __align__(1024) unsigned char dsm[];
  __shared__ float s_ref[W][16], s_sum[W][16];
  __shared__ int s_last;
  float4* s_merge = reinterpret_cast<float4*>(dsm + W * S * Sh::kStage);
  chain_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  unsigned char* ring = dsm + warp * S * Sh::kStage;
  const uint32_t ring_s = smem_u32(ring);

  PdCursor cu;
  long long total;
  const long long per = pd_deal<TILE>(cu, total, c, r, wk.blocks), t0 = blockIdx.x * per;
  const int mine = t0 >= total ? 0 : (int)(t0 + per <= total ? per : total - t0);
  PdCursor ci = cu;
  int issued = 0;

  auto page_of = [&](const PdCursor& u) -> int {  // of this lane's slot: -1 where there is none
    const int slot = u.tile * TILE + warp * 16 + (lane & 15);
    return slot < u.n ? paged_page(c, r, u.row, slot / c.P) : -1;
  };
  int pg = mine > 0 ? page_of(ci) : -1;  // of the tile that is issued next
  auto issue = [&]() {
    if (issued < mine) {
      const int slot0 = ci.tile * TILE + warp * 16, st = issued % S;
      if (slot0 < ci.n) {
        const int slot = slot0 + (lane & 15);
        const long long off = pg < 0 ? -1 : (long long)paged_row(c, layer, pg, ci.head, slot % c.P);
        int* s_page = reinterpret_cast<int*>(ring + st * Sh::kStage + Sh::kRaw + 4 * D);
        if (lane < 16) s_page[lane] = pg;
        const uint32_t sk = ring_s + st * Sh::kStage, sv = sk + 16 * Sh::kRow;
        const int fresh = a.k && ci.n - 1 - slot0 < 16 ? ci.n - 1 - slot0 : -1;  // the new token's row comes from the caller
#pragma unroll
        for (int i = 0; i < RC / 2; ++i) {
          const int row = i * (32 / RC) + lane / RC, ch = lane % RC;
          const long long o = shfl_ll(off, row);
          const bool in = o >= 0 && row != fresh;
          const size_t at = in ? (size_t)o + ch * 16 : 0;
          cp_async16(sk + pd_at<RC>(row, ch), c.k + at, in ? 16 : 0);
          cp_async16(sv + pd_at<RC>(row, ch), c.v + at, in ? 16 : 0);
        }
        if (fresh >= 0 && lane < D / 8) {
          const size_t at = ci.row * a.kv_stride + ((size_t)ci.head * D + lane * 8) * 2;
          cp_async16(ring_s + st * Sh::kStage + Sh::kRaw + lane * 16, a.k + at, 16);
          cp_async16(ring_s + st * Sh::kStage + Sh::kRaw + 2 * D + lane * 16, a.v + at, 16);
        }
      }
      if (++issued < mine) {
        pd_advance<TILE>(ci, c, r, wk.blocks);
        pg = page_of(ci);
      }
    }
    cp_async_commit();
  };
#pragma unroll 1
  for (int i = 0; i < S - 1; ++i) issue();

  uint32_t qb[NT][DT][2];
  float sc[NT][2];      // logits' factor of this lane's heads
  float O[NT][DT][4], ref[NT][2], sum[NT][2];
  bool whole = false;   // the unit has begun in this CTA
  for (int at = 0; at < mine; ++at) {
    if (at == 0 || cu.tile == 0) {  // a unit begins: its queries
      whole = cu.tile == 0;
      const float ks = c.ks ? c.ks[cu.head] : 1.f;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int in_group = cu.block * H + nt * 8 + g;
        const unsigned char* qr = a.q + cu.row * a.q_stride + ((size_t)cu.head * c.G + in_group) * D * 2;
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          // (8-bit rows: a 16-byte chunk is one step of 16, of which a lane holds four neighbours)
          const int e = KIND == kPdE4m3 ? i * 16 + q4 * 4 : i * 16 + q4 * 2;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int el = KIND == kPdE4m3 ? e + 2 * j : e + 8 * j;
            qb[nt][i][j] = in_group < c.G ? *reinterpret_cast<const uint32_t*>(qr + el * 2) : 0u;
            most = max(most, max(qb[nt][i][j] & 0x7fffu, (qb[nt][i][j] >> 16) & 0x7fffu));
          }
        }
        float back = 1.f;
        if (KIND == kPdE4m3 && c.type == LTRI_TYPE_BF16) {
          // bf16 queries as halves: a power of two brings the row's largest element to [2^14, 2^15); what then falls below
          // the halves' range is 2^-39 of it
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
          const int ex = (int)(most >> 7);  // biased exponent
          const int up = ex == 0 || ex == 255 ? 0 : 127 + 14 - ex;
#pragma unroll
          for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float2 f = paged_unpack(LTRI_TYPE_BF16, qb[nt][i][j]);
              qb[nt][i][j] = paged_pack(LTRI_TYPE_FP16, ldexpf(f.x, up), ldexpf(f.y, up));
            }
          back = ldexpf(1.f, -up);
        }
        // (the queries lie with head g, the logits with heads 2 q4 and 2 q4 + 1)
#pragma unroll
        for (int e = 0; e < 2; ++e) sc[nt][e] = c.scale * ks * __shfl_sync(0xffffffffu, back, (2 * q4 + e) * 4);
        ref[nt][0] = ref[nt][1] = -INFINITY;
        sum[nt][0] = sum[nt][1] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) O[nt][i][0] = O[nt][i][1] = O[nt][i][2] = O[nt][i][3] = 0.f;
      }
    }
    cp_async_wait<S - 2>();
    __syncwarp();
    const int slot0 = cu.tile * TILE + warp * 16, st = at % S;
    if (slot0 < cu.n) {
      unsigned char* stage = ring + st * Sh::kStage;
      const uint32_t sk = ring_s + st * Sh::kStage, sv = sk + 16 * Sh::kRow;
      const int* s_page = reinterpret_cast<const int*>(stage + Sh::kRaw + 4 * D);
      const int fresh = a.k && cu.n - 1 - slot0 < 16 ? cu.n - 1 - slot0 : -1;
      if (fresh >= 0 && s_page[fresh] >= 0) {  // the new token's row into the tile and into its page
        const int page = s_page[fresh], place = (cu.n - 1) % c.P;
        if (lane < D / 8) {
          const uint4 kx = *reinterpret_cast<const uint4*>(stage + Sh::kRaw + lane * 16);
          const uint4 vx = *reinterpret_cast<const uint4*>(stage + Sh::kRaw + 2 * D + lane * 16);
          const size_t to = paged_row(c, layer, page, cu.head, place);
          if (KIND == kPdE4m3) {
            const uint2 ky = paged_quantise(c.type, kx, c.ks[cu.head]), vy = paged_quantise(c.type, vx, c.vs[cu.head]);
            const uint32_t in = pd_at<RC>(fresh, lane / 2) + (lane & 1) * 8;
            *reinterpret_cast<uint2*>(stage + in) = ky;
            *reinterpret_cast<uint2*>(stage + 16 * Sh::kRow + in) = vy;
            if (cu.block == 0) {
              *reinterpret_cast<uint2*>(c.k + to + lane * 8) = ky;
              *reinterpret_cast<uint2*>(c.v + to + lane * 8) = vy;
            }
          } else {
            const uint32_t in = pd_at<RC>(fresh, lane);
            *reinterpret_cast<uint4*>(stage + in) = kx;
            *reinterpret_cast<uint4*>(stage + 16 * Sh::kRow + in) = vx;
            if (cu.block == 0) {
              *reinterpret_cast<uint4*>(c.k + to + lane * 16) = kx;
              *reinterpret_cast<uint4*>(c.v + to + lane * 16) = vx;
            }
          }
        }
        if (c.w && cu.block == 0 && lane == 0) {
          const size_t word = paged_word(c, layer, page, cu.head, place);
          c.w[word] = 0.f;
          c.pos[word] = a.row_pos ? a.row_pos[cu.row] : cu.n - 1;
        }
        __syncwarp();
      }
      float x[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) x[nt][0] = x[nt][1] = x[nt][2] = x[nt][3] = 0.f;
      if (KIND == kPdE4m3) {
#pragma unroll
        for (int i = 0; i < DT; i += 2) {
          uint32_t b[4];
          ldsm_x4(b, sk + pd_at<RC>(lane & 15, i + (lane >> 4)));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t f[4] = {pd_halves(b[2 * j]), pd_halves(b[2 * j + 1]), pd_halves(b[2 * j] >> 16),
                                   pd_halves(b[2 * j + 1] >> 16)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) pd_mma<KIND>(x[nt], f, qb[nt][i + j][0], qb[nt][i + j][1]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          uint32_t f[4];
          ldsm_x4(f, sk + pd_at<RC>(lane & 15, 2 * i + (lane >> 4)));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) pd_mma<KIND>(x[nt], f, qb[nt][i][0], qb[nt][i][1]);
        }
      }
      // lane: slots slot0 + g and + 8 (x[0..1], x[2..3]), heads 2 q4 and 2 q4 + 1
      const int p0 = s_page[g], p1 = s_page[g + 8];
      bool grow = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[nt][e] = (e < 2 ? p0 : p1) >= 0 ? x[nt][e] * sc[nt][e & 1] : -INFINITY;
          grow |= x[nt][e] > ref[nt][e & 1] + (kOff + kGrow);
        }
      if (c.w) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int page = e ? p1 : p0;
          if (page < 0) continue;
          const size_t word = ((size_t)page * c.Hkv + cu.head) * c.P + (slot0 + g + 8 * e) % c.P;
          float2* to = reinterpret_cast<float2*>(wk.logits + word * (wk.blocks * H) + cu.block * H);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) to[nt * 4 + q4] = make_float2(x[nt][2 * e], x[nt][2 * e + 1]);
        }
      }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(x[nt][e], x[nt][e + 2]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float to = fmaxf(ref[nt][e], top - kOff);
            const float by = to == -INFINITY ? 1.f : pd_exp2(ref[nt][e] - to);
            ref[nt][e] = to;
            sum[nt][e] *= by;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
              O[nt][i][e] *= by;
              O[nt][i][e + 2] *= by;
            }
          }
      }
      // probabilities as two terms of the products' type, as V^T P^T takes them
      uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float m = ref[nt][e & 1];
          p[e] = pd_exp2(x[nt][e] - (m == -INFINITY ? 0.f : m));
          sum[nt][e & 1] += p[e];
        }
        constexpr int T = KIND == kPdBf16 ? LTRI_TYPE_BF16 : LTRI_TYPE_FP16;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t h = paged_pack(T, p[2 * e], p[2 * e + 1]);
          const float2 back = paged_unpack(T, h);
          hi[nt][e] = pd_transpose(h);
          lo[nt][e] = pd_transpose(paged_pack(T, p[2 * e] - back.x, p[2 * e + 1] - back.y));
        }
      }
#pragma unroll
      for (int i = 0; i < DT; i += KIND == kPdE4m3 ? 2 : 1) {
        uint32_t b[4];
        if (KIND == kPdE4m3) {
          // a 16-byte chunk's 8 pairs of neighbours are the 8 rows of a transposed matrix: row g has elements 2g and 2g + 1
          ldsm_x4_t(b, sv + pd_at<RC>(lane & 15, i + (lane >> 4)));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t f[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {  // slots 2 q4, 2 q4 + 1 and, with e, 8 further
              const uint32_t l = pd_halves(b[2 * j + e]), h = pd_halves(b[2 * j + e] >> 16);
              f[2 * e] = __byte_perm(l, h, 0x5410);
              f[2 * e + 1] = __byte_perm(l, h, 0x7632);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              pd_mma<KIND>(O[nt][i + j], f, hi[nt][0], hi[nt][1]);
              pd_mma<KIND>(O[nt][i + j], f, lo[nt][0], lo[nt][1]);
            }
          }
        } else {
          ldsm_x4_t(b, sv + pd_at<RC>((lane & 7) + (lane >> 4) * 8, 2 * i + ((lane >> 3) & 1)));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            pd_mma<KIND>(O[nt][i], b, hi[nt][0], hi[nt][1]);
            pd_mma<KIND>(O[nt][i], b, lo[nt][0], lo[nt][1]);
          }
        }
      }
    }
    __syncwarp();
    issue();
    const bool ends = cu.tile + 1 == cu.tiles;
    if (ends || at + 1 == mine) {
      // ---- the warps' sums, brought to one reference ----
      float top[NT][2], tot[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], d);
          if (g == 0) {
            s_ref[warp][nt * 8 + 2 * q4 + e] = ref[nt][e];
            s_sum[warp][nt * 8 + 2 * q4 + e] = sum[nt][e];
          }
        }
      __syncthreads();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int h = nt * 8 + 2 * q4 + e;
          float m = -INFINITY, t = 0.f;
#pragma unroll
          for (int w = 0; w < W; ++w) m = fmaxf(m, s_ref[w][h]);
          const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int w = 0; w < W; ++w) t += s_sum[w][h] * pd_exp2(s_ref[w][h] - mu);
          top[nt][e] = m;
          tot[nt][e] = t;
          const float by = pd_exp2(ref[nt][e] - mu);
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            O[nt][i][e] *= by;
            O[nt][i][e + 2] *= by;
          }
        }
      // the upper half of the warps hands its accumulators to the lower, then every warp adds up slices of the lower's
      float4 got[kSlices];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (warp >= W / 2) {
#pragma unroll
          for (int i = 0; i < DT; ++i)
            s_merge[((warp - W / 2) * DT + i) * 32 + lane] = make_float4(O[nt][i][0], O[nt][i][1], O[nt][i][2], O[nt][i][3]);
        }
        __syncthreads();
        if (warp < W / 2) {
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            float4& z = s_merge[(warp * DT + i) * 32 + lane];
            z.x += O[nt][i][0];
            z.y += O[nt][i][1];
            z.z += O[nt][i][2];
            z.w += O[nt][i][3];
          }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSlices; ++k) {
          const int sl = k * W + warp - nt * DT;  // slice of this block of eight heads
          if (sl >= 0 && sl < DT) {
            float4 z = s_merge[sl * 32 + lane];
#pragma unroll
            for (int w = 1; w < W / 2; ++w) {
              const float4 y = s_merge[(w * DT + sl) * 32 + lane];
              z.x += y.x;
              z.y += y.y;
              z.z += y.z;
              z.w += y.w;
            }
            got[k] = z;
          }
        }
        __syncthreads();
      }
      // ---- one CTA has all of the unit, or the last of its CTAs joins the parts ----
      bool write = whole && ends;
      if (!write) {
        const long long begin = t0 + at - cu.tile;  // of the unit, in the line
        const int first = (int)(begin / per), pieces = (int)((begin + cu.tiles - 1) / per) - first + 1;
        float* part = wk.part + (size_t)(2 * blockIdx.x + (whole ? 1 : 0)) * wk.part_stride;
        if (warp == 0 && g == 0)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              __stcg(part + nt * 8 + 2 * q4 + e, top[nt][e]);
              __stcg(part + 16 + nt * 8 + 2 * q4 + e, tot[nt][e]);
            }
#pragma unroll
        for (int k = 0; k < kSlices; ++k)
          if (k * W + warp < NT * DT) __stcg(reinterpret_cast<float4*>(part + 32) + (k * W + warp) * 32 + lane, got[k]);
        __threadfence();
        __syncthreads();
        int* count = wk.count + ((size_t)cu.row * c.Hkv + cu.head) * wk.blocks + cu.block;
        if (threadIdx.x == 0) {
          s_last = atomicAdd(count, 1) == pieces - 1;
          if (s_last) *count = 0;
        }
        __syncthreads();
        write = s_last;
        if (write) {
          __threadfence();
          auto piece = [&](int i) { return wk.part + (size_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * wk.part_stride; };
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float m = -INFINITY;
              for (int i = g; i < pieces; i += 8) m = fmaxf(m, __ldcg(piece(i) + nt * 8 + 2 * q4 + e));
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
              top[nt][e] = m;
              tot[nt][e] = 0.f;
            }
#pragma unroll
          for (int k = 0; k < kSlices; ++k) got[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int i = 0; i < pieces; ++i) {
            const float* from = piece(i);
            float by[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float2 m = __ldcg(reinterpret_cast<const float2*>(from + nt * 8) + q4);
              const float2 s = __ldcg(reinterpret_cast<const float2*>(from + 16 + nt * 8) + q4);
              by[nt][0] = pd_exp2(m.x - (top[nt][0] == -INFINITY ? 0.f : top[nt][0]));
              by[nt][1] = pd_exp2(m.y - (top[nt][1] == -INFINITY ? 0.f : top[nt][1]));
              tot[nt][0] += s.x * by[nt][0];
              tot[nt][1] += s.y * by[nt][1];
            }
#pragma unroll
            for (int k = 0; k < kSlices; ++k) {
              if (k * W + warp >= NT * DT) continue;
              const int nt = (k * W + warp) / DT;
              const float4 z = __ldcg(reinterpret_cast<const float4*>(from + 32) + (k * W + warp) * 32 + lane);
              const float b0 = NT == 1 || nt == 0 ? by[0][0] : by[NT - 1][0], b1 = NT == 1 || nt == 0 ? by[0][1] : by[NT - 1][1];
              got[k].x += z.x * b0;
              got[k].y += z.y * b1;
              got[k].z += z.z * b0;
              got[k].w += z.w * b1;
            }
          }
        }
      }
      if (write) {
        const float vs = c.vs ? c.vs[cu.head] : 1.f;
        const size_t head0 = (size_t)cu.row * c.Hq + (size_t)cu.head * c.G + cu.block * H;
        const int heads = min(H, c.G - cu.block * H);
#pragma unroll
        for (int k = 0; k < kSlices; ++k) {
          if (k * W + warp >= NT * DT) continue;
          const int nt = (k * W + warp) / DT, i = (k * W + warp) % DT;
          const float z[4] = {got[k].x, got[k].y, got[k].z, got[k].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int h = nt * 8 + 2 * q4 + (e & 1);
            if (h >= heads) continue;
            const float t = NT == 1 || nt == 0 ? tot[0][e & 1] : tot[NT - 1][e & 1];
            const int d = KIND == kPdE4m3 ? i * 16 + 2 * g + (e >> 1) : i * 16 + g + 8 * (e >> 1);
            const uint32_t y = paged_pack(c.type, t == 0.f ? 0.f : z[e] / t * vs, 0.f);
            reinterpret_cast<uint16_t*>(a.out)[(head0 + h) * D + d] = (uint16_t)y;
          }
        }
        if (warp == 0 && g == 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = nt * 8 + 2 * q4 + e;
              if (h >= heads) continue;
              const float l2 = tot[nt][e] == 0.f ? -INFINITY : top[nt][e] + log2f(tot[nt][e]);
              if (a.lse) a.lse[head0 + h] = l2 * 0.69314718055994531f;
              if (c.w) wk.lse2[head0 + h] = l2;
            }
        }
      }
    }
    pd_advance<TILE>(cu, c, r, wk.blocks);
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

// weights[j] = decay * weights[j] + sum over the group's heads of 2^(x_j - L), from the logits that the attention left.
constexpr int kPwThreads = 256;
__global__ void __launch_bounds__(kPwThreads) k_paged_weights(PagedCache c, PagedRows r, int layer, PdWork wk) {
  chain_wait();
  PdCursor u;
  long long total;
  const long long per = pd_deal<kPwThreads>(u, total, c, r, 1), t0 = blockIdx.x * per;
  const int row = wk.blocks * wk.heads;
  for (long long t = t0; t < t0 + per && t < total; ++t) {
    const int slot = u.tile * kPwThreads + threadIdx.x;
    const int page = slot < u.n ? paged_page(c, r, u.row, slot / c.P) : -1;
    if (page >= 0) {
      const size_t word = ((size_t)page * c.Hkv + u.head) * c.P + slot % c.P;
      const float* x = wk.logits + word * row;
      const float* l2 = wk.lse2 + (size_t)u.row * c.Hq + (size_t)u.head * c.G;
      float p = 0.f;
      for (int h = 0; h < c.G; ++h) p += pd_exp2(x[h] - l2[h]);
      float* w = c.w + (size_t)layer * c.n_pages * c.Hkv * c.P + word;
      *w = *w * c.decay + p;
    }
    pd_advance<kPwThreads>(u, c, r, 1);
  }
}

namespace {

template <int KIND, int D, int NT>
cudaError_t prepare_one() {
  return allow_smem(k_paged_decode<KIND, D, NT>, PdShape<KIND, D>::kSmem);
}
template <int KIND, int D>
cudaError_t prepare_dim() {
  return first_error(prepare_one<KIND, D, 1>(), prepare_one<KIND, D, 2>());
}
template <int KIND>
cudaError_t prepare_kind() {
  return first_error(prepare_dim<KIND, 64>(), first_error(prepare_dim<KIND, 128>(), prepare_dim<KIND, 256>()));
}

template <int KIND, int D>
cudaError_t launch_dim(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, const PdWork& w, int grid, cudaStream_t s) {
  using Sh = PdShape<KIND, D>;
  if (w.heads == 8)
    return launch_chained(k_paged_decode<KIND, D, 1>, dim3(grid), dim3(Sh::kWarps * 32), Sh::kSmem, s, c, r, layer, a, w);
  return launch_chained(k_paged_decode<KIND, D, 2>, dim3(grid), dim3(Sh::kWarps * 32), Sh::kSmem, s, c, r, layer, a, w);
}
template <int KIND>
cudaError_t launch_kind(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, const PdWork& w, int grid, cudaStream_t s) {
  if (c.D == 64) return launch_dim<KIND, 64>(c, r, layer, a, w, grid, s);
  if (c.D == 128) return launch_dim<KIND, 128>(c, r, layer, a, w, grid, s);
  return launch_dim<KIND, 256>(c, r, layer, a, w, grid, s);
}

}  // namespace

cudaError_t prepare_paged() {
  return first_error(prepare_kind<kPdBf16>(), first_error(prepare_kind<kPdFp16>(), prepare_kind<kPdE4m3>()));
}

PagedBlocks paged_blocks(int group) {
  PagedBlocks b;
  b.heads = group <= 8 ? 8 : 16;
  b.count = (group + b.heads - 1) / b.heads;
  return b;
}
size_t paged_part_floats(int head_dim) { return 32 + (size_t)16 * head_dim; }

int paged_decode_kernels(const PagedCache& c) { return c.w ? 2 : 1; }

cudaError_t launch_paged_decode(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, cudaStream_t s) {
  const PagedBlocks b = paged_blocks(c.G);
  const PdWork w{b.heads, b.count, c.part, (int)paged_part_floats(c.D), c.count, c.logits, c.lse2};
  cudaError_t e;
  if (c.cache_type == LTRI_TYPE_E4M3) e = launch_kind<kPdE4m3>(c, r, layer, a, w, c.sms, s);
  else if (c.type == LTRI_TYPE_BF16) e = launch_kind<kPdBf16>(c, r, layer, a, w, c.sms, s);
  else e = launch_kind<kPdFp16>(c, r, layer, a, w, c.sms, s);
  if (e != cudaSuccess || !c.w) return e;
  return launch_chained(k_paged_weights, dim3(c.sms * 4), dim3(kPwThreads), 0, s, c, r, layer, w);
}

}  // namespace ltri
