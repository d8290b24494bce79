// Slots of ragged rows out of the pages of a caller-owned cache, as dense rows of the model's type.
//
// Bound: HBM, every row is read once and written once.  A lane has up to CHUNKS 16-byte chunks of a token's dense K row and as
// many of its V row on their way; consecutive lanes take consecutive chunks, so both sides move whole rows whatever the order of
// the axes.  Measured: four ragged rows of up to 32768 slots of eight KV heads of 128 out of 4-bit pages, 301 MB read and written,
// 54 to 55 us (5.5 TB/s, 0.86 of the copy rate).
#include "paged_int4.cuh"

namespace ltri {

constexpr int kRdThreads = 256;

// Eight numbers of a row times their scale, as elements of `type` (exactly: they have no more than seven significant bits).
__device__ __forceinline__ uint4 i4_elements(int type, uint32_t w, unsigned scale) {
  const __half s = __ushort_as_half((unsigned short)(scale << 7));
  uint32_t v[4];
  if (type == LTRI_TYPE_FP16) {
    i4_values(v, w, i4_factors(scale * 0x00800080u));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i4_mul(v[i], 0x48004800u);  // (kI4Back)
  } else {
    // four bits below an exponent of 2^7 are 128 + number + 8 in bf16; 136 times a scale has eight significant bits
    const float f = __half2float(s);
    const uint32_t s2 = paged_pack(LTRI_TYPE_BF16, f, f), c2 = paged_pack(LTRI_TYPE_BF16, -136.f * f, -136.f * f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("{\n.reg .b32 t;\nlop3.b32 t, %1, 0x000f000f, %2, 0xEA;\nfma.rn.bf16x2 %0, t, %3, %4;\n}\n"
          : "=r"(v[i])
          : "r"(w >> (4 * i)), "r"(0x43004300u), "r"(s2), "r"(c2));
  }
  // v[i]: elements i and i + 4
  return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632),
                    __byte_perm(v[2], v[3], 0x7632));
}

// x * y as fp32, where inexact the odd one of its two neighbours (rounding to odd: S. Boldo and G. Melquiond, 2008), so that a rounding
// to fewer bits is that of the exact product: it lies on no midpoint that the product does not lie on.  (No slower: 11193
// tokens of eight KV heads of 128 take 18 to 20 us either way.)
__device__ __forceinline__ float mul_odd(float x, float y) {
  const float down = __fmul_rd(x, y), up = __fmul_ru(x, y);
  return __float_as_uint(down) & 1u ? down : up;
}

__device__ __forceinline__ uint4 e4m3_elements(int type, const uint2& x, float scale) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t in = i < 2 ? x.x : x.y;
    const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(in >> (16 * (i & 1)));
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[i] = paged_pack(type, mul_odd(f.x, scale), mul_odd(f.y, scale));
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// BYTES of the cache are 16 bytes of a dense row.
template <int BYTES, int CHUNKS>
__global__ void __launch_bounds__(kRdThreads)
    k_paged_read(PagedCache c, PagedRows r, int layer, PagedRead a, int lanes, int parts) {
  chain_wait();
  const int chunks = c.D / 8, shift = 31 - __clz(chunks), per_token = c.Hkv * chunks;
  // `lanes` of a warp have a part of CHUNKS * lanes chunks of a token
  const int lane = threadIdx.x & 31, sub = lane / lanes, together = 32 / lanes;
  const long long items = a.n_tokens * parts, step = (long long)gridDim.x * (kRdThreads / 32) * together;
  const long long begin = ((long long)blockIdx.x * (kRdThreads / 32) + threadIdx.x / 32) * together + sub;
  for (long long item = begin; item < items; item += step) {
    const long long tok = parts == 1 ? item : item / parts;
    const int in0 = (int)(item - tok * parts) * (CHUNKS * lanes) + lane % lanes;
    // the last row that starts at or in front of the token
    int lo = 0, hi = r.n;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.starts[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    if (lo >= r.n || a.starts[lo] > tok) continue;
    const int row = lo, n = paged_len(c, r, row);
    const long long slot = (a.first ? (long long)a.first[row] - a.starts[row] : (long long)n - a.starts[row + 1]) + tok;
    int page = -1, place = 0;
    if (slot >= 0 && slot < n) {
      const int in_row = paged_nth(c, (int)slot);
      page = paged_page(c, r, row, in_row);
      place = (int)slot - in_row * c.P;
    } else {
      paged_status(c, row);
    }
    const size_t at0 = page < 0 ? 0 : paged_row(c, layer, page, 0, place);
    const size_t word0 = page < 0 ? 0 : paged_word(c, layer, page, 0, place);
    uint4 x[2][CHUNKS];
    unsigned sc[2][CHUNKS];
    float f[2][CHUNKS];
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int in = in0 + u * lanes, head = in >> shift, ch = in & (chunks - 1);
      const size_t at = at0 + head * c.hs + ch * BYTES;
      const unsigned char* scales = c.sc + (word0 + (unsigned)head * (unsigned)c.P) * (c.D / 16) + ch / 4;
#pragma unroll
      for (int of_v = 0; of_v < 2; ++of_v) {
        x[of_v][u] = make_uint4(0u, 0u, 0u, 0u);
        sc[of_v][u] = 0u;
        f[of_v][u] = 0.f;
        if (in >= per_token || page < 0 || !(of_v ? a.v : a.k)) continue;
        const unsigned char* from = (of_v ? c.v : c.k) + at;
        if (BYTES == 16) x[of_v][u] = __ldcs(reinterpret_cast<const uint4*>(from));
        if (BYTES == 8) {
          const uint2 y = __ldcs(reinterpret_cast<const uint2*>(from));
          x[of_v][u].x = y.x;
          x[of_v][u].y = y.y;
          f[of_v][u] = (of_v ? c.vs : c.ks)[head];
        }
        if (BYTES == 4) {
          x[of_v][u].x = __ldcs(reinterpret_cast<const uint32_t*>(from));
          sc[of_v][u] = scales[of_v ? c.D / kI4Block : 0];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int in = in0 + u * lanes;
      if (in >= per_token) continue;
#pragma unroll
      for (int of_v = 0; of_v < 2; ++of_v) {
        unsigned char* out = of_v ? a.v : a.k;
        if (!out) continue;
        uint4 y = x[of_v][u];
        if (BYTES == 8) y = e4m3_elements(c.type, make_uint2(y.x, y.y), f[of_v][u]);
        if (BYTES == 4) y = i4_elements(c.type, y.x, sc[of_v][u]);
        __stcs(reinterpret_cast<uint4*>(out + tok * a.stride + in * 16), y);
      }
    }
  }
}

cudaError_t launch_paged_read(const PagedCache& c, const PagedRows& r, int layer, const PagedRead& a, cudaStream_t s) {
  const int per_token = c.Hkv * (c.D / 8), lanes = per_token <= 8 ? 8 : per_token <= 16 ? 16 : 32;
  const bool few = a.n_tokens * per_token <= c.sms * 2048ll;
  const int chunks = few ? 1 : 4, parts = (per_token + chunks * lanes - 1) / (chunks * lanes);
  const long long per_block = (kRdThreads / 32) * (32 / lanes), blocks = (a.n_tokens * parts + per_block - 1) / per_block;
  const int grid = (int)(blocks < c.sms * 16ll ? blocks : c.sms * 16ll);
  const int bytes = 16 * c.row_bytes / (2 * c.D);
  const auto kernel = bytes == 16 ? (few ? k_paged_read<16, 1> : k_paged_read<16, 4>)
                      : bytes == 8 ? (few ? k_paged_read<8, 1> : k_paged_read<8, 4>)
                                   : (few ? k_paged_read<4, 1> : k_paged_read<4, 4>);
  return launch_chained(kernel, dim3(grid), dim3(kRdThreads), 0, s, c, r, layer, a, lanes, parts);
}

}  // namespace ltri
