// Slots of ragged rows out of the pages of a caller-owned cache, as dense rows of the model's type.
//
// Bound: HBM, every row is read once and written once.  A lane has up to CHUNKS 16-byte chunks of a token's dense K row and as
// many of its V row on their way; consecutive lanes take consecutive chunks, so both sides move whole rows whatever the order of
// the axes.
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
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"((w >> (4 * i) & 0x000f000fu) | 0x43004300u), "r"(s2), "r"(c2));
  }
  // v[i]: elements i and i + 4
  return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632),
                    __byte_perm(v[2], v[3], 0x7632));
}

__device__ __forceinline__ uint4 e4m3_elements(int type, const uint2& x, float scale) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t in = i < 2 ? x.x : x.y;
    const __nv_fp8x2_storage_t two = (__nv_fp8x2_storage_t)(in >> (16 * (i & 1)));
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[i] = paged_pack(type, f.x * scale, f.y * scale);
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
#pragma unroll
    for (int of_v = 0; of_v < 2; ++of_v) {
      unsigned char* out = of_v ? a.v : a.k;
      if (!out) continue;
      const unsigned char* pages = of_v ? c.v : c.k;
      const float* scales = of_v ? c.vs : c.ks;
      uint4 x[CHUNKS];
      unsigned sc[CHUNKS];
      float f[CHUNKS];
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) {
        const int in = in0 + u * lanes, head = in >> shift, ch = in & (chunks - 1);
        x[u] = make_uint4(0u, 0u, 0u, 0u);
        sc[u] = 0u;
        f[u] = 0.f;
        if (in >= per_token || page < 0) continue;
        const unsigned char* from = pages + paged_row(c, layer, page, head, place) + ch * BYTES;
        if (BYTES == 16) x[u] = __ldcs(reinterpret_cast<const uint4*>(from));
        if (BYTES == 8) {
          const uint2 y = __ldcs(reinterpret_cast<const uint2*>(from));
          x[u].x = y.x;
          x[u].y = y.y;
          f[u] = scales[head];
        }
        if (BYTES == 4) {
          x[u].x = __ldcs(reinterpret_cast<const uint32_t*>(from));
          sc[u] = c.sc[(paged_word(c, layer, page, head, place) * 2 + of_v) * (c.D / kI4Block) + ch / 4];
        }
      }
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) {
        const int in = in0 + u * lanes;
        if (in >= per_token) continue;
        uint4 y = x[u];
        if (BYTES == 8) y = e4m3_elements(c.type, make_uint2(x[u].x, x[u].y), f[u]);
        if (BYTES == 4) y = i4_elements(c.type, x[u].x, sc[u]);
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
