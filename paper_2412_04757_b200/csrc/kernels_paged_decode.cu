// Attention of one new token per row over a caller-owned paged cache.
#include "paged.cuh"

namespace ltri {

constexpr int kPdThreads = 256;
constexpr int kPdWarps = kPdThreads / 32;

// Element pair (2 lane-owned neighbours) of a cached row as fp32.
__device__ __forceinline__ float2 pd_pair(const PagedCache& c, const unsigned char* row, int pair) {
  if (c.cache_type == LTRI_TYPE_E4M3) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(reinterpret_cast<const __nv_fp8x2_storage_t*>(row)[pair], __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
  }
  return paged_unpack(c.type, reinterpret_cast<const uint32_t*>(row)[pair]);
}

template <int D>
__global__ void __launch_bounds__(kPdThreads) k_paged_decode(PagedCache c, PagedRows r, int layer, PagedStep a) {
  constexpr int kPairs = D / 64;  // element pairs of a lane
  __shared__ float s_m[kPdWarps], s_l[kPdWarps], s_o[kPdWarps][D], s_lse[64];
  chain_wait();
  const int head = blockIdx.x, row = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int n = paged_len(c, r, row);
  const float ks = c.ks ? c.ks[head] : 1.f, vs = c.vs ? c.vs[head] : 1.f;
  if (a.k && n > 0) {  // the new token's rows
    const int slot = n - 1, page = paged_page(c, r, row, slot / c.P);
    if (page >= 0) {
      const size_t at = paged_row(c, layer, page, head, slot % c.P);
      for (int i = threadIdx.x; i < D / 4; i += kPdThreads) {
        const int ch = i % (D / 8);
        const bool is_v = i >= D / 8;
        const uint4 x = *reinterpret_cast<const uint4*>((is_v ? a.v : a.k) + row * a.kv_stride + head * D * 2 + ch * 16);
        unsigned char* to = (is_v ? c.v : c.k) + at;
        if (c.cache_type == LTRI_TYPE_E4M3) *reinterpret_cast<uint2*>(to + ch * 8) = paged_quantise(c.type, x, is_v ? vs : ks);
        else *reinterpret_cast<uint4*>(to + ch * 16) = x;
      }
      if (c.w && threadIdx.x == 0) {
        const size_t word = paged_word(c, layer, page, head, slot % c.P);
        c.w[word] = 0.f;
        c.pos[word] = a.row_pos ? a.row_pos[row] : slot;
      }
    }
    __syncthreads();
  }
  for (int g = 0; g < c.G; ++g) {
    const int h = head * c.G + g;
    float2 q[kPairs], o[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      q[i] = paged_unpack(c.type, reinterpret_cast<const uint32_t*>(a.q + row * a.q_stride + (size_t)h * D * 2)[i * 32 + lane]);
      o[i] = make_float2(0.f, 0.f);
    }
    auto logit = [&](size_t at) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 f = pd_pair(c, c.k + at, i * 32 + lane);
        x = fmaf(q[i].x, f.x, fmaf(q[i].y, f.y, x));
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      return x * c.scale * ks;
    };
    float m = -INFINITY, l = 0.f;
    for (int slot = warp; slot < n; slot += kPdWarps) {
      const int page = paged_page(c, r, row, slot / c.P);
      if (page < 0) continue;
      const size_t at = paged_row(c, layer, page, head, slot % c.P);
      const float x = logit(at), mn = fmaxf(m, x), al = mn == -INFINITY ? 0.f : exp2f(m - mn);
      const float p = mn == -INFINITY ? 0.f : exp2f(x - mn);
      l = l * al + p;
      m = mn;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 f = pd_pair(c, c.v + at, i * 32 + lane);
        o[i].x = o[i].x * al + p * f.x;
        o[i].y = o[i].y * al + p * f.y;
      }
    }
    if (lane == 0) s_m[warp] = m, s_l[warp] = l;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      s_o[warp][(i * 32 + lane) * 2] = o[i].x;
      s_o[warp][(i * 32 + lane) * 2 + 1] = o[i].y;
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
    for (int w = 0; w < kPdWarps; ++w) top = fmaxf(top, s_m[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < kPdWarps; ++w) sum += s_l[w] * exp2f(s_m[w] - ref);
    for (int i = threadIdx.x; i < D / 2; i += kPdThreads) {
      float x = 0.f, y = 0.f;
      for (int w = 0; w < kPdWarps; ++w) {
        const float e = exp2f(s_m[w] - ref);
        x += e * s_o[w][2 * i];
        y += e * s_o[w][2 * i + 1];
      }
      const float inv = sum > 0.f ? vs / sum : 0.f;
      reinterpret_cast<uint32_t*>(a.out + ((size_t)row * c.Hq + h) * D * 2)[i] = paged_pack(c.type, x * inv, y * inv);
    }
    if (threadIdx.x == 0) {
      s_lse[g] = ref + log2f(sum);
      if (a.lse) a.lse[(size_t)row * c.Hq + h] = sum > 0.f ? (ref + log2f(sum)) * 0.69314718055994531f : -INFINITY;
    }
    __syncthreads();
  }
  if (!c.w) return;
  for (int slot = warp; slot < n; slot += kPdWarps) {
    const int page = paged_page(c, r, row, slot / c.P);
    if (page < 0) continue;
    const size_t at = paged_row(c, layer, page, head, slot % c.P);
    float p = 0.f;
    for (int g = 0; g < c.G; ++g) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 f = pd_pair(c, c.k + at, i * 32 + lane);
        const float2 q = paged_unpack(
            c.type, reinterpret_cast<const uint32_t*>(a.q + row * a.q_stride + (size_t)(head * c.G + g) * D * 2)[i * 32 + lane]);
        x = fmaf(q.x, f.x, fmaf(q.y, f.y, x));
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      p += exp2f(x * c.scale * ks - s_lse[g]);
    }
    if (lane == 0) {
      float* w = c.w + paged_word(c, layer, page, head, slot % c.P);
      *w = *w * c.decay + p;
    }
  }
}

cudaError_t prepare_paged(const PagedCache&) { return cudaSuccess; }

cudaError_t launch_paged_decode(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, cudaStream_t s) {
  const dim3 grid(c.Hkv, r.n), block(kPdThreads);
  if (c.D == 64) return launch_chained(k_paged_decode<64>, grid, block, 0, s, c, r, layer, a);
  if (c.D == 128) return launch_chained(k_paged_decode<128>, grid, block, 0, s, c, r, layer, a);
  return launch_chained(k_paged_decode<256>, grid, block, 0, s, c, r, layer, a);
}

}  // namespace ltri
