// Eviction from a caller-owned paged cache by accumulated attention weight.
#include <limits.h>

#include "paged.cuh"

namespace ltri {

constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;

// Order of a slot: larger is kept first.  Protected positions come before every weight, NaN counts as -infinity, and the
// two zeros are equal.
__device__ __forceinline__ unsigned ev_key(float w, bool stays) {
  if (stays) return 0xffffffffu;
  if (w != w) w = -INFINITY;
  const unsigned u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive prefix sum of x over the CTA and the total; s: kEvWarps + 1 ints.
__device__ __forceinline__ int ev_scan(int x, int* s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  int inc = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 31) s[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    int y = s[lane], z = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, z, d);
      if (lane >= d) z += u;
    }
    s[lane] = z - y;
    if (lane == 31) s[32] = z;
  }
  __syncthreads();
  *total = s[32];
  return s[warp] + inc - x;
}

// One CTA per (KV head, row, layer).
__global__ void __launch_bounds__(kEvThreads) k_paged_evict(PagedCache c, PagedRows r, int layer_begin, int budget, int n_sink,
                                                            int recent) {
  __shared__ int s_scan[kEvWarps + 1], s_newest;
  __shared__ unsigned s_hist[256], s_prefix, s_need;
  chain_wait();
  const int head = blockIdx.x, row = blockIdx.y, layer = layer_begin + blockIdx.z;
  const int n = paged_len(c, r, row);
  if (n <= budget) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  auto word = [&](int slot) -> long long {  // -1: no page
    const int page = paged_page(c, r, row, paged_nth(c, slot));
    return page < 0 ? -1 : (long long)paged_word(c, layer, page, head, slot % c.P);
  };
  if (tid == 0) s_newest = INT_MIN, s_prefix = 0, s_need = budget;
  __syncthreads();
  int newest = INT_MIN;
  for (int j = tid; j < n; j += kEvThreads) {
    const long long at = word(j);
    if (at >= 0) newest = max(newest, c.pos[at]);
  }
  atomicMax(&s_newest, newest);
  __syncthreads();
  const long long first_recent = (long long)s_newest - recent;
  auto key = [&](int slot) -> unsigned {
    const long long at = word(slot);
    if (at < 0) return 0u;
    const int pos = c.pos[at];
    return ev_key(c.w[at], pos < n_sink || pos > first_recent);
  };
  // the budget-th largest key, eight bits a pass
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    const unsigned prefix = s_prefix;
    for (int j = tid; j < n; j += kEvThreads) {
      const unsigned x = key(j);
      if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(x >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      unsigned need = s_need;
      int b = 255;
      while (b > 0 && s_hist[b] < need) need -= s_hist[b--];
      s_need = need;
      s_prefix = prefix | (unsigned)b << shift;
    }
    __syncthreads();
  }
  const unsigned cut = s_prefix;
  const int ties = (int)s_need;  // slots of the cut's key that stay: the lowest
  // lists: the i-th slot to be filled in the word of slot budget + i, the i-th that moves in the word of slot i
  int eq0 = 0, hole0 = 0, mover0 = 0;
  for (int base = 0; base < n; base += kEvThreads) {
    const int j = base + tid;
    const unsigned x = j < n ? key(j) : 0u;
    int total;
    const bool eq = j < n && x == cut;
    const int e = eq0 + ev_scan(eq, s_scan, &total);
    eq0 += total;
    const bool kept = j < n && (x > cut || (eq && e < ties));
    const bool hole = j < budget && !kept, mover = j >= budget && kept;
    const int hi = hole0 + ev_scan(hole, s_scan, &total);
    hole0 += total;
    const int mi = mover0 + ev_scan(mover, s_scan, &total);
    mover0 += total;
    if (hole) {
      const long long at = word(budget + hi);
      if (at >= 0) c.list[at] = j;
    }
    if (mover) {
      const long long at = word(mi);
      if (at >= 0) c.list[at] = j;
    }
  }
  __syncthreads();
  for (int i = warp; i < mover0; i += kEvWarps) {
    const long long a0 = word(i), a1 = word(budget + i);
    if (a0 < 0 || a1 < 0) continue;
    const int src = c.list[a0], dst = c.list[a1];
    const int sp = paged_page(c, r, row, paged_nth(c, src)), dp = paged_page(c, r, row, paged_nth(c, dst));
    if (sp < 0 || dp < 0) continue;
    const size_t from = paged_row(c, layer, sp, head, src % c.P), to = paged_row(c, layer, dp, head, dst % c.P);
    for (int b = lane * 16; b < 2 * c.row_bytes; b += 512) {
      unsigned char* base = b < c.row_bytes ? c.k : c.v;
      const int o = b < c.row_bytes ? b : b - c.row_bytes;
      *reinterpret_cast<uint4*>(base + to + o) = *reinterpret_cast<const uint4*>(base + from + o);
    }
    if (lane == 0) {
      const size_t ws = paged_word(c, layer, sp, head, src % c.P), wd = paged_word(c, layer, dp, head, dst % c.P);
      c.w[wd] = c.w[ws];
      c.pos[wd] = c.pos[ws];
    }
  }
}

__global__ void k_paged_lens(PagedCache c, PagedRows r, int* new_lens, int budget) {
  chain_wait();
  const int row = blockIdx.x * blockDim.x + threadIdx.x;
  if (row < r.n) new_lens[row] = min(paged_len(c, r, row), budget);
}

cudaError_t launch_paged_evict(const PagedCache& c, const PagedRows& r, int layer_begin, int layer_count, int* new_lens,
                               int budget, int n_sink, int recent, cudaStream_t s) {
  cudaError_t e = launch_chained(k_paged_evict, dim3(c.Hkv, r.n, layer_count), dim3(kEvThreads), 0, s, c, r, layer_begin, budget,
                                 n_sink, recent);
  if (e != cudaSuccess) return e;
  return launch_chained(k_paged_lens, dim3((r.n + 255) / 256), dim3(256), 0, s, c, r, new_lens, budget);
}

}  // namespace ltri
