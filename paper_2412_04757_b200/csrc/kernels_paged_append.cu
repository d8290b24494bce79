// Rows of ragged prompts into the pages of a caller-owned cache.
//
// Bound: HBM, every row is read once and written once.  A thread takes 16 bytes of a K row and the same 16 of the V row;
// consecutive threads take consecutive chunks of a token, so both sides move whole rows whatever the order of the axes.
#include "paged.cuh"

namespace ltri {

constexpr int kAppThreads = 256;

__global__ void __launch_bounds__(kAppThreads) k_paged_append(PagedCache c, PagedRows r, int layer, PagedAppend a) {
  chain_wait();
  const int chunks = c.D / 8;  // of a row
  const long long per_token = (long long)c.Hkv * chunks;
  const long long total = a.n_tokens * per_token;
  for (long long i = blockIdx.x * (long long)kAppThreads + threadIdx.x; i < total; i += (long long)gridDim.x * kAppThreads) {
    const long long tok = i / per_token;
    const int in = (int)(i - tok * per_token), head = in / chunks, ch = in - head * chunks;
    // the last row that starts at or in front of the token
    int lo = 0, hi = r.n;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.starts[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    if (lo >= r.n || a.starts[lo] > tok) continue;
    const int row = lo, nth = (int)(tok - a.starts[row]);
    const long long slot = (long long)paged_len(c, r, row) - (a.starts[row + 1] - a.starts[row]) + nth;
    if (slot < 0) {
      paged_status(c, row);
      continue;
    }
    const int in_row = paged_nth(c, (int)slot), page = paged_page(c, r, row, in_row), place = (int)slot - in_row * c.P;
    if (page < 0) continue;
    const uint4 kx = *reinterpret_cast<const uint4*>(a.k + tok * a.stride + in * 16);
    const uint4 vx = *reinterpret_cast<const uint4*>(a.v + tok * a.stride + in * 16);
    const size_t at = paged_row(c, layer, page, head, place);
    if (c.cache_type == LTRI_TYPE_E4M3) {
      *reinterpret_cast<uint2*>(c.k + at + ch * 8) = paged_quantise(c.type, kx, c.ks[head]);
      *reinterpret_cast<uint2*>(c.v + at + ch * 8) = paged_quantise(c.type, vx, c.vs[head]);
    } else {
      *reinterpret_cast<uint4*>(c.k + at + ch * 16) = kx;
      *reinterpret_cast<uint4*>(c.v + at + ch * 16) = vx;
    }
    if (c.w && ch == 0) {
      const size_t word = paged_word(c, layer, page, head, place);
      c.w[word] = a.weights ? a.weights[tok * c.Hkv + head] : 0.f;
      c.pos[word] = a.row_pos ? a.row_pos[row] + nth : (int)slot;
    }
  }
}

cudaError_t launch_paged_append(const PagedCache& c, const PagedRows& r, int layer, const PagedAppend& a, cudaStream_t s) {
  const long long total = a.n_tokens * c.Hkv * (c.D / 8);
  const long long blocks = (total + kAppThreads - 1) / kAppThreads;
  const int grid = (int)(blocks < c.sms * 8ll ? blocks : c.sms * 8ll);
  return launch_chained(k_paged_append, dim3(grid), dim3(kAppThreads), 0, s, c, r, layer, a);
}

}  // namespace ltri
