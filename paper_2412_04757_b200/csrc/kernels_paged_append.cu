// Rows of ragged prompts into the pages of a caller-owned cache.
//
// Bound: HBM, every row is read once and written once.  A warp's lanes ask for up to CHUNKS 16-byte chunks each of a token's K
// rows and as many of its V rows before they look up the token's row, slot and page, which the loads do not depend on.
// Consecutive lanes take consecutive chunks, so both sides move whole rows whatever the order of the axes.  (A chunk a thread,
// behind the lookups: 38 us for 22700 tokens of eight KV heads, 33 so.)
#include "paged.cuh"

namespace ltri {

constexpr int kAppThreads = 256;

template <int CHUNKS>
__global__ void __launch_bounds__(kAppThreads)
    k_paged_append(PagedCache c, PagedRows r, int layer, PagedAppend a, int lanes, int parts) {
  chain_wait();
  const int chunks = c.D / 8, shift = 31 - __clz(chunks), per_token = c.Hkv * chunks;
  // `lanes` of a warp have a part of CHUNKS * lanes chunks of a token
  const int lane = threadIdx.x & 31, sub = lane / lanes, together = 32 / lanes;
  const long long items = a.n_tokens * parts, step = (long long)gridDim.x * (kAppThreads / 32) * together;
  const long long begin = ((long long)blockIdx.x * (kAppThreads / 32) + threadIdx.x / 32) * together + sub;
  for (long long item = begin; item < items; item += step) {
    const long long tok = parts == 1 ? item : item / parts;
    const int in0 = (int)(item - tok * parts) * (CHUNKS * lanes) + lane % lanes;
    uint4 kx[CHUNKS], vx[CHUNKS];
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int in = in0 + u * lanes;
      if (in < per_token) {
        kx[u] = __ldcs(reinterpret_cast<const uint4*>(a.k + tok * a.stride + in * 16));
        vx[u] = __ldcs(reinterpret_cast<const uint4*>(a.v + tok * a.stride + in * 16));
      }
    }
    // the last row that starts at or in front of the token; the next one has been seen to start behind it, so the slot lies
    // below the row's length even if the starts do not ascend
    int lo = 0, hi = r.n;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.starts[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    if (lo >= r.n || a.starts[lo] > tok) continue;
    const int row = lo;
    const long long nth = tok - a.starts[row], slot = (long long)paged_len(c, r, row) - a.starts[row + 1] + tok;
    if (slot < 0) {
      paged_status(c, row);
      continue;
    }
    const int in_row = paged_nth(c, (int)slot), page = paged_page(c, r, row, in_row), place = (int)slot - in_row * c.P;
    if (page < 0) continue;
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int in = in0 + u * lanes, head = in >> shift, ch = in & (chunks - 1);
      if (in >= per_token) continue;
      const size_t at = paged_row(c, layer, page, head, place);
      if (c.cache_type == LTRI_TYPE_E4M3) {
        *reinterpret_cast<uint2*>(c.k + at + ch * 8) = paged_quantise(c.type, kx[u], c.ks[head]);
        *reinterpret_cast<uint2*>(c.v + at + ch * 8) = paged_quantise(c.type, vx[u], c.vs[head]);
      } else {
        *reinterpret_cast<uint4*>(c.k + at + ch * 16) = kx[u];
        *reinterpret_cast<uint4*>(c.v + at + ch * 16) = vx[u];
      }
      if (c.w && ch == 0) {
        const size_t word = paged_word(c, layer, page, head, place);
        c.w[word] = a.weights ? a.weights[tok * c.Hkv + head] : 0.f;
        c.pos[word] = a.row_pos ? a.row_pos[row] + (int)nth : (int)slot;
      }
    }
  }
}

cudaError_t launch_paged_append(const PagedCache& c, const PagedRows& r, int layer, const PagedAppend& a, cudaStream_t s) {
  const int per_token = c.Hkv * (c.D / 8), lanes = per_token <= 8 ? 8 : per_token <= 16 ? 16 : 32;
  // calls that do not fill the GPU's threads take a chunk a lane (9 prompts of 1097 tokens, four KV heads, 8-bit pages: 3.6 us,
  // with four chunks 4.5), calls that do have four of each on their way
  const bool few = a.n_tokens * per_token <= c.sms * 2048ll;
  const int chunks = few ? 1 : 4, parts = (per_token + chunks * lanes - 1) / (chunks * lanes);
  const long long per_block = (kAppThreads / 32) * (32 / lanes), blocks = (a.n_tokens * parts + per_block - 1) / per_block;
  const int grid = (int)(blocks < c.sms * 16ll ? blocks : c.sms * 16ll);
  const auto kernel = few ? k_paged_append<1> : k_paged_append<4>;
  return launch_chained(kernel, dim3(grid), dim3(kAppThreads), 0, s, c, r, layer, a, lanes, parts);
}

}  // namespace ltri
