// Shared declarations of the caller-owned paged K/V cache: the device-side view of a handle and the launch wrappers of its
// kernel files (kernels_paged_*.cu).
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "../../include/ltri.h"
#include "common.cuh"

namespace ltri {

// Device-side view of one handle.  Passed to kernels by value.
struct PagedCache {
  int Hq, Hkv, G, D, P;
  // slot / P = slot * p_mul >> p_shift for slots below 2^31: p_mul = floor(2^p_shift / P) + 1 with p_shift = 31 + ceil(log2 P),
  // so that slot * (p_mul * P - 2^p_shift) < 2^p_shift
  unsigned p_mul;
  int p_shift;
  int type, cache_type;
  int row_bytes;                // bytes of a cached row
  int n_pages;
  long long ls, ps, hs, ts;     // layer, page, head and place strides of the pages, bytes
  float scale;                  // softmax_scale * log2(e)
  float decay;
  unsigned char *k, *v;
  const float *ks, *vs;         // per KV head, or null
  unsigned char* sc;            // [L][n_pages][Hkv][P][2][D / 32], K's and V's scales of 4-bit rows, or null
  float* w;                     // [L][n_pages][Hkv][P], or null
  int* pos;
  int* status;                  // [4]
  int* list;                    // [L][n_pages][Hkv][P]: an eviction's moves, in the words of the unit's own slots
  float* part;                  // [sms][2][paged_part_floats]: partial sums of units that several CTAs share
  float* lead;                  // [sms][kPagedWarps][paged_part_floats]: of units that several warps share
  int* count;                   // [max_rows][Hkv][blocks of heads]: CTAs of the unit that have finished; zero between calls
  float* logits;                // [n_pages][Hkv][P][paged_even(G)], with weights: a decode call's logits
  float* lse2;                  // [max_rows][Hq], with weights: their sums, log2
  int* seen;                    // [max_rows]: CTAs of an eviction that have read the row's length; zero between calls
  int sms, evict_cluster;
  long long wait_limit;         // of an attend call's waits, SM cycles
  int held;                     // tests: bit 0: K rows, bit 1: V rows never arrive there
};

// One call's rows.
struct PagedRows {
  const int* table;
  long long table_stride;
  int cap;                      // slots that the table has columns for
  const int* lens;
  int n;
};

struct PagedAppend {
  const int* starts;
  long long n_tokens;
  const unsigned char *k, *v;
  long long stride;             // bytes between tokens
  const int* row_pos;
  const float* weights;
};

struct PagedRead {
  const int *starts, *first;
  long long n_tokens;
  unsigned char *k, *v;         // either may be null
  long long stride;             // bytes between tokens
};

struct PagedQueries {
  const int* starts;
  long long n_tokens;
  const unsigned char* q;
  long long q_stride;           // bytes between tokens
  unsigned char* out;
  float* lse;
};

struct PagedStep {
  const unsigned char *q, *k, *v;
  long long q_stride, kv_stride;  // bytes between rows
  const int* row_pos;
  unsigned char* out;
  float* lse;
};

// Query heads of a KV head in blocks that the attention kernel takes at a time.
struct PagedBlocks {
  int heads, count;
};
PagedBlocks paged_blocks(int group);
__host__ __device__ constexpr int paged_even(int x) { return (x + 1) & ~1; }
size_t paged_part_floats(int group, int head_dim);  // partial sums of one block
constexpr int kPagedWarps = 16;                     // of an attention CTA, at most
int paged_decode_kernels(const PagedCache& c);  // launches of a decode call

// (for the handle's own type and head_dim)
cudaError_t prepare_paged(const PagedCache& c);
cudaError_t prepare_paged_evict();
cudaError_t prepare_paged_attend(const PagedCache& c);
size_t paged_attend_workspace(const PagedCache& c, long long n_tokens, long long n_rows);
cudaError_t launch_paged_attend(const PagedCache& c, const PagedRows& r, int layer, const PagedQueries& a, unsigned char* workspace,
                                cudaStream_t s);
int paged_evict_cluster();
cudaError_t launch_paged_append(const PagedCache& c, const PagedRows& r, int layer, const PagedAppend& a, cudaStream_t s);
cudaError_t launch_paged_read(const PagedCache& c, const PagedRows& r, int layer, const PagedRead& a, cudaStream_t s);
cudaError_t launch_paged_decode(const PagedCache& c, const PagedRows& r, int layer, const PagedStep& a, cudaStream_t s);
cudaError_t launch_paged_evict(const PagedCache& c, const PagedRows& r, int layer_begin, int layer_count, int* new_lens,
                               int budget, int n_sink, int recent, cudaStream_t s);

#ifdef __CUDACC__
// (out of line: the checks are everywhere, and never taken)
static __device__ __noinline__ void paged_status(const PagedCache& c, int detail) {
  if (atomicCAS(&c.status[0], 0, (int)LTRI_EDEVICE) == 0) c.status[1] = detail;
}

// Adds one; what this thread has seen or written is visible to whoever finds it added.
__device__ __forceinline__ int paged_arrive(int* count) {
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(count) : "memory");
  return before;
}

// Slots of row r: 0 (and the status word) where the length says more than the table can hold.
__device__ __forceinline__ int paged_len(const PagedCache& c, const PagedRows& r, int row) {
  const int n = r.lens[row];
  if ((unsigned)n <= (unsigned)r.cap) return n;
  paged_status(c, row);
  return 0;
}

// Which of its row's pages a slot lies in.
__device__ __forceinline__ int paged_nth(const PagedCache& c, int slot) {
  return (int)(((unsigned long long)(unsigned)slot * c.p_mul) >> c.p_shift);
}

// The nth page of a row, or -1 (and the status word) where the table names none.
__device__ __forceinline__ int paged_page(const PagedCache& c, const PagedRows& r, int row, int nth) {
  const int page = r.table[row * r.table_stride + nth];
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  paged_status(c, row);
  return -1;
}

// Index of a slot's word in weights, positions and lists.
__device__ __forceinline__ size_t paged_word(const PagedCache& c, int layer, int page, int head, int place) {
  return (((size_t)layer * c.n_pages + page) * c.Hkv + head) * c.P + place;
}

__device__ __forceinline__ size_t paged_row(const PagedCache& c, int layer, int page, int head, int place) {
  return layer * c.ls + page * c.ps + head * c.hs + place * c.ts;  // (the strides are 64-bit)
}

// Two fp32 values as elements of `type`, the first in the lower half.
__device__ __forceinline__ uint32_t paged_pack(int type, float a, float b) {
  if (type == LTRI_TYPE_BF16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  const __half2 x = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float2 paged_unpack(int type, uint32_t x) {
  if (type == LTRI_TYPE_BF16) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

// Eight elements of `type` as e4m3: the nearest value to element / scale (fp32's quotient), ties to even, clamped to the
// largest.  The quotient lies within 2^-22 of the product with 1 / scale; where 2^-21 to either side rounds to the same value,
// as it does unless the quotient almost is a midpoint of two, no division is needed.  (Appending 22700 tokens of eight KV heads
// of 128: 34 us, with eight divisions a chunk 44.)
__device__ __forceinline__ uint2 paged_quantise(int type, const uint4& x, float scale) {
  const uint32_t in[4] = {x.x, x.y, x.z, x.w};
  uint32_t out[2] = {0u, 0u}, other[2] = {0u, 0u};
  const float r = __fdiv_rn(1.f, scale), lo = r * (1.f - 0x1p-21f), hi = r * (1.f + 0x1p-21f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = paged_unpack(type, in[i]);
    const float2 a = make_float2(f.x * lo, f.y * lo), b = make_float2(f.x * hi, f.y * hi);
    out[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3) << (16 * (i & 1));
    other[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(b, __NV_SATFINITE, __NV_E4M3) << (16 * (i & 1));
  }
  const bool normal = fabsf(lo) >= 0x1p-126f && fabsf(hi) <= 3.0e38f;
  if (normal && out[0] == other[0] && out[1] == other[1]) return make_uint2(out[0], out[1]);
  out[0] = out[1] = 0u;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    float2 f = paged_unpack(type, i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w);
    f.x = __fdiv_rn(f.x, scale);
    f.y = __fdiv_rn(f.y, scale);
    const uint32_t y = (uint32_t)__nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3) << (16 * (i & 1));
    if (i < 2) out[0] |= y;
    else out[1] |= y;
  }
  return make_uint2(out[0], out[1]);
}
#endif

}  // namespace ltri
