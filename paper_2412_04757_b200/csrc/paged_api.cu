// C ABI of the caller-owned paged K/V cache: checks of the arguments, the workspace's layout and the launches.
#include <cmath>
#include <new>

#include "paged.cuh"

using namespace ltri;

struct ltri_paged {
  ltri_paged_params p;
  PagedCache c;
  int device = 0;
  int blocks = 1;  // of a KV head's query heads
  int last_cuda = 0;
  cudaError_t attend = cudaSuccess;  // of its kernels' preparation: what its calls end with
  int64_t launches = 0;
};

namespace {

constexpr int64_t kPagedMaxTokens = 1 << 24;  // of an attend call: query rows of a KV head are counted in 32 bits
// Upper bound of any wait of an attend call, in SM cycles (about ten seconds: a CTA's longest run of tiles lies far below)
constexpr long long kPagedWaitLimit = 20000000000ll;
constexpr int kPagedMaxSms = 256;  // CTAs that a decode call can have partial sums of

int element_bits(int type) { return type == LTRI_TYPE_INT4 ? 4 : type == LTRI_TYPE_E4M3 ? 8 : 16; }

bool aligned(const void* p, uintptr_t a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool validate(const ltri_paged_params* p) {
  if (!p) return false;
  if (p->n_layers < 1 || p->n_layers > 65535 || p->n_kv_heads < 1 || p->n_kv_heads > 65535 || p->n_q_heads < 1) return false;
  if (p->n_q_heads % p->n_kv_heads || p->n_q_heads / p->n_kv_heads > 64) return false;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return false;
  if (p->type != LTRI_TYPE_BF16 && p->type != LTRI_TYPE_FP16) return false;
  if (p->cache_type != p->type && p->cache_type != LTRI_TYPE_E4M3 && p->cache_type != LTRI_TYPE_INT4) return false;
  if (p->page_tokens < 1 || p->page_tokens > 65536 || p->max_rows < 1 || p->max_rows > 65535) return false;
  if (p->n_pages < 1 || p->n_pages > 0x7fffffffll || p->n_pages * p->page_tokens > (1ll << 40)) return false;
  const long long bits = element_bits(p->cache_type);
  // an axis of one entry may have any stride; the others keep 16-byte chunks aligned and rows apart from each other
  const struct { long long n, stride; } axes[4] = {{p->n_layers, p->layer_stride}, {p->n_pages, p->page_stride},
                                                   {p->n_kv_heads, p->head_stride}, {p->page_tokens, p->token_stride}};
  double extent = 0.0;  // bytes; far from where 64 bits end, as are the workspace's
  for (const auto& a : axes) {
    if (a.n == 1) continue;
    if (a.stride < p->head_dim || a.stride > (1ll << 42) || a.stride * bits % 128) return false;
    extent += (double)(a.n - 1) * (double)a.stride * (double)bits / 8.0;
  }
  if (extent > 0x1p56 || (double)p->n_layers * (double)p->n_pages * p->page_tokens * p->n_kv_heads > 0x1p48) return false;
  if (!std::isfinite(p->softmax_scale) || p->softmax_scale < 0.f) return false;
  if (!(p->weight_decay >= 0.f && p->weight_decay <= 1.f)) return false;
  return true;
}

// Carves the workspace; returns its size.  The status word and the counts come first and start at zero.
size_t layout(const ltri_paged_params& p, int sms, PagedCache* c, unsigned char* base, size_t* zeroed) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* at = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  const PagedBlocks b = paged_blocks(p.n_q_heads / p.n_kv_heads);
  const size_t slots = (size_t)p.n_pages * p.n_kv_heads * p.page_tokens;
  unsigned char* status = take(256);
  unsigned char* count = take((size_t)p.max_rows * p.n_kv_heads * b.count * sizeof(int));
  unsigned char* seen = take((size_t)p.max_rows * sizeof(int));
  if (zeroed) *zeroed = off;
  const size_t part_bytes = paged_part_floats(p.n_q_heads / p.n_kv_heads, p.head_dim) * sizeof(float);
  unsigned char *part = take(sms * 2 * part_bytes), *lead = take(sms * kPagedWarps * part_bytes);
  unsigned char *list = nullptr, *logits = nullptr, *lse2 = nullptr;
  if (p.weights) {
    list = take(p.n_layers * slots * sizeof(int));
    logits = take(slots * paged_even(p.n_q_heads / p.n_kv_heads) * sizeof(float));
    lse2 = take((size_t)p.max_rows * p.n_q_heads * sizeof(float));
  }
  if (c) {
    c->status = reinterpret_cast<int*>(status);
    c->count = reinterpret_cast<int*>(count);
    c->seen = reinterpret_cast<int*>(seen);
    c->part = reinterpret_cast<float*>(part);
    c->lead = reinterpret_cast<float*>(lead);
    c->list = reinterpret_cast<int*>(list);
    c->logits = reinterpret_cast<float*>(logits);
    c->lse2 = reinterpret_cast<float*>(lse2);
  }
  return off;
}

// The handle's device for the length of a call.
struct OnDevice {
  int before = -1;
  bool ok = true;
  explicit OnDevice(int device) {
    int now = -1;
    if (cudaGetDevice(&now) != cudaSuccess) ok = false;
    else if (now != device) {
      before = now;
      ok = cudaSetDevice(device) == cudaSuccess;
    }
  }
  ~OnDevice() {
    if (before >= 0) cudaSetDevice(before);
  }
};

int done(ltri_paged* c, cudaError_t e, int kernels) {
  if (e != cudaSuccess) {
    cudaGetLastError();
    c->last_cuda = (int)e;
    return LTRI_ECUDA;
  }
  c->launches += kernels;
  return LTRI_OK;
}

// The arguments that every call has: LTRI_OK or the error.
int check_rows(const ltri_paged* c, const int32_t* table, int table_pages, int64_t table_stride, const int32_t* lens,
               int n_rows, PagedRows* r) {
  if (!aligned(table, 4) || !aligned(lens, 4) || n_rows < 1 || table_pages < 1) return LTRI_EINVAL;
  if (table_stride < 0 || (n_rows > 1 && table_stride < table_pages)) return LTRI_EINVAL;
  if (n_rows > c->p.max_rows) return LTRI_ECAPACITY;
  // the kernels count the 16-slot tiles of all rows in 32 bits, and a row's slots with a stride of theirs behind its end
  const int64_t cap = (int64_t)table_pages * c->p.page_tokens;
  const int64_t units = (int64_t)c->p.n_kv_heads * c->blocks;
  if (cap > 0x7fff0000ll || (cap / 16 + 1) * n_rows > (1ll << 30) / units) return LTRI_ECAPACITY;
  *r = PagedRows{table, table_stride, (int)cap, lens, n_rows};
  return LTRI_OK;
}

// Bytes between rows of `heads` heads; 0: not allowed.
long long row_stride(const ltri_paged* c, int64_t stride, int heads) {
  const long long dense = (long long)heads * c->p.head_dim;
  if (stride == 0) return dense * 2;
  if (stride < dense || stride > (1ll << 42) || stride % 8) return 0;
  return stride * 2;
}

// Whether `bytes` bytes at a meet one of n rows of `row` bytes at b, `stride` apart.
bool meets(const void* a, long long bytes, const void* b, long long n, long long row, long long stride) {
  const long long d = (long long)(reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b));  // (addresses have 57 bits)
  const long long first = d < row ? 0 : (d - row) / stride + 1;  // the first row that ends behind a
  return first < n && first * stride < d + bytes;
}

// block_scales: 4-bit pages' (not looked at beside others).
int create(const ltri_paged_params* p, uint8_t* block_scales, cudaStream_t s, ltri_paged** out) {
  if (!aligned(p->k_pages, 16) || !aligned(p->v_pages, 16) || !aligned(p->workspace, 256)) return LTRI_EINVAL;
  const bool scaled = p->cache_type == LTRI_TYPE_E4M3;
  if (scaled ? !aligned(p->k_scale, 4) || !aligned(p->v_scale, 4) : p->k_scale || p->v_scale) return LTRI_EINVAL;
  if (!p->weights != !p->positions) return LTRI_EINVAL;
  if (p->weights && (!aligned(p->weights, 4) || !aligned(p->positions, 4))) return LTRI_EINVAL;
  if (p->workspace_bytes < ltri_paged_workspace_bytes(p)) return LTRI_ECAPACITY;
  ltri_paged* c = new (std::nothrow) ltri_paged();
  if (!c) return LTRI_ECAPACITY;
  c->p = *p;
  c->blocks = paged_blocks(p->n_q_heads / p->n_kv_heads).count;
  PagedCache& d = c->c;
  d = PagedCache{};
  size_t zeroed = 0;
  layout(*p, kPagedMaxSms, &d, static_cast<unsigned char*>(p->workspace), &zeroed);
  const long long bits = element_bits(p->cache_type);
  auto bytes = [bits](long long elements) { return elements / 8 * bits; };  // (strides are multiples of 16 bytes)
  d.Hq = p->n_q_heads;
  d.Hkv = p->n_kv_heads;
  d.G = d.Hq / d.Hkv;
  d.D = p->head_dim;
  d.P = p->page_tokens;
  d.type = p->type;
  d.cache_type = p->cache_type;
  d.row_bytes = (int)bytes(d.D);
  d.n_pages = (int)p->n_pages;
  int log = 0;
  while ((1 << log) < d.P) ++log;
  d.p_shift = 31 + log;
  d.p_mul = (unsigned)((1ull << d.p_shift) / d.P + 1);
  d.ls = p->n_layers > 1 ? bytes(p->layer_stride) : 0;
  d.ps = p->n_pages > 1 ? bytes(p->page_stride) : 0;
  d.hs = p->n_kv_heads > 1 ? bytes(p->head_stride) : 0;
  d.ts = p->page_tokens > 1 ? bytes(p->token_stride) : 0;
  d.scale = (p->softmax_scale > 0.f ? p->softmax_scale : 1.f / std::sqrt((float)d.D)) * 1.4426950408889634f;
  d.decay = p->weight_decay;
  d.wait_limit = kPagedWaitLimit;
  d.k = static_cast<unsigned char*>(p->k_pages);
  d.v = static_cast<unsigned char*>(p->v_pages);
  d.ks = p->k_scale;
  d.vs = p->v_scale;
  d.sc = p->cache_type == LTRI_TYPE_INT4 ? block_scales : nullptr;
  d.w = p->weights;
  d.pos = p->positions;
  cudaError_t e = cudaGetDevice(&c->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, c->device);
  if (d.sms > kPagedMaxSms) d.sms = kPagedMaxSms;
  if (e == cudaSuccess) e = first_error(prepare_paged(d), prepare_paged_evict());
  if (e == cudaSuccess) c->attend = prepare_paged_attend(d);
  if (c->attend != cudaSuccess) cudaGetLastError();
  if (e == cudaSuccess) d.evict_cluster = paged_evict_cluster();
  if (e == cudaSuccess) e = cudaMemsetAsync(p->workspace, 0, zeroed, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) {
    cudaGetLastError();
    delete c;
    return LTRI_ECUDA;
  }
  *out = c;
  return LTRI_OK;
}

}  // namespace

extern "C" {

size_t ltri_paged_workspace_bytes(const ltri_paged_params* p) {
  return validate(p) ? layout(*p, kPagedMaxSms, nullptr, nullptr, nullptr) : 0;
}

int ltri_paged_create(const ltri_paged_params* p, void* cuda_stream, ltri_paged** out) {
  if (!out) return LTRI_EINVAL;
  *out = nullptr;
  if (!validate(p) || p->cache_type == LTRI_TYPE_INT4) return LTRI_EINVAL;
  return create(p, nullptr, static_cast<cudaStream_t>(cuda_stream), out);
}

int ltri_paged_create_int4(const ltri_paged_params* p, uint8_t* block_scales, void* cuda_stream, ltri_paged** out) {
  if (!out) return LTRI_EINVAL;
  *out = nullptr;
  if (!validate(p) || p->cache_type != LTRI_TYPE_INT4 || !aligned(block_scales, 16)) return LTRI_EINVAL;
  return create(p, block_scales, static_cast<cudaStream_t>(cuda_stream), out);
}

int ltri_paged_destroy(ltri_paged* cache) {
  if (!cache) return LTRI_EINVAL;
  delete cache;
  return LTRI_OK;
}

int ltri_paged_append(ltri_paged* cache, int layer, const int32_t* table, int table_pages, int64_t table_stride,
                      const int32_t* lens, int n_rows, const int32_t* starts, int64_t n_tokens, const void* k, const void* v,
                      int64_t kv_stride, const int32_t* row_pos, const float* weights, void* cuda_stream) {
  if (!cache || layer < 0 || layer >= cache->p.n_layers || !aligned(starts, 4) || n_tokens < 0) return LTRI_EINVAL;
  PagedRows r;
  if (const int rc = check_rows(cache, table, table_pages, table_stride, lens, n_rows, &r)) return rc;
  if (n_tokens > 0x7fffffffll) return LTRI_ECAPACITY;
  if (n_tokens == 0) return LTRI_OK;
  const long long stride = row_stride(cache, kv_stride, cache->p.n_kv_heads);
  if (!aligned(k, 16) || !aligned(v, 16) || !stride) return LTRI_EINVAL;
  if ((row_pos && !aligned(row_pos, 4)) || (weights && !aligned(weights, 4))) return LTRI_EINVAL;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  const PagedAppend a{starts, n_tokens, static_cast<const unsigned char*>(k), static_cast<const unsigned char*>(v), stride,
                      row_pos, weights};
  return done(cache, launch_paged_append(cache->c, r, layer, a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int ltri_paged_read(ltri_paged* cache, int layer, const int32_t* table, int table_pages, int64_t table_stride,
                    const int32_t* lens, int n_rows, const int32_t* starts, const int32_t* first, int64_t n_tokens, void* k,
                    void* v, int64_t kv_stride, void* cuda_stream) {
  if (!cache || layer < 0 || layer >= cache->p.n_layers || !aligned(starts, 4) || n_tokens < 0) return LTRI_EINVAL;
  PagedRows r;
  if (const int rc = check_rows(cache, table, table_pages, table_stride, lens, n_rows, &r)) return rc;
  if (n_tokens > 0x7fffffffll) return LTRI_ECAPACITY;
  if (n_tokens == 0) return LTRI_OK;
  const long long stride = row_stride(cache, kv_stride, cache->p.n_kv_heads);
  if ((!k && !v) || (k && !aligned(k, 16)) || (v && !aligned(v, 16)) || !stride) return LTRI_EINVAL;
  if (first && !aligned(first, 4)) return LTRI_EINVAL;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  const PagedRead a{starts, first, n_tokens, static_cast<unsigned char*>(k), static_cast<unsigned char*>(v), stride};
  return done(cache, launch_paged_read(cache->c, r, layer, a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int ltri_paged_decode(ltri_paged* cache, int layer, const int32_t* table, int table_pages, int64_t table_stride,
                      const int32_t* lens, int n_rows, const void* q, int64_t q_stride, const void* k, const void* v,
                      int64_t kv_stride, const int32_t* row_pos, void* out, float* lse, void* cuda_stream) {
  if (!cache || layer < 0 || layer >= cache->p.n_layers) return LTRI_EINVAL;
  PagedRows r;
  if (const int rc = check_rows(cache, table, table_pages, table_stride, lens, n_rows, &r)) return rc;
  const long long qs = row_stride(cache, q_stride, cache->p.n_q_heads), kvs = row_stride(cache, kv_stride, cache->p.n_kv_heads);
  if (!aligned(q, 16) || !aligned(out, 16) || !qs || !kvs || !k != !v) return LTRI_EINVAL;
  if (k && (!aligned(k, 16) || !aligned(v, 16))) return LTRI_EINVAL;
  if ((row_pos && !aligned(row_pos, 4)) || (lse && !aligned(lse, 4))) return LTRI_EINVAL;
  // outputs are written while other rows' queries are still to be read
  const long long row = (long long)cache->p.n_q_heads * cache->p.head_dim * 2;
  if (!(out == q && (qs == row || n_rows == 1)) && meets(out, n_rows * row, q, n_rows, row, qs)) return LTRI_EINVAL;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  const PagedStep a{static_cast<const unsigned char*>(q), static_cast<const unsigned char*>(k),
                    static_cast<const unsigned char*>(v), qs, kvs, row_pos, static_cast<unsigned char*>(out), lse};
  return done(cache, launch_paged_decode(cache->c, r, layer, a, static_cast<cudaStream_t>(cuda_stream)),
              paged_decode_kernels(cache->c));
}

size_t ltri_paged_attend_workspace_bytes(const ltri_paged* cache, int64_t max_tokens) {
  if (!cache || max_tokens < 1 || max_tokens > kPagedMaxTokens) return 0;
  return paged_attend_workspace(cache->c, max_tokens, cache->p.max_rows);
}

int ltri_paged_attend(ltri_paged* cache, int layer, const int32_t* table, int table_pages, int64_t table_stride,
                      const int32_t* lens, int n_rows, const int32_t* starts, int64_t n_tokens, const void* q, int64_t q_stride,
                      void* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!cache || layer < 0 || layer >= cache->p.n_layers || !aligned(starts, 4) || n_tokens < 0) return LTRI_EINVAL;
  PagedRows r;
  if (const int rc = check_rows(cache, table, table_pages, table_stride, lens, n_rows, &r)) return rc;
  if (n_tokens > kPagedMaxTokens) return LTRI_ECAPACITY;
  if (n_tokens == 0) return LTRI_OK;
  const long long qs = row_stride(cache, q_stride, cache->p.n_q_heads);
  if (!aligned(q, 16) || !aligned(out, 16) || !qs || (lse && !aligned(lse, 4)) || !aligned(workspace, 256)) return LTRI_EINVAL;
  if (workspace_bytes < paged_attend_workspace(cache->c, n_tokens, n_rows)) return LTRI_ECAPACITY;
  // outputs are written while other tokens' queries are still to be read
  const long long row = (long long)cache->p.n_q_heads * cache->p.head_dim * 2;
  if (!(out == q && (qs == row || n_tokens == 1)) && meets(out, n_tokens * row, q, n_tokens, row, qs)) return LTRI_EINVAL;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  if (cache->attend != cudaSuccess) return done(cache, cache->attend, 0);
  const PagedQueries a{starts, n_tokens, static_cast<const unsigned char*>(q), qs, static_cast<unsigned char*>(out), lse};
  return done(cache, launch_paged_attend(cache->c, r, layer, a, static_cast<unsigned char*>(workspace),
                                         static_cast<cudaStream_t>(cuda_stream)), 3);
}

int ltri_paged_evict(ltri_paged* cache, int layer_begin, int layer_count, const int32_t* table, int table_pages,
                     int64_t table_stride, const int32_t* lens, int32_t* new_lens, int n_rows, int budget, int n_sink,
                     int recent, void* cuda_stream) {
  if (!cache || !cache->p.weights || layer_begin < 0 || layer_count < 1 || layer_count > cache->p.n_layers - layer_begin)
    return LTRI_EINVAL;
  PagedRows r;
  if (const int rc = check_rows(cache, table, table_pages, table_stride, lens, n_rows, &r)) return rc;
  if (!aligned(new_lens, 4) || budget < 1 || n_sink < 0 || recent < 0 || (int64_t)n_sink + recent > budget) return LTRI_EINVAL;
  // the same lengths or others: where one row's new length replaced another's old one, its CTAs would disagree about it
  const uintptr_t l0 = reinterpret_cast<uintptr_t>(lens), l1 = reinterpret_cast<uintptr_t>(new_lens);
  if (l0 != l1 && (l0 < l1 ? l1 - l0 : l0 - l1) < (uintptr_t)n_rows * sizeof(int32_t)) return LTRI_EINVAL;
  // (a cluster for every layer, row and KV head)
  if ((int64_t)layer_count * n_rows > (1ll << 24) / cache->p.n_kv_heads) return LTRI_ECAPACITY;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  return done(cache, launch_paged_evict(cache->c, r, layer_begin, layer_count, new_lens, budget, n_sink, recent,
                                        static_cast<cudaStream_t>(cuda_stream)), 1);
}

int ltri_paged_sync_status(ltri_paged* cache, void* cuda_stream) {
  if (!cache) return LTRI_EINVAL;
  OnDevice on(cache->device);
  if (!on.ok) return done(cache, cudaErrorInvalidDevice, 0);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int w[4] = {0, 0, 0, 0};
  cudaError_t e = cudaMemcpyAsync(w, cache->c.status, sizeof(w), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && w[0] != 0) {
    e = cudaMemsetAsync(cache->c.status, 0, sizeof(w), s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  }
  if (e != cudaSuccess) return done(cache, e, 0);
  return w[0];
}

int ltri_paged_debug_wait(ltri_paged* cache, int64_t limit_cycles, int held) {
  if (!cache || limit_cycles < 0 || limit_cycles > 100000000 || held < 0 || held > 3 || (held && !limit_cycles)) return LTRI_EINVAL;
  cache->c.wait_limit = limit_cycles ? limit_cycles : kPagedWaitLimit;
  cache->c.held = held;
  return LTRI_OK;
}

int ltri_paged_last_cuda_error(const ltri_paged* cache) { return cache ? cache->last_cuda : 0; }

int64_t ltri_paged_launch_count(const ltri_paged* cache) { return cache ? cache->launches : 0; }

}  // extern "C"
