// Runs the paged cache's C entry points on the host over a runtime and kernels that are none: what they do with errors.
#include <cuda_runtime.h>

#include <cstdio>
#include <cstring>

static int atomicCAS(int*, int, int) { return 0; }
static int __shfl_xor_sync(unsigned, int x, int) { return x; }
static int __shfl_up_sync(unsigned, int x, int) { return x; }
static int __shfl_sync(unsigned, int x, int) { return x; }
static struct { int x; } threadIdx;
namespace ltri {
static cudaError_t first_error(cudaError_t a, cudaError_t b) { return a != cudaSuccess ? a : b; }
}

#include "../paper_2412_04757_b200/csrc/paged_api.cu"

static cudaError_t attend_fails = cudaSuccess;
static int attends = 0, prepared = 0;

namespace ltri {
PagedBlocks paged_blocks(int) { return PagedBlocks{8, 1}; }
size_t paged_part_floats(int, int head_dim) { return 10 * head_dim; }
int paged_decode_kernels(const PagedCache&) { return 1; }
int paged_evict_cluster() { return 1; }
cudaError_t prepare_paged(const PagedCache&) { return cudaSuccess; }
cudaError_t prepare_paged_evict() { return cudaSuccess; }
cudaError_t prepare_paged_attend(const PagedCache&) { return ++prepared, attend_fails; }
size_t paged_attend_workspace(const PagedCache&, long long, long long) { return 256; }
cudaError_t launch_paged_attend(const PagedCache&, const PagedRows&, int, const PagedQueries&, unsigned char*, cudaStream_t) {
  return ++attends, cudaSuccess;
}
cudaError_t launch_paged_append(const PagedCache&, const PagedRows&, int, const PagedAppend&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_paged_read(const PagedCache&, const PagedRows&, int, const PagedRead&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_paged_decode(const PagedCache&, const PagedRows&, int, const PagedStep&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_paged_evict(const PagedCache&, const PagedRows&, int, int, int*, int, int, int, cudaStream_t) { return cudaSuccess; }
}  // namespace ltri

extern "C" {
cudaError_t cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* x, cudaDeviceAttr, int) { return *x = 148, cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void* to, const void*, size_t n, cudaMemcpyKind, cudaStream_t) { return memset(to, 0, n), cudaSuccess; }
}

#define CHECK(x) \
  if (!(x)) return printf("%s\n", #x), 1

int main() {
  ltri_paged_params p{};
  p.n_layers = p.n_kv_heads = p.max_rows = 1;
  p.n_q_heads = 4;
  p.head_dim = 128;
  p.page_tokens = 16;
  p.n_pages = 8;
  p.page_stride = 16 * 128;
  p.token_stride = 128;
  p.weight_decay = 1.f;
  auto at = [](size_t x) { return reinterpret_cast<void*>(x); };  // (nothing is looked at)
  p.k_pages = at(1 << 20);
  p.v_pages = at(2 << 20);
  p.workspace = at(3 << 20);
  p.workspace_bytes = ltri_paged_workspace_bytes(&p);
  const int32_t* ints = static_cast<int32_t*>(at(4 << 20));
  for (cudaError_t fails : {cudaSuccess, cudaErrorInvalidConfiguration}) {
    attend_fails = fails;
    attends = prepared = 0;
    ltri_paged* h = nullptr;
    // a device or build that has no room for attend's kernels has handles all the same, and all other calls
    CHECK(ltri_paged_create(&p, nullptr, &h) == LTRI_OK && h && prepared == 1);
    CHECK(ltri_paged_append(h, 0, ints, 8, 8, ints, 1, ints, 4, at(5 << 20), at(6 << 20), 0, nullptr, nullptr, nullptr) == LTRI_OK);
    CHECK(ltri_paged_read(h, 0, ints, 8, 8, ints, 1, ints, nullptr, 4, at(5 << 20), at(6 << 20), 0, nullptr) == LTRI_OK);
    CHECK(ltri_paged_decode(h, 0, ints, 8, 8, ints, 1, at(5 << 20), 0, nullptr, nullptr, 0, nullptr, at(6 << 20), nullptr, nullptr) ==
          LTRI_OK);
    CHECK(ltri_paged_last_cuda_error(h) == 0);
    CHECK(ltri_paged_attend_workspace_bytes(h, 4) == 256);
    const int rc = ltri_paged_attend(h, 0, ints, 8, 8, ints, 1, ints, 4, at(5 << 20), 0, at(6 << 20), nullptr, at(7 << 20), 256, nullptr);
    CHECK(rc == (fails == cudaSuccess ? LTRI_OK : LTRI_ECUDA) && attends == (fails == cudaSuccess));
    CHECK(ltri_paged_last_cuda_error(h) == (int)fails);
    CHECK(ltri_paged_launch_count(h) == (fails == cudaSuccess ? 6 : 3));
    CHECK(ltri_paged_destroy(h) == LTRI_OK);
  }
  puts("ok");
  return 0;
}
