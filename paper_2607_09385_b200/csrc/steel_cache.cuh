// What the kernels of the paged 4-bit cache share: the memory's layout (include/steel_cache.h), checks of what the device finds
// in tables and batches, and the launch interface.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/steel_cache.h"

namespace steel {

constexpr int kUnitTokens = 16;   // tokens of a unit: one tensor-core operand's rows
constexpr int kGroup = 64;        // channels that share a scale
constexpr int kMaxSlots = 8192, kMaxCachePages = 1 << 20;

// bytes of a unit: 16 tokens of one head, keys and values, codes and scales
__host__ __device__ constexpr int unit_bytes(int head_dim) { return kUnitTokens * head_dim + head_dim / kGroup * 128; }

// The cache as a kernel sees it; `pool` is one layer's for the calls that name a layer.
struct CacheView {
  unsigned char *pool;
  int32_t *table, *lens, *refs, *status;
  int64_t layer_bytes, page_bytes;
  int32_t layers, pages, page_shift, heads_kv, slots, max_pages;  // page_tokens = 1 << page_shift
};

constexpr long long kWaitCycles = 1ll << 32;  // the bound of a wait on the device: about two seconds

// Odd numbers that memory does not hold by chance, another for each launch: a flag in memory that nobody has cleared is set only if it equals its
// launch's.  (A launch in a graph keeps its number: steel_cache_wait.cuh.)
uint64_t next_token();

struct Rows {  // steel_cache_tensor_t
  unsigned char *data;
  int64_t batch, head, seq;  // strides in bytes
};

struct CacheBatch {
  const int32_t *slots, *counts;  // either may be null
  int32_t batch;
};

__device__ __forceinline__ void report(int32_t *status, int32_t code) { atomicCAS(status, STEEL_OK, code); }

// Slot of a batch's sequence i, or -1.
__device__ __forceinline__ int slot_of(const CacheView &c, const int32_t *slots, int i) {
  const int s = slots ? slots[i] : i;
  return s >= 0 && s < c.slots ? s : -1;
}

__device__ __forceinline__ int max_tokens(const CacheView &c) { return c.max_pages << c.page_shift; }

// Whether sequence i of the batch has the slot of an earlier one (asked by a whole warp).
__device__ __forceinline__ bool slot_taken_before(const int32_t *slots, int i, int slot, int lane) {
  if (!slots) return false;
  bool same = false;
  for (int j = lane; j < i; j += 32) same |= slots[j] == slot;
  return __any_sync(0xffffffffu, same);
}

// Launches that carry the programmatic-serialisation attribute: a kernel's blocks may be set up while the kernel before it
// drains; every thread waits (griddepcontrol.wait) before it touches global memory.
template <class... Params, class... Args>
cudaError_t launch_overlapping(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                               Args... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Kernels' launchers (steel_cache_tokens.cu, steel_cache_attend.cu, steel_cache_pages.cu).
cudaError_t launch_append(const CacheView &c, int head_dim, const CacheBatch &b, int seq, const Rows &k, const Rows &v,
                          cudaStream_t stream);
cudaError_t launch_read(const CacheView &c, int head_dim, const int32_t *slots, const int32_t *begin, int batch, int seq,
                        const Rows &k, const Rows &v, cudaStream_t stream);

struct AttendProblem {
  CacheBatch b;
  int32_t heads_q, seq_q, head_dim;
  uint32_t flags;
  float scale;
  int64_t window;
  Rows q;
  void *o;
  float *lse;
  unsigned char *workspace;
  long long wait_cycles;
};
bool attend_fits(const CacheView &c, int batch, int heads_q, int seq_q);  // the work counts within 32 bits
int64_t attend_workspace(int head_dim, int sms);
cudaError_t configure_attend();
cudaError_t launch_attend(const CacheView &c, const AttendProblem &p, int sms, cudaStream_t stream);

int64_t pages_scratch_bytes(int slots, int max_pages, int pages);
cudaError_t configure_pages();
cudaError_t launch_extend(const CacheView &c, int head_dim, void *scratch, const CacheBatch &b, int sms, cudaStream_t stream);
cudaError_t launch_fork(const CacheView &c, void *scratch, int n, const int32_t *src, const int32_t *dst, cudaStream_t stream);
cudaError_t launch_free(const CacheView &c, const CacheBatch &b, cudaStream_t stream);
cudaError_t launch_compact(const CacheView &c, int head_dim, void *scratch, int32_t *live, int sms, cudaStream_t stream);

}  // namespace steel
