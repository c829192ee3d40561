// C ABI of the paged 4-bit cache (include/steel_cache.h): checks of arguments and launches.  Nothing here allocates device
// memory or waits, but steel_cache_last_status.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <chrono>
#include <cmath>
#include <tuple>
#include <new>

#include "steel_cache.cuh"

using namespace steel;

uint64_t steel::next_token() {
  static std::atomic<uint64_t> count{uint64_t(std::chrono::system_clock::now().time_since_epoch().count()) * 2654435761u};
  uint64_t z = count.fetch_add(0x9E3779B97F4A7C15ull);  // splitmix64
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return (z ^ (z >> 31)) | 1;  // not 0
}

struct steel_cache {
  steel_cache_params_t params;
  steel_cache_memory_t memory;
  CacheView view;  // pool of layer 0
  int device, sms;
  long long wait_cycles;  // of attend, for another CTA's part
};

namespace {

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int log2_of(int n) {
  int s = 0;
  while ((1 << s) < n) ++s;
  return s;
}

steel_status_t check(const steel_cache_params_t *p) {
  if (!p) return STEEL_ERR_INVALID_ARG;
  if (p->layers <= 0 || p->pages <= 0 || p->page_tokens <= 0 || p->heads_kv <= 0 || p->head_dim <= 0 || p->slots <= 0 ||
      p->max_pages <= 0)
    return STEEL_ERR_INVALID_ARG;
  if (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128)
    return STEEL_ERR_UNSUPPORTED;
  if ((p->head_dim != 64 && p->head_dim != 128) || p->layers > 4096 || p->pages > kMaxCachePages || p->heads_kv > 1024 ||
      p->slots > kMaxSlots || p->max_pages > kMaxCachePages || int64_t(p->max_pages) * p->page_tokens > (int64_t(1) << 30) ||
      (int64_t(p->max_pages) * (p->page_tokens / kUnitTokens) + 1) * p->heads_kv > (int64_t(1) << 30))
    return STEEL_ERR_UNSUPPORTED;
  return STEEL_OK;
}

void fill_sizes(const steel_cache_params_t &p, steel_cache_sizes_t *s) {
  s->unit_bytes = unit_bytes(p.head_dim);
  s->page_bytes = s->unit_bytes * (p.page_tokens / kUnitTokens) * p.heads_kv;
  s->pool_bytes = s->page_bytes * p.pages * p.layers;  // at most 2^12 * 2^20 * 2^10 * 2^15
  s->table_bytes = int64_t(p.slots) * p.max_pages * int64_t(sizeof(int32_t));
  s->lens_bytes = int64_t(p.slots) * int64_t(sizeof(int32_t));
  s->refs_bytes = int64_t(p.pages) * int64_t(sizeof(int32_t));
  s->status_bytes = sizeof(int32_t);
  s->scratch_bytes = pages_scratch_bytes(p.slots, p.max_pages, p.pages);
}

// The call's device is the cache's, and the batch can be one.
steel_status_t check_call(const steel_cache *c, int32_t batch, bool distinct, const int32_t *slots) {
  if (!c || batch < 0 || !aligned(slots, 4)) return STEEL_ERR_INVALID_ARG;
  if ((distinct || !slots) && batch > c->params.slots) return STEEL_ERR_INVALID_ARG;
  if (batch > 65535) return STEEL_ERR_UNSUPPORTED;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) {
    cudaGetLastError();
    return STEEL_ERR_CUDA;
  }
  return device == c->device ? STEEL_OK : STEEL_ERR_INVALID_ARG;
}

bool check_rows(const steel_cache_tensor_t *t, int batch, int heads, int seq, Rows *out) {
  if (!t || !t->data || !aligned(t->data, 16)) return false;
  constexpr int64_t kMost = int64_t(1) << 40;
  // a stride along which there is one element is never used
  const int64_t b = batch > 1 ? t->stride_batch : 0, h = heads > 1 ? t->stride_head : 0, s = seq > 1 ? t->stride_seq : 0;
  for (int64_t stride : {b, h, s})
    if (stride < 0 || stride > kMost || stride % 8) return false;
  *out = Rows{static_cast<unsigned char *>(t->data), b * 2, h * 2, s * 2};
  return true;
}

CacheView layer_view(const steel_cache *c, int layer) {
  CacheView v = c->view;
  v.pool += v.layer_bytes * layer;
  return v;
}

steel_status_t launched(cudaError_t e) {
  if (e == cudaSuccess) return STEEL_OK;
  cudaGetLastError();
  return STEEL_ERR_CUDA;
}

}  // namespace

extern "C" {

steel_status_t steel_cache_sizes(const steel_cache_params_t *params, steel_cache_sizes_t *sizes) {
  if (!sizes) return STEEL_ERR_INVALID_ARG;
  const steel_status_t st = check(params);
  if (st == STEEL_OK) fill_sizes(*params, sizes);
  return st;
}

steel_status_t steel_cache_create(const steel_cache_params_t *params, const steel_cache_memory_t *m, steel_cache_t **out) {
  if (!out) return STEEL_ERR_INVALID_ARG;
  *out = nullptr;
  const steel_status_t st = check(params);
  if (st != STEEL_OK) return st;
  if (!m || !m->pool || !m->table || !m->lens || !m->refs || !m->status || !m->scratch || !aligned(m->pool, 128) ||
      !aligned(m->scratch, 128) || !aligned(m->status, 128) || !aligned(m->table, 4) || !aligned(m->lens, 4) ||
      !aligned(m->refs, 4))
    return STEEL_ERR_INVALID_ARG;
  int device = 0, major = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || major != 10 ||
      configure_attend() != cudaSuccess || configure_pages() != cudaSuccess) {
    cudaGetLastError();
    return STEEL_ERR_CUDA;
  }
  steel_cache *c = new (std::nothrow) steel_cache();
  if (!c) return STEEL_ERR_ALLOC;
  steel_cache_sizes_t sizes;
  fill_sizes(*params, &sizes);
  c->params = *params;
  c->memory = *m;
  c->device = device;
  c->sms = sms;
  c->wait_cycles = kWaitCycles;
  c->view = CacheView{static_cast<unsigned char *>(m->pool), m->table, m->lens, m->refs, m->status,
                      sizes.page_bytes * params->pages, sizes.page_bytes, params->layers, params->pages,
                      log2_of(params->page_tokens), params->heads_kv, params->slots, params->max_pages};
  *out = c;
  return STEEL_OK;
}

steel_status_t steel_cache_destroy(steel_cache_t *c) {
  delete c;
  return STEEL_OK;
}

steel_status_t steel_cache_reset(steel_cache_t *c, void *cuda_stream) {
  steel_status_t st = check_call(c, 0, true, nullptr);
  if (st != STEEL_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  steel_cache_sizes_t s;
  fill_sizes(c->params, &s);
  for (auto [p, value, bytes] : {std::make_tuple(c->memory.table, 0xff, s.table_bytes), std::make_tuple(c->memory.lens, 0, s.lens_bytes),
                                 std::make_tuple(c->memory.refs, 0, s.refs_bytes),
                                 std::make_tuple(c->memory.status, 0, s.status_bytes)})
    if (st == STEEL_OK) st = launched(cudaMemsetAsync(p, value, size_t(bytes), stream));
  return st;
}

steel_status_t steel_cache_extend(steel_cache_t *c, int32_t batch, const int32_t *slots, const int32_t *counts,
                                  void *cuda_stream) {
  steel_status_t st = check_call(c, batch, true, slots);
  if (st != STEEL_OK) return st;
  if (batch == 0) return STEEL_OK;
  if (!counts || !aligned(counts, 4)) return STEEL_ERR_INVALID_ARG;
  return launched(launch_extend(c->view, c->params.head_dim, c->memory.scratch, CacheBatch{slots, counts, batch}, c->sms,
                                static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_append(steel_cache_t *c, int32_t layer, int32_t batch, const int32_t *slots, const int32_t *counts,
                                  int32_t seq, const steel_cache_tensor_t *k, const steel_cache_tensor_t *v, void *cuda_stream) {
  steel_status_t st = check_call(c, batch, true, slots);
  if (st != STEEL_OK) return st;
  Rows rk, rv;
  if (layer < 0 || layer >= c->params.layers || seq < 0 || seq > (1 << 30) || !aligned(counts, 4)) return STEEL_ERR_INVALID_ARG;
  if (batch == 0 || seq == 0) return STEEL_OK;
  if (!check_rows(k, batch, c->params.heads_kv, seq, &rk) || !check_rows(v, batch, c->params.heads_kv, seq, &rv))
    return STEEL_ERR_INVALID_ARG;
  return launched(launch_append(layer_view(c, layer), c->params.head_dim, CacheBatch{slots, counts, batch}, seq, rk, rv,
                                static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_read(steel_cache_t *c, int32_t layer, int32_t batch, const int32_t *slots, const int32_t *begin,
                                int32_t seq, const steel_cache_tensor_t *k, const steel_cache_tensor_t *v, void *cuda_stream) {
  steel_status_t st = check_call(c, batch, false, slots);
  if (st != STEEL_OK) return st;
  Rows rk, rv;
  if (layer < 0 || layer >= c->params.layers || seq < 0 || seq > (1 << 30) || !aligned(begin, 4)) return STEEL_ERR_INVALID_ARG;
  if (batch == 0 || seq == 0) return STEEL_OK;
  if (!check_rows(k, batch, c->params.heads_kv, seq, &rk) || !check_rows(v, batch, c->params.heads_kv, seq, &rv))
    return STEEL_ERR_INVALID_ARG;
  return launched(launch_read(layer_view(c, layer), c->params.head_dim, slots, begin, batch, seq, rk, rv,
                              static_cast<cudaStream_t>(cuda_stream)));
}

int64_t steel_cache_attend_workspace(const steel_cache_t *c, int32_t batch, int32_t heads_q, int32_t seq_q) {
  if (!c || batch < 0 || heads_q <= 0 || heads_q % c->params.heads_kv || seq_q < 0) return -1;
  return attend_workspace(c->params.head_dim, c->sms);
}

steel_status_t steel_cache_attend(steel_cache_t *c, const steel_cache_attend_t *a, void *cuda_stream) {
  if (!a) return STEEL_ERR_INVALID_ARG;
  steel_status_t st = check_call(c, a->batch, false, a->slots);
  if (st != STEEL_OK) return st;
  if (a->layer < 0 || a->layer >= c->params.layers || a->heads_q <= 0 || a->heads_q % c->params.heads_kv || a->seq_q < 0 ||
      !aligned(a->counts, 4) || (a->flags & ~uint32_t(STEEL_MASK_CAUSAL | STEEL_MASK_WINDOW)) || !std::isfinite(a->scale) ||
      a->scale <= 0.f || ((a->flags & STEEL_MASK_WINDOW) && a->window <= 0))
    return STEEL_ERR_INVALID_ARG;
  if (a->batch == 0 || a->seq_q == 0) return STEEL_OK;
  if (!attend_fits(c->view, a->batch, a->heads_q, a->seq_q)) return STEEL_ERR_UNSUPPORTED;
  Rows q;
  if (!check_rows(&a->q, a->batch, a->heads_q, a->seq_q, &q) || !a->o || !aligned(a->o, 16) || !aligned(a->lse, 4) ||
      !a->workspace || !aligned(a->workspace, 128) ||
      a->workspace_bytes < steel_cache_attend_workspace(c, a->batch, a->heads_q, a->seq_q))
    return STEEL_ERR_INVALID_ARG;
  AttendProblem p{CacheBatch{a->slots, a->counts, a->batch}, a->heads_q, a->seq_q, c->params.head_dim, a->flags, a->scale,
                  a->window, q, a->o, a->lse, static_cast<unsigned char *>(a->workspace), c->wait_cycles};
  return launched(launch_attend(layer_view(c, a->layer), p, c->sms, static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_fork(steel_cache_t *c, int32_t n, const int32_t *src, const int32_t *dst, void *cuda_stream) {
  steel_status_t st = check_call(c, n, true, src);
  if (st != STEEL_OK) return st;
  if (n == 0) return STEEL_OK;
  if (!src || !dst || !aligned(dst, 4)) return STEEL_ERR_INVALID_ARG;
  return launched(launch_fork(c->view, c->memory.scratch, n, src, dst, static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_free(steel_cache_t *c, int32_t batch, const int32_t *slots, const int32_t *keep, void *cuda_stream) {
  steel_status_t st = check_call(c, batch, true, slots);
  if (st != STEEL_OK) return st;
  if (!aligned(keep, 4)) return STEEL_ERR_INVALID_ARG;
  if (batch == 0) return STEEL_OK;
  return launched(launch_free(c->view, CacheBatch{slots, keep, batch}, static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_compact(steel_cache_t *c, int32_t *live, void *cuda_stream) {
  steel_status_t st = check_call(c, 0, true, nullptr);
  if (st != STEEL_OK) return st;
  if (!aligned(live, 4)) return STEEL_ERR_INVALID_ARG;
  return launched(launch_compact(c->view, c->params.head_dim, c->memory.scratch, live, c->sms,
                                 static_cast<cudaStream_t>(cuda_stream)));
}

steel_status_t steel_cache_debug_wait(steel_cache_t *c, int64_t cycles) {
  if (!c) return STEEL_ERR_INVALID_ARG;
  c->wait_cycles = cycles < 0 ? kWaitCycles : std::min<long long>(cycles, 1ll << 46);
  return STEEL_OK;
}

steel_status_t steel_cache_last_status(steel_cache_t *c, void *cuda_stream) {
  steel_status_t st = check_call(c, 0, true, nullptr);
  if (st != STEEL_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  int32_t word = 0;
  if (cudaMemcpyAsync(&word, c->memory.status, sizeof word, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
      cudaStreamSynchronize(stream) != cudaSuccess ||
      (word != 0 && (cudaMemsetAsync(c->memory.status, 0, sizeof word, stream) != cudaSuccess ||
                     cudaStreamSynchronize(stream) != cudaSuccess))) {
    cudaGetLastError();
    return STEEL_ERR_CUDA;
  }
  return static_cast<steel_status_t>(word);
}

}  // extern "C"
