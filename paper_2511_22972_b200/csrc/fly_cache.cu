// Host side of the C ABI declared in include/fly_cache.h: argument checks and kernel launches.  No torch types, no
// allocation outside fly_attention_create.
#include "fly_cache.h"

#include <cmath>
#include <new>

#include "attention_kernel.cuh"
#include "cache_kernel.cuh"
#include "device_guard.h"

struct fly_attention {
  fly_attention_config_t cfg;
  int last_launches = 0;
  int last_cuda_error = 0;
};

namespace {

namespace K = fly::cache;

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// FLY_ERR_INVALID_ARG: nothing could serve it.  FLY_ERR_UNSUPPORTED: alignment, strides and shapes that the kernels do not take.
fly_status_t check_cache(const fly_cache_t* c, int32_t B, int32_t n) {
  if (!c || c->device < 0 || !c->k_pages || !c->v_pages || !c->block_table || !c->lengths) return FLY_ERR_INVALID_ARG;
  if (c->format != FLY_CACHE_BF16 && c->format != FLY_CACHE_E4M3) return FLY_ERR_INVALID_ARG;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  if (e4m3 != (c->k_scales != nullptr) || e4m3 != (c->v_scales != nullptr)) return FLY_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1 || c->max_pages < 1 || c->sequences < 1 ||
      c->table_stride < c->max_pages)
    return FLY_ERR_INVALID_ARG;
  if (B < 1 || B > c->sequences || n < 1) return FLY_ERR_INVALID_ARG;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return FLY_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FLY_ERR_UNSUPPORTED;
  if (c->page_size < 8 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0) return FLY_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > (int64_t)1 << 30 || n > 1 << 30) return FLY_ERR_UNSUPPORTED;
  const int64_t unit = e4m3 ? 16 : 8;  // elements in 16 bytes
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || (e4m3 && (!aligned(c->k_scales, 8) || !aligned(c->v_scales, 8))))
    return FLY_ERR_UNSUPPORTED;
  if ((c->num_pages > 1 && c->page_stride % unit) || c->token_stride % unit || (c->kv_heads > 1 && c->head_stride % unit))
    return FLY_ERR_UNSUPPORTED;
  return FLY_OK;
}

fly_status_t check_rows(const fly_rows_t* r) {
  if (!r || !r->data || r->batch_stride < 0 || r->token_stride < 0 || r->head_stride < 0) return FLY_ERR_INVALID_ARG;
  return aligned(r->data, 2) ? FLY_OK : FLY_ERR_UNSUPPORTED;
}

// Whether every row starts on 16 bytes.
bool wide(const fly_rows_t* r, int32_t B, int32_t n, int32_t heads) {
  return aligned(r->data, 16) && (B == 1 || r->batch_stride % 8 == 0) && (n == 1 || r->token_stride % 8 == 0) &&
         (heads == 1 || r->head_stride % 8 == 0);
}

K::View view_of(const fly_cache_t* c) {
  K::View v;
  v.k_pages = static_cast<uint8_t*>(c->k_pages);
  v.v_pages = static_cast<uint8_t*>(c->v_pages);
  v.k_scales = c->k_scales;
  v.v_scales = c->v_scales;
  v.page_stride = c->page_stride;
  v.token_stride = c->token_stride;
  v.head_stride = c->head_stride;
  v.table = c->block_table;
  v.table_stride = c->table_stride;
  v.lengths = c->lengths;
  v.num_pages = c->num_pages;
  v.page_shift = 0;
  while (1 << v.page_shift < c->page_size) ++v.page_shift;
  v.kv_heads = c->kv_heads;
  v.head_dim = c->head_dim;
  v.capacity = c->max_pages * c->page_size;
  return v;
}

K::Rows rows_of(const fly_rows_t* r) { return {static_cast<uint8_t*>(r->data), r->batch_stride, r->token_stride, r->head_stride}; }

// One group of head_dim / 8 threads per (token, head), sequences along y.
bool row_grid(const fly_cache_t* c, int32_t B, int32_t n, dim3* grid) {
  const int64_t per_block = K::kThreads / (c->head_dim / 8), blocks = ((int64_t)n * c->kv_heads + per_block - 1) / per_block;
  if (blocks > 0x7fffffff) return false;
  *grid = dim3((unsigned)blocks, (unsigned)(B < 65535 ? B : 65535));
  return true;
}

}  // namespace

extern "C" {

fly_status_t fly_cache_append(const fly_cache_t* c, int32_t B, int32_t n, const fly_rows_t* k, const fly_rows_t* v,
                              const int32_t* counts, uint32_t* row_flags, void* cuda_stream) {
  fly_status_t s = check_cache(c, B, n);
  if (s != FLY_OK || (s = check_rows(k)) != FLY_OK || (s = check_rows(v)) != FLY_OK) return s;
  DeviceGuard g(c->device);
  if (!g.ok) return FLY_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, 1, K::kThreads, static_cast<cudaStream_t>(cuda_stream), true);
  if (!row_grid(c, B, n, &cfg.gridDim)) return FLY_ERR_UNSUPPORTED;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  auto kernel = c->head_dim == 128 ? (e4m3 ? K::append_kernel<128, true> : K::append_kernel<128, false>)
                                   : (e4m3 ? K::append_kernel<64, true> : K::append_kernel<64, false>);
  const int aligned_rows = (wide(k, B, n, c->kv_heads) ? 1 : 0) | (wide(v, B, n, c->kv_heads) ? 2 : 0);
  return cudaLaunchKernelEx(&cfg, kernel, view_of(c), rows_of(k), rows_of(v), (int)B, (int)n, counts, row_flags, aligned_rows) == cudaSuccess
             ? FLY_OK
             : FLY_ERR_CUDA;
}

fly_status_t fly_cache_read(const fly_cache_t* c, int32_t B, int32_t n, const int32_t* starts, const fly_rows_t* k, const fly_rows_t* v,
                            void* cuda_stream) {
  fly_status_t s = check_cache(c, B, n);
  if (s != FLY_OK || (s = check_rows(k)) != FLY_OK || (s = check_rows(v)) != FLY_OK) return s;
  DeviceGuard g(c->device);
  if (!g.ok) return FLY_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, 1, K::kThreads, static_cast<cudaStream_t>(cuda_stream), true);
  if (!row_grid(c, B, n, &cfg.gridDim)) return FLY_ERR_UNSUPPORTED;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  auto kernel = c->head_dim == 128 ? (e4m3 ? K::read_kernel<128, true> : K::read_kernel<128, false>)
                                   : (e4m3 ? K::read_kernel<64, true> : K::read_kernel<64, false>);
  const int aligned_rows = (wide(k, B, n, c->kv_heads) ? 1 : 0) | (wide(v, B, n, c->kv_heads) ? 2 : 0);
  return cudaLaunchKernelEx(&cfg, kernel, view_of(c), rows_of(k), rows_of(v), (int)B, (int)n, starts, aligned_rows) == cudaSuccess ? FLY_OK
                                                                                                                                  : FLY_ERR_CUDA;
}

fly_status_t fly_attention_create(const fly_attention_config_t* c, fly_attention_t** out) {
  if (out) *out = nullptr;
  if (!c || !out) return FLY_ERR_INVALID_ARG;
  if (c->device < 0 || c->max_batch < 1 || c->max_tokens < 1 || c->kv_heads < 1 || c->heads < 1 || c->heads % c->kv_heads != 0 || c->head_dim < 1)
    return FLY_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->heads / c->kv_heads > 128) return FLY_ERR_UNSUPPORTED;
  fly_attention* h = new (std::nothrow) fly_attention();
  if (!h) return FLY_ERR_INVALID_ARG;
  h->cfg = *c;
  *out = h;
  return FLY_OK;
}

fly_status_t fly_attention_destroy(fly_attention_t* h) {
  delete h;
  return FLY_OK;
}

fly_status_t fly_attention_run(fly_attention_t* h, const fly_cache_t* c, const fly_attention_args_t* a, void* cuda_stream) {
  if (!h || !a) return FLY_ERR_INVALID_ARG;
  fly_status_t s = check_cache(c, a->B, a->n);
  if (s != FLY_OK || (s = check_rows(&a->q)) != FLY_OK || (s = check_rows(&a->out)) != FLY_OK) return s;
  if (a->B > h->cfg.max_batch || a->n > h->cfg.max_tokens || c->device != h->cfg.device || c->kv_heads != h->cfg.kv_heads ||
      c->head_dim != h->cfg.head_dim)
    return FLY_ERR_INVALID_ARG;
  if (a->window < 0 || a->sinks < 0 || (a->sinks > 0 && a->window == 0)) return FLY_ERR_INVALID_ARG;
  if (!(a->scale >= 0.0) || !std::isfinite(a->scale)) return FLY_ERR_INVALID_ARG;
  if (!wide(&a->q, a->B, a->n, h->cfg.heads) || !wide(&a->out, a->B, a->n, h->cfg.heads)) return FLY_ERR_UNSUPPORTED;
  if ((a->B > 1 && a->q.batch_stride == 0) || (a->n > 1 && a->q.token_stride == 0) || (h->cfg.heads > 1 && a->q.head_stride == 0))
    return FLY_ERR_UNSUPPORTED;
  DeviceGuard g(h->cfg.device);
  if (!g.ok) return FLY_ERR_CUDA;
  fly::attn::Params p;
  p.c = view_of(c);
  p.q = rows_of(&a->q);
  p.out = rows_of(&a->out);
  p.lse = a->lse;
  p.counts = a->counts;
  p.B = a->B;
  p.n = a->n;
  p.heads = h->cfg.heads;
  p.group = h->cfg.heads / h->cfg.kv_heads;
  p.window = a->window;
  p.sinks = a->sinks;
  p.scale = (float)((a->scale == 0.0 ? 1.0 / std::sqrt((double)c->head_dim) : a->scale) * 1.4426950408889634);
  const int64_t blocks = ((int64_t)p.B * p.n * p.heads + 3) / 4;
  if (blocks > 0x7fffffff) return FLY_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, (unsigned)blocks, fly::attn::kThreads, static_cast<cudaStream_t>(cuda_stream), true);
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  auto kernel = c->head_dim == 128 ? (e4m3 ? fly::attn::attention_kernel<128, true> : fly::attn::attention_kernel<128, false>)
                                   : (e4m3 ? fly::attn::attention_kernel<64, true> : fly::attn::attention_kernel<64, false>);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  if (e != cudaSuccess) {
    h->last_cuda_error = (int)e;
    return FLY_ERR_CUDA;
  }
  h->last_launches = 1;
  return FLY_OK;
}

int32_t fly_attention_last_launch_count(const fly_attention_t* h) { return h ? h->last_launches : 0; }
int32_t fly_attention_last_cuda_error(const fly_attention_t* h) { return h ? h->last_cuda_error : 0; }

}  // extern "C"
