// Host side of the C ABI declared in include/fly_cache.h: argument checks and kernel launches.  No torch types, no
// allocation outside fly_attention_create.
#include "fly_cache.h"

#include <cmath>
#include <initializer_list>
#include <new>

#include <cudaTypedefs.h>

#include "attention_kernel.cuh"
#include "cache_kernel.cuh"
#include "device_guard.h"

struct fly_attention {
  fly_attention_config_t cfg;
  int sm_count = 148;
  float4* part_o = nullptr;  // one block: parts of items | their references and sums | how the ranges begin | status word
  float2* part_ml = nullptr;
  int* desc = nullptr;
  int* status = nullptr;
  PFN_cuTensorMapEncodeTiled encode_tiled = nullptr;
  int last_launches = 0;
  int last_cuda_error = 0;
};

namespace {

namespace K = fly::cache;
namespace A = fly::attn;

constexpr int kMaxTokens = 1 << 28;  // of a chunk: a position and a chunk's end are int32

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
  if ((int64_t)c->max_pages * c->page_size > (int64_t)1 << 30 || n > kMaxTokens) return FLY_ERR_UNSUPPORTED;
  const int64_t unit = e4m3 ? 16 : 8;  // elements in 16 bytes
  if (!aligned(c->block_table, 4) || !aligned(c->lengths, 4)) return FLY_ERR_UNSUPPORTED;
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || (e4m3 && (!aligned(c->k_scales, 8) || !aligned(c->v_scales, 8))))
    return FLY_ERR_UNSUPPORTED;
  if ((c->num_pages > 1 && c->page_stride % unit) || c->token_stride % unit || (c->kv_heads > 1 && c->head_stride % unit))
    return FLY_ERR_UNSUPPORTED;
  // (rows that overlap hold nothing)
  if ((c->num_pages > 1 && c->page_stride < c->head_dim) || c->token_stride < c->head_dim || (c->kv_heads > 1 && c->head_stride < c->head_dim))
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

// Whether no dimension of rows that are written is a broadcast.
bool apart(const fly_rows_t* r, int32_t B, int32_t n, int32_t heads, int32_t head_dim) {
  return (B == 1 || r->batch_stride >= head_dim) && (n == 1 || r->token_stride >= head_dim) && (heads == 1 || r->head_stride >= head_dim);
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

// Groups of head_dim / 16 threads with `each` rows (tokens x heads) to a group, sequences along y.
bool row_grid(const fly_cache_t* c, int32_t B, int32_t n, int threads, int each, dim3* grid) {
  const int64_t per_block = (int64_t)(threads / (c->head_dim / 16)) * each, rows = (int64_t)n * c->kv_heads;
  if (rows > 0x7fffff00) return false;  // (rows of a sequence are counted in 32 bits)
  *grid = dim3((unsigned)((rows + per_block - 1) / per_block), (unsigned)(B < 65535 ? B : 65535));
  return true;
}

template <int D, bool E4M3, bool PAIR>
cudaError_t set_attrs() {
  return cudaFuncSetAttribute(A::attention_kernel<D, E4M3, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, A::Shape<D, E4M3, PAIR>::kSmem);
}
cudaError_t set_attention_attrs() {
  cudaError_t e = cudaSuccess;
  for (cudaError_t x : {set_attrs<64, false, false>(), set_attrs<64, false, true>(), set_attrs<64, true, false>(), set_attrs<64, true, true>(),
                        set_attrs<128, false, false>(), set_attrs<128, false, true>(), set_attrs<128, true, false>(), set_attrs<128, true, true>()})
    if (e == cudaSuccess) e = x;
  return e;
}

// The queries [B, n, heads, D] in boxes of 64 values x the heads of a group x the tokens of a row tile.
bool encode_q(fly_attention* h, CUtensorMap* map, const fly_rows_t* q, const A::Params& p) {
  const cuuint64_t D = (cuuint64_t)h->cfg.head_dim;
  const cuuint64_t dims[4] = {D, (cuuint64_t)p.heads, (cuuint64_t)p.n, (cuuint64_t)p.B};
  const int64_t strides[3] = {q->head_stride, q->token_stride, q->batch_stride};
  cuuint64_t bytes[3];
  for (int i = 0; i < 3; ++i) bytes[i] = 2 * (dims[i + 1] > 1 ? (cuuint64_t)strides[i] : D);  // (of a dimension of one entry: anything)
  const cuuint32_t box[4] = {64, (cuuint32_t)p.group, (cuuint32_t)p.tpt, 1}, one[4] = {1, 1, 1, 1};
  return h->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, q->data, dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pages.  bf16: boxes of eight tokens with all their values, 64 at a time and swizzled.  E4M3: boxes of a page's (or 128) tokens' codes; keys swizzled, values as they lie.
bool encode_pages(fly_attention* h, CUtensorMap* map, const fly_cache_t* c, bool keys) {
  void* const pages = keys ? c->k_pages : c->v_pages;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  const cuuint64_t D = (cuuint64_t)c->head_dim, esz = e4m3 ? 1 : 2;
  const cuuint64_t token = (cuuint64_t)c->token_stride * esz;
  const cuuint64_t head = c->kv_heads > 1 ? (cuuint64_t)c->head_stride * esz : D * esz, page = c->num_pages > 1 ? (cuuint64_t)c->page_stride * esz : D * esz;
  const cuuint64_t tokens = (cuuint64_t)c->page_size, heads = (cuuint64_t)c->kv_heads, count = (cuuint64_t)c->num_pages;
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  if (e4m3) {
    const cuuint64_t dims[4] = {D, tokens, heads, count}, bytes[3] = {token, head, page};
    const cuuint32_t box[4] = {(cuuint32_t)D, (cuuint32_t)(c->page_size < A::kTile ? c->page_size : A::kTile), 1, 1};
    return h->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pages, dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           !keys ? CU_TENSOR_MAP_SWIZZLE_NONE : D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  const cuuint64_t dims[5] = {64, tokens, D / 64, heads, count}, bytes[4] = {token, 128, head, page};
  const cuuint32_t box[5] = {64, 8, (cuuint32_t)(D / 64), 1, 1};
  return h->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, pages, dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool E4M3, bool PAIR>
cudaError_t launch(fly_attention* h, const CUtensorMap* maps, const A::Params& p, cudaStream_t st) {
  using S = A::Shape<D, E4M3, PAIR>;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, (unsigned)h->sm_count, S::kThreads, st, true);
  cfg.dynamicSmemBytes = S::kSmem;
  cudaError_t e = cudaLaunchKernelEx(&cfg, A::attention_kernel<D, E4M3, PAIR>, maps[0], maps[1], maps[2], p);
  if (e != cudaSuccess) return e;
  h->last_launches++;
  if (h->sm_count < 2) return e;
  // (one kernel less: a context of 300 positions 12.0 -> 10.6 us) Nothing is cut where every item is short enough to stay whole, whatever the lengths are.
  if (p.groups <= 32 && (int64_t)p.groups * p.c.kv_heads <= h->sm_count && p.c.capacity <= A::kWholeItem * A::kTile) return e;
  // (blocks for as many cut items as there can be, at most four per SM)
  const int64_t items = (int64_t)p.groups * p.c.kv_heads, most = (items < h->sm_count - 1 ? items : h->sm_count - 1) * (PAIR ? S::kItemRows : p.tpt * p.group) * (D / 4);
  const int64_t blocks = (most + A::kCombineThreads - 1) / A::kCombineThreads;
  fill_launch(&cfg, attr, (unsigned)(blocks < 4 * h->sm_count ? blocks : 4 * h->sm_count), A::kCombineThreads, st, true);
  e = cudaLaunchKernelEx(&cfg, A::attention_combine_kernel<D, S::kItemRows>, p, h->sm_count);
  if (e == cudaSuccess) h->last_launches++;
  return e;
}

}  // namespace

extern "C" {

fly_status_t fly_cache_append(const fly_cache_t* c, int32_t B, int32_t n, const fly_rows_t* k, const fly_rows_t* v,
                              const int32_t* counts, uint32_t* row_flags, void* cuda_stream) {
  fly_status_t s = check_cache(c, B, n);
  if (s != FLY_OK || (s = check_rows(k)) != FLY_OK || (s = check_rows(v)) != FLY_OK) return s;
  if (!aligned(counts, 4) || !aligned(row_flags, 4)) return FLY_ERR_UNSUPPORTED;
  DeviceGuard g(c->device);
  if (!g.ok) return FLY_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, 1, K::kAppendThreads, static_cast<cudaStream_t>(cuda_stream), true);
  if (!row_grid(c, B, n, K::kAppendThreads, 1, &cfg.gridDim)) return FLY_ERR_UNSUPPORTED;
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
  if (!aligned(starts, 4) || !apart(k, B, n, c->kv_heads, c->head_dim) || !apart(v, B, n, c->kv_heads, c->head_dim)) return FLY_ERR_UNSUPPORTED;
  DeviceGuard g(c->device);
  if (!g.ok) return FLY_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  fill_launch(&cfg, attr, 1, K::kReadThreads, static_cast<cudaStream_t>(cuda_stream), true);
  if (!row_grid(c, B, n, K::kReadThreads, 1, &cfg.gridDim)) return FLY_ERR_UNSUPPORTED;
  // Several rows to a group where that still leaves every SM its eight blocks.
  constexpr int R = K::kReadRows;
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, c->device) != cudaSuccess) return FLY_ERR_CUDA;
  const bool several = (int64_t)n * c->kv_heads * B / (K::kReadThreads / (c->head_dim / 16) * R) >= sms * 8;
  if (several && !row_grid(c, B, n, K::kReadThreads, R, &cfg.gridDim)) return FLY_ERR_UNSUPPORTED;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  auto kernel = c->head_dim == 128 ? (e4m3 ? (several ? K::read_kernel<128, true, R> : K::read_kernel<128, true, 1>)
                                           : (several ? K::read_kernel<128, false, R> : K::read_kernel<128, false, 1>))
                                   : (e4m3 ? (several ? K::read_kernel<64, true, R> : K::read_kernel<64, true, 1>)
                                           : (several ? K::read_kernel<64, false, R> : K::read_kernel<64, false, 1>));
  const int aligned_rows = (wide(k, B, n, c->kv_heads) ? 1 : 0) | (wide(v, B, n, c->kv_heads) ? 2 : 0);
  return cudaLaunchKernelEx(&cfg, kernel, view_of(c), rows_of(k), rows_of(v), (int)B, (int)n, starts, aligned_rows) == cudaSuccess ? FLY_OK
                                                                                                                                  : FLY_ERR_CUDA;
}

fly_status_t fly_attention_create(const fly_attention_config_t* c, fly_attention_t** out) {
  if (out) *out = nullptr;
  if (!c || !out) return FLY_ERR_INVALID_ARG;
  if (c->device < 0 || c->max_batch < 1 || c->max_tokens < 1 || c->kv_heads < 1 || c->heads < 1 || c->heads % c->kv_heads != 0 || c->head_dim < 1)
    return FLY_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->heads / c->kv_heads > A::kTileRows || c->max_tokens > kMaxTokens) return FLY_ERR_UNSUPPORTED;
  fly_attention* h = new (std::nothrow) fly_attention();
  if (!h) return FLY_ERR_INVALID_ARG;
  h->cfg = *c;
  DeviceGuard g(c->device);
  cudaStream_t st = nullptr;
  cudaError_t e = g.ok ? cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, c->device) : cudaErrorInvalidDevice;
  if (e == cudaSuccess) e = set_attention_attrs();
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (e == cudaSuccess) e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found);
  if (e == cudaSuccess && !fn) e = cudaErrorUnknown;
  const size_t rows = (size_t)h->sm_count * 2 * (c->max_tokens > A::kTileRows / (c->heads / c->kv_heads) ? 2 * A::kTileRows : A::kTileRows);
  const size_t o_bytes = rows * c->head_dim * sizeof(float), ml_bytes = rows * sizeof(float2), d_bytes = (size_t)h->sm_count * 8 * sizeof(int);
  if (e == cudaSuccess) e = cudaMalloc(&h->part_o, o_bytes + ml_bytes + d_bytes + 128);
  if (e == cudaSuccess) {
    h->part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(h->part_o) + o_bytes);
    h->desc = reinterpret_cast<int*>(h->part_ml + rows);
    h->status = h->desc + (size_t)h->sm_count * 8 + 16;
    // (on a stream of its own: making a handle does not wait for what is queued on the default stream)
    e = cudaStreamCreateWithFlags(&st, cudaStreamNonBlocking);
  }
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (st) cudaStreamDestroy(st);
  if (e != cudaSuccess) {
    if (g.ok) cudaFree(h->part_o);
    delete h;
    return FLY_ERR_CUDA;
  }
  h->encode_tiled = reinterpret_cast<PFN_cuTensorMapEncodeTiled>(fn);
  *out = h;
  return FLY_OK;
}

fly_status_t fly_attention_destroy(fly_attention_t* h) {
  if (!h) return FLY_OK;
  DeviceGuard g(h->cfg.device);
  if (g.ok) cudaFree(h->part_o);
  delete h;
  return FLY_OK;
}

fly_status_t fly_attention_run(fly_attention_t* h, const fly_cache_t* c, const fly_attention_args_t* a, void* cuda_stream) {
  if (!h || !a) return FLY_ERR_INVALID_ARG;
  fly_status_t s = check_cache(c, a->B, a->n);
  if (s != FLY_OK || (s = check_rows(&a->q)) != FLY_OK || (s = check_rows(&a->out)) != FLY_OK) return s;
  const int heads = h->cfg.heads, kv_heads = h->cfg.kv_heads, D = h->cfg.head_dim;
  if (a->B > h->cfg.max_batch || a->n > h->cfg.max_tokens || c->device != h->cfg.device || c->kv_heads != kv_heads || c->head_dim != D)
    return FLY_ERR_INVALID_ARG;
  if (a->window < 0 || a->sinks < 0 || (a->sinks > 0 && a->window == 0)) return FLY_ERR_INVALID_ARG;
  if (!(a->scale >= 0.0) || !std::isfinite(a->scale)) return FLY_ERR_INVALID_ARG;
  if (a->scale > 0x1p127) return FLY_ERR_UNSUPPORTED;  // (infinite in fp32, times log2(e); a score of 0 would become NaN)
  if (!wide(&a->q, a->B, a->n, heads) || !wide(&a->out, a->B, a->n, heads)) return FLY_ERR_UNSUPPORTED;
  if ((a->B > 1 && a->q.batch_stride == 0) || (a->n > 1 && a->q.token_stride == 0) || (heads > 1 && a->q.head_stride == 0))
    return FLY_ERR_UNSUPPORTED;
  if (!aligned(a->counts, 4) || !aligned(a->lse, 4) || !apart(&a->out, a->B, a->n, heads, D)) return FLY_ERR_UNSUPPORTED;
  DeviceGuard g(h->cfg.device);
  if (!g.ok) return FLY_ERR_CUDA;
  A::Params p;
  p.c = view_of(c);
  p.q = rows_of(&a->q);
  p.out = rows_of(&a->out);
  p.lse = a->lse;
  p.counts = a->counts;
  p.B = a->B;
  p.n = a->n;
  p.heads = heads;
  p.group = heads / kv_heads;
  // (a window that no position is outside of is none)
  const bool window = a->window > 0 && (int64_t)a->window < (int64_t)p.c.capacity + a->n;
  p.window = window ? a->window : 0;
  p.sinks = window ? (a->sinks < p.c.capacity ? a->sinks : p.c.capacity) : 0;
  p.scale = A::positive((float)((a->scale == 0.0 ? 1.0 / std::sqrt((double)D) : a->scale) * 1.4426950408889634));
  const int most = A::kTileRows / p.group;  // whole tokens in a row tile
  const bool pair = a->n > most;
  p.tpt = a->n < most ? a->n : most;
  p.tpi = pair ? 2 * p.tpt : p.tpt;
  p.rt = (a->n + p.tpi - 1) / p.tpi;
  const int64_t groups = (int64_t)p.B * p.rt;
  // (tiles of positions are counted in 32 bits, lengths are not known here)
  // What an item takes besides its tiles, in tiles (its queries, the joining of the slots, its end).  us a call at 0 / 2 / 4: 64 sequences of one token
  // 222 / 193 / 191, 16 of nine over e4m3 169 / 158 / 147, window of one token over e4m3 36.4 / 32.6 / 34.7 (3 for e4m3: 151 and 33.0).
  // (193 and 191 are as good as equal: repeated runs differ by 1 % and more.)
  const int item_cost = c->format == FLY_CACHE_E4M3 ? 3 : 2;
  if (groups > 1 << 28 || groups * kv_heads * ((int64_t)p.c.capacity / A::kTile + 2 + item_cost) > 0x7fffffff) return FLY_ERR_UNSUPPORTED;
  p.groups = (int)groups;
  p.item_cost = item_cost;
  p.part_o = h->part_o;
  p.part_ml = h->part_ml;
  p.desc = h->desc;
  p.status = h->status;
  const bool e4m3 = c->format == FLY_CACHE_E4M3;
  CUtensorMap maps[3];
  if (!encode_q(h, &maps[0], &a->q, p) || !encode_pages(h, &maps[1], c, true) || !encode_pages(h, &maps[2], c, false))
    return FLY_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  h->last_launches = 0;
  cudaError_t e = D == 128 ? (e4m3 ? (pair ? launch<128, true, true>(h, maps, p, st) : launch<128, true, false>(h, maps, p, st))
                                   : (pair ? launch<128, false, true>(h, maps, p, st) : launch<128, false, false>(h, maps, p, st)))
                           : (e4m3 ? (pair ? launch<64, true, true>(h, maps, p, st) : launch<64, true, false>(h, maps, p, st))
                                   : (pair ? launch<64, false, true>(h, maps, p, st) : launch<64, false, false>(h, maps, p, st)));
  if (e != cudaSuccess) {
    h->last_cuda_error = (int)e;
    return FLY_ERR_CUDA;
  }
  return FLY_OK;
}

fly_status_t fly_attention_device_status(fly_attention_t* h, void* cuda_stream) {
  if (!h) return FLY_ERR_INVALID_ARG;
  DeviceGuard g(h->cfg.device);
  if (!g.ok) return FLY_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, h->status, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && word != 0) e = cudaMemsetAsync(h->status, 0, sizeof(int), st);
  if (e != cudaSuccess) {
    h->last_cuda_error = (int)e;
    return FLY_ERR_CUDA;
  }
  return word == 0 ? FLY_OK : FLY_ERR_TIMEOUT;
}

fly_status_t fly_attention_selftest_wait(fly_attention_t* h, void* cuda_stream) {
  if (!h) return FLY_ERR_INVALID_ARG;
  DeviceGuard g(h->cfg.device);
  if (!g.ok) return FLY_ERR_CUDA;
  A::attention_selftest_kernel<<<1, 1, 0, static_cast<cudaStream_t>(cuda_stream)>>>(h->status, 2000000ull);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) h->last_cuda_error = (int)e;
  return e == cudaSuccess ? FLY_OK : FLY_ERR_CUDA;
}

int32_t fly_attention_last_launch_count(const fly_attention_t* h) { return h ? h->last_launches : 0; }
int32_t fly_attention_last_cuda_error(const fly_attention_t* h) { return h ? h->last_cuda_error : 0; }

}  // extern "C"
