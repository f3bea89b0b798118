/*
 * fly_cache.h - C ABI of the paged key/value cache next to the verification step of fly_verify.h, and of the attention of a
 * chunk of new tokens over it, for NVIDIA B200 (sm_100a).
 *
 * A round of speculative decoding runs a chunk of n = K+1 tokens per sequence (the last token and the K drafts that
 * fly_pld_draft or another drafter proposes) through the target: in every layer the chunk's keys and values are appended to
 * the cache (fly_cache_append) and its queries attend to what is there (fly_attention_run); the last layer's hidden states go
 * into the fused LM head of fly_verify_run.  Afterwards the cache keeps the s = accept_len tokens of the chunk that the
 * sequence keeps: the caller sets lengths[b] += accept_len[b] - rollback[b], and the next round's append overwrites the rest.
 * fly_cache_read gives a range of the cache back as plain tensors.
 *
 * Conventions
 *   - As in fly_verify.h: pointers marked "dev" are device memory of the named device, owned by the caller; the calls are
 *     asynchronous on `cuda_stream`, allocate nothing and never synchronise; no function throws, aborts or traps.  What the
 *     host can see is refused with a return code before anything is launched.  lengths, counts, starts and block_table are device data:
 *     no value in them makes a call read or write outside the cache and the caller's buffers (what each bad one does stands
 *     beside it).
 *     They must not change until the step that was given them has ended; if they do, its results mean nothing, but it ends
 *     (attention: with FLY_ERR_TIMEOUT from fly_attention_device_status where its parts no longer agreed on what to do).
 *   - Position p of sequence b is slot p % page_size of page block_table[b][p / page_size].
 *   - The chunk of sequence b starts at position lengths[b]: lengths is what the cache held BEFORE the chunk, in all calls.
 *     lengths[b] has to lie in [0, max_pages * page_size]; another one counts as a sequence without any position: nothing
 *     is written or read for it, and its chunk sees nothing.
 *   - counts (dev [B] or NULL): the tokens of the chunk that sequence b really has, 0 .. n (another value counts as 0); NULL = n for all.
 *     Rows of a chunk from counts[b] on are not written and have no influence, whatever they hold (attention may read its queries there).
 */
#ifndef FLY_CACHE_H_
#define FLY_CACHE_H_

#include "fly_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How a cache holds the keys and values.
 * BF16  as they are.
 * E4M3  one byte a value, and one byte of scale per token, head and tensor: value = code * 2^(scale - 127).  A row of head_dim values
 *       is written with the smallest scale >= 7 for which its largest magnitude does not exceed 448 * 2^(scale - 127), every
 *       value rounded to the nearest code (ties to even; with scale 247, the largest, to at most 240, since 256 * 2^120 is not
 *       a bf16 number).  The scale is a power of two, so scaling rounds nothing, and what is read back (and what attention
 *       computes with) is exact in bf16.  A row that holds a NaN or an infinity gets scale 255 and reads back as NaN. */
typedef enum { FLY_CACHE_BF16 = 0, FLY_CACHE_E4M3 = 1 } fly_cache_format_t;

typedef struct {
  int32_t device;
  fly_cache_format_t format;
  void* k_pages;            /* dev [num_pages, page_size, kv_heads, head_dim], at the strides below; 16-byte aligned */
  void* v_pages;            /* the same for the values */
  uint8_t* k_scales;        /* dev [num_pages, kv_heads, page_size] contiguous, 8-byte aligned; E4M3 only, else NULL */
  uint8_t* v_scales;
  int32_t num_pages;        /* >= 1 */
  int32_t page_size;        /* tokens per page: a power of two, 8 .. 65536 */
  int32_t kv_heads;         /* >= 1 */
  int32_t head_dim;         /* 64 or 128, contiguous */
  int64_t page_stride;      /* elements from one page, token and head to the next: whole 16-byte units, at least head_dim, any order */
  int64_t token_stride;     /* of the three dimensions (a dimension of one entry may have any stride) */
  int64_t head_stride;
  const int32_t* block_table; /* dev [sequences, max_pages] page ids, rows table_stride entries apart.  A page id outside
                                 [0, num_pages) is never followed: tokens for it are not written, and it is read as a
                                 page that is not visible */
  int64_t table_stride;     /* >= max_pages */
  int32_t max_pages;        /* >= 1; max_pages * page_size <= 2^30 */
  int32_t sequences;        /* rows of block_table and lengths */
  const int32_t* lengths;   /* dev [sequences] */
} fly_cache_t;

/* A bf16 tensor [B, n, heads, head_dim], head_dim contiguous, the other strides in elements (>= 0). */
typedef struct {
  void* data;
  int64_t batch_stride;
  int64_t token_stride;
  int64_t head_stride;
} fly_rows_t;

/* Writes token i of sequence b's chunk to position lengths[b] + i, i < counts[b].
 *   k, v       [B, n, kv_heads, head_dim], at any alignment of their type
 *   row_flags  dev [B, n] or NULL: 0, or bit 5 where the token was not written (its position is past the block table, its page id
 *              is out of range, or lengths[b] is).  Rows from counts[b] on are left as they are.
 * Two tokens of one call must not have the same page and slot.  1 <= B <= cache->sequences, n >= 1. */
fly_status_t fly_cache_append(const fly_cache_t* cache, int32_t B, int32_t n, const fly_rows_t* k, const fly_rows_t* v,
                              const int32_t* counts, uint32_t* row_flags, void* cuda_stream);

/* Reads positions starts[b] .. starts[b] + n - 1 of every sequence (starts dev [B], NULL = 0) into k and v [B, n, kv_heads, head_dim].
 * Exact: both formats hold bf16 values.  Rows of positions that sequence b does not hold - negative ones, those from
 * lengths[b] on, and those on a page whose id is out of range - are left as they are.  Strides of k and v are at least head_dim. */
fly_status_t fly_cache_read(const fly_cache_t* cache, int32_t B, int32_t n, const int32_t* starts, const fly_rows_t* k,
                            const fly_rows_t* v, void* cuda_stream);

/* Attention of a chunk over the cache.  Query head h reads key/value head h / (heads / kv_heads).  Row i of sequence b
 * (position P = lengths[b] + i) sees the positions p <= P that the cache holds - its own and the chunk's earlier ones among
 * them, so append first - and with a window only those with p > P - window or p < sinks:
 *   s_p = scale * <q, k_p>,   lse = ln sum_p e^{s_p},   out = sum_p e^{s_p - lse} v_p.
 * A row that sees nothing, or only scores of -inf, gets out 0 and lse -inf.  Keys and values that a row does not see have no
 * influence on it, whatever they hold.  Products are added up in fp32 (weights rounded to bf16; over E4M3 a query is
 * exact down to 2^-13.8 of the largest of its row and off by at most 2^-21.8 of that, or 2^-134, below), so magnitudes beyond 2^100 may
 * overflow on the way, and a row with scores beyond 2^30, of whose weights fp32 leaves nothing, may come out as NaN.
 * out may be q itself; otherwise the two do not overlap.
 *
 * A handle owns the scratch in which the parts of a long context meet, so steps of one handle run one after the other
 * on the GPU (one handle per stream, as in fly_verify.h), and graphs captured with it too. */
typedef struct fly_attention fly_attention_t;

typedef struct {
  int32_t device;
  int32_t max_batch;   /* largest B, >= 1 */
  int32_t max_tokens;  /* largest n, >= 1 */
  int32_t heads;       /* a multiple of kv_heads, at most 128 times it */
  int32_t kv_heads;
  int32_t head_dim;    /* 64 or 128 */
} fly_attention_config_t;

fly_status_t fly_attention_create(const fly_attention_config_t* config, fly_attention_t** out);
fly_status_t fly_attention_destroy(fly_attention_t* handle);

typedef struct {
  int32_t B;              /* 1 .. max_batch, at most cache->sequences */
  int32_t n;              /* 1 .. max_tokens */
  fly_rows_t q;           /* [B, n, heads, head_dim]; 16-byte aligned, strides whole 16-byte units and not 0 */
  fly_rows_t out;         /* the same shape, strides at least head_dim; rows from counts[b] on are left as they are */
  float* lse;             /* dev [B, n, heads] contiguous or NULL */
  const int32_t* counts;  /* dev [B] or NULL */
  int32_t window;         /* 0: everything up to the row's own position; >= 1: the last `window` positions (its own among them) */
  int32_t sinks;          /* >= 0: first positions that stay visible; only with a window */
  double scale;           /* > 0 and at most 2^127, or 0 for 1 / sqrt(head_dim) */
} fly_attention_args_t;

/* One kernel, and another one for the parts of long contexts where there may be any.  FLY_ERR_UNSUPPORTED where the sequences' tables
 * together span more than 2^31 tiles of 128 positions per key/value head and row tile. */
fly_status_t fly_attention_run(fly_attention_t* handle, const fly_cache_t* cache, const fly_attention_args_t* args,
                               void* cuda_stream);

/* The kernel waits on hardware barriers (loads, tensor cores); every such wait is bounded (200 ms without a step forward of the
 * block, however long a context is).  If one runs out, the kernel
 * records it and returns without hanging, and rows that it could not form are NaN (out and lse).  This call synchronises
 * `cuda_stream` and returns FLY_ERR_TIMEOUT if that happened since the last call (the record is cleared), else FLY_OK.  While
 * a record is pending, every further step of the handle comes back as NaN. */
fly_status_t fly_attention_device_status(fly_attention_t* handle, void* cuda_stream);

/* Self-test of that mechanism, safe to run anywhere: enqueues a one-thread kernel that waits, with a 2 ms limit, on a barrier
 * that nothing completes.  It gives up and returns normally, and fly_attention_device_status reports FLY_ERR_TIMEOUT. */
fly_status_t fly_attention_selftest_wait(fly_attention_t* handle, void* cuda_stream);

/* Number of kernels the last fly_attention_run enqueued, and the cudaError_t of the last failed CUDA call (0 if none). */
int32_t fly_attention_last_launch_count(const fly_attention_t* handle);
int32_t fly_attention_last_cuda_error(const fly_attention_t* handle);

#ifdef __cplusplus
}
#endif
#endif /* FLY_CACHE_H_ */
