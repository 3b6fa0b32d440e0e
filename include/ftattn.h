/*
 * ftattn.h -- C ABI of the attention side of a decoder layer on NVIDIA B200 (sm_100a): what stands in front of the
 * expert-cached MoE layer of ftmoe.h in every layer of a served model.  Same library (libftmoe.so), same conventions.
 *
 * The keys and values of all requests live in fixed-size pages.  Per step the caller runs
 *
 *     ft_attn_slots                                        once per step
 *     ft_attn_qk_rope -> ft_attn_forward -> (ft_moe_...)   once per layer
 *
 * slots   : from the requests' lengths, on the device: page allocation and release, block tables, position and cache
 *           slot of every new token, and the work partition of ft_attn_forward.
 * qk_rope : RMS norm of every query and key head, rotation by position, write of keys and values into the cache.
 * forward : causal attention of the step's new tokens (single tokens, chunks, whole prompts, mixed) over the cache.
 *
 * Conventions
 *   - Every function returns an ft_status_t, never aborts, never throws, never traps on the device.
 *   - "dev" pointers are device pointers; streams are cudaStream_t passed as void*.  One host thread per handle, and
 *     the calls of a handle are ordered on the device by the caller (one stream, or events): they share the handle's
 *     work partition and scratch.  No call allocates or synchronises except create, destroy, sync_status.
 *   - Indices found on the device that cannot be (a page id outside the pool, a slot outside the cache, a position
 *     beyond the rotation table, lengths that contradict the host's bounds) are skipped, never followed, and latched
 *     in a device status word: ft_attn_sync_status returns FT_ERR_INVALID_ARG once.
 *     A page id outside the pool in a block table counts as a page of zeros for ft_attn_forward: no other request's
 *     keys and values are read for it.
 *   - T = 0 or n_req = 0 is a no-op (ft_attn_slots and ft_attn_plan still record an empty step, and ft_attn_slots writes
 *     its outputs: q_start[0] = 0, n_free_out, rows of -1).  Arrays without elements may be NULL.
 *
 * Cache of one layer: [n_pages][2][n_kv_heads][page_tokens][head_dim] in the handle's dtype, contiguous, 16-byte aligned,
 *   keys at index 0 and values at index 1 of the second axis.  Slot of a token = page id * page_tokens + offset.
 *   Elements that hold no token of a request may hold anything (NaN and infinities included) and never reach a result.
 * Block table: int32 [n_req][max_pages], entry b of a row = page of the request's tokens b*page_tokens ...
 */
#ifndef FTATTN_H_
#define FTATTN_H_

#include "ftmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ft_attn ft_attn_t; /* opaque: work partition, scratch of split requests, status word */

typedef enum { FT_ATTN_BF16 = 0, FT_ATTN_FP16 = 1 } ft_attn_dtype_t;

typedef struct {
  uint32_t struct_size;   /* = sizeof(ft_attn_config_t) */
  int32_t device;         /* CUDA device ordinal */
  int32_t dtype;          /* ft_attn_dtype_t: queries, keys, values, outputs, norm weights */
  int32_t n_q_heads;      /* Hq, <= 1024 */
  int32_t n_kv_heads;     /* Hkv, divides Hq; query head h reads key/value head h / (Hq/Hkv); Hq/Hkv <= 64 */
  int32_t head_dim;       /* D: 64 or 128 */
  int32_t page_tokens;    /* 16, 32, 64 or 128 */
  int32_t n_pages;        /* pages of a layer's cache, < 2^22; n_pages * page_tokens < 2^31 */
  int32_t max_requests;   /* requests of one step, <= 1024 */
  int32_t max_tokens;     /* new tokens of one step, <= 2^20 */
  int32_t max_pages;      /* columns of the block table; max_pages * page_tokens < 2^31 */
  int32_t window;         /* 0: a token attends to every token up to itself; W > 0: to the W latest ones */
} ft_attn_config_t;

/* Bytes of one layer's cache (0 if the configuration is not supported). */
size_t ft_attn_cache_bytes(const ft_attn_config_t *cfg);

/* FT_ERR_INVALID_ARG: a value out of its range; FT_ERR_UNSUPPORTED: head_dim or page_tokens that is not listed above, or a
 * step whose work units (key blocks of 64 tokens x n_kv_heads, of max_pages * page_tokens tokens for each of max_requests
 * requests, and for each of max_tokens / (2 * floor(128 * Hkv / Hq)) + max_requests pieces) would not be counted in 31 bits;
 * FT_ERR_OOM: no device memory for the scratch. */
ft_status_t ft_attn_create(const ft_attn_config_t *cfg, ft_attn_t **out);
ft_status_t ft_attn_destroy(ft_attn_t *h);

/* Block tables and slot maps of a step.  All arrays DEVICE int32.
 *   in     : new_len[n_req]  new tokens of the request in this step; < 0 = the request is finished
 *            ctx_len[n_req]  tokens it has in the cache
 *            n_free[1]       valid entries of the stack free_pages[n_pages]
 *            max_new, T      HOST bounds: largest new_len, length of position/slot (>= the sum of new_len)
 *   in/out : table[n_req][table_stride]  the first ceil(ctx_len / page_tokens) entries of a row are read, new pages are
 *            appended behind them;  free_pages
 *   out    : q_start[n_req + 1]  first packed row of each request;  kv_len[n_req]  tokens in the cache after the step;
 *            n_free_out[1];  admitted[n_req];  position[T], slot[T]  of every packed token
 * Finished requests first push their pages on the stack (in order of request and page).  A request needs
 * ceil((ctx + new) / page) - ceil(ctx / page) pages; it is admitted if it needs none or if the needs up to and including
 * its own fit on the stack; pages are taken from the top, in order.  A request that is not admitted keeps its state
 * (kv_len = ctx_len): its tokens get position and slot -1, are not written to the cache, and attend to nothing.  A
 * finished request gets kv_len 0 and admitted 0.  Rows of position/slot past the last request's tokens get -1.
 * Counts are not updated in place (n_free_out != n_free, kv_len != ctx_len): the call can be repeated on its inputs. */
ft_status_t ft_attn_slots(ft_attn_t *h, int n_req, int T, int max_new, const int32_t *new_len, const int32_t *ctx_len,
                          int32_t *table, int64_t table_stride, int32_t *free_pages, const int32_t *n_free,
                          int32_t *q_start, int32_t *kv_len, int32_t *n_free_out, int32_t *admitted, int32_t *position,
                          int32_t *slot, void *stream);

/* The work partition alone, for callers that keep their own block tables: request r has the packed rows
 * q_start[r] .. q_start[r+1] - 1 (q_start[0] = 0, DEVICE int32 [n_req + 1]) and kv_len[r] cached tokens, its new ones
 * included (DEVICE int32 [n_req]); max_new >= every request's rows, T >= q_start[n_req] (HOST).  Valid for every
 * ft_attn_forward until the next ft_attn_slots or ft_attn_plan. */
ft_status_t ft_attn_plan(ft_attn_t *h, int n_req, int T, int max_new, const int32_t *q_start, const int32_t *kv_len,
                         void *stream);

/* y = x * rsqrt(mean(x^2) + eps) * w over each query and key head (w_q, w_k DEVICE [D] in the dtype; NULL: no norm), then
 * the rotation (a, b) -> (a cos - b sin, b cos + a sin) of the pairs (i, i + rot_dim/2) or, interleaved, (2i, 2i + 1),
 * i < rot_dim/2, with cos_sin DEVICE float [max_pos][rot_dim] = the cosines, then the sines, of row `position`
 * (rot_dim % 8 == 0, <= D; 0: no rotation).  Computed in float and rounded once.
 *   q [T][Hq][D], k, v [T][Hkv][D]: DEVICE, heads contiguous, *_stride elements from token to token; 8-byte aligned
 *   q_out [T][Hq][D] with q_out_stride (may be q itself); kv_cache: keys and values of the token go to its slot
 * A token with slot < 0 is not written to the cache; one with position < 0 (not admitted, padding) gets zeros in q_out. */
ft_status_t ft_attn_qk_rope(ft_attn_t *h, int T, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                            const void *v, int64_t v_stride, const void *w_q, const void *w_k, float eps,
                            const float *cos_sin, int max_pos, int rot_dim, int interleaved, const int32_t *position,
                            const int32_t *slot, void *q_out, int64_t q_out_stride, void *kv_cache, void *stream);

/* Attention over the requests of the latest ft_attn_slots / ft_attn_plan: row i of a request with n rows stands at
 * position P = kv_len - n + i and attends to the cached tokens j <= P (and j > P - window):
 * out = sum_j softmax_j(scale * q.k_j) v_j, lse = log(sum_j exp(scale * q.k_j)).  A row that attends to nothing gets
 * zeros and lse = -infinity; a row with an infinite positive or NaN score among those it attends to gets NaN in both.
 * The weights are rounded to the dtype before they multiply the values (as matrix operands); scores, maxima and sums are float.
 * A value v_j that is itself infinite or NaN can make rows of the same request and step NaN that do not attend to j (weight 0).
 * Rows of no request are not written.
 *   q, out: DEVICE [T][Hq][D], strides in elements from token to token, 16-byte aligned, strides % 8 == 0
 *           and <= 2^23
 *   lse   : DEVICE float [T][Hq] or NULL
 * FT_ERR_STATE before the first slots/plan call. */
ft_status_t ft_attn_forward(ft_attn_t *h, const void *q, int64_t q_stride, const void *kv_cache, const int32_t *table,
                            int64_t table_stride, void *out, int64_t out_stride, float *lse, float scale, void *stream);

/* Waits for the device and returns (and clears) the latched device status. */
ft_status_t ft_attn_sync_status(ft_attn_t *h);
/* Test hook for the failure path of the bounded device-side waits, as ft_moe_debug_inject: withhold_mask names kernels whose
 * first producer leaves out one copy, wait_polls is the poll limit of every wait from now on (0 = the default, 2^22).  The
 * kernel then gives up, latches FT_ERR_TIMEOUT and runs to completion; ft_attn_sync_status reports it once and makes the
 * handle usable again.  Per process and device; (0, 0) restores normal operation.  Waits for the device. */
enum { FT_ATTN_DEBUG_WITHHOLD_STREAM = 1,   /* attention of requests with few rows */
       FT_ATTN_DEBUG_WITHHOLD_TILE = 2,     /* attention of requests with many rows */
       FT_ATTN_DEBUG_WITHHOLD_ROPE = 4 };   /* norm and rotation of many tokens */
ft_status_t ft_attn_debug_inject(ft_attn_t *h, uint32_t withhold_mask, uint32_t wait_polls);
/* Number of kernels this handle has launched since create. */
ft_status_t ft_attn_launch_count(ft_attn_t *h, uint64_t *out);
/* Text of the CUDA runtime error behind the most recent FT_ERR_CUDA / FT_ERR_OOM of a ft_attn_ call. */
const char *ft_attn_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FTATTN_H_ */
