/*
 * ftdense.h -- C ABI of what a decoder's step has besides its attention (ftattn.h) and its experts (ftmoe.h) on NVIDIA B200
 * (sm_100a).  Same library (libftmoe.so), same conventions.
 *
 *     ft_dense_add_norm     between two blocks: the block's output joins the residual stream, the next block's input is normed
 *     ft_dense_w4_forward   a projection or the output head with 4-bit weights and group scales (single tokens to whole prompts)
 *     ft_dense_logprobs     from the logits: log probabilities of given tokens, entropy, the most likely alternatives
 *
 * Conventions
 *   - Every function returns an ft_status_t, never aborts, never throws, never traps on the device.
 *   - "dev" pointers are device pointers; streams are cudaStream_t passed as void*.  One host thread per handle.  The kernels have no
 *     workspace: calls of a handle may run at the same time on several streams or from several captured graphs, as far as their
 *     own inputs and outputs allow.  No call allocates or synchronises except create, destroy, sync_status.
 *   - Sizes of zero tokens are a no-op (pointers may then be NULL); strides are in elements, from token to token.
 *   - A call that is refused launches nothing and writes nothing.
 */
#ifndef FTDENSE_H_
#define FTDENSE_H_

#include "ftmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ft_dense ft_dense_t; /* opaque: device, status word, counters */

typedef enum { FT_DENSE_BF16 = 0, FT_DENSE_FP16 = 1, FT_DENSE_FP32 = 2 } ft_dense_dtype_t;

ft_status_t ft_dense_create(int device, ft_dense_t **out);
ft_status_t ft_dense_destroy(ft_dense_t *h);

/* u  = y,  or with FT_DENSE_NORM_POST  y * rsqrt(mean(y^2) + eps) * (w_offset + w_post)
 * r' = res_scale * res + y_scale * gate * u                                   -> res_out (if given)
 * h  = r' * rsqrt(mean(r'^2) + eps) * (w_offset + w_pre)                      -> out (if given)
 * over rows of d <= 16384 elements.  y, w_post, gate, w_pre and out are of `dtype` (bf16 or fp16), res and res_out of `res_dtype`
 * (the same, or fp32).  Computed in float, r' and h each rounded once (h from the r' that is not rounded yet);
 * a mean whose squares leave the range of float is taken of the row times a power of two.
 *   y [T][d] or NULL (then r' = res_scale * res);  res [T][d] or NULL (then r' = y_scale * gate * u); not both
 *   gate NULL (one), else its element (t, i) stands at gate[t * gate_stride + i * gate_step], gate_step 0 or 1: a gate per element,
 *        per token (gate_step 0), per channel (gate_stride 0)
 *   w_post, w_pre [d] or NULL (no weights: the factor is 1, whatever w_offset says)
 *   res_out may be res, out may be y (the same rows with the same stride); no other overlap.
 * Any alignment of whole elements; rows whose addresses, strides and d are multiples of 16 bytes are read in 16-byte pieces. */
enum { FT_DENSE_NORM_POST = 1 };
ft_status_t ft_dense_add_norm(ft_dense_t *h, int T, int d, int dtype, int res_dtype, int flags, const void *y, int64_t y_stride,
                              const void *res, int64_t res_stride, const void *gate, int64_t gate_stride, int gate_step,
                              const void *w_post, const void *w_pre, float w_offset, float eps, float res_scale, float y_scale,
                              void *res_out, int64_t res_out_stride, void *out, int64_t out_stride, void *stream);

/* 4-bit weights with group scales: w[n][k] = scale[n][k / group] * (code[n][k] - zero[n][k / group]), codes 0 .. 15, zero points 0 .. 15
 * (8 where none are given), group 32, 64 or 128, k a multiple of it and <= 65536, n <= 2^24.
 * ft_dense_w4_pack lays them out once, into an image of ft_dense_w4_bytes (0: not supported) DEVICE bytes, 16-byte aligned:
 *   codes DEVICE [n][k / 2] bytes, codes_stride bytes from row to row, the even k in the low half of a byte;
 *   scales DEVICE [n][k / group] of `dtype` (bf16 or fp16), zeros DEVICE [n][k / group] bytes or NULL (values above 15 count as 15).
 * An image is for activations of the scales' type. */
size_t ft_dense_w4_bytes(int64_t n, int64_t k, int group, int has_zeros);
ft_status_t ft_dense_w4_pack(ft_dense_t *h, int64_t n, int64_t k, int group, int dtype, const uint8_t *codes, int64_t codes_stride,
                             const void *scales, const uint8_t *zeros, void *image, void *stream);

/* y[t][i] = sum_k x[t][k] * w[i][k] + bias[i].  x DEVICE [T][k] of `dtype`, 16-byte aligned, x_stride a multiple of 8 and < 2^38; T <= 2^20; bias
 * DEVICE [n] of `dtype` or NULL; y DEVICE [T][n] of out_dtype (`dtype` or fp32), any alignment of whole elements.  Up to 16 tokens, and for fp32
 * results at any number, the codes less their zero point are multiplied exactly, sums are float, and scales are applied to the sums of a
 * group in float (a group's sum without its scale has to be a float too: x beyond 10^35 may give infinities).  For 16-bit results of more tokens
 * each weight is rounded once to `dtype` before it is multiplied (an error of the size of the result's own rounding); rows with a scale above 1/15 of
 * the type's largest value, whose weights it may not hold, are then computed in the exact form all the same, slowly.  y is rounded once; it overlaps
 * none of the inputs.  n, k, group, dtype and has_zeros must be those of the image. */
ft_status_t ft_dense_w4_forward(ft_dense_t *h, int T, int64_t n, int64_t k, int group, int dtype, int has_zeros, const void *x,
                                int64_t x_stride, const void *image, const void *bias, void *y, int64_t y_stride, int out_dtype,
                                void *stream);

/* With l_i = scale * logits[t][i] (0 < scale <= 2^126) and lse = log(sum_i exp(l_i)):
 *   logprob[t][j] = l_i - lse for i = tokens[t][j], j < n_tokens   (a negative token is none: 0)
 *   entropy[t]    = -sum_i p_i log(p_i),  p_i = exp(l_i - lse)
 *   top_ids[t][j], top_logprobs[t][j], j < top_k <= 32: the largest logits in descending order, the lowest id first among equals,
 *                   and their log probabilities
 * logits DEVICE [T][vocab] bf16, fp16 or fp32, vocab <= 2^30, `stride` elements from row to row, any alignment of whole elements; tokens
 * DEVICE int32, tokens_stride from row to row; outputs DEVICE float (ids int32), contiguous, each may be NULL (top_ids and
 * top_logprobs: both, or neither with top_k 0; logprob goes with tokens).
 * A logit of -infinity has probability 0 and is no alternative: where fewer than top_k are left, ids are -1 and log probabilities
 * -infinity.  A row of nothing but -infinity: entropy 0, log probabilities -infinity.  A row that holds NaN or +infinity has no
 * distribution: its results are NaN, its ids -1.  A token >= vocab gets NaN and is latched: ft_dense_sync_status returns
 * FT_ERR_INVALID_ARG once. */
ft_status_t ft_dense_logprobs(ft_dense_t *h, int T, int64_t vocab, int dtype, const void *logits, int64_t stride, float scale,
                              const int32_t *tokens, int64_t tokens_stride, int n_tokens, float *logprob, float *entropy, int top_k,
                              int32_t *top_ids, float *top_logprobs, void *stream);

/* Waits for the device and returns (and clears) the latched device status. */
ft_status_t ft_dense_sync_status(ft_dense_t *h);
/* Test hook for the failure path of the bounded device-side waits, as ft_moe_debug_inject: withhold_mask names kernels whose first producer
 * leaves out one copy, wait_polls is the poll limit of every wait from now on (0 = the default, 2^22).  The kernel then gives up, latches
 * FT_ERR_TIMEOUT and runs to completion; ft_dense_sync_status reports it once.  Per process and device; (0, 0) restores normal operation.
 * Waits for the device. */
enum { FT_DENSE_DEBUG_WITHHOLD_STREAM = 1,   /* 4-bit products of few tokens */
       FT_DENSE_DEBUG_WITHHOLD_TILE = 2 };   /* 4-bit products of many tokens */
ft_status_t ft_dense_debug_inject(ft_dense_t *h, uint32_t withhold_mask, uint32_t wait_polls);
/* Number of kernels this handle has launched since create. */
ft_status_t ft_dense_launch_count(ft_dense_t *h, uint64_t *out);
/* Text of the CUDA runtime error behind the most recent FT_ERR_CUDA / FT_ERR_OOM of a ft_dense_ call. */
const char *ft_dense_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FTDENSE_H_ */
