/*
 * blendstep_bits.h - the two resources of a blended step in fewer bits: a paged cache in four bits, which is what its
 * memory-bound rows read, and products of 8-bit integers, which is what its compute-bound rows do.  The conventions are those of
 * blendstep.h and blendstep_stream.h: device pointers and streams belong to the caller, every function returns BS_OK or a negative
 * bs_status, the message is kept for bs_last_error of the context, nothing throws, a malformed argument is an error code before
 * anything is enqueued, all device calls are asynchronous on the given stream.
 *
 *   bs_window_cache      which cache the plans of a bs_window are for: bs_rope_append and bs_window_attention of
 *                        blendstep_stream.h then write and read a pool in four bits
 *   bs_kv4_*             sizes, conversion and copies of such a pool's pages
 *   bs_w8_*              rows as 8-bit integers, and their product with a weight in 8-bit integers
 */
#ifndef BLENDSTEP_BITS_H
#define BLENDSTEP_BITS_H

#include "blendstep_stream.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- a cache in four bits ----------------------------------------------------------------------------------------
 * Pages of 16 tokens as in blendstep.h, with codes 0 .. 15 in place of bf16 numbers.  The keys (turned by their positions, in 32 bits) and
 * the values of a token and KV head are cut into groups of `group` channels: 32, 64 or 128, at most head_dim.  A group has two bf16
 * numbers, scale and mid, and code c stands for mid + scale (c - 8):
 *     mid   = the place of code 8 where 0 .. 15 span the group's least and greatest value, rounded to bf16
 *     scale = the smallest bf16 number, at least 2^-126, with which the codes reach both
 *     c     = round((v - mid) / scale) + 8, ties to even
 * so that no value is further than scale / 2 from what is kept of it, and equal bf16 values (zeros among them) are kept as they are.
 * A group that holds a NaN or an infinity, or whose values are further apart than 32-bit numbers reach, stands for NaN throughout.
 * A page takes n_kv_heads (16 head_dim + 128 head_dim / group) bytes: 3.2 to 3.8 times less than in bf16.  Bytes of zero stand for zeros. */

/* Bytes of a page; 0 for a group that is not supported. */
int64_t bs_kv4_page_bytes(const bs_ctx *ctx, int32_t group);

/* The cache that the steps planned on `w` from now on are for: bits 16 (group 0; what a new bs_window has), or 4 with the group's size.
 * Ends the planned step.  With four bits kv_pool of bs_rope_append and bs_window_attention is such a pool, 16-byte aligned.  All
 * that blendstep_stream.h says of them holds, but:
 *   - probabilities are rounded to bf16 after a multiplication with the scales of values
 *   - a query with an infinity gives NaN
 *   - sums carry 16 of every code, which cancel: 31 times the sum of |q| over a group, the same times a key's scale, |mid| times that sum, and 31 times a value's scale
 *     have to be in range; and a probability times a scale is a bf16 number, which keeps fewer digits below 2^-126
 *   - the wide_blocks of bs_window_division are units of one KV head too, of about eight times the rows of a narrow unit, with all of their pages. */
int bs_window_cache(bs_window *w, int32_t bits, int32_t group);

/* k, v: device bf16, token-major [n_pages][16][n_kv_heads][head_dim], 16-byte aligned; kv_pool: n_pages pages in four bits, n_pages * n_kv_heads
 * below 2^24.  kv4_unpack gives what the codes stand for, rounded to bf16. */
int bs_kv4_pack(bs_ctx *ctx, const void *k, const void *v, void *kv_pool, int64_t n_pages, int32_t group, void *stream);
int bs_kv4_unpack(bs_ctx *ctx, const void *kv_pool, void *k, void *v, int64_t n_pages, int32_t group, void *stream);

/* bs_kv_copy_pages and bs_kv_compact for pools in four bits. */
int bs_kv4_copy_pages(bs_ctx *ctx, void *const *pools, int32_t n_pools, int64_t n_pages, int32_t group, const int32_t *src, const int32_t *dst,
                      int32_t n, void *stream);
int bs_kv4_compact(bs_ctx *ctx, void *const *pools, int32_t n_pools, int64_t n_pages, int32_t group, const int32_t *tables, int64_t n,
                   int32_t *tables_out, int32_t *n_live, void *stream);

/* ---- products of 8-bit integers ----------------------------------------------------------------------------------
 * y[m, n] = scales[m] weight_scales[n] * sum over k of q[m, k] w[n, k].  Sums are exact; k is a multiple of 16 up to 131072; m and n any. */

/* Rows as 8-bit integers, of activations (a scale for each token) or of a weight (a scale for each output): scale = the greatest magnitude
 * of the row / 127 (at least 2^-100 / 127), q = x / scale to the nearest integer, ties to even, in 32 bits.  A row with a NaN or an infinity: its scale is
 * NaN and its integers 0, so that all of its results are NaN.
 * x: device bf16, row i at x + i * x_stride elements (x_stride a multiple of 8, 16-byte aligned).  q: device int8 [m, k], 16-byte aligned; scales: device
 * float [m]. */
int bs_w8_quantize(bs_ctx *ctx, const void *x, int64_t x_stride, int64_t m, int64_t k, void *q, float *scales, void *stream);

/* q: device int8 [m, k], weight: device int8 [n, k] (any values of either, -128 included), 16-byte aligned; scales: device float [m], weight_scales: device float [n];
 * y: device bf16, row i at y + i * y_stride, rounded once; it must not overlap what is read.  The calls on one context, those of bs_w8_linear_rows too, share a
 * workspace and must not overlap in time on different streams. */
int bs_w8_linear(bs_ctx *ctx, const void *q, const float *scales, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
                 int64_t y_stride, void *stream);

/* How bs_w8_linear divides a product, for tests (host only): rows and outputs of a workgroup, ranges of k that are added up by a second kernel. */
int bs_w8_division(bs_ctx *ctx, int64_t m, int64_t n, int64_t k, int32_t *rows, int32_t *outputs, int32_t *ranges);

/* Both for rows of bf16 (as for bs_w8_quantize), in one launch where rows are few.  scratch: device, bs_w8_scratch_bytes(m, k) bytes (0: may be NULL),
 * 16-byte aligned, the call's own until its work is done. */
int64_t bs_w8_scratch_bytes(int64_t m, int64_t k);
int bs_w8_linear_rows(bs_ctx *ctx, const void *x, int64_t x_stride, const void *weight, const float *weight_scales, int64_t m, int64_t n, int64_t k, void *y,
                      int64_t y_stride, void *scratch, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BLENDSTEP_BITS_H */
