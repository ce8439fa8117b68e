/*
 * blendstep_stream.h - operators for streams: sequences that decode for so long that a layer looks at their last
 * `window` tokens and their first `sinks` ones only, whose pages behind the window are given up, that are forked
 * where a prompt is answered several ways, and that are so few at the end of a pool that the step is bound by
 * the weights.  They work on the paged cache and the contexts of blendstep.h, whose conventions hold here:
 * device pointers and streams belong to the caller, every function returns BS_OK or a negative bs_status, the
 * message is kept for bs_last_error of the context, nothing throws, a malformed argument is an error code before
 * anything is enqueued.  All device calls are asynchronous on the given stream.
 *
 *   bs_window_*       sliding-window attention with sinks over the paged cache, and the rotary positions (with
 *                     several axes) and the append that go before it; both work from one plan of the step
 *   bs_w4_*           products of few rows with 4-bit weights that have a scale per group of inputs
 *   bs_pages_*        book-keeping of a cache's pages: fork, extend, trim, free, compact (host only)
 *   bs_kv_copy_pages, bs_kv_compact    the copies behind it, in the pools of all layers at once
 */
#ifndef BLENDSTEP_STREAM_H
#define BLENDSTEP_STREAM_H

#include "blendstep.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- window attention, rotary positions and append -----------------------------------------------------------
 *
 * A plan holds what one step needs on the device: where rows stand, where their keys and values go, the pages that
 * each row sees, how the work is divided.  It is made once per step and used by every layer whose window and sinks
 * it has.  bs_window_plan may allocate device memory (it keeps the largest size seen); the calls that use the plan
 * allocate nothing and can be captured into a graph.  A graph holds the plan of its capture: planning again
 * on the same handle ends it.  Calls on one handle must not overlap in time on different streams (they share its partial
 * states), and a call on another stream than the plan's must be ordered behind it by the caller.  The context must outlive its
 * plans. */
typedef struct bs_window bs_window;

/* A page-table entry whose page was given up (bs_pages_trim): no row of the step sees a token of it. */
#define BS_PAGE_NONE (-1)

int bs_window_create(bs_ctx *ctx, bs_window **out); /* a host-only context: bs_window_plan validates and divides only */
void bs_window_destroy(bs_window *w);

/* Plans one step.  `batch`: n_seq, n_rows, row_start, kv_len, page_start and page_ids as in blendstep.h (n_prefill and the
 * nodes are not looked at), with these differences:
 *   - a sequence may have any number of rows, none included, and kv_len may be smaller than their number: row j of
 *     n stands at position p = kv_len - n + j, and rows with p < 0 (padding in front, idle slots of a batch with
 *     kv_len 0) see nothing, append nothing, and their attention output is zero;
 *   - entries of pages that no row of the step sees or appends to may be BS_PAGE_NONE;
 *   - kv_len is not limited by max_positions (positions are, see below).
 * A row at position p sees token t of its sequence if t <= p and (t > p - window or t < sinks).  window >= 1;
 * sinks >= 0; either may exceed every length.
 *
 * positions: HOST [n_axes][n_rows], the position of each row along each axis (time, height, width for images and
 * video; all equal for text), each in [0, max_positions) of the context.  axis_of_pair: HOST [head_dim / 2], the axis whose position
 * turns the pair (i, i + head_dim / 2); it allows sections as well as axes in turn.  Both NULL with n_axes = 0: every pair is turned by the row's
 * position in its sequence, as in bs_blend_step (rows in front of their sequence: 0).  1 <= n_axes <= 8 otherwise. */
int bs_window_plan(bs_window *w, const bs_batch *batch, int64_t n_pages, int32_t window, int32_t sinks,
                   int32_t n_axes, const int32_t *positions, const int32_t *axis_of_pair, void *stream);

/* Turns the queries and keys of fused rows and appends keys and values to the pages of their positions.
 * qkv: device bf16, row r at qkv + r * qkv_stride elements: Hq query heads, Hkv key heads, Hkv value heads of head_dim each.
 * q: device bf16, row r at q + r * q_stride, Hq heads; may be qkv itself (the same stride: turned in place), and must not overlap it otherwise.
 * Rows are 16-byte aligned: strides are multiples of 8 elements.  Angles: pos * rope_theta^(-2i/dh) from the
 * context's table (evaluated in 64 bits, kept in 32); products in 32 bits, rounded once. */
int bs_rope_append(bs_window *w, const void *qkv, int64_t qkv_stride, void *q, int64_t q_stride, void *kv_pool, void *stream);

/* Attention of the plan's rows over the pool (this step's keys and values are in it already).  q, out: device bf16, Hq heads a row,
 * strides as above; out may be q itself where both strides are equal, and must not overlap it otherwise.  Softmax statistics and sums in 32
 * bits (they begin at -1e30: a row that sees nothing above that gives zeros, as one that sees nothing);
 * probabilities enter their product with V in bf16.  Tokens that no row of a sequence's call sees do not reach any result, whatever bits
 * their slots hold; a NaN or an infinity in a value that one row sees may also reach
 * rows of the same sequence that do not see it. */
int bs_window_attention(bs_window *w, const void *q, int64_t q_stride, void *out, int64_t out_stride, const void *kv_pool,
                        void *stream);

/* How the last planned step is divided, for tests (host only). */
typedef struct bs_window_parts {
  int32_t units;         /* narrow work: units of one KV head, at most 16 / group rows and a run of pages */
  int32_t longest_pages; /* pages of the longest of them */
  int32_t split_rows;    /* rows whose pages are split over several units and joined */
  int32_t wide_blocks;   /* wide work: blocks of rows of longer segments (per group of heads) */
  int32_t wide_cut;      /* of these, blocks whose pages are cut into ranges and joined */
  int32_t waves;         /* wavefronts of a workgroup that share a unit's pages (1, 2, 4 or 8) */
  int64_t pages;         /* pages that the units and blocks name */
} bs_window_parts;
int bs_window_division(const bs_window *w, bs_window_parts *out);

/* ---- 4-bit products --------------------------------------------------------------------------------------------
 * y[m, n] = sum over groups g of scale[n, g] * sum over k in g of x[m, k] * (w[n, k] - zero[n, g]),  w in 0 .. 15.
 * group is 32, 64 or 128; k a multiple of it; n any; m >= 0.  Meant for few rows (up to 64 the weights come from
 * memory once; beyond, once for every 64 rows). */

/* Bytes of the laid-out weight; 0 for a shape that is not supported. */
int64_t bs_w4_bytes(int64_t n, int64_t k, int32_t group, int32_t with_zeros);

/* Lays a weight out for bs_w4_linear, once.  packed: device uint8 [n, k / 2], the even input in the low four bits.
 * scales: device bf16 [n, k / group].  zeros: device uint8 [n, k / group], values 0 .. 15, or NULL (8 everywhere).
 * weight: device, bs_w4_bytes bytes, 16-byte aligned. */
int bs_w4_pack(bs_ctx *ctx, const void *packed, const void *scales, const void *zeros, int64_t n, int64_t k, int32_t group,
               void *weight, void *stream);

/* x: device bf16, row i at x + i * x_stride elements (x_stride a multiple of 8, 16-byte aligned); y: device bf16, row i at
 * y + i * y_stride; with_zeros as the weight was packed.  Sums in 32 bits, y rounded once.  (They carry an offset of the weights that
 * cancels: an infinity in a row of x makes its outputs NaN, and sums of 143 |x| have to be in range.)  The calls on one context share
 * a workspace and must not overlap in time on different streams. */
int bs_w4_linear(bs_ctx *ctx, const void *x, int64_t x_stride, const void *weight, int64_t m, int64_t n, int64_t k, int32_t group,
                 int32_t with_zeros, void *y, int64_t y_stride, void *stream);

/* ---- pages -------------------------------------------------------------------------------------------------------
 * Book-keeping of the pages of a cache (page_size 16), on the host.  Every sequence has a page table; pages are
 * counted by reference and the free ones are handed out smallest number first.  A call that fails changes
 * nothing.  Copies that a call asks for are returned as pairs (src, dst): they are to be made in the pools of all layers
 * (bs_kv_copy_pages) before the next step writes; within one call no dst is a src or another dst. */
typedef struct bs_pages bs_pages;
int bs_pages_create(int32_t n_pages, bs_pages **out);
void bs_pages_destroy(bs_pages *p);
const char *bs_pages_last_error(const bs_pages *p); /* NULL: of the last failed bs_pages_create of this thread */
/* n new, empty sequences; their ids (smallest free ids first) to ids[n]. */
int bs_pages_open(bs_pages *p, int32_t n, int32_t *ids);
/* `children` new sequences for each of the n parents (all of the first parent's first), which share every page with it;
 * their ids to out[n * children]. */
int bs_pages_fork(bs_pages *p, const int32_t *parents, int32_t n, int32_t children, int32_t *out);
/* Makes room for tokens[i] >= 0 further tokens of sequence ids[i], in order (an id may come once).  Where a
 * sequence's last page is open (not full) and shared, it gets a copy of its own, which is a pair.  src, dst: arrays of n
 * entries; *n_copies pairs are written.  BS_ENOMEM: not enough free pages. */
int bs_pages_extend(bs_pages *p, const int32_t *ids, const int32_t *tokens, int32_t n, int32_t *src, int32_t *dst, int32_t *n_copies);
/* Gives up the pages that no later row of the sequences sees through `window` and `sinks` (their entries become BS_PAGE_NONE). */
int bs_pages_trim(bs_pages *p, const int32_t *ids, int32_t n, int32_t window, int32_t sinks);
/* Ends sequences; their ids are free again. */
int bs_pages_free(bs_pages *p, const int32_t *ids, int32_t n);
/* Moves the live pages to the numbers below their count, each number above it to the smallest free one in ascending order, and
 * rewrites the tables.  src, dst: arrays of n_pages entries. */
int bs_pages_compact(bs_pages *p, int32_t *src, int32_t *dst, int32_t *n_moves, int32_t *n_live);
/* Lengths, and tables one behind the other (page_start[n + 1]; page_ids of `room` entries).  With page_ids = NULL or room for fewer than
 * page_start[n] entries only the lengths and page_start are written. */
int bs_pages_tables(const bs_pages *p, const int32_t *ids, int32_t n, int32_t *tokens, int32_t *page_start, int32_t *page_ids, int64_t room);
int bs_pages_stats(const bs_pages *p, int32_t *n_free, int32_t *n_sequences);

/* Copies page src[i] to page dst[i], i < n, in each of n_pools pools of n_pages pages.  pools, src, dst: HOST.  No dst may
 * be a src or another dst (BS_EINVAL). */
int bs_kv_copy_pages(bs_ctx *ctx, void *const *pools, int32_t n_pools, int64_t n_pages, const int32_t *src, const int32_t *dst,
                     int32_t n, void *stream);
/* The same for page tables that the caller holds: the pages that tables[0 .. n) name (entries repeat where pages are
 * shared; BS_PAGE_NONE is kept) are moved as by bs_pages_compact, in each pool, and the tables with the new
 * numbers written to tables_out (which may be tables).  *n_live: pages named. */
int bs_kv_compact(bs_ctx *ctx, void *const *pools, int32_t n_pools, int64_t n_pages, const int32_t *tables, int64_t n,
                  int32_t *tables_out, int32_t *n_live, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BLENDSTEP_STREAM_H */
