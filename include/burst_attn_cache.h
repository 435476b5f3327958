/*
 * libburstattn -- rotary positions, a paged key-value cache, and the attention of one new token over it.  Same library, same
 * conventions as burst_attn.h: device pointers owned by the caller, nothing allocated, retained or synchronised, work enqueued
 * on the given stream only, every argument checked on the host before any launch, BURST_OK (0) or a negative burst_status_t.
 *
 * A chunk may be without rows (sq = 0): burst_attn_rope and burst_attn_cache_append then check what they are given and do nothing, and the pointers of
 * its tensors and positions may be NULL.
 *
 * A model turns the queries and keys of a device's chunk by their positions before the ring's attention (burst_attn_rope), and turns
 * the gradients that the backward step leaves in fp32 back again (the same call, inverse).  A sequence that is to be continued keeps its
 * turned keys and its values in pages (burst_attn_cache_append); every further token attends to them (burst_attn_decode).  A cache that is
 * sharded over the devices of a ring is decoded by each device over its own rows; burst_attn_lse_merge joins the (O, Lse) pairs.
 */
#ifndef BURST_ATTN_CACHE_H
#define BURST_ATTN_CACHE_H

#include <stdint.h>

#include "burst_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A third type of burst_tensor_t, for the cache alone: e4m3 (4 exponent bits, 3 of mantissa, largest number 448, no infinity). */
#define BURST_F8E4M3 2

#define BURST_ROPE_MAX_AXES 3

/*
 * A rotation by positions.  The first rotary_dim elements of a head are rotary_dim / 2 pairs; pair i is elements
 * (i, i + rotary_dim / 2), or with adjacent != 0 (2i, 2i + 1), and is turned by the angle
 *     a_i = positions[axis_of_pair[i]][b][s] * inv_freq[i]:    (x1, x2) -> (x1 cos a - x2 sin a, x2 cos a + x1 sin a).
 * The elements behind them are copied.  Text has one axis; images and video have a position on each of two or three (time, height,
 * width), and each pair belongs to one of them, in runs or in turns as axis_of_pair says.
 *   rotary_dim  : a positive multiple of 16, at most head_dim (0 < rotary_dim: INVALID_ARG otherwise; not a multiple of 16: UNSUPPORTED).
 *   inv_freq    : fp32 [rotary_dim / 2], device; any values.
 *   positions   : int32 [n_axes][batch][rows], device, rows contiguous, strides in elements (0 broadcasts); any values, negative too.
 * Angles are formed in 64 bits, by three roundings, so that far positions keep their place on the circle: sine and cosine are off by at most
 * 2^-24 + 3 * 2^-53 |a| (a in radians: 1e-7 up to 10^8, 8e-7 at position 2^31 with frequency 1; without meaning from 10^15 on).
 */
typedef struct {
  int32_t n_axes;     /* 1 .. BURST_ROPE_MAX_AXES */
  int32_t rotary_dim;
  int32_t adjacent;
  int32_t _pad;
  const float* inv_freq;
  const int32_t* positions;
  int64_t stride_axis, stride_b;   /* of positions, >= 0 */
  uint8_t axis_of_pair[64];        /* entries below rotary_dim / 2 are read; each below n_axes */
} burst_rope_t;

/*
 * Turns the heads of a chunk: q -> q_out, and with k != NULL k -> k_out, in one launch.  inverse != 0 turns back (by -a), which is
 * also the gradient: with dQ, dK of the backward step as q and k the result is the gradient of what was turned.  Inputs and
 * outputs are bf16 or fp32, each on its own; a result is rounded once.  An output may be its input itself (same pointer, strides and type:
 * the rotation in place); otherwise outputs must not share memory with inputs or each other.
 * shape: batch, q_heads, kv_heads, head_dim and sq (rows of the chunk, of q and of k) are read.  batch * sq of 2^31 or more: UNSUPPORTED.
 */
int burst_attn_rope(const burst_shape_t* shape, const burst_rope_t* rope, const burst_tensor_t* q, const burst_tensor_t* q_out,
                    const burst_tensor_t* k, const burst_tensor_t* k_out, int32_t inverse, void* hip_stream);

/*
 * A paged cache.  k and v are [page, row, kv_head, head_dim] (stride_b is a page's stride, stride_s a row's), bf16 or e4m3, of one type and
 * with the same strides (UNSUPPORTED otherwise); pointers and strides are multiples of 16 bytes.  Row t of sequence b is row
 * t % page_rows of page table[b * table_stride + t / page_rows].  rows[b] is the number of rows that sequence b has, 0 .. table_cols *
 * page_rows; a number outside is taken as the nearest of these.  An entry of the table that is no page (negative, or n_pages and
 * more) is no error: its rows are not written by an append, and not seen by the attention.
 * e4m3 holds numbers over a scale of their head: the value is number * k_scale[kv_head] (v_scale); NULL: 1.  The scales are the
 * caller's, positive; numbers beyond +-448 are stored as +-448 (infinities too), NaN stays NaN.  With bf16 the scales must be NULL.
 * Pages of a multiple of 16 rows are read fastest, and heads whose rows lie one after the other in a page (head stride above row stride).
 */
typedef struct {
  burst_tensor_t k, v;
  int64_t n_pages;         /* 1 .. 2^31 - 1 */
  int32_t page_rows;       /* 1 .. 2^20 */
  int32_t table_cols;      /* pages a sequence may have, 1 .. 2^30; table_cols * page_rows at most 2^30 */
  const int32_t* table;    /* device */
  int64_t table_stride;    /* >= table_cols, or 0: one row of the table for all sequences */
  const int32_t* rows;     /* device, [batch] */
  const float* k_scale;    /* device, [kv_heads], or NULL */
  const float* v_scale;
} burst_cache_t;

/*
 * Puts new rows into the cache.  k and v are bf16 [batch, sq, kv_heads, head_dim]; sequence b brings its first new_rows[b] rows (device
 * int32 [batch], 0 .. sq, a number outside is taken as the nearest; NULL: sq for all), which become its rows rows[b] - new_rows[b] ..
 * rows[b] - 1: rows counts them already, so that one update of it serves all layers of a model, and the attention after it.
 * rope, if not NULL, turns the keys; its positions are [n_axes][batch][sq], those of the new rows.  q, if not NULL, is bf16
 * [batch, sq, q_heads, head_dim] and is turned into q_out (bf16; may be q itself) by the same positions, in the same launch.
 * Rows of q_out at and behind new_rows[b] are left as they were, and so is everything in the cache but the new rows.  No two new rows
 * may fall on one row of a page.  shape: batch, q_heads, kv_heads, head_dim and sq are read.  batch * sq of 2^31 or more: UNSUPPORTED.
 */
int burst_attn_cache_append(const burst_shape_t* shape, const burst_cache_t* cache, const burst_tensor_t* k, const burst_tensor_t* v,
                            const int32_t* new_rows, const burst_rope_t* rope, const burst_tensor_t* q, const burst_tensor_t* q_out,
                            void* hip_stream);

/*
 * Attention of one new token of every sequence over its rows in the cache, as a step of the ring gives it: for query head h and the rows
 * t = first_row[b] .. rows[b] - 1 (first_row: device int32 [batch], a negative number is taken as 0; NULL: 0; a sliding window is
 * first_row = rows - window)
 *     S_t = scale * q . K_t;  Lse = log sum exp S_t (natural log);  O = sum exp(S_t - Lse) V_t;   without a row O = 0, Lse = -inf.
 * q is bf16 [batch, 1, q_heads, head_dim], o bf16 or fp32 of that shape, lse [batch, q_heads, 1], or NULL: not wanted.
 * shape: sq must be 1; sk is a bound on every sequence's rows, at most table_cols * page_rows (INVALID_ARG): rows at and behind it are
 * not seen.  batch * q_heads above 2^21, or batch * sk of about 2^36 and more: UNSUPPORTED.  Work is dealt by the rows that are there, not by
 * the bound; but a bound that keeps all keys and values of a head within 256 KiB (512 with 256 (sequence, key head) pairs and more) makes the call
 * one launch instead of two.  O is exact to fp32 rounding before it is cast: the numbers
 * exp(S - Lse) are multiplied in the three bf16 parts that their 24 bits are.  An infinity among the values that are seen is its element of O
 * for every query head whose weight there is 2^-90 of the largest or more (below that it may be NaN, as it is where infinities of both signs meet).  A row's result depends on the other sequences of the batch by roundings in fp32 alone.
 * Rows that are not seen may hold anything, NaN too.  o and lse share memory with nothing that the call reads.
 * workspace: burst_attn_decode_workspace_bytes(shape) bytes, 256-byte aligned, contents on entry irrelevant, on return unspecified; calls
 * that share one must be ordered on one stream.  The size depends on batch, the heads, head_dim and sk; it is 0 for some shapes, for which
 * workspace may be NULL.
 */
int64_t burst_attn_decode_workspace_bytes(const burst_shape_t* shape);   /* host only; -1 for an invalid shape */
int burst_attn_decode(const burst_shape_t* shape, const burst_cache_t* cache, const burst_tensor_t* q, const int32_t* first_row,
                      const burst_tensor_t* o, const burst_rowvec_t* lse, void* workspace, int64_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* BURST_ATTN_CACHE_H */
