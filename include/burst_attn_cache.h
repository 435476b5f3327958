/*
 * libburstattn -- rotary positions, a paged key-value cache, the attention of one new token or of a tree of drafted ones over it, and
 * pages and rows of the cache copied.  Same library, same
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
 * Where several next tokens were guessed they are appended together, attend to the cache and to each other as their tree says (burst_attn_tree), and the
 * rows of those that turn out right are moved to the front (burst_attn_cache_keep_rows).  A sequence that is continued in several ways shares its full
 * pages through the table and has its last one copied (burst_attn_cache_copy_pages).
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

#define BURST_TREE_MAX_TOKENS 64

/*
 * What new tokens see of a cache.  Sequence b has tokens[b] of them (device int32 [batch], 0 .. sq, a number outside is taken as the nearest; NULL: sq
 * for all).  Their own rows are the last tokens[b] ones of its rows[b], as an append leaves them; the rows before those are older.
 *   seen      : device, a word of 64 bits for each token, [batch][sq] (stride in words, 0: one tree for all): token i sees new token j iff bit j is
 *               set; bits of tokens that are not there are not looked at.  A token sees itself by its own bit.  NULL: a chain, i sees 0 .. i.
 *   first_row : device int32 [batch][sq] (stride in numbers, 0 broadcasts): token i sees of the older rows those from first_row on and, whatever it says, the
 *               first sink_rows ones of the sequence.  Any number; NULL: 0, all of them.  (A sliding window of w tokens is first_row = position - w + 1;
 *               new tokens are hidden by their bits alone.)
 *   elsewhere : != 0: the new tokens' own rows are not in this cache (a ring's devices but one): every row here is older, seen is not looked at.
 */
typedef struct {
  const uint64_t* seen;
  int64_t seen_stride;
  const int32_t* first_row;
  int64_t first_stride;
  const int32_t* tokens;
  int32_t sink_rows;   /* >= 0 */
  int32_t elsewhere;
} burst_tree_t;

/*
 * Attention of a few new tokens of every sequence over its rows in the cache, each over the rows t that it sees, as a step of the ring gives it:
 *     S_t = scale * q . K_t;  Lse = log sum exp S_t (natural log);  O = sum exp(S_t - Lse) V_t;   without a row O = 0, Lse = -inf.
 * q is bf16 [batch, sq, q_heads, head_dim], o bf16 or fp32 of that shape, lse [batch, q_heads, sq], or NULL: not wanted.  Tokens behind a sequence's last
 * one (padding) are not read, and their rows of o and lse are left as they were.
 * shape: sq is 1 .. BURST_TREE_MAX_TOKENS (more: UNSUPPORTED; a longer chain goes by several calls, each behind its append); sk is a bound on every
 * sequence's rows, the new ones among them, at most table_cols * page_rows (INVALID_ARG): rows at and behind it are not seen.  batch * q_heads * sq above 2^25, or
 * batch * sk of about 2^36 and more: UNSUPPORTED.
 * O is exact to fp32 rounding before it is cast: the numbers exp(S - Lse) are multiplied in the three bf16 parts that their 24 bits are.  Where O is bf16 and
 * sq * q_heads / kv_heads is above 32 they are multiplied in two, which hold them to 2^-16.  A row that is seen by none of a sequence's tokens, or that has no page, may hold anything, NaN too.  An infinity or NaN in a
 * row that one of them sees reaches those that see it, and may reach the sequence's other tokens.  A token's result depends on the other tokens and sequences by
 * roundings in fp32 alone, and where two parts are taken by those of 2^-16 of each number, before O is cast.  o and lse share memory with nothing that the call reads.
 * workspace: burst_attn_tree_workspace_bytes(shape) bytes, 256-byte aligned, contents on entry irrelevant, on return unspecified; calls that share one must be
 * ordered on one stream.  The size depends on batch, sq, the heads, head_dim and sk; it is 0 for some shapes, for which workspace may be NULL.
 */
int64_t burst_attn_tree_workspace_bytes(const burst_shape_t* shape);   /* host only; -1 for an invalid shape */
int burst_attn_tree(const burst_shape_t* shape, const burst_cache_t* cache, const burst_tree_t* tree, const burst_tensor_t* q, const burst_tensor_t* o,
                    const burst_rowvec_t* lse, void* workspace, int64_t workspace_bytes, void* hip_stream);

/*
 * The first rows of pages copied to other pages, in n_layers caches (at most BURST_CACHE_MAX_LAYERS, in as few launches as they allow) that are alike
 * but for where k and v lie: types, strides, n_pages, page_rows (INVALID_ARG otherwise; table, rows and scales are not looked at).  moves: device
 * int32 [n_moves][3]: from, to, and the number of rows (a number outside 0 .. page_rows is taken as the nearest).  A move from or to what is no page does nothing, nor does one
 * from a page to itself.  No page may be the destination of two moves that are carried out, or of one and the source of another.  shape: kv_heads and head_dim are read.
 */
#define BURST_CACHE_MAX_LAYERS 1024
int burst_attn_cache_copy_pages(const burst_shape_t* shape, int32_t n_layers, const burst_cache_t* caches, const int32_t* moves, int64_t n_moves,
                                void* hip_stream);

/*
 * Of each sequence's last new_rows[b] rows (device int32 [batch], 0 .. sq, a number outside is taken as the nearest; NULL: sq) those that stay, moved to the
 * front of them, in n_layers caches as above, which also share one table and its rows: for i < kept[b] (device int32 [batch], taken as at most new_rows[b]) row i of them
 * becomes what row from[b][i] of them was before the call (device int32 [batch][sq], stride in numbers, 0 broadcasts).  A row may be named more than once, in
 * any order; where from is outside 0 .. new_rows[b] - 1, or either row has no page, the row stays as it is, and so do rows from kept[b] on.  rows itself
 * is not changed: the program takes new_rows[b] - kept[b] off it afterwards.  No two of the rows may be one row of a page.
 * shape: batch, kv_heads, head_dim and sq are read; sq is at most BURST_TREE_MAX_TOKENS (UNSUPPORTED).
 */
int burst_attn_cache_keep_rows(const burst_shape_t* shape, int32_t n_layers, const burst_cache_t* caches, const int32_t* from, int64_t from_stride,
                               const int32_t* new_rows, const int32_t* kept, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* BURST_ATTN_CACHE_H */
