/*
 * libburstattn -- sequence-level fusion of the language-modelling head and the loss function
 * (Sec. 3.3, Eq. 9, Alg. 3), the second single-device kernel family of the method.  Same library,
 * same conventions as burst_attn.h: every data pointer is DEVICE memory unless marked host, the
 * caller owns every buffer, the library allocates nothing, retains nothing, does not synchronise
 * and enqueues only on the given stream; all argument checks run on the host before any launch;
 * calls return BURST_OK (0) or a negative burst_status_t.
 *
 * For hidden states H_last (N x d), head weights W_head (v x d) and targets Y (N):
 *   Logits = H_last W_head^T;  Lse_i = log sum_j exp(Logits_ij);  loss_i = Lse_i - Logits_i,Y_i
 *   dLogits = grad_scale * (exp(Logits - Lse) - E),  E_ij = 1 iff j == Y_i
 *   dH = dLogits W_head;   dW = dLogits^T H_last
 * computed one sequence tile of tile_tokens rows at a time (the B_s of Alg. 3): the logits of the
 * tile are kept in the workspace between the forward sweep and the backward sweep, so nothing of
 * size N x v is ever stored and no logit is computed twice.  E is subtracted: the algorithm prints
 * it added, which is not the gradient of the loss it prints.  A target outside [0, v) marks an
 * ignored token: loss 0, no gradient.
 */
#ifndef BURST_LM_HEAD_H
#define BURST_LM_HEAD_H

#include <stdint.h>

#include "burst_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int64_t n_tokens;    /* N >= 0: rows of H_last on this device */
  int64_t d_model;     /* d: a positive multiple of 256 */
  int64_t vocab;       /* v >= 1 */
  int64_t tile_tokens; /* B_s: a positive multiple of 256; the workspace grows with it, the number
                          of passes over dW shrinks with it */
  float grad_scale;    /* gradient of the caller's scalar w.r.t. each token's loss (1: sum, 1/N: mean) */
  int32_t _pad;
} burst_lm_head_shape_t;

/* Bytes of workspace burst_lm_head_loss needs for this shape (n_tokens and grad_scale play no
 * part), or -1 for an invalid shape.  Host only. */
int64_t burst_lm_head_workspace_bytes(const burst_lm_head_shape_t* shape);

/*
 * Alg. 3, forward and backward in one call.
 *   h_last : bf16 [N][ld_h], w_head : bf16 [v][ld_w]  (row-major, leading dimensions in elements,
 *            multiples of 8, >= d; base pointers 16-byte aligned); y : int64 [N].  With N = 0
 *            the per-token pointers (h_last, y, loss, lse, d_h) are not looked at.
 *   loss   : fp32 [N], written.  lse : fp32 [N], written; may be NULL.
 *   d_h    : [N][ld_dh], BURST_F32 or BURST_BF16 (burst_dtype_t), OVERWRITTEN; NULL: not wanted.
 *   d_w    : fp32 [v][ld_dw]; accumulate_dw != 0 adds to its contents, else it is overwritten;
 *            NULL: not wanted.  With both gradients NULL only the forward sweep runs.
 *   workspace : at least burst_lm_head_workspace_bytes(shape) bytes, 256-byte aligned; contents
 *            on entry are irrelevant, contents on return are unspecified.  Calls that share a
 *            workspace must be ordered on one stream.
 * Non-finite inputs give non-finite outputs, possibly also in other rows of the same tile.
 * Errors: BURST_ERR_INVALID_ARG (null / misaligned pointers, bad sizes or leading dimensions,
 * workspace too small), BURST_ERR_UNSUPPORTED (d not a multiple of 256, sizes beyond 2^31 - 1
 * rows or a workspace row beyond 2^31 bytes), BURST_ERR_HIP (launch failed).
 */
int burst_lm_head_loss(const burst_lm_head_shape_t* shape, const void* h_last, int64_t ld_h,
                       const void* w_head, int64_t ld_w, const int64_t* y, float* loss, float* lse,
                       void* d_h, int32_t d_h_dtype, int64_t ld_dh, float* d_w, int64_t ld_dw,
                       int32_t accumulate_dw, void* workspace, int64_t workspace_bytes, void* hip_stream);

/*
 * The same computation for callers that cannot allocate device memory or hand over a workspace of
 * their own: code running under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Arguments, results and errors are those of burst_lm_head_loss without the workspace
 * pair: the scratch memory is an array built into the library's code object, 256 MiB on a GPU from the
 * first call there until the process ends (the HIP runtime loads this code object, by default, when it is
 * first needed, under capture too; a process that makes no such call has none of it).  The call itself
 * allocates nothing and frees nothing, on the host or on the device.
 *   - A shape whose burst_lm_head_workspace_bytes() exceeds 64 MiB is refused with BURST_ERR_SCRATCH and
 *     nothing is enqueued (64 MiB holds e.g. tile_tokens = 256 with a 32000-word vocabulary and d = 4096);
 *     choose a smaller tile_tokens or use burst_lm_head_loss.  burst_lm_head_static_scratch_bytes()
 *     returns this limit, not the size of the array, whose rest is there to join short tiles.
 *   - Sequence tiles of 256 tokens get what the array holds: they are joined, and contractions are split
 *     where few work-groups would run, which changes the order in which fp32 sums are taken; longer tiles
 *     are taken as asked for and give the bits of burst_lm_head_loss.
 *   - The array used is that of the GPU that is current on the calling thread when the call is
 *     made; the stream must belong to that GPU.
 *   - Every call on a GPU shares that GPU's array, which keeps whatever the last call left in it
 *     (no call depends on its previous contents).  Calls that may overlap on one GPU -- different
 *     streams, or this entry point from two threads -- race on it: order them on one stream.
 */
int64_t burst_lm_head_static_scratch_bytes(void);
int burst_lm_head_loss_noalloc(const burst_lm_head_shape_t* shape, const void* h_last, int64_t ld_h,
                               const void* w_head, int64_t ld_w, const int64_t* y, float* loss, float* lse,
                               void* d_h, int32_t d_h_dtype, int64_t ld_dh, float* d_w, int64_t ld_dw,
                               int32_t accumulate_dw, void* hip_stream);

/*
 * Scores of tokens from logits that the program has (of drafted or generated tokens, of a prompt, of answers that are trained on).  With
 * x = scale * logits (scale: 1 / temperature):
 *   lse_i = log sum_j exp x_ij;  logp_i = x_i,y_i - lse_i;  entropy_i = - sum_j p_ij log p_ij,  p_ij = exp(x_ij - lse_i);
 *   top_ids_i: the n_top words of the largest logits, the largest first, among equal ones (0 and -0 are) the lowest index first; top_logp_i their log probabilities.
 *   logits : [n_tokens][ld], BURST_BF16 or BURST_F32, 16-byte aligned, ld >= vocab, any number (rows that are multiples of 16 bytes are read a little faster).
 *   y      : int64 [n_tokens]; a word outside [0, vocab) marks an ignored token: logp 0.  NULL with logp == NULL.
 *   logp, lse, entropy : fp32 [n_tokens], each NULL if not wanted.  top_logp fp32, top_ids int64 : [n_tokens][n_top], each NULL if not wanted.
 * Exponentials, logp and top_logp are of differences from the row's largest logit: words and whole rows at large finite numbers (-1e10, the type's lowest) have the scores of these formulas;
 * a lse beyond the largest fp32 number is an infinity.
 * Words at -inf (masked ones) have no share; where all are, lse = logp = top_logp = -inf and entropy = 0.  A NaN or +inf among a token's logits makes its scores NaN; with a NaN
 * its top_ids are words, but no particular ones.
 * workspace: burst_lm_head_scores_workspace_bytes(shape) bytes, 256-byte aligned, or NULL where that is 0; contents on entry irrelevant; calls that share one must be ordered
 * on one stream.  With n_tokens = 0 pointers are not looked at.
 * Errors: INVALID_ARG; UNSUPPORTED beyond 64 n_top, 2^30 words or 2^25 tokens.
 */
#define BURST_SCORES_MAX_TOP 64
typedef struct {
  int64_t n_tokens;   /* >= 0 */
  int64_t vocab;      /* >= 1 */
  int32_t n_top;      /* 0 .. 64, at most vocab */
  float scale;        /* positive, finite */
} burst_scores_shape_t;

int64_t burst_lm_head_scores_workspace_bytes(const burst_scores_shape_t* shape);   /* host only; -1 for an invalid shape */
int burst_lm_head_scores(const burst_scores_shape_t* shape, const void* logits, int32_t logits_dtype, int64_t ld, const int64_t* y, float* logp, float* lse,
                         float* entropy, float* top_logp, int64_t* top_ids, void* workspace, int64_t workspace_bytes, void* hip_stream);

/*
 * The gradient of the logits from those of the scores (fp32, of the shapes above, each NULL if there is none, not all of them):
 *   d_logits_ij = scale * ( p_ij (g_lse_i - g_logp_i - sum_k g_top_ik - g_entropy_i (log p_ij + entropy_i)) + g_logp_i [j = y_i] + sum_k g_top_ik [j = top_ids_ik] )
 * lse, and entropy with g_entropy, are those that burst_lm_head_scores gave; y comes with g_logp, top_ids with g_top.  A word outside [0, vocab) takes its gradient with it, among
 * top_ids too; one that is named several times gets the sum.  Where lse is -inf the gradient is 0; where |lse| is above 4096, of which an fp32 number says too little for p, the row's own
 * sum is formed again (such rows take several times as long).  d_logits: [n_tokens][ld_d], bf16 or fp32, overwritten
 * (words 0 .. vocab - 1 of each row); it may be logits itself (same type and ld), else they share no memory.
 */
int burst_lm_head_scores_bwd(const burst_scores_shape_t* shape, const void* logits, int32_t logits_dtype, int64_t ld, const int64_t* y, const float* lse,
                             const float* entropy, const int64_t* top_ids, const float* g_logp, const float* g_lse, const float* g_entropy, const float* g_top,
                             void* d_logits, int32_t d_logits_dtype, int64_t ld_d, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
