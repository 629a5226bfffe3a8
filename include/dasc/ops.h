/*
 * dasc/ops.h -- the operators a serving engine runs on the states of dasc.h.
 *
 * dasc.h stores, restores and refreshes recurrent states; the calls here use them:
 *
 *   dasc_linear_attn    linear attention with a decay for each head (the gated delta rule
 *                       of GDN heads, or the plain rule), from and into pool states, for
 *                       prompts, single tokens and drafted tokens
 *   dasc_verify_drafts  accepts or rejects drafted tokens against the target's probabilities,
 *                       from given random numbers
 *   dasc_block_norm     the norms before and after a block, with its gate and residual scale
 *
 * A recurrent state cannot be cut back to an earlier token as a KV cache can.  A speculative
 * step therefore runs dasc_linear_attn over the drafted tokens with no destination slots,
 * verifies, and runs it again without an output over the tokens that were kept
 * (lens = n_emitted), which advances the states.
 *
 * The conventions of dasc.h hold: status codes, no exceptions; every argument that the host
 * can see is checked before any launch; the caller owns all memory; calls are asynchronous
 * on the given stream, allocate nothing and keep nothing.  Forward only.
 */
#ifndef DASC_OPS_H
#define DASC_OPS_H

#include "../dasc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear attention with a decay for each head ------------------------------------ */

/* Token streams of one call.  Tokens of all requests lie one after another (row t of every
 * tensor belongs to token t); strides are in elements, the last dimension is contiguous. */
typedef struct dasc_linear_io {
  const uint16_t *q;  /* bf16 bits [n_tokens, Hqk, dk]; may be NULL if o is              */
  const uint16_t *k;  /* bf16 bits [n_tokens, Hqk, dk]                                   */
  const uint16_t *v;  /* bf16 bits [n_tokens, H, dv]                                     */
  const float *g;     /* log-decays [n_tokens, H]; a stride of 0 repeats a value         */
  const float *beta;  /* [n_tokens, H]: the delta rule; NULL: the plain rule             */
  uint16_t *o;        /* bf16 bits [n_tokens, H, dv]; NULL: states only                  */
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;
  int64_t g_tok, g_head, beta_tok, beta_head, o_tok, o_head;
} dasc_linear_io;

/* Device workspace of dasc_linear_attn for these sizes (0 for many).  It does for every call of
 * this shape with no more requests and tokens than these and none longer, so that one allocation
 * serves an engine's largest batch and all smaller ones.  delta: whether beta is given.
 * Errors: DASC_E_INVAL (NULL, n_req < 1, n_tokens < 0, max_len < 0), DASC_E_SHAPE. */
int dasc_linear_attn_workspace_bytes(const dasc_shape *shape, int32_t n_req, int64_t n_tokens,
                                     int32_t max_len, int32_t delta, size_t *bytes);

/* For each request i < n_req and each head h of layer `layer`, over the request's tokens t in
 * order, with S' = S^T as in dasc.h and key head h / (H / Hqk):
 *     S~  = exp(g_t) S'_{t-1}
 *     u_t = v_t (plain rule)   or   beta_t (v_t - S~^T k_t) (delta rule)
 *     S'_t = S~ + k_t u_t^T
 *     o_t = scale * S'_t^T q_t
 * A request's tokens are rows cu_seqlens[i] .. cu_seqlens[i + 1] - 1, of which the first
 * lens[i] are taken if lens is given (a lens outside the range is clamped to it, and so are
 * cu_seqlens to [0, n_tokens]).  A request without tokens carries its state over.
 *   states: device fp32 pool [n_pool, L, H, dk, dv], 16-byte aligned.
 *   src_slot: device int32 [n_req], slot of S'_0; an index outside [0, n_pool), -1 say, means
 *     zero.  NULL: all zero.
 *   dst_slot: device int32 [n_req], slot that receives the last state; an index outside
 *     [0, n_pool) means that it is not written.  NULL: none is written.  A slot may be a
 *     request's source and destination at once; no two requests may share a destination, and
 *     none may have another's source as its destination.
 *   cu_seqlens: device int32 [n_req + 1], ascending.  lens: device int32 [n_req] or NULL.
 *   max_len: tokens of the longest request, as the caller knows it.  It chooses between the
 *     token-by-token and the chunked form and decides nothing else: results do not depend on it
 *     beyond rounding (and an infinite query's own outputs, infinite in one form, may be NaN in
 *     the other).
 *   io: q, k, v and o 16-byte aligned, their strides multiples of 8 elements (o and v: of 4);
 *     all strides >= 0.  o must not overlap an input, nor its rows (token, head) each other: they
 *     lie dv or more apart, all heads of a token (or tokens of a head) before the next one's.
 *     Rows of o of tokens that no request
 *     takes are not written.
 *   workspace: device, at least dasc_linear_attn_workspace_bytes, 16-byte aligned (may be NULL
 *     if that is 0); overlapping calls must not share one.
 * Log-decays may be any value: -inf clears the state, and a state of zero stays zero whatever it
 * grows by.  What is not finite stays where the rule has it: an infinity or NaN of a token reaches
 * its own and later outputs of its request, heads and columns, no others.  Columns that end so, and
 * heads with log-decays above 0.17, are taken token by token at any length: right, but slow.
 * Heads may share a key head; keys and queries are taken as they are.
 * Precision: values and outputs are bf16; states, sums and decays fp32 (running sums of
 * log-decays 64-bit), and states are as good as fp32 arithmetic makes them.  The chunked form
 * holds what only an output needs to 16 bits a factor before the output's rounding to bf16: an
 * output whose terms cancel is good to 2^-14 |scale| |q_t| |column of S'_t|.
 * Errors: DASC_E_INVAL (NULL shape, states, io or cu_seqlens; k, v or g NULL with n_tokens > 0; q
 * NULL with o given; neither o nor dst_slot given with n_tokens > 0; misalignment, a bad stride
 * or rows of o that overlap; layer out of [0, L), n_req < 1, n_tokens < 0 or above 2^31 - 1,
 * max_len < 0, n_pool < 1, scale not finite), DASC_E_SHAPE (bad shape, dv % 4 != 0),
 * DASC_E_WORKSPACE, DASC_E_UNSUPPORTED (arch KDA, whose decay is by channel; dk not in
 * {16, 32, 64, 128} or dv > 256), DASC_E_HIP. */
int dasc_linear_attn(const dasc_shape *shape, int32_t layer, float *states, int64_t n_pool,
                     const int32_t *src_slot, const int32_t *dst_slot, const dasc_linear_io *io,
                     const int32_t *cu_seqlens, const int32_t *lens, int32_t n_req,
                     int64_t n_tokens, int32_t max_len, float scale, void *workspace,
                     size_t workspace_bytes, dasc_stream_t stream);

/* ---- verification of drafted tokens -------------------------------------------------- */

#define DASC_DTYPE_BF16 0
#define DASC_DTYPE_F16  1
#define DASC_DTYPE_F32  2

/* Device workspace of dasc_verify_drafts: partial sums of each request's row.
 * Errors: DASC_E_INVAL (NULL bytes, n_req < 0, vocab < 1), DASC_E_SHAPE (vocab above 2^24). */
int dasc_verify_drafts_workspace_bytes(int32_t n_req, int64_t vocab, size_t *bytes);

/* Speculative sampling: for each request r, with n = n_draft[r] drafted tokens x_0 .. x_{n-1}
 * (n_draft NULL: n = max_draft), target probabilities p_0 .. p_n and the draft model's
 * q_0 .. q_{n-1}:
 *     x_i is accepted iff u_accept[r][i] * q_i(x_i) < p_i(x_i), the product rounded to fp32;
 *     a = the number accepted before the first that is not;
 *     w = max(p_a - q_a, 0) if a < n (the difference rounded to fp32), p_n if a = n;
 *     out_tokens[r] = x_0 .. x_{a-1}, y, -1, ...;   n_emitted[r] = a + 1,
 * with y drawn from w by u_sample[r].  draft NULL stands for drafts without probabilities:
 * q_i is 1 at x_i and, in w, takes x_i's weight away.
 * The draw is exact: W_v = floor(min(w_v, 1) 2^36) (0 for negative values and NaN),
 * R = floor(u_sample 2^24) clamped to [0, 2^24 - 1], y = the lowest v with
 * W_0 + .. + W_v > floor(R * sum W / 2^24).  Integer sums make it independent of the order in
 * which the row is summed; a probability below 2^-36 is never drawn.  If all weights are 0,
 * w = p_a; if those are too, y = -1.  A drafted token outside [0, vocab) is not accepted.  n_draft
 * is clamped to max_draft; a negative one marks a request to leave out: all its tokens -1, n_emitted 0.
 *   target: device [n_req, max_draft + 1, vocab], draft: device [n_req, max_draft, vocab] or
 *     NULL; both of type dtype (DASC_DTYPE_*), rows contiguous, strides of requests and
 *     positions in elements.  Aligned to their element.
 *   draft_tokens: device int32 [n_req, max_draft]; u_accept: device fp32 [n_req, max_draft];
 *     u_sample: device fp32 [n_req]; n_draft: device int32 [n_req] or NULL.
 *   out_tokens: device int32 [n_req, max_draft + 1]; n_emitted: device int32 [n_req].  Neither
 *     may overlap an input.
 * Errors: DASC_E_INVAL (NULL or misaligned pointer, n_req < 0, max_draft < 0, bad dtype or
 * stride), DASC_E_SHAPE (vocab < 1 or above 2^24, max_draft above 1023), DASC_E_WORKSPACE,
 * DASC_E_HIP. */
int dasc_verify_drafts(int32_t n_req, int32_t max_draft, int64_t vocab, int32_t dtype,
                       const void *target, int64_t target_req, int64_t target_pos,
                       const void *draft, int64_t draft_req, int64_t draft_pos,
                       const int32_t *draft_tokens, const int32_t *n_draft,
                       const float *u_accept, const float *u_sample, int32_t *out_tokens,
                       int32_t *n_emitted, void *workspace, size_t workspace_bytes,
                       dasc_stream_t stream);

/* ---- norms before and after a block --------------------------------------------------- */

#define DASC_ACT_NONE    0
#define DASC_ACT_SIGMOID 1
#define DASC_ACT_SILU    2

/* Rows are [outer, inner, dim]: row (i, j) of a tensor starts at i * _out + j * _in elements,
 * dim is contiguous.  A stride of 0 repeats a row of an input. */
typedef struct dasc_norm_io {
  const void *y;      /* the block's output, dtype                                        */
  const void *gate;   /* dtype, or NULL: no gate                                          */
  const void *x;      /* the residual, res_dtype, or NULL: none is added                  */
  void *x_out;        /* res_dtype, or NULL: not written                                  */
  void *h_out;        /* dtype, the normed input of the next block, or NULL               */
  const void *w_post; /* [dim] weight of the norm after the block, or NULL: no such norm  */
  const void *w_pre;  /* [dim] weight of the norm before the next, needed with h_out      */
  const void *channel_scale; /* [dim], or NULL                                            */
  int64_t y_out, y_in, gate_out, gate_in, x_row_out, x_row_in;
  int64_t xo_out, xo_in, h_row_out, h_row_in;
  int64_t outer;
  int32_t inner, dim;
  int32_t dtype;      /* DASC_DTYPE_* of y, gate and h_out                                */
  int32_t res_dtype;  /* dtype, or DASC_DTYPE_F32: of x and x_out                         */
  int32_t w_dtype;    /* dtype, or DASC_DTYPE_F32: of the weights and channel_scale       */
  int32_t act;        /* DASC_ACT_*; with a gate SIGMOID or SILU                          */
  float scale, eps;
} dasc_norm_io;

/* For each row, in fp32, each output rounded once:
 *     b  = act(gate) * y / sqrt(mean(y^2) + eps) * w_post   (without w_post: act(gate) * y)
 *     x' = x + scale * channel_scale * b                    -> x_out
 *     h  = x' / sqrt(mean(x'^2) + eps) * w_pre              -> h_out (from x' before its rounding)
 * With x NULL, x' = scale * channel_scale * b: the gated norm of a linear-attention layer's
 * heads is y = o, [n_tokens, H, dv].  All rows share the weights.  x_out or h_out may be x, y or
 * gate itself (same address, type and strides); otherwise outputs overlap neither inputs nor each
 * other.
 * outer = 0 is an empty call.
 * Errors: DASC_E_INVAL (NULL io or y, neither x_out nor h_out, h_out without w_pre, a bad
 * dtype, act or stride, a gate without act or the reverse, a pointer not aligned to its element,
 * output rows that overlap, eps < 0, eps or scale not finite), DASC_E_SHAPE (outer < 0, inner or
 * dim < 1, outer * inner above 2^31 - 1), DASC_E_UNSUPPORTED (dim > 32768), DASC_E_HIP. */
int dasc_block_norm(const dasc_norm_io *io, dasc_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DASC_OPS_H */
