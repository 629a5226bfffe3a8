/*
 * dasc/cache.h -- the full-attention layers and the beams of a hybrid model.
 *
 * dasc.h and dasc/ops.h serve the recurrent states of linear-attention layers.  The layers
 * between them attend over a paged cache of keys and values, and a search with several beams
 * reorders both:
 *
 *   dasc_cache_append  rotates new queries and keys by their positions (of one or several axes)
 *                      and writes the keys and values to their slots of the cache
 *   dasc_cache_attn    attention of each request's new tokens over its pages: single tokens,
 *                      drafts, chunks of a prompt, whole prompts
 *   dasc_beam_select   the best continuations over beams and vocabulary
 *   dasc_move_slots    pool slots (states of dasc.h, or pages) reordered all at once
 *
 * A step appends, then attends: the keys of the new tokens are read from the cache.  Drafts that
 * a verification rejects need no undoing here; their slots are overwritten, and kv_lens decides
 * what is seen.
 *
 * The conventions of dasc.h hold: status codes, no exceptions; every argument that the host
 * can see is checked before any launch; the caller owns all memory; calls are asynchronous
 * on the given stream, allocate nothing and keep nothing.  Forward only.
 */
#ifndef DASC_CACHE_H
#define DASC_CACHE_H

#include "ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One layer's cache: position p of page b, head h, starts at b * _page + p * _tok + h * _head
 * elements, its head_dim elements are contiguous.  Any order of the three is possible: pages
 * with tokens or with heads first, pages of several layers side by side.  Here and below
 * any stride from 0 on will do for a dimension of one element. */
typedef struct dasc_kv_cache {
  void *k, *v;              /* [n_pages, page_size, n_kv_heads, head_dim], dtype            */
  int64_t k_page, k_tok, k_head, v_page, v_tok, v_head;
  int64_t n_pages;
  int32_t page_size, n_kv_heads, head_dim;
  int32_t dtype;            /* DASC_DTYPE_BF16 or DASC_DTYPE_F16                            */
} dasc_kv_cache;

/* ---- append --------------------------------------------------------------------------- */

/* New tokens [n_tokens, heads, head_dim], the cache's dtype; strides in elements. */
typedef struct dasc_append_io {
  const void *q;            /* [n_tokens, n_q_heads, head_dim], or NULL: keys and values only */
  void *q_out;              /* the rotated queries; NULL if q is                            */
  const void *k, *v;        /* [n_tokens, n_kv_heads, head_dim]                             */
  const int64_t *slots;     /* [n_tokens]: page * page_size + place in the page             */
  const int32_t *pos;       /* [n_tokens, n_axes], or NULL if rot is 0                      */
  const float *inv_freq;    /* [rot / 2], or NULL if rot is 0                               */
  const int32_t *pair_axis; /* [rot / 2], the axis whose position turns a pair; NULL: 0     */
  int64_t q_tok, q_head, qo_tok, qo_head, k_tok, k_head, v_tok, v_head, pos_tok, pos_axis;
  int64_t n_tokens;
  int32_t n_q_heads, n_axes;
  int32_t rot;              /* elements of a head that are rotated, its first; even; 0: none */
  int32_t adjacent;         /* 0: pairs (i, i + rot / 2); 1: pairs (2 i, 2 i + 1)           */
} dasc_append_io;

/* For each token t and each pair i of the first rot elements of each head of q and k,
 *     angle = pos[t][pair_axis[i]] * inv_freq[i]
 *     (x, y) -> (x cos - y sin, x sin + y cos)
 * and the rest as it is; queries to q_out, keys and values to the cache at slots[t].  A token
 * whose slot lies outside [0, n_pages * page_size), -1 say, is not stored (a padded batch); its
 * query is rotated all the same.  Everything else in the cache is left as it was.
 * The angle is the exact product, its turns counted in 64 bits: cosine and sine are good to 2^-22
 * at any position, for |inv_freq| up to 2^20.  Arithmetic is fp32, rounded once.  A pair_axis outside [0, n_axes) turns a pair by
 * nothing.
 * No two tokens may share a slot.  q_out may be q itself (same address and strides); otherwise
 * outputs overlap neither inputs nor each other.  Rows need no alignment beyond their element.
 * n_tokens = 0 is an empty call.
 * Errors: DASC_E_INVAL (NULL cache, io, k, v, slots or cache arrays; q without q_out or the
 * reverse; rot without pos or inv_freq; a bad dtype or stride; a pointer not aligned to its
 * element; rows of q_out or of the cache that overlap), DASC_E_SHAPE (n_pages, page_size,
 * n_kv_heads, n_axes or, with q, n_q_heads < 1, head_dim < 8 or above 256 or no multiple of 8, rot odd,
 * negative or above head_dim, n_axes above 8, n_tokens < 0 or above 2^31 - 1, heads above 65536),
 * DASC_E_HIP. */
int dasc_cache_append(const dasc_kv_cache *cache, const dasc_append_io *io, dasc_stream_t stream);

/* ---- attention over the cache --------------------------------------------------------- */

/* New tokens of all requests lie one after another; strides in elements, the last dimension
 * of q and o is contiguous. */
typedef struct dasc_attn_io {
  const void *q;              /* [n_tokens, n_q_heads, head_dim], the cache's dtype          */
  void *o;                    /* [n_tokens, n_q_heads, head_dim], the cache's dtype          */
  float *lse;                 /* [n_tokens, n_q_heads], or NULL                              */
  const int32_t *block_table; /* [n_req, table_width]: the pages of each request in order    */
  const int32_t *cu_seqlens;  /* [n_req + 1], ascending                                      */
  const int32_t *kv_lens;     /* [n_req]: positions of each request, the new tokens included */
  int64_t q_tok, q_head, o_tok, o_head, lse_tok, lse_head, table_req;
  int64_t n_tokens;
  int32_t n_req, n_q_heads, table_width;
  int32_t max_len;            /* new tokens of the longest request, as the caller knows it   */
  int32_t max_kv;             /* the largest kv_lens, as the caller knows it                 */
  int32_t causal;             /* 0 or 1                                                      */
  int32_t window;             /* 0: none                                                     */
  float scale;
} dasc_attn_io;

/* Device workspace of dasc_cache_attn for these sizes (0 for many).  It does for every call with
 * these heads with no more requests and tokens than these and none longer.
 * Errors: DASC_E_INVAL (NULL bytes), DASC_E_SHAPE (as dasc_cache_attn). */
int dasc_cache_attn_workspace_bytes(int32_t n_req, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                                    int32_t head_dim, int32_t max_len, int32_t max_kv, size_t *bytes);

/* For token j of request i's len = cu_seqlens[i + 1] - cu_seqlens[i] new tokens, at position
 * here = kv_lens[i] - len + j, and query head h over the keys p of key head
 * h / (n_q_heads / n_kv_heads):
 *     seen = { p : 0 <= p < kv_lens[i], p <= here if causal, p > here - window if window > 0,
 *              its page in [0, n_pages) }
 *     s_p = scale q . k_p,   lse = log sum_seen e^{s_p},   o = sum_seen e^{s_p - lse} v_p
 * A token that sees nothing (kv_lens[i] < len, say, or pages of -1) gets o = 0 and lse = -inf.
 * What is not seen is not read into a result, whatever it holds (infinities, NaN): the rest of a
 * page, pages of -1, later tokens.
 * What is seen follows the formulas: a score of NaN makes lse and o NaN, one of +inf makes lse +inf
 * and o NaN, one of -inf weighs nothing; an infinity or NaN in a value reaches the outputs of its
 * column (an infinity as NaN where its weight is too small for the cache's dtype).
 * cu_seqlens is clamped to [0, n_tokens], kv_lens to [0, table_width * page_size]; rows of o and
 * lse of tokens that no request takes are not written.  max_len and max_kv choose launch shapes
 * and decide nothing else: a call whose requests are longer is right, but slow.
 * Precision: scores, running maxima and sums are fp32; the weights e^{s - m} are rounded to
 * the cache's dtype before they multiply the values, as the output is after; their sum takes them unrounded.
 * (fp16: a weight below 2^-21 of its row's largest is off by up to 2^-32 of that.)
 * Scores are meant to stay below 2^27, where fp32's numbers are 8 apart.
 *   q and o: 16-byte aligned, strides multiples of 8 elements; k and v too.  All strides >= 0.
 *   o must not overlap an input, nor its rows (token, head) each other; lse as o.  Requests may
 *   share pages.
 *   workspace: device, at least dasc_cache_attn_workspace_bytes, 16-byte aligned (may be NULL if
 *   that is 0); overlapping calls must not share one.
 * Errors: DASC_E_INVAL (NULL cache, io or arrays of them (q and o with n_tokens > 0, k and v); misalignment, a bad
 * dtype or stride, rows of o or lse that overlap; n_req < 1, table_width, max_len, max_kv or window
 * < 0, causal not 0 or 1, scale not finite or below 2^-126), DASC_E_SHAPE (n_pages or page_size < 1,
 * head_dim < 8 or above 256 or no multiple of 8, n_kv_heads < 1, n_q_heads no multiple of it or
 * above 65535, n_tokens < 0 or above 2^31 - 1, n_tokens times heads per key head or table_width *
 * page_size above 2^31 - 1), DASC_E_UNSUPPORTED (a page's stride above 2^32 - 1, a
 * token's above 2^27 - 1), DASC_E_WORKSPACE, DASC_E_HIP. */
int dasc_cache_attn(const dasc_kv_cache *cache, const dasc_attn_io *io, void *workspace,
                    size_t workspace_bytes, dasc_stream_t stream);

/* ---- beams ------------------------------------------------------------------------------ */

/* Device workspace of dasc_beam_select.
 * Errors: DASC_E_INVAL (NULL bytes), DASC_E_SHAPE (as dasc_beam_select). */
int dasc_beam_select_workspace_bytes(int32_t n_req, int32_t beams, int64_t vocab, int32_t n_out, size_t *bytes);

/* For each request r, beam b and token x,
 *     s = scores[r][b] + logits[r][b][x] - log sum_y e^{logits[r][b][y]}
 * in 64-bit arithmetic (the log-sum good to 2^-35); the n_out largest of all beams and tokens, in descending order:
 *     out_scores = s rounded to fp32, out_tokens = x, out_parents = b, out_slots = slots[r][b].
 * Equal ones go to the lower beam, then to the lower token; two tokens of one beam compare by
 * their logits.  A candidate needs a score above -inf: a logit of -inf, a beam whose score is -inf
 * (one that is not in use), and beams with a score or a logit of NaN or +inf give none.  Places
 * that are left over get -inf, -1, -1 and -1.
 *   logits: device [n_req, beams, vocab], dtype, rows contiguous, strides in elements, aligned
 *     to their element.  scores: device fp32 [n_req, beams].
 *   out_*: device [n_req, n_out], fp32 or int32.  slots: device int32 [n_req, beams] and out_slots
 *     both given or both NULL.  Outputs overlap neither inputs nor each other.
 *   workspace: device, 16-byte aligned; overlapping calls must not share one.
 * n_req = 0 is an empty call.
 * Errors: DASC_E_INVAL (NULL or misaligned pointer, bad dtype or stride), DASC_E_SHAPE (n_req < 0,
 * beams or n_out < 1 or above 64, vocab < 1 or above 2^24, n_req * beams above 2^24), DASC_E_WORKSPACE,
 * DASC_E_HIP. */
int dasc_beam_select(int32_t n_req, int32_t beams, int64_t vocab, int32_t n_out, int32_t dtype, const void *logits,
                     int64_t logits_req, int64_t logits_beam, const float *scores, const int32_t *slots,
                     float *out_scores, int32_t *out_tokens, int32_t *out_parents, int32_t *out_slots, void *workspace,
                     size_t workspace_bytes, dasc_stream_t stream);

/* For each group g and each j < m: slot dst[g][j] of the pool becomes what slot src[g][j] was
 * before the call.  The moves of a group happen all at once: its slots may be each other's
 * sources and destinations, and a source may serve several destinations, as the beams of a
 * request do.  A move whose src or dst lies outside [0, n_slots) is left out.
 *   pool: device, 16-byte aligned, n_slots slots of slot_bytes at a distance of slot_stride bytes, both
 *     multiples of 16: a state pool [n_pool, L, H, dk, dv] in whole slots, or a cache's pages.
 *   src, dst: device int32 [groups, m], rows src_group and dst_group elements apart.
 * No two moves may share a destination, and none of a group may have another group's source as its
 * destination.  groups = 0 or m = 0 is an empty call.
 * Errors: DASC_E_INVAL (NULL or misaligned pointer, n_slots < 1, slot_bytes < 16 or no multiple of 16 or above
 * slot_stride, a negative stride), DASC_E_SHAPE (groups or m < 0, groups above 65535, m above 64), DASC_E_HIP. */
int dasc_move_slots(void *pool, int64_t n_slots, int64_t slot_bytes, int64_t slot_stride, const int32_t *src,
                    int64_t src_group, const int32_t *dst, int64_t dst_group, int32_t groups, int32_t m,
                    dasc_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DASC_CACHE_H */
