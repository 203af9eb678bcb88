/*
 * xkv_paged - rotary positions, and a paged 16-bit cache of many sequences with grouped heads.
 *
 * Where xkv.h holds ONE stream per cache, packed and evicted jointly over its heads, this part serves many
 * sequences from one pool of pages: their new tokens are turned by their positions and written to their pages
 * (kv_paged_append), attend to what their sequence holds (attn_paged_causal), leave on every cached token the
 * weight that they gave it (kv_paged_weights), and the tokens with little weight are evicted (kv_paged_evict).
 * xkv_rotary turns tensors that go anywhere else, such as the frames of kv_append.
 *
 * Conventions are those of xkv.h.  In particular
 *   - a token tensor is addressed as  base[head*head_stride + token*tok_stride + c], c = 0..head_dim-1 contiguous,
 *     strides in ELEMENTS and multiples of 8; [H][n][d] and [n][H*d] are both of that form.
 *   - q, k, v, out, pages, weights, lse, positions, tables, lengths and workspaces are DEVICE pointers on the
 *     current device, token tensors and pages 16-byte aligned, the others aligned to their type.
 *   - Calls are stream-ordered, never synchronise (exception: xkv_paged_poll_status), allocate no device memory
 *     and read no device data on the host, so they may be captured into graphs.  Tensor contents, lengths
 *     and tables are read when the kernels run: a captured call may be replayed with new ones in the same places.
 *   - All calls through one handle use its workspace: order them (one stream, or events).  Two graphs captured
 *     from one handle must not run at the same time.  Give sequences that run side by side a handle each; handles
 *     may share their pages.
 */
#ifndef XKV_PAGED_H_
#define XKV_PAGED_H_

#include "xkv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { XKV_BF16 = 0, XKV_FP16 = 1 } xkv_dtype;

/* A token tensor, see above.  (Calls take their token tensors as one array of these: few arguments, which bindings pay for one by one.) */
typedef struct {
  const void* data;          /* null: absent, where a call allows that.  Outputs are written through it. */
  int64_t tok_stride, head_stride;
} xkv_rows;

/* ---- rotary positions --------------------------------------------------------- */

/* A token at position p has the pairs (x1, x2) of its channels turned:
 *     (x1, x2) -> magnitude * (x1 cos a - x2 sin a, x2 cos a + x1 sin a),   a = p * w_i,  w_i = base^(-2i/rotary_dim).
 * With n_axes axes (the row and the column of a patch, say), channels [a*rotary_dim, (a+1)*rotary_dim) are
 * turned by the token's position on axis a; the channels behind n_axes*rotary_dim stay as they are.
 * Within an axis pair i is channels (i, i + rotary_dim/2), or (2i, 2i+1) when interleaved.
 * For contexts longer than the trained one the w_i shrink:
 *     original_tokens = 0:  all of them, w_i / factor;
 *     otherwise by bands: a pair that turns r = original_tokens * w_i / 2pi times over the trained length keeps
 *     w_i if r >= beta_fast, has w_i / factor if r <= beta_slow, and between them a blend that is linear in r.
 *     (In r, not in the pair's index i: checkpoints whose frequencies blend linearly in i, between the pairs that turn beta_fast and
 *     beta_slow times, have others in between, which this struct cannot state.)
 * Angles are formed in 64 bits (positions far beyond 2^24 keep theirs), sine, cosine and products in 32. */
typedef struct {
  int32_t rotary_dim;        /* turned channels of one axis: even, n_axes * rotary_dim <= head_dim  */
  int32_t n_axes;            /* 1..4                                                                */
  int32_t interleaved;       /* 0: pairs (i, i + rotary_dim/2); 1: pairs (2i, 2i + 1)               */
  int32_t original_tokens;   /* trained length for scaling by bands, 0: none                        */
  double  base;              /* > 1                                                                 */
  double  factor;            /* >= 1, 1: no scaling                                                 */
  double  beta_fast, beta_slow;  /* turns, beta_fast > beta_slow >= 0; read if original_tokens > 0  */
  double  magnitude;         /* > 0, usually 1                                                      */
} xkv_rotary_params;

/* Turns n tokens of q (n_q_heads heads) and of k (n_k_heads heads; 0: absent) into q_out and k_out.
 * tensors: q, q_out, k, k_out.  positions: int32 [n_axes][pos_stride], the first n of each.  An output may be its input (same
 * pointer, same strides); other overlaps are not allowed.  inverse != 0 turns by -a: undoes the rotation (magnitude 1),
 * and takes gradients of the outputs to gradients of the inputs.  n = 0 does nothing.
 * Errors: XKV_E_INVALID for bad parameters, pointers or strides. */
XKV_API int xkv_rotary(const xkv_rotary_params* params, int32_t dtype, int32_t head_dim, const int32_t* positions, int64_t pos_stride,
               int32_t n, const xkv_rows tensors[4], int32_t n_q_heads, int32_t n_k_heads, int32_t inverse, xkv_stream stream);

/* ---- the paged cache ----------------------------------------------------------- */

typedef struct xkv_paged xkv_paged;         /* opaque, host-side handle */

/* Keys and values live in two pools of n_pages pages.  Token slot t of page p, key head h is the row
 *     pool[p*page_stride + h*head_stride + t*slot_stride + c]      (strides in elements, multiples of 8)
 * so that [page][head][token][d] and [page][token][head][d] both fit.  Slot j of a sequence (its j-th cached
 * token) is slot j mod page_tokens of the page that its table names at j / page_tokens.  Query head g reads key
 * head g / (n_heads / n_kv_heads).  weights (optional) holds one float per slot, [n_pages][n_kv_heads][page_tokens]. */
typedef struct {
  int32_t n_heads;           /* query heads, a multiple of n_kv_heads, at most 64 for each           */
  int32_t n_kv_heads;        /* key heads, 1..64                                                    */
  int32_t head_dim;          /* 64 or 128                                                           */
  int32_t dtype;             /* XKV_BF16 or XKV_FP16: q, k, v, out and the pages                     */
  int32_t page_tokens;       /* 16, 32, 64, 128 or 256                                              */
  int32_t n_pages;           /* >= 1                                                                */
  int32_t max_seqs;          /* most sequences of one call, 1..1024                                  */
  int32_t reserved;          /* 0                                                                   */
  int64_t page_stride, head_stride, slot_stride;
} xkv_paged_params;

/* The sequences of a call.  Rows q_start[b] .. q_start[b+1]-1 of the token tensors are the new tokens of sequence b,
 * which holds lens[b] tokens with them: new token i is slot lens[b] - new + i.  Rows behind q_start[n_seqs] belong
 * to nobody and are neither read nor written.  A sequence may have no new tokens and no tokens at all.  The pages
 * behind a sequence's last token, and their table entries, may hold anything, as may the slots behind it.
 * The numbers are checked on the device: a sequence that reaches outside its bounds (rows, max_new, table_width,
 * n_pages) is left out, a token on a page that does not exist is not written and reads as zero, and the status
 * word becomes XKV_E_INVALID (xkv_paged_poll_status). */
typedef struct {
  int32_t n_seqs;            /* 1..max_seqs                                                         */
  int32_t n_tokens;          /* rows of the token tensors, >= 0                                     */
  int32_t max_new;           /* no sequence has more new tokens, >= 0                               */
  int32_t table_width;       /* entries of a table row; table_width * page_tokens < 2^31 - 2^16      */
  const int32_t* q_start;    /* [n_seqs + 1], from 0, not decreasing                                */
  const int32_t* lens;       /* [n_seqs]                                                            */
  const int32_t* table;      /* [n_seqs][table_width] page numbers                                  */
} xkv_paged_batch;

/* What a new token sees: its predecessors and itself, or every token of its sequence (as the tokens of one frame do). */
typedef enum { XKV_MASK_CAUSAL = 0, XKV_MASK_FULL = 1 } xkv_mask;

/* Bytes of device workspace a handle needs on a device of `multiprocessors` multiprocessors; 0 if the parameters are invalid. */
XKV_API size_t xkv_paged_workspace_bytes(const xkv_paged_params* params, int32_t multiprocessors);

/* A handle on pages that the caller owns.  dev_workspace: 256-byte aligned, at least xkv_paged_workspace_bytes
 * for the current device; zero-filled on `stream`.  The pages are not touched.  weights may be null (then
 * kv_paged_weights and kv_paged_evict answer XKV_E_STATE). */
XKV_API int xkv_paged_create(const xkv_paged_params* params, void* k_pages, void* v_pages, float* weights,
                     void* dev_workspace, size_t bytes, xkv_stream stream, xkv_paged** out);
XKV_API int xkv_paged_destroy(xkv_paged* cache);

/* The new tokens into the cache.  tensors: k, v, q, q_out.  k and v (n_kv_heads heads) go to their slots, k turned by `rotary` if that is not
 * null (positions as in xkv_rotary, one column per row), v as it is; the weights of the slots become 0.  If q is
 * present, q_out receives it turned the same way (or copied); q_out may be q.  New tokens for which the sequence has no slot (more new
 * tokens than lens[b]) are not written.  Slots written by two tokens of a call (two sequences that share the
 * page) hold one of them. */
XKV_API int kv_paged_append(xkv_paged* cache, const xkv_paged_batch* batch, const xkv_rows tensors[4],
                    const xkv_rotary_params* rotary, const int32_t* positions, int64_t pos_stride, xkv_stream stream);

/* tensors: q, out.  out = softmax(q K^T * softmax_scale) V per head over the tokens that `mask` lets a new token see, and, if lse is not
 * null, lse[head*n_tokens + row] = log sum exp of its scaled scores (natural logarithm).  The new tokens' own keys and
 * values have to be in the cache (kv_paged_append).  A token that sees nothing (more new tokens than lens[b])
 * gets zeros and an lse of -infinity.  Scores, maxima, sums and accumulators are fp32; the
 * weights are rounded to the type of v before their product with it, each against a reference maximum of its row.
 * impl: 0 = default, 1 = a simple kernel without tensor cores, kept as a cross-check (fp32 throughout).
 * Values that a token does not see never reach it, whatever they are: NaN and infinities of later tokens, and what the memory
 * holds behind the end of its sequence.  (A token before a value that is not finite may be computed a second time, by a slow
 * kernel.)  out may be q where all values are finite.
 * Errors: XKV_E_LIMIT if n_seqs * n_kv_heads * (table_width * page_tokens / 128) * (max_new * group / 128) could pass 2^32. */
XKV_API int attn_paged_causal(xkv_paged* cache, const xkv_paged_batch* batch, const xkv_rows tensors[2],
                      float* lse, float softmax_scale, int32_t mask, int32_t impl, xkv_stream stream);

/* weights[slot of head h] = decay * weights[slot] + the softmax weights that the new tokens gave the slot, added up
 * over the new tokens and over the query heads of h: exp(q.k * softmax_scale - lse).  q and lse are those of attn_paged_causal
 * with the same mask.  Every slot of every sequence with new tokens is updated.  decay >= 0; with 0 the old
 * weights are not read.  A row with a NaN (in its query or its lse) makes every slot that it sees NaN; a row that saw nothing (lse
 * -infinity) gives nothing.  Sums are formed in a fixed order: the same call repeats exactly, but for shared slots.
 * Sequences of one call that share a page (a common prefix): with decay 1 its slots get the updates of all of them, added in
 * any order; with another decay that of one of them, which one is not determined.  (A handle per sequence, on the same pages with
 * weights of its own, keeps what each gave apart.)  Errors: XKV_E_LIMIT as above. */
XKV_API int kv_paged_weights(xkv_paged* cache, const xkv_paged_batch* batch, const xkv_rows* q, const float* lse,
                     float softmax_scale, float decay, int32_t mask, xkv_stream stream);

/* Every sequence with more than `keep` tokens keeps, per key head, its first n_first and last n_recent tokens and the
 * heaviest of the others, keep tokens in all (equal weights: the lower slot wins; a NaN weighs less than any number); the
 * others keep all their tokens.  The survivors' keys, values and weights go, in their order, to slots 0, 1, ... of
 * the pages that dst_table [n_seqs][dst_width] names, which must not be pages that any sequence of the call reads; the old pages
 * stay as they are (they may be shared), the caller frees them.  kept: int32 [n_seqs][n_kv_heads][keep], the
 * survivors' old slots, -1 behind them.  lens_out: int32 [n_seqs], not lens, the new lengths, 0 for a sequence that was left out.
 * Of the batch n_seqs, lens, table and table_width are read.  Errors: XKV_E_INVALID if n_first + n_recent > keep,
 * keep < 1, dst_width * page_tokens < keep, lens_out overlaps lens, or dst_table is the batch's table. */
XKV_API int kv_paged_evict(xkv_paged* cache, const xkv_paged_batch* batch, const int32_t* dst_table, int32_t dst_width,
                   int32_t keep, int32_t n_first, int32_t n_recent, int32_t* kept, int32_t* lens_out, xkv_stream stream);

/* Synchronises `stream` and returns the handle's status word: XKV_OK, XKV_E_INVALID (see xkv_paged_batch) or
 * XKV_E_TIMEOUT (a bounded wait inside a kernel ran out; the kernel ended in order, its results are void).
 * The word is then cleared. */
XKV_API int xkv_paged_poll_status(xkv_paged* cache, xkv_stream stream);

#ifdef __cplusplus
}
#endif
#endif  /* XKV_PAGED_H_ */
