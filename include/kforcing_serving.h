/*
 * kforcing_serving.h - serving operators of libkforcing.so for models with
 * grouped heads over a paged cache: attention of whole prompts and of the
 * newest rows, the cache's pages (room, append, fork, free, compact, copy), and scores of tokens
 * with their gradient.
 *
 * Device pointers only, caller-owned; work is enqueued on `stream`
 * (cudaStream_t, NULL = legacy default) and nothing is allocated or
 * synchronised, so every call may be captured in a CUDA graph.  A call that
 * needs scratch takes `work`, at least kf_op_*_work(...) bytes (0: it may be NULL), 256-byte
 * aligned, with any contents; it is free again when the call's work is done,
 * and calls that may overlap on the GPU take different ones.
 *
 * Return KF_OK or a negative KF_E_* status (kforcing.h; kf_last_error(NULL)
 * says why).  What only the device can see (a page id outside the pool, a pool
 * without enough free pages, a token outside the vocabulary) sets bits of a device error
 * word that stays set until kf_op_status reads it (KF_E_DEVICE); what such a
 * call then leaves is said at each entry.  No call reads or writes outside the
 * arrays that its arguments describe, whatever the arrays hold.
 */
#ifndef KFORCING_SERVING_H
#define KFORCING_SERVING_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define KF_TYPE_FP32 0
#define KF_TYPE_BF16 1
#define KF_TYPE_FP16 2

/* bits of the device error word that kf_op_status reports */
#define KF_DEV_BAD_TOKEN 1     /* a token outside the vocabulary                 */
#define KF_DEV_BAD_PAGE 2      /* a page id outside the pool, or no page         */
#define KF_DEV_TIMEOUT 4       /* a bounded wait ran out                         */
#define KF_DEV_BAD_ROW 8       /* a slot, length or start out of range           */
#define KF_DEV_NO_PAGES 32     /* not enough free pages                          */

/*
 * Causal attention over n packed prompts: tokens starts[i] .. starts[i+1]-1 are
 * sequence i, query row t of it sees its keys 0 .. t, and
 *   out[t][h] = sum_j p_j v[j][h / (Hq / Hkv)],
 *   p = softmax_j(scale q[t][h] . k[j][h / (Hq / Hkv)]).
 * type: KF_TYPE_BF16 or KF_TYPE_FP16 (q, k, v and out alike); hd: 64 or 128;
 * Hq a multiple of Hkv.  q [T][Hq][hd], k and v [T][Hkv][hd], out [T][Hq][hd]:
 * elements of a head contiguous, *_row / *_head the strides of tokens and heads in elements
 * (multiples of 8), so that q, k and v may be parts of one projection's output;
 * out must not overlap them.  starts: int32 [n+1], on the device,
 * starts[0] = 0, not falling, starts[n] = T; longest: at least the longest sequence's
 * tokens (host; at most 524288).  scale: a finite number > 0, for instance 1/sqrt(hd).  A sequence of
 * no tokens is allowed.  Scores, maxima, sums and the output's accumulation
 * are fp32; the probabilities are rounded to `type` for the product with V.
 * A NaN or infinity in a sequence's q, k or v stays in that sequence, and in a V
 * row it reaches the rows of the 128-row tiles that hold or follow it.
 * Starts that are not as said: KF_DEV_BAD_ROW, and out is left as it was.
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int64_t kf_op_prompt_attention_work(int32_t n, int64_t T);
int kf_op_prompt_attention(int32_t type, int32_t n, int64_t T, int32_t longest, int32_t Hq, int32_t Hkv,
                           int32_t hd, const void* q, int64_t q_row, int64_t q_head, const void* k,
                           int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                           void* out, int64_t out_row, int64_t out_head, const int32_t* starts,
                           float scale, void* work, void* stream);

/*
 * Attention of the newest `rows` rows of each of B sequences over a paged
 * cache that already holds their own K and V: with len = lens[b], row i of
 * sequence b is token len - rows + i and sees keys 0 .. len - rows + i.  A row
 * that sees no key (len < rows) is zeros.  rows = 1 is the ordinary decode
 * step, rows = P + k a joint one.
 * type: KF_TYPE_BF16 or KF_TYPE_FP16; hd: 64 or 128; Hq a multiple of Hkv.
 * q [B][rows][Hq][hd] with strides q_seq / q_row / q_head (multiples of 8
 * elements); out [B][rows][Hq][hd] contiguous.
 * pool: one layer's pages [n_pages][2: K, V][Hkv][page][hd], contiguous, page a
 * multiple of 16; table: int32 [B][width] page ids; lens: int32 [B], 0 ..
 * width * page.  Scores, maxima, sums and the accumulation are fp32.
 * KV beyond a sequence's length is never used, whatever it holds; a NaN or infinity in
 * the V of the newest rows reaches all of that sequence's rows.
 * A page id outside the pool: KF_DEV_BAD_PAGE, its keys count as unseen.
 * A length outside 0 .. width * page: KF_DEV_BAD_ROW, clamped.
 * The same lengths in a table of the same width and a pool of the same size give the same bits on one
 * device, whatever the pages' order (a call's kernels and their split go by these).
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int64_t kf_op_paged_attention_work(int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd, int32_t page, int32_t width);
int kf_op_paged_attention(int32_t type, int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd,
                          const void* q, int64_t q_seq, int64_t q_row, int64_t q_head, const void* pool,
                          int64_t n_pages, int32_t page, const int32_t* table, int32_t width,
                          const int32_t* lens, float scale, void* out, void* work, void* stream);

/*
 * The book of a cache: ref int32 [n_pages], the references to each page (0:
 * free); table int32 [slots][width], the pages of each sequence in order (-1:
 * none); lens int32 [slots], its tokens.  A sequence of len tokens has
 * ceil(len / page) pages.  Calls change it in place, in stream order.  Pages
 * are handed out lowest id first, in the order of the call's list and then of
 * the table's columns, so a book and a call give one result.
 * A call that cannot be done as a whole (a slot out of range or twice in a
 * list, a length past width * page, pages run out, a table that contradicts the
 * references where the call looks) sets KF_DEV_BAD_ROW, KF_DEV_NO_PAGES or KF_DEV_BAD_PAGE and
 * leaves book and pool as they were.  Free and fork look at the listed slots' rows, compact at the whole
 * table, grow at the columns that it fills, which have to be -1: a page without references that a
 * table still lists elsewhere is handed out again.
 *
 * No call shortens a sequence.  Rows that are not all kept (a joint step's) take room ahead: grow to the
 * kept tokens and those rows, and give append and paged attention lengths of the step's own, which may be
 * below the book's; the next step's rows then overwrite what was not kept.  Fork shares every page that the
 * book's length fills, so it wants a book whose length counts kept tokens only (before the first such step).
 *
 * kf_op_pages_grow: slot slots[i] (i < n, all different) gets pages for
 *   new_lens[i] >= lens tokens, and that length.
 * kf_op_pages_free: the listed slots (all different) give up their pages:
 *   each reference count falls by one, the table row becomes -1, the length 0.
 * kf_op_pages_fork: the sequence of slot src[i] continues in slot dst[i] too (all
 *   dst different, empty and no src): full pages are shared (one reference more), a
 *   last page that is not full is copied to a page of its own, in every layer of the pool,
 *   so appending to either never touches the other.
 * kf_op_pages_compact: with L live pages, the i-th lowest live page at or above L moves to
 *   the i-th lowest free page below L, in every layer; tables and references
 *   follow, and live (int32, device, or NULL) receives L.  Page ids >= L are free afterwards.
 * kf_op_pages_copy: page src[i] to page dst[i], in every layer; the dst pages are
 *   different from each other and from every src.  Ids outside the pool: KF_DEV_BAD_PAGE, that copy is
 *   left out.
 * pool: [layers][n_pages][page_bytes], page_bytes a multiple of 16.
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int64_t kf_op_pages_work(int32_t n_pages, int32_t slots, int32_t n);
int kf_op_pages_grow(int32_t n, const int32_t* which, const int32_t* new_lens, int32_t* ref, int32_t n_pages,
                     int32_t* table, int32_t slots, int32_t width, int32_t* lens, int32_t page, void* work,
                     void* stream);
int kf_op_pages_free(int32_t n, const int32_t* which, int32_t* ref, int32_t n_pages, int32_t* table,
                     int32_t slots, int32_t width, int32_t* lens, int32_t page, void* work, void* stream);
int kf_op_pages_fork(int32_t n, const int32_t* src, const int32_t* dst, int32_t* ref, int32_t n_pages,
                     int32_t* table, int32_t slots, int32_t width, int32_t* lens, int32_t page, void* pool,
                     int32_t layers, int64_t page_bytes, void* work, void* stream);
int kf_op_pages_compact(int32_t* ref, int32_t n_pages, int32_t* table, int32_t slots, int32_t width,
                        void* pool, int32_t layers, int64_t page_bytes, int32_t* live, void* work,
                        void* stream);
int kf_op_pages_copy(int32_t n, const int32_t* src, const int32_t* dst, void* pool, int32_t layers,
                     int32_t n_pages, int64_t page_bytes, void* stream);

/*
 * K and V rows of new tokens into their pages of one layer: rows starts[i] ..
 * starts[i+1]-1 of k and v (T rows of Hkv heads, strides in elements, multiples of
 * 8; 16-bit elements) are the last tokens of slot which[i], at positions lens[slot]
 * - count .. lens[slot] - 1.  pool: that layer's [n_pages][2][Hkv][page][hd], hd a
 * multiple of 8.  The pages must not be shared (kf_op_pages_fork leaves none of them so).
 * A token whose slot, position or page is out of range: KF_DEV_BAD_ROW or
 * KF_DEV_BAD_PAGE, and it is not written.
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int kf_op_pages_append(int32_t n, const int32_t* which, const int32_t* starts, int64_t T, int32_t Hkv,
                       int32_t hd, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                       int64_t v_head, void* pool, int32_t n_pages, int32_t page, const int32_t* table,
                       int32_t slots, int32_t width, const int32_t* lens, void* stream);

/*
 * Scores of R rows of logits [R][V] (type fp32, bf16 or fp16; rows `stride`
 * elements apart, at most 1 MiB each; log2(e) / tau a finite fp32 number).  With x = logits * (1 / tau) in fp32, lse = log sum_v exp(x_v) and lp_v = x_v - lse:
 *   logp[r] = lp_token, entropy[r] = -sum_v exp(lp_v) lp_v, lse[r], and the top
 *   alternatives: the `top` (0 .. 64, <= V) ids of the largest x, largest first, ties to the
 *   lowest id, in top_ids [R][top], their lp in top_logp [R][top].
 * tokens: int64 [R]; a negative one is padding (logp 0).  logp, entropy, lse: fp32 [R]; NULL skips
 * one.  Logits of -inf are closed tokens (probability 0, no part in the
 * entropy).  A row with every logit -inf: lse, logp and top_logp -inf, entropy 0, top_ids 0,
 * 1, ...  A row with a NaN or +inf: NaN numbers (padding keeps logp 0), top_ids -1.
 * A token >= V: KF_DEV_BAD_TOKEN, logp NaN.
 * kf_op_token_scores_grad: the scores, and for loss weights g_logp and g_entropy
 * (fp32 [R], NULL: zeros) the gradient of sum_r g_logp logp + g_entropy entropy:
 *   grad_v = (g_logp (1[v = token] - p_v) - g_entropy p_v (lp_v + entropy)) / tau, p = exp(lp),
 * in grad [R][V] (the logits' type, rows grad_stride apart; it may be the logits themselves).
 * Padding and bad tokens: g_logp counts as 0; a p below 2^-126 is 0.  A row with every logit -inf: zeros;
 * with a NaN or +inf: NaN.
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int kf_op_token_scores(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                       const int64_t* tokens, float tau, int32_t top, float* logp, float* entropy, float* lse,
                       int32_t* top_ids, float* top_logp, void* stream);
int kf_op_token_scores_grad(int32_t type, int64_t R, int32_t V, const void* logits, int64_t stride,
                            const int64_t* tokens, float tau, const float* g_logp, const float* g_entropy,
                            float* logp, float* entropy, float* lse, void* grad, int64_t grad_stride,
                            void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KFORCING_SERVING_H */
