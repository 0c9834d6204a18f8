/*
 * kforcing_serving.h - serving operators of libkforcing.so for models with
 * grouped heads over a paged cache: attention of the newest rows, and scores
 * of tokens with their gradient.
 *
 * Device pointers only, caller-owned; work is enqueued on `stream`
 * (cudaStream_t, NULL = legacy default) and nothing is allocated or
 * synchronised, so every call may be captured in a CUDA graph.  A call that
 * needs scratch takes `work`, at least kf_op_*_work(...) bytes, 256-byte
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
 * KV beyond a sequence's length is never used, whatever it holds.
 * A page id outside the pool: KF_DEV_BAD_PAGE, its keys count as unseen.
 * A length outside 0 .. width * page: KF_DEV_BAD_ROW, clamped.
 * The same lengths give the same bits, whatever the pages' order.
 * Errors: KF_E_ARG, KF_E_CUDA.
 */
int64_t kf_op_paged_attention_work(int32_t hd);
int kf_op_paged_attention(int32_t type, int32_t B, int32_t rows, int32_t Hq, int32_t Hkv, int32_t hd,
                          const void* q, int64_t q_seq, int64_t q_row, int64_t q_head, const void* pool,
                          int64_t n_pages, int32_t page, const int32_t* table, int32_t width,
                          const int32_t* lens, float scale, void* out, void* work, void* stream);

/*
 * Scores of R rows of logits [R][V] (type fp32, bf16 or fp16; rows `stride`
 * elements apart).  With x = logits * (1 / tau) in fp32, lse = log sum_v exp(x_v) and lp_v = x_v - lse:
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
 * Padding and bad tokens: g_logp counts as 0.  A row with every logit -inf: zeros;
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
