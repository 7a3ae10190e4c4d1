/*
 * pqtopk_probs.h -- the scoring head as a distribution over the catalogue: log-probabilities of given items with the entropy and
 * the likeliest items, and distillation from a teacher's list of items with scores.
 *
 * For a position with the scores r_qi of all N items and a temperature T,
 *
 *     p_qi = exp(r_qi / T - lse_q)      lse_q = log sum_i exp(r_qi / T)      entropy_q = - sum_i p_qi log p_qi
 *
 * Scores are Eq. 5's sums of m sub-item scores (pq_log_probs, pq_distillation) or the default scorer's W phi (pq_default_*).  The
 * distillations, and log-probabilities without likeliest items, keep neither a score nor a probability of the N items.
 *
 * Conventions are those of pqtopk.h and pqtopk_train.h (device pointers, row-major, caller's stream, no allocation, no
 * synchronisation, arguments checked before anything is enqueued, results the same from run to run), and besides:
 *   - T is a finite number of 1e-4 to 1e4.  Scores over it are float32 numbers of magnitude below 5.8e6: those below count as -inf (also a
 *     mask of some other large number, -1e30 say: its items have the log-probability -inf, beside other items and alone), those above as +inf.
 *   - Item ids are int32.  One outside [0, N) names no item (padding).
 *   - A position all of whose scores are -inf has lse = -inf.
 *   - Workspaces of the log-probabilities with K > 0 hold lists of scored items, 8 bytes for every position and item of a piece of the
 *     catalogue (the likeliest few come from them): up to 16,384 items (and positions) are one piece, of longer catalogues the largest has most of
 *     the items, as far as 2 GiB of lists go (of more than 32,768 positions 4.3, where K is over 496).  64 positions of 1.27M items take 614 MiB, twice
 *     what their scores would; 16 KB a position and up to 128 MiB of sums come on top.  By sub-ids and few positions there are no lists: the ranking
 *     follows the pass.
 */
#ifndef PQTOPK_PROBS_H
#define PQTOPK_PROBS_H

#include "pqtopk_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Log-probabilities of n given items a position, the entropy and the K likeliest items, by sub-ids.
 *   codes          in   uint8 [N][m] (uint16 for the _u16 call; 16-byte aligned);   S  in  float [B][m][b]
 *   items          in   int32 [B][n]       an item may be given more than once.  n may be 0 (items and log_probs may be NULL then)
 *   log_probs      out  float [B][n]       log p of these; 0 where there is no item
 *   entropy        out  float [B]          in nats;  0 for a position all of whose scores are -inf
 *   lse            out  float [B]
 *   top_items      out  int32 [B][K]       by score descending, then id ascending, as pq_score_topk() ranks them.  K may be 0 (top_items and
 *   top_log_probs  out  float [B][K]         top_log_probs may be NULL then)
 * Table entries may be -inf (a sub-id out of play; entries below -1e32 count as that): items of score -inf have the log-probability -inf and
 * come last, by id; those whose scores are numbers that count as -inf come before them, by their scores.  Of a position that meets a NaN or +inf
 * every number is NaN, top_items are different items of the catalogue in no particular order; no other position is touched by it.
 * Errors: PQ_ERR_NULL, PQ_ERR_SHAPE (N, B, m, b < 1; n, K < 0; b too large; K > N; N >= 2^31; T no positive number), PQ_ERR_UNSUPPORTED
 *         (K > PQ_MAX_K, n > 65536, T out of its range, and as pq_cross_entropy()), PQ_ERR_WORKSPACE, PQ_ERR_ALIGN, PQ_ERR_HIP.
 */
size_t pq_log_probs_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_log_probs(const uint8_t* codes, const float* S, const int* items, long long N, int B, int m, int b, int n, int K, float temperature,
                 float* log_probs, float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace,
                 size_t workspace_bytes, void* stream);
size_t pq_log_probs_u16_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_log_probs_u16(const uint16_t* codes, const float* S, const int* items, long long N, int B, int m, int b, int n, int K, float temperature,
                     float* log_probs, float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * The same by the default scorer: r_qi = W[i] . phi_q, W and queries of `type` (PQ_FLOAT32, PQ_BFLOAT16, PQ_FLOAT16).
 *   W  in  type [N][d];  queries  in  type [B][d]  (both 16-byte aligned)
 * The catalogue's scores are float32 sums as in pq_default_cross_entropy().  The K + 16 best of them (all N if there are no more) are scored again in
 * 64 bits, which ranks them, and so are the given items.  (Of more than 16 items beyond the K-th whose scores lie within a float32 sum's rounding of
 * its score, near copies of one item, that rounding decides which come; equal rows of W have equal sums.)
 * Errors: as pq_log_probs() and pq_default_cross_entropy().
 */
size_t pq_default_log_probs_workspace_bytes(long long N, int B, int d, int type, int K);
int pq_default_log_probs(const void* W, const void* queries, const int* items, long long N, int B, int d, int type, int n, int K,
                         float temperature, float* log_probs, float* entropy, float* lse, int* top_items, float* top_log_probs,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Distillation: a teacher's list of K items a position with its scores of them, as pq_log_probs(), pq_score_topk() or any other model gives them.
 *     w_qk = softmax over the list of teacher_scores[q][k] / T        loss_q = T^2 sum_k w_qk (log w_qk - log p_{q, items_qk})
 *     d loss_q / d r_qi = T (p_qi - sum_{k: items_qk = i} w_qk)
 *   teacher_items   in   int32 [B][K]   an id outside [0, N) is no entry (a shorter list, or padding); an item that is listed twice has two entries
 *   teacher_scores  in   float [B][K]   -inf: an entry of no weight.  A list that holds a NaN or +inf makes the position's loss and gradient NaN
 *   loss            out  float [B];  lse  out  float [B]   log sum_i exp(r_qi / T)
 * A position whose list has no entry of weight (or all of whose scores are -inf) has the loss 0 and adds nothing to any gradient, whatever
 * its query holds.  An entry of weight whose own score is -inf, or counts as that, makes the loss +inf, and the gradient stays finite.
 * A list of one item has the loss -T^2 log p, so the gradient of sum_q g_q log p_{q,t_q} is that of lists of the one item t_q (of any score) with
 * grad_loss_q = -g_q / T^2; that of several items' sum_k g_qk log p_{q,i_qk}, g_qk > 0, that of lists of these with the scores T log g_qk
 * and grad_loss_q = -sum_k g_qk / T^2.  (The entropy's gradient has no call.)
 * Errors: PQ_ERR_NULL, PQ_ERR_SHAPE (N, B, m, b, K < 1; b too large; N >= 2^31; T no positive number), PQ_ERR_UNSUPPORTED (K > PQ_MAX_K,
 *         T out of its range, and as pq_cross_entropy()), PQ_ERR_WORKSPACE, PQ_ERR_ALIGN, PQ_ERR_HIP.
 */
size_t pq_distillation_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_distillation(const uint8_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, long long N, int B,
                    int m, int b, int K, float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);
size_t pq_distillation_u16_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_distillation_u16(const uint16_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, long long N, int B,
                        int m, int b, int K, float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradient of sum_q grad_loss[q] * loss[q] with respect to the score tables: lse as pq_distillation() returned it for the same arguments.
 *   dS  out  float [B][m][b].   Sums are whole multiples of 2^-62 in 64 bits, as in pq_cross_entropy_backward().
 * Errors: as pq_distillation().
 */
size_t pq_distillation_backward_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_distillation_backward(const uint8_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, const float* lse,
                             const float* grad_loss, long long N, int B, int m, int b, int K, float temperature, float* dS,
                             void* workspace, size_t workspace_bytes, void* stream);
size_t pq_distillation_u16_backward_workspace_bytes(long long N, int B, int m, int b, int K);
int pq_distillation_u16_backward(const uint16_t* codes, const float* S, const int* teacher_items, const float* teacher_scores,
                                 const float* lse, const float* grad_loss, long long N, int B, int m, int b, int K, float temperature,
                                 float* dS, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Distillation of the default scorer, and its gradients with respect to queries and W (each in `type`, every element written).  Arithmetic,
 * what dz is held in and its limits are those of pq_default_cross_entropy() and its gradient, with T grad_loss for the positions' weights;
 * of 33 to 64 positions of 16 bits and up to 512 elements (float16: 72 and more) listed items' dz, too, is held with what its rounding leaves.
 * Of more positions of 16 bits it is rounded to their type: the gradients are then off by up to two roundings of it instead of one, sqrt(2) of
 * one in the mean square.  Float32 W and queries have it in float32.
 * A list that holds a NaN or +inf makes its position's row of dqueries NaN, and the rows of dW of the items that it names.
 * Errors: as pq_distillation() and pq_default_cross_entropy().
 */
size_t pq_default_distillation_workspace_bytes(long long N, int B, int d, int type, int K);
int pq_default_distillation(const void* W, const void* queries, const int* teacher_items, const float* teacher_scores, long long N, int B,
                            int d, int type, int K, float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream);
size_t pq_default_distillation_backward_workspace_bytes(long long N, int B, int d, int type, int K);
int pq_default_distillation_backward(const void* W, const void* queries, const int* teacher_items, const float* teacher_scores,
                                     const float* lse, const float* grad_loss, long long N, int B, int d, int type, int K,
                                     float temperature, void* dqueries, void* dW, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PQTOPK_PROBS_H */
