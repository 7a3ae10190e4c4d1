/*
 * pqtopk_train.h -- training the scoring head: the catalogue's softmax cross entropy and its gradients.
 *
 * The items of the catalogue are the model's vocabulary.  For the sequence embedding phi_q of a position with the
 * target item t_q, and the scores r_qi of all N items,
 *
 *     lse_q  = log sum_i exp r_qi            loss_q = lse_q - r_{q,t_q}
 *     d loss_q / d r_qi = exp(r_qi - lse_q) - [i = t_q]
 *
 * Scores are either Eq. 5's sums of m sub-item scores (pq_cross_entropy: the codebook stands for the items, the gradient
 * is the score tables' and pq_subitem_scores_backward() takes it on to phi and Psi) or the default scorer's W phi
 * (pq_default_cross_entropy: gradients of phi and W).  No score and no probability of the N items is kept: the backward
 * calls compute them again, piece by piece.
 *
 * Conventions are those of pqtopk.h (device pointers, row-major, caller's stream, no allocation, no synchronisation,
 * arguments checked before anything is enqueued), and besides:
 *   - targets are int32 item ids.  A position whose target lies outside [0, N) has none (padding): its lse is computed,
 *     its loss is 0 and it adds nothing to any gradient, whatever its query holds (NaN too).  (Its rows of dS are zeros:
 *     Eq. 4's gradients, which know of no targets, multiply these with its query, so there it has to be finite.)
 *   - grad_loss is float [B], the gradient of the final objective with respect to loss_q (1 / count for a mean).
 *   - Scores are float32 numbers of magnitude below 5.8e6 (2^23 ln 2; probabilities of larger ones would be rounding alone): those
 *     below count as -inf (also a mask of some other large number, -1e30 say), those above as +inf.  A position all of whose
 *     scores are -inf has lse = -inf, loss 0 and no gradient.
 *   - Softmax statistics and all sums are held in 32 bits or more.  Every result is the same from run to run: no sum
 *     depends on the order in which workgroups or waves finish.
 *   - workspace: at least the bytes that the call's _workspace_bytes function names, 16-byte aligned; contents on entry
 *     are irrelevant; calls that share one must not overlap in time.  Those functions are host arithmetic and return 0
 *     for arguments that the call would reject.
 */
#ifndef PQTOPK_TRAIN_H
#define PQTOPK_TRAIN_H

#include "pqtopk.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Loss and log-sum of B positions by sub-ids: r_qi = sum_k S[q][k][codes[i][k]].
 *   codes    in   uint8 [N][m]     codebook G (Eq. 1), sub-ids < b (16-byte aligned);  uint16 [N][m] for the _u16 call
 *   S        in   float [B][m][b]  from pq_subitem_scores().  Entries may be -inf (a sub-id out of play: its items have
 *                                  probability 0); a position that meets a NaN or +inf has lse, loss and gradient NaN, and no other
 *                                  position has
 *   targets  in   int32 [B]
 *   loss     out  float [B];  lse  out  float [B]
 * b <= 256 for one-byte sub-ids, <= 65536 for two bytes.  A sub-id >= b makes the result unspecified; nothing outside the
 * arguments is touched.
 * Errors: PQ_ERR_NULL, PQ_ERR_SHAPE (N, B, m, b < 1; b too large; N >= 2^31), PQ_ERR_UNSUPPORTED (m > PQ_MAX_M,
 *         B > PQ_MAX_B, or for two-byte sub-ids one query's table too large for LDS: m * b > 36864), PQ_ERR_WORKSPACE,
 *         PQ_ERR_ALIGN, PQ_ERR_HIP.
 */
size_t pq_cross_entropy_workspace_bytes(long long N, int B, int m, int b);
int pq_cross_entropy(const uint8_t* codes, const float* S, const int* targets, long long N, int B, int m, int b,
                     float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);
size_t pq_cross_entropy_u16_workspace_bytes(long long N, int B, int m, int b);
int pq_cross_entropy_u16(const uint16_t* codes, const float* S, const int* targets, long long N, int B, int m, int b,
                         float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradient of sum_q grad_loss[q] * loss[q] with respect to the score tables:
 *     dS[q][k][j] = grad_loss[q] * ( sum_{i: codes[i][k] = j} exp(r_qi - lse_q) - [codes[t_q][k] = j] )
 *   lse  in  float [B]  as returned by pq_cross_entropy() for the same codes and S
 *   dS   out float [B][m][b]
 * Probabilities are summed as whole multiples of 2^-62 in 64 bits, so the order of the additions does not matter.
 * Errors: as pq_cross_entropy().
 */
size_t pq_cross_entropy_backward_workspace_bytes(long long N, int B, int m, int b);
int pq_cross_entropy_backward(const uint8_t* codes, const float* S, const int* targets, const float* lse,
                              const float* grad_loss, long long N, int B, int m, int b, float* dS, void* workspace,
                              size_t workspace_bytes, void* stream);
size_t pq_cross_entropy_u16_backward_workspace_bytes(long long N, int B, int m, int b);
int pq_cross_entropy_u16_backward(const uint16_t* codes, const float* S, const int* targets, const float* lse,
                                  const float* grad_loss, long long N, int B, int m, int b, float* dS, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * Eq. 4's gradients: for S[q][k][j] = psi_{k,j} . phi_{q,k} and a gradient dS of the tables,
 *     dqueries[q][k s + e] = sum_j dS[q][k][j] * psi[k][j][e]      dcentroids[k][j][e] = sum_q dS[q][k][j] * phi[q][k s + e]
 * with s = d / m.  Either output may be NULL (not both): it is not computed.
 *   dS float [B][m][b];  queries float [B][d];  centroids float [m][b][s];  dqueries float [B][d];  dcentroids float [m][b][s]
 * Sums in float32, in an order that depends on the shape alone.  From 1024 queries on, products are made of bfloat16 pieces, with
 * the limits that pq_default_cross_entropy() states for float32; below that they are float32 products.
 * Errors: PQ_ERR_NULL, PQ_ERR_SHAPE (B, d, m, b < 1; d % m; b > 65536), PQ_ERR_UNSUPPORTED (B > PQ_MAX_B, m > PQ_MAX_M,
 *         or gradients of 2^33 elements and more), PQ_ERR_WORKSPACE, PQ_ERR_ALIGN, PQ_ERR_HIP.
 */
size_t pq_subitem_scores_backward_workspace_bytes(int B, int d, int m, int b);
int pq_subitem_scores_backward(const float* dS, const float* queries, const float* centroids, float* dqueries,
                               float* dcentroids, int B, int d, int m, int b, void* workspace, size_t workspace_bytes,
                               void* stream);

#define PQ_FLOAT32  0        /* `type` of the calls below: what W, queries and their gradients hold */
#define PQ_BFLOAT16 1
#define PQ_FLOAT16  2

/*
 * Loss and log-sum of B positions by the default scorer: r_qi = W[i] . phi_q.
 *   W        in   type [N][d]   (16-byte aligned);   queries  in  type [B][d]  (16-byte aligned)
 *   targets  in   int32 [B];    loss, lse  out  float [B]
 * Scores are float32 sums of the products on the matrix cores; they are never stored.  Products of 16-bit inputs are exact.  Those
 * of float32 are made of three bfloat16 pieces of each factor: to 2^-24 of themselves for factors of 2^-100 and more (a smaller
 * one's last piece, below 2^-126, may be lost), and a factor that is infinite or above 3.396e38 makes NaN of the sums it enters.
 * Errors: PQ_ERR_NULL, PQ_ERR_SHAPE (N, B, d < 1; an unknown type; N >= 2^31), PQ_ERR_UNSUPPORTED (B > PQ_MAX_B, d > 16384,
 *         d no multiple of 16 bytes of elements: 4 of float32, 8 of 16-bit types), PQ_ERR_WORKSPACE, PQ_ERR_ALIGN, PQ_ERR_HIP.
 */
size_t pq_default_cross_entropy_workspace_bytes(long long N, int B, int d, int type);
int pq_default_cross_entropy(const void* W, const void* queries, const int* targets, long long N, int B, int d, int type,
                             float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradients of sum_q grad_loss[q] * loss[q] with respect to queries and W:
 *     dz_qi = grad_loss[q] * (exp(r_qi - lse_q) - [i = t_q])     dqueries = dz W     dW = dz^T queries
 *   lse  in  float [B]  as returned by pq_default_cross_entropy() for the same W and queries
 *   dqueries  out  type [B][d];  dW  out  type [N][d]  (both 16-byte aligned, every element written)
 * The items are taken in pieces whose dz fits the workspace: about 1 GB of it (at most a third more, where positions are padded;
 * a quarter for 16-bit rows of up to 64 elements), or 2048 items of every position.  dz is
 * held in the inputs' type (for up to 32 positions of 16 bits together with what that rounding leaves).  Float16 keeps probabilities
 * down to 2^-39 in dqueries, however small a position's weight is beside others.  In dW it keeps them down to 2^-39 times the
 * largest weight over the position's own (up to 64 positions and 512 elements), or keeps the position's query elements down to
 * 2^-39 of the largest product of a weight and an element.  The products' sums are float32, rounded to the type once.
 * Errors: as pq_default_cross_entropy().
 */
size_t pq_default_cross_entropy_backward_workspace_bytes(long long N, int B, int d, int type);
int pq_default_cross_entropy_backward(const void* W, const void* queries, const int* targets, const float* lse,
                                      const float* grad_loss, long long N, int B, int d, int type, void* dqueries, void* dW,
                                      void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PQTOPK_TRAIN_H */
