/*
 * Distillation from a teacher's top logits, for MI355X (gfx950); part of libechoattn.so: the loss that trains a student's output layer on the K
 * likeliest words of a large model in the place of one label per row (echovocab.h), and its gradients.  As there, no logits are kept.
 *
 * Rows h [N, D], words W [V, D], of row n the teacher's words w[n,k] and logits t[n,k], temperature T:
 *   q[n,k]   = exp(t[n,k] / T) / sum_j exp(t[n,j] / T)         over the row's entries
 *   z[n,v]   = sum_d h[n,d] W[v,d]                             lse[n] = log sum_v exp(z[n,v] / T)
 *   loss[n]  = T^2 sum_k q[n,k] (log q[n,k] - z[n,w[n,k]] / T + lse[n])
 *   dz[n,v]  = dloss[n] T (exp(z[n,v] / T - lse[n]) - sum_{k: w[n,k] = v} q[n,k])
 *   dh[n,:]  = sum_v dz[n,v] W[v,:]                            dW[v,:] = sum_n dz[n,v] h[n,:]
 * the divergence of the student's distribution over all words from the teacher's over its K, with Hinton, Vinyals and Dean's factor T^2
 * ("Distilling the Knowledge in a Neural Network", 2015), which keeps the gradients' size as T grows.
 *
 * An entry (n, k) takes part if its word is one, i.e. in [0, V), and its logit is not minus infinity; a list may be shorter than K, have gaps and name a word
 * more than once (its shares add up in dz; in the loss each is a term of its own).  A row without entries takes part in nothing: loss, lse and dh of
 * that row are zero whatever h and dloss hold there (NaN included), and it adds nothing to dW.  Such rows cost next to nothing.
 *
 * What persists from the forward to the backward pass is lse (N floats).
 *
 * The descriptor is echovocab.h's: in_dtype of h and W, out_dtype of dh and dW; t, loss, lse and dloss are fp32.  Conventions, products, their error and
 * ranges: as those of echo_vocab_loss_fwd and echo_vocab_loss_bwd, with T dloss in the place of dloss.  A logit t that is NaN or plus infinity
 * makes its row's loss and gradients NaN (lse does not depend on t).
 * The loss is the difference of sum_k q log q and sum_k q log p, each of them good to some 2^-23 of its own size times the roundings of the sums behind it: where
 * student and teacher are nearly sure of the same word both are small and the loss keeps its digits, as that of a sure label does; where they agree on
 * several words it may be far smaller than either.
 * Errors, before anything is launched: ECHO_ERR_NULL, ECHO_ERR_DTYPE, ECHO_ERR_SHAPE (the descriptor's limits, K outside
 * 1 .. ECHO_DISTILL_MAX_K, T outside 2^-64 .. 2^64), ECHO_ERR_ALIGN, ECHO_ERR_WORKSPACE; ECHO_ERR_HIP for a failed launch.
 */
#ifndef ECHODISTILL_H
#define ECHODISTILL_H

#include "echovocab.h" /* echo_vocab_desc_t */

#ifdef __cplusplus
extern "C" {
#endif

#define ECHO_DISTILL_MAX_K 128

/* loss [N] and lse [N] from h [N,D], W [V,D], words [N,K] and logits [N,K].  Keep lse for the backward call.  (Sizes: 0 where a call would be refused.) */
size_t echo_distill_fwd_workspace_bytes(const echo_vocab_desc_t *desc, int32_t K);
echo_status_t echo_distill_fwd(const echo_vocab_desc_t *desc, const void *h, const void *W, const int32_t *words, const float *logits,
                               int32_t K, float T, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* dh [N,D] and dW [V,D] (out_dtype, overwritten) from dloss [N], lse as the forward call left it, and the forward inputs.
 * dh or dW may be NULL: that gradient is not wanted, and its product is left out. */
size_t echo_distill_bwd_workspace_bytes(const echo_vocab_desc_t *desc, int32_t K);
echo_status_t echo_distill_bwd(const echo_vocab_desc_t *desc, const float *dloss, const float *lse, const void *h, const void *W,
                               const int32_t *words, const float *logits, int32_t K, float T, void *dh, void *dW, void *workspace,
                               size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECHODISTILL_H */
