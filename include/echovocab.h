/*
 * The two ends of a language model that touch its vocabulary, for MI355X (gfx950); part of libechoattn.so: the token
 * embedding with its gradient, and the output layer's softmax cross entropy with its gradients, whose logits are
 * recomputed in the backward pass instead of being kept.
 *
 * The Echo paper (Section 2) maps every word to a row of H numbers at the front of the model and computes a loss from the decoded
 * sequence at its end; Section 3.2 counts the output layer among the holders of feature maps.  It prints no formula for
 * either; these are the usual ones.
 *
 * Embedding of words t_n with a table E [V, D] and a scale s (often sqrt(D)):
 *   out[n,:] = s E[t_n,:]                     zeros where t_n is no word, i.e. outside [0, V)
 *   dE[v,:]  = s sum_{n: t_n = v} dout[n,:]   zeros for words that do not occur
 *
 * Loss of rows h [N, D] against words W [V, D], labels y_n and a label smoothing e:
 *   z[n,v]   = sum_d h[n,d] W[v,d]            lse[n] = log sum_v exp(z[n,v])
 *   loss[n]  = lse[n] - (1 - e) z[n,y_n] - e / V sum_v z[n,v]
 *   dz[n,v]  = dloss[n] (exp(z[n,v] - lse[n]) - (1 - e) [v = y_n] - e / V)
 *   dh[n,:]  = sum_v dz[n,v] W[v,:]           dW[v,:] = sum_n dz[n,v] h[n,:]
 * A row whose label is no word (outside [0, V): padding behind short sentences, say) takes part in nothing: loss, lse and dh
 * of that row are zero whatever h and dloss hold there (NaN included), and it adds nothing to dW.  Such rows cost next to nothing:
 * the others are gathered first.
 *
 * What persists from the forward to the backward pass is lse (N floats) in the place of N V logits.  Neither pass holds all of the logits at any
 * time: the forward pass keeps one maximum and sum per row and group of 64, 128 or 256 words, the backward pass forms dz for one piece of
 * the vocabulary after another (512 MB of dz at most, one piece has 256 words or more).
 *
 * Conventions: as in echoattn.h (caller-owned 16-byte aligned DEVICE memory, row-major and contiguous, work
 * enqueued on `stream`, no synchronisation, no allocation, results bit-identical from run to run, calls that share a workspace
 * ordered by the caller, workspace contents in any state before and undefined after).  Arithmetic and sums are fp32.  Inputs
 * and outputs must not overlap.
 *   - in_dtype: storage of E, h and W.  out_dtype: storage of embedded rows and of dout; of dh and dW.  Each is rounded once, to
 *     nearest even, from its fp32 sum.  loss, lse, dloss and dE are fp32.  The loss takes out_dtype ECHO_BF16 with in_dtype
 *     ECHO_BF16 only (ECHO_ERR_DTYPE); the embedding takes all four pairs.
 *   - Products run on the matrix cores with fp32 sums.  f32 storage: an operand is taken as the sum of three bf16 numbers, which add up to it
 *     exactly (below 2^-110 they are off by up to 2^-134), a product of two of them as the six that matter (error as of fp32 products), and
 *     so is dz, with a factor of 2^24 until the sums are done; infinities in h or W, numbers past 2^127, and dloss, dh or dW from 2^104
 *     on give NaN or infinities.
 *   - bf16 storage: the gradients' operands are fp16.  h and W are exact in it, scaled by a power of two, down to 2^-32 of their largest
 *     finite value (of the rows with a label, of all words), and off by up to 2^-40 of that below.  dz is taken as two fp16 numbers behind
 *     f32 gradients (off by up to 2^-22 of it) and as one behind bf16 gradients (2^-11, an eighth of what the rounding of
 *     the result is off by).  For dh both hold down to 2^-28 of the row's own dloss; a smaller dz is off by up to 2^-50 (two numbers) or 2^-39
 *     (one) of that dloss.  For dW they hold down to 2^-10 of the largest |dz| of the word, however small that is (to 2^-130 of the largest
 *     finite |dloss| among the rows with a label); a smaller dz is off by up to 2^-31 (two numbers) or 2^-20 (one) of that largest |dz|.
 *   - Errors, before anything is launched: ECHO_ERR_NULL, ECHO_ERR_DTYPE, ECHO_ERR_SHAPE (a limit below; label smoothing outside
 *     [0, 1); a scale that is not finite), ECHO_ERR_ALIGN, ECHO_ERR_WORKSPACE; ECHO_ERR_HIP for a failed launch.
 */
#ifndef ECHOVOCAB_H
#define ECHOVOCAB_H

#include <stddef.h>
#include <stdint.h>

#include "echoattn.h" /* echo_status_t, echo_dtype_t */

#ifdef __cplusplus
extern "C" {
#endif

/* Limits: 1 <= N <= ECHO_VOCAB_MAX_ROWS, 1 <= V <= ECHO_VOCAB_MAX_ROWS, 1 <= D <= ECHO_VOCAB_MAX_D; N D and V D may pass 2^32. */
#define ECHO_VOCAB_MAX_ROWS (1 << 24)
#define ECHO_VOCAB_MAX_D 16384

typedef struct {
    int32_t N;         /* tokens: rows of h, of embedded rows        */
    int32_t V;         /* words: rows of the table E, of W           */
    int32_t D;         /* row width                                  */
    int32_t in_dtype;  /* echo_dtype_t of E, h, W                    */
    int32_t out_dtype; /* echo_dtype_t of out, dout; of dh, dW       */
} echo_vocab_desc_t;

/* out [N,D] from tokens [N] and table [V,D].  in_dtype: table, out_dtype: out. */
echo_status_t echo_embed_fwd(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *table, float scale,
                             void *out, void *stream);

/* dtable [V,D] fp32 from tokens [N] and dout [N,D] (out_dtype).  echo_embed_bwd writes all of dtable;
 * echo_embed_bwd_accumulate adds to it and touches the rows of words that occur only, for a table that the output layer
 * shares (its dW comes first) or for several batches in turn.  The rows of a word are added in the order of n, long ones in
 * groups, so that a result does not depend on the run. */
size_t echo_embed_bwd_workspace_bytes(const echo_vocab_desc_t *desc);
echo_status_t echo_embed_bwd(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *dout, float scale,
                             float *dtable, void *workspace, size_t workspace_bytes, void *stream);
echo_status_t echo_embed_bwd_accumulate(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *dout,
                                        float scale, float *dtable, void *workspace, size_t workspace_bytes,
                                        void *stream);

/* loss [N] and lse [N] from h [N,D], W [V,D] and labels [N].  Keep lse for the backward call. */
size_t echo_vocab_loss_fwd_workspace_bytes(const echo_vocab_desc_t *desc);
echo_status_t echo_vocab_loss_fwd(const echo_vocab_desc_t *desc, const void *h, const void *W, const int32_t *labels,
                                  float label_smoothing, float *loss, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream);

/* dh [N,D] and dW [V,D] (out_dtype, overwritten) from dloss [N], lse as the forward call left it, and the forward inputs.
 * dh or dW may be NULL: that gradient is not wanted, and its product is left out. */
size_t echo_vocab_loss_bwd_workspace_bytes(const echo_vocab_desc_t *desc);
echo_status_t echo_vocab_loss_bwd(const echo_vocab_desc_t *desc, const float *dloss, const float *lse, const void *h,
                                  const void *W, const int32_t *labels, float label_smoothing, void *dh, void *dW,
                                  void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECHOVOCAB_H */
