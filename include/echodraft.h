/*
 * Verification of drafted words against the model's own probabilities, for MI355X (gfx950); part of libechoattn.so.
 *
 * A small student proposes the next K words of a sentence one by one, the model of the Echo paper (Section 2) scores all of them in one
 * pass, and this call decides how many stand, so that the words come out distributed as the model alone would draw them (Leviathan, Kalman,
 * Matias, "Fast Inference from Transformers via Speculative Decoding", 2023).  With p the model's and q the student's probabilities, n drafted words d
 * of sequence b and given random numbers u and r from [0, 1):
 *
 *   word d[i] is taken while   u[i] q[i, d[i]] < p[i, d[i]],   i = 0, 1, .. n - 1;   a = number of words taken
 *   one more word is drawn from the weights w:
 *     a < n   w[v] = max(p[a, v] - q[a, v], 0), or p[a, v] if none of these is positive
 *     a = n   w[v] = p[n, v]
 *   as the first v with   sum_{x <= v} w[x] > r sum_x w[x]
 *
 * All comparisons and sums are in 64 bits.  p and q need not be normalised.
 *   - A drafted word outside [0, V) is not taken.  NaN in p, q or u at a drafted word: not taken.
 *   - Weights that are no positive finite numbers (NaN, infinities) count as zero.  Where p[a] has no other ones there is no word to draw: -1.
 *   - r below 0 or NaN counts as 0; r of 1 and more draws the last word with a weight.
 *   - What p holds behind position n, and q, d and u from position n on, does not matter.  n below 0 counts as 0, above K as K.
 *
 * Conventions: as in echoattn.h (caller-owned 16-byte aligned DEVICE memory, row-major and contiguous, work enqueued on `stream`, no
 * synchronisation, no allocation, results bit-identical from run to run, calls that share a workspace ordered by the caller, workspace contents in any
 * state before and undefined after).  Outputs must not overlap inputs.
 * Errors, before anything is launched: ECHO_ERR_NULL, ECHO_ERR_DTYPE, ECHO_ERR_SHAPE (a limit below), ECHO_ERR_ALIGN, ECHO_ERR_WORKSPACE;
 * ECHO_ERR_HIP for a failed launch.
 */
#ifndef ECHODRAFT_H
#define ECHODRAFT_H

#include <stddef.h>
#include <stdint.h>

#include "echoattn.h" /* echo_status_t, echo_dtype_t */

#ifdef __cplusplus
extern "C" {
#endif

/* Limits: 1 <= B <= ECHO_DRAFT_MAX_B, 1 <= K <= ECHO_DRAFT_MAX_K, 1 <= V <= ECHO_DRAFT_MAX_V; B (K + 1) V may pass 2^32. */
#define ECHO_DRAFT_MAX_B (1 << 20)
#define ECHO_DRAFT_MAX_K 1024
#define ECHO_DRAFT_MAX_V (1 << 24)

typedef struct {
    int32_t B;     /* sequences                          */
    int32_t K;     /* drafted words of each, at most     */
    int32_t V;     /* words of the vocabulary            */
    int32_t dtype; /* echo_dtype_t of draft and target   */
} echo_draft_desc_t;

/* tokens [B,K+1] (the words taken, the word drawn, -1 behind it) and taken [B] (a) from drafted [B,K], n_drafted [B], draft [B,K,V] (q),
 * target [B,K+1,V] (p), u [B,K] and r [B].  n_drafted may be NULL: K for all.  The workspace may be NULL where its size is 0. */
size_t echo_draft_verify_workspace_bytes(const echo_draft_desc_t *desc);
echo_status_t echo_draft_verify(const echo_draft_desc_t *desc, const int32_t *drafted, const int32_t *n_drafted, const void *draft,
                                const void *target, const float *u, const float *r, int32_t *tokens, int32_t *taken, void *workspace,
                                size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECHODRAFT_H */
