/*
 * A gated linear recurrence over whole sequences, forward and backward, for MI355X (gfx950); part of libechoattn.so.
 *
 * It is what the LSTM cell (echolstm.h) becomes when its gates no longer depend on the previous hidden state: then all gates of a
 * sequence come out of one matrix product over all of its steps, and what is left to do step by step is linear in the state
 * and is done for all steps at once.  A layer of it in the place of an LSTM layer makes a student of the Echo paper's model
 * (Section 2) that reads a prompt, and trains, without a chain of small products.  The paper has no such layer; the usual formulas are taken, gates sliced
 * in the order forget, candidate, output:
 *
 *   f[t] = sigmoid(G[b, t, 0:H])      g[t] = tanh(G[b, t, H:2H])      o[t] = sigmoid(G[b, t, 2H:3H])
 *   c[t] = f[t] c[t-1] + (1 - f[t]) g[t]          h[t] = o[t] c[t]
 * over steps 0 .. len[b] - 1, starting with c0[b], and
 *   r[t] = dh[t] o[t] + f[t+1] r[t+1]             (at the last step dc_last[b] in the place of f[t+1] r[t+1])
 *   dG[t] = [r[t] (c[t-1] - g[t]) f[t] (1 - f[t]),   r[t] (1 - f[t]) (1 - g[t]^2),   dh[t] c[t] o[t] (1 - o[t])]
 *   dc0 = f[0] r[0]
 * With `reverse`, a sequence's steps run from position len[b] - 1 to 0 (the other direction of an encoder): h, G, dh and dG of a step stand at its
 * position; c0 is in front of position len[b] - 1, c_last behind position 0.
 *
 * Positions from len[b] on take no part, whatever G and dh hold there (NaN included): h and dG are zero there.  A length below 0 counts
 * as 0, one above T as T; a sequence of length 0 hands c0 to c_last, and dc_last to dc0.
 *
 * What persists from the forward to the backward pass is one state per ECHO_SCAN_CHUNK steps; those between are formed again.
 *
 * One step of decoding is the forward call with T = 1: c_last is the next step's c0.  It may be the same buffer.
 *
 * Conventions: as in echoattn.h (caller-owned 16-byte aligned DEVICE memory, row-major and contiguous, work enqueued on `stream`, no
 * synchronisation, no allocation, results bit-identical from run to run, calls that share a workspace ordered by the caller, workspace contents in any
 * state before and undefined after).  Outputs are overwritten and must not overlap inputs, but for c_last and c0, and dc0 and
 * dc_last, which may be one buffer.
 *   - dtype: storage of G, h, dh and dG, each rounded once, to nearest even, from fp32.  c0, c_last, dc_last, dc0 and the kept states are
 *     fp32, and so are all gates, states and sums.
 *   - f and 1 - f = sigmoid(-x) are each good to a few units of their own last place: what a gate that is nearly closed lets through, and its gradient, keep their
 *     digits as those of a gate that forgets next to nothing do.  o (1 - o) and 1 - g^2 are formed from o and g as fp32 has them, off by up to 2^-23.
 *   - An infinite c0 stays infinite in h and c_last, an infinite dc_last or dh in dc0, as long as the product of the gates in between is a number of fp32's; behind that
 *     it is NaN.  In dG, which multiplies and subtracts them, what they reach is infinite or NaN.  Other channels and sequences do not notice.
 *   - Errors, before anything is launched: ECHO_ERR_NULL, ECHO_ERR_DTYPE, ECHO_ERR_SHAPE (a limit below), ECHO_ERR_ALIGN,
 *     ECHO_ERR_WORKSPACE; ECHO_ERR_HIP for a failed launch.
 */
#ifndef ECHOSCAN_H
#define ECHOSCAN_H

#include <stddef.h>
#include <stdint.h>

#include "echoattn.h" /* echo_status_t, echo_dtype_t */

#ifdef __cplusplus
extern "C" {
#endif

/* Limits: 1 <= B, T <= ECHO_SCAN_MAX_ROWS, 1 <= H <= ECHO_SCAN_MAX_H, B T H <= 2^40; B T H may pass 2^32. */
#define ECHO_SCAN_MAX_ROWS (1 << 24)
#define ECHO_SCAN_MAX_H (1 << 20)
#define ECHO_SCAN_CHUNK 128

typedef struct {
    int32_t B;       /* sequences                                  */
    int32_t T;       /* positions of each                          */
    int32_t H;       /* channels                                   */
    int32_t dtype;   /* echo_dtype_t of G, h, dh, dG               */
    int32_t reverse; /* 0: from position 0 on, 1: from the end     */
} echo_scan_desc_t;

/* Bytes of the states that the forward call keeps for the backward call: B ceil(T / ECHO_SCAN_CHUNK) H floats. */
size_t echo_scan_states_bytes(const echo_scan_desc_t *desc);

/* h [B,T,H] and c_last [B,H] from G [B,T,3H], c0 [B,H] and len [B].  c0 may be NULL (zeros), len may be NULL (T for all), c_last may be
 * NULL (not wanted), states may be NULL (no backward call follows).  The workspace may be NULL where its size is 0. */
size_t echo_scan_fwd_workspace_bytes(const echo_scan_desc_t *desc);
echo_status_t echo_scan_fwd(const echo_scan_desc_t *desc, const void *G, const float *c0, const int32_t *len, void *h,
                            float *c_last, float *states, void *workspace, size_t workspace_bytes, void *stream);

/* dG [B,T,3H] and dc0 [B,H] from dh [B,T,H], dc_last [B,H], the forward inputs and the states as the forward call left them.
 * dc_last may be NULL (zeros), dc0 may be NULL (not wanted).  The workspace may be NULL where its size is 0. */
size_t echo_scan_bwd_workspace_bytes(const echo_scan_desc_t *desc);
echo_status_t echo_scan_bwd(const echo_scan_desc_t *desc, const void *dh, const float *dc_last, const void *G, const int32_t *len,
                            const float *states, void *dG, float *dc0, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECHOSCAN_H */
