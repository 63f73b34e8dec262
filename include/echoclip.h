/*
 * The global norm of many gradient tensors, and their clipping by it, for MI355X (gfx950); part of libechoattn.so.
 *
 * The gradients of a recurrent network grow without bound now and then, so its training step ends with (Pascanu, Mikolov,
 * Bengio, "On the difficulty of training recurrent neural networks", ICML 2013)
 *
 *   norm = sqrt(sum over all tensors and elements of g^2)
 *   g    = g * max_norm / norm     if norm > max_norm, otherwise g as it is
 *
 * Squares and sums are fp64: they neither overflow nor lose small entries, whatever the number of elements.  A norm that is
 * not finite (an infinity or a NaN among the gradients, or finite ones whose norm is past fp32's largest number) clips nothing: the
 * gradients stay as they are, and `norm` says so to whoever reads it.  `norm` is the norm before clipping, rounded to fp32.
 *
 * Conventions: `grads` is HOST memory, read before the call returns (a HIP graph that captures the call keeps what it held).  The data
 * pointers in it are caller-owned DEVICE memory, contiguous and 16-byte aligned; `clipped` may be the very pointer `grad`
 * (in place: nothing is written when the factor is 1) or memory of its own that overlaps no tensor of the call, and is not looked at by
 * echo_grad_norm.  A tensor listed twice counts twice and must not be clipped in place.  n may be 0 (the pointers are
 * then not looked at).  bf16 results are rounded to nearest even once.  norm: one fp32 number on the device, 16-byte aligned
 * like the workspace.  Work is enqueued on `stream`, no synchronisation, no allocation; results are bit-identical from run to run.
 * Calls that share a workspace must be ordered by the caller.
 * Errors: ECHO_ERR_NULL, ECHO_ERR_SHAPE (count outside [1, ECHO_GRAD_MAX_COUNT], n outside [0, 2^40], max_norm not above 0 or
 * NaN; infinity is allowed and clips nothing), ECHO_ERR_DTYPE, ECHO_ERR_ALIGN, ECHO_ERR_WORKSPACE, ECHO_ERR_HIP.
 */
#ifndef ECHOCLIP_H
#define ECHOCLIP_H

#include <stddef.h>
#include <stdint.h>

#include "echoattn.h" /* echo_status_t, echo_dtype_t */

#ifdef __cplusplus
extern "C" {
#endif

#define ECHO_GRAD_MAX_COUNT 16384

typedef struct {
    const void *grad;  /* n elements                                   */
    void *clipped;     /* where they go: `grad` itself or other memory */
    int64_t n;
    int32_t dtype;     /* echo_dtype_t of both                         */
    int32_t reserved;  /* 0                                            */
} echo_grad_t;

/* Scratch of both calls, in bytes (host arithmetic; 0 for a count outside its limits). */
size_t echo_grad_workspace_bytes(const echo_grad_t *grads, int32_t count);

/* norm alone; nothing is clipped. */
echo_status_t echo_grad_norm(const echo_grad_t *grads, int32_t count, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream);

/* norm, and every tensor clipped by it. */
echo_status_t echo_grad_clip(const echo_grad_t *grads, int32_t count, float max_norm, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECHOCLIP_H */
