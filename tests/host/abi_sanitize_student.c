/* As abi_sanitize_driver.c, for the calls of echoscan.h, echodistill.h, echodraft.h and those of echovocab.h and echoclip.h next to them: argument checks and
 * size queries, up to the largest descriptors.  Nothing is launched.  Prints "ok" at the end. */
#include <stdint.h>
#include <stdio.h>

#include "echoclip.h"
#include "echodistill.h"
#include "echodraft.h"
#include "echoscan.h"
#include "echovocab.h"

#define EXPECT(call, want)                                                                     \
    do {                                                                                       \
        int got_ = (int)(call);                                                                \
        if (got_ != (int)(want)) {                                                             \
            fprintf(stderr, "%s:%d: %s returned %d, expected %d\n", __FILE__, __LINE__, #call, got_, (int)(want)); \
            return 1;                                                                          \
        }                                                                                      \
    } while (0)
#define MUST(what)                                                                             \
    do {                                                                                       \
        if (!(what)) {                                                                         \
            fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #what);                         \
            return 1;                                                                          \
        }                                                                                      \
    } while (0)

#define ALL ((size_t)-1)
static void *const A = (void *)0x10000;     /* aligned, never dereferenced */
static void *const M = (void *)0x10004;     /* misaligned */

static int scan_fwd(const echo_scan_desc_t *d, void *G, void *len, void *ws, size_t bytes) {
    return (int)echo_scan_fwd(d, G, (const float *)A, (const int32_t *)len, A, (float *)A, (float *)A, ws, bytes, NULL);
}
static int scan_bwd(const echo_scan_desc_t *d, void *dh, void *states, void *ws, size_t bytes) {
    return (int)echo_scan_bwd(d, dh, (const float *)A, A, (const int32_t *)A, (const float *)states, A, (float *)A, ws, bytes, NULL);
}
static int distill_fwd(const echo_vocab_desc_t *d, void *words, int32_t K, float T, void *ws, size_t bytes) {
    return (int)echo_distill_fwd(d, A, A, (const int32_t *)words, (const float *)A, K, T, (float *)A, (float *)A, ws, bytes, NULL);
}
static int distill_bwd(const echo_vocab_desc_t *d, void *dloss, int32_t K, float T, void *dh, void *dW, void *ws, size_t bytes) {
    return (int)echo_distill_bwd(d, (const float *)dloss, (const float *)A, A, A, (const int32_t *)A, (const float *)A, K, T, dh, dW, ws, bytes, NULL);
}
static int verify(const echo_draft_desc_t *d, void *drafted, void *taken, void *ws, size_t bytes) {
    return (int)echo_draft_verify(d, (const int32_t *)drafted, (const int32_t *)A, A, A, (const float *)A, (const float *)A, (int32_t *)A, (int32_t *)taken, ws,
                                  bytes, NULL);
}

static int scan(void) {
    static const echo_scan_desc_t largest[] = {{1 << 24, 1 << 16, 1, ECHO_F32, 0}, {1 << 16, 1 << 24, 1, ECHO_BF16, 1}, {1, 1 << 20, 1 << 20, ECHO_F32, 0},
                                               {1 << 24, 257, 255, ECHO_F32, 1}, {1 << 12, 256, 1 << 20, ECHO_BF16, 0}, {1 << 20, 1, 1 << 20, ECHO_F32, 0},
                                               {3, 300, 1022, ECHO_BF16, 1}, {1, 129, 1, ECHO_F32, 0}};
    echo_scan_desc_t d = {4, 600, 70, ECHO_F32, 0}, x;
    const size_t need = echo_scan_fwd_workspace_bytes(&d);
    MUST(need > 0 && echo_scan_bwd_workspace_bytes(&d) == need && echo_scan_states_bytes(&d) == (size_t)4 * 5 * 70 * 4);
    MUST(echo_scan_fwd_workspace_bytes(NULL) == 0 && echo_scan_bwd_workspace_bytes(NULL) == 0 && echo_scan_states_bytes(NULL) == 0);
    EXPECT(scan_fwd(NULL, A, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(scan_fwd(&d, NULL, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(scan_fwd(&d, A, A, NULL, ALL), ECHO_ERR_NULL);
    EXPECT(scan_fwd(&d, M, A, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(scan_fwd(&d, A, M, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(scan_fwd(&d, A, A, A, need - 1), ECHO_ERR_WORKSPACE);
    EXPECT(scan_bwd(NULL, A, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(scan_bwd(&d, A, NULL, A, ALL), ECHO_ERR_NULL);
    EXPECT(scan_bwd(&d, M, A, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(scan_bwd(&d, A, A, A, need - 1), ECHO_ERR_WORKSPACE);
    x = d, x.dtype = 2;
    EXPECT(scan_fwd(&x, A, A, A, ALL), ECHO_ERR_DTYPE);
    x = d, x.reverse = 2;
    EXPECT(scan_bwd(&x, A, A, A, ALL), ECHO_ERR_SHAPE);
    x = d, x.B = INT32_MIN;
    EXPECT(scan_fwd(&x, A, A, A, ALL), ECHO_ERR_SHAPE);
    x = d, x.T = INT32_MAX;
    EXPECT(scan_fwd(&x, A, A, A, ALL), ECHO_ERR_SHAPE);
    x.B = x.T = ECHO_SCAN_MAX_ROWS, x.H = ECHO_SCAN_MAX_H;
    EXPECT(scan_fwd(&x, A, A, A, ALL), ECHO_ERR_SHAPE);                         /* above 2^40 together */
    MUST(echo_scan_states_bytes(&x) == 0 && echo_scan_fwd_workspace_bytes(&x) == 0);
    for (size_t i = 0; i < sizeof largest / sizeof *largest; ++i) {
        const size_t bytes = echo_scan_fwd_workspace_bytes(&largest[i]), chunks = ((size_t)largest[i].T + ECHO_SCAN_CHUNK - 1) / ECHO_SCAN_CHUNK;
        MUST(echo_scan_states_bytes(&largest[i]) == (size_t)largest[i].B * chunks * (size_t)largest[i].H * 4);
        MUST(bytes < (size_t)1 << 46 && (chunks > 1 || bytes == 0));
        EXPECT(scan_fwd(&largest[i], NULL, A, A, ALL), ECHO_ERR_NULL);
        if (bytes) EXPECT(scan_fwd(&largest[i], A, A, A, bytes - 1), ECHO_ERR_WORKSPACE);
        if (bytes) EXPECT(scan_bwd(&largest[i], A, A, A, bytes - 1), ECHO_ERR_WORKSPACE);
    }
    return 0;
}

static int distill(void) {
    static const echo_vocab_desc_t largest[] = {{ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_D, ECHO_F32, ECHO_F32},
                                                {ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_D, ECHO_BF16, ECHO_BF16},
                                                {1, ECHO_VOCAB_MAX_ROWS, 1, ECHO_BF16, ECHO_F32}, {ECHO_VOCAB_MAX_ROWS, 1, ECHO_VOCAB_MAX_D, ECHO_F32, ECHO_F32},
                                                {1, 1, 1, ECHO_F32, ECHO_F32}, {64, 32000, 512, ECHO_F32, ECHO_F32}, {65, 100003, 2047, ECHO_BF16, ECHO_BF16}};
    echo_vocab_desc_t d = {50, 700, 90, ECHO_F32, ECHO_F32}, x;
    const size_t fwd = echo_distill_fwd_workspace_bytes(&d, 9), bwd = echo_distill_bwd_workspace_bytes(&d, 9);
    MUST(fwd > echo_vocab_loss_fwd_workspace_bytes(&d) && bwd > echo_vocab_loss_bwd_workspace_bytes(&d));
    MUST(echo_distill_fwd_workspace_bytes(NULL, 9) == 0 && echo_distill_bwd_workspace_bytes(NULL, 9) == 0);
    MUST(echo_distill_fwd_workspace_bytes(&d, 0) == 0 && echo_distill_bwd_workspace_bytes(&d, ECHO_DISTILL_MAX_K + 1) == 0 &&
         echo_distill_fwd_workspace_bytes(&d, INT32_MIN) == 0);
    EXPECT(distill_fwd(NULL, A, 9, 1.f, A, ALL), ECHO_ERR_NULL);
    EXPECT(distill_fwd(&d, NULL, 9, 1.f, A, ALL), ECHO_ERR_NULL);
    EXPECT(distill_fwd(&d, M, 9, 1.f, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(distill_fwd(&d, A, 0, 1.f, A, ALL), ECHO_ERR_SHAPE);
    EXPECT(distill_fwd(&d, A, INT32_MAX, 1.f, A, ALL), ECHO_ERR_SHAPE);
    EXPECT(distill_fwd(&d, A, 9, 0.f, A, ALL), ECHO_ERR_SHAPE);
    EXPECT(distill_fwd(&d, A, 9, 0x1p65f, A, ALL), ECHO_ERR_SHAPE);
    EXPECT(distill_fwd(&d, A, 9, 1.f, A, fwd - 1), ECHO_ERR_WORKSPACE);
    EXPECT(distill_fwd(&d, A, 9, 1.f, NULL, ALL), ECHO_ERR_NULL);
    EXPECT(distill_bwd(&d, NULL, 9, 1.f, A, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(distill_bwd(&d, A, 9, 1.f, NULL, NULL, A, ALL), ECHO_ERR_NULL);
    EXPECT(distill_bwd(&d, A, 9, 1.f, NULL, M, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(distill_bwd(&d, A, 9, 0x1p-65f, A, A, A, ALL), ECHO_ERR_SHAPE);
    EXPECT(distill_bwd(&d, A, 9, 1.f, A, NULL, A, bwd - 1), ECHO_ERR_WORKSPACE);
    x = d, x.out_dtype = ECHO_BF16;
    EXPECT(distill_bwd(&x, A, 9, 1.f, A, A, A, ALL), ECHO_ERR_DTYPE);
    x = d, x.in_dtype = -1;
    EXPECT(distill_fwd(&x, A, 9, 1.f, A, ALL), ECHO_ERR_DTYPE);
    x = d, x.V = 0;
    EXPECT(distill_fwd(&x, A, 9, 1.f, A, ALL), ECHO_ERR_SHAPE);
    x = d, x.D = ECHO_VOCAB_MAX_D + 1;
    EXPECT(distill_bwd(&x, A, 9, 1.f, A, A, A, ALL), ECHO_ERR_SHAPE);
    for (size_t i = 0; i < sizeof largest / sizeof *largest; ++i)
        for (int32_t K = 1; K <= ECHO_DISTILL_MAX_K; K += 127) {
            const size_t f = echo_distill_fwd_workspace_bytes(&largest[i], K), b = echo_distill_bwd_workspace_bytes(&largest[i], K);
            const size_t lists = (size_t)largest[i].N * (size_t)(12 + 8 * K + largest[i].V / 128);
            MUST(f >= echo_vocab_loss_fwd_workspace_bytes(&largest[i]) + lists && b >= echo_vocab_loss_bwd_workspace_bytes(&largest[i]) + lists);
            MUST(f < (size_t)1 << 50 && b < (size_t)1 << 50);
            EXPECT(distill_fwd(&largest[i], A, K, 0x1p64f, A, f - 1), ECHO_ERR_WORKSPACE);
            EXPECT(distill_bwd(&largest[i], A, K, 0x1p-64f, A, A, A, b - 1), ECHO_ERR_WORKSPACE);
        }
    return 0;
}

static int draft(void) {
    static const echo_draft_desc_t largest[] = {{ECHO_DRAFT_MAX_B, ECHO_DRAFT_MAX_K, ECHO_DRAFT_MAX_V, ECHO_F32}, {1, 1, ECHO_DRAFT_MAX_V, ECHO_BF16},
                                                {64, ECHO_DRAFT_MAX_K, ECHO_DRAFT_MAX_V, ECHO_BF16}, {ECHO_DRAFT_MAX_B, 1, 1, ECHO_F32}};
    echo_draft_desc_t d = {3, 4, 50000, ECHO_F32}, x;
    const size_t need = echo_draft_verify_workspace_bytes(&d);
    MUST(need > 0 && echo_draft_verify_workspace_bytes(NULL) == 0);
    EXPECT(verify(NULL, A, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(verify(&d, NULL, A, A, ALL), ECHO_ERR_NULL);
    EXPECT(verify(&d, A, NULL, A, ALL), ECHO_ERR_NULL);
    EXPECT(verify(&d, A, A, NULL, ALL), ECHO_ERR_NULL);
    EXPECT(verify(&d, A, M, A, ALL), ECHO_ERR_ALIGN);
    EXPECT(verify(&d, A, A, M, ALL), ECHO_ERR_ALIGN);
    EXPECT(verify(&d, A, A, A, need - 1), ECHO_ERR_WORKSPACE);
    x = d, x.dtype = 7;
    EXPECT(verify(&x, A, A, A, ALL), ECHO_ERR_DTYPE);
    x = d, x.K = ECHO_DRAFT_MAX_K + 1;
    EXPECT(verify(&x, A, A, A, ALL), ECHO_ERR_SHAPE);
    x = d, x.V = INT32_MIN;
    EXPECT(verify(&x, A, A, A, ALL), ECHO_ERR_SHAPE);
    MUST(echo_draft_verify_workspace_bytes(&x) == 0);
    for (size_t i = 0; i < sizeof largest / sizeof *largest; ++i) {
        const size_t bytes = echo_draft_verify_workspace_bytes(&largest[i]);
        EXPECT(verify(&largest[i], NULL, A, A, ALL), ECHO_ERR_NULL);
        if (bytes) EXPECT(verify(&largest[i], A, A, A, bytes - 1), ECHO_ERR_WORKSPACE);
    }
    return 0;
}

static int vocabulary(void) {
    echo_vocab_desc_t d = {50, 700, 90, ECHO_F32, ECHO_F32}, most = {ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_ROWS, ECHO_VOCAB_MAX_D, ECHO_BF16, ECHO_F32};
    echo_grad_t g[2] = {{NULL, NULL, 0, ECHO_F32, 0}, {NULL, NULL, 0, ECHO_F32, 0}};
    g[0].grad = g[0].clipped = g[1].clipped = A, g[0].n = 10, g[1].grad = M, g[1].n = INT64_MAX;
    MUST(echo_vocab_loss_bwd_workspace_bytes(&most) < (size_t)1 << 50 && echo_embed_bwd_workspace_bytes(&most) > 0);
    EXPECT(echo_embed_fwd(&d, (const int32_t *)A, NULL, 1.f, A, NULL), ECHO_ERR_NULL);
    EXPECT(echo_embed_bwd(&most, (const int32_t *)A, A, 1.f, (float *)A, A, echo_embed_bwd_workspace_bytes(&most) - 1, NULL), ECHO_ERR_WORKSPACE);
    EXPECT(echo_embed_bwd_accumulate(&d, (const int32_t *)M, A, 1.f, (float *)A, A, ALL, NULL), ECHO_ERR_ALIGN);
    EXPECT(echo_vocab_loss_fwd(&d, A, A, (const int32_t *)A, 2.f, (float *)A, (float *)A, A, ALL, NULL), ECHO_ERR_SHAPE);
    EXPECT(echo_vocab_loss_bwd(&most, (const float *)A, (const float *)A, A, A, (const int32_t *)A, 0.f, A, A, A,
                               echo_vocab_loss_bwd_workspace_bytes(&most) - 1, NULL), ECHO_ERR_WORKSPACE);
    MUST(echo_grad_norm(g, 2, (float *)A, A, ALL, NULL) != ECHO_OK && echo_grad_clip(g, 1, 1.f, NULL, A, ALL, NULL) != ECHO_OK);
    EXPECT(echo_grad_clip(NULL, 1, 1.f, (float *)A, A, ALL, NULL), ECHO_ERR_NULL);
    return 0;
}

int main(void) {
    if (scan() || distill() || draft() || vocabulary()) return 1;
    puts("ok");
    return 0;
}
