// Verification of drafted words (include/echodraft.h has the rules): a block per sequence.
//
// Which words are taken takes K pairs of probabilities; the word that is drawn behind them takes one row of the model's and, if a word was not taken,
// one of the student's.  The block sums the weights of that row by segments, finds the segment in which the sum passes r of the whole, and goes over
// that segment again.  All sums are in 64 bits and in an order that depends on V alone.
#include "../../include/echodraft.h"

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kDraftWaves = 16;

struct DraftArgs {
    const int *drafted, *n_drafted;
    const void *draft, *target;
    const float *u, *r;
    int B, K, V;
    int *tokens, *taken;
};

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
// inclusive sums over the lanes
__device__ __forceinline__ double wave_scan_f64(double x, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    return x;
}

// the weight of a word: positive and finite, or zero
template <typename T> __device__ __forceinline__ double weight(const T *p, const T *q, int v) {
    const float x = ld(p, v);
    const double w = q ? (double)x - (double)ld(q, v) : (double)x;
    return w > 0.0 && w < __builtin_inf() ? w : 0.0;
}

template <typename T> __global__ __launch_bounds__(64 * kDraftWaves) void k_draft_verify(const DraftArgs a) {
    __shared__ double s_sum[kDraftWaves][4];
    __shared__ double s_before;
    __shared__ int s_segment;
    const int b = blockIdx.x, lane = lane_id(), w = wave_id(), V = a.V;
    const int n = a.n_drafted ? clamp_len(a.n_drafted[b], a.K) : a.K;
    const T *p = static_cast<const T *>(a.target) + (size_t)b * (a.K + 1) * V, *q = static_cast<const T *>(a.draft) + (size_t)b * a.K * V;
    // the first word that is not taken: every wave for itself
    int take = n;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = min(i0 + lane, n - 1), d = a.drafted[(size_t)b * a.K + i];
        const bool word = (unsigned)d < (unsigned)V;
        const size_t at = (size_t)i * V + (word ? d : 0);
        const bool good = word && (double)a.u[(size_t)b * a.K + i] * (double)ld(q, at) < (double)ld(p, at);
        const unsigned long long bad = __ballot(!good);
        if (bad) {
            take = min(n, i0 + __builtin_ctzll(bad));
            break;
        }
    }
    p += (size_t)take * V;
    q = take < n ? q + (size_t)take * V : nullptr;
    int *tokens = a.tokens + (size_t)b * (a.K + 1);
    for (int i = threadIdx.x; i <= a.K; i += 64 * kDraftWaves)
        if (i != take) tokens[i] = i < take ? a.drafted[(size_t)b * a.K + i] : -1;
    if (threadIdx.x == 0) a.taken[b] = take;

    // segments of whole groups of 64 words, four a wave
    constexpr int SEGMENTS = 4 * kDraftWaves;
    const int size = ((V + SEGMENTS - 1) / SEGMENTS + 63) / 64 * 64;
    double total = 0.0;
    for (int attempt = 0; attempt < 2; ++attempt) {
        double sum[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int begin = (w * 4 + k) * size, end = min(V, begin + size);
            sum[k] = 0.0;
            for (int v = begin + lane; v < end; v += 64) sum[k] += weight(p, q, v);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sum[k] = wave_sum_f64(sum[k]);
            if (lane == 0) s_sum[w][k] = sum[k];
        }
        __syncthreads();
        total = 0.0;
        for (int k = 0; k < SEGMENTS; ++k) total += s_sum[k >> 2][k & 3];
        if (total > 0.0 || !q) break;
        q = nullptr;                                       // nothing is left of p behind q: p itself
        __syncthreads();
    }
    if (!(total > 0.0)) {
        if (threadIdx.x == 0) tokens[take] = -1;
        return;
    }
    if (threadIdx.x == 0) {
        const float r = a.r[b];
        const double at = r > 0.f ? (double)r * total : 0.0;
        double before = 0.0, found_before = 0.0;
        int found = -1, last = 0;
        double last_before = 0.0;
        for (int k = 0; k < SEGMENTS; ++k) {
            const double x = s_sum[k >> 2][k & 3];
            if (x > 0.0) last = k, last_before = before;
            if (found < 0 && before + x > at) found = k, found_before = before;
            before += x;
        }
        s_segment = found < 0 ? last : found;
        s_before = found < 0 ? last_before : found_before;
    }
    __syncthreads();
    if (w != 0) return;
    const float r = a.r[b];
    const double at = r > 0.f ? (double)r * total : 0.0;
    const int begin = s_segment * size, end = min(V, begin + size);
    double before = s_before;
    int word = -1;                                         // the last word with a weight, until one passes
    for (int v0 = begin; v0 < end; v0 += 64) {
        const int v = v0 + lane;
        const double x = v < end ? weight(p, q, v) : 0.0;
        const double upto = before + wave_scan_f64(x, lane);
        const unsigned long long pass = __ballot(x > 0.0 && upto > at), any = __ballot(x > 0.0);
        if (pass) {
            word = v0 + __builtin_ctzll(pass);
            break;
        }
        if (any) word = v0 + 63 - __builtin_clzll(any);
        before = __shfl(upto, 63);
    }
    if (lane == 0) tokens[take] = word;
}

static echo_status_t check_draft(const echo_draft_desc_t *d) {
    if (!d) return ECHO_ERR_NULL;
    if (d->dtype != ECHO_F32 && d->dtype != ECHO_BF16) return ECHO_ERR_DTYPE;
    if (d->B < 1 || d->K < 1 || d->V < 1 || d->B > ECHO_DRAFT_MAX_B || d->K > ECHO_DRAFT_MAX_K || d->V > ECHO_DRAFT_MAX_V) return ECHO_ERR_SHAPE;
    return ECHO_OK;
}

}  // namespace echo

extern "C" {

size_t echo_draft_verify_workspace_bytes(const echo_draft_desc_t *desc) { return 0; }

echo_status_t echo_draft_verify(const echo_draft_desc_t *desc, const int32_t *drafted, const int32_t *n_drafted, const void *draft,
                                const void *target, const float *u, const float *r, int32_t *tokens, int32_t *taken, void *workspace,
                                size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_draft(desc)) return s;
    if (!drafted || !draft || !target || !u || !r || !tokens || !taken) return ECHO_ERR_NULL;
    uintptr_t m = 0;
    for (const void *p : {(const void *)drafted, (const void *)n_drafted, draft, target, (const void *)u, (const void *)r, (const void *)tokens,
                          (const void *)taken, (const void *)workspace})
        m |= (uintptr_t)p;
    if (m & 15u) return ECHO_ERR_ALIGN;
    const DraftArgs a{drafted, n_drafted, draft, target, u, r, desc->B, desc->K, desc->V, tokens, taken};
    hipStream_t st = static_cast<hipStream_t>(stream);
    LaunchRecord rec = launch_begin("draft_verify", st);
    if (desc->dtype == ECHO_F32) k_draft_verify<float><<<desc->B, 64 * kDraftWaves, 0, st>>>(a);
    else k_draft_verify<bf16_t><<<desc->B, 64 * kDraftWaves, 0, st>>>(a);
    return launch_end(rec);
}

}  // extern "C"
