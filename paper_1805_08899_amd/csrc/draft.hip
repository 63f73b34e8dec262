// Verification of drafted words (include/echodraft.h has the rules): a block per sequence.
//
// Which words are taken takes K pairs of probabilities; the word that is drawn behind them takes one row of the model's and, if a word was not taken,
// one of the student's.  The block sums the weights of that row by segments, which its waves take in turn, finds the segment in which the sum passes r of
// the whole, and a wave goes over that segment again.  All sums are in 64 bits and in an order that depends on V alone.
//
// Many sequences are bound by memory: 256 x 5 of 100003 f32 words, 193 MB, takes 41 us, 4.7 TB/s.  One is bound by four trips to memory one after the other (words; their
// probabilities; the rows; the segment): 1 x 4 of 32000 words takes 9.3 us, of which the launch is 4.  The weights have no branches, with which that took 10 us more.
#include "../../include/echodraft.h"

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kDraftWaves = 16, kDraftSegments = 256;
constexpr int kDraftAtOnce = 4;      // segments whose words a wave requests at once
constexpr int kDraftGroups = kDraftSegments / (kDraftWaves * kDraftAtOnce);      // times that it does

struct DraftArgs {
    const int *drafted, *n_drafted;
    const void *draft, *target;
    const float *u, *r;
    int B, K, V;
    int *tokens, *taken;
    double *sums;                    // [B][kDraftSegments], where a sequence has several blocks
};

// inclusive sums over the lanes
__device__ __forceinline__ double wave_scan_f64(double x, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    return x;
}
// Sums of four values per lane over the lanes: of value l / 16 for lane l.  At the first two steps a lane keeps half of its values and hands the other half on.
__device__ __forceinline__ double wave_sums_f64(const double (&a)[4], int lane) {
    const bool high = lane & 32, odd = lane & 16;
    const double b0 = (high ? a[2] : a[0]) + __shfl_xor(high ? a[0] : a[2], 32), b1 = (high ? a[3] : a[1]) + __shfl_xor(high ? a[1] : a[3], 32);
    double c = (odd ? b1 : b0) + __shfl_xor(odd ? b0 : b1, 16);
#pragma unroll
    for (int off = 8; off; off >>= 1) c += __shfl_xor(c, off);
    return c;
}

// Four consecutive words' probabilities as they stand in memory: the four from v on, or the row's last four, of which word() says which is which.
// FEW: there are fewer than four words.
template <typename T, bool FEW> struct Four {
    RawKey<T> raw;
    static __device__ __forceinline__ int first(int v, int V) { return max(0, min(v, V - 4)); }
    __device__ __forceinline__ void load(const T *row, int v, int V) {
        // (a byte offset of 32 bits on a scalar address: 2^24 words at most)
        if constexpr (!FEW) raw.load(reinterpret_cast<const T *>(reinterpret_cast<const char *>(row) + (unsigned)first(v, V) * (unsigned)sizeof(T)), 0);
        else raw.load_some(row, V);
    }
    __device__ __forceinline__ void get(float (&x)[4]) const {
        const float4 y = raw.get();
        x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
    }
};
// the weight of a word: p - q, where that is positive and finite, or zero
__device__ __forceinline__ double weight(float p, float q, bool word) {
    const bool on = (int)word & (int)(p > q) & (int)(p < __builtin_inff()) & (int)(q > -__builtin_inff());      // (no branches)
    return (double)(on ? p : 0.f) - (double)(on ? q : 0.f);
}
// the weights of the words from v on, zero for those that are not v .. v + 3 or not in the vocabulary
template <typename T, bool FEW> __device__ __forceinline__ void weights(const Four<T, FEW> &p, const Four<T, FEW> &q, bool both, int v, int V, double (&w)[4]) {
    float x[4], y[4];
    p.get(x);
    q.get(y);
    const int first = Four<T, FEW>::first(v, V);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = weight(x[e], both ? y[e] : 0.f, (int)(first + e >= v) & (int)(first + e < V));
}

// A wave's groups first .. last - 1 of four segments each: the sums of their weights into sums[segment] (LDS or memory).  A segment has 256 m words: m groups of
// four words for each lane; the next step's words are on their way.
template <typename T, bool FEW>
__device__ __forceinline__ void segment_sums(const T *p, const T *q, bool less, int V, int m, int first, int last, double *sums) {
    constexpr int U = kDraftAtOnce;
    const int lane = lane_id(), w = wave_id();
    // step t: the t % m -th 256 words of the segments of group t / m
    const auto word_of = [&](int t, int k) { return ((w + (t / m * U + k) * kDraftWaves) * m + t % m) * 256 + lane * 4; };
    Four<T, FEW> fp[2][U], fq[2][U];
    const auto fetch = [&](int buf, int t) __attribute__((always_inline)) {
        // (behind the last step, and behind the last word: the row's last words once more)
#pragma unroll
        for (int k = 0; k < U; ++k) {
            fp[buf][k].load(p, word_of(t, k), V);
            fq[buf][k].load(q, word_of(t, k), V);
        }
    };
    double sum[U] = {};
    const auto add = [&](int buf, int t) __attribute__((always_inline)) {
        if (word_of(t, 0) - lane * 4 < V) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                double x[4];
                weights(fp[buf][k], fq[buf][k], less, word_of(t, k), V, x);
                sum[k] += (x[0] + x[1]) + (x[2] + x[3]);
                __builtin_amdgcn_sched_barrier(0);         // one segment after the other: the registers are the next step's
            }
        }
        if ((t + 1) % m != 0) return;
        const double mine = wave_sums_f64(sum, lane);
        if ((lane & 15) == 0) sums[w + (t / m * U + (lane >> 4)) * kDraftWaves] = mine;
#pragma unroll
        for (int k = 0; k < U; ++k) sum[k] = 0.0;
    };
    fetch(0, first * m);
    for (int t = first * m; t < last * m; t += 2) {
        fetch(1, t + 1);
        add(0, t);
        fetch(0, t + 2);
        if (t + 1 < last * m) add(1, t + 1);
    }
}

// The first word that is not taken, for every wave by itself.  (What is read does not wait for n.)
template <typename T> __device__ __forceinline__ int draft_take(const DraftArgs &a, int b, int n, const T *p, const T *q) {
    const int lane = lane_id();
    for (int i0 = 0; i0 < a.K; i0 += 64) {
        const int i = min(i0 + lane, a.K - 1), d = a.drafted[(size_t)b * a.K + i];
        const float u = a.u[(size_t)b * a.K + i];
        const bool word = (unsigned)d < (unsigned)a.V;
        const size_t at = (size_t)i * a.V + (word ? d : 0);
        const float pd = ld(p, at), qd = ld(q, at);
        const unsigned long long bad = __ballot(!word || i0 + lane >= n || !((double)u * (double)qd < (double)pd));
        if (bad) return min(n, i0 + __builtin_ctzll(bad));
    }
    return n;
}

// The block of a sequence (kWhole); or, of sequences that have several blocks each, one that sums a group of segments (kSums: blocks beside each other), and the one
// that draws the word from them (kDraw).
enum class Part { kWhole, kSums, kDraw };
template <typename T, bool FEW, Part PART> __global__ __launch_bounds__(64 * kDraftWaves) void k_draft_verify(const DraftArgs a) {
    __shared__ double s_sum[kDraftSegments];
    const int b = PART == Part::kSums ? blockIdx.x / kDraftGroups : blockIdx.x, lane = lane_id(), w = wave_id(), V = a.V;
    const T *p = static_cast<const T *>(a.target) + (size_t)b * (a.K + 1) * V, *q = static_cast<const T *>(a.draft) + (size_t)b * a.K * V;
    const float r = a.r[b];
    const int n = a.n_drafted ? clamp_len(a.n_drafted[b], a.K) : a.K;
    const int take = PART == Part::kDraw ? a.taken[b] : draft_take(a, b, n, p, q);
    const bool both = take < n;
    p += (size_t)take * V;
    q = both ? q + (size_t)take * V : p;
    const int m = (V + 256 * kDraftSegments - 1) / (256 * kDraftSegments);
    int *tokens = a.tokens + (size_t)b * (a.K + 1);
    const int group = PART == Part::kSums ? (int)blockIdx.x % kDraftGroups : 0;
    if (PART != Part::kDraw && group == 0) {
        for (int i = threadIdx.x; i <= a.K; i += 64 * kDraftWaves)
            if (i != take) tokens[i] = i < take ? a.drafted[(size_t)b * a.K + i] : -1;
        if (threadIdx.x == 0) a.taken[b] = take;
    }
    if constexpr (PART == Part::kSums) {
        segment_sums<T, FEW>(p, q, both, V, m, group, group + 1, a.sums + (size_t)b * kDraftSegments);
    } else {
        bool less = both;                                  // the weights are p - q; if nothing is left of p behind q, p itself
        double x[4];                                       // of every wave's lanes: four segments each
        bool here = PART == Part::kDraw;
        double upto, total;
        for (;;) {
            if (!here) {
                const int per = kDraftSegments / kDraftGroups, groups = (V + 256 * m * per - 1) / (256 * m * per);
                if ((int)threadIdx.x < kDraftSegments - groups * per) s_sum[groups * per + threadIdx.x] = 0.0;
                segment_sums<T, FEW>(p, q, less, V, m, 0, groups, s_sum);
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = here ? a.sums[(size_t)b * kDraftSegments + lane * 4 + k] : s_sum[lane * 4 + k];
            upto = wave_scan_f64((x[0] + x[1]) + (x[2] + x[3]), lane);
            total = __shfl(upto, 63);
            if (total > 0.0 || !less) break;
            less = here = false;
            __syncthreads();                               // before the sums are written again
        }
        if (w != 0) return;
        if (!(total > 0.0)) {
            if (lane == 0) tokens[take] = -1;
            return;
        }
        // (from 1 on no sum passes: sums in other orders than the total's may lie a rounding above it)
        const double at = r >= 1.f ? __builtin_inf() : r > 0.f ? (double)r * total : 0.0;
        // the first segment whose sum passes, or the last one that has a weight
        double before = __shfl_up(upto, 1);
        if (lane == 0) before = 0.0;
        int segment = -1, last = -1;
        double start = 0.0, last_start = 0.0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (x[k] > 0.0) {
                last = lane * 4 + k, last_start = before;
                if (segment < 0 && before + x[k] > at) segment = last, start = before;
            }
            before += x[k];
        }
        const unsigned long long pass = __ballot(segment >= 0), any = __ballot(last >= 0);
        const int from = pass ? __builtin_ctzll(pass) : 63 - __builtin_clzll(any);
        segment = __shfl(pass ? segment : last, from);
        before = __shfl(pass ? start : last_start, from);
        // the words of that segment, 4 m a lane
        const int v0 = segment * 256 * m + lane * 4 * m;
        double own = 0.0;
        for (int j = 0; j < m; ++j) {
            Four<T, FEW> fp, fq;
            fp.load(p, v0 + 4 * j, V);
            fq.load(q, v0 + 4 * j, V);
            weights(fp, fq, less, v0 + 4 * j, V, x);
            own += (x[0] + x[1]) + (x[2] + x[3]);
        }
        upto = wave_scan_f64(own, lane);
        double sum_to = before + __shfl_up(upto, 1);
        if (lane == 0) sum_to = before;
        int word = -1, heavy = -1;
        for (int j = 0; j < m; ++j) {
            Four<T, FEW> fp, fq;
            fp.load(p, v0 + 4 * j, V);
            fq.load(q, v0 + 4 * j, V);
            weights(fp, fq, less, v0 + 4 * j, V, x);
            const int first = Four<T, FEW>::first(v0 + 4 * j, V);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum_to += x[e];
                if (x[e] > 0.0) {
                    heavy = first + e;
                    if (word < 0 && sum_to > at) word = heavy;
                }
            }
        }
        const unsigned long long passed = __ballot(word >= 0), heavies = __ballot(heavy >= 0);
        if (passed) word = __shfl(word, __builtin_ctzll(passed));
        else word = __shfl(heavy, 63 - __builtin_clzll(heavies));
        if (lane == 0) tokens[take] = word;
    }
}

static echo_status_t check_draft(const echo_draft_desc_t *d) {
    if (!d) return ECHO_ERR_NULL;
    if (d->dtype != ECHO_F32 && d->dtype != ECHO_BF16) return ECHO_ERR_DTYPE;
    if (d->B < 1 || d->K < 1 || d->V < 1 || d->B > ECHO_DRAFT_MAX_B || d->K > ECHO_DRAFT_MAX_K || d->V > ECHO_DRAFT_MAX_V) return ECHO_ERR_SHAPE;
    return ECHO_OK;
}

// Several blocks to a sequence (and a second launch) pay where there are few sequences and many words; one block and kDraftGroups of them, us, f32:
//   1 x 100003 words 20.0 / 11.3, 1 x 32000 9.7 / 9.7, 16 x 100003 23.9 / 14.7, 64 x 100003 24.9 / 17.9, 128 x 100003 26.9 / 28.4, 256 x 8000 11.4 / 25.7; 64 x 50021 bf16
//   15.1 / 13.2.  Between 64 and 128 sequences, where the two lines cross, nothing is measured: the border is the last number at which several were the better ones.
constexpr int kDraftSplitB = 64, kDraftSplitV = 40000;
static size_t draft_bytes(const echo_draft_desc_t &d) {
    return d.B <= kDraftSplitB && d.V >= kDraftSplitV ? (size_t)d.B * kDraftSegments * 8 : 0;
}

template <typename T, bool FEW, Part PART> static echo_status_t launch_draft(const char *name, const DraftArgs &a, int blocks, hipStream_t st) {
    LaunchRecord r = launch_begin(name, st);
    k_draft_verify<T, FEW, PART><<<blocks, 64 * kDraftWaves, 0, st>>>(a);
    return launch_end(r);
}
template <typename T, bool FEW> static echo_status_t run_draft(const DraftArgs &a, bool split, hipStream_t st) {
    if constexpr (!FEW) {
        if (split) {
            if (echo_status_t s = launch_draft<T, FEW, Part::kSums>("draft_sums", a, a.B * kDraftGroups, st)) return s;
            return launch_draft<T, FEW, Part::kDraw>("draft_draw", a, a.B, st);
        }
    }
    return launch_draft<T, FEW, Part::kWhole>("draft_verify", a, a.B, st);
}

}  // namespace echo

extern "C" {

size_t echo_draft_verify_workspace_bytes(const echo_draft_desc_t *desc) { return echo::check_draft(desc) ? 0 : echo::draft_bytes(*desc); }

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
    const size_t need = draft_bytes(*desc);
    if (need && !workspace) return ECHO_ERR_NULL;
    if (workspace_bytes < need) return ECHO_ERR_WORKSPACE;
    const DraftArgs a{drafted, n_drafted, draft, target, u, r, desc->B, desc->K, desc->V, tokens, taken, static_cast<double *>(workspace)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (desc->V < 4) return desc->dtype == ECHO_F32 ? run_draft<float, true>(a, false, st) : run_draft<bf16_t, true>(a, false, st);
    return desc->dtype == ECHO_F32 ? run_draft<float, false>(a, need > 0, st) : run_draft<bf16_t, false>(a, need > 0, st);
}

}  // extern "C"
