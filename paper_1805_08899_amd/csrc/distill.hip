// The teacher's lists made ready for the products (distill.hpp): a wave per row.  Its words are K at most, so each lane compares its own with all of
// them: whether the word stood in front already, the share of all its places, and how many words are below it.
#include "distill.hpp"

#include "launch.hpp"

namespace echo {

__global__ __launch_bounds__(256) void k_distill_lists(const TeacherLists a) {
    constexpr int MOST = ECHO_DISTILL_MAX_K, U = MOST / 64, kNone = 0x7fffffff;
    __shared__ int s_word[4][MOST], s_once[4][MOST], s_sorted[4][MOST];
    __shared__ float s_share[4][MOST];
    const int lane = lane_id(), w = wave_id(), n = blockIdx.x * 4 + w;
    if (n >= a.N) return;
    const auto settle = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };      // a wave's own exchange through LDS
    int word[U];
    float x[U], q[U];
    bool in[U];
    float top = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int e = lane + 64 * k;
        word[k] = e < a.K ? a.words[(size_t)n * a.K + e] : -1;
        x[k] = e < a.K ? a.logits[(size_t)n * a.K + e] : 0.f;
        in[k] = (unsigned)word[k] < (unsigned)a.V && x[k] != -__builtin_inff();
        if (in[k]) top = fmaxf(top, x[k]);
    }
    top = wave_max(top);
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        x[k] = (x[k] - top) / a.temperature;
        q[k] = in[k] ? expf(x[k]) : 0.f;
        sum += q[k];
    }
    sum = wave_sum(sum);
    const float log_sum = logf(sum);
    float own = 0.f;
    int label = -1;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        q[k] /= sum;
        if (in[k] && q[k] != 0.f) own += q[k] * (x[k] - log_sum);
        const unsigned long long m = __ballot(in[k]);
        if (label < 0 && m) label = __builtin_amdgcn_readlane(word[k], __builtin_ctzll(m));
        s_word[w][lane + 64 * k] = in[k] ? word[k] : kNone;
        s_share[w][lane + 64 * k] = q[k];
    }
    own = wave_sum(own);
    settle();
    bool first[U];
    float share[U];
#pragma unroll
    for (int k = 0; k < U; ++k) first[k] = in[k], share[k] = 0.f;
    for (int j = 0; j < a.K; ++j) {
        const int other = s_word[w][j];
        const float y = s_share[w][j];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool same = in[k] && other == word[k];
            share[k] += same ? y : 0.f;
            first[k] = first[k] && !(same && j < lane + 64 * k);
        }
    }
    int many = 0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        s_once[w][lane + 64 * k] = first[k] ? word[k] : kNone;
        many += __builtin_popcountll(__ballot(first[k]));
    }
    settle();
    int below[U] = {};
    for (int j = 0; j < a.K; ++j) {
        const int other = s_once[w][j];
#pragma unroll
        for (int k = 0; k < U; ++k) below[k] += other < word[k];
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        if (!first[k]) continue;
        s_sorted[w][below[k]] = word[k];
        a.words_out[(size_t)n * a.K + below[k]] = word[k];
        a.shares[(size_t)n * a.K + below[k]] = share[k];
    }
    settle();
    for (int m = lane; m < a.marks; m += 64) {
        const long long border = (long long)m * kMarkWords;
        int lo = 0, hi = many;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (s_sorted[w][mid] < border) lo = mid + 1;
            else hi = mid;
        }
        a.start[(size_t)n * a.marks + m] = (unsigned char)lo;
    }
    if (lane != 0) return;
    a.labels[n] = label;
    a.own[n] = label < 0 ? 0.f : own;
    if (a.dloss) a.dloss_out[n] = label < 0 ? 0.f : a.temperature * a.dloss[n];
}

echo_status_t launch_teacher_lists(const TeacherLists &l, hipStream_t st) {
    LaunchRecord r = launch_begin("distill_lists", st);
    k_distill_lists<<<(l.N + 3) / 4, 256, 0, st>>>(l);
    return launch_end(r);
}

}  // namespace echo
