// The teacher's lists made ready for the products (distill.hpp): a wave per row.  An entry's place among the row's words in ascending order is the number of
// entries with a smaller key, word and place in the list in one number: with K entries at most each lane compares its own with all, four at a time.  Equal words
// then stand beside each other, and the first of them takes the shares of all, in the list's order.
#include "distill.hpp"

#include "launch.hpp"

namespace echo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(256) void k_distill_lists(const TeacherLists a) {
    constexpr int MOST = ECHO_DISTILL_MAX_K, U = MOST / 64, kNone = 0x7fffffff;          // (no key is above it)
    static_assert(ECHO_VOCAB_MAX_ROWS <= 1 << 24 && MOST <= 128, "keys of 31 bits");
    __shared__ __align__(16) int s_key[4][MOST], s_sorted[4][MOST + 1], s_once[4][MOST];
    __shared__ float s_share[4][MOST];
    const int lane = lane_id(), w = wave_id(), n = blockIdx.x * 4 + w;
    if (n >= a.N) return;
    const auto settle = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };      // a wave's own exchange through LDS
    int word[U], key[U];
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
    // the sum without the first of the largest, which is 1: log(1 + rest) keeps the digits of a teacher that is sure of a word
    float rest = 0.f;
    bool out = false;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        x[k] = (x[k] - top) / a.temperature;
        q[k] = in[k] ? expf(x[k]) : 0.f;
        const unsigned long long ones = __ballot(q[k] == 1.f);
        rest += !out && ones && lane == __builtin_ctzll(ones) ? 0.f : q[k];
        out |= ones != 0;
    }
    rest = wave_sum(rest);
    const float sum = 1.f + rest, log_sum = log1pf(rest);
    float own = 0.f;
    int label = -1, many = 0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        q[k] /= sum;
        if (in[k] && q[k] != 0.f) own += q[k] * (x[k] - log_sum);
        const unsigned long long m = __ballot(in[k]);
        if (label < 0 && m) label = __builtin_amdgcn_readlane(word[k], __builtin_ctzll(m));
        many += __builtin_popcountll(m);
        key[k] = in[k] ? word[k] << 7 | (lane + 64 * k) : kNone;
        s_key[w][lane + 64 * k] = key[k];
    }
    own = wave_sum(own);
    settle();
    int below[U] = {};
    for (int j = 0; j < a.K; j += 4) {
        const i32x4 other = *reinterpret_cast<const i32x4 *>(&s_key[w][j]);
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) below[k] += other[i] < key[k];
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (in[k]) s_sorted[w][below[k]] = word[k], s_share[w][below[k]] = q[k];
    if (lane == 0) s_sorted[w][many] = kNone;
    settle();
    int once = 0;                                          // words so far, each once
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int at = lane + 64 * k, mine = s_sorted[w][min(at, many)];
        const bool first = at < many && (at == 0 || s_sorted[w][at - 1] != mine);
        const unsigned long long m = __ballot(first);
        if (first) {
            float share = s_share[w][at];
            for (int j = at + 1; s_sorted[w][j] == mine; ++j) share += s_share[w][j];
            const int to = once + __builtin_popcountll(m & ((1ull << lane) - 1));
            s_once[w][to] = mine;
            a.words_out[(size_t)n * a.K + to] = mine;
            a.shares[(size_t)n * a.K + to] = share;
        }
        once += __builtin_popcountll(m);
    }
    settle();
    // four marks a lane, whose searches go on side by side
    constexpr int S = 4;
    for (int m0 = lane; m0 < a.marks; m0 += 64 * S) {
        int lo[S];
#pragma unroll
        for (int i = 0; i < S; ++i) lo[i] = 0;
#pragma unroll
        for (int step = MOST / 2; step; step >>= 1) {
#pragma unroll
            for (int i = 0; i < S; ++i) {
                const int at = lo[i] + step - 1;
                if (at < once && s_once[w][at] < (m0 + 64 * i) * kMarkWords) lo[i] += step;
            }
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            // (of 128 words the steps reach 127)
            if (lo[i] < once && s_once[w][lo[i]] < (m0 + 64 * i) * kMarkWords) ++lo[i];
            if (m0 + 64 * i < a.marks) a.start[(size_t)n * a.marks + m0 + 64 * i] = (unsigned char)lo[i];
        }
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
