// The target of a distillation as the products of the vocabulary loss meet it (include/echodistill.h has the formulas): of every row its words in
// ascending order, each once, with their shares, and where among them each range of kMarkWords words of the vocabulary begins.
//
// The products bound it, as they bound the vocabulary loss: 8192 x 100003 x 2048 bf16 12.5 ms, both passes.  What the teacher adds to it: the lists (24 us each pass; 64 rows of
// 16 entries 5 us), in the forward pass a pass over the logits in registers (4 % of the labels' time there, 12 % of
// 6400 x 32000 x 1024) and a look at the maxima of the entries' tiles (8 us; 3 us of 6400 rows), in the backward pass 2 %.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/echodistill.h"
#include "common.hpp"

namespace echo {

constexpr int kMarkWords = 128;

struct Teacher {
    const int *words;                // [N][K], ascending
    const float *shares;             // [N][K]
    const unsigned char *start;      // [N][marks]: how many of the row's words are below kMarkWords times the mark's number
    const float *own;                // [N]: sum of share log share, small for a teacher that is sure of a word
    int K, marks;
    float inv_t, temperature;
    __device__ __forceinline__ void from_row(int n) {
        words += (size_t)n * K;
        shares += (size_t)n * K;
        start += (size_t)n * marks;
        own += n;
    }
};

// What makes it
struct TeacherLists {
    const int *words;
    const float *logits, *dloss;     // dloss: or null (forward)
    int N, V, K, marks;
    float temperature;
    int *labels, *words_out;         // labels [N]: a word of the row, or -1: the row takes part in nothing
    float *own, *dloss_out, *shares; // dloss_out: dloss by the temperature
    unsigned char *start;
};
echo_status_t launch_teacher_lists(const TeacherLists &l, hipStream_t st);

// The shares of TN times 16 rows and of WORDS words for a wave that holds their logits as the matrix cores leave them (lane l: row l % 16 of each): put into LDS
// where they are, read by everybody, and taken out again.  Four lanes look after a row.  What a row has among these words is hardly ever more than an entry or
// two; the first four of all TN rows are requested together, in three trips to the caches (one row after the other, each with its own three, took 18 % of a
// tile of 256 x 256 x 1024).
// Where they stand: the row, and first and last entry + 1 in 8 bits each.  What does not depend on the logits may be requested in front of their product.
template <int TN> struct TeacherRanges {
    int row[TN], range[TN];
    // row_of(j): the lane's row among rows j, below 0: none; first_word: the wave's
    template <typename RowOf> __device__ __forceinline__ void look_up(const Teacher &t, int first_word, RowOf row_of) {
        const int mark = min(first_word / kMarkWords, t.marks - 2);
        const bool there = first_word / kMarkWords == mark;
#pragma unroll
        for (int j = 0; j < TN; ++j) row[j] = row_of(j);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const unsigned char *start = t.start + (size_t)max(row[j], 0) * t.marks + mark;
            range[j] = row[j] >= 0 && there ? start[0] | start[1] << 8 : 0;
        }
    }
};
template <int WORDS, int TN> struct TeacherTile {
    static constexpr int PITCH = WORDS + 4, BYTES = 16 * PITCH * 4;            // 4 more floats a row: a fragment's 16 rows take all banks
    const Teacher &t;
    float *mine;
    int v0;
    int row[TN], range[TN], word[TN];
    float share[TN];
    // `on`: it is used; lds: BYTES of every wave, nobody else's from here to the last clear()
    __device__ __forceinline__ TeacherTile(const Teacher &teacher, float *lds, int first_word, bool on, const TeacherRanges<TN> &r) : t(teacher), v0(first_word) {
        mine = lds + wave_id() * 16 * PITCH;
        if (!on) return;
        zero();
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            row[j] = r.row[j], range[j] = r.range[j];
            const int e = begin(j) + (lane_id() >> 4);
            const size_t at = (size_t)max(row[j], 0) * t.K + min(e, t.K - 1);
            word[j] = t.words[at];
            share[j] = t.shares[at];
        }
    }
    __device__ __forceinline__ int begin(int j) const { return range[j] & 255; }
    __device__ __forceinline__ int end(int j) const { return range[j] >> 8; }
    __device__ __forceinline__ void zero() {
        for (int k = lane_id(); k < 16 * PITCH / 4; k += 64) reinterpret_cast<f32x4 *>(mine)[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ float *place(int v) const { return mine + (lane_id() & 15) * PITCH + v; }
    __device__ __forceinline__ bool any(int j) const { return __ballot(begin(j) < end(j)) != 0; }
    __device__ __forceinline__ bool many(int j) const { return __ballot(begin(j) + 4 < end(j)) != 0; }
    __device__ __forceinline__ bool first(int j) const { return begin(j) + (lane_id() >> 4) < end(j) && (unsigned)(word[j] - v0) < (unsigned)WORDS; }
    __device__ __forceinline__ void put(int j) {
        if (!any(j)) return;
        wait();
        if (first(j)) *place(word[j] - v0) = share[j];
        if (many(j)) {
            constexpr int U = 4;
            for (int e0 = begin(j) + 4 + (lane_id() >> 4); __ballot(e0 < end(j)); e0 += 4 * U) {
                int w[U];
                float x[U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const size_t at = (size_t)max(row[j], 0) * t.K + min(e0 + 4 * k, t.K - 1);
                    w[k] = t.words[at], x[k] = t.shares[at];
                }
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (e0 + 4 * k < end(j) && (unsigned)(w[k] - v0) < (unsigned)WORDS) *place(w[k] - v0) = x[k];
            }
        }
        wait();
    }
    __device__ __forceinline__ f32x4 get(int j, int v) const {                 // of the lane's row, words v0 + v .. + 3
        return any(j) ? *reinterpret_cast<const f32x4 *>(place(v)) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void clear(int j) {
        if (!any(j)) return;
        wait();
        if (many(j)) zero();
        else if (first(j)) *place(word[j] - v0) = 0.f;
    }
    // what this wave has written or read in LDS is done: the lanes' exchange needs no more
    static __device__ __forceinline__ void wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
};

}  // namespace echo
