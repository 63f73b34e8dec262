// The target of a distillation as the products of the vocabulary loss meet it (include/echodistill.h has the formulas): of every row its words in
// ascending order, each once, with their shares, and where among them each range of kMarkWords words of the vocabulary begins.
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
    const float *own;                // [N]: sum of share log share
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

// The shares of words v .. v + 3 in row n (below 0: none), v a multiple of 4.  For few rows: the lane looks through the row's words of v's range.
__device__ __forceinline__ f32x4 teacher_shares(const Teacher &t, int n, int v) {
    f32x4 q = {0.f, 0.f, 0.f, 0.f};
    const int mark = v / kMarkWords;
    if (n < 0 || mark + 1 >= t.marks) return q;
    const unsigned char *start = t.start + (size_t)n * t.marks + mark;
    for (int e = start[0]; e < start[1]; ++e) {
        const int r = t.words[(size_t)n * t.K + e] - v;
        const float x = t.shares[(size_t)n * t.K + e];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r == k) q[k] = x;
    }
    return q;
}

// The shares of 16 rows and WORDS words for a wave that holds their logits as the matrix cores leave them (lane l: row l % 16): put into LDS where they are,
// read by everybody, and taken out again.  Nothing of it but the few words that a row has among these costs more than one read.
template <int WORDS> struct TeacherTile {
    static constexpr int PITCH = WORDS + 4, BYTES = 16 * PITCH * 4;            // 4 more floats a row: a fragment's 16 rows take all banks
    const Teacher &t;
    float *mine;
    int v0, row, begin, end;
    bool any;
    // `on`: it is used; lds: BYTES of every wave, nobody else's from here to the last clear()
    __device__ __forceinline__ TeacherTile(const Teacher &teacher, float *lds, int first_word, bool on) : t(teacher), v0(first_word) {
        mine = lds + wave_id() * 16 * PITCH;
        if (!on) return;
        for (int k = lane_id(); k < 16 * PITCH / 4; k += 64) reinterpret_cast<f32x4 *>(mine)[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void put(int n) {                               // the lane's row, below 0: none
        row = n;
        begin = end = 0;
        const int mark = v0 / kMarkWords;
        if (n >= 0 && mark + 1 < t.marks) {
            const unsigned char *start = t.start + (size_t)n * t.marks + mark;
            begin = start[0], end = start[1];
        }
        any = __ballot(begin < end) != 0;
        if (any) write(false);
    }
    __device__ __forceinline__ void clear() {
        if (any) write(true);
    }
    __device__ __forceinline__ f32x4 get(int v) const {                        // of the lane's row, words v0 + v .. + 3
        return any ? *reinterpret_cast<const f32x4 *>(mine + (lane_id() & 15) * PITCH + v) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // four lanes share a row
    __device__ __forceinline__ void write(bool zero) {
        wait();
        for (int e = begin + (lane_id() >> 4); e < end; e += 4) {
            const int v = t.words[(size_t)row * t.K + e] - v0;
            if ((unsigned)v < (unsigned)WORDS) mine[(lane_id() & 15) * PITCH + v] = zero ? 0.f : t.shares[(size_t)row * t.K + e];
        }
        wait();
    }
    // what this wave has written or read in LDS is done: the lanes' exchange needs no more
    static __device__ __forceinline__ void wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
};

}  // namespace echo
