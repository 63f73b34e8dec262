// Tiled products of bf16 matrices with fp32 sums on the matrix cores, for the vocabulary loss: C[m, n] += sum_k A(m, k) B(n, k).
//
// An operand lies in memory in one of two ways, both with rows of `pitch` elements, a multiple of 8, from a 16-byte aligned address:
//   rows along k   element (m, k) at m * pitch + k    (logits: words and rows of h; dh: dz)
//   k along rows   element (m, k) at k * pitch + m    (dh: words; dW: dz and rows of h)
// and may consist of several planes, whose sum it is; the product then is the sum over a list of plane pairs, one pair's whole k axis after
// another's, which for the loop is one long k axis.
//
// A block computes a BM x BN tile.  Its operands pass through LDS in steps of 64 k, straight from memory (buffer loads to LDS, 16
// bytes per lane, no registers), STAGES - 1 steps ahead.  Such a load puts 64 x 16 consecutive bytes into LDS; which bytes of
// memory each lane asks for is free, and is chosen so that the reads below spread over all banks:
//   rows along k   a row is 8 groups of 16 bytes; group c of row r goes to place c ^ (r % 8).  A wave's fragment of 32 rows is read as 16
//                  bytes per lane.
//   k along rows   a row is BM / 32 groups of 64 bytes; group g of row k goes to place g ^ (k % 4).  A fragment is read with the transposing
//                  LDS load: sixteen lanes address 4 rows x 16 columns, and each receives a column's 4 numbers.
// Every lane checks its own rows, columns and k against the operand's ends, and asks for an address past the end of the buffer
// descriptor where it is outside: the load then delivers zeros.
#pragma once
#include "common.hpp"
#include "split.hpp"

namespace echo {

struct Operand {
    const bf16_t *p;        // element (0, 0) of plane 0
    size_t plane;           // elements from plane to plane
    int pitch;              // elements from row to row
    int rows;               // extent along m (or n)
};
// plane pairs, the small terms first: nibble i of a and b
struct PlanePairs {
    unsigned n, a, b;
};

constexpr int kStepK = 64;

template <int BM_, int BN_, int WM_, int WN_, int STAGES_> struct TileConfig {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;                // 32 x 32 tiles of a wave
    static constexpr int STAGE_BYTES = (BM + BN) * kStepK * 2;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
    static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "whole tiles");
    static_assert(BM / 8 % WAVES == 0 && BN / 8 % WAVES == 0, "whole loads per wave");
};

constexpr unsigned kOutside = 0x80000000u;                                     // past every descriptor below

typedef __attribute__((address_space(3))) void *lds_ptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));

// One operand's way from memory to LDS: ROWS = BM or BN, of which this block's tile begins at row0.
template <int ROWS, int WAVES, bool ALONG_ROWS> struct Loader {
    static constexpr int N = ROWS / 8 / WAVES;                                 // loads of 1 KB per wave and step
    static constexpr int ROW_BYTES = ALONG_ROWS ? ROWS * 2 : kStepK * 2, PER_ROW = ROW_BYTES / 16;
    unsigned off[N];                                                           // bytes from the step's base
    int k_of[N];                                                               // the first k of the lane's 16 bytes
    const char *base0, *base;                                                  // plane 0 at k = 0; the step under way
    size_t plane_bytes, step_bytes;

    __device__ __forceinline__ void init(const Operand &o, int row0, int w, int lane) {
        plane_bytes = o.plane * 2;
        step_bytes = ALONG_ROWS ? (size_t)kStepK * o.pitch * 2 : kStepK * 2;
        base0 = reinterpret_cast<const char *>(o.p) + (ALONG_ROWS ? (size_t)row0 * 2 : (size_t)row0 * o.pitch * 2);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (w * N + i) * 64 + lane, row = at / PER_ROW, slot = at % PER_ROW;
            if (ALONG_ROWS) {
                const int col = (((slot >> 2) ^ (row & 3)) * 4 + (slot & 3)) * 8;
                k_of[i] = row;
                off[i] = row0 + col < o.rows ? (unsigned)(row * o.pitch + col) * 2u : kOutside;
            } else {
                const int k = (slot ^ (row & 7)) * 8;
                k_of[i] = k;
                off[i] = row0 + row < o.rows ? (unsigned)(row * o.pitch + k) * 2u : kOutside;
            }
        }
    }
    __device__ __forceinline__ void plane(unsigned p) { base = base0 + p * plane_bytes; }
    // `left`: k from this step's begin to the end of the axis
    __device__ __forceinline__ void load(char *lds, int w, int left) {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0x7ffffff0, 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned o = left >= kStepK || k_of[i] < left ? off[i] : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(lds + (w * N + i) * 1024), 16, o, 0, 0, 0);
        }
        base += step_bytes;
    }
};

// Fragments of 32 rows x 16 k from LDS: lane l holds row l % 32, k = 8 (l / 32) .. + 7.
template <int ROWS, bool ALONG_ROWS, int TILES> struct Reader {
    static constexpr int ROW_BYTES = ALONG_ROWS ? ROWS * 2 : kStepK * 2;
    unsigned at[ALONG_ROWS ? TILES : kStepK / 16];
    __device__ __forceinline__ void init(int row0, int lane) {                 // row0: the wave's first row in the tile
        if (ALONG_ROWS) {
            const int k = 8 * (lane >> 5) + ((lane & 15) >> 2), in = (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
#pragma unroll
            for (int i = 0; i < TILES; ++i) at[i] = k * ROW_BYTES + (((row0 / 32 + i) ^ (k & 3)) * 64) + in;
        } else {
#pragma unroll
            for (int s = 0; s < kStepK / 16; ++s)
                at[s] = (row0 + (lane & 31)) * ROW_BYTES + (((2 * s + (lane >> 5)) ^ (lane & 7)) * 16);
        }
    }
    __device__ __forceinline__ u32x4 get(const char *lds, int i, int s) const {  // tile i, 16 k from 16 s on
        if constexpr (ALONG_ROWS) {
            const char *p = lds + at[i] + s * 16 * ROW_BYTES;
            typedef __attribute__((address_space(3))) s16x4 *tr_ptr;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + 4 * ROW_BYTES));
            const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
            return u32x4{a.x, a.y, b.x, b.y};
        } else {
            return *reinterpret_cast<const u32x4 *>(lds + at[s] + i * 32 * ROW_BYTES);
        }
    }
};

template <int N> __device__ __forceinline__ void wait_loads() {                // at most N loads of this wave still under way
    static_assert(N >= 0 && N < 64, "counter");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// (this wave's LDS reads have arrived: what it read may be overwritten behind the barrier)
__device__ __forceinline__ void block_barrier() { lds_barrier(); }

// acc[i][j]: rows m0 + 32 (wm TM + i), columns n0 + 32 (wn TN + j) of the product.  k_begin, k_end: this block's part of the k axis
// (k_begin a multiple of 64).  On return every wave has read its last fragment from LDS (the caller puts a barrier in
// front of other uses of it).
template <class C, bool A_ALONG, bool B_ALONG>
__device__ __forceinline__ void tile_product(f32x16 (&acc)[C::TM][C::TN], const Operand &A, const Operand &B, int m0, int n0, int k_begin,
                                             int k_end, const PlanePairs &pairs, char *lds) {
    const int lane = lane_id(), w = wave_id(), wm = w / C::WN, wn = w % C::WN;
    Loader<C::BM, C::WAVES, A_ALONG> la;
    Loader<C::BN, C::WAVES, B_ALONG> lb;
    la.init(A, m0, w, lane);
    lb.init(B, n0, w, lane);
    la.base0 += (size_t)(k_begin / kStepK) * la.step_bytes;
    lb.base0 += (size_t)(k_begin / kStepK) * lb.step_bytes;
    Reader<C::BM, A_ALONG, C::TM> ra;
    Reader<C::BN, B_ALONG, C::TN> rb;
    ra.init(wm * C::TM * 32, lane);
    rb.init(wn * C::TN * 32, lane);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j] = zero16();
    const int len = k_end - k_begin, steps = (len + kStepK - 1) / kStepK, total = steps * (int)pairs.n;
    int issued = 0, k_issued = 0, pair = 0;
    auto issue = [&]() {
        if (k_issued == 0) {
            la.plane(pairs.a >> (4 * pair) & 15u);
            lb.plane(pairs.b >> (4 * pair) & 15u);
            ++pair;
        }
        char *s = lds + (issued % C::STAGES) * C::STAGE_BYTES;
        la.load(s, w, len - k_issued);
        lb.load(s + C::BM * kStepK * 2, w, len - k_issued);
        ++issued;
        k_issued += kStepK;
        if (k_issued >= len) k_issued = 0;
    };
    constexpr int LOADS = decltype(la)::N + decltype(lb)::N;
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s)
        if (s < total) issue();
    for (int t = 0; t < total; ++t) {
        // this wave's loads of step t are there, then everybody's; and everybody is done with the stage that is written next
        if (issued - t >= C::STAGES - 1) wait_loads<LOADS *(C::STAGES - 2)>();
        else wait_loads<0>();
        block_barrier();
        if (issued < total) issue();
        const char *a = lds + (t % C::STAGES) * C::STAGE_BYTES, *b = a + C::BM * kStepK * 2;
#pragma unroll
        for (int s = 0; s < kStepK / 16; ++s) {
            u32x4 fa[C::TM], fb[C::TN];
#pragma unroll
            for (int i = 0; i < C::TM; ++i) fa[i] = ra.get(a, i, s);
#pragma unroll
            for (int j = 0; j < C::TN; ++j) fb[j] = rb.get(b, j, s);
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j) acc[i][j] = mfma32(fa[i], fb[j], acc[i][j]);
        }
    }
}

}  // namespace echo
