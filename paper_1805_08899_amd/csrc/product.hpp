// Tiled products of bf16 (HALF: fp16) matrices with fp32 sums on the matrix cores, for the vocabulary loss: C[m, n] = sum_k A(m, k) B(n, k).
//
// Both operands have their rows along k: element (m, k) at m * pitch + k, pitch a multiple of 8, first element 16-byte aligned.  An operand may
// consist of several planes, whose sum it is; the product then is the sum over a list of plane pairs, one pair's whole k axis after another's, which
// for the loop is one long k axis.
//
// A block computes a BM x BN tile with v_mfma_f32_16x16x32_bf16 (on operands of this kind the chip's power limit lets them run at 1941 TFLOP/s,
// v_mfma_f32_32x32x16_bf16 at 1735).  Its operands pass through LDS in steps of 64 k, two stages, straight from memory (buffer loads to LDS, 16 bytes
// per lane, no registers in between).  Such a load puts 64 x 16 consecutive bytes into LDS, eight rows of 128 bytes; which bytes of memory a lane asks
// for is free: the 8 groups of 16 bytes of row r stand in the order c ^ (r / 2 % 8), so that the 16 rows of a fragment, read as 16 bytes per lane, take
// all 64 banks (c ^ (r % 8): half of the LDS time went to conflicts).
// Every lane checks its own row and k against the operand's ends, and asks for an address past the end of the buffer descriptor where
// it is outside: the load then delivers zeros.
//
// What bounds it (8192^3, TFLOP/s, same data): matrix instructions alone 1600 to 1940 by the power limit, with the reads from LDS 1480, with a barrier
// per step 1420, with the loads 1300 (the library's product 1500); for 64 x 128 per wave the reads take 1536 and the arriving operands 512
// of a step's 2048 clocks of LDS bandwidth.
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
// plane pairs, the small terms first: nibble i of a and b.  HALF: of two pairs the first one's operand was stored kLowScale times as large (its
// values, 2^-11 of the other plane's, would meet the end of fp16's exponents): its sums are scaled back before the second pair.
struct PlanePairs {
    unsigned n, a, b;
};
constexpr float kLowScale = 0x1p11f;

constexpr int kStepK = 64;
constexpr int kStepBytes = kStepK * 2;

// AHEAD: fragments of the next 32 k and of the next step are read while the matrix cores work on these (one block of 8 waves per
// compute unit: 1250 -> 1315); without it (blocks of 4 waves, two to a compute unit, which fill each other's gaps: 1130, with it 990).
template <int BM_, int BN_, int WM_, int WN_, bool AHEAD_> struct TileConfig {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr bool AHEAD = AHEAD_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;                // 16 x 16 tiles of a wave
    static constexpr int LDS_BYTES = 2 * (BM + BN) * kStepBytes;
    static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole tiles");
    static_assert(BM / 8 % WAVES == 0 && BN / 8 % WAVES == 0, "whole loads per wave");
};

constexpr unsigned kOutside = 0x80000000u;                                     // past every descriptor below

typedef __attribute__((address_space(3))) void *lds_ptr;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <bool HALF = false> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {   // 32 k: lane l: row l % 16, k = 8 (l / 16) .. + 7
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// accumulator r of lane l: row 4 (l / 16) + r, column l % 16

// One operand's way from memory to LDS: ROWS = BM or BN, of which this block's tile begins at row0.
template <int ROWS, int WAVES> struct Loader {
    static constexpr int N = ROWS / 8 / WAVES;                                 // loads of 1 KB per wave and step
    unsigned off[N];                                                           // bytes from the step's base
    const char *base0, *base;                                                  // plane 0 at the first k; the step under way
    size_t plane_bytes;

    static __device__ __forceinline__ int row_of(int i, int w, int lane) { return (w * N + i) * 8 + (lane >> 3); }
    static __device__ __forceinline__ int k_of(int i, int w, int lane) { return ((lane & 7) ^ (row_of(i, w, lane) >> 1 & 7)) * 8; }

    __device__ __forceinline__ void init(const Operand &o, int row0, int k_begin, int w, int lane) {
        plane_bytes = o.plane * 2;
        // from the wave's first row, so that a lane's offset stays below 2^31 for every pitch up to 2^24 (32 rows and less per wave)
        static_assert(N * 8 <= 32, "offsets");
        base0 = reinterpret_cast<const char *>(o.p) + ((size_t)(row0 + w * N * 8) * o.pitch + k_begin) * 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row_of(i, w, lane);
            off[i] = row0 + row < o.rows ? (unsigned)((row - w * N * 8) * o.pitch + k_of(i, w, lane)) * 2u : kOutside;
        }
    }
    __device__ __forceinline__ void plane(unsigned p) { base = base0 + p * plane_bytes; }
    // `left`: k from this step's begin to the end of the axis
    __device__ __forceinline__ void load(int i, char *lds, int w, int left) {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0x7ffffff0, 0x00020000);
        unsigned o = off[i];
        if (left < kStepK && k_of(i, w, lane_id()) >= left) o = kOutside;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(lds + (w * N + i) * 1024), 16, o, 0, 0, 0);
        if (i == N - 1) base += kStepBytes;
    }
};

// At most N loads of this wave are still under way.  (The builtin, not a statement: the compiler counts the loads itself and would wait
// once more in front of the next read from LDS.)
template <int N> __device__ __forceinline__ void wait_loads() {
    static_assert(N >= 0 && N < 64, "counter");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
    asm volatile("" ::: "memory");
}

template <class C, bool HALF> struct Pipeline {
    static constexpr int TM = C::TM, TN = C::TN, F = TM + TN;
    typedef Loader<C::BM, C::WAVES> LoadA;
    typedef Loader<C::BN, C::WAVES> LoadB;
    static constexpr int LA = LoadA::N, L = LA + LoadB::N;
    static constexpr int A_BYTES = C::BM * kStepBytes, B_BYTES = C::BN * kStepBytes;
    typedef f32x4 Acc[TM][TN];
    LoadA la;
    LoadB lb;
    unsigned a_at[2], b_at[2];                                                 // this lane's place in a stage, by half step
    u32x4 fa[C::AHEAD ? 2 : 1][TM], fb[C::AHEAD ? 2 : 1][TN];
    PlanePairs pairs;
    int w, len, total, issued, k_issued, pair, scale_at;

    // fragment f of half step s: A 0, then B, then the rest of A
    __device__ __forceinline__ void read(int buf, const char *a, const char *b, int s, int f) {
        if (f == 0) fa[buf][0] = *reinterpret_cast<const u32x4 *>(a + a_at[s]);
        else if (f <= TN) fb[buf][f - 1] = *reinterpret_cast<const u32x4 *>(b + b_at[s] + (f - 1) * 16 * kStepBytes);
        else fa[buf][f - TN] = *reinterpret_cast<const u32x4 *>(a + a_at[s] + (f - TN) * 16 * kStepBytes);
    }
    __device__ __forceinline__ void begin_load() {
        if (k_issued == 0) {
            la.plane(pairs.a >> (4 * pair) & 15u);
            lb.plane(pairs.b >> (4 * pair) & 15u);
            ++pair;
        }
    }
    __device__ __forceinline__ void end_load() {
        ++issued;
        k_issued += kStepK;
        if (k_issued >= len) k_issued = 0;
    }
    __device__ __forceinline__ void load(int l, char *a, char *b) {
        if (l < LA) la.load(l, a, w, len - k_issued);
        else lb.load(l - LA, b, w, len - k_issued);
    }
    __device__ __forceinline__ void load_all(char *a, char *b) {
        begin_load();
#pragma unroll
        for (int l = 0; l < L; ++l) load(l, a, b);
        end_load();
    }

    // G groups of products per half step, each followed by its share of the reads for the next half step and of the loads
    static constexpr int PER = 16, G = TM * TN / PER;
    __device__ __forceinline__ void multiply(Acc &acc, int buf, int g) {
#pragma unroll
        for (int x = g * PER; x < (g + 1) * PER; ++x) acc[x / TN][x % TN] = mfma16<HALF>(fa[buf][x / TN], fb[buf][x % TN], acc[x / TN][x % TN]);
    }
    __device__ __forceinline__ void scale_low(Acc &acc, int t) {
        if constexpr (HALF) {
            if (t != scale_at) return;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] *= 1.f / kLowScale;
        }
    }
    __device__ __forceinline__ void step_ahead(Acc &acc, int t, char *a, char *b, const char *next_a, const char *next_b) {
        scale_low(acc, t);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            multiply(acc, 0, g);
#pragma unroll
            for (int f = g * F / G; f < (g + 1) * F / G; ++f) read(1, a, b, 1, f);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the last fragments of this step have arrived, and the next step's operands: for all waves, so this stage may be filled again
        const bool more = t + 1 < total, fill = issued < total;
        if (more) {
            wait_loads<0>();
            lds_barrier();
        }
        if (fill) begin_load();
#pragma unroll
        for (int g = 0; g < G; ++g) {
            multiply(acc, 1, g);
            if (more) {
#pragma unroll
                for (int f = g * F / G; f < (g + 1) * F / G; ++f) read(0, next_a, next_b, 0, f);
            }
            if (fill) {
#pragma unroll
                for (int l = g * L / G; l < (g + 1) * L / G; ++l) load(l, a, b);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (fill) end_load();
    }
    __device__ __forceinline__ void run(Acc &acc, char *lds) {
        char *a0 = lds, *a1 = lds + A_BYTES, *b0 = lds + 2 * A_BYTES, *b1 = b0 + B_BYTES;      // (offsets within 16 bits of either)
        load_all(a0, b0);
        if constexpr (C::AHEAD) {
            wait_loads<0>();
            lds_barrier();
            if (issued < total) load_all(a1, b1);
#pragma unroll
            for (int f = 0; f < F; ++f) read(0, a0, b0, 0, f);
            for (int t = 0; t < total; t += 2) {
                step_ahead(acc, t, a0, b0, a1, b1);
                if (t + 1 < total) step_ahead(acc, t + 1, a1, b1, a0, b0);
            }
        } else {
            for (int t = 0; t < total; ++t) {
                scale_low(acc, t);
                // step t's operands are there, for all waves; and everybody is done with the stage that is filled next
                wait_loads<0>();
                lds_barrier();
                char *a = t & 1 ? a1 : a0, *b = t & 1 ? b1 : b0;
                if (issued < total) load_all(t & 1 ? a0 : a1, t & 1 ? b0 : b1);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
#pragma unroll
                    for (int f = 0; f < F; ++f) read(0, a, b, s, f);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[i][j] = mfma16<HALF>(fa[0][i], fb[0][j], acc[i][j]);
                }
            }
        }
    }
};

// acc[i][j]: rows m0 + 16 (wm TM + i), columns n0 + 16 (wn TN + j) of the product over k_begin <= k < k_end (k_begin a multiple of 64).
// On return all waves are done with LDS.
template <class C, bool HALF = false>
__device__ __forceinline__ void tile_product(f32x4 (&acc)[C::TM][C::TN], const Operand &A, const Operand &B, int m0, int n0, int k_begin,
                                             int k_end, const PlanePairs &pairs, char *lds) {
    const int lane = lane_id(), w = wave_id(), wm = w / C::WN, wn = w % C::WN;
    Pipeline<C, HALF> p;
    p.la.init(A, m0, k_begin, w, lane);
    p.lb.init(B, n0, k_begin, w, lane);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int r = lane & 15, c = ((4 * s + (lane >> 4)) ^ (r >> 1)) * 16;
        p.a_at[s] = (wm * C::TM * 16 + r) * kStepBytes + c;
        p.b_at[s] = (wn * C::TN * 16 + r) * kStepBytes + c;
    }
    p.pairs = pairs;
    p.w = w;
    p.len = k_end - k_begin;
    p.total = p.len > 0 ? (p.len + kStepK - 1) / kStepK * (int)pairs.n : 0;
    p.issued = p.k_issued = p.pair = 0;
    p.scale_at = pairs.n == 2 ? p.total / 2 : -1;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (p.total > 0) p.run(acc, lds);
    lds_barrier();
}

}  // namespace echo
