// Softmax cross entropy over a vocabulary without kept logits, and its gradients (include/echovocab.h has the formulas).
//
//   rows, pack   the rows with a label are gathered (whoever has none takes part in nothing); f32 rows and words are stored as bf16 planes, words piece
//                by piece; for the gradients both are turned as well, so that every product's operands have their rows along k
//   logits       z = W h^T tile by tile on the matrix cores; a tile never leaves its block:
//                  forward   maximum and sum of exponentials of its 128 or 256 words but the label, for label smoothing their sum, for every row; the
//                            label's logit
//                  backward  dz = dloss (exp(z - lse) - target) of one piece of the vocabulary, as it is and turned, in planes
//   finish       joins a row's tiles: loss and lse
//   grads        dW of the piece = dz^T h, dh += dz W, both kinds of tiles in one launch
//   dh finish    puts the sums of dh into the rows' places
//
// Bound by the matrix cores: 2 N V D forward, 8 N V D for both directions (the logits are formed twice, as the tanh map of the attention is: to keep
// them would take 4 N V bytes written and read twice), times the number of plane pairs (product.hpp, split.hpp).
// Measured (8192 rows x 100003 words x 2048, bf16): logits 2.5 ms (1340 TFLOP/s), logits and dz 3.25 (the stores of dz and of its turned form, 3.3 GB, are
// not hidden: a compute unit holds one block), dW and dh 6.1 (1100: by the power limit; pieces whose tiles fill whole rounds gained nothing),
// all else 0.4.  One of 3520 x 32000 x 1024 with f32 gradients: 0.23, 0.45, 0.88, 0.12.
// The same kernels with a teacher's words in the place of a label (TEACHER; distill.hpp) are the distillation's.
#include "../../include/echodistill.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "distill.hpp"
#include "kernels.hpp"
#include "launch.hpp"
#include "product.hpp"

namespace echo {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kDzExponent = 24;
constexpr float kDzScale = 1 << kDzExponent;          // on dz while it is in bf16 planes: small probabilities keep their digits (split.hpp)

typedef TileConfig<256, 256, 2, 4, true> BigTile;
typedef TileConfig<128, 128, 2, 2, false> MidTile;

// How a piece's tiles of dW and dh are cut along k, so that the units fill whole rounds of the chip: with few tiles, and with k axes of
// very different lengths (rows for dW, the piece's words for dh), uncut ones leave most of it idle.  Among lengths of 1 / q of either axis, the one
// with the least rounds x (length + what a unit costs besides) + what the parts cost that are written and read again.  The number of rows
// is known on the device only: k_vocab_rows works it out for all launches behind it.
struct Cut {
    int dw, dh;                      // parts of each kind
};
struct CutArgs {
    int words, D;                    // of a whole piece: the last one, which may be narrower, is cut into as many parts
    int most_dw, most_dh;            // parts there is room for, of either gradient whether it is wanted or not: each is the same beside the other and alone
    int tile, slots;                 // tile x tile; blocks that run at once
    int pairs;
    float round;                     // what a step of a round takes, against one of 256 blocks of 256 x 256
};
constexpr int kMostParts = 64;
constexpr float kUnitSteps = 8.f;                       // steps that a unit's start and end take
constexpr float kPartSteps = 1.f / 1.1e6f;              // steps (of 1.7 us) that it takes to write and read one number of a part (8 bytes at 5 TB/s)
constexpr int kCutChoices = 28;                         // q = 1 .. 8, 12, 16, 24 .. 64 of either axis
__host__ __device__ inline Cut cut_choice(const CutArgs &a, int count, int i, float &cost) {
    const int tm = (a.D + a.tile - 1) / a.tile, tw = tm * ((a.words + a.tile - 1) / a.tile), th = tm * ((count + a.tile - 1) / a.tile);
    const int kw = count > 0 ? (count + 63) / 64 : 1, kh = (a.words + 63) / 64;
    const int j = i / 2, q = j < 8 ? j + 1 : (j % 2 ? 16 : 12) << (j - 8) / 2, len = ((i % 2 ? kw : kh) + q - 1) / q;
    Cut c = {(kw + len - 1) / len, (kh + len - 1) / len};
    c.dw = c.dw < a.most_dw ? c.dw : a.most_dw;
    c.dh = c.dh < a.most_dh ? c.dh : a.most_dh;
    const int lw = (kw + c.dw - 1) / c.dw, lh = (kh + c.dh - 1) / c.dh, longest = lw > lh ? lw : lh;
    const long long units = (long long)tw * c.dw + (long long)th * c.dh;
    const float rounds = (float)((units + a.slots - 1) / a.slots);
    cost = rounds * ((float)(longest * a.pairs) + kUnitSteps) * a.round +
           ((c.dw > 1 ? (float)c.dw * a.words : 0.f) + (c.dh > 1 ? (float)(c.dh - 1) * count : 0.f)) * a.D * kPartSteps;
    return c;
}
static Cut cut_of(const CutArgs &a, int count, float &least) {
    Cut best = {1, 1};
    least = 3e38f;
    for (int i = 0; i < kCutChoices; ++i) {
        float cost;
        const Cut c = cut_choice(a, count, i, cost);
        if (cost < least) least = cost, best = c;
    }
    return best;
}

// ---- fp16 operands of the gradients of bf16 storage ------------------------------------------------------------------------
// h and W, bf16, have 8 digits, which are exact in fp16; so dz may be fp16 as well, with 11 digits to a plane where bf16 has 8.
//   bf16 gradients  are rounded by up to 2^-8 of themselves: one plane of dz, rounded by up to 2^-11 (one of bf16, by 2^-8, would double the
//                   results' variance; two of bf16 take twice the products and bytes: 8192 x 100003 x 2048 17.9 ms, this 12.1).
//   f32 gradients   two planes, together rounded by up to 2^-22: a dz has larger errors from its logit (three of bf16: 6400 x 32000 x 1024
//                   2.15 ms, this 1.59).
// fp16 ends at 2^-24 and 2^16, so the operands are scaled by powers of two: h and W so that their largest value has exponent 15, dz so that the
// largest dloss times p = 1 has 14.  What of h or W is below 2^-29 of its largest is rounded by up to 2^-40 of that instead.
// The rows of dh are scaled each for itself (dloss is multiplied with them at the end), so none suffers from another's large dloss.  What of
// dz is below 2^-29 of its row's dloss is rounded by up to 2^-40 of that, with two planes 2^-51; p - 1 itself has an error of 2^-25 in fp32.
// The rows of dW are scaled each for itself as well: a word that is unlikely in every row, or that only rows of small dloss know, has nothing but small dz
// (at p = 1e-12 everywhere one plane scaled like the others left its row of dW with an error of 26 to 87 %, at 1e-14 there was nothing left of it).
// A tile of dz is formed where nothing is known of a word's other rows, so it scales its share by 2^(16 k), k by the largest |dz| in it (dz_steps()); where
// tiles of a word took different k, k_vocab_level brings them to the least one, and the sums are scaled back by that.  Steps of 16, so that hardly any
// word has tiles that differ; the least k leaves a word's largest |dz| at 2^-4 or above, where fp16's places are 2^-20 of it.  All of it costs 0.5 to
// 2.5 % of a step (6400 x 32000 x 1024 1628 -> 1670 us, 8192 x 100003 x 2048 12.21 -> 12.30 ms, 300 x 8000 x 512 75 -> 76.5 us).
struct Largest {                     // bits of |x| as fp32, among the finite values
    unsigned h, W, dloss;            // of the rows with a label; of all words
};
// n: 2^n x has exponent 15
__device__ __forceinline__ int exponent_for(unsigned largest) { return 142 - (int)(largest >> 23); }
__device__ __forceinline__ float scaled(float x, int n) { return __builtin_amdgcn_ldexpf(x, n); }
__device__ __forceinline__ f32x4 scaled(f32x4 x, int n) { return f32x4{scaled(x[0], n), scaled(x[1], n), scaled(x[2], n), scaled(x[3], n)}; }
__device__ __forceinline__ unsigned half_pair(float a, float b) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, f16x2{(_Float16)a, (_Float16)b});
}

constexpr unsigned kNoDz = 8;         // steps of a tile in which all dz of a word are zero
__device__ __forceinline__ unsigned dz_steps(unsigned largest) {              // bits of a magnitude: 2^(16 steps) of it is 2^-4 or more
    return largest == 0u ? kNoDz : largest >= 123u << 23 ? 0u : min(7u, (138u - (largest >> 23)) / 16u);
}
// Of N values per lane the largest of 16 lanes: lane l ends with those of values N / 16 (l % 16) .. in a[0 .. N / 16 - 1].  At each step a lane keeps half of
// its values and hands the other half on (row_ror:8, row_half_mirror, two quad permutations).
template <int CTRL, int HALF, int N> __device__ __forceinline__ void row16_max_step(float (&a)[N], bool upper) {
#pragma unroll
    for (int k = 0; k < HALF; ++k) a[k] = fmaxf(upper ? a[HALF + k] : a[k], dpp_get<CTRL>(upper ? a[k] : a[HALF + k]));
}
template <int N> __device__ __forceinline__ void row16_max(float (&a)[N], int lane) {
    static_assert(N % 16 == 0, "values for every lane");
    row16_max_step<0x128, N / 2>(a, lane & 8);
    row16_max_step<0x141, N / 4>(a, lane & 4);
    row16_max_step<0x4E, N / 8>(a, lane & 2);
    row16_max_step<0xB1, N / 16>(a, lane & 1);
}

// ---- rows with a label ------------------------------------------------------------------------------------------------
// rows[p] = n of the p-th row with a label, place[n] = p or -1.  A block writes kRowsBlock labels' entries and counts all labels in
// front of them by itself.
struct Rows {
    int count;                       // rows with a label
    Cut cut;
    Largest most;
};
constexpr int kRowsBlock = 2048;
__global__ __launch_bounds__(256) void k_vocab_rows(const int *__restrict__ labels, int N, int V, int *__restrict__ rows,
                                                    int *__restrict__ place, Rows *__restrict__ out, const CutArgs cut) {
    __shared__ int s_wave[4];
    const int lane = lane_id(), w = wave_id(), begin = blockIdx.x * kRowsBlock;
    int before = 0;
    for (int i = threadIdx.x * 4; i < begin; i += 1024) {
        const int4 t = *reinterpret_cast<const int4 *>(labels + i);
        before += ((unsigned)t.x < (unsigned)V) + ((unsigned)t.y < (unsigned)V) + ((unsigned)t.z < (unsigned)V) + ((unsigned)t.w < (unsigned)V);
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) before += __shfl_xor(before, off);
    if (lane == 0) s_wave[w] = before;
    __syncthreads();
    int at = s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3];
    constexpr int U = kRowsBlock / 256;
    __shared__ int s_in[U * 4];
    int t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) t[u] = begin + u * 256 + (int)threadIdx.x < N ? labels[begin + u * 256 + threadIdx.x] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned long long m = __ballot((unsigned)t[u] < (unsigned)V);
        if (lane == 0) s_in[u * 4 + w] = __builtin_popcountll(m);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = (unsigned)t[u] < (unsigned)V;
        int p = at + __builtin_popcountll(__ballot(in) & ((1ull << lane) - 1));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k < w) p += s_in[u * 4 + k];
            at += s_in[u * 4 + k];
        }
        const int n = begin + u * 256 + threadIdx.x;
        if (in) rows[p] = n;
        if (n < N) place[n] = in ? p : -1;
    }
    if (blockIdx.x != gridDim.x - 1 || w != 0) return;
    // a lane per choice: the least cost, the first of equal ones
    float cost = 3e38f;
    Cut c = {0, 0};
    if (cut.slots && lane < kCutChoices) c = cut_choice(cut, at, lane, cost);
    float least = cost;
#pragma unroll
    for (int off = 32; off; off >>= 1) least = fminf(least, __shfl_xor(least, off));
    if (lane == __builtin_ctzll(__ballot(cost == least))) *out = Rows{at, c, Largest{0, 0, 0}};
}

// Largest values: blocks in front of h_block0 take the words, the others a row per wave of h, and dloss.  Bound by reading them once.
struct LargestArgs {
    const bf16_t *h, *W;
    const float *dloss;
    const int *labels;
    int N, V, D, h_block0;
    Rows *out;
};
__global__ __launch_bounds__(256) void k_vocab_largest(const LargestArgs a) {
    __shared__ unsigned s[2][4];
    const int lane = lane_id(), w = wave_id();
    const auto finite = [](unsigned x) { return x < 0x7f80u ? x : 0u; };
    const auto largest8 = [&](u32x4 u) {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = max(m, max(finite(u[j] & 0x7fffu), finite(u[j] >> 16 & 0x7fffu)));
        return m;
    };
    unsigned m = 0, g = 0;
    const bool words = (int)blockIdx.x < a.h_block0;
    if (words) {
        const long long n = (long long)a.V * a.D, step = (long long)a.h_block0 * 256;
        const u32x4 *W = reinterpret_cast<const u32x4 *>(a.W);
        constexpr int U = 4;
        for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n / 8; i += U * step) {
            u32x4 u[U];
#pragma unroll
            for (int k = 0; k < U; ++k) u[k] = W[min(i + k * step, n / 8 - 1)];
#pragma unroll
            for (int k = 0; k < U; ++k) m = max(m, largest8(u[k]));
        }
        if (blockIdx.x == 0 && threadIdx.x < n % 8) m = max(m, finite(a.W[n / 8 * 8 + threadIdx.x].bits & 0x7fffu));
    } else {
        for (int n = ((int)blockIdx.x - a.h_block0) * 4 + w; n < a.N; n += ((int)gridDim.x - a.h_block0) * 4) {
            if ((unsigned)a.labels[n] >= (unsigned)a.V) continue;
            const bf16_t *h = a.h + (size_t)n * a.D;
            const unsigned x = __float_as_uint(a.dloss[n]) & 0x7fffffffu;
            if (x < 0x7f800000u) g = max(g, x);
            if (a.D % 8 == 0)
                for (int d = lane * 8; d < a.D; d += 512) m = max(m, largest8(*reinterpret_cast<const u32x4 *>(h + d)));
            else
                for (int d = lane; d < a.D; d += 64) m = max(m, finite(h[d].bits & 0x7fffu));
        }
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, off));
    if (lane == 0) s[0][w] = m, s[1][w] = g;
    __syncthreads();
    if (threadIdx.x != 0) return;
    m = max(max(s[0][0], s[0][1]), max(s[0][2], s[0][3])) << 16;
    g = max(max(s[1][0], s[1][1]), max(s[1][2], s[1][3]));
    // A maximum of integers does not depend on the order.  (Only where it raises it: 2000 blocks' atomics in a row took 30 us.)
    const auto raise = [](unsigned *to, unsigned x) {
        if (x > __hip_atomic_load(to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(to, x);
    };
    if (words) {
        raise(&a.out->most.W, m);
    } else {
        raise(&a.out->most.h, m);
        raise(&a.out->most.dloss, g);
    }
}

// ---- bf16 planes ------------------------------------------------------------------------------------------------------
// Rows of src as bf16 planes, once with their columns in a row (dst, `pitch` elements a row, zeros behind D) and once turned (turned: a
// row per column, `turned_pitch` elements, zeros behind the last row up to a multiple of 8), either of them optional.  Row r is row list[r] of
// src (r < *count) or row first + r (r < n_rows).  A block takes 64 rows and 64 columns.  HALF: the turned form is fp16, scaled.
struct PackArgs {
    const void *src;
    int D, first, n_rows, pitch, turned_pitch;
    const int *list;                 // or null: consecutive rows
    const Rows *rows;
    bf16_t *dst, *turned;
    size_t plane, turned_plane;
};
template <typename T, bool HALF> __global__ __launch_bounds__(256) void k_vocab_pack(const PackArgs a) {
    constexpr int PLANES = sizeof(T) == 4 ? 3 : 1, LP = 72;                    // LDS pitch: 144 bytes, 16-byte aligned, spread over the banks
    __shared__ __align__(16) unsigned short s[64 * LP];
    const int rows = a.list ? a.rows->count : a.n_rows, r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
    if (r0 >= rows) return;
    const int tr = threadIdx.x >> 2, tc = (threadIdx.x & 3) * 16, r = r0 + tr, c = c0 + tc;
    const bool row = r < rows;
    const T *src = static_cast<const T *>(a.src) + (row ? (size_t)(a.list ? a.list[r] : a.first + r) * a.D : 0);
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = 0.f;
    if (row) {
        if (c + 16 <= a.D) {                     // loads of 16 bytes may begin at any value (2 bytes each: 1536 columns 10 us, 1534 58)
            struct __attribute__((packed, aligned(sizeof(T)))) Any { u32x4 u; };
            constexpr int PER = 16 / sizeof(T);
#pragma unroll
            for (int j = 0; j < 16; j += PER) {
                const u32x4 u = reinterpret_cast<const Any *>(src + c + j)->u;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if constexpr (PER == 4) x[j + i] = __uint_as_float(u[i]);
                    else x[j + i] = __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < a.D) x[j] = ld(src, c + j);
        }
    }
#pragma unroll
    for (int k = 0; k < PLANES; ++k) {
        unsigned u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
            x[2 * j] -= __uint_as_float(u[j] << 16);
            x[2 * j + 1] -= __uint_as_float(u[j] & 0xffff0000u);
        }
        if (a.dst && row) {
            bf16_t *to = a.dst + k * a.plane + (size_t)r * a.pitch + c;
            if (c < a.pitch) *reinterpret_cast<u32x4 *>(to) = u32x4{u[0], u[1], u[2], u[3]};
            if (c + 8 < a.pitch) *reinterpret_cast<u32x4 *>(to + 8) = u32x4{u[4], u[5], u[6], u[7]};
        }
        if (a.turned) {
            if constexpr (HALF) {
                static_assert(PLANES == 1, "bf16 values are exact in fp16");
                const int e = exponent_for(a.list ? a.rows->most.h : a.rows->most.W);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = half_pair(scaled(__uint_as_float(u[j] << 16), e), scaled(__uint_as_float(u[j] & 0xffff0000u), e));
            }
            if (k > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[(tc + 2 * j) * LP + tr] = (unsigned short)u[j];
                s[(tc + 2 * j + 1) * LP + tr] = (unsigned short)(u[j] >> 16);
            }
            __syncthreads();
            // here tr is the column and tc the first of 16 rows
            if (c0 + tr < a.pitch) {
                bf16_t *to = a.turned + k * a.turned_plane + (size_t)(c0 + tr) * a.turned_pitch + r0 + tc;
                const u32x4 *from = reinterpret_cast<const u32x4 *>(s + tr * LP + tc);
                if (r0 + tc < rows) *reinterpret_cast<u32x4 *>(to) = from[0];
                if (r0 + tc + 8 < rows) *reinterpret_cast<u32x4 *>(to + 8) = from[1];
            }
        }
    }
}

// ---- order of the tiles -------------------------------------------------------------------------------------------------
// Tile of block b of a grid of at least tm tn blocks: consecutive tiles to the same XCD (blocks are dealt to the 8 XCDs in turn), and
// among them groups of 8 rows of tiles, column by column, so that what runs at the same time shares operands in the XCD's L2.
__device__ __forceinline__ bool tile_of_block(int b, int tm, int tn, int &im, int &in) {
    const int total = tm * tn, q = total / 8, rem = total % 8, x = b % 8, k = b / 8;
    if (k >= q + (x < rem ? 1 : 0)) return false;
    const int id = x * q + min(x, rem) + k;
    constexpr int G = 8;
    const int first = id / (G * tn) * G, size = min(G, tm - first), r = id - first * tn;
    im = first + r % size;
    in = r / size;
    return true;
}

// ---- logits -----------------------------------------------------------------------------------------------------------
struct LogitsArgs {
    Operand W, h;                    // words of this piece; gathered rows
    int D;
    PlanePairs pairs;
    const Rows *count;
    const int *rows, *labels;
    int V, v0;                       // words of the vocabulary; this piece's first word
    float eps;                       // label smoothing
    Teacher teacher;                 // in the place of labels
    // forward: [tiles][pitch] maximum, sum, sum of logits; the label's logit.  Against a teacher: maximum, rest, how far its words are below the maximum
    float *part_max, *part_sum, *part_z, *z_label;
    int first_tile;
    size_t pitch;
    // backward
    const float *lse, *dloss;
    bf16_t *dz, *turned;             // [N][dz_pitch]; [words][turned_pitch]
    size_t dz_plane, turned_plane;
    int dz_pitch, turned_pitch;
    unsigned char *steps;            // [row tiles][dz_pitch]: dz_steps() of the words of `turned`, of fp16
};
// Forward, or backward by what dz is: three bf16 planes (f32 storage), two of fp16 (bf16 storage, f32 gradients), one of fp16 (bf16 gradients)
enum class Mode { kForward, kPlanes, kHalves, kHalf };
constexpr bool half_of(Mode m) { return m == Mode::kHalves || m == Mode::kHalf; }

// a sum of exponentials relative to `from`, relative to `to` >= from (both may be minus infinity: an empty sum)
__device__ __forceinline__ float scaled_sum(float sum, float from, float to) {
    return from == to ? sum : sum * fast_exp2((from - to) * kLog2e);
}

// Against a teacher, whose row may be as sure of a word as the student's, a sum of exponentials is kept without the largest one, which is 1 next to the
// maximum: `rest` and `top` stand for (1 + rest) exp(top), -1 and minus infinity for no exponentials at all.  log(1 + rest) has the digits of a small rest.
// Where the sum is 1.25 or more, 1 off it leaves rest 5 times the sum's error at most; below that the numbers are added by their fractions: of those in (0, 1] only the 1
// has none (a forward pass of 6400 x 32000 x 512 bf16, 64 entries a row, 311 us; all numbers by their fractions 322; one sum with the 1 in it 297).
__device__ __forceinline__ void join_rest(float &top, float &rest, float t, float r) {
    const bool more = t > top;
    const float high = more ? t : top, low = more ? top : t;
    rest = (more ? r : rest) + scaled_sum(1.f + (more ? rest : r), low, high);
    top = high;
}
// The rest of a row of the matrix cores' results (lanes l, l + 16, l + 32, l + 48) from each lane's sum and, where they are wanted, its sum of fractions
template <bool ASK, typename Fractions> __device__ __forceinline__ float row_rest(float top, float sum, Fractions fractions) {
    float all = sum + __shfl_xor(sum, 16);
    all += __shfl_xor(all, 32);
    float rest = all - 1.f;
    if (!ASK || __ballot(all < 1.25f)) {                   // (of a few numbers not worth the question)
        float part = fractions();
        const float ones = rintf(sum - part);              // likeliest words: the first lane that has one leaves one out
        const int lane = lane_id();
        const unsigned long long in_front = (lane < 16 ? 0ull : 0x0001000100010001ull >> (64 - 16 * (lane >> 4)) << (lane & 15));
        part += ones > 0.f && (__ballot(ones > 0.f) & in_front) == 0 ? ones - 1.f : ones;
        part += __shfl_xor(part, 16);
        part += __shfl_xor(part, 32);
        if (all < 1.25f) rest = top == -__builtin_inff() ? part - 1.f : part;
    }
    return rest;
}
// The cross entropy of a row is kept as far as it goes beyond the maximum's: the mean, by their shares, of how far its words' logits are below it.  `far` and
// `share` of a part of the words go to another maximum `to` >= from.
__device__ __forceinline__ float far_from(float far, float share, float from, float to) {
    return share != 0.f && from != to ? far + share * (to - from) : far;
}

// TEACHER: the target is a row's shares among the teacher's words (distill.hpp) instead of its label, and logits are divided by the temperature.
template <class C, Mode MODE, bool TEACHER = false>
__global__ __launch_bounds__(C::THREADS) void k_vocab_logits(const LogitsArgs a) {
    extern __shared__ __align__(16) char lds[];
    const int count = a.count->count;
    int im, in;
    if (!tile_of_block(blockIdx.x, (a.W.rows + C::BM - 1) / C::BM, (count + C::BN - 1) / C::BN, im, in)) return;
    const int m0 = im * C::BM, n0 = in * C::BN;
    const int lane = lane_id(), w = wave_id(), wm = w / C::WN, wn = w % C::WN, lr = 4 * (lane >> 4);
    // The large tile of dz has no registers for the ranges besides its product's.
    constexpr bool EARLY = MODE == Mode::kForward || C::BM < 256;
    TeacherRanges<C::TN> ranges;
    const auto look_up = [&] {
        ranges.look_up(a.teacher, a.v0 + m0 + wm * C::TM * 16, [&](int j) {
            const int n = n0 + (wn * C::TN + j) * 16 + (lane & 15);
            return n < count ? a.rows[n] : -1;
        });
    };
    if constexpr (TEACHER && EARLY) look_up();
    f32x4 acc[C::TM][C::TN];
    Operand h = a.h;
    h.rows = count;
    tile_product<C>(acc, a.W, h, m0, n0, 0, a.D, a.pairs, lds);
    if constexpr (TEACHER && !EARLY) look_up();
    const int vw = a.v0 + m0 + wm * C::TM * 16 + lr;                           // this lane's first word: it holds words vw + 16 i + r
    const bool tail = a.v0 + m0 + C::BM > a.V;
    typedef TeacherTile<C::TM * 16, C::TN> Shares;
    if constexpr (MODE == Mode::kForward) {
        float *s_max = reinterpret_cast<float *>(lds), *s_sum = s_max + C::WM * C::BN, *s_z = s_sum + C::WM * C::BN, *s_share = s_z + C::WM * C::BN;
        static_assert(4 * C::WM * C::BN * 4 + C::WAVES * Shares::BYTES <= C::LDS_BYTES, "room for the shares");
        Shares shares(a.teacher, reinterpret_cast<float *>(lds) + 4 * C::WM * C::BN, vw - lr, TEACHER, ranges);
        // the teacher's temperature is taken into the exponent, and off maxima and means
        const float log2e = TEACHER ? kLog2e * a.teacher.inv_t : kLog2e;
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            const int nt = (wn * C::TN + j) * 16 + (lane & 15), n = n0 + nt;
            const int y = !TEACHER && n < count ? a.labels[a.rows[n]] - vw : -1;
            float z = 0.f;
            if (!TEACHER && a.eps > 0.f) {
#pragma unroll
                for (int i = 0; i < C::TM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z += !tail || vw + i * 16 + r < a.V ? acc[i][j][r] : 0.f;
                z += __shfl_xor(z, 16);
                z += __shfl_xor(z, 32);
            }
            if (!TEACHER && __ballot(y >= 0 && y < C::TM * 16 && y % 16 < 4)) {   // the label's logit: the lane that holds it writes it and leaves it out of maximum and sum
#pragma unroll
                for (int i = 0; i < C::TM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (y == i * 16 + r) {
                            a.z_label[n] = acc[i][j][r];
                            acc[i][j][r] = -__builtin_inff();
                        }
            }
            if (tail) {
#pragma unroll
                for (int i = 0; i < C::TM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (vw + i * 16 + r >= a.V) acc[i][j][r] = -__builtin_inff();
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float at = top == -__builtin_inff() ? 0.f : top;             // nothing but the label and words past the end
            float sum = 0.f, share = 0.f;
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += fast_exp2((acc[i][j][r] - at) * log2e);
            if constexpr (TEACHER) {
                sum = row_rest<true>(top, sum, [&] {
                    float x = 0.f;
#pragma unroll
                    for (int i = 0; i < C::TM; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) x += __builtin_amdgcn_fractf(fast_exp2((acc[i][j][r] - at) * log2e));
                    return x;
                });
                if (shares.any(j)) {
                    shares.put(j);
                    f32x4 far = {0.f, 0.f, 0.f, 0.f}, of = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < C::TM; ++i) {
                        const f32x4 q = shares.get(j, i * 16 + lr);
#pragma unroll
                        for (int r = 0; r < 4; ++r) far[r] += q[r] != 0.f ? q[r] * (at - acc[i][j][r]) : 0.f, of[r] += q[r];
                    }
                    shares.clear(j);
                    z = a.teacher.inv_t * ((far[0] + far[1]) + (far[2] + far[3]));
                    share = (of[0] + of[1]) + (of[2] + of[3]);
                    z += __shfl_xor(z, 16);
                    z += __shfl_xor(z, 32);
                    share += __shfl_xor(share, 16);
                    share += __shfl_xor(share, 32);
                }
            } else {
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
            }
            if (lane < 16) {
                s_max[wm * C::BN + nt] = TEACHER ? top * a.teacher.inv_t : top;
                s_sum[wm * C::BN + nt] = sum;
                s_z[wm * C::BN + nt] = z;
                if constexpr (TEACHER) s_share[wm * C::BN + nt] = share;
            }
        }
        __syncthreads();
        for (int nt = threadIdx.x; nt < C::BN; nt += C::THREADS) {
            if (n0 + nt >= count) break;
            float top = s_max[nt], z = 0.f, sum = 0.f;
            if constexpr (TEACHER) {
                sum = s_sum[nt];
#pragma unroll
                for (int k = 1; k < C::WM; ++k) join_rest(top, sum, s_max[k * C::BN + nt], s_sum[k * C::BN + nt]);
#pragma unroll
                for (int k = 0; k < C::WM; ++k) z += far_from(s_z[k * C::BN + nt], s_share[k * C::BN + nt], s_max[k * C::BN + nt], top);
            } else {
#pragma unroll
                for (int k = 1; k < C::WM; ++k) top = fmaxf(top, s_max[k * C::BN + nt]);
#pragma unroll
                for (int k = 0; k < C::WM; ++k) {
                    sum += scaled_sum(s_sum[k * C::BN + nt], s_max[k * C::BN + nt], top);
                    z += s_z[k * C::BN + nt];
                }
            }
            const size_t at = (size_t)(a.first_tile + im) * a.pitch + n0 + nt;
            a.part_max[at] = top;
            a.part_sum[at] = sum;
            if (TEACHER || a.eps > 0.f) a.part_z[at] = z;
        }
    } else {
        const float off = 1.0f - a.eps, low = a.eps / (float)a.V;
        if (n0 + C::BN > count) {                                              // rows behind the last one have no logits: zero times an infinite word is NaN
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int i = 0; i < C::TM; ++i)
                    if (n0 + (wn * C::TN + j) * 16 + (lane & 15) >= count) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        Shares shares(a.teacher, reinterpret_cast<float *>(lds), vw - lr, TEACHER, ranges);
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            const int n = n0 + (wn * C::TN + j) * 16 + (lane & 15);
            const bool row = n < count;
            const int at = row ? a.rows[n] : 0;
            const int y = !TEACHER && row ? a.labels[at] - vw : -1;
            if constexpr (TEACHER) shares.put(j);
            const float lse = row ? a.lse[at] : 0.f, g = !row ? 0.f : half_of(MODE) ? 0x1p15f : a.dloss[at] * kDzScale;
#pragma unroll
            for (int i = 0; i < C::TM; ++i) {
                f32x4 q;
                if constexpr (TEACHER) {
                    q = shares.get(j, i * 16 + lr);
                    acc[i][j] *= a.teacher.inv_t;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int v = i * 16 + r;
                    // a probability: a logit of a million has an error of one half, and what that makes of it must not leave fp16
                    const float e = fast_exp2((acc[i][j][r] - lse) * kLog2e), p = (e > 1.f ? 1.f : e) - (TEACHER ? q[r] : v == y ? off + low : low);
                    float x = vw + v < a.V ? p * g : 0.f;
                    // kHalves: rounded to fp32 for both planes alike, see below.  TEACHER: computed here, between the shares' way into LDS and out of it
                    // (put off to the stores, it takes more registers than there are)
                    if constexpr (MODE == Mode::kHalves || TEACHER) asm("" : "+v"(x));
                    acc[i][j][r] = x;
                }
            }
            if constexpr (TEACHER) shares.clear(j);
        }
        if constexpr (TEACHER) lds_barrier();                                  // the shares' place is the other waves' for dz
        // dz passes through LDS a plane at a time, [row][word]: each lane writes four words of a row; whole rows leave for dz, and read
        // with the transposing load 16 words x 32 rows leave for its turned form
        constexpr int PITCH = C::BM * 2 + 16;                                  // bytes; 16 more per row spread the rows over the banks
        const int rows = min(C::BN, (count - n0 + 7) / 8 * 8);                 // zeros up to a multiple of 8
        const auto place = [&](int j, int i) { return lds + ((wn * C::TN + j) * 16 + (lane & 15)) * PITCH + (wm * C::TM * 16 + lr) * 2 + i * 32; };
        const auto store_rows = [&](bf16_t *plane) {
            bf16_t *out = plane + (size_t)n0 * a.dz_pitch + m0;
            for (int c = threadIdx.x; c < rows * (C::BM / 8); c += C::THREADS) {
                const int nt = c / (C::BM / 8), g = c % (C::BM / 8);
                if (m0 + g * 8 < a.dz_pitch)
                    *reinterpret_cast<u32x4 *>(out + (size_t)nt * a.dz_pitch + g * 8) = *reinterpret_cast<const u32x4 *>(lds + nt * PITCH + g * 16);
            }
        };
        const auto store_turned = [&](bf16_t *plane) {
            bf16_t *out = plane + (size_t)m0 * a.turned_pitch + n0;
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 *tr_ptr;
            // block (x, y): words 16 x .., rows 32 y ..; lanes 16 g .. 16 g + 15 address 4 rows x 16 words and get a word's 4 rows each
            for (int c = w; c < (C::BM / 16) * (C::BN / 32); c += C::WAVES) {
                const int x = c / (C::BN / 32), y = c % (C::BN / 32), nt = y * 32 + 8 * (lane >> 4), v = 16 * x + (lane & 15);
                const char *from = lds + (nt + ((lane & 15) >> 2)) * PITCH + (16 * x + 4 * (lane & 3)) * 2;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)from);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(from + 4 * PITCH));
                const u32x2 p = __builtin_bit_cast(u32x2, lo), q = __builtin_bit_cast(u32x2, hi);
                if (nt < rows && a.v0 + m0 + v < a.V) *reinterpret_cast<u32x4 *>(out + (size_t)v * a.turned_pitch + nt) = u32x4{p.x, p.y, q.x, q.y};
            }
        };
        if constexpr (half_of(MODE)) {
            // x, and of two planes what fp16 left of it
            const auto put = [&](char *to, f32x4 x, int k) {
                u32x2 u = {half_pair(x[0], x[1]), half_pair(x[2], x[3])};
                if (k > 0) {
                    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
                    const f16x4 top = __builtin_bit_cast(f16x4, u);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = (x[r] - (float)top[r]) * kLowScale;
                    u = u32x2{half_pair(x[0], x[1]), half_pair(x[2], x[3])};
                }
                *reinterpret_cast<u32x2 *>(to) = u;
            };
            constexpr int PLANES = MODE == Mode::kHalf ? 1 : 2;
            const auto put_all = [&](int k) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
#pragma unroll
                    for (int i = 0; i < C::TM; ++i) put(place(j, i), acc[i][j], k);
                lds_barrier();
            };
            if (a.dz)
#pragma unroll
                for (int k = 0; k < PLANES; ++k) {
                    if (k > 0) lds_barrier();
                    put_all(k);
                    store_rows(a.dz + k * a.dz_plane);
                }
            if (a.turned) {
                const int e = exponent_for(a.count->most.dloss) - 16;
#pragma unroll
                for (int j = 0; j < C::TN; ++j) {
                    const int n = n0 + (wn * C::TN + j) * 16 + (lane & 15);
                    const float g = n < count ? scaled(a.dloss[a.rows[n]], e) : 0.f;
                    // Rounded to fp32 here, for both planes: a product that goes straight to fp16, rounded once, may end at the other one of two
                    // neighbours than the one whose rest the second plane holds.
#pragma unroll
                    for (int i = 0; i < C::TM; ++i) {
                        acc[i][j] *= g;
#pragma unroll
                        for (int r = 0; r < 4; ++r) asm("" : "+v"(acc[i][j][r]));
                    }
                }
                // Each word's largest |dz| in this tile: over the wave's rows (dealt to the lanes: 30 exchanges where a reduction of each word by itself takes
                // 128), then over the waves that share its words, one of which works out the steps.
                constexpr int OWN = C::TM * 4 / 16;                            // words of a lane: from number OWN (lane % 16) of the wave's on
                float *s_top = reinterpret_cast<float *>(lds + C::BN * PITCH) + wm * C::TM * 16, *s_up = s_top + C::WN * C::BM;
                const int own = (lane & 15) * OWN, at = own / 4 * 16 + lr + own % 4;
                float top[C::TM * 4];
#pragma unroll
                for (int i = 0; i < C::TM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        top[i * 4 + r] = 0.f;
#pragma unroll
                        for (int j = 0; j < C::TN; ++j) top[i * 4 + r] = fmaxf(top[i * 4 + r], fabsf(acc[i][j][r]));
                    }
                row16_max(top, lane);
#pragma unroll
                for (int k = 0; k < OWN; ++k) s_top[wn * C::BM + at + k] = top[k];
                lds_barrier();
                if (wn == 0) {
                    unsigned char *steps = a.steps + (size_t)in * a.dz_pitch + m0 + wm * C::TM * 16 + at;
#pragma unroll
                    for (int k = 0; k < OWN; ++k) {
#pragma unroll
                        for (int x = 1; x < C::WN; ++x) top[k] = fmaxf(top[k], s_top[x * C::BM + at + k]);
                        const unsigned n = dz_steps(__float_as_uint(top[k]));
                        s_up[at + k] = n == kNoDz ? 1.f : __uint_as_float((127u + 16u * n) << 23);
                        steps[k] = (unsigned char)n;
                    }
                }
                lds_barrier();
                f32x4 up[C::TM];
                bool any = false;
#pragma unroll
                for (int i = 0; i < C::TM; ++i) {
                    up[i] = *reinterpret_cast<const f32x4 *>(s_up + i * 16 + lr);
#pragma unroll
                    for (int r = 0; r < 4; ++r) any |= up[i][r] != 1.f;
                }
                if (__ballot(any)) {
#pragma unroll
                    for (int i = 0; i < C::TM; ++i)
#pragma unroll
                        for (int j = 0; j < C::TN; ++j) acc[i][j] *= up[i];
                }
#pragma unroll
                for (int k = 0; k < PLANES; ++k) {
                    if (k > 0) lds_barrier();
                    put_all(k);
                    store_turned(a.turned + k * a.turned_plane);
                }
            }
        } else {
#pragma unroll 1
            for (int k = 0; k < 3; ++k) {
                if (k > 0) lds_barrier();
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
#pragma unroll
                    for (int i = 0; i < C::TM; ++i) {
                        f32x4 &x = acc[i][j];
                        const u32x2 u = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
                        x[0] -= __uint_as_float(u.x << 16);
                        x[1] -= __uint_as_float(u.x & 0xffff0000u);
                        x[2] -= __uint_as_float(u.y << 16);
                        x[3] -= __uint_as_float(u.y & 0xffff0000u);
                        *reinterpret_cast<u32x2 *>(place(j, i)) = u;
                    }
                lds_barrier();
                if (a.dz) store_rows(a.dz + k * a.dz_plane);
                if (a.turned) store_turned(a.turned + k * a.turned_plane);
            }
        }
    }
}

// Brings the turned dz of words whose row tiles took different steps to the least of them: the block's 64 words by a lane each, tiles by waves and
// blockIdx.y.  Where none differ, which is the rule, it reads a byte per word and tile (5 us a piece).  Nothing is rounded but what falls below fp16's
// places: two planes are taken together and apart again.  Words at 0 to -48 at random in each tile of 8192 rows (32000 x 1024): 100 us a piece, the step
// 2313 -> 2438 us with bf16 gradients, 3304 -> 3718 with f32 ones.
template <int PLANES>
__global__ __launch_bounds__(256) void k_vocab_level(const Rows *__restrict__ rows, const unsigned char *__restrict__ steps, int steps_pitch, int tile,
                                                     bf16_t *__restrict__ turned, size_t plane, int pitch, int words, unsigned char *__restrict__ level) {
    __shared__ unsigned s_least[4][64];
    const int count = rows->count, tiles = (count + tile - 1) / tile, lane = lane_id(), w = wave_id(), v0 = blockIdx.x * 64;
    const unsigned char *mine = steps + v0 + lane;
    unsigned least = kNoDz;
    for (int t0 = w; t0 < tiles; t0 += 32) {
        unsigned k[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) k[u] = mine[(size_t)min(t0 + 4 * u, tiles - 1) * steps_pitch];
#pragma unroll
        for (int u = 0; u < 8; ++u) least = min(least, k[u]);
    }
    s_least[w][lane] = least;
    __syncthreads();
    least = min(min(s_least[0][lane], s_least[1][lane]), min(s_least[2][lane], s_least[3][lane]));
    if (blockIdx.y == 0 && w == 0) level[v0 + lane] = (unsigned char)least;
    constexpr int U = 2;                                                       // words of half a wave, whose loads leave together
    for (int t = blockIdx.y * 4 + w; t < tiles; t += gridDim.y * 4) {
        const int k = mine[(size_t)t * steps_pitch], down = 16 * (k - (int)least);
        const int n0 = t * tile, n = min(tile, (count - n0 + 7) / 8 * 8), c = (lane & 31) * 8;     // a lane's eight rows: 32 lanes take a tile of up to 256
        unsigned long long off = __ballot(v0 + lane < words && k < (int)kNoDz && down > 0);
        while (off) {
            u32x4 *row[U], u[U], low[U];
            int by[U];
            bool here[U];
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int a = __builtin_ctzll(off);                            // the lower half's word, the upper half's
                const unsigned long long rest = off & (off - 1);
                const int b = rest ? __builtin_ctzll(rest) : a;
                here[x] = off != 0 && (lane < 32 || rest != 0) && c < n;
                const int l = off == 0 ? 0 : lane < 32 ? a : b;
                by[x] = off == 0 ? 0 : lane < 32 ? __builtin_amdgcn_readlane(down, a) : __builtin_amdgcn_readlane(down, b);
                row[x] = reinterpret_cast<u32x4 *>(turned + (size_t)(v0 + l) * pitch + n0 + c);
                off = rest & (rest - 1);
                if (here[x]) {
                    u[x] = *row[x];
                    if constexpr (PLANES == 2) low[x] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const bf16_t *>(row[x]) + plane);
                }
            }
#pragma unroll
            for (int x = 0; x < U; ++x) {
                if (!here[x]) continue;
                const f16x8 top = __builtin_bit_cast(f16x8, u[x]);
                f16x8 new_top, new_low;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    float y = (float)top[r];
                    if constexpr (PLANES == 2) y += (float)__builtin_bit_cast(f16x8, low[x])[r] * (1.f / kLowScale);
                    y = scaled(y, -by[x]);
                    new_top[r] = (_Float16)y;
                    if constexpr (PLANES == 2) new_low[r] = (_Float16)((y - (float)new_top[r]) * kLowScale);
                }
                *row[x] = __builtin_bit_cast(u32x4, new_top);
                if constexpr (PLANES == 2) *reinterpret_cast<u32x4 *>(reinterpret_cast<bf16_t *>(row[x]) + plane) = __builtin_bit_cast(u32x4, new_low);
            }
        }
    }
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// A decoder step scored, one token: bound by reading the words once.  Every wave takes words straight from memory as operands (f32 ones are split in
// registers) and multiplies them with all rows; no rows are gathered, no words packed, and a block's maxima, sums and label logits go to
// part [row][tile].  Up to 16 rows each wave works on its own, the rows coming to it from the caches as operands too (one of 32000 x 1024 bf16
// 13.8 us).  For more rows that would be more bytes than the caches deliver (64 f32 rows as planes: 256 MB, 36 us), so a block of eight waves passes
// 64 rows through LDS as planes (32000 x 512 f32 22.4 us); several such groups read the words together.
// Against the tiles, which pack f32 words first (us; words x D: 68832 x 696, 32000 x 1024, 8000 x 512):
//   f32   128 rows 141 / 373,  72 / 212, 23 / 57    256   242 / 408, 148 / 216, 26 / 58    512   447 / 507, 272 / 249, 45 / 60
//   bf16  128 rows  49 / 57,   30 / 38,  14 / 24    256    78 / 70,   51 / 36,  14 / 24    512   132 / 97,   92 / 45,  20 / 25
// few_pays() has what these (and 96, 192 and 384 rows) come to in rounds of 256 blocks.
// The backward pass of f32 takes the same kernel for dz, with the rows as they were gathered; only the turned words are packed then (forward and
// backward of 38 rows of 19710 x 1256 454 -> 270 us, of 64 of 32000 x 1024 440 -> 292, of 300 of 60000 x 1500 2546 -> 2196).  Where it does is decided by
// the forward's rule, which knows neither the packed rows nor the 2-byte stores of the turned dz: measured at these sizes and 556 of 2180 x 936 only.
constexpr int kFewGroup = 64, kFewAlone = 16;
template <typename T> static bool few_pays(size_t N, size_t V, size_t D) {
    // rows of whole 16-byte groups, and offsets of 31 bits among them
    if (D % (16 / sizeof(T)) != 0 || N * D * sizeof(T) >= 0x7fff0000u) return false;
    if (N <= kFewGroup) return true;
    const auto cover = [](size_t x, size_t a) { return (x + a - 1) / a; };
    const float few = 6.f + (float)cover(cover(V, 128) * cover(N, kFewGroup), 256) * (sizeof(T) == 4 ? 5.f + 0.03f * D : 3.f + 0.007f * D);
    const float mid = (float)cover(cover(V, 128) * cover(N, 128), 512) * 1.1f, big = (float)cover(cover(V, 256) * cover(N, 256), 256) * 1.7f;
    const float steps = (float)cover(D, 64) * (sizeof(T) == 4 ? 6.f : 1.f), pack = sizeof(T) == 4 ? (float)V * D * 2e-6f : 0.f;
    return few < 15.f + pack + steps * std::min(mid, big);
}
constexpr int few_words(int rows) { return rows <= kFewAlone ? 64 : 128; }     // per block of four or eight waves of 16 words

struct FewArgs {
    const void *h, *W;
    const int *labels;
    int N, V, D, tiles, groups;      // groups of 64 rows
    float eps;
    float *part_max, *part_sum, *part_z, *z_label;
    // backward (f32): V words from v0 of all_words, rows as gathered, dz and its turned form as three planes
    int v0, all_words;
    const Rows *count;
    const int *rows;
    const float *lse, *dloss;
    bf16_t *dz, *turned;
    size_t dz_plane, turned_plane;
    int dz_pitch, turned_pitch;
    Teacher teacher;
};

// 16 rows x 32 k of a matrix as an operand: as loaded (lane l: row l % 16, k = 8 (l / 16) .. + 7), and as planes
template <typename T> struct FewFragment {
    static constexpr int LOADS = (int)sizeof(T) / 2, PLANES = sizeof(T) == 4 ? 3 : 1;
    u32x4 raw[LOADS];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rsrc, unsigned row_off, int k, int D) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = k + 4 * i;
            raw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at < D ? row_off + at * (unsigned)sizeof(T) : kOutside, 0, 0));
        }
    }
    __device__ __forceinline__ void planes(u32x4 (&p)[PLANES]) const {
        if constexpr (PLANES == 1) {
            p[0] = raw[0];
        } else {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(raw[j / 4][j % 4]);
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned u = bf16_pair(x[2 * j], x[2 * j + 1]);
                    x[2 * j] -= __uint_as_float(u << 16);
                    x[2 * j + 1] -= __uint_as_float(u & 0xffff0000u);
                    p[i][j] = u;
                }
        }
    }
};
// A product of f32 rows is six of planes, five of them small.  APART: those have a sum of their own, which join() adds at the end: to the large one, every 32 k, they
// are six roundings at its size instead of one (lse of 16 rows of D = 2048 off by 4.4e-7 of itself instead of 8e-8, 64 of 1024 by 2.8e-7 instead of 9e-8; a
// plain fp32 product 8e-8, 9e-8; 0 to 0.5 % of the time).  Labels have one sum, so that their results stay as they were.
template <int PLANES, bool APART> struct FewSum {
    f32x4 large = {0.f, 0.f, 0.f, 0.f}, small = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void multiply(const u32x4 (&a)[PLANES], const u32x4 (&b)[PLANES]) {
        f32x4 &c = APART ? small : large;
        if constexpr (PLANES == 3) {                                           // the small terms first
            c = mfma16(a[1], b[1], c);
            c = mfma16(a[2], b[0], c);
            c = mfma16(a[0], b[2], c);
            c = mfma16(a[1], b[0], c);
            c = mfma16(a[0], b[1], c);
        }
        large = mfma16(a[0], b[0], large);
    }
    __device__ __forceinline__ f32x4 join() const {
        if constexpr (APART && PLANES == 3) return large + small;
        else return large;
    }
};

// The logits of 16 NT rows and a wave's 16 words, joined over the block: s_*: WAVES x 16 NT floats
template <int NT, int WAVES, bool TEACHER>
__device__ __forceinline__ void few_join(const FewArgs &a, f32x4 (&acc)[NT], int tile, int v0, float *s_max, float *s_sum, float *s_z, float *s_share,
                                         float *s_shares) {
    constexpr int ROWS = 16 * NT;
    const int lane = lane_id(), w = wave_id(), vw = v0 + 4 * (lane >> 4);       // this lane holds words vw + r
    TeacherRanges<NT> ranges;
    if constexpr (TEACHER) ranges.look_up(a.teacher, v0, [&](int j) { return 16 * j + (lane & 15) < a.N ? 16 * j + (lane & 15) : -1; });
    TeacherTile<16, NT> shares(a.teacher, s_shares, v0, TEACHER, ranges);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = 16 * j + (lane & 15), y = !TEACHER && n < a.N ? a.labels[n] - vw : -1;
        f32x4 q = {0.f, 0.f, 0.f, 0.f};
        if constexpr (TEACHER) {
            acc[j] *= a.teacher.inv_t;
            shares.put(j);
            q = shares.get(j, vw - v0);
            shares.clear(j);
        }
        float z = 0.f, top = -__builtin_inff(), sum = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (vw + r >= a.V) {
                acc[j][r] = -__builtin_inff();
            } else {
                z += acc[j][r];
                if (y == r) {                                                  // the label's logit is left out of maximum and sum
                    a.z_label[n] = acc[j][r];
                    acc[j][r] = -__builtin_inff();
                }
            }
            top = fmaxf(top, acc[j][r]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float at = top == -__builtin_inff() ? 0.f : top;
        float share = 0.f;
        if constexpr (TEACHER) {
            z = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) z += q[r] != 0.f ? q[r] * (at - acc[j][r]) : 0.f, share += q[r];
            share += __shfl_xor(share, 16);
            share += __shfl_xor(share, 32);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += fast_exp2((acc[j][r] - at) * kLog2e);
        if constexpr (TEACHER) {
            sum = row_rest<false>(top, sum, [&] {
                float x = 0.f;
#pragma unroll
                for (int r = 0; r < 4; ++r) x += __builtin_amdgcn_fractf(fast_exp2((acc[j][r] - at) * kLog2e));
                return x;
            });
        } else {
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
        }
        z += __shfl_xor(z, 16);
        z += __shfl_xor(z, 32);
        if (lane < 16) {
            s_max[w * ROWS + n] = top, s_sum[w * ROWS + n] = sum, s_z[w * ROWS + n] = z;
            if constexpr (TEACHER) s_share[w * ROWS + n] = share;
        }
    }
    __syncthreads();
    const int n = threadIdx.x;
    if (n >= a.N) return;
    float top = s_max[n], sum = 0.f, z = 0.f;
    if constexpr (TEACHER) {
        sum = s_sum[n];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) join_rest(top, sum, s_max[k * ROWS + n], s_sum[k * ROWS + n]);
#pragma unroll
        for (int k = 0; k < WAVES; ++k) z += far_from(s_z[k * ROWS + n], s_share[k * ROWS + n], s_max[k * ROWS + n], top);
    } else {
#pragma unroll
        for (int k = 1; k < WAVES; ++k) top = fmaxf(top, s_max[k * ROWS + n]);
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            sum += scaled_sum(s_sum[k * ROWS + n], s_max[k * ROWS + n], top);
            z += s_z[k * ROWS + n];
        }
    }
    const size_t at = (size_t)n * a.tiles + tile;
    a.part_max[at] = top;
    a.part_sum[at] = sum;
    a.part_z[at] = z;
}

// dz of the same: few enough to be stored as the lanes hold it.  Rows n0 .. n0 + a.N, and zeros up to a multiple of 8 and for words past the end
template <int NT, bool TEACHER> __device__ __forceinline__ void few_dz(const FewArgs &a, f32x4 (&acc)[NT], int n0, int v0, float *s_shares) {
    const int lane = lane_id(), vw = v0 + 4 * (lane >> 4);
    TeacherRanges<NT> ranges;
    if constexpr (TEACHER) ranges.look_up(a.teacher, a.v0 + v0, [&](int j) { return 16 * j + (lane & 15) < a.N ? a.rows[16 * j + (lane & 15)] : -1; });
    TeacherTile<16, NT> shares(a.teacher, s_shares, a.v0 + v0, TEACHER, ranges);
    const float low = a.eps / (float)a.all_words, off = 1.0f - a.eps;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = 16 * j + (lane & 15);
        f32x4 q = {0.f, 0.f, 0.f, 0.f};
        if constexpr (TEACHER) {
            acc[j] *= a.teacher.inv_t;
            shares.put(j);
            q = shares.get(j, vw - v0);
            shares.clear(j);
        }
        if (n >= (a.N + 7) / 8 * 8) continue;
        const bool row = n < a.N;
        const int at = a.rows[min(n, a.N - 1)], y = TEACHER ? -1 : a.labels[at] - a.v0 - vw;
        const float lse = a.lse[at], g = a.dloss[at] * kDzScale;
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float e = fast_exp2((acc[j][r] - lse) * kLog2e), p = (e > 1.f ? 1.f : e) - (TEACHER ? q[r] : r == y ? off + low : low);
            x[r] = row && vw + r < a.V ? p * g : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const u32x2 u = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
            x[0] -= __uint_as_float(u.x << 16);
            x[1] -= __uint_as_float(u.x & 0xffff0000u);
            x[2] -= __uint_as_float(u.y << 16);
            x[3] -= __uint_as_float(u.y & 0xffff0000u);
            if (a.dz && row) *reinterpret_cast<u32x2 *>(a.dz + k * a.dz_plane + (size_t)(n0 + n) * a.dz_pitch + vw) = u;
            if (a.turned) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (vw + r < a.V)
                        a.turned[k * a.turned_plane + (size_t)(vw + r) * a.turned_pitch + n0 + n].bits = (unsigned short)(u[r / 2] >> (16 * (r & 1)));
            }
        }
    }
}

// AHEAD: how many times 32 k are on their way.
template <typename T, int AHEAD, bool TEACHER>
__global__ __launch_bounds__(256, 2) void k_vocab_few_alone(const FewArgs a) {
    constexpr int PLANES = FewFragment<T>::PLANES;
    __shared__ float s_max[64], s_sum[64], s_z[64], s_share[TEACHER ? 64 : 1];
    const int lane = lane_id(), v0 = (blockIdx.x * 4 + wave_id()) * 16, steps = (a.D + 31) / 32, k_lane = 8 * (lane >> 4);
    const int first = min(v0, a.V - 1);
    const __amdgpu_buffer_rsrc_t words = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(static_cast<const T *>(a.W) + (size_t)first * a.D), 0, 0x7ffffff0, 0x00020000);
    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.h), 0, 0x7ffffff0, 0x00020000);
    const unsigned word_off = (unsigned)(min(lane & 15, a.V - 1 - first) * a.D) * sizeof(T);
    const unsigned row_off = (unsigned)(min(lane & 15, a.N - 1) * a.D) * sizeof(T);
    FewFragment<T> fw[AHEAD], fh[AHEAD];
    auto fetch = [&](int d, int t) __attribute__((always_inline)) {
        fw[d].load(words, word_off, 32 * t + k_lane, a.D);
        fh[d].load(rows, row_off, 32 * t + k_lane, a.D);
        loads_stay();
    };
    FewSum<PLANES, TEACHER> sum;
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (d < steps) fetch(d, d);
    for (int t0 = 0; t0 < steps; t0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            if (t0 + d >= steps) break;
            u32x4 pw[PLANES], ph[PLANES];
            fw[d].planes(pw);
            fh[d].planes(ph);
            if (t0 + d + AHEAD < steps) fetch(d, t0 + d + AHEAD);
            sum.multiply(pw, ph);
        }
    f32x4 acc[1] = {sum.join()};
    __shared__ __align__(16) float s_shares[TEACHER ? 4 * TeacherTile<16, 1>::BYTES / 4 : 1];
    few_join<1, 4, TEACHER>(a, acc, blockIdx.x, v0, s_max, s_sum, s_z, s_share, s_shares);
}

// 128 k at a time: the words' next 256 and the rows' next 128 are on their way; the rows stand in LDS twice.
// A row takes 256 bytes of LDS, its groups of 16 bytes in the order c ^ (row % 16): the 16 rows of a fragment take all banks, whichever of its lanes are
// served together (16 more bytes a row instead: 41 % of the LDS time went to conflicts).
constexpr int kFewK = 128, kFewPitch = kFewK * 2;
template <typename T, int NT, bool BWD, bool TEACHER>
__global__ __launch_bounds__(512) void k_vocab_few_shared(const FewArgs all) {
    constexpr int PLANES = FewFragment<T>::PLANES, SUB = kFewK / 32, ROWS = 16 * NT, WAVES = 8;
    constexpr int GROUPS = ROWS * kFewK / 8, ITEMS = (GROUPS + 64 * WAVES - 1) / (64 * WAVES);      // groups of 8 numbers of the rows, per thread
    constexpr int STAGE = PLANES * ROWS * kFewPitch;
    __shared__ __align__(16) char s_h[2 * STAGE];
    __shared__ float s_max[WAVES * ROWS], s_sum[WAVES * ROWS], s_z[WAVES * ROWS], s_share[TEACHER ? WAVES * ROWS : 1];
    // the groups' blocks of a tile side by side: its words are read from memory once
    const int tile = blockIdx.x / all.groups, n0 = (blockIdx.x - tile * all.groups) * kFewGroup;
    FewArgs a = all;
    if constexpr (BWD) {
        a.N = min(ROWS, all.count->count - n0);
        if (a.N <= 0) return;
        a.rows += n0;
    } else {
        a.N = min(ROWS, all.N - n0);
        a.h = static_cast<const T *>(all.h) + (size_t)n0 * all.D;
        if constexpr (TEACHER) {
            a.teacher.from_row(n0);
        } else {
            a.labels += n0;
            a.z_label += n0;
        }
        a.part_max += (size_t)n0 * all.tiles;
        a.part_sum += (size_t)n0 * all.tiles;
        a.part_z += (size_t)n0 * all.tiles;
    }
    const int lane = lane_id(), v0 = (tile * WAVES + wave_id()) * 16, steps = (a.D + kFewK - 1) / kFewK, k_lane = 8 * (lane >> 4);
    const int first = min(v0, a.V - 1);
    const __amdgpu_buffer_rsrc_t words = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(static_cast<const T *>(a.W) + (size_t)first * a.D), 0, 0x7ffffff0, 0x00020000);
    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.h), 0, 0x7ffffff0, 0x00020000);
    const unsigned word_off = (unsigned)(min(lane & 15, a.V - 1 - first) * a.D) * sizeof(T);
    FewFragment<T> fw[2][SUB], fh[ITEMS];
    auto fetch_words = [&](int buf, int t) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) fw[buf][s].load(words, word_off, t * kFewK + 32 * s + k_lane, a.D);
    };
    unsigned row_off[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int n = min((i * 64 * WAVES + (int)threadIdx.x) / (kFewK / 8), a.N - 1);
        row_off[i] = (unsigned)((BWD ? a.rows[n] : n) * a.D) * sizeof(T);
    }
    auto fetch_rows = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) fh[i].load(rows, row_off[i], t * kFewK + (i * 64 * WAVES + (int)threadIdx.x) % (kFewK / 8) * 8, a.D);
    };
    auto put_rows = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int g = i * 64 * WAVES + threadIdx.x;
            u32x4 p[PLANES];
            fh[i].planes(p);
            if (GROUPS % (64 * WAVES) == 0 || g < GROUPS) {
#pragma unroll
                for (int k = 0; k < PLANES; ++k)
                    *reinterpret_cast<u32x4 *>(s_h + (t & 1) * STAGE + (k * ROWS + g / (kFewK / 8)) * kFewPitch + (g % (kFewK / 8) ^ g / (kFewK / 8) % 16) * 16) = p[k];
            }
        }
    };
    FewSum<PLANES, TEACHER> sum[NT];
    fetch_rows(0);
    fetch_words(0, 0);
    fetch_words(1, 1);
    loads_stay();
    put_rows(0);
    lds_barrier();
    auto step = [&](int t, FewFragment<T> (&f)[SUB]) __attribute__((always_inline)) {
        u32x4 pw[SUB][PLANES];
        if (t + 1 < steps) fetch_rows(t + 1);                                  // in front of the words behind it: loads arrive in order
        loads_stay();
#pragma unroll
        for (int s = 0; s < SUB; ++s) f[s].planes(pw[s]);
        if (t + 2 < steps) {
#pragma unroll
            for (int s = 0; s < SUB; ++s) f[s].load(words, word_off, (t + 2) * kFewK + 32 * s + k_lane, a.D);
        }
        loads_stay();
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const char *from = s_h + (t & 1) * STAGE + (lane & 15) * kFewPitch + ((4 * s + (lane >> 4)) ^ (lane & 15)) * 16;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                u32x4 ph[PLANES];
#pragma unroll
                for (int k = 0; k < PLANES; ++k) ph[k] = *reinterpret_cast<const u32x4 *>(from + (k * ROWS + 16 * j) * kFewPitch);
                sum[j].multiply(pw[s], ph);
            }
        }
        if (t + 1 < steps) put_rows(t + 1);
        lds_barrier();
    };
    for (int t = 0; t < steps; t += 2) {
        step(t, fw[0]);
        if (t + 1 < steps) step(t + 1, fw[1]);
    }
    f32x4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = sum[j].join();
    static_assert(WAVES * TeacherTile<16, NT>::BYTES <= sizeof(s_h), "room for the shares");      // (behind the last barrier nobody reads the rows)
    float *s_shares = reinterpret_cast<float *>(s_h);
    if constexpr (BWD) few_dz<NT, TEACHER>(a, acc, n0, v0, s_shares);
    else few_join<NT, WAVES, TEACHER>(a, acc, tile, v0, s_max, s_sum, s_z, s_share, s_shares);
}

// loss and lse of a row from its maximum, sum and sum of logits without and with the label:
// -log p of the label: log(1 + sum over the other words of exp(z - z_label)), which keeps the digits of a sure label's loss.  lse from whichever of the label's
// logit and the maximum is larger: the digits of a label far below (from -infinity, a word that is shut out) are not in it.
__device__ __forceinline__ void loss_of_row(float top, float sum, float z, float zl, int V, float eps, float &loss, float &lse) {
    const float t = top - zl;
    const float rest = t > 0.f ? logf(sum + expf(-t)) : log1pf(sum * expf(t));
    lse = (t > 0.f ? top : zl) + rest;
    loss = t > 0.f ? t + rest : rest;
    if (zl == __builtin_inff()) loss = __builtin_nanf("");
    if (eps > 0.f) loss += eps * (zl - z / (float)V);
}

// The same against a teacher: from its maximum, the rest of its exponentials and how far its words are below the maximum; `own` is the sum of share log share.  Each
// of the terms is small where student and teacher are sure of the same word.  The temperature's square by itself may leave fp32's range.
__device__ __forceinline__ void loss_of_row(float top, float rest, float far, const Teacher &t, int n, float &loss, float &lse) {
    const float log_sum = log1pf(rest);
    lse = top + log_sum;
    loss = t.temperature * (t.temperature * (t.own[n] + (far + log_sum)));
}
// How far a row's entries of a part of its list are below their tiles' largest maximum, `top`
struct EntriesFar {
    float top = -__builtin_inff(), share = 0.f, far = 0.f;
    __device__ __forceinline__ void add(float q, float tile_top) {
        const float to = fmaxf(top, tile_top);
        far = far_from(far, share, top, to);
        if (q != 0.f && tile_top != to) far += q * (to - tile_top);
        share += q;
        top = to;
    }
};

// A block per row.
template <bool TEACHER>
__global__ __launch_bounds__(256) void k_vocab_few_finish(const FewArgs a, float *__restrict__ loss, float *__restrict__ lse) {
    __shared__ float s_max[4], s_sum[4], s_z[4];
    const int n = blockIdx.x, lane = lane_id(), w = wave_id(), y = a.labels[n];
    if ((unsigned)y >= (unsigned)a.V) {
        if (threadIdx.x == 0) loss[n] = 0.f, lse[n] = 0.f;
        return;
    }
    float top = -__builtin_inff(), sum = TEACHER ? -1.f : 0.f, z = 0.f;
    EntriesFar entries;
    if (TEACHER && w == 0) {
        const int count = a.teacher.start[(size_t)n * a.teacher.marks + a.teacher.marks - 1];
        for (int k = lane; k < count; k += 64) {
            const size_t at = (size_t)n * a.teacher.K + k;
            entries.add(a.teacher.shares[at], a.part_max[(size_t)n * a.tiles + a.teacher.words[at] / few_words(a.N)]);
        }
    }
    for (int t0 = threadIdx.x; t0 < a.tiles; t0 += 1024) {
        float m[4], s[4], zz[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const size_t at = (size_t)n * a.tiles + min(t0 + 256 * u, a.tiles - 1);
            m[u] = a.part_max[at], s[u] = a.part_sum[at], zz[u] = a.part_z[at];
        }
        if constexpr (TEACHER) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (t0 + 256 * u < a.tiles) join_rest(top, sum, m[u], s[u]), z += zz[u];
        } else {
            float next = top;
#pragma unroll
            for (int u = 0; u < 4; ++u) next = fmaxf(next, m[u]);
            sum = scaled_sum(sum, top, next);
            top = next;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (t0 + 256 * u < a.tiles) sum += scaled_sum(s[u], m[u], top), z += zz[u];
        }
    }
    const float wave_top = wave_max(top);
    if constexpr (TEACHER) {
        // (of all lanes, whose exponentials are none, ones or more, one keeps its likeliest out)
        const bool out = lane == __builtin_ctzll(__ballot(top == wave_top));
        sum = wave_sum(out ? sum : scaled_sum(1.f + sum, top, wave_top));
        if (w == 0) {
            const float to = wave_max(entries.top);
            z += far_from(entries.far, entries.share, entries.top, to);
            entries.share = wave_sum(entries.share), entries.top = to;
        }
    } else {
        sum = wave_sum(scaled_sum(sum, top, wave_top));
    }
    z = wave_sum(z);
    if (lane == 0) s_max[w] = wave_top, s_sum[w] = sum, s_z[w] = z;
    __syncthreads();
    if (threadIdx.x != 0) return;
    if constexpr (TEACHER) {
        top = wave_top;
#pragma unroll
        for (int k = 1; k < 4; ++k) join_rest(top, sum, s_max[k], s_sum[k]), z += s_z[k];
        loss_of_row(top, sum, far_from(z, entries.share, entries.top, top), a.teacher, n, loss[n], lse[n]);
    } else {
        top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
        sum = 0.f, z = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += scaled_sum(s_sum[k], s_max[k], top), z += s_z[k];
        loss_of_row(top, sum, z, a.z_label[n], a.V, a.eps, loss[n], lse[n]);
    }
}

// Joins the tiles of 64 rows, of 2^tile_bits words each: four waves take a quarter of the tiles each, lanes are rows.  Rows without a label get zeros.
template <bool TEACHER>
__global__ __launch_bounds__(256) void k_vocab_loss_finish(const float *__restrict__ part_max, const float *__restrict__ part_sum,
                                                           const float *__restrict__ part_z, const float *__restrict__ z_label,
                                                           const int *__restrict__ place, int N, int V, int tiles, size_t pitch,
                                                           float eps, const Teacher teacher, int tile_bits, float *__restrict__ loss,
                                                           float *__restrict__ lse) {
    __shared__ float s_max[4][64], s_sum[4][64], s_z[4][64], s_top[4][TEACHER ? 64 : 1], s_share[4][TEACHER ? 64 : 1];
    const int lane = lane_id(), w = wave_id(), n = blockIdx.x * 64 + lane, p = n < N ? place[n] : -1;
    const int share = (tiles + 3) / 4, t0 = w * share, t1 = min(tiles, t0 + share);
    float top = -__builtin_inff(), sum = TEACHER ? -1.f : 0.f, z = 0.f;
    EntriesFar entries;
    if (TEACHER && p >= 0) {                               // the waves share a row's entries too (what stands behind the last one is nothing)
        constexpr int U = 8;
        const int count = teacher.start[(size_t)n * teacher.marks + teacher.marks - 1];
        for (int k0 = w; k0 < teacher.K; k0 += 4 * U) {
            float q[U], m[U];
            int word[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t at = (size_t)n * teacher.K + min(k0 + 4 * u, teacher.K - 1);
                word[u] = teacher.words[at];
                q[u] = teacher.shares[at];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) m[u] = part_max[(size_t)(k0 + 4 * u < count ? word[u] >> tile_bits : 0) * pitch + p];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k0 + 4 * u < count) entries.add(q[u], m[u]);
        }
    }
    if (p >= 0) {
        for (int t = t0; t < t1; t += 8) {
            float m[8], s[8], zz[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const size_t at = (size_t)min(t + u, t1 - 1) * pitch + p;
                m[u] = part_max[at];
                s[u] = part_sum[at];
                zz[u] = TEACHER || eps > 0.f ? part_z[at] : 0.f;
            }
            if constexpr (TEACHER) {
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (t + u >= t1) m[u] = -__builtin_inff(), s[u] = -1.f, zz[u] = 0.f;
#pragma unroll
                for (int d = 1; d < 8; d *= 2)
#pragma unroll
                    for (int u = 0; u < 8; u += 2 * d) join_rest(m[u], s[u], m[u + d], s[u + d]), zz[u] += zz[u + d];
                join_rest(top, sum, m[0], s[0]);
                z += zz[0];
            } else {
                float next = top;
#pragma unroll
                for (int u = 0; u < 8; ++u) next = fmaxf(next, m[u]);
                sum = scaled_sum(sum, top, next);
                top = next;
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (t + u < t1) {
                        sum += scaled_sum(s[u], m[u], top);
                        z += zz[u];
                    }
            }
        }
    }
    if constexpr (TEACHER) {
        s_top[w][lane] = entries.top;
        s_share[w][lane] = entries.share;
        z += entries.far;
    }
    s_max[w][lane] = top;
    s_sum[w][lane] = sum;
    s_z[w][lane] = z;
    __syncthreads();
    if (w != 0 || n >= N) return;
    float l = 0.f, e = 0.f;
    if (p >= 0) {
        if constexpr (TEACHER) {
#pragma unroll
            for (int k = 1; k < 4; ++k) join_rest(top, sum, s_max[k][lane], s_sum[k][lane]);
            z = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) z += far_from(s_z[k][lane], s_share[k][lane], s_top[k][lane], top);
            loss_of_row(top, sum, z, teacher, n, l, e);
        } else {
            float all = fmaxf(fmaxf(s_max[0][lane], s_max[1][lane]), fmaxf(s_max[2][lane], s_max[3][lane]));
            sum = 0.f;
            z = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum += scaled_sum(s_sum[k][lane], s_max[k][lane], all);
                z += s_z[k][lane];
            }
            loss_of_row(all, sum, z, z_label[p], V, eps, l, e);
        }
    }
    loss[n] = l;
    lse[n] = e;
}

// ---- gradients ----------------------------------------------------------------------------------------------------------
struct GradsArgs {
    Operand dz, dz_turned;           // rows of dz; words of dz
    Operand h_turned, W_turned;      // columns of h; of this piece's words
    const Rows *rows;
    int words, D;                    // of this piece
    PlanePairs pairs;
    void *dW;                        // this piece's first row
    const unsigned char *level;      // fp16: steps of 16 by which the words' rows of dz_turned were scaled up
    float *dw_sum, *dh_sum;          // [parts][words][D]; [parts][N][D], in the rows' gathered places
    size_t dw_part, dh_part;
    bool add;                        // not the first piece
};
// powers of two that the sums carry
__device__ __forceinline__ int dw_exponent(const Rows &r, bool half) {
    return half ? exponent_for(r.most.dloss) - 1 + exponent_for(r.most.h) : kDzExponent;
}
__device__ __forceinline__ int dh_exponent(const Rows &r, bool half) { return half ? 15 + exponent_for(r.most.W) : kDzExponent; }

// Four consecutive columns of a row, of which `left` exist.  Wide loads and stores may begin at any value.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ f32x4 get4(const float *from, int left) {
    if (left >= 4) return *reinterpret_cast<const f32x4_any *>(from);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 3; ++r)
        if (r < left) x[r] = from[r];
    return x;
}
__device__ __forceinline__ void put4(float *to, f32x4 x, int left) {
    if (left >= 4) {
        __builtin_nontemporal_store(x, reinterpret_cast<f32x4_any *>(to));
    } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < left) to[r] = x[r];
    }
}
__device__ __forceinline__ void put4(bf16_t *to, f32x4 x, int left) {
    const u32x2 u = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    if (left >= 4) {
        __builtin_nontemporal_store(u, reinterpret_cast<u32x2_any *>(to));
    } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < left) to[r].bits = (unsigned short)(u[r / 2] >> (16 * (r & 1)));
    }
}

// Units of dW (columns of h x words, over rows) and, behind them, of dh (columns of W x rows, over the piece's words): a lane holds
// four consecutive columns of a result row.
template <class C, Mode MODE>
__global__ __launch_bounds__(C::THREADS) void k_vocab_grads(const GradsArgs a) {
    extern __shared__ __align__(16) char lds[];
    const int count = a.rows->count, words = a.words, D = a.D, tm = (D + C::BM - 1) / C::BM;
    Cut cut = a.rows->cut;
    if (!a.dW) cut.dw = 0;
    if (!a.dh_sum) cut.dh = 0;
    const int tw = (words + C::BN - 1) / C::BN, th = (count + C::BN - 1) / C::BN;
    const int lane = lane_id(), w = wave_id(), wm = w / C::WN, wn = w % C::WN;
    const int dw_blocks = (tm * tw * cut.dw + 7) / 8 * 8;
    f32x4 acc[C::TM][C::TN];
    int im, in;
    if ((int)blockIdx.x < dw_blocks) {
        if (!tile_of_block(blockIdx.x, tm, tw * cut.dw, im, in)) return;
        const int part = in / tw, m0 = im * C::BM, n0 = (in - part * tw) * C::BN;
        const int len = ((count + kStepK - 1) / kStepK + cut.dw - 1) / cut.dw * kStepK, k0 = min(count, part * len);
        tile_product<C, half_of(MODE)>(acc, a.h_turned, a.dz_turned, m0, n0, k0, min(count, k0 + len), a.pairs, lds);
        const int d0 = m0 + wm * C::TM * 16 + 4 * (lane >> 4), e = dw_exponent(*a.rows, half_of(MODE));
        typedef std::conditional_t<MODE == Mode::kHalf, bf16_t, float> grad_t;
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
            const int v = n0 + (wn * C::TN + j) * 16 + (lane & 15);
            if (v >= words) continue;
            const size_t at = (size_t)v * D + d0;
            const int back = -(half_of(MODE) ? e + 16 * a.level[v] : e);
#pragma unroll
            for (int i = 0; i < C::TM; ++i) {
                if (cut.dw > 1) put4(a.dw_sum + part * a.dw_part + at + 16 * i, acc[i][j], D - d0 - 16 * i);
                else put4(static_cast<grad_t *>(a.dW) + at + 16 * i, scaled(acc[i][j], back), D - d0 - 16 * i);
            }
        }
        return;
    }
    if (!tile_of_block(blockIdx.x - dw_blocks, tm, th * cut.dh, im, in)) return;
    const int part = in / th, m0 = im * C::BM, n0 = (in - part * th) * C::BN;
    const int len = ((words + kStepK - 1) / kStepK + cut.dh - 1) / cut.dh * kStepK, k0 = min(words, part * len);
    Operand dz = a.dz;
    dz.rows = count;
    tile_product<C, half_of(MODE)>(acc, a.W_turned, dz, m0, n0, k0, min(words, k0 + len), a.pairs, lds);
    float *sums = a.dh_sum + part * a.dh_part;
    const int d0 = m0 + wm * C::TM * 16 + 4 * (lane >> 4);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
        const int n = n0 + (wn * C::TN + j) * 16 + (lane & 15);
        if (n >= count) continue;
        float *to = sums + (size_t)n * D + d0;
        const int left = D - d0;
        f32x4 old[C::TM];
#pragma unroll
        for (int i = 0; i < C::TM; ++i) old[i] = a.add ? get4(to + 16 * i, left - 16 * i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            const f32x4 x = old[i] + acc[i][j];
            if (left - 16 * i >= 4) {
                *reinterpret_cast<f32x4_any *>(to + 16 * i) = x;               // read again soon
            } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                    if (r < left - 16 * i) to[16 * i + r] = x[r];
            }
        }
    }
}

// Parts of dW added in order and scaled back, where there are any.  level: of fp16, otherwise null
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_dw_finish(const Rows *__restrict__ rows, const unsigned char *__restrict__ level, const float *__restrict__ sums,
                                                         size_t part, int words, int D, T *__restrict__ dW) {
    const int parts = rows->cut.dw, v = blockIdx.x * 4 + wave_id();
    if (parts < 2 || v >= words) return;
    const int e = dw_exponent(*rows, level != nullptr) + (level ? 16 * level[v] : 0);
    for (int d = lane_id() * 4; d < D; d += 256) {
        const size_t at = (size_t)v * D + d;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = 0; k < parts; ++k) x += get4(sums + k * part + at, D - d);
        put4(dW + at, scaled(x, -e), D - d);
    }
}

// dh[n] = sum of the parts of row place[n], scaled back; zeros for rows without a label.  A wave per 256 columns of a row.  half: dloss is not in the sums yet.
template <typename T>
__global__ __launch_bounds__(256) void k_vocab_dh_finish(const Rows *__restrict__ rows, bool half, const float *__restrict__ sums, size_t part,
                                                         const int *__restrict__ place, const float *__restrict__ dloss, int N, int D,
                                                         T *__restrict__ dh) {
    const int n = blockIdx.x * 4 + wave_id(), d = blockIdx.y * 256 + lane_id() * 4;
    if (n >= N || d >= D) return;
    const int p = place[n], parts = rows->cut.dh, e = dh_exponent(*rows, half);
    const float g = p >= 0 && half ? dloss[n] : 1.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (p >= 0) {
        const float *from = sums + (size_t)p * D + d;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) x += get4(from + k * part, D - d);
    }
    put4(dh + (size_t)n * D + d, scaled(x, -e) * g, D - d);
}

// ---- host ---------------------------------------------------------------------------------------------------------------
static size_t up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr size_t kPackBytes = (size_t)128 << 20;      // of f32 words' planes at a time
constexpr size_t kDzBytes = (size_t)512 << 20;        // of dz and its turned form at a time
constexpr size_t kTurnedBytes = (size_t)512 << 20;    // of words' turned form at a time (with few rows a piece may be all words)
constexpr size_t kPartBytes = (size_t)256 << 20;      // of the parts of dW, and of dh
// A round of 512 blocks of 128 x 128 against one of 256 blocks of 256 x 256, twice its work at 1315 instead of 1130 TFLOP/s.
constexpr float kMidRound = 0.5f * 1315 / 1130;
constexpr size_t kMaxTiles = (size_t)1 << 22;         // of 128 x 128 in a launch: a grid has fewer than 2^32 threads

struct VocabPlan {
    int planes, pitch, turned_pitch;                  // of h and, if packed, of W; of h and dz turned
    bool pack_words, few;                             // few: of few rows, whose words are not packed (forward; backward of f32, turned ones are)
    int piece;                                        // words per piece, a multiple of 256
    int dz_planes;
    bool big_grads;
    CutArgs cut;
    size_t count, rows, place, hp, ht, wp, wt, dzt, dw, part_max, part_sum, part_z, z_label, dz, dh, steps, level, total;
    size_t h_plane, ht_plane, w_plane, wt_plane, dz_plane, dzt_plane, part_pitch;
    int tiles;                                        // most tiles along the vocabulary
};

static VocabPlan vocab_plan(const echo_vocab_desc_t &d, bool bwd) {
    VocabPlan p{};
    const size_t N = d.N, V = d.V, D = d.D;
    p.planes = d.in_dtype == ECHO_F32 ? 3 : 1;
    p.pitch = (int)up(D, 8);
    p.dz_planes = d.in_dtype == ECHO_F32 ? 3 : d.out_dtype == ECHO_F32 ? 2 : 1;
    p.few = d.in_dtype == ECHO_F32 ? few_pays<float>(N, V, D) : !bwd && few_pays<bf16_t>(N, V, D);
    if (p.few && !bwd) {
        p.tiles = (int)((V + few_words(d.N) - 1) / few_words(d.N));
        const size_t part = up(N * p.tiles * 4, 256);
        p.part_sum = part;
        p.part_z = 2 * part;
        p.z_label = 3 * part;
        p.total = 3 * part + up(N * 4, 256);
        return p;
    }
    p.pack_words = !p.few && (d.in_dtype == ECHO_F32 || D % 8 != 0);
    size_t piece = std::min(up(V, 256), std::max<size_t>(kMaxTiles * 128 * 128 / N / 256 * 256, 256));
    if (p.pack_words) piece = std::min(piece, std::max<size_t>(kPackBytes / (2 * p.planes * p.pitch) / 256 * 256, 256));
    if (bwd) {
        piece = std::min(piece, std::max<size_t>(kDzBytes / (4 * p.dz_planes * N) / 256 * 256, 256));
        piece = std::min(piece, std::max<size_t>(kTurnedBytes / (2 * p.planes * p.pitch) / 256 * 256, 256));
    }
    piece = up((V + (V + piece - 1) / piece - 1) / ((V + piece - 1) / piece), 256);   // pieces of about the same width
    p.piece = (int)piece;
    p.h_plane = N * p.pitch;
    p.w_plane = piece * p.pitch;
    p.turned_pitch = (int)up(N, 8);
    p.ht_plane = (size_t)p.pitch * p.turned_pitch;
    p.wt_plane = (size_t)p.pitch * piece;
    p.dz_plane = up(N, 8) * piece;
    p.dzt_plane = piece * p.turned_pitch;
    p.part_pitch = up(N, 64);
    p.tiles = (int)(up(V, piece) / piece * (piece / 128));
    if (bwd) {
        CutArgs cuts[2];
        float times[2];
        for (int big = 0; big < 2; ++big) {
            CutArgs &c = cuts[big];
            c = CutArgs{(int)std::min(piece, V), (int)D, 1, 1, big ? 256 : 128, big ? 256 : 512, p.planes == 3 ? 6 : p.dz_planes, big ? 1.f : kMidRound};
            c.most_dw = (int)std::min<size_t>(kMostParts, std::max<size_t>(1, kPartBytes / (piece * D * 4)));
            c.most_dh = (int)std::min<size_t>(kMostParts, std::max<size_t>(1, kPartBytes / (N * D * 4)));
            // room for what some numbers of rows with a label from a quarter to all of N ask for
            Cut most = {1, 1};
            for (int k = 4; k <= 16; k += 3) {
                const Cut x = cut_of(c, (int)((N * k + 15) / 16), times[big]);
                most.dw = std::max(most.dw, x.dw);
                most.dh = std::max(most.dh, x.dh);
            }
            c.most_dw = most.dw;
            c.most_dh = most.dh;
        }
        p.big_grads = times[1] <= times[0];
        p.cut = cuts[p.big_grads];
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes, 256);
        return here;
    };
    p.count = take(sizeof(Rows));
    p.rows = take(N * 4);
    p.place = take(N * 4);
    if (!p.few) p.hp = take(p.planes * p.h_plane * 2);
    if (p.pack_words) p.wp = take(p.planes * p.w_plane * 2);
    if (!bwd) {
        p.part_max = take(p.tiles * p.part_pitch * 4);
        p.part_sum = take(p.tiles * p.part_pitch * 4);
        p.part_z = take(p.tiles * p.part_pitch * 4);
        p.z_label = take(N * 4);
    } else {
        p.ht = take(p.planes * p.ht_plane * 2);
        p.wt = take(p.planes * p.wt_plane * 2);
        p.dz = take(p.dz_planes * p.dz_plane * 2);
        p.dzt = take(p.dz_planes * p.dzt_plane * 2);
        if (d.in_dtype == ECHO_BF16) {
            p.steps = take((N + 127) / 128 * piece);
            p.level = take(piece);
        }
        if (p.cut.most_dw > 1) p.dw = take(p.cut.most_dw * piece * D * 4);
        p.dh = take(p.cut.most_dh * N * D * 4);
    }
    p.total = at;
    return p;
}

// Which tile the logits take: rounds of 256 blocks of 256 x 256 against rounds of 512 (two to a compute unit) of 128 x 128.
static bool big_logits(size_t words, size_t N) {
    const size_t big = (up(words, 256) / 256) * (up(N, 256) / 256), mid = (up(words, 128) / 128) * (up(N, 128) / 128);
    return (float)((big + 255) / 256) <= kMidRound * (float)((mid + 511) / 512);
}

static PlanePairs pairs_of(int a, int b) {             // planes of the operands: nibbles, the small terms first
    if (a == 3 && b == 3) return {6, 0x001021u, 0x010201u};
    if (a == 1 && b == 2) return {2, 0u, 0x01u};
    return {1, 0u, 0u};
}

template <class C> static size_t product_lds() {
    return std::max<size_t>(C::LDS_BYTES, (size_t)C::BN * (C::BM * 2 + 16) + (C::WN + 1) * C::BM * 4);    // dz, and of its words the largest values and factors
}

// Launches a kernel whose LDS is above the default limit.
template <typename K, typename A>
static echo_status_t launch_tiles(const char *name, K *kernel, LdsGrants &granted, size_t lds, long long blocks, int threads, const A &args, hipStream_t st) {
    LaunchRecord r = launch_begin(name, st);
    if (ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), lds, granted) == hipSuccess) kernel<<<(unsigned)blocks, threads, lds, st>>>(args);
    return launch_end(r);
}

template <typename T, bool TEACHER> static void launch_few(const FewArgs &a, hipStream_t st) {
    if (a.N <= kFewAlone) k_vocab_few_alone<T, sizeof(T) == 2 ? 8 : 6, TEACHER><<<a.tiles, 256, 0, st>>>(a);
    else if (a.N <= 32) k_vocab_few_shared<T, 2, false, TEACHER><<<a.tiles, 512, 0, st>>>(a);
    else k_vocab_few_shared<T, 4, false, TEACHER><<<a.tiles * a.groups, 512, 0, st>>>(a);
}
template <bool TEACHER> static echo_status_t launch_few_dz(const FewArgs &a, hipStream_t st) {
    LaunchRecord r = launch_begin("vocab_few_dz", st);
    if (a.N <= 32) k_vocab_few_shared<float, 2, true, TEACHER><<<a.tiles, 512, 0, st>>>(a);
    else k_vocab_few_shared<float, 4, true, TEACHER><<<a.tiles * a.groups, 512, 0, st>>>(a);
    return launch_end(r);
}
template <class C, Mode MODE, bool TEACHER> static echo_status_t launch_logits(const LogitsArgs &a, int N, hipStream_t st) {
    static LdsGrants granted{};
    const long long blocks = (long long)((a.W.rows + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN);
    constexpr bool BWD = MODE != Mode::kForward;
    constexpr const char *name = C::BM == 256 ? (BWD ? "vocab_dlogits_256" : "vocab_logits_256") : (BWD ? "vocab_dlogits_128" : "vocab_logits_128");
    return launch_tiles(name, &k_vocab_logits<C, MODE, TEACHER>, granted, BWD ? product_lds<C>() : (size_t)C::LDS_BYTES, blocks,
                        C::THREADS, a, st);
}
template <class C, Mode MODE> static echo_status_t launch_grads(const GradsArgs &a, const CutArgs &cut, int N, hipStream_t st) {
    static LdsGrants granted{};
    const long long tm = (a.D + C::BM - 1) / C::BM, tw = (a.words + C::BN - 1) / C::BN, th = (N + C::BN - 1) / C::BN;
    const long long blocks = (tm * tw * (a.dW ? cut.most_dw : 0) + 7) / 8 * 8 + tm * th * (a.dh_sum ? cut.most_dh : 0);
    return launch_tiles(C::BM == 256 ? "vocab_grads_256" : "vocab_grads_128", &k_vocab_grads<C, MODE>, granted, C::LDS_BYTES, blocks, C::THREADS, a, st);
}

static echo_status_t check_vocab(const echo_vocab_desc_t *d, float eps) {
    if (!d) return ECHO_ERR_NULL;
    if ((d->in_dtype != ECHO_F32 && d->in_dtype != ECHO_BF16) || (d->out_dtype != ECHO_F32 && d->out_dtype != ECHO_BF16)) return ECHO_ERR_DTYPE;
    if (d->in_dtype == ECHO_F32 && d->out_dtype == ECHO_BF16) return ECHO_ERR_DTYPE;
    if (d->N < 1 || d->V < 1 || d->D < 1 || d->N > ECHO_VOCAB_MAX_ROWS || d->V > ECHO_VOCAB_MAX_ROWS || d->D > ECHO_VOCAB_MAX_D) return ECHO_ERR_SHAPE;
    if (!(eps >= 0.f) || !(eps < 1.f)) return ECHO_ERR_SHAPE;
    return ECHO_OK;
}

static bool unaligned(std::initializer_list<const void *> ps) {
    uintptr_t m = 0;
    for (const void *p : ps) m |= (uintptr_t)p;
    return (m & 15u) != 0;
}

struct VocabRun {
    echo_vocab_desc_t d;
    VocabPlan p;
    char *ws;
    const void *h, *W;
    const int *labels;
    hipStream_t st;
    template <typename T> T *at(size_t off) const { return reinterpret_cast<T *>(ws + off); }

    bool half() const { return d.in_dtype == ECHO_BF16; }                     // backward: dz and the turned forms in fp16

    // the rows with a label; turned: in their turned form too
    echo_status_t gather(bool turned, const CutArgs &cut, const LargestArgs &largest) const {
        LaunchRecord r = launch_begin("vocab_rows", st);
        k_vocab_rows<<<(d.N + kRowsBlock - 1) / kRowsBlock, 256, 0, st>>>(labels, d.N, d.V, at<int>(p.rows), at<int>(p.place), at<Rows>(p.count),
                                                                             cut);
        if (echo_status_t s = launch_end(r)) return s;
        if (largest.h || largest.W) {
            LargestArgs a = largest;
            a.out = at<Rows>(p.count);
            const long long per = 4 * 256 * 8;                                 // values of a block at a time
            a.h_block0 = a.W ? (int)std::min<long long>(((long long)d.V * d.D + per - 1) / per, 1024) : 0;
            r = launch_begin("vocab_largest", st);
            k_vocab_largest<<<a.h_block0 + (a.h ? std::min((d.N + 3) / 4, 1024) : 0), 256, 0, st>>>(a);
            if (echo_status_t s = launch_end(r)) return s;
        }
        if (p.few && !turned) return ECHO_OK;
        return pack("vocab_pack_rows", half() && turned, PackArgs{h, d.D, 0, d.N, p.pitch, p.turned_pitch, at<int>(p.rows), at<Rows>(p.count), p.few ? nullptr : at<bf16_t>(p.hp),
                                                turned ? at<bf16_t>(p.ht) : nullptr, p.h_plane, p.ht_plane});
    }
    echo_status_t pack(const char *name, bool half, const PackArgs &a) const {
        LaunchRecord r = launch_begin(name, st);
        const dim3 grid((a.n_rows + 63) / 64, (a.pitch + 63) / 64);
        if (d.in_dtype == ECHO_F32) k_vocab_pack<float, false><<<grid, 256, 0, st>>>(a);
        else if (half) k_vocab_pack<bf16_t, true><<<grid, 256, 0, st>>>(a);
        else k_vocab_pack<bf16_t, false><<<grid, 256, 0, st>>>(a);
        return launch_end(r);
    }
    // the words of a piece as an operand, and their turned form if it is wanted
    echo_status_t words(int v0, int n, bool turned, Operand &o) const {
        // (few rows: the operand is not used)
        o = p.pack_words ? Operand{at<bf16_t>(p.wp), p.w_plane, p.pitch, n} : Operand{static_cast<const bf16_t *>(W) + (size_t)v0 * d.D, 0, d.D, n};
        if (!p.pack_words && !turned) return ECHO_OK;
        return pack("vocab_pack_words", half() && turned, PackArgs{W, d.D, v0, n, p.pitch, p.piece, nullptr, at<Rows>(p.count), p.pack_words ? at<bf16_t>(p.wp) : nullptr,
                                                 turned ? at<bf16_t>(p.wt) : nullptr, p.w_plane, p.wt_plane});
    }
    Operand rows() const { return Operand{at<bf16_t>(p.hp), p.h_plane, p.pitch, d.N}; }
};

// the few-row form of a backward launch over n words from a.v0
static FewArgs few_dz_args(const VocabRun &x, const LogitsArgs &a, int n) {
    FewArgs f{};
    f.h = x.h;
    f.W = static_cast<const float *>(x.W) + (size_t)a.v0 * x.d.D;
    f.labels = a.labels;
    f.N = x.d.N, f.V = n, f.D = x.d.D;
    f.tiles = (n + few_words(kFewGroup) - 1) / few_words(kFewGroup);
    f.groups = (x.d.N + kFewGroup - 1) / kFewGroup;
    f.eps = a.eps;
    f.v0 = a.v0, f.all_words = a.V;
    f.count = a.count;
    f.rows = a.rows;
    f.lse = a.lse, f.dloss = a.dloss;
    f.dz = a.dz, f.turned = a.turned;
    f.dz_plane = a.dz_plane, f.turned_plane = a.turned_plane;
    f.dz_pitch = a.dz_pitch, f.turned_pitch = a.turned_pitch;
    f.teacher = a.teacher;
    return f;
}

// TEACHER: x.labels holds a word of every row that takes part, which is what the rows are gathered by; eps is 0
template <bool TEACHER>
static echo_status_t run_forward(const VocabRun &x, float eps, const Teacher &teacher, float *loss, float *lse) {
    const int N = x.d.N, V = x.d.V;
    if (x.p.few) {
        FewArgs a{x.h, x.W, x.labels, N, V, x.d.D, x.p.tiles, (N + kFewGroup - 1) / kFewGroup, eps, x.at<float>(x.p.part_max), x.at<float>(x.p.part_sum),
                        x.at<float>(x.p.part_z), x.at<float>(x.p.z_label)};
        a.teacher = teacher;
        LaunchRecord r = launch_begin("vocab_few", x.st);
        if (x.d.in_dtype == ECHO_F32) launch_few<float, TEACHER>(a, x.st);
        else launch_few<bf16_t, TEACHER>(a, x.st);
        if (echo_status_t s = launch_end(r)) return s;
        r = launch_begin("vocab_few_finish", x.st);
        k_vocab_few_finish<TEACHER><<<N, 256, 0, x.st>>>(a, loss, lse);
        return launch_end(r);
    }
    if (echo_status_t s = x.gather(false, CutArgs{}, LargestArgs{})) return s;
    LogitsArgs a{};
    a.h = x.rows();
    a.D = x.p.pitch;
    a.pairs = pairs_of(x.p.planes, x.p.planes);
    a.count = x.at<Rows>(x.p.count);
    a.rows = x.at<int>(x.p.rows);
    a.labels = x.labels;
    a.V = V;
    a.eps = eps;
    a.teacher = teacher;
    a.part_max = x.at<float>(x.p.part_max);
    a.part_sum = x.at<float>(x.p.part_sum);
    a.part_z = x.at<float>(x.p.part_z);
    a.z_label = x.at<float>(x.p.z_label);
    a.pitch = x.p.part_pitch;
    const bool big = big_logits(std::min(x.p.piece, V), N);
    int tiles = 0;
    for (int v0 = 0; v0 < V; v0 += x.p.piece) {
        const int n = std::min(x.p.piece, V - v0);
        if (echo_status_t s = x.words(v0, n, false, a.W)) return s;
        a.v0 = v0;
        a.first_tile = tiles;
        if (echo_status_t s = big ? launch_logits<BigTile, Mode::kForward, TEACHER>(a, N, x.st) : launch_logits<MidTile, Mode::kForward, TEACHER>(a, N, x.st)) return s;
        tiles += big ? (n + 255) / 256 : (n + 127) / 128;
    }
    LaunchRecord r = launch_begin("vocab_loss_finish", x.st);
    k_vocab_loss_finish<TEACHER><<<(N + 63) / 64, 256, 0, x.st>>>(a.part_max, a.part_sum, a.part_z, a.z_label, x.at<int>(x.p.place), N, V, tiles, a.pitch,
                                                                  eps, teacher, big ? 8 : 7, loss, lse);
    return launch_end(r);
}

template <bool TEACHER>
static echo_status_t run_backward(const VocabRun &x, float eps, const Teacher &teacher, const float *dloss, const float *lse, void *dh, void *dW) {
    const int N = x.d.N, V = x.d.V, D = x.d.D;
    const VocabPlan &p = x.p;
    LargestArgs l{};
    if (x.half()) l = LargestArgs{dW ? static_cast<const bf16_t *>(x.h) : nullptr, dh ? static_cast<const bf16_t *>(x.W) : nullptr, dloss, x.labels, N, V, D};
    if (echo_status_t s = x.gather(dW != nullptr, x.p.cut, l)) return s;
    LogitsArgs a{};
    a.h = x.rows();
    a.D = p.pitch;
    a.pairs = pairs_of(p.planes, p.planes);
    a.count = x.at<Rows>(p.count);
    a.rows = x.at<int>(p.rows);
    a.labels = x.labels;
    a.V = V;
    a.eps = eps;
    a.teacher = teacher;
    a.lse = lse;
    a.dloss = dloss;
    a.dz = dh ? x.at<bf16_t>(p.dz) : nullptr;
    a.dz_plane = p.dz_plane;
    a.dz_pitch = p.piece;
    a.turned = dW ? x.at<bf16_t>(p.dzt) : nullptr;
    a.turned_plane = p.dzt_plane;
    a.turned_pitch = p.turned_pitch;
    a.steps = x.at<unsigned char>(p.steps);
    GradsArgs g{};
    g.dz = Operand{a.dz, p.dz_plane, p.piece, N};
    g.h_turned = Operand{x.at<bf16_t>(p.ht), p.ht_plane, p.turned_pitch, p.pitch};
    g.W_turned = Operand{x.at<bf16_t>(p.wt), p.wt_plane, p.piece, p.pitch};
    g.rows = a.count;
    g.D = D;
    g.pairs = pairs_of(p.planes, p.dz_planes);
    g.dw_sum = x.at<float>(p.dw);
    g.dw_part = (size_t)p.piece * D;
    g.dh_sum = dh ? x.at<float>(p.dh) : nullptr;
    g.dh_part = (size_t)N * D;
    const bool bf16_out = x.d.out_dtype == ECHO_BF16;
    const size_t out_bytes = bf16_out ? 2 : 4;
    const bool big = big_logits(std::min(p.piece, V), N);
    const int row_tile = big ? 256 : 128, row_tiles = (N + row_tile - 1) / row_tile;
    if (x.half()) g.level = row_tiles > 1 ? x.at<unsigned char>(p.level) : a.steps;
    for (int v0 = 0; v0 < V; v0 += p.piece) {
        const int n = std::min(p.piece, V - v0);
        if (echo_status_t s = x.words(v0, n, dh != nullptr, a.W)) return s;
        a.v0 = v0;
        echo_status_t s;
        if (p.few) s = launch_few_dz<TEACHER>(few_dz_args(x, a, n), x.st);
        else if (!x.half()) s = big ? launch_logits<BigTile, Mode::kPlanes, TEACHER>(a, N, x.st) : launch_logits<MidTile, Mode::kPlanes, TEACHER>(a, N, x.st);
        else if (bf16_out) s = big ? launch_logits<BigTile, Mode::kHalf, TEACHER>(a, N, x.st) : launch_logits<MidTile, Mode::kHalf, TEACHER>(a, N, x.st);
        else s = big ? launch_logits<BigTile, Mode::kHalves, TEACHER>(a, N, x.st) : launch_logits<MidTile, Mode::kHalves, TEACHER>(a, N, x.st);
        if (s) return s;
        if (dW && x.half() && row_tiles > 1) {
            LaunchRecord r = launch_begin("vocab_level", x.st);
            const dim3 grid((n + 63) / 64, std::min(64, (row_tiles + 15) / 16));
            if (bf16_out) k_vocab_level<1><<<grid, 256, 0, x.st>>>(a.count, a.steps, p.piece, row_tile, a.turned, p.dzt_plane, p.turned_pitch, n, x.at<unsigned char>(p.level));
            else k_vocab_level<2><<<grid, 256, 0, x.st>>>(a.count, a.steps, p.piece, row_tile, a.turned, p.dzt_plane, p.turned_pitch, n, x.at<unsigned char>(p.level));
            if (echo_status_t s = launch_end(r)) return s;
        }
        g.words = n;
        g.dz_turned = Operand{a.turned, p.dzt_plane, p.turned_pitch, n};
        g.dW = dW ? static_cast<char *>(dW) + (size_t)v0 * D * out_bytes : nullptr;
        g.add = v0 > 0;
        if (!x.half()) s = p.big_grads ? launch_grads<BigTile, Mode::kPlanes>(g, p.cut, N, x.st) : launch_grads<MidTile, Mode::kPlanes>(g, p.cut, N, x.st);
        else if (bf16_out) s = p.big_grads ? launch_grads<BigTile, Mode::kHalf>(g, p.cut, N, x.st) : launch_grads<MidTile, Mode::kHalf>(g, p.cut, N, x.st);
        else s = p.big_grads ? launch_grads<BigTile, Mode::kHalves>(g, p.cut, N, x.st) : launch_grads<MidTile, Mode::kHalves>(g, p.cut, N, x.st);
        if (s) return s;
        if (dW && p.cut.most_dw > 1) {
            LaunchRecord r = launch_begin("vocab_dw_finish", x.st);
            if (bf16_out) k_vocab_dw_finish<<<(n + 3) / 4, 256, 0, x.st>>>(g.rows, g.level, g.dw_sum, g.dw_part, n, D, static_cast<bf16_t *>(g.dW));
            else k_vocab_dw_finish<<<(n + 3) / 4, 256, 0, x.st>>>(g.rows, g.level, g.dw_sum, g.dw_part, n, D, static_cast<float *>(g.dW));
            if (echo_status_t s = launch_end(r)) return s;
        }
    }
    if (!dh) return ECHO_OK;
    LaunchRecord r = launch_begin("vocab_dh_finish", x.st);
    if (bf16_out) k_vocab_dh_finish<<<dim3((N + 3) / 4, (D + 255) / 256), 256, 0, x.st>>>(g.rows, x.half(), g.dh_sum, g.dh_part, x.at<int>(p.place), dloss, N, D, static_cast<bf16_t *>(dh));
    else k_vocab_dh_finish<<<dim3((N + 3) / 4, (D + 255) / 256), 256, 0, x.st>>>(g.rows, x.half(), g.dh_sum, g.dh_part, x.at<int>(p.place), dloss, N, D, static_cast<float *>(dh));
    return launch_end(r);
}

// ---- distillation: the workspace of the loss, and behind it what the teacher's lists are made into ---------------------------
struct TeacherPlan {
    int marks;
    size_t labels, own, dloss, words, shares, start, total;
};
static TeacherPlan teacher_plan(const echo_vocab_desc_t &d, int K, size_t at) {
    TeacherPlan p{};
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes, 256);
        return here;
    };
    const size_t N = d.N;
    p.marks = (d.V + kMarkWords - 1) / kMarkWords + 1;
    p.labels = take(N * 4);
    p.own = take(N * 4);
    p.dloss = take(N * 4);
    p.words = take(N * K * 4);
    p.shares = take(N * K * 4);
    p.start = take(N * p.marks);
    p.total = at;
    return p;
}
static echo_status_t check_distill(const echo_vocab_desc_t *d, int K, float T) {
    if (echo_status_t s = check_vocab(d, 0.f)) return s;
    return K < 1 || K > ECHO_DISTILL_MAX_K || !(T >= 0x1p-64f && T <= 0x1p64f) ? ECHO_ERR_SHAPE : ECHO_OK;
}
// the lists, sorted, and the run that works on them
static echo_status_t distill_begin(VocabRun &x, const TeacherPlan &p, const int *words, const float *logits, int K, float T, const float *dloss,
                                   Teacher &teacher) {
    TeacherLists l{};
    l.words = words, l.logits = logits, l.dloss = dloss;
    l.N = x.d.N, l.V = x.d.V, l.K = K, l.marks = p.marks;
    l.temperature = T;
    l.labels = x.at<int>(p.labels);
    l.own = x.at<float>(p.own);
    l.dloss_out = x.at<float>(p.dloss);
    l.words_out = x.at<int>(p.words);
    l.shares = x.at<float>(p.shares);
    l.start = x.at<unsigned char>(p.start);
    x.labels = l.labels;
    teacher = Teacher{l.words_out, l.shares, l.start, l.own, K, p.marks, 1.f / T, T};
    return launch_teacher_lists(l, x.st);
}

}  // namespace echo

extern "C" {

size_t echo_vocab_loss_fwd_workspace_bytes(const echo_vocab_desc_t *desc) {
    if (echo::check_vocab(desc, 0.f)) return 0;
    return echo::vocab_plan(*desc, false).total;
}

size_t echo_vocab_loss_bwd_workspace_bytes(const echo_vocab_desc_t *desc) {
    if (echo::check_vocab(desc, 0.f)) return 0;
    return echo::vocab_plan(*desc, true).total;
}

echo_status_t echo_vocab_loss_fwd(const echo_vocab_desc_t *desc, const void *h, const void *W, const int32_t *labels,
                                  float label_smoothing, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                                  void *stream) {
    using namespace echo;
    if (echo_status_t s = check_vocab(desc, label_smoothing)) return s;
    if (!h || !W || !labels || !loss || !lse || !workspace) return ECHO_ERR_NULL;
    if (unaligned({h, W, labels, loss, lse, workspace})) return ECHO_ERR_ALIGN;
    const VocabRun x{*desc, vocab_plan(*desc, false), static_cast<char *>(workspace), h, W, labels, static_cast<hipStream_t>(stream)};
    if (workspace_bytes < x.p.total) return ECHO_ERR_WORKSPACE;
    return run_forward<false>(x, label_smoothing, Teacher{}, loss, lse);
}

echo_status_t echo_vocab_loss_bwd(const echo_vocab_desc_t *desc, const float *dloss, const float *lse, const void *h, const void *W,
                                  const int32_t *labels, float label_smoothing, void *dh, void *dW, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_vocab(desc, label_smoothing)) return s;
    if (!dloss || !lse || !h || !W || !labels || (!dh && !dW) || !workspace) return ECHO_ERR_NULL;
    if (unaligned({dloss, lse, h, W, labels, dh, dW, workspace})) return ECHO_ERR_ALIGN;
    const VocabRun x{*desc, vocab_plan(*desc, true), static_cast<char *>(workspace), h, W, labels, static_cast<hipStream_t>(stream)};
    if (workspace_bytes < x.p.total) return ECHO_ERR_WORKSPACE;
    return run_backward<false>(x, label_smoothing, Teacher{}, dloss, lse, dh, dW);
}

size_t echo_distill_fwd_workspace_bytes(const echo_vocab_desc_t *desc, int32_t K) {
    if (echo::check_distill(desc, K, 1.f)) return 0;
    return echo::teacher_plan(*desc, K, echo::vocab_plan(*desc, false).total).total;
}

size_t echo_distill_bwd_workspace_bytes(const echo_vocab_desc_t *desc, int32_t K) {
    if (echo::check_distill(desc, K, 1.f)) return 0;
    return echo::teacher_plan(*desc, K, echo::vocab_plan(*desc, true).total).total;
}

echo_status_t echo_distill_fwd(const echo_vocab_desc_t *desc, const void *h, const void *W, const int32_t *words, const float *logits,
                               int32_t K, float T, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_distill(desc, K, T)) return s;
    if (!h || !W || !words || !logits || !loss || !lse || !workspace) return ECHO_ERR_NULL;
    if (unaligned({h, W, words, logits, loss, lse, workspace})) return ECHO_ERR_ALIGN;
    VocabRun x{*desc, vocab_plan(*desc, false), static_cast<char *>(workspace), h, W, nullptr, static_cast<hipStream_t>(stream)};
    const TeacherPlan p = teacher_plan(*desc, K, x.p.total);
    if (workspace_bytes < p.total) return ECHO_ERR_WORKSPACE;
    Teacher teacher;
    if (echo_status_t s = distill_begin(x, p, words, logits, K, T, nullptr, teacher)) return s;
    return run_forward<true>(x, 0.f, teacher, loss, lse);
}

echo_status_t echo_distill_bwd(const echo_vocab_desc_t *desc, const float *dloss, const float *lse, const void *h, const void *W,
                               const int32_t *words, const float *logits, int32_t K, float T, void *dh, void *dW, void *workspace,
                               size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_distill(desc, K, T)) return s;
    if (!dloss || !lse || !h || !W || !words || !logits || (!dh && !dW) || !workspace) return ECHO_ERR_NULL;
    if (unaligned({dloss, lse, h, W, words, logits, dh, dW, workspace})) return ECHO_ERR_ALIGN;
    VocabRun x{*desc, vocab_plan(*desc, true), static_cast<char *>(workspace), h, W, nullptr, static_cast<hipStream_t>(stream)};
    const TeacherPlan p = teacher_plan(*desc, K, x.p.total);
    if (workspace_bytes < p.total) return ECHO_ERR_WORKSPACE;
    Teacher teacher;
    if (echo_status_t s = distill_begin(x, p, words, logits, K, T, dloss, teacher)) return s;
    return run_backward<true>(x, 0.f, teacher, x.at<float>(p.dloss), lse, dh, dW);
}

}  // extern "C"
