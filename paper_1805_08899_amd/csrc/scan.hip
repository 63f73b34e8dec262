// A gated linear recurrence over whole sequences, forward and backward (include/echoscan.h has the formulas).
//
// A thread owns kSteps consecutive steps of VEC channels; 16 such threads stand side by side, GROUPS of them one behind the other, and together take
// GROUPS kSteps steps of 16 VEC channels.  A thread's steps are a linear map of the state, c -> A c + b (backward: q -> A q + R).  A wave folds the maps of
// its four groups in LDS, a lane per channel, and every wave those of the waves in front of it; from the state in front of its own, every thread goes on
// by itself.  A sequence longer than a chunk is a chain of them, whose chunks are one block's or many blocks' (below).
//
// f and u = 1 - f = sigmoid(-x) are each good to a few units of their own last place, the smaller one as e / (1 + e) with e = 2^(-|x| log2 e): with f as 1 - u, what
// a gate at -12 lets through would be off by 1 % and nothing be left from -17 on.  A thread that keeps a gate keeps the smaller of both, f with its sign
// set (Forget below).  It costs a selection per gate where either is wanted: both passes of 64 x 50 x 512 f32 11.7 -> 12.4 us, of 4 x 16384 x 1280 bf16 414 -> 433,
// of f32 none.
//
// Every gate is read once and every result written once, which is what bounds long sequences: 4 x 16384 x 1280 f32 takes 250 + 420 us, 5.4 TB/s (a large copy: 6.4).
// Shorter ones are bound by trips to memory: a launch and one unit are 4 us (64 x 1 x 512), one sequence of 4001 x 768 bf16 is 10 us behind the clearing's 2.
// 16 threads x 4 channels are 256 bytes of a row in f32 and 128 in bf16; four steps a thread keep a unit's gates in registers from the map to the result (a chunk of 128
// steps: two blocks of 512 threads to a compute unit).
#include "../../include/echoscan.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kSteps = 4;
template <int GROUPS> constexpr int kThreads = GROUPS > 16 ? 512 : 256;
constexpr int kBlocks = 2;            // to a compute unit
constexpr int kXcds = 8;
constexpr int kQueues = 32, kTicketStride = 16;            // (words of 8 bytes: a cache line)
constexpr int kChunkGroups = ECHO_SCAN_CHUNK / kSteps;
constexpr float kLog2eS = 1.4426950408889634f;

// sigmoid(x) = 1 / (1 + 2^(-x log2 e)); tanh(x) = 1 - 2 / (2^(2 x log2 e) + 1).  exp2 overflows to infinity, whose reciprocal is 0.
__device__ __forceinline__ float gate(float x) { return fast_rcp(1.0f + fast_exp2(-kLog2eS * x)); }
// f = sigmoid(x) and u = 1 - f from the smaller one, `least`, as a thread keeps it: f with its sign set, or u; 0, an open gate, for a step that is none of the sequence's
struct Forget {
    float least;
    bool f_least;
    static __device__ __forceinline__ float pack(float x) {
        const float e = fast_exp2(-kLog2eS * fabsf(x));
        return copysignf(e * fast_rcp(1.0f + e), x);
    }
    __device__ __forceinline__ explicit Forget(float packed) : least(fabsf(packed)), f_least(__float_as_int(packed) < 0) {}
    __device__ __forceinline__ float f() const { return f_least ? least : 1.0f - least; }
    __device__ __forceinline__ float u() const { return f_least ? 1.0f - least : least; }
    // f c + u g: from the one of c and g that counts more, `least` of the way to the other
    __device__ __forceinline__ float step(float c, float g) const {
        const float more = f_least ? g : c, less = f_least ? c : g;
        return __builtin_fmaf(least, less - more, more);
    }
};
__device__ __forceinline__ float candidate(float x) {
    return __builtin_fmaf(-2.0f, fast_rcp(fast_exp2(kTwoLog2e * x) + 1.0f), 1.0f);
}
// A thread's map of its steps up to step i, from that of those in front: c -> A c + b.  x: the forget gate's; in: the step is the sequence's
template <int VEC> __device__ __forceinline__ void add_step(float (&A)[kSteps][VEC], float (&b)[kSteps][VEC], int i, int v, float x, float g, bool in) {
    const float e = fast_exp2(-kLog2eS * fabsf(x)), most = fast_rcp(1.0f + e), least = e * most;
    const float f = x < 0.f ? least : most, u = x < 0.f ? most : least;
    const float b0 = i ? b[i ? i - 1 : 0][v] : 0.f, A0 = i ? A[i ? i - 1 : 0][v] : 1.f;
    b[i][v] = in ? __builtin_fmaf(f, b0, u * g) : b0;
    A[i][v] = in ? f * A0 : A0;
}

// VEC consecutive channels of a row as they stand in memory; rows begin at any element
template <typename T, int VEC> struct Lanes;
template <typename T> struct Lanes<T, 4> {
    RawKey<T> raw;
    __device__ __forceinline__ void load(const T *p) { raw.load(p, 0); }
    __device__ __forceinline__ void get(float (&x)[4]) const {
        const float4 v = raw.get();
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    }
};
template <typename T> struct Lanes<T, 1> {
    typename RawElem<T>::type raw;
    __device__ __forceinline__ void load(const T *p) { raw = RawElem<T>::load(p, 0); }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = RawElem<T>::value(raw); }
};
typedef unsigned u32x4_any __attribute__((ext_vector_type(4)));
typedef __bf16 bf16_hw;
__device__ __forceinline__ unsigned bf16_bits(float x) { return __builtin_bit_cast(unsigned short, (bf16_hw)x); }
__device__ __forceinline__ void put_one(float *p, float x) { *p = x; }
__device__ __forceinline__ void put_one(bf16_t *p, float x) { p->bits = (unsigned short)bf16_bits(x); }
// whole: the rows consist of whole groups of 16 bytes
template <int VEC> __device__ __forceinline__ void put(float *p, const float (&x)[VEC], bool whole) {
    if constexpr (VEC == 4) {
        const f32x4 v = {x[0], x[1], x[2], x[3]};
        if (whole) __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(p));
        else *reinterpret_cast<f32x4_any *>(p) = v;
    } else {
        *p = x[0];
    }
}
template <int VEC> __device__ __forceinline__ void put(bf16_t *p, const float (&x)[VEC], bool whole) {
    if constexpr (VEC == 4) {
        const u32x2 v = {bf16_bits(x[0]) | bf16_bits(x[1]) << 16, bf16_bits(x[2]) | bf16_bits(x[3]) << 16};
        if (whole) __builtin_nontemporal_store(v, reinterpret_cast<u32x2 *>(p));
        else *reinterpret_cast<u32x2_any *>(p) = v;
    } else {
        p->bits = (unsigned short)bf16_bits(x[0]);
    }
}
// x[skip ..]: what a lane's neighbour has in front of that is not its own
template <typename T, int VEC> __device__ __forceinline__ void put_from(T *p, const float (&x)[VEC], int skip, bool whole) {
    if (skip == 0) {
        put<VEC>(p, x, whole);
    } else {
#pragma unroll
        for (int v = 1; v < VEC; ++v)
            if (v >= skip) put_one(p + v, x[v]);
    }
}

struct ScanArgs {
    const void *G, *dh;
    const float *first;              // c0; dc_last
    const int *len;
    int B, T, H, reverse, chunks, groups_h;   // groups_h: units along the channels
    long long chains, chain0;        // B groups_h; the launch's first
    void *out;                       // h; dG
    float *last;                     // c_last; dc0
    float *states;
    unsigned long long *words, *tickets;      // [chunks][chains][WIDTH]; [queues], kTicketStride apart: the next to be taken
    int queues;
    bool whole;                      // rows are whole groups of 16 bytes
};

// What a thread is in a unit: its channels of a sequence, kSteps steps of a chunk
template <int VEC, int GROUPS> struct Place {
    static constexpr int SUBS = kThreads<GROUPS> / 16 / GROUPS, WIDTH = 16 * VEC;
    int group, sub, slot, b, ch, skip, s0;                 // skip: of its VEC channels, those in front that are the neighbour's
    bool on;                         // it has channels of its own
    int n;                           // steps of the sequence
    __device__ __forceinline__ Place(const ScanArgs &a, long long first_chain, int chunk) {
        group = (threadIdx.x >> 4) % GROUPS;
        sub = SUBS == 1 ? 0 : (threadIdx.x >> 4) / GROUPS;
        const long long chain = min(first_chain + sub, a.chains - 1);
        b = (int)(chain / a.groups_h);
        channels(a, (int)(chain - (long long)b * a.groups_h), first_chain + sub < a.chains);
        n = a.len ? clamp_len(a.len[b], a.T) : a.T;
        s0 = (chunk * GROUPS + group) * kSteps;
    }
    __device__ __forceinline__ Place(const ScanArgs &a, int b_, int g, int n_, int chunk) : sub(0), b(b_), n(n_) {
        static_assert(SUBS == 1, "a chunk of one chain");
        group = (threadIdx.x >> 4) % GROUPS;
        channels(a, g, true);
        s0 = (chunk * GROUPS + group) * kSteps;
    }
    __device__ __forceinline__ void channels(const ScanArgs &a, int g, bool there) {
        slot = (threadIdx.x & 15) * VEC;
        on = there && g * WIDTH + slot < a.H;
        ch = min(g * WIDTH + slot, a.H - VEC);             // the last lane steps back to a whole group of channels
        skip = g * WIDTH + slot - ch;
    }
    __device__ __forceinline__ bool in(int i) const { return s0 + i < n; }
    // position of the thread's step i; steps from n on stand at their own number
    __device__ __forceinline__ int position(const ScanArgs &a, int i) const { return a.reverse && in(i) ? n - 1 - s0 - i : s0 + i; }
};

// What a lane is where a wave folds maps: a channel
template <int VEC> struct Folder {
    static constexpr int WIDTH = 16 * VEC;
    int lane, ch;
    bool on, own;                    // it is one; the unit's own
    size_t row;                      // of c0 and c_last
    __device__ __forceinline__ Folder(const ScanArgs &a, int b, int g, bool there) {
        lane = lane_id() % WIDTH;
        const int c = g * WIDTH + lane / VEC * VEC;
        ch = max(0, min(c, a.H - VEC)) + lane % VEC;
        on = lane_id() < WIDTH;
        own = on && there && c < a.H && ch >= c;
        row = (size_t)b * a.H + ch;
    }
};
// a wave's own exchange through LDS
__device__ __forceinline__ void settle() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A number that was requested is here
__device__ __forceinline__ void here(float &x) { asm volatile("" : "+v"(x)); }

// The maps of a wave's four groups, a lane per channel, and of all four; BACK: in their order backwards
template <int WIDTH, bool BACK> struct FourMaps {
    float A[4], b[4];
    static __device__ __forceinline__ int order(int k) { return BACK ? 3 - k : k; }
    __device__ __forceinline__ void read(const float (*sa)[WIDTH], const float (*sb)[WIDTH], int lane) {
#pragma unroll
        for (int k = 0; k < 4; ++k) A[k] = sa[order(k)][lane], b[k] = sb[order(k)][lane];
    }
    __device__ __forceinline__ void total(float &all, float &sum) const {
        all = A[0], sum = b[0];
#pragma unroll
        for (int k = 1; k < 4; ++k) sum = __builtin_fmaf(A[k], sum, b[k]), all *= A[k];
    }
    // the state in front of each group takes the place of its b; the one behind all is returned
    __device__ __forceinline__ float write(float (*sb)[WIDTH], int lane, float state) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sb[order(k)][lane] = state;
            state = __builtin_fmaf(A[k], state, b[k]);
        }
        return state;
    }
};
// The maps of W waves
template <int WIDTH, int W, bool BACK> struct WaveMaps {
    float A[W], b[W];
    static __device__ __forceinline__ int order(int k) { return BACK ? W - 1 - k : k; }
    __device__ __forceinline__ void read(const float (&sa)[W][WIDTH], const float (&sb)[W][WIDTH], int lane) {
#pragma unroll
        for (int k = 0; k < W; ++k) A[k] = sa[order(k)][lane], b[k] = sb[order(k)][lane];
    }
    __device__ __forceinline__ void total(float &all, float &sum) const {
        all = A[0], sum = b[0];
#pragma unroll
        for (int k = 1; k < W; ++k) sum = __builtin_fmaf(A[k], sum, b[k]), all *= A[k];
    }
    // the state in front of wave w
    __device__ __forceinline__ float state(float start, int w) const {
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
            if (k < order(w)) start = __builtin_fmaf(A[k], start, b[k]);
        return start;
    }
};

// A thread's rows.  FULL: all steps of the unit are the sequence's, and all of its addresses are one 32-bit offset behind scalar ones.
template <typename T, bool FULL> struct Row {
    T *base;
    unsigned off;                    // bytes
    int step;                        // elements from step to step
    // rows of `width` elements, of which the thread's channels of array k stand `between` elements behind those of array k - 1
    template <typename P> __device__ __forceinline__ Row(const ScanArgs &a, const void *array, int width, const P &p, int chunk) {
        base = (T *)array + (size_t)p.b * a.T * width;
        if constexpr (FULL) {
            const int low = a.reverse ? p.n - (chunk + 1) * ECHO_SCAN_CHUNK : chunk * ECHO_SCAN_CHUNK;
            base += (size_t)low * width;
            step = a.reverse ? -width : width;
            // (at most 127 rows of 3 2^20 elements: 2^31 bytes)
            off = ((unsigned)(a.reverse ? ECHO_SCAN_CHUNK - 1 - p.group * kSteps : p.group * kSteps) * (unsigned)width + (unsigned)p.ch) * (unsigned)sizeof(T);
        } else {
            base += p.ch;
        }
    }
    template <typename P> __device__ __forceinline__ T *at(const ScanArgs &a, const P &p, int i, int width, int behind, bool load) const {
        if constexpr (FULL) return (T *)((const char *)(base + ((long long)i * step + behind)) + off);
        else return base + (size_t)(load && !p.in(i) ? 0 : p.position(a, i)) * width + behind;
    }
};

// A wave's channels where there are no chains: of its unit, which GROUPS / 4 waves share (GROUPS of 1: nothing is folded)
template <int VEC, int GROUPS> __device__ __forceinline__ Folder<VEC> wave_folder(const ScanArgs &a, long long first_chain) {
    const long long mine = first_chain + wave_id() / (GROUPS > 4 ? GROUPS / 4 : 1), chain = min(mine, a.chains - 1);
    const int b = (int)(chain / a.groups_h);
    return Folder<VEC>(a, b, (int)(chain - (long long)b * a.groups_h), mine < a.chains);
}

// ---- one chunk ---------------------------------------------------------------------------------------------------------------
template <typename T, int VEC, int GROUPS>
__global__ __launch_bounds__(kThreads<GROUPS>, 4) void k_scan_fwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    constexpr int ALL = P::SUBS * GROUPS, W = GROUPS / 4;
    __shared__ float s_a[ALL][P::WIDTH], s_b[ALL][P::WIDTH], s_wa[W > 1 ? W : 1][P::WIDTH], s_wb[W > 1 ? W : 1][P::WIDTH];
    const int w = wave_id(), own = threadIdx.x >> 4;       // the thread's group in the block
    const long long first_chain = a.chain0 + (long long)blockIdx.x * P::SUBS;
    const P p(a, first_chain, 0);
    const Row<const T, false> G(a, a.G, 3 * a.H, p, 0);
    const Row<T, false> h(a, a.out, a.H, p, 0);
    Lanes<T, VEC> x[kSteps][3];
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) x[i][k].load(G.at(a, p, i, 3 * a.H, k * a.H, true));
    const Folder<VEC> f = wave_folder<VEC, GROUPS>(a, first_chain);
    float state = GROUPS > 1 && a.first ? a.first[f.row] : 0.f;
    float c[VEC];
    if constexpr (GROUPS == 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) c[v] = a.first ? a.first[(size_t)p.b * a.H + p.ch + v] : 0.f;
        if (a.states && p.on) {
#pragma unroll
            for (int v = 0; v < VEC; ++v)
                if (v >= p.skip) a.states[(size_t)p.b * a.H + p.ch + v] = c[v];
        }
    }
    // GROUPS of 1: the forget gate as kept, and the candidate, step by step; else the maps of the thread's first steps
    float A[kSteps][VEC], b[kSteps][VEC];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float y[VEC], z[VEC];
        x[i][0].get(y);
        x[i][1].get(z);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            const float g = candidate(z[v]);
            if constexpr (GROUPS == 1) {
                A[i][v] = p.in(i) ? Forget::pack(y[v]) : 0.f;
                b[i][v] = p.in(i) ? g : 0.f;
            } else {
                add_step(A, b, i, v, y[v], g, p.in(i));
            }
        }
    }
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            s_a[own][p.slot + v] = A[kSteps - 1][v];
            s_b[own][p.slot + v] = b[kSteps - 1][v];
        }
        if (a.states && f.own && w % W == 0) a.states[f.row] = state;
        settle();
        FourMaps<P::WIDTH, false> m;
        m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
        if constexpr (W > 1) {
            float all, sum;
            m.total(all, sum);
            if (f.on) s_wa[w][f.lane] = all, s_wb[w][f.lane] = sum;
            here(state);                                   // in front of the barrier: behind it the unit's last wave writes c_last, which may be c0
            lds_barrier();
            WaveMaps<P::WIDTH, W, false> wm;
            wm.read(s_wa, s_wb, f.lane);
            state = wm.state(state, w);
        }
        if (f.on) state = m.write(s_b + 4 * w, f.lane, state);
        if (a.last && f.own && w % W == W - 1) a.last[f.row] = state;
        settle();
#pragma unroll
        for (int v = 0; v < VEC; ++v) c[v] = s_b[own][p.slot + v];
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float y[VEC];
        x[i][2].get(y);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            float at;
            if constexpr (GROUPS == 1) {
                // step by step from call to call: f as a factor would lose a third of a percent of a gate that forgets 1e-5 to its rounding, the same in every step
                const Forget k(A[i][v]);
                at = c[v] = fabsf(c[v]) == __builtin_inff() ? k.f() * c[v] : k.step(c[v], b[i][v]);
            } else {
                at = __builtin_fmaf(A[i][v], c[v], b[i][v]);
            }
            y[v] = p.in(i) ? gate(y[v]) * at : 0.f;
        }
        if (p.on && p.s0 + i < a.T) put_from<T, VEC>(h.at(a, p, i, a.H, 0, false), y, p.skip, a.whole);
    }
    if constexpr (GROUPS == 1) {
        if (a.last && p.on) {
#pragma unroll
            for (int v = 0; v < VEC; ++v)
                if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = c[v];
        }
    }
}

// A thread's kSteps steps backwards: its gates, u as kept, and dh (u = g = o = d = 0 at steps that are none of the sequence's)
template <int VEC> struct Back {
    float u[kSteps][VEC], g[kSteps][VEC], o[kSteps][VEC], d[kSteps][VEC];
    template <bool FULL, typename T, typename P>
    __device__ __forceinline__ void load(const ScanArgs &a, const P &p, const Row<const T, FULL> &G, const Row<const T, FULL> &dh) {
        Lanes<T, VEC> x[kSteps][3], up[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G.at(a, p, i, 3 * a.H, k * a.H, true));
            up[i].load(dh.at(a, p, i, a.H, 0, true));
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = FULL || p.in(i);
            float y[VEC];
            x[i][0].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[i][v] = in ? Forget::pack(y[v]) : 0.f;
            x[i][1].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) g[i][v] = in ? candidate(y[v]) : 0.f;
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) o[i][v] = in ? gate(y[v]) : 0.f;
            up[i].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) d[i][v] = in ? y[v] : 0.f;
        }
    }
    // the maps of the state, forwards, and of q, backwards, which share the factor
    __device__ __forceinline__ void maps(int v, float &A, float &b, float &R) const {
        A = 1.f, b = 0.f, R = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const Forget at(u[i][v]);
            b = __builtin_fmaf(at.f(), b, at.u() * g[i][v]);
            A *= at.f();
            const int k = kSteps - 1 - i;
            R = Forget(u[k][v]).f() * __builtin_fmaf(d[k][v], o[k][v], R);
        }
    }
    // dG from the state in front of the thread's steps and the q behind them; q: that in front of them
    template <bool FULL, typename T, typename P>
    __device__ __forceinline__ void store(const ScanArgs &a, const P &p, const Row<T, FULL> &dG, float (&c)[VEC], float (&q)[VEC]) const {
        float before[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                before[i][v] = c[v];
                c[v] = Forget(u[i][v]).step(c[v], g[i][v]);
            }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = kSteps - 1 - k;
            float df[VEC], dg[VEC], dout[VEC];
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float r = __builtin_fmaf(d[i][v], o[i][v], q[v]);
                const Forget k(u[i][v]);
                const float part = r * k.least, rest = r - part, ru = k.f_least ? rest : part;
                df[v] = __builtin_fmaf(-part, k.least, part) * (before[i][v] - g[i][v]);
                dg[v] = ru * __builtin_fmaf(-g[i][v], g[i][v], 1.f);
                dout[v] = d[i][v] * c[v] * __builtin_fmaf(-o[i][v], o[i][v], o[i][v]);
                c[v] = before[i][v];
                q[v] = k.f_least ? part : rest;
            }
            if (p.on && (FULL || p.s0 + i < a.T)) {
                put_from<T, VEC>(dG.at(a, p, i, 3 * a.H, 0, false), df, p.skip, a.whole);
                put_from<T, VEC>(dG.at(a, p, i, 3 * a.H, a.H, false), dg, p.skip, a.whole);
                put_from<T, VEC>(dG.at(a, p, i, 3 * a.H, 2 * a.H, false), dout, p.skip, a.whole);
            }
        }
    }
};

template <typename T, int VEC, int GROUPS>
__global__ __launch_bounds__(kThreads<GROUPS>, 4) void k_scan_bwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    constexpr int ALL = P::SUBS * GROUPS, W = GROUPS / 4, WS = W > 1 ? W : 1;
    __shared__ float s_a[ALL][P::WIDTH], s_b[ALL][P::WIDTH], s_r[ALL][P::WIDTH], s_wa[WS][P::WIDTH], s_wb[WS][P::WIDTH], s_wr[WS][P::WIDTH];
    const int w = wave_id(), own = threadIdx.x >> 4;       // the thread's group in the block
    const long long first_chain = a.chain0 + (long long)blockIdx.x * P::SUBS;
    const P p(a, first_chain, 0);
    const Folder<VEC> f = wave_folder<VEC, GROUPS>(a, first_chain);
    float state = GROUPS > 1 ? a.states[f.row] : 0.f, back = GROUPS > 1 && a.first ? a.first[f.row] : 0.f;
    Back<VEC> x;
    x.template load<false, T>(a, p, Row<const T, false>(a, a.G, 3 * a.H, p, 0), Row<const T, false>(a, a.dh, a.H, p, 0));
    float c[VEC], q[VEC], dc0[VEC];
    if constexpr (GROUPS == 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            c[v] = a.states[(size_t)p.b * a.H + p.ch + v];
            q[v] = a.first ? a.first[(size_t)p.b * a.H + p.ch + v] : 0.f;
            // dc0 by the steps' map, as it is of longer sequences
            float A, b, R;
            x.maps(v, A, b, R);
            dc0[v] = __builtin_fmaf(A, q[v], R);
        }
    } else {
#pragma unroll
        for (int v = 0; v < VEC; ++v) x.maps(v, s_a[own][p.slot + v], s_b[own][p.slot + v], s_r[own][p.slot + v]);
        settle();
        FourMaps<P::WIDTH, false> m;
        FourMaps<P::WIDTH, true> r;
        m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
        r.read(s_a + 4 * w, s_r + 4 * w, f.lane);
        if constexpr (W > 1) {
            float all, sum, rest;
            m.total(all, sum);
            r.total(all, rest);
            if (f.on) s_wa[w][f.lane] = all, s_wb[w][f.lane] = sum, s_wr[w][f.lane] = rest;
            here(back);                                    // (as in the forward pass: dc0 may be dc_last)
            lds_barrier();
            WaveMaps<P::WIDTH, W, false> wm;
            wm.read(s_wa, s_wb, f.lane);
            state = wm.state(state, w);
            WaveMaps<P::WIDTH, W, true> wr;
            wr.read(s_wa, s_wr, f.lane);
            back = wr.state(back, w);
        }
        if (f.on) {
            m.write(s_b + 4 * w, f.lane, state);
            back = r.write(s_r + 4 * w, f.lane, back);
        }
        if (a.last && f.own && w % W == 0) a.last[f.row] = back;
        settle();
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            c[v] = s_b[own][p.slot + v];
            q[v] = s_r[own][p.slot + v];
        }
    }
    x.template store<false, T>(a, p, Row<T, false>(a, a.out, 3 * a.H, p, 0), c, q);
    if constexpr (GROUPS == 1) {
        if (a.last && p.on) {
#pragma unroll
            for (int v = 0; v < VEC; ++v)
                if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = dc0[v];
        }
    }
}

// ---- chains of chunks -----------------------------------------------------------------------------------------------------------
// The chunks of a sequence's channels are a chain, up to the one that holds its last step: each hands the state behind it to the next.  A chunk publishes its map
// (A, b) as soon as it has it, and the state behind it (C) as soon as it knows the one in front of it; the next one takes C from the chunk in front, or from one up
// to kLookBack in front and applies the maps of those between, in order, with the same operation that each of them applies to its own: results do not
// depend on how far it looked.  Map and state go out in one 64-bit word, b or C below and above it A, which is 0 to 1 and leaves the upper two bits for
// what it is (A that is NaN comes with a b that is), so that nothing has to be waited for in between; the words are cleared in front of the launch.
// Units are taken by ticket, chunk after chunk: whoever waits, waits for a unit that has been taken already and waits for lower tickets only.  The chains are
// dealt to up to kQueues queues with a ticket counter and blocks each: one counter for all gives out a ticket every 15 to 20 ns, no matter who asks
// (4 x 16384 x 1280 bf16, forward: 181 us of 10240 tickets).
struct Queue {
    unsigned *ticket;
    unsigned first, chains;          // chain; neighbours are one queue's, and with it one XCD's: they share cache lines where rows are not whole ones
    __device__ __forceinline__ Queue(const ScanArgs &a) {
        const int q = (int)(blockIdx.x % (unsigned)a.queues);
        ticket = reinterpret_cast<unsigned *>(a.tickets + q * kTicketStride);
        first = (unsigned)(a.chains * q / a.queues);
        chains = (unsigned)(a.chains * (q + 1) / a.queues) - first;
    }
    __device__ __forceinline__ unsigned take() const { return atomicAdd(ticket, 1u); }          // one lane's
};
typedef unsigned long long Word;
constexpr Word kMapMark = 1ull << 62, kStateMark = 1ull << 63;
__device__ __forceinline__ Word map_word(float A, float b) {
    return kMapMark | (Word)(__float_as_uint(A) & 0x3fffffffu) << 32 | __float_as_uint(b);
}
__device__ __forceinline__ Word state_word(float c) { return kStateMark | __float_as_uint(c); }
__device__ __forceinline__ float factor_of(Word w) { return __uint_as_float((unsigned)(w >> 32) & 0x3fffffffu); }
__device__ __forceinline__ float value_of(Word w) { return __uint_as_float((unsigned)w); }

// From the marks of the chunks in front (bit d: the one d + 1 in front): the nearest whose state is there while the maps of all nearer ones are, or -1
__device__ __forceinline__ int nearest_state(unsigned states, unsigned maps) {
    if (states == 0) return -1;
    const int d = __builtin_ctz(states);
    return (~maps & ((1u << d) - 1)) == 0 ? d : -1;
}

// How a block gets the state in front of its chunk.  One wave, a lane per channel, publishes the map and looks at the nearest four chunks; if they do not
// tell, all eight waves look at four each, as often as it takes.
constexpr int kLookBack = 32, kLookWaves = kThreads<kChunkGroups> / 64;
template <int WIDTH> struct Chain {
    float s_factor[kLookBack][WIDTH], s_value[kLookBack][WIDTH];
    unsigned s_marks[kLookWaves];
    int s_from;                      // -1: not known yet

    // words d0 + 1 .. d0 + 4 in front; bit d of the marks: states, bit 4 + d: maps.  back: words from a chunk's to those of the one in front
    static __device__ __forceinline__ unsigned look(const Word *unit, int lane, long long back, int d0, int ahead, Word (&w)[4]) {
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] = load_agent(unit - (min(d0 + d, ahead - 1) + 1) * back + lane);
        unsigned marks = 0;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if (d0 + d >= ahead) break;
            if (__all((w[d] & kStateMark) != 0)) marks |= 1u << d;
            if (__all((w[d] & kMapMark) != 0)) marks |= 16u << d;
        }
        return marks;
    }
    // The word of the chunk in front, requested early: in the middle of a long chain it has the state by the time it is wanted
    static __device__ __forceinline__ Word early(const Word *unit, int lane, long long back, int ahead) {
        return ahead > 0 ? load_agent(unit - back + lane) : 0;
    }
    // The wave's first look; `carry` is what it gives where it returns true.
    static __device__ __forceinline__ bool first_look(Word *unit, int lane, long long back, int ahead, Word front, float A, float b, float &carry) {
        if (ahead == 0) return true;
        if (__all((front & kStateMark) != 0)) {
            carry = value_of(front);
            return true;
        }
        store_agent(unit + lane, map_word(A, b));
        Word w[4];
        const unsigned marks = look(unit, lane, back, 0, ahead, w);
        const int from = nearest_state(marks & 15u, marks >> 4);
        if (from < 0) return false;
#pragma unroll
        for (int d = 3; d >= 0; --d) {
            if (d == from) carry = value_of(w[d]);
            else if (d < from) carry = __builtin_fmaf(factor_of(w[d]), carry, value_of(w[d]));
        }
        return true;
    }
    // All waves: until it is known.  The values are in LDS then.
    __device__ __forceinline__ int look_on(const Word *unit, long long back, int ahead) {
        const int lane = lane_id(), w = wave_id();
        const long long t0 = wall_clock64();
        for (;;) {
            unsigned marks = 0;
            if (lane < WIDTH && 4 * w < ahead) {
                Word x[4];
                marks = look(unit, lane, back, 4 * w, ahead, x);
#pragma unroll
                for (int d = 0; d < 4; ++d) s_factor[4 * w + d][lane] = factor_of(x[d]), s_value[4 * w + d][lane] = value_of(x[d]);
            }
            // (a chunk that never hands on is given up after kSpinLimitTicks: NaN makes the failure visible)
            if (w == 0 && wall_clock64() - t0 > kSpinLimitTicks) {
                marks |= 256u;
            }
            if (lane == 0) s_marks[w] = marks;
            lds_barrier();
            unsigned states = 0, maps = 0, end = 0;
#pragma unroll
            for (int k = 0; k < kLookWaves; ++k) {
                const unsigned m = s_marks[k];
                states |= (m & 15u) << 4 * k;
                maps |= (m >> 4 & 15u) << 4 * k;
                end |= m >> 8;
            }
            const int from = __builtin_amdgcn_readfirstlane(end ? kLookBack : nearest_state(states, maps));
            if (from >= 0) return from;
            lds_barrier();                                 // before they are written again
        }
    }
    __device__ __forceinline__ float carry_from(int lane, int from) const {
        if (from >= kLookBack) return __builtin_nanf("");
        float carry = s_value[from][lane];
        for (int d = from - 1; d >= 0; --d) carry = __builtin_fmaf(s_factor[d][lane], carry, s_value[d][lane]);
        return carry;
    }
    static __device__ __forceinline__ void hand_on(Word *unit, int lane, float A, float carry, float b) {
        store_agent(unit + lane, state_word(__builtin_fmaf(factor_of(map_word(A, b)), carry, b)));
    }
};

__global__ __launch_bounds__(256) void k_scan_clear(u32x4_any *p, long long n) {
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) p[i] = u32x4_any{0u, 0u, 0u, 0u};
}

// A unit of a chain, the same for the whole block
struct Unit {
    int b, g, n, chunk, last;        // last: the chunk of the sequence's last step
    unsigned chain;
    bool there;
    __device__ __forceinline__ Unit(const ScanArgs &a, const Queue &queue, unsigned ticket, bool backwards) {
        const unsigned turn = ticket / queue.chains;
        chain = queue.first + (ticket - turn * queue.chains);
        there = turn < (unsigned)a.chunks;
        chunk = backwards ? a.chunks - 1 - (int)turn : (int)turn;          // backwards from the last one on
        b = (int)(chain / (unsigned)a.groups_h);
        g = (int)(chain - (unsigned)b * (unsigned)a.groups_h);
        n = there ? a.len ? clamp_len(a.len[b], a.T) : a.T : 0;
        last = n > 0 ? (n - 1) / ECHO_SCAN_CHUNK : 0;
    }
    __device__ __forceinline__ bool full() const { return (chunk + 1) * ECHO_SCAN_CHUNK <= n; }
};

template <typename T, int VEC> struct FwdChain {
    static constexpr int GROUPS = kChunkGroups, WIDTH = 16 * VEC;
    typedef Place<VEC, GROUPS> P;
    static constexpr int W = GROUPS / 4;
    float s_a[GROUPS][WIDTH], s_b[GROUPS][WIDTH], s_wa[2][W][WIDTH], s_wb[2][W][WIDTH], s_carry[2][WIDTH];
    Chain<WIDTH> chain;
    int s_known[2];

    template <bool FULL> __device__ __forceinline__ void run(const ScanArgs &a, const Queue &queue, Unit &unit, int buf, unsigned *s_ticket) {
        unsigned next = 0;
        if (threadIdx.x == kThreads<GROUPS> - 64) next = queue.take();
        const P p(a, unit.b, unit.g, unit.n, unit.chunk);
        Word *words = a.words + ((long long)unit.chunk * a.chains + unit.chain) * WIDTH;
        const long long back = a.chains * WIDTH;
        const Folder<VEC> f(a, unit.b, unit.g, true);
        const int w = wave_id();
        const Word front = w == 0 ? Chain<WIDTH>::early(words, f.lane, back, unit.chunk) : 0;
        const Row<const T, FULL> G(a, a.G, 3 * a.H, p, unit.chunk);
        Lanes<T, VEC> x[kSteps][3];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G.at(a, p, i, 3 * a.H, k * a.H, true));
        float A[kSteps][VEC], b[kSteps][VEC];              // the maps of the thread's first steps
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC], z[VEC];
            x[i][0].get(y);
            x[i][1].get(z);
#pragma unroll
            for (int v = 0; v < VEC; ++v) add_step(A, b, i, v, y[v], candidate(z[v]), FULL || p.in(i));
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            s_a[p.group][p.slot + v] = A[kSteps - 1][v];
            s_b[p.group][p.slot + v] = b[kSteps - 1][v];
        }
        float carry = w == 0 && unit.chunk == 0 && a.first ? a.first[f.row] : 0.f;
        settle();
        // (what is read from LDS here is read again behind the barriers: there are no registers to keep it)
        float all, sum;
        {
            FourMaps<WIDTH, false> m;
            m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
            m.total(all, sum);
        }
        if (f.on) s_wa[buf][w][f.lane] = all, s_wb[buf][w][f.lane] = sum;
        lds_barrier();
        if (w == 0) {
            WaveMaps<WIDTH, W, false> wm;
            wm.read(s_wa[buf], s_wb[buf], f.lane);
            wm.total(all, sum);
        }
        const auto finish = [&]() __attribute__((always_inline)) {
            if (unit.chunk < unit.last) Chain<WIDTH>::hand_on(words, f.lane, all, carry, sum);
            s_carry[buf][f.lane] = carry;
            if (a.states && f.own) a.states[((size_t)unit.b * a.chunks + unit.chunk) * a.H + f.ch] = carry;
        };
        if (w == 0 && f.on) {
            const bool known = Chain<WIDTH>::first_look(words, f.lane, back, unit.chunk, front, all, sum, carry);
            if (known) finish();
            if (f.lane == 0) s_known[buf] = known;
        }
        if (threadIdx.x == kThreads<GROUPS> - 64) s_ticket[buf] = next;
        lds_barrier();
        if (!__builtin_amdgcn_readfirstlane(s_known[buf])) {
            const int from = chain.look_on(words, back, unit.chunk);
            if (w == 0 && f.on) {
                carry = chain.carry_from(f.lane, from);
                finish();
            }
            lds_barrier();
        }
        if (f.on) {
            WaveMaps<WIDTH, W, false> wm;
            wm.read(s_wa[buf], s_wb[buf], f.lane);
            FourMaps<WIDTH, false> m;
            m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
            const float end = m.write(s_b + 4 * w, f.lane, wm.state(s_carry[buf][f.lane], w));
            if (a.last && f.own && unit.chunk == unit.last && w == W - 1) a.last[f.row] = end;
        }
        settle();
        const Row<T, FULL> h(a, a.out, a.H, p, unit.chunk);
        unit = Unit(a, queue, __builtin_amdgcn_readfirstlane(s_ticket[buf]), false);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC];
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float c = __builtin_fmaf(A[i][v], s_b[p.group][p.slot + v], b[i][v]);
                y[v] = FULL || p.in(i) ? gate(y[v]) * c : 0.f;
            }
            if (p.on && (FULL || p.s0 + i < a.T)) put_from<T, VEC>(h.at(a, p, i, a.H, 0, false), y, p.skip, a.whole);
        }
    }
};

template <typename T, int VEC> struct BwdChain {
    static constexpr int GROUPS = kChunkGroups, WIDTH = 16 * VEC;
    typedef Place<VEC, GROUPS> P;
    static constexpr int W = GROUPS / 4;
    float s_a[GROUPS][WIDTH], s_b[GROUPS][WIDTH], s_r[GROUPS][WIDTH], s_wa[2][W][WIDTH], s_wb[2][W][WIDTH], s_wr[2][W][WIDTH], s_carry[2][WIDTH];
    Chain<WIDTH> chain;
    int s_known[2];

    template <bool FULL> __device__ __forceinline__ void run(const ScanArgs &a, const Queue &queue, Unit &unit, int buf, unsigned *s_ticket) {
        unsigned next = 0;
        if (threadIdx.x == kThreads<GROUPS> - 64) next = queue.take();
        const P p(a, unit.b, unit.g, unit.n, unit.chunk);
        const int w = wave_id(), link = unit.last - unit.chunk;                // links from the last chunk on
        Word *words = a.words + ((long long)unit.chunk * a.chains + unit.chain) * WIDTH;
        const long long back = -a.chains * WIDTH;
        const Folder<VEC> f(a, unit.b, unit.g, true);
        Back<VEC> x;
        x.template load<FULL, T>(a, p, Row<const T, FULL>(a, a.G, 3 * a.H, p, unit.chunk), Row<const T, FULL>(a, a.dh, a.H, p, unit.chunk));
#pragma unroll
        for (int v = 0; v < VEC; ++v) x.maps(v, s_a[p.group][p.slot + v], s_b[p.group][p.slot + v], s_r[p.group][p.slot + v]);
        settle();
        float all, sum;
        {
            FourMaps<WIDTH, false> m;
            m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
            m.total(all, sum);
        }
        if (f.on) s_wa[buf][w][f.lane] = all, s_wb[buf][w][f.lane] = sum;
        {
            FourMaps<WIDTH, true> r;
            r.read(s_a + 4 * w, s_r + 4 * w, f.lane);
            r.total(all, sum);
        }
        if (f.on) s_wr[buf][w][f.lane] = sum;
        const float state = a.states[((size_t)unit.b * a.chunks + unit.chunk) * a.H + f.ch];      // (wanted behind the barrier)
        float carry = 0.f;
        lds_barrier();
        const auto finish = [&]() __attribute__((always_inline)) {
            if (unit.chunk > 0) Chain<WIDTH>::hand_on(words, f.lane, all, carry, sum);
            s_carry[buf][f.lane] = carry;
        };
        if (w == 0 && f.on) {
            if (link == 0 && a.first) carry = a.first[f.row];
            WaveMaps<WIDTH, W, true> wr;
            wr.read(s_wa[buf], s_wr[buf], f.lane);
            wr.total(all, sum);
            const bool known = Chain<WIDTH>::first_look(words, f.lane, back, link, 0, all, sum, carry);
            if (known) finish();
            if (f.lane == 0) s_known[buf] = known;
        }
        // the states in front of the groups meanwhile
        if (f.on) {
            WaveMaps<WIDTH, W, false> wm;
            wm.read(s_wa[buf], s_wb[buf], f.lane);
            FourMaps<WIDTH, false> m;
            m.read(s_a + 4 * w, s_b + 4 * w, f.lane);
            m.write(s_b + 4 * w, f.lane, wm.state(state, w));
        }
        if (threadIdx.x == kThreads<GROUPS> - 64) s_ticket[buf] = next;
        lds_barrier();
        if (!__builtin_amdgcn_readfirstlane(s_known[buf])) {
            const int from = chain.look_on(words, back, link);
            if (w == 0 && f.on) {
                carry = chain.carry_from(f.lane, from);
                finish();
            }
            lds_barrier();
        }
        if (f.on) {
            WaveMaps<WIDTH, W, true> wr;
            wr.read(s_wa[buf], s_wr[buf], f.lane);
            FourMaps<WIDTH, true> r;
            r.read(s_a + 4 * w, s_r + 4 * w, f.lane);
            const float end = r.write(s_r + 4 * w, f.lane, wr.state(s_carry[buf][f.lane], w));
            if (a.last && f.own && unit.chunk == 0 && w == 0) a.last[f.row] = end;
        }
        settle();
        float c[VEC], q[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            c[v] = s_b[p.group][p.slot + v];
            q[v] = s_r[p.group][p.slot + v];
        }
        const Row<T, FULL> dG(a, a.out, 3 * a.H, p, unit.chunk);
        x.template store<FULL, T>(a, p, dG, c, q);
        unit = Unit(a, queue, __builtin_amdgcn_readfirstlane(s_ticket[buf]), true);
    }
};

// Positions behind a sequence's end, a whole chunk of them
template <typename T, int VEC> __device__ __forceinline__ void put_zeros(const ScanArgs &a, int b, int g, int n, int chunk, int arrays) {
    const Place<VEC, kChunkGroups> p(a, b, g, n, chunk);
    const Row<T, false> out(a, a.out, arrays * a.H, p, chunk);
    float zero[VEC] = {};
#pragma unroll
    for (int v = 0; v < VEC; ++v) asm volatile("" : "+v"(zero[v]));           // (made here: in front of the loop over the units they would hold registers)
    for (int i = 0; i < kSteps; ++i)
        for (int k = 0; k < arrays; ++k)
            if (p.on && p.s0 + i < a.T) put_from<T, VEC>(out.at(a, p, i, arrays * a.H, k * a.H, false), zero, p.skip, a.whole);
}

template <typename T, int VEC, bool BWD>
__global__ __launch_bounds__(kThreads<kChunkGroups>, 4) void k_scan_chain(const ScanArgs a) {
    __shared__ std::conditional_t<BWD, BwdChain<T, VEC>, FwdChain<T, VEC>> s;
    __shared__ unsigned s_ticket[2];
    constexpr int THREADS = kThreads<kChunkGroups>;
    const Queue queue(a);
    if (threadIdx.x == 0) s_ticket[1] = queue.take();
    __syncthreads();
    Unit unit(a, queue, __builtin_amdgcn_readfirstlane(s_ticket[1]), BWD);
    for (int buf = 0; unit.there; buf ^= 1) {
        if (unit.chunk > unit.last) {
            if (threadIdx.x == THREADS - 64) s_ticket[buf] = queue.take();
            put_zeros<T, VEC>(a, unit.b, unit.g, unit.n, unit.chunk, BWD ? 3 : 1);
            lds_barrier();
            unit = Unit(a, queue, __builtin_amdgcn_readfirstlane(s_ticket[buf]), BWD);
        } else if (unit.full()) {
            s.template run<true>(a, queue, unit, buf, s_ticket);
        } else {
            s.template run<false>(a, queue, unit, buf, s_ticket);
        }
    }
}

// ---- chains that are a block's ---------------------------------------------------------------------------------------------
// A short chain, or one of so many that they keep all compute units busy to the end, is better off with one block for all of its chunks: the state stays in LDS,
// nothing is cleared and nobody looks at others' words.  Chain of blocks / blocks' chains, us, forward and backward:
//   two chunks: 1 x 200 x 1024 bf16 8.8 / 8.1 and 11.3 / 11.1, 16 x 200 x 1024 bf16 12.4 / 10.2 and 15.6 / 13.9 (f32 16.3 / 13.4 and 24.1 / 23.7), 128 x 200 x 1024 bf16
//     58 / 47 and 96 / 82
//   three and four, 512 chains and more, a multiple of 256 or little less: 32 x 300 x 1022 bf16 28.4 / 22.2 and 43.6 / 36.6, 64 x 300 x 512 f32 36.6 / 34.4 and 61.6 / 56.8,
//     128 x 500 x 1024 f32 188 / 171 and 328 / 320; a few chains more than that: 33 x 500 x 1024 bf16 34 / 36 and 55 / 59
//   three and four, 256 chains: 16 x 500 x 1024 bf16 20.8 / 19.2 and 30.7 / 31.3, f32 28.6 / 26.9 and 48.4 / 45.9: one of the four is slower, so they are left out; 128
//     chains: 8 x 500 x 1024 bf16 12.5 / 14.5 and 16.7 / 22.2
//   more chunks: 32 x 1000 x 1024 bf16 59 / 53 and 101 / 100; of unequal length 64 x 2000 x 512 f32 159 / 163 and 301 / 314
// (The next chunk's gates requested while this one's maps are folded: 17 registers in memory with bf16 gates, 22 -> 30.5 us of 32 x 300 x 1022.)
static bool walks(long long chains, int chunks) {
    if (chunks < 2 || chains > 1 << 22) return false;      // (a grid has fewer than 2^32 threads)
    if (chunks == 2) return true;
    return chunks <= 4 && chains >= 512 && (chains + 255) / 256 * 256 <= chains + chains / 16;
}
template <bool BWD> struct Walk {
    int b, g, n, last, chunk;
    bool there;
    __device__ __forceinline__ explicit Walk(const ScanArgs &a) {
        // neighbours are one XCD's
        const int q = (int)(blockIdx.x % kXcds);
        const unsigned first = (unsigned)(a.chains * q / kXcds), chain = first + blockIdx.x / kXcds;
        there = chain < (unsigned)(a.chains * (q + 1) / kXcds);
        b = (int)(chain / (unsigned)a.groups_h);
        g = (int)(chain - (unsigned)b * (unsigned)a.groups_h);
        n = there && a.len ? clamp_len(a.len[b], a.T) : a.T;
        last = n > 0 ? (n - 1) / ECHO_SCAN_CHUNK : 0;
        chunk = BWD ? last : 0;
    }
    __device__ __forceinline__ bool full(int c) const { return (c + 1) * ECHO_SCAN_CHUNK <= n; }
};

template <typename T, int VEC> struct FwdWalk {
    static constexpr int GROUPS = kChunkGroups, WIDTH = 16 * VEC, W = GROUPS / 4;
    typedef Place<VEC, GROUPS> P;
    struct Shared { float a[GROUPS][WIDTH], b[GROUPS][WIDTH], wa[2][W][WIDTH], wb[2][W][WIDTH], carry[2][WIDTH]; };
    template <bool FULL> static __device__ __forceinline__ void run(const ScanArgs &a, const Walk<false> &k, int buf, Shared &s) {
        const P p(a, k.b, k.g, k.n, k.chunk);
        const Folder<VEC> f(a, k.b, k.g, true);
        const int w = wave_id();
        const Row<const T, FULL> G(a, a.G, 3 * a.H, p, k.chunk);
        Lanes<T, VEC> x[kSteps][3];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int j = 0; j < 3; ++j) x[i][j].load(G.at(a, p, i, 3 * a.H, j * a.H, true));
        float A[kSteps][VEC], b[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC], z[VEC];
            x[i][0].get(y);
            x[i][1].get(z);
#pragma unroll
            for (int v = 0; v < VEC; ++v) add_step(A, b, i, v, y[v], candidate(z[v]), FULL || p.in(i));
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            s.a[p.group][p.slot + v] = A[kSteps - 1][v];
            s.b[p.group][p.slot + v] = b[kSteps - 1][v];
        }
        settle();
        {
            float all, sum;
            FourMaps<WIDTH, false> m;
            m.read(s.a + 4 * w, s.b + 4 * w, f.lane);
            m.total(all, sum);
            if (f.on) s.wa[buf][w][f.lane] = all, s.wb[buf][w][f.lane] = sum;
        }
        lds_barrier();
        if (f.on) {
            WaveMaps<WIDTH, W, false> wm;
            wm.read(s.wa[buf], s.wb[buf], f.lane);
            FourMaps<WIDTH, false> m;
            m.read(s.a + 4 * w, s.b + 4 * w, f.lane);
            const float state = wm.state(s.carry[buf][f.lane], w), end = m.write(s.b + 4 * w, f.lane, state);
            if (w == 0 && a.states && f.own) a.states[((size_t)k.b * a.chunks + k.chunk) * a.H + f.ch] = state;
            if (w == W - 1) {
                s.carry[buf ^ 1][f.lane] = end;
                if (a.last && f.own && k.chunk == k.last) a.last[f.row] = end;
            }
        }
        settle();
        const Row<T, FULL> h(a, a.out, a.H, p, k.chunk);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC];
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float c = __builtin_fmaf(A[i][v], s.b[p.group][p.slot + v], b[i][v]);
                y[v] = FULL || p.in(i) ? gate(y[v]) * c : 0.f;
            }
            if (p.on && (FULL || p.s0 + i < a.T)) put_from<T, VEC>(h.at(a, p, i, a.H, 0, false), y, p.skip, a.whole);
        }
    }
};

template <typename T, int VEC> __global__ __launch_bounds__(kThreads<kChunkGroups>, 4) void k_scan_fwd_walk(const ScanArgs a) {
    typedef FwdWalk<T, VEC> F;
    __shared__ typename F::Shared s;
    Walk<false> k(a);
    if (!k.there) return;
    const Folder<VEC> f(a, k.b, k.g, true);
    if (wave_id() == 0 && f.on) s.carry[0][f.lane] = a.first ? a.first[f.row] : 0.f;
    for (int buf = 0; k.chunk <= k.last; ++k.chunk, buf ^= 1) {
        if (k.full(k.chunk)) F::template run<true>(a, k, buf, s);
        else F::template run<false>(a, k, buf, s);
    }
    for (; k.chunk < a.chunks; ++k.chunk) put_zeros<T, VEC>(a, k.b, k.g, k.n, k.chunk, 1);
}

template <typename T, int VEC> struct BwdWalk {
    static constexpr int GROUPS = kChunkGroups, WIDTH = 16 * VEC, W = GROUPS / 4;
    typedef Place<VEC, GROUPS> P;
    struct Shared { float a[GROUPS][WIDTH], b[GROUPS][WIDTH], r[GROUPS][WIDTH], wa[2][W][WIDTH], wb[2][W][WIDTH], wr[2][W][WIDTH], carry[2][WIDTH]; };
    template <bool FULL> static __device__ __forceinline__ void run(const ScanArgs &a, const Walk<true> &k, int buf, Shared &s) {
        const P p(a, k.b, k.g, k.n, k.chunk);
        const Folder<VEC> f(a, k.b, k.g, true);
        const int w = wave_id();
        Back<VEC> x;
        const float first = a.states[((size_t)k.b * a.chunks + k.chunk) * a.H + f.ch];
        x.template load<FULL, T>(a, p, Row<const T, FULL>(a, a.G, 3 * a.H, p, k.chunk), Row<const T, FULL>(a, a.dh, a.H, p, k.chunk));
#pragma unroll
        for (int v = 0; v < VEC; ++v) x.maps(v, s.a[p.group][p.slot + v], s.b[p.group][p.slot + v], s.r[p.group][p.slot + v]);
        settle();
        {
            float all, sum, rest;
            FourMaps<WIDTH, false> m;
            m.read(s.a + 4 * w, s.b + 4 * w, f.lane);
            m.total(all, sum);
            FourMaps<WIDTH, true> r;
            r.read(s.a + 4 * w, s.r + 4 * w, f.lane);
            r.total(all, rest);
            if (f.on) s.wa[buf][w][f.lane] = all, s.wb[buf][w][f.lane] = sum, s.wr[buf][w][f.lane] = rest;
        }
        lds_barrier();
        if (f.on) {
            {
                WaveMaps<WIDTH, W, false> wm;
                wm.read(s.wa[buf], s.wb[buf], f.lane);
                FourMaps<WIDTH, false> m;
                m.read(s.a + 4 * w, s.b + 4 * w, f.lane);
                m.write(s.b + 4 * w, f.lane, wm.state(first, w));
            }
            WaveMaps<WIDTH, W, true> wr;
            wr.read(s.wa[buf], s.wr[buf], f.lane);
            FourMaps<WIDTH, true> r;
            r.read(s.a + 4 * w, s.r + 4 * w, f.lane);
            const float end = r.write(s.r + 4 * w, f.lane, wr.state(s.carry[buf][f.lane], w));
            if (w == 0) {
                s.carry[buf ^ 1][f.lane] = end;
                if (a.last && f.own && k.chunk == 0) a.last[f.row] = end;
            }
        }
        settle();
        float c[VEC], q[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            c[v] = s.b[p.group][p.slot + v];
            q[v] = s.r[p.group][p.slot + v];
        }
        x.template store<FULL, T>(a, p, Row<T, FULL>(a, a.out, 3 * a.H, p, k.chunk), c, q);
    }
};

template <typename T, int VEC> __global__ __launch_bounds__(kThreads<kChunkGroups>, 4) void k_scan_bwd_walk(const ScanArgs a) {
    typedef BwdWalk<T, VEC> B;
    __shared__ typename B::Shared s;
    Walk<true> k(a);
    if (!k.there) return;
    const Folder<VEC> f(a, k.b, k.g, true);
    if (wave_id() == 0 && f.on) s.carry[0][f.lane] = a.first ? a.first[f.row] : 0.f;
    for (int buf = 0; k.chunk >= 0; --k.chunk, buf ^= 1) {
        if (k.full(k.chunk)) B::template run<true>(a, k, buf, s);
        else B::template run<false>(a, k, buf, s);
    }
    for (int chunk = k.last + 1; chunk < a.chunks; ++chunk) put_zeros<T, VEC>(a, k.b, k.g, k.n, chunk, 3);
}

static echo_status_t check_scan(const echo_scan_desc_t *d) {
    if (!d) return ECHO_ERR_NULL;
    if (d->dtype != ECHO_F32 && d->dtype != ECHO_BF16) return ECHO_ERR_DTYPE;
    if (d->B < 1 || d->T < 1 || d->H < 1 || d->B > ECHO_SCAN_MAX_ROWS || d->T > ECHO_SCAN_MAX_ROWS || d->H > ECHO_SCAN_MAX_H) return ECHO_ERR_SHAPE;
    // (B T fits 64 bits, B T H may not)
    if ((d->reverse != 0 && d->reverse != 1) || (size_t)d->B * d->T > ((size_t)1 << 40) / d->H) return ECHO_ERR_SHAPE;
    return ECHO_OK;
}
static size_t scan_chunks(const echo_scan_desc_t &d) { return ((size_t)d.T + ECHO_SCAN_CHUNK - 1) / ECHO_SCAN_CHUNK; }

static bool unaligned_scan(std::initializer_list<const void *> ps) {
    uintptr_t m = 0;
    for (const void *p : ps) m |= (uintptr_t)p;
    return (m & 15u) != 0;
}

// Words and tickets of the chains.  Nothing where all steps are one chunk's, or a chain is one block's.
struct ScanPlan {
    int vec, groups_h, chunks;
    long long chains;
    int queues;
    size_t bytes;
};
static ScanPlan scan_plan(const echo_scan_desc_t &d) {
    ScanPlan p{};
    p.vec = d.H < 4 ? 1 : 4;
    p.groups_h = (d.H + 16 * p.vec - 1) / (16 * p.vec);
    p.chunks = (int)scan_chunks(d);
    p.chains = (long long)d.B * p.groups_h;
    if (p.chunks > 1 && !walks(p.chains, p.chunks)) {
        p.bytes = kQueues * kTicketStride * 8 + (size_t)p.chains * p.chunks * 16 * p.vec * 8;
        // as many queues as there are chains, or a number up to kQueues that deals them out evenly
        long long least = p.chains * 2;
        for (int q = (int)std::min<long long>(p.chains, kQueues); q > (int)std::min<long long>(p.chains, kQueues) / 2; --q) {
            const long long most = (p.chains + q - 1) / q * q;
            if (most < least) least = most, p.queues = q;
        }
    }
    return p;
}

template <typename T, int VEC, int GROUPS> static echo_status_t launch_scan(ScanArgs a, bool bwd, hipStream_t st) {
    constexpr int SUBS = Place<VEC, GROUPS>::SUBS;
    constexpr long long MOST = 1 << 22;                    // blocks of a launch: a grid has fewer than 2^32 threads
    for (; a.chain0 < a.chains; a.chain0 += MOST * SUBS) {
        const unsigned blocks = (unsigned)std::min(MOST, (a.chains - a.chain0 + SUBS - 1) / SUBS);
        LaunchRecord r = launch_begin(bwd ? "scan_bwd" : "scan_fwd", st);
        if (bwd) k_scan_bwd<T, VEC, GROUPS><<<blocks, kThreads<GROUPS>, 0, st>>>(a);
        else k_scan_fwd<T, VEC, GROUPS><<<blocks, kThreads<GROUPS>, 0, st>>>(a);
        if (echo_status_t s = launch_end(r)) return s;
    }
    return ECHO_OK;
}
template <typename T, int VEC> static echo_status_t launch_scan(const ScanArgs &a, bool bwd, hipStream_t st) {
    if (walks(a.chains, a.chunks)) {
        const unsigned blocks = (unsigned)((a.chains + kXcds - 1) / kXcds * kXcds);
        LaunchRecord r = launch_begin(bwd ? "scan_bwd_walk" : "scan_fwd_walk", st);
        if (bwd) k_scan_bwd_walk<T, VEC><<<blocks, kThreads<kChunkGroups>, 0, st>>>(a);
        else k_scan_fwd_walk<T, VEC><<<blocks, kThreads<kChunkGroups>, 0, st>>>(a);
        return launch_end(r);
    }
    if (a.chunks > 1) {
        // as many blocks as the chip holds, the same number for each queue
        const unsigned blocks = (unsigned)((std::min<long long>(a.chains * a.chunks, 256 * kBlocks) + a.queues - 1) / a.queues * a.queues);
        LaunchRecord r = launch_begin(bwd ? "scan_bwd_chain" : "scan_fwd_chain", st);
        if (bwd) k_scan_chain<T, VEC, true><<<blocks, kThreads<kChunkGroups>, 0, st>>>(a);
        else k_scan_chain<T, VEC, false><<<blocks, kThreads<kChunkGroups>, 0, st>>>(a);
        return launch_end(r);
    }
    if (a.T <= kSteps) return launch_scan<T, VEC, 1>(a, bwd, st);
    if (a.T <= 4 * kSteps) return launch_scan<T, VEC, 4>(a, bwd, st);
    if (a.T <= 16 * kSteps) return launch_scan<T, VEC, 16>(a, bwd, st);
    return launch_scan<T, VEC, kChunkGroups>(a, bwd, st);
}
static echo_status_t run_scan(const echo_scan_desc_t &d, const ScanPlan &p, ScanArgs a, bool bwd, void *workspace, hipStream_t st) {
    a.B = d.B, a.T = d.T, a.H = d.H, a.reverse = d.reverse;
    a.queues = 1;
    a.whole = d.H % (d.dtype == ECHO_F32 ? 4 : 8) == 0;
    a.chunks = p.chunks, a.groups_h = p.groups_h, a.chains = p.chains;
    if (p.bytes) {
        a.tickets = static_cast<unsigned long long *>(workspace);
        a.words = a.tickets + kQueues * kTicketStride;
        a.queues = p.queues;
        const long long n = (long long)(p.bytes / 16);
        LaunchRecord r = launch_begin("scan_clear", st);
        k_scan_clear<<<(unsigned)std::min<long long>((n + 255) / 256, 2048), 256, 0, st>>>(static_cast<u32x4_any *>(workspace), n);
        if (echo_status_t s = launch_end(r)) return s;
    }
    if (d.dtype == ECHO_F32) return p.vec == 4 ? launch_scan<float, 4>(a, bwd, st) : launch_scan<float, 1>(a, bwd, st);
    return p.vec == 4 ? launch_scan<bf16_t, 4>(a, bwd, st) : launch_scan<bf16_t, 1>(a, bwd, st);
}

}  // namespace echo

extern "C" {

size_t echo_scan_states_bytes(const echo_scan_desc_t *desc) {
    if (echo::check_scan(desc)) return 0;
    return (size_t)desc->B * echo::scan_chunks(*desc) * desc->H * 4;
}
size_t echo_scan_fwd_workspace_bytes(const echo_scan_desc_t *desc) { return echo::check_scan(desc) ? 0 : echo::scan_plan(*desc).bytes; }
size_t echo_scan_bwd_workspace_bytes(const echo_scan_desc_t *desc) { return echo_scan_fwd_workspace_bytes(desc); }

echo_status_t echo_scan_fwd(const echo_scan_desc_t *desc, const void *G, const float *c0, const int32_t *len, void *h, float *c_last,
                            float *states, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_scan(desc)) return s;
    const ScanPlan p = scan_plan(*desc);
    if (!G || !h || (p.bytes && !workspace)) return ECHO_ERR_NULL;
    if (unaligned_scan({G, c0, len, h, c_last, states, workspace})) return ECHO_ERR_ALIGN;
    if (workspace_bytes < p.bytes) return ECHO_ERR_WORKSPACE;
    ScanArgs a{};
    a.G = G, a.first = c0, a.len = len, a.out = h, a.last = c_last, a.states = states;
    return run_scan(*desc, p, a, false, workspace, static_cast<hipStream_t>(stream));
}

echo_status_t echo_scan_bwd(const echo_scan_desc_t *desc, const void *dh, const float *dc_last, const void *G, const int32_t *len,
                            const float *states, void *dG, float *dc0, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_scan(desc)) return s;
    const ScanPlan p = scan_plan(*desc);
    if (!dh || !G || !states || !dG || (p.bytes && !workspace)) return ECHO_ERR_NULL;
    if (unaligned_scan({dh, dc_last, G, len, states, dG, dc0, workspace})) return ECHO_ERR_ALIGN;
    if (workspace_bytes < p.bytes) return ECHO_ERR_WORKSPACE;
    ScanArgs a{};
    a.G = G, a.dh = dh, a.first = dc_last, a.len = len, a.out = dG, a.last = dc0, a.states = const_cast<float *>(states);
    return run_scan(*desc, p, a, true, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
