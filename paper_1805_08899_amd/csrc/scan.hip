// A gated linear recurrence over whole sequences, forward and backward (include/echoscan.h has the formulas).
//
// A thread owns kSteps consecutive steps of VEC channels; 16 such threads stand side by side, GROUPS of them one behind the other, and together take
// GROUPS kSteps steps of 16 VEC channels (a unit).  A thread's steps are a linear map of the state, c -> A c + b (backward: q -> A q + R): a wave folds
// the GROUPS maps of each channel through LDS, and every thread goes over its steps once more from the state in front of them.  A sequence longer
// than a unit is taken unit by unit.
//
// With u = 1 - f = sigmoid(-x):  c += u (g - c),  r = dh o + q,  q = r - u r  keep the digits of a u next to zero.
#include "../../include/echoscan.h"

#include <hip/hip_runtime.h>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kSteps = 4;
constexpr int kScanThreads = 512;
constexpr int kChunkGroups = ECHO_SCAN_CHUNK / kSteps;
constexpr float kLog2eS = 1.4426950408889634f;

// sigmoid(x) = 1 / (1 + 2^(-x log2 e)); tanh(x) = 1 - 2 / (2^(2 x log2 e) + 1).  exp2 overflows to infinity, whose reciprocal is 0.
__device__ __forceinline__ float gate(float x) { return fast_rcp(1.0f + fast_exp2(-kLog2eS * x)); }
__device__ __forceinline__ float forget_rest(float x) { return fast_rcp(1.0f + fast_exp2(kLog2eS * x)); }   // 1 - sigmoid(x)
__device__ __forceinline__ float candidate(float x) {
    return __builtin_fmaf(-2.0f, fast_rcp(fast_exp2(kTwoLog2e * x) + 1.0f), 1.0f);
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
typedef __bf16 bf16_hw;
__device__ __forceinline__ unsigned bf16_bits(float x) { return __builtin_bit_cast(unsigned short, (bf16_hw)x); }
__device__ __forceinline__ void put_one(float *p, float x) { *p = x; }
__device__ __forceinline__ void put_one(bf16_t *p, float x) { p->bits = (unsigned short)bf16_bits(x); }
template <int VEC> __device__ __forceinline__ void put(float *p, const float (&x)[VEC]) {
    if constexpr (VEC == 4) __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4_any *>(p));
    else store_streaming(p, x[0]);
}
template <int VEC> __device__ __forceinline__ void put(bf16_t *p, const float (&x)[VEC]) {
    if constexpr (VEC == 4)
        __builtin_nontemporal_store(u32x2{bf16_bits(x[0]) | bf16_bits(x[1]) << 16, bf16_bits(x[2]) | bf16_bits(x[3]) << 16}, reinterpret_cast<u32x2_any *>(p));
    else p->bits = (unsigned short)bf16_bits(x[0]);
}

// x[skip ..]: what a lane's neighbour has in front of that is not its own
template <typename T, int VEC> __device__ __forceinline__ void put_from(T *p, const float (&x)[VEC], int skip) {
    if (skip == 0) {
        put<VEC>(p, x);
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
    long long units;                 // B groups_h
    void *out;                       // h; dG
    float *last;                     // c_last; dc0
    float *states;
};

// What a thread is
template <int VEC, int GROUPS> struct Place {
    static constexpr int SUBS = kScanThreads / 16 / GROUPS, WIDTH = 16 * VEC;
    int lane16, group, sub, b, ch, slot;
    int skip;                        // of its VEC channels, those in front that are the neighbour's
    bool on;                         // it has channels of its own
    int n;                           // steps of the sequence
    __device__ __forceinline__ Place(const ScanArgs &a) {
        lane16 = threadIdx.x & 15;
        group = (threadIdx.x >> 4) % GROUPS;
        sub = (threadIdx.x >> 4) / GROUPS;
        const long long unit = (long long)blockIdx.x * SUBS + sub, u = unit < a.units ? unit : a.units - 1;
        b = (int)(u / a.groups_h);
        const int c = (int)(u - (long long)b * a.groups_h) * WIDTH + lane16 * VEC;
        on = unit < a.units && c < a.H;
        ch = min(c, a.H - VEC);                            // the last lane steps back to a whole group of channels
        skip = c - ch;
        slot = lane16 * VEC;
        n = a.len ? clamp_len(a.len[b], a.T) : a.T;
    }
    // position of step s; steps from n on stand at their own number
    __device__ __forceinline__ int position(const ScanArgs &a, int s) const { return a.reverse && s < n ? n - 1 - s : s; }
};

template <typename T, int VEC, int GROUPS>
__global__ __launch_bounds__(kScanThreads) void k_scan_fwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    __shared__ float s_a[GROUPS > 1 ? P::SUBS : 1][GROUPS][P::WIDTH], s_b[GROUPS > 1 ? P::SUBS : 1][GROUPS][P::WIDTH];
    const P p(a);
    const size_t row = (size_t)p.b * a.T;
    const T *G = static_cast<const T *>(a.G) + row * 3 * a.H + p.ch;
    T *h = static_cast<T *>(a.out) + row * a.H + p.ch;
    float carry[VEC];                                      // the state in front of the chunk: of every thread's own channels
#pragma unroll
    for (int v = 0; v < VEC; ++v) carry[v] = a.first ? a.first[(size_t)p.b * a.H + p.ch + v] : 0.f;
    for (int chunk = 0; chunk < a.chunks; ++chunk) {
        const int s0 = chunk * GROUPS * kSteps + p.group * kSteps;
        if (a.states && p.group == 0 && p.on) {
#pragma unroll
            for (int v = 0; v < VEC; ++v)
                if (v >= p.skip) a.states[((size_t)p.b * a.chunks + chunk) * a.H + p.ch + v] = carry[v];
        }
        Lanes<T, VEC> x[kSteps][3];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const size_t at = (size_t)(s0 + i < p.n ? p.position(a, s0 + i) : 0) * 3 * a.H;
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G + at + (size_t)k * a.H);
        }
        float u[kSteps][VEC], g[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = s0 + i < p.n;
            float y[VEC];
            x[i][0].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[i][v] = in ? forget_rest(y[v]) : 0.f;
            x[i][1].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) g[i][v] = in ? candidate(y[v]) : 0.f;
        }
        float c[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) c[v] = carry[v];
        if constexpr (GROUPS > 1) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float A = 1.f, b = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    b = __builtin_fmaf(u[i][v], g[i][v] - b, b);
                    A = __builtin_fmaf(-u[i][v], A, A);
                }
                s_a[p.sub][p.group][p.slot + v] = A;
                s_b[p.sub][p.group][p.slot + v] = b;
            }
            __syncthreads();
            // every thread folds the maps of the groups in front of it, and goes on to the end for the next chunk's start
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float state = carry[v];
#pragma unroll 4
                for (int k = 0; k < GROUPS; ++k) {
                    if (k == p.group) c[v] = state;
                    state = __builtin_fmaf(s_a[p.sub][k][p.slot + v], state, s_b[p.sub][k][p.slot + v]);
                }
                carry[v] = state;
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = s0 + i < p.n;
            float y[VEC];
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                c[v] = __builtin_fmaf(u[i][v], g[i][v] - c[v], c[v]);
                y[v] = in ? gate(y[v]) * c[v] : 0.f;
            }
            if (p.on && s0 + i < a.T) put_from<T, VEC>(h + (size_t)p.position(a, s0 + i) * a.H, y, p.skip);
        }
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) carry[v] = c[v];
        }
    }
    if (a.last && p.group == 0 && p.on) {
#pragma unroll
        for (int v = 0; v < VEC; ++v)
            if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = carry[v];
    }
}

template <typename T, int VEC, int GROUPS>
__global__ __launch_bounds__(kScanThreads) void k_scan_bwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    constexpr int SUBS = GROUPS > 1 ? P::SUBS : 1;
    __shared__ float s_a[SUBS][GROUPS][P::WIDTH], s_b[SUBS][GROUPS][P::WIDTH], s_r[SUBS][GROUPS][P::WIDTH];
    const P p(a);
    const size_t row = (size_t)p.b * a.T;
    const T *G = static_cast<const T *>(a.G) + row * 3 * a.H + p.ch;
    const T *dh = static_cast<const T *>(a.dh) + row * a.H + p.ch;
    T *dG = static_cast<T *>(a.out) + row * 3 * a.H + p.ch;
    float carry[VEC];                                      // f r of the step behind the chunk
#pragma unroll
    for (int v = 0; v < VEC; ++v) carry[v] = a.first ? a.first[(size_t)p.b * a.H + p.ch + v] : 0.f;
    for (int chunk = a.chunks - 1; chunk >= 0; --chunk) {
        const int s0 = chunk * GROUPS * kSteps + p.group * kSteps;
        Lanes<T, VEC> x[kSteps][3], up[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const size_t at = s0 + i < p.n ? p.position(a, s0 + i) : 0;
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G + (at * 3 + k) * a.H);
            up[i].load(dh + at * a.H);
        }
        float c[VEC], q[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            c[v] = a.states[((size_t)p.b * a.chunks + chunk) * a.H + p.ch + v];
            q[v] = carry[v];
        }
        float u[kSteps][VEC], g[kSteps][VEC], o[kSteps][VEC], d[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = s0 + i < p.n;
            float y[VEC];
            x[i][0].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[i][v] = in ? forget_rest(y[v]) : 0.f;
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
        if constexpr (GROUPS > 1) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float A = 1.f, b = 0.f, R = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    b = __builtin_fmaf(u[i][v], g[i][v] - b, b);
                    A = __builtin_fmaf(-u[i][v], A, A);
                    const int k = kSteps - 1 - i;
                    const float r = __builtin_fmaf(d[k][v], o[k][v], R);
                    R = __builtin_fmaf(-u[k][v], r, r);
                }
                s_a[p.sub][p.group][p.slot + v] = A;
                s_b[p.sub][p.group][p.slot + v] = b;
                s_r[p.sub][p.group][p.slot + v] = R;
            }
            __syncthreads();
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float state = c[v], back = carry[v];
#pragma unroll 4
                for (int k = 0; k < GROUPS; ++k) {
                    const int j = GROUPS - 1 - k;
                    if (k == p.group) c[v] = state;
                    if (j == p.group) q[v] = back;
                    state = __builtin_fmaf(s_a[p.sub][k][p.slot + v], state, s_b[p.sub][k][p.slot + v]);
                    back = __builtin_fmaf(s_a[p.sub][j][p.slot + v], back, s_r[p.sub][j][p.slot + v]);
                }
                carry[v] = back;
            }
            __syncthreads();
        }
        float before[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                before[i][v] = c[v];
                c[v] = __builtin_fmaf(u[i][v], g[i][v] - c[v], c[v]);
            }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = kSteps - 1 - k;
            float df[VEC], dg[VEC], dout[VEC];
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float r = __builtin_fmaf(d[i][v], o[i][v], q[v]);
                const float ru = r * u[i][v];
                df[v] = ru * (1.f - u[i][v]) * (before[i][v] - g[i][v]);
                dg[v] = ru * __builtin_fmaf(-g[i][v], g[i][v], 1.f);
                dout[v] = d[i][v] * c[v] * o[i][v] * (1.f - o[i][v]);
                c[v] = before[i][v];
                q[v] = r - ru;
            }
            if (p.on && s0 + i < a.T) {
                T *to = dG + (size_t)p.position(a, s0 + i) * 3 * a.H;
                put_from<T, VEC>(to, df, p.skip);
                put_from<T, VEC>(to + a.H, dg, p.skip);
                put_from<T, VEC>(to + 2 * (size_t)a.H, dout, p.skip);
            }
        }
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) carry[v] = q[v];
        }
    }
    if (a.last && p.group == 0 && p.on) {
#pragma unroll
        for (int v = 0; v < VEC; ++v)
            if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = carry[v];
    }
}

static echo_status_t check_scan(const echo_scan_desc_t *d) {
    if (!d) return ECHO_ERR_NULL;
    if (d->dtype != ECHO_F32 && d->dtype != ECHO_BF16) return ECHO_ERR_DTYPE;
    if (d->B < 1 || d->T < 1 || d->H < 1 || d->B > ECHO_SCAN_MAX_ROWS || d->T > ECHO_SCAN_MAX_ROWS || d->H > ECHO_SCAN_MAX_H) return ECHO_ERR_SHAPE;
    if ((d->reverse != 0 && d->reverse != 1) || (size_t)d->B * d->T * d->H > (size_t)1 << 40) return ECHO_ERR_SHAPE;
    return ECHO_OK;
}
static size_t scan_chunks(const echo_scan_desc_t &d) { return ((size_t)d.T + ECHO_SCAN_CHUNK - 1) / ECHO_SCAN_CHUNK; }

static bool unaligned_scan(std::initializer_list<const void *> ps) {
    uintptr_t m = 0;
    for (const void *p : ps) m |= (uintptr_t)p;
    return (m & 15u) != 0;
}

template <typename T, int VEC, int GROUPS> static echo_status_t launch_scan(const ScanArgs &a, bool bwd, hipStream_t st) {
    constexpr int SUBS = Place<VEC, GROUPS>::SUBS;
    const unsigned blocks = (unsigned)((a.units + SUBS - 1) / SUBS);
    LaunchRecord r = launch_begin(bwd ? "scan_bwd" : "scan_fwd", st);
    if (bwd) k_scan_bwd<T, VEC, GROUPS><<<blocks, kScanThreads, 0, st>>>(a);
    else k_scan_fwd<T, VEC, GROUPS><<<blocks, kScanThreads, 0, st>>>(a);
    return launch_end(r);
}
template <typename T, int VEC> static echo_status_t launch_scan(const ScanArgs &a, bool bwd, hipStream_t st) {
    if (a.T <= kSteps) return launch_scan<T, VEC, 1>(a, bwd, st);
    if (a.T <= 4 * kSteps) return launch_scan<T, VEC, 4>(a, bwd, st);
    if (a.T <= 16 * kSteps) return launch_scan<T, VEC, 16>(a, bwd, st);
    return launch_scan<T, VEC, kChunkGroups>(a, bwd, st);
}
static echo_status_t run_scan(const echo_scan_desc_t &d, ScanArgs a, bool bwd, hipStream_t st) {
    const int vec = d.H < 4 ? 1 : 4;
    a.B = d.B, a.T = d.T, a.H = d.H, a.reverse = d.reverse;
    a.chunks = (int)scan_chunks(d);
    a.groups_h = (d.H + 16 * vec - 1) / (16 * vec);
    a.units = (long long)d.B * a.groups_h;
    if (d.dtype == ECHO_F32) return vec == 4 ? launch_scan<float, 4>(a, bwd, st) : launch_scan<float, 1>(a, bwd, st);
    return vec == 4 ? launch_scan<bf16_t, 4>(a, bwd, st) : launch_scan<bf16_t, 1>(a, bwd, st);
}

}  // namespace echo

extern "C" {

size_t echo_scan_states_bytes(const echo_scan_desc_t *desc) {
    if (echo::check_scan(desc)) return 0;
    return (size_t)desc->B * echo::scan_chunks(*desc) * desc->H * 4;
}
size_t echo_scan_fwd_workspace_bytes(const echo_scan_desc_t *desc) { return 0; }
size_t echo_scan_bwd_workspace_bytes(const echo_scan_desc_t *desc) { return 0; }

echo_status_t echo_scan_fwd(const echo_scan_desc_t *desc, const void *G, const float *c0, const int32_t *len, void *h, float *c_last,
                            float *states, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_scan(desc)) return s;
    if (!G || !h) return ECHO_ERR_NULL;
    if (unaligned_scan({G, c0, len, h, c_last, states, workspace})) return ECHO_ERR_ALIGN;
    ScanArgs a{};
    a.G = G, a.first = c0, a.len = len, a.out = h, a.last = c_last, a.states = states;
    return run_scan(*desc, a, false, static_cast<hipStream_t>(stream));
}

echo_status_t echo_scan_bwd(const echo_scan_desc_t *desc, const void *dh, const float *dc_last, const void *G, const int32_t *len,
                            const float *states, void *dG, float *dc0, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace echo;
    if (echo_status_t s = check_scan(desc)) return s;
    if (!dh || !G || !states || !dG) return ECHO_ERR_NULL;
    if (unaligned_scan({dh, dc_last, G, len, states, dG, dc0, workspace})) return ECHO_ERR_ALIGN;
    ScanArgs a{};
    a.G = G, a.dh = dh, a.first = dc_last, a.len = len, a.out = dG, a.last = dc0, a.states = const_cast<float *>(states);
    return run_scan(*desc, a, true, static_cast<hipStream_t>(stream));
}

}  // extern "C"
