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

#include <algorithm>
#include <initializer_list>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kSteps = 4;
template <int GROUPS> constexpr int kThreads = GROUPS > 16 ? 512 : 256;
constexpr int kBlocks = 2;            // to a compute unit
constexpr int kQueues = 32, kTicketStride = 16;            // (words of 8 bytes: a cache line)
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
    long long chains, units, chain0; // B groups_h; chains by chunks; the launch's first
    void *out;                       // h; dG
    float *last;                     // c_last; dc0
    float *states;
    unsigned long long *words, *tickets;      // [units][WIDTH]; [queues], kTicketStride apart: the next to be taken
    int queues;
    bool whole;                      // rows are whole groups of 16 bytes
};

// What a thread is in a unit
template <int VEC, int GROUPS> struct Place {
    static constexpr int SUBS = kThreads<GROUPS> / 16 / GROUPS, WIDTH = 16 * VEC;
    int group, sub, slot, b, base, ch, skip, chunk, s0;    // skip: of its VEC channels, those in front that are the neighbour's
    bool on;                         // it has channels of its own
    int n;                           // steps of the sequence
    long long chain;
    __device__ __forceinline__ Place(const ScanArgs &a, long long unit, int chunk_) : chunk(chunk_) {
        const int lane16 = threadIdx.x & 15;
        group = (threadIdx.x >> 4) % GROUPS;
        sub = (threadIdx.x >> 4) / GROUPS;
        chain = min(unit + sub, a.chains - 1);
        b = (int)(chain / a.groups_h);
        base = (int)(chain - (long long)b * a.groups_h) * WIDTH;
        slot = lane16 * VEC;
        on = unit + sub < a.chains && base + slot < a.H;
        ch = min(base + slot, a.H - VEC);                  // the last lane steps back to a whole group of channels
        skip = base + slot - ch;
        n = a.len ? clamp_len(a.len[b], a.T) : a.T;
        s0 = (chunk * GROUPS + group) * kSteps;
    }
    __device__ __forceinline__ bool in(int i) const { return s0 + i < n; }
    // position of the thread's step i; steps from n on stand at their own number
    __device__ __forceinline__ int position(const ScanArgs &a, int i) const { return a.reverse && in(i) ? n - 1 - s0 - i : s0 + i; }
};

// What a lane is where a wave folds the maps of unit w: a channel each
template <int VEC, int GROUPS> struct Folder {
    typedef Place<VEC, GROUPS> P;
    int lane, ch;
    bool on, own;
    size_t row, state;               // of c0 and c_last; of the kept states
    long long chain;
    __device__ __forceinline__ Folder(const ScanArgs &a, long long unit, int w, int chunk) {
        lane = lane_id();
        chain = min(unit + w, a.chains - 1);
        const int b = (int)(chain / a.groups_h), c = (int)(chain - (long long)b * a.groups_h) * P::WIDTH + lane / VEC * VEC;
        on = w < P::SUBS && lane < P::WIDTH;
        ch = max(0, min(c, a.H - VEC)) + lane % VEC;
        own = on && unit + w < a.chains && c < a.H && ch >= c;
        row = (size_t)b * a.H + ch;
        state = ((size_t)b * a.chunks + chunk) * a.H + ch;
    }
};

// ---- chains ---------------------------------------------------------------------------------------------------------------
// The chunks of a sequence's channels are a chain: each hands the state behind it to the next.  A chunk publishes its map (A, b) as soon as it has it, and the
// state behind it (C) as soon as it knows the one in front of it; the next one takes C from the chunk in front, or from one up to kLookBack in front and applies
// the maps of those between, in order, with the same operation that each of them applies to its own: results do not depend on how far it looked.
// Map and state go out in one 64-bit word, b or C below and above it A, which is 0 to 1 and leaves the upper two bits for what it is (A that is NaN comes with
// a b that is), so that nothing has to be waited for in between; the words are cleared in front of the launch.
// Units are taken by ticket, chunk after chunk: whoever waits, waits for a unit that has been taken already and waits for lower tickets only.  The chains are
// dealt to up to kQueues queues with a ticket counter and blocks each: one counter for all gives out a ticket every 15 to 20 ns, no matter who asks
// (4 x 16384 x 1280 bf16, forward: 181 us of 10240 tickets).
struct Queue {
    unsigned *ticket;
    long long first;                 // chain; neighbours are one queue's, and with it one XCD's: they share cache lines where rows are not whole ones
    int chains;
    __device__ __forceinline__ Queue(const ScanArgs &a) {
        const int q = (int)blockIdx.x % a.queues;
        ticket = reinterpret_cast<unsigned *>(a.tickets + q * kTicketStride);
        first = a.chains * q / a.queues;
        chains = (int)(a.chains * (q + 1) / a.queues - first);
    }
    __device__ __forceinline__ unsigned take() const { return atomicAdd(ticket, 1u); }
    // the unit of a ticket: link of the chain, chain; false: there is none
    __device__ __forceinline__ bool unit(unsigned t, int links, int &link, long long &chain) const {
        link = (int)(t / (unsigned)chains);
        chain = first + (t - (unsigned)link * chains);
        return link < links;
    }
};
typedef unsigned long long Word;
constexpr Word kMapMark = 1ull << 62, kStateMark = 1ull << 63;
__device__ __forceinline__ Word map_word(float A, float b) {
    return kMapMark | (Word)(__float_as_uint(A) & 0x3fffffffu) << 32 | __float_as_uint(b);
}
__device__ __forceinline__ Word state_word(float c) { return kStateMark | __float_as_uint(c); }
__device__ __forceinline__ float factor_of(Word w) { return __uint_as_float((unsigned)(w >> 32) & 0x3fffffffu); }
__device__ __forceinline__ float value_of(Word w) { return __uint_as_float((unsigned)w); }

// The state in front of this chunk from the words of the W chunks in front of it (`ahead` of them exist), a lane per channel; false: it can't be told yet.
// `back`: words from a chunk's to those of the one in front of it.
template <int W> __device__ __forceinline__ bool look_back(const Word *unit, int lane, long long back, int ahead, float &carry) {
    Word w[W];
#pragma unroll
    for (int d = 0; d < W; ++d) w[d] = load_agent(unit - (min(d, ahead - 1) + 1) * back + lane);
    int from = -1;                                         // the nearest chunk whose state is there, the maps of all nearer ones being there
    bool maps = true;
#pragma unroll
    for (int d = 0; d < W; ++d) {
        if (from < 0 && maps && d < ahead && __all((w[d] & kStateMark) != 0)) from = d;
        maps = maps && __all((w[d] & kMapMark) != 0);
    }
    if (from < 0) return false;
#pragma unroll
    for (int d = W - 1; d >= 0; --d) {
        if (d == from) carry = value_of(w[d]);
        else if (d < from) carry = __builtin_fmaf(factor_of(w[d]), carry, value_of(w[d]));
    }
    return true;
}
// Publishes this chunk's map, returns the state in front of it (`start` if it is the first) and publishes the one behind it.
template <int W> __device__ __forceinline__ float chain_carry(Word *unit, int lane, long long back, int ahead, float start, float A, float b) {
    float carry = start;
    if (ahead > 0) {
        store_agent(unit + lane, map_word(A, b));
        const long long t0 = wall_clock64();
        while (!look_back<W>(unit, lane, back, ahead, carry)) {
            if (wall_clock64() - t0 > kSpinLimitTicks) {
                carry = __builtin_nanf("");                // make the failure visible
                break;
            }
        }
    }
    store_agent(unit + lane, state_word(__builtin_fmaf(factor_of(map_word(A, b)), carry, b)));
    return carry;
}

__global__ __launch_bounds__(256) void k_scan_clear(u32x4_any *p, long long n) {
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) p[i] = u32x4_any{0u, 0u, 0u, 0u};
}

template <typename T, int VEC, int GROUPS, bool CHAIN>
__global__ __launch_bounds__(kThreads<GROUPS>, 4) void k_scan_fwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    __shared__ float s_a[CHAIN ? 2 : 1][P::SUBS][GROUPS][P::WIDTH], s_b[CHAIN ? 2 : 1][P::SUBS][GROUPS][P::WIDTH];
    __shared__ unsigned s_ticket[2];
    const int w = wave_id();
    const Queue queue(a);
    unsigned ticket = 0;
    int buf = 0;
    if constexpr (CHAIN) {
        if (threadIdx.x == 0) s_ticket[1] = queue.take();
        __syncthreads();
        ticket = __builtin_amdgcn_readfirstlane(s_ticket[1]);
    }
    for (;;) {
        int link = 0;
        long long first_chain = a.chain0 + (long long)blockIdx.x * P::SUBS;
        if (CHAIN && !queue.unit(ticket, a.chunks, link, first_chain)) break;
        unsigned next = 0;
        if (CHAIN && threadIdx.x == kThreads<GROUPS> - 64) next = queue.take();
        const int chunk = link;
        const P p(a, first_chain, chunk);
        const size_t row = (size_t)p.b * a.T;
        const T *G = static_cast<const T *>(a.G) + row * 3 * a.H + p.ch;
        T *h = static_cast<T *>(a.out) + row * a.H + p.ch;
        Lanes<T, VEC> x[kSteps][3];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const size_t at = (size_t)(p.in(i) ? p.position(a, i) : 0) * 3 * a.H;
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G + at + (size_t)k * a.H);
        }
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
        float u[kSteps][VEC], g[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC];
            x[i][0].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[i][v] = p.in(i) ? forget_rest(y[v]) : 0.f;
            x[i][1].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) g[i][v] = p.in(i) ? candidate(y[v]) : 0.f;
        }
        if constexpr (GROUPS > 1) {
            float A[VEC], b[VEC];
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                A[v] = 1.f, b[v] = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    b[v] = __builtin_fmaf(u[i][v], g[i][v] - b[v], b[v]);
                    A[v] = __builtin_fmaf(-u[i][v], A[v], A[v]);
                }
                s_a[buf][p.sub][p.group][p.slot + v] = A[v];
                s_b[buf][p.sub][p.group][p.slot + v] = b[v];
            }
            lds_barrier();
            if (w < P::SUBS) {
                const Folder<VEC, GROUPS> f(a, first_chain, w, chunk);
                if (f.on) {
                    float(&fa)[GROUPS][P::WIDTH] = s_a[buf][w], (&fb)[GROUPS][P::WIDTH] = s_b[buf][w];
                    float state = (!CHAIN || chunk == 0) && a.first ? a.first[f.row] : 0.f;
                    if constexpr (CHAIN) {
                        float all = 1.f, sum = 0.f;
#pragma unroll 4
                        for (int k = 0; k < GROUPS; ++k) {
                            sum = __builtin_fmaf(fa[k][f.lane], sum, fb[k][f.lane]);
                            all *= fa[k][f.lane];
                        }
                        state = chain_carry<8>(a.words + (link * a.chains + f.chain) * P::WIDTH, f.lane, a.chains * P::WIDTH, chunk, state, all, sum);
                    }
                    if (a.states && f.own) a.states[f.state] = state;
#pragma unroll 4
                    for (int k = 0; k < GROUPS; ++k) {
                        const float x = __builtin_fmaf(fa[k][f.lane], state, fb[k][f.lane]);
                        fb[k][f.lane] = state;
                        state = x;
                    }
                    if (a.last && f.own && chunk == a.chunks - 1) a.last[f.row] = state;
                }
            }
            if (CHAIN && threadIdx.x == kThreads<GROUPS> - 64) s_ticket[buf] = next;
            lds_barrier();
#pragma unroll
            for (int v = 0; v < VEC; ++v) c[v] = s_b[buf][p.sub][p.group][p.slot + v];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC];
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                c[v] = __builtin_fmaf(u[i][v], g[i][v] - c[v], c[v]);
                y[v] = p.in(i) ? gate(y[v]) * c[v] : 0.f;
            }
            if (p.on && p.s0 + i < a.T) put_from<T, VEC>(h + (size_t)p.position(a, i) * a.H, y, p.skip, a.whole);
        }
        if constexpr (GROUPS == 1) {
            if (a.last && p.on) {
#pragma unroll
                for (int v = 0; v < VEC; ++v)
                    if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = c[v];
            }
        }
        if constexpr (!CHAIN) break;
        ticket = __builtin_amdgcn_readfirstlane(s_ticket[buf]);
        buf ^= 1;
    }
}

template <typename T, int VEC, int GROUPS, bool CHAIN>
__global__ __launch_bounds__(kThreads<GROUPS>, 4) void k_scan_bwd(const ScanArgs a) {
    typedef Place<VEC, GROUPS> P;
    constexpr int BUFS = CHAIN ? 2 : 1;
    __shared__ float s_a[BUFS][P::SUBS][GROUPS][P::WIDTH], s_b[BUFS][P::SUBS][GROUPS][P::WIDTH], s_r[BUFS][P::SUBS][GROUPS][P::WIDTH];
    __shared__ unsigned s_ticket[2];
    const int w = wave_id();
    const Queue queue(a);
    unsigned ticket = 0;
    int buf = 0;
    if constexpr (CHAIN) {
        if (threadIdx.x == 0) s_ticket[1] = queue.take();
        __syncthreads();
        ticket = __builtin_amdgcn_readfirstlane(s_ticket[1]);
    }
    for (;;) {
        int link = 0;
        long long first_chain = a.chain0 + (long long)blockIdx.x * P::SUBS;
        if (CHAIN && !queue.unit(ticket, a.chunks, link, first_chain)) break;
        unsigned next = 0;
        if (CHAIN && threadIdx.x == kThreads<GROUPS> - 64) next = queue.take();
        const int chunk = a.chunks - 1 - link;             // from the last one on
        const P p(a, first_chain, chunk);
        const size_t row = (size_t)p.b * a.T;
        const T *G = static_cast<const T *>(a.G) + row * 3 * a.H + p.ch;
        const T *dh = static_cast<const T *>(a.dh) + row * a.H + p.ch;
        T *dG = static_cast<T *>(a.out) + row * 3 * a.H + p.ch;
        Lanes<T, VEC> x[kSteps][3], up[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const size_t at = p.in(i) ? p.position(a, i) : 0;
#pragma unroll
            for (int k = 0; k < 3; ++k) x[i][k].load(G + (at * 3 + k) * a.H);
            up[i].load(dh + at * a.H);
        }
        float c[VEC], q[VEC];
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                c[v] = a.states[(size_t)p.b * a.H + p.ch + v];
                q[v] = a.first ? a.first[(size_t)p.b * a.H + p.ch + v] : 0.f;
            }
        }
        float u[kSteps][VEC], g[kSteps][VEC], o[kSteps][VEC], d[kSteps][VEC];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float y[VEC];
            x[i][0].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[i][v] = p.in(i) ? forget_rest(y[v]) : 0.f;
            x[i][1].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) g[i][v] = p.in(i) ? candidate(y[v]) : 0.f;
            x[i][2].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) o[i][v] = p.in(i) ? gate(y[v]) : 0.f;
            up[i].get(y);
#pragma unroll
            for (int v = 0; v < VEC; ++v) d[i][v] = p.in(i) ? y[v] : 0.f;
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
                s_a[buf][p.sub][p.group][p.slot + v] = A;
                s_b[buf][p.sub][p.group][p.slot + v] = b;
                s_r[buf][p.sub][p.group][p.slot + v] = R;
            }
            lds_barrier();
            // the states in front of the groups, and behind them f r of the next step: two waves' work in a chain, otherwise one's
            if (w < (CHAIN ? 2 : P::SUBS)) {
                const int sub = CHAIN ? 0 : w;
                const Folder<VEC, GROUPS> f(a, first_chain, sub, chunk);
                float(&fa)[GROUPS][P::WIDTH] = s_a[buf][sub], (&fb)[GROUPS][P::WIDTH] = s_b[buf][sub], (&fr)[GROUPS][P::WIDTH] = s_r[buf][sub];
                if (f.on && (!CHAIN || w == 0)) {
                    float state = a.states[f.state];
#pragma unroll 4
                    for (int k = 0; k < GROUPS; ++k) {
                        const float x = __builtin_fmaf(fa[k][f.lane], state, fb[k][f.lane]);
                        fb[k][f.lane] = state;
                        state = x;
                    }
                }
                if (f.on && (!CHAIN || w == 1)) {
                    float back = (!CHAIN || link == 0) && a.first ? a.first[f.row] : 0.f;
                    if constexpr (CHAIN) {
                        float all = 1.f, sum = 0.f;
#pragma unroll 4
                        for (int k = GROUPS - 1; k >= 0; --k) {
                            sum = __builtin_fmaf(fa[k][f.lane], sum, fr[k][f.lane]);
                            all *= fa[k][f.lane];
                        }
                        back = chain_carry<4>(a.words + (link * a.chains + f.chain) * P::WIDTH, f.lane, a.chains * P::WIDTH, link, back, all, sum);
                    }
#pragma unroll 4
                    for (int k = GROUPS - 1; k >= 0; --k) {
                        const float x = __builtin_fmaf(fa[k][f.lane], back, fr[k][f.lane]);
                        fr[k][f.lane] = back;
                        back = x;
                    }
                    if (a.last && f.own && chunk == 0) a.last[f.row] = back;
                }
            }
            if (CHAIN && threadIdx.x == kThreads<GROUPS> - 64) s_ticket[buf] = next;
            lds_barrier();
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                c[v] = s_b[buf][p.sub][p.group][p.slot + v];
                q[v] = s_r[buf][p.sub][p.group][p.slot + v];
            }
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
            if (p.on && p.s0 + i < a.T) {
                T *to = dG + (size_t)p.position(a, i) * 3 * a.H;
                put_from<T, VEC>(to, df, p.skip, a.whole);
                put_from<T, VEC>(to + a.H, dg, p.skip, a.whole);
                put_from<T, VEC>(to + 2 * (size_t)a.H, dout, p.skip, a.whole);
            }
        }
        if constexpr (GROUPS == 1) {
            if (a.last && p.on) {
#pragma unroll
                for (int v = 0; v < VEC; ++v)
                    if (v >= p.skip) a.last[(size_t)p.b * a.H + p.ch + v] = q[v];
            }
        }
        if constexpr (!CHAIN) break;
        ticket = __builtin_amdgcn_readfirstlane(s_ticket[buf]);
        buf ^= 1;
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

// Words and ticket of the chains.  Nothing where all steps are one chunk's.
struct ScanPlan {
    int vec, groups_h, chunks;
    long long chains, units;
    int queues;
    size_t bytes;
};
static ScanPlan scan_plan(const echo_scan_desc_t &d) {
    ScanPlan p{};
    p.vec = d.H < 4 ? 1 : 4;
    p.groups_h = (d.H + 16 * p.vec - 1) / (16 * p.vec);
    p.chunks = (int)scan_chunks(d);
    p.chains = (long long)d.B * p.groups_h;
    p.units = p.chains * p.chunks;
    if (p.chunks > 1) {
        p.bytes = kQueues * kTicketStride * 8 + (size_t)p.units * 16 * p.vec * 8;
        // as many queues as there are chains, or a number up to kQueues that deals them out evenly
        long long least = p.chains * 2;
        for (int q = (int)std::min<long long>(p.chains, kQueues); q > (int)std::min<long long>(p.chains, kQueues) / 2; --q) {
            const long long most = (p.chains + q - 1) / q * q;
            if (most < least) least = most, p.queues = q;
        }
    }
    return p;
}

template <typename T, int VEC, int GROUPS, bool CHAIN> static echo_status_t launch_scan(const ScanArgs &a, bool bwd, hipStream_t st) {
    constexpr int SUBS = Place<VEC, GROUPS>::SUBS;
    const auto launch = [&](const ScanArgs &x, long long blocks) {
        LaunchRecord r = launch_begin(bwd ? "scan_bwd" : "scan_fwd", st);
        if (bwd) k_scan_bwd<T, VEC, GROUPS, CHAIN><<<(unsigned)blocks, kThreads<GROUPS>, 0, st>>>(x);
        else k_scan_fwd<T, VEC, GROUPS, CHAIN><<<(unsigned)blocks, kThreads<GROUPS>, 0, st>>>(x);
        return launch_end(r);
    };
    // as many blocks as the chip holds, the same number for each queue
    if (CHAIN) return launch(a, (std::min<long long>(a.units, 256 * kBlocks) + a.queues - 1) / a.queues * a.queues);
    ScanArgs x = a;
    constexpr long long MOST = 1 << 22;                    // blocks of a launch: a grid has fewer than 2^32 threads
    for (; x.chain0 < a.chains; x.chain0 += MOST * SUBS)
        if (echo_status_t s = launch(x, std::min(MOST, (a.chains - x.chain0 + SUBS - 1) / SUBS))) return s;
    return ECHO_OK;
}
template <typename T, int VEC> static echo_status_t launch_scan(const ScanArgs &a, bool bwd, hipStream_t st) {
    if (a.chunks > 1) return launch_scan<T, VEC, kChunkGroups, true>(a, bwd, st);
    if (a.T <= kSteps) return launch_scan<T, VEC, 1, false>(a, bwd, st);
    if (a.T <= 4 * kSteps) return launch_scan<T, VEC, 4, false>(a, bwd, st);
    if (a.T <= 16 * kSteps) return launch_scan<T, VEC, 16, false>(a, bwd, st);
    return launch_scan<T, VEC, kChunkGroups, false>(a, bwd, st);
}
static echo_status_t run_scan(const echo_scan_desc_t &d, const ScanPlan &p, ScanArgs a, bool bwd, void *workspace, hipStream_t st) {
    a.B = d.B, a.T = d.T, a.H = d.H, a.reverse = d.reverse;
    a.queues = 1;
    a.whole = d.H % (d.dtype == ECHO_F32 ? 4 : 8) == 0;
    a.chunks = p.chunks, a.groups_h = p.groups_h, a.chains = p.chains, a.units = p.units;
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
