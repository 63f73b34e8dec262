// The global norm of many gradient tensors and their clipping by it: norm = sqrt(sum g^2), g *= max_norm / norm where
// norm > max_norm.  Two launches: sums of squares per block, then every block adds all of those (at most kClipParts numbers from the
// caches), derives the same factor from them and scales its share.
//
// Bound by HBM: the tensors are read once for the norm, once more to be scaled and written once (their norm is a sum over all of them,
// and nothing on the chip holds more than the 256 MB of the last cache).  The second launch therefore walks the tensors from the end:
// what the first one read last is still in that cache.  Measured (400M bf16 values in 40 tensors): 137 + 289 us, 5.8 and 5.5 TB/s; 1.5M f32
// values in 18 tensors 7 + 8 us, of which a launch of nothing is 2 to 3: a trip for the table, one for the values, one for the sums.
//
// Squares and sums are fp64: an exploding gradient (1e20) overflows fp32 squares, which would clip everything to zero.  The vector unit does
// an fp64 multiply-add per 4 clocks and wave, a tenth of what the loads leave it.
//
// The tensors' addresses and sizes travel as kernel arguments, kClipBatch tensors to a launch, so that nothing has to be
// copied to the device and a captured graph holds them.  A block's work is whole spans of kSpanBytes of one tensor, dealt round robin.
#include "../../include/echoclip.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

constexpr int kClipBatch = 96;        // 32 bytes each: with the rest below the 4 KB of a launch's arguments
constexpr int kClipThreads = 256;
constexpr int kSpanBytes = 16384;     // four 16-byte loads per thread
constexpr int kClipParts = 1024;      // blocks of the norm launches together, four to a compute unit

struct ClipTensor {
    const void *src;
    void *dst;
    long long n;                      // elements
    long long first_bf16;             // first span of this tensor in the launch, times two; bit 0: bf16
};
struct ClipTable {
    ClipTensor t[kClipBatch];
    long long spans;
    int count;
};

// A span: where it begins, and how much of its tensor is left there.  The tensor is the last one whose first span is not behind this one
// (tensors without elements have no span: they are not in the table); the lanes look at all of the table at once, one trip to
// memory where a search would take seven.
typedef unsigned u4 __attribute__((ext_vector_type(4)));
constexpr int kSpanLoads = kSpanBytes / 16 / kClipThreads;
struct ClipSpan {
    const char *src;
    char *dst;
    long long left;                   // elements
    bool bf16;
    __device__ __forceinline__ bool whole() const { return left * (bf16 ? 2 : 4) >= kSpanBytes; }
    __device__ __forceinline__ void find(const ClipTable &tab, long long s) {
        static_assert(kClipBatch <= 128, "two tensors per lane");
        const int l = lane_id();
        const int i = __builtin_popcountll(__ballot(l < tab.count && (tab.t[min(l, kClipBatch - 1)].first_bf16 >> 1) <= s)) +
                      __builtin_popcountll(__ballot(l + 64 < tab.count && (tab.t[min(l + 64, kClipBatch - 1)].first_bf16 >> 1) <= s)) - 1;
        const ClipTensor &t = tab.t[i];
        bf16 = t.first_bf16 & 1;
        const long long size = bf16 ? 2 : 4, begin = (s - (t.first_bf16 >> 1)) * (kSpanBytes / size);
        src = static_cast<const char *>(t.src) + begin * size;
        dst = static_cast<char *>(t.dst) + begin * size;
        left = t.n - begin;
    }
    __device__ __forceinline__ void load(u4 (&v)[kSpanLoads]) const {          // of a whole span
#pragma unroll
        for (int k = 0; k < kSpanLoads; ++k) v[k] = *reinterpret_cast<const u4 *>(src + (k * kClipThreads + threadIdx.x) * 16);
    }
};

__device__ __forceinline__ void clip_square(double &acc, float x) { acc = __builtin_fma((double)x, (double)x, acc); }
__device__ __forceinline__ float bf_lo(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(unsigned u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ unsigned short bf16_round(float x) {
    return __builtin_bit_cast(unsigned short, (__bf16)x);
}
__device__ __forceinline__ unsigned bf16_round2(float a, float b) { return (unsigned)bf16_round(a) | (unsigned)bf16_round(b) << 16; }

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
// Sum over the block, in every thread; fixed order.
__device__ __forceinline__ double block_sum_f64(double x, double *s) {
    x = wave_sum_f64(x);
    if (lane_id() == 0) s[wave_id()] = x;
    __syncthreads();
    double t = 0.;
#pragma unroll
    for (int w = 0; w < kClipThreads / 64; ++w) t += s[w];
    return t;
}

__global__ __launch_bounds__(kClipThreads) void k_grad_norm(const ClipTable tab, double *parts) {
    __shared__ double s_sum[kClipThreads / 64];
    double acc[4] = {0., 0., 0., 0.};
    ClipSpan s;
    if (blockIdx.x < tab.spans) s.find(tab, blockIdx.x);
    for (long long span = blockIdx.x; span < tab.spans; span += gridDim.x) {
        const ClipSpan here = s;
        u4 v[kSpanLoads];
        if (here.whole()) here.load(v);
        if (span + gridDim.x < tab.spans) s.find(tab, span + gridDim.x);      // while the loads are under way
        if (here.whole()) {
#pragma unroll
            for (int k = 0; k < kSpanLoads; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (here.bf16) {
                        clip_square(acc[j], bf_lo(v[k][j]));
                        clip_square(acc[j], bf_hi(v[k][j]));
                    } else {
                        clip_square(acc[j], __uint_as_float(v[k][j]));
                    }
                }
        } else {
            for (int i = threadIdx.x; i < (int)here.left; i += kClipThreads)
                clip_square(acc[0], here.bf16 ? __uint_as_float((unsigned)reinterpret_cast<const unsigned short *>(here.src)[i] << 16)
                                              : reinterpret_cast<const float *>(here.src)[i]);
        }
    }
    const double sum = block_sum_f64((acc[0] + acc[1]) + (acc[2] + acc[3]), s_sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__device__ __forceinline__ double grad_norm_of(const double *parts, int n_parts, double *s) {
    double x = 0.;
    for (int i = threadIdx.x; i < n_parts; i += kClipThreads) x += parts[i];
    return sqrt(block_sum_f64(x, s));
}

__global__ __launch_bounds__(kClipThreads) void k_grad_norm_finish(const double *parts, int n_parts, float *norm) {
    __shared__ double s[kClipThreads / 64];
    const double x = grad_norm_of(parts, n_parts, s);
    if (threadIdx.x == 0) *norm = (float)x;
}

__global__ __launch_bounds__(kClipThreads) void k_grad_scale(const ClipTable tab, const double *parts, int n_parts,
                                                             float max_norm, float *norm) {
    __shared__ double s_sum[kClipThreads / 64];
    // the block's first span is on its way before the norm is worked out
    ClipSpan s;
    u4 v[kSpanLoads];
    const bool any = blockIdx.x < tab.spans;
    if (any) s.find(tab, tab.spans - 1 - blockIdx.x);
    if (any && s.whole()) s.load(v);
    const double x = grad_norm_of(parts, n_parts, s_sum);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
    // false for NaN; a norm that fp32 rounds to infinity, which is what the caller reads, clips nothing either
    const bool clip = x > (double)max_norm && (float)x < __builtin_inff();
    // f 2^k: a factor below 2^-100 (down to 2^-277) would lose digits in fp32; f has [1/2, 1) then, so that no product overflows
    const double factor = clip ? (double)max_norm / x : 1.;
    const int k = factor < 0x1p-100 ? (int)(__builtin_bit_cast(unsigned long long, factor) >> 52) - 1022 : 0;
    const float f = (float)__builtin_amdgcn_ldexp(factor, -k);
    const auto scaled = [&](float v) { return __builtin_amdgcn_ldexpf(v * f, k); };
    for (long long r = blockIdx.x; r < tab.spans; r += gridDim.x) {
        if (r > blockIdx.x) {
            s.find(tab, tab.spans - 1 - r);
            if (s.whole() && (clip || s.src != s.dst)) s.load(v);
        }
        if (!clip && s.src == s.dst) continue;
        if (s.whole()) {
            if (clip) {
#pragma unroll
                for (int l = 0; l < kSpanLoads; ++l)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[l][j] = s.bf16 ? bf16_round2(scaled(bf_lo(v[l][j])), scaled(bf_hi(v[l][j]))) : __float_as_uint(scaled(__uint_as_float(v[l][j])));
            }
#pragma unroll
            for (int k = 0; k < kSpanLoads; ++k)
                __builtin_nontemporal_store(v[k], reinterpret_cast<u4 *>(s.dst + (k * kClipThreads + threadIdx.x) * 16));
        } else {
            for (int i = threadIdx.x; i < (int)s.left; i += kClipThreads) {
                if (s.bf16) {
                    const unsigned short u = reinterpret_cast<const unsigned short *>(s.src)[i];
                    reinterpret_cast<unsigned short *>(s.dst)[i] = clip ? bf16_round(scaled(__uint_as_float((unsigned)u << 16))) : u;
                } else {
                    const float u = reinterpret_cast<const float *>(s.src)[i];
                    reinterpret_cast<float *>(s.dst)[i] = clip ? scaled(u) : u;
                }
            }
        }
    }
}

static echo_status_t check_grads(const echo_grad_t *grads, int32_t count, bool clip, const float *norm, const void *workspace,
                                 size_t workspace_bytes) {
    if (!grads || !norm || !workspace) return ECHO_ERR_NULL;
    if (count < 1 || count > ECHO_GRAD_MAX_COUNT) return ECHO_ERR_SHAPE;
    uintptr_t bits = (uintptr_t)norm | (uintptr_t)workspace;
    for (int i = 0; i < count; ++i) {
        const echo_grad_t &g = grads[i];
        if (g.dtype != ECHO_F32 && g.dtype != ECHO_BF16) return ECHO_ERR_DTYPE;
        if (g.n < 0 || g.n > (int64_t(1) << 40)) return ECHO_ERR_SHAPE;
        if (g.n == 0) continue;
        if (!g.grad || (clip && !g.clipped)) return ECHO_ERR_NULL;
        bits |= (uintptr_t)g.grad | (clip ? (uintptr_t)g.clipped : 0);
    }
    if (bits & 15u) return ECHO_ERR_ALIGN;
    if (workspace_bytes < echo_grad_workspace_bytes(grads, count)) return ECHO_ERR_WORKSPACE;
    return ECHO_OK;
}

// Calls f(table) for the tensors, kClipBatch with elements at a time (once with an empty table if there are none).
template <typename F> static echo_status_t for_tables(const echo_grad_t *grads, int32_t count, F f) {
    ClipTable tab;
    tab.spans = 0;
    tab.count = 0;
    int tables = 0;
    for (int i = 0; i < count; ++i) {
        const echo_grad_t &g = grads[i];
        if (g.n > 0) {
            const bool bf = g.dtype == ECHO_BF16;
            const long long per = kSpanBytes / (bf ? 2 : 4);
            tab.t[tab.count++] = ClipTensor{g.grad, g.clipped, g.n, tab.spans * 2 + (bf ? 1 : 0)};
            tab.spans += (g.n + per - 1) / per;
        }
        if (tab.count == kClipBatch || (i == count - 1 && (tab.count > 0 || tables == 0))) {
            if (echo_status_t s = f(tab)) return s;
            ++tables;
            tab.spans = 0;
            tab.count = 0;
        }
    }
    return ECHO_OK;
}

static echo_status_t grad_impl(const echo_grad_t *grads, int32_t count, bool clip, float max_norm, float *norm, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (echo_status_t s = check_grads(grads, count, clip, norm, workspace, workspace_bytes)) return s;
    if (clip && !(max_norm > 0.f)) return ECHO_ERR_SHAPE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *parts = static_cast<double *>(workspace);
    const int tables = (count + kClipBatch - 1) / kClipBatch, most = std::max(1, kClipParts / tables);
    int n_parts = 0;
    echo_status_t s = for_tables(grads, count, [&](const ClipTable &tab) {
        const int blocks = (int)std::min<long long>(std::max<long long>(tab.spans, 1), most);
        LaunchRecord r = launch_begin("grad_norm", st);
        k_grad_norm<<<blocks, kClipThreads, 0, st>>>(tab, parts + n_parts);
        n_parts += blocks;
        return launch_end(r);
    });
    if (s) return s;
    if (!clip) {
        LaunchRecord r = launch_begin("grad_norm_finish", st);
        k_grad_norm_finish<<<1, kClipThreads, 0, st>>>(parts, n_parts, norm);
        return launch_end(r);
    }
    float *to = norm;                                                          // the first launch writes the norm
    return for_tables(grads, count, [&](const ClipTable &tab) {
        const int blocks = (int)std::min<long long>(std::max<long long>(tab.spans, 1), 2 * kClipParts);
        LaunchRecord r = launch_begin("grad_scale", st);
        k_grad_scale<<<blocks, kClipThreads, 0, st>>>(tab, parts, n_parts, max_norm, to);
        to = nullptr;
        return launch_end(r);
    });
}

}  // namespace echo

extern "C" {

size_t echo_grad_workspace_bytes(const echo_grad_t *, int32_t count) {
    if (count < 1 || count > ECHO_GRAD_MAX_COUNT) return 0;
    return sizeof(double) * echo::kClipParts;
}

echo_status_t echo_grad_norm(const echo_grad_t *grads, int32_t count, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream) {
    return echo::grad_impl(grads, count, false, 0.f, norm, workspace, workspace_bytes, stream);
}

echo_status_t echo_grad_clip(const echo_grad_t *grads, int32_t count, float max_norm, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream) {
    return echo::grad_impl(grads, count, true, max_norm, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"
