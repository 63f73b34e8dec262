// Token embedding out[n] = s E[t_n] and its gradient dE[v] = s sum_{t_n = v} dout[n], by sorted tokens.
//
// Both are bound by HBM: the forward pass reads N rows and writes N rows, the backward pass reads N rows of dout and writes all V
// rows of dE (or, adding, reads and writes those of the words that occur).
//
// Backward, three launches and no floating-point atomics:
//   k_embed_sort   a stable counting sort of the tokens.  A block owns every 256th word; it reads all tokens (from the caches: N words of 4
//                  bytes, a D-th of what the rows are) and so knows by itself how many tokens the blocks in front of it have and
//                  where each of its own goes: no exchange between blocks, one launch.
//   k_embed_sum    a wave per word with up to kRun tokens adds their rows in order; a wave per kRun sorted tokens adds what of them belongs to
//                  longer runs (the commonest word of Zipf's law has a tenth of all tokens, padding more) into parts.
//   k_embed_join   adds the parts of a long run in order.
// Measured: forward 12800 bf16 rows of 1024 7 us, one of 64 f32 rows 2.6.  Backward, V = 32000, 12800 f32 rows of 512, 40 % padding: 8.5 + 12.6 (66 MB
// written at 5.7 TB/s) + 5.1 us; V = 50021, 9601 bf16 rows of 1020 added: 8.5 + 16.3 + 5.8.  The first and the last are trips to memory one after
// the other (tokens, counters, positions; first of a run, parts, row), not bytes.  Rows that are no multiple of four are taken value by value, twice the time where bf16
// ones come from the caches (12800 rows of 1001 values instead of 1000: forward bf16 7.9 -> 15.7, f32 16.9 -> 18.1 us; backward 40.5 -> 62.7, 39.7 -> 58.7).
#include "../../include/echovocab.h"

#include <hip/hip_runtime.h>

#include "common.hpp"
#include "launch.hpp"

namespace echo {

typedef __bf16 bf16_hw;
__device__ __forceinline__ unsigned short bf16_bits(float x) { return __builtin_bit_cast(unsigned short, (bf16_hw)x); }

// VEC consecutive elements (VEC 4: aligned, 1: any)
template <int VEC> struct Quad { float v[VEC]; };
template <int VEC> __device__ __forceinline__ Quad<VEC> load_vec(const float *p, size_t i) {
    if constexpr (VEC == 4) {
        const float4 x = ld4(p, i);
        return {{x.x, x.y, x.z, x.w}};
    } else {
        return {{p[i]}};
    }
}
template <int VEC> __device__ __forceinline__ Quad<VEC> load_vec(const bf16_t *p, size_t i) {
    if constexpr (VEC == 4) {
        const float4 x = ld4(p, i);
        return {{x.x, x.y, x.z, x.w}};
    } else {
        return {{ld(p, i)}};
    }
}
template <int VEC> __device__ __forceinline__ void store_vec(float *p, size_t i, const Quad<VEC> &q) {
    if constexpr (VEC == 4) store4_streaming(p + i, make_float4(q.v[0], q.v[1], q.v[2], q.v[3]));
    else store_streaming(p + i, q.v[0]);
}
template <int VEC> __device__ __forceinline__ void store_vec(bf16_t *p, size_t i, const Quad<VEC> &q) {
    if constexpr (VEC == 4) {
        const u32x2 u = {(unsigned)bf16_bits(q.v[0]) | (unsigned)bf16_bits(q.v[1]) << 16,
                         (unsigned)bf16_bits(q.v[2]) | (unsigned)bf16_bits(q.v[3]) << 16};
        __builtin_nontemporal_store(u, reinterpret_cast<u32x2 *>(p + i));
    } else {
        p[i].bits = bf16_bits(q.v[0]);
    }
}

// ---- forward: a wave per row and up to kFwdPieces x 64 VEC columns, whose loads leave together ------------------------
constexpr int kFwdPieces = 4;
template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(256) void k_embed_fwd(const int *__restrict__ tokens, const TI *__restrict__ table, float scale,
                                                   TO *__restrict__ out, int N, int V, int D) {
    const int n = blockIdx.x * 4 + wave_id(), c0 = ((int)blockIdx.y * kFwdPieces * 64 + lane_id()) * VEC;
    if (n >= N) return;
    const int t = tokens[n];
    Quad<VEC> q[kFwdPieces];
#pragma unroll
    for (int k = 0; k < kFwdPieces; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) q[k].v[j] = 0.f;
    if ((unsigned)t < (unsigned)V) {
#pragma unroll
        for (int k = 0; k < kFwdPieces; ++k)
            if (c0 + k * 64 * VEC < D) q[k] = load_vec<VEC>(table, (size_t)t * D + c0 + k * 64 * VEC);
#pragma unroll
        for (int k = 0; k < kFwdPieces; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) q[k].v[j] *= scale;
    }
#pragma unroll
    for (int k = 0; k < kFwdPieces; ++k)
        if (c0 + k * 64 * VEC < D) store_vec<VEC>(out, (size_t)n * D + c0 + k * 64 * VEC, q[k]);
}

// ---- backward --------------------------------------------------------------------------------------------------------
// Tokens per part of a long run; longer runs than this are long.  It is also what a wave adds one after the other: with 32, 9600 bf16 rows of
// 1020 take 37 us in k_embed_sum, with 16 21, with 8 12 (more parts for k_embed_join: 2 -> 4).
constexpr int kRun = 8;
constexpr int kSortWaves = 16;
constexpr int kSortMaxWords = 512;    // of a block: 32 KB of counters

// Words are dealt to the blocks in turn, so that the commonest ones (the first, by Zipf's law) are with different blocks: word v is number v >> shift of
// block v & (blocks - 1), and stands at slot() in the sorted order.  256 blocks, one to a compute unit, as long as one takes no more than kSortMaxWords.
struct Deal {
    int shift, per_block;
    __host__ __device__ int blocks() const { return 1 << shift; }
    __host__ __device__ size_t slots() const { return (size_t)per_block << shift; }
    __device__ __forceinline__ int slot(int v) const { return (v & ((1 << shift) - 1)) * per_block + (v >> shift); }
};
static Deal deal_of(int V) {
    Deal d{8, (V + 255) / 256};
    while (d.per_block > kSortMaxWords) {
        ++d.shift;
        d.per_block = (V + (1 << d.shift) - 1) >> d.shift;
    }
    return d;
}

// order[p] = token's place n, word[p] = its word, for sorted positions p; first[slot of v] = position of word v's first token, first[slots] = number
// of tokens that are words.  s_count: kSortWaves x R counters, in turn: tokens per wave and word, then the next position of each.
constexpr int kSortKeep = 16;         // groups of 64 tokens that a wave keeps in registers between its two looks at them
__global__ __launch_bounds__(64 * kSortWaves) void k_embed_sort(const int *__restrict__ tokens, int N, int V, const Deal deal,
                                                                int *__restrict__ order, int *__restrict__ word,
                                                                int *__restrict__ first) {
    extern __shared__ int s_count[];
    __shared__ int s_before[kSortWaves], s_upto[kSortWaves];
    const int lane = lane_id(), w = wave_id(), R = deal.per_block, own = blockIdx.x, mask = deal.blocks() - 1;
    const int share = ((N + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;      // a wave's tokens: whole groups of 64
    const int begin = min(N, w * share), end = min(N, begin + share);
    int t[kSortKeep];
    auto look = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kSortKeep; ++u) t[u] = i0 + 64 * u + lane < end ? tokens[i0 + 64 * u + lane] : -1;
    };
    look(begin);
    for (int i = threadIdx.x; i < kSortWaves * R; i += 64 * kSortWaves) s_count[i] = 0;
    __syncthreads();
    int *mine = s_count + w * R;
    int before = 0;
    for (int i0 = begin; i0 < end; i0 += 64 * kSortKeep) {
        if (i0 > begin) look(i0);
#pragma unroll
        for (int u = 0; u < kSortKeep; ++u) {
            const bool is = (unsigned)t[u] < (unsigned)V;
            before += is && (t[u] & mask) < own ? 1 : 0;
            if (is && (t[u] & mask) == own) atomicAdd(&mine[t[u] >> deal.shift], 1);
        }
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) before += __shfl_xor(before, off);
    if (lane == 0) s_before[w] = before;
    __syncthreads();
    // positions, in the order of words, then of waves: a thread per word
    const int r = threadIdx.x;
    int mine_of[kSortWaves], total = 0, upto = 0;
    if (r < R) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) mine_of[k] = s_count[k * R + r];
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const int x = mine_of[k];
            mine_of[k] = total;
            total += x;
        }
    }
    upto = total;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(upto, off);
        if (lane >= off) upto += x;
    }
    if (lane == 63) s_upto[w] = upto;
    __syncthreads();
    int at = upto - total, all = 0;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        at += s_before[k] + (k < w ? s_upto[k] : 0);
        all += s_upto[k];
    }
    if (r < R) {
        first[(size_t)own * R + r] = at;
        if (r == R - 1 && own == mask) first[deal.slots()] = at + total;
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) s_count[k * R + r] = at + mine_of[k];
    }
    if (all == 0) return;
    __syncthreads();
    if (end - begin > 64 * kSortKeep) look(begin);
    volatile int *next = mine;
    for (int i0 = begin; i0 < end; i0 += 64 * kSortKeep) {
        if (i0 > begin) look(i0);
#pragma unroll
        for (int u = 0; u < kSortKeep; ++u) {
            const bool in = (unsigned)t[u] < (unsigned)V && (t[u] & mask) == own;
            unsigned long long left = __ballot(in);
            int p = 0;
            while (left) {                                                     // one word after the other: there are few in a group of 64 tokens
                const int l = __builtin_ctzll(left), v = __builtin_amdgcn_readlane(t[u], l);
                const unsigned long long same = __ballot(t[u] == v);
                const int at = next[v >> deal.shift];
                if (t[u] == v) p = at + __builtin_popcountll(same & ((1ull << lane) - 1));
                if (lane == l) next[v >> deal.shift] = at + __builtin_popcountll(same);
                left &= ~same;
            }
            if (in) {
                order[p] = i0 + 64 * u + lane;
                word[p] = t[u];
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// Up to kPieces x 64 VEC columns of a row at a time, a lane's VEC of each: their loads leave together.
constexpr int kPieces = 4;
template <int VEC> struct RowPieces {
    Quad<VEC> q[kPieces];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) q[k].v[j] = 0.f;
    }
    template <typename T> __device__ __forceinline__ void load(const T *row, int c, int D) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (c + k * 64 * VEC < D) q[k] = load_vec<VEC>(row, c + k * 64 * VEC);
    }
    __device__ __forceinline__ void add(const RowPieces &o) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) q[k].v[j] += o.q[k].v[j];
    }
    __device__ __forceinline__ void scale(float s) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) q[k].v[j] *= s;
    }
    __device__ __forceinline__ void store(float *row, int c, int D) const {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (c + k * 64 * VEC < D) store_vec<VEC>(row, c + k * 64 * VEC, q[k]);
    }
};

// Rows of dout, columns c .., added in order: row k is row at(k) of dout, `at` held by lane k (a run of up to 64 positions is one load).
// All lanes of the wave have to be here: lanes past the last column too hold numbers that are read.
template <typename T, int VEC>
__device__ __forceinline__ void add_rows(RowPieces<VEC> &sum, const T *dout, int at, int k0, int n, int D, int c) {
    constexpr int U = 2;
    for (int k = k0; k < n; k += U) {
        RowPieces<VEC> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].zero();
            if (k + u < n) x[u].load(dout + (size_t)__builtin_amdgcn_readlane(at, k + u) * D, c, D);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u < n) sum.add(x[u]);
    }
}

template <int VEC> __device__ __forceinline__ void put_row(float *dtable, size_t i, Quad<VEC> q, float scale, bool acc) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) q.v[j] *= scale;
    if (acc) {
        const Quad<VEC> old = load_vec<VEC>(dtable, i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) q.v[j] += old.v[j];
    }
    store_vec<VEC>(dtable, i, q);
}

// Blocks of four waves: first those of the groups of kRun sorted tokens, then those of the words (all of them are written), or, to add,
// of the sorted tokens, of which the first of each word acts (the other words stay as they are).
// parts: two rows of pitch P per group: 0 the long run that holds the group's first token, 1 the long run that begins behind it
template <typename T, int VEC>
__global__ __launch_bounds__(256) void k_embed_sum(const T *__restrict__ dout, const int *__restrict__ order,
                                                   const int *__restrict__ word, const int *__restrict__ first, const Deal deal, float scale,
                                                   float *__restrict__ dtable, float *__restrict__ parts, int N, int V, int D, int P,
                                                   int groups, int group_blocks, bool acc) {
    constexpr int WIDTH = kPieces * 64 * VEC;
    const int lane = lane_id();
    RowPieces<VEC> sum;
    if ((int)blockIdx.x < group_blocks) {
        const int g = blockIdx.x * 4 + wave_id(), p0 = g * kRun;
        if (g >= groups) return;
        const int mine = min(p0 + (lane & (kRun - 1)), N - 1), at = order[mine], v = word[mine], total = first[deal.slots()];
        if (p0 >= total) return;
        const int n = min(kRun, total - p0), a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, n - 1);
        const int sa = deal.slot(a), sb = deal.slot(b), a0 = first[sa], a1 = first[sa + 1], b0 = first[sb], b1 = first[sb + 1];
        float *to = parts + (size_t)g * 2 * P;
        if (a1 - a0 > kRun)
            for (int c0 = 0; c0 < D; c0 += WIDTH) {
                sum.zero();
                add_rows<T, VEC>(sum, dout, at, 0, min(n, a1 - p0), D, c0 + lane * VEC);
                sum.store(to, c0 + lane * VEC, D);
            }
        if (b != a && b1 - b0 > kRun)
            for (int c0 = 0; c0 < D; c0 += WIDTH) {
                sum.zero();
                add_rows<T, VEC>(sum, dout, at, b0 - p0, n, D, c0 + lane * VEC);
                sum.store(to + P, c0 + lane * VEC, D);
            }
        return;
    }
    const int i = ((int)blockIdx.x - group_blocks) * 4 + wave_id();
    if (acc) {
        // everything that depends on the position alone is requested at once, then what depends on its word
        if (i >= N) return;
        const int at = order[min(i + (lane & (kRun - 1)), N - 1)], v = word[i], before = word[max(i - 1, 0)];
        if (i >= first[deal.slots()] || (i > 0 && before == v)) return;
        const int end = first[deal.slot(v) + 1];
        float *row = dtable + (size_t)v * D;
        for (int c0 = 0; c0 < D; c0 += WIDTH) {
            RowPieces<VEC> old;
            old.zero();
            old.load(row, c0 + lane * VEC, D);
            sum.zero();
            sum.load(dout + (size_t)__builtin_amdgcn_readlane(at, 0) * D, c0 + lane * VEC, D);
            if (end - i > kRun) return;
            add_rows<T, VEC>(sum, dout, at, 1, end - i, D, c0 + lane * VEC);
            sum.scale(scale);
            sum.add(old);
            sum.store(row, c0 + lane * VEC, D);
        }
        return;
    }
    if (i >= V) return;
    const int s = deal.slot(i), p0 = first[s], n = first[s + 1] - p0;
    if (n > kRun) return;
    const int at = lane < n ? order[p0 + lane] : 0;
    for (int c0 = 0; c0 < D; c0 += WIDTH) {
        sum.zero();
        add_rows<T, VEC>(sum, dout, at, 0, n, D, c0 + lane * VEC);
        sum.scale(scale);
        sum.store(dtable + (size_t)i * D, c0 + lane * VEC, D);
    }
}

// A block per group and 64 VEC columns: the long run that begins in the group, if there is one.  The four waves add a quarter of
// its parts each, in order.
template <int VEC>
__global__ __launch_bounds__(256) void k_embed_join(const int *__restrict__ word, const int *__restrict__ first, const Deal deal, float scale,
                                                    const float *__restrict__ parts, float *__restrict__ dtable, int N, int D, int P,
                                                    bool acc) {
    const int g = blockIdx.x, p0 = g * kRun, last = word[min(p0 + kRun, N) - 1], total = first[deal.slots()];
    if (p0 >= total) return;
    // a long run that begins here reaches past the group: it holds its last token
    const int v = p0 + kRun <= total ? last : word[total - 1];
    const int s = deal.slot(v), begin = first[s], end = first[s + 1];
    if (end - begin <= kRun || begin < p0) return;        // (begin < p0: it began in an earlier group)
    __shared__ Quad<VEC> s_sum[4][64];
    const int w = wave_id(), lane = lane_id(), c = (int)blockIdx.y * 64 * VEC + lane * VEC;
    const int n = (end - 1) / kRun - g + 1, share = (n + 3) / 4;
    Quad<VEC> sum;
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum.v[j] = 0.f;
    if (c < D) {
        const int k1 = min(n, (w + 1) * share);
        for (int k0 = w * share; k0 < k1; k0 += 8) {
            Quad<VEC> x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int k = min(k0 + u, k1 - 1);
                x[u] = load_vec<VEC>(parts, ((size_t)(g + k) * 2 + (k == 0 && begin != p0 ? 1 : 0)) * P + c);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k0 + u < k1)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sum.v[j] += x[u].v[j];
        }
    }
    s_sum[w][lane] = sum;
    __syncthreads();
    if (w == 0 && c < D) {
        sum = s_sum[0][lane];
#pragma unroll
        for (int k = 1; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum.v[j] += s_sum[k][lane].v[j];
        put_row<VEC>(dtable, (size_t)v * D + c, sum, scale, acc);
    }
}

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct EmbedWs {
    size_t order, word, first, parts, total;
    int groups, pitch;
    Deal deal;
};
static EmbedWs embed_layout(const echo_vocab_desc_t &d) {
    EmbedWs w;
    w.groups = (d.N + kRun - 1) / kRun;
    w.deal = deal_of(d.V);
    w.pitch = (d.D + 3) / 4 * 4;
    w.order = 0;
    w.word = w.order + up256((size_t)d.N * 4);
    w.first = w.word + up256((size_t)d.N * 4);
    w.parts = w.first + up256((w.deal.slots() + 1) * 4);
    w.total = w.parts + (size_t)w.groups * 2 * w.pitch * 4;
    return w;
}

static echo_status_t check_embed(const echo_vocab_desc_t *d, float scale) {
    if (!d) return ECHO_ERR_NULL;
    if ((d->in_dtype != ECHO_F32 && d->in_dtype != ECHO_BF16) || (d->out_dtype != ECHO_F32 && d->out_dtype != ECHO_BF16)) return ECHO_ERR_DTYPE;
    if (d->N < 1 || d->V < 1 || d->D < 1 || d->N > ECHO_VOCAB_MAX_ROWS || d->V > ECHO_VOCAB_MAX_ROWS || d->D > ECHO_VOCAB_MAX_D) return ECHO_ERR_SHAPE;
    if (!(scale - scale == 0.f)) return ECHO_ERR_SHAPE;                        // infinite or NaN
    return ECHO_OK;
}

template <typename TI, typename TO>
static void embed_fwd_launch(const echo_vocab_desc_t &d, const int *tokens, const void *table, float scale, void *out, hipStream_t st) {
    const TI *e = static_cast<const TI *>(table);
    TO *o = static_cast<TO *>(out);
    const int vec = d.D % 4 == 0 ? 4 : 1, width = kFwdPieces * 64 * vec;
    const dim3 grid((d.N + 3) / 4, (d.D + width - 1) / width);
    if (vec == 4) k_embed_fwd<TI, TO, 4><<<grid, 256, 0, st>>>(tokens, e, scale, o, d.N, d.V, d.D);
    else k_embed_fwd<TI, TO, 1><<<grid, 256, 0, st>>>(tokens, e, scale, o, d.N, d.V, d.D);
}

template <typename T, int VEC>
static void embed_sum_launch(const echo_vocab_desc_t &d, const EmbedWs &w, const void *dout, const int *order, const int *word,
                             const int *first, float scale, float *dtable, float *parts, bool acc, hipStream_t st) {
    const int group_blocks = (w.groups + 3) / 4, word_blocks = ((acc ? d.N : d.V) + 3) / 4;
    k_embed_sum<T, VEC><<<group_blocks + word_blocks, 256, 0, st>>>(static_cast<const T *>(dout), order, word, first, w.deal, scale, dtable, parts,
                                                                    d.N, d.V, d.D, w.pitch, w.groups, group_blocks, acc);
}

static echo_status_t embed_bwd_impl(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *dout, float scale, float *dtable,
                                    void *workspace, size_t workspace_bytes, bool acc, void *stream) {
    if (echo_status_t s = check_embed(desc, scale)) return s;
    if (!tokens || !dout || !dtable || !workspace) return ECHO_ERR_NULL;
    if (((uintptr_t)tokens | (uintptr_t)dout | (uintptr_t)dtable | (uintptr_t)workspace) & 15u) return ECHO_ERR_ALIGN;
    const echo_vocab_desc_t d = *desc;
    const EmbedWs w = embed_layout(d);
    if (workspace_bytes < w.total) return ECHO_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    int *order = reinterpret_cast<int *>(ws + w.order), *word = reinterpret_cast<int *>(ws + w.word), *first = reinterpret_cast<int *>(ws + w.first);
    float *parts = reinterpret_cast<float *>(ws + w.parts);
    LaunchRecord r = launch_begin("embed_sort", st);
    k_embed_sort<<<w.deal.blocks(), 64 * kSortWaves, (size_t)kSortWaves * w.deal.per_block * 4, st>>>(tokens, d.N, d.V, w.deal, order, word, first);
    if (echo_status_t s = launch_end(r)) return s;
    r = launch_begin("embed_sum", st);
    const bool quads = d.D % 4 == 0;
    if (d.out_dtype == ECHO_F32) {
        if (quads) embed_sum_launch<float, 4>(d, w, dout, order, word, first, scale, dtable, parts, acc, st);
        else embed_sum_launch<float, 1>(d, w, dout, order, word, first, scale, dtable, parts, acc, st);
    } else {
        if (quads) embed_sum_launch<bf16_t, 4>(d, w, dout, order, word, first, scale, dtable, parts, acc, st);
        else embed_sum_launch<bf16_t, 1>(d, w, dout, order, word, first, scale, dtable, parts, acc, st);
    }
    if (echo_status_t s = launch_end(r)) return s;
    if (d.N <= kRun) return ECHO_OK;                                           // no run is long
    r = launch_begin("embed_join", st);
    if (quads) k_embed_join<4><<<dim3(w.groups, (d.D + 255) / 256), 256, 0, st>>>(word, first, w.deal, scale, parts, dtable, d.N, d.D, w.pitch, acc);
    else k_embed_join<1><<<dim3(w.groups, (d.D + 63) / 64), 256, 0, st>>>(word, first, w.deal, scale, parts, dtable, d.N, d.D, w.pitch, acc);
    return launch_end(r);
}

}  // namespace echo

extern "C" {

echo_status_t echo_embed_fwd(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *table, float scale, void *out,
                             void *stream) {
    if (echo_status_t s = echo::check_embed(desc, scale)) return s;
    if (!tokens || !table || !out) return ECHO_ERR_NULL;
    if (((uintptr_t)tokens | (uintptr_t)table | (uintptr_t)out) & 15u) return ECHO_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    echo::LaunchRecord r = echo::launch_begin("embed_fwd", st);
    const bool ib = desc->in_dtype == ECHO_BF16, ob = desc->out_dtype == ECHO_BF16;
    if (ib && ob) echo::embed_fwd_launch<echo::bf16_t, echo::bf16_t>(*desc, tokens, table, scale, out, st);
    else if (ib) echo::embed_fwd_launch<echo::bf16_t, float>(*desc, tokens, table, scale, out, st);
    else if (ob) echo::embed_fwd_launch<float, echo::bf16_t>(*desc, tokens, table, scale, out, st);
    else echo::embed_fwd_launch<float, float>(*desc, tokens, table, scale, out, st);
    return echo::launch_end(r);
}

size_t echo_embed_bwd_workspace_bytes(const echo_vocab_desc_t *desc) {
    if (echo::check_embed(desc, 1.f)) return 0;
    return echo::embed_layout(*desc).total;
}

echo_status_t echo_embed_bwd(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *dout, float scale, float *dtable,
                             void *workspace, size_t workspace_bytes, void *stream) {
    return echo::embed_bwd_impl(desc, tokens, dout, scale, dtable, workspace, workspace_bytes, false, stream);
}

echo_status_t echo_embed_bwd_accumulate(const echo_vocab_desc_t *desc, const int32_t *tokens, const void *dout, float scale,
                                        float *dtable, void *workspace, size_t workspace_bytes, void *stream) {
    return echo::embed_bwd_impl(desc, tokens, dout, scale, dtable, workspace, workspace_bytes, true, stream);
}

}  // extern "C"
