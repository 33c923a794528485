// Log probabilities of given tokens with entropy and top alternatives, and the gradient of the logits.
//
// For a row x of V logits and a scale c (1 / temperature), with z = c x:
//     lse = log sum_j exp z_j        logprob = z_t - lse        H = -sum_j p_j log p_j,  p_j = exp(z_j - lse)
//     dL/dx_j = c ( g (delta_jt - p_j) - h p_j (log p_j + H) )        for upstream gradients g of logprob, h of H
//
// All sums are kept relative to the running maximum m: s = sum 2^d, u = sum d 2^d with d = (x - m) c log2(e) <= 0,
// so that H = ln 2 (log2 s - u / s) has no cancellation between large logits.  x - m is formed before the
// multiplication, so that rows of the type's lowest value stay a distribution.  Statistics are fp32.
//
// small_vocab_kernel   a row in the registers of a group of 4-32 lanes (V <= 1024): one read, everything from registers.
// row_kernel           a row in the shared memory of a cluster of 1-8 CTAs: the logits are read once, by bulk copies of
//                      16 KiB that are all under way before the first is used, and the alternatives and the gradient are
//                      taken from shared memory.
// stream_kernel        many long rows, statistics and alternatives: blocks that stay, loads that run on from row to row.
// grad_kernel          gradient from saved row statistics: one read, one write.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>

#include "../../include/hpl.h"
#include "device_async.h"

namespace hpl {
namespace {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -INFINITY;
constexpr int kThreads = 256;              // of row_kernel and grad_kernel
constexpr int kBatch = 4;                  // vectors of a thread per bulk copy of the block
constexpr int kChunkVecs = kThreads * kBatch;
constexpr int kGroups = 64;                // thread groups whose maxima bound the k-th largest element from below
constexpr int kCandidates = 512;           // candidates for the top_k list held at once
constexpr int kMaxCluster = 8;
constexpr int kSmallVocab = 1024;          // small_vocab_kernel up to here
constexpr int64_t kSegment = 54 << 10;     // bytes of a row that one CTA is meant to hold
constexpr size_t kMaxSegment = 200 << 10;  // ... and that it can
constexpr int kMaxChunks = (int)((kMaxSegment / 16 + kChunkVecs - 1) / kChunkVecs);

struct LogprobsParams {
    const void* logits;
    const int64_t* targets;      // may be null: no tokens
    float* logprob;              // any output may be null
    float* entropy;
    float* top_logprob;
    int64_t* top_index;
    float4* row_stats;           // {max of x, log2 sum 2^d, H, lse}
    const float* d_logprob;      // may be null: zero
    const float* d_entropy;
    void* d_logits;
    int64_t rows, row_stride, d_row_stride;
    int32_t vocab, top_k;
    float scale, scale_log2e;
    uint32_t seg_vecs;           // 16-byte vectors of a row per CTA of the cluster
};

// ------------------------------------------------------------------ scalar and packed arithmetic
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// exponents below -150 give 0 like -150 does; keeps 0 * -inf out of u for masked logits, lets NaN through
__device__ __forceinline__ float floor_exponent(float d) {
    float y;
    asm("max.NaN.f32 %0, %1, 0fC3160000;" : "=f"(y) : "f"(d));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
using pair_t = unsigned long long;
__device__ __forceinline__ pair_t pack2(float a, float b) {
    pair_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(pair_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
    pair_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
    pair_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
    pair_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// ------------------------------------------------------------------ element types
template <bool BF16>
struct Elem {
    static constexpr int kBytes = BF16 ? 2 : 4;
    static constexpr int kPerVec = 16 / kBytes;
    __device__ static float load(const void* p, int64_t i) {
        if constexpr (BF16) return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
        else return ((const float*)p)[i];
    }
    __device__ static void store(void* p, int64_t i, float v) {
        if constexpr (BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
        else ((float*)p)[i] = v;
    }
    __device__ static void widen(const uint4& v, float (&x)[kPerVec]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                x[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ static uint4 narrow(const float (&x)[kPerVec]) {   // one rounding, to nearest even
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
            else w[i] = __float_as_uint(x[i]);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // largest element of NV vectors, NaN if there is one
    template <int NV>
    __device__ static float max_of(const uint4 (&v)[NV]) {
        if constexpr (BF16) {
            auto mx = [](uint32_t a, uint32_t b) {
                uint32_t r;
                asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
                return r;
            };
            uint32_t m = 0xFF80FF80u;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = mx(m, mx(mx(v[i].x, v[i].y), mx(v[i].z, v[i].w)));
            return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
        } else {
            float m = kNegInf;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                m = max_nan(m, max_nan(max_nan(__uint_as_float(v[i].x), __uint_as_float(v[i].y)), max_nan(__uint_as_float(v[i].z), __uint_as_float(v[i].w))));
            return m;
        }
    }
};

// ------------------------------------------------------------------ running statistics of a set of logits
struct Stats {
    float m, s, u;   // maximum, sum 2^d, sum d 2^d
};

// The same sums relative to another maximum M >= m.  An empty part (or one of NaN only) has m = -inf and s = u = 0 (NaN).
__device__ __forceinline__ Stats rebase(const Stats& a, float M, float c) {
    if (a.m == kNegInf || a.m == M) return {M, a.s, a.u};
    const float d = floor_exponent((a.m - M) * c), f = ex2(d);
    return {M, a.s * f, (a.u + a.s * d) * f};
}
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, float c) {
    const float M = fmaxf(a.m, b.m);
    const Stats x = rebase(a, M, c), y = rebase(b, M, c);
    return {M, x.s + y.s, x.u + y.u};
}

struct Running {
    float m = kNegInf;
    pair_t s = 0, u = 0;   // two independent halves

    // returns the largest of the added (NaN if there is one); the maximum passes NaN over, the sums do not
    template <bool BF16, int NV>
    __device__ __forceinline__ float add(const uint4 (&v)[NV], float c) {
        constexpr int E = Elem<BF16>::kPerVec;
        const float cm = Elem<BF16>::template max_of<NV>(v);
        if (cm > m) {
            if (m != kNegInf) {
                const float d = floor_exponent((m - cm) * c), f = ex2(d);
                const pair_t ff = pack2(f, f), dd = pack2(d, d);
                u = mul2(fma2(s, dd, u), ff);
                s = mul2(s, ff);
            }
            m = cm;
        }
        const float base = m == kNegInf ? 0.f : -m;
        const pair_t nm = pack2(base, base), cc = pack2(c, c);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[E];
            Elem<BF16>::widen(v[i], x);
#pragma unroll
            for (int j = 0; j < E; j += 2) {
                float d0, d1;
                unpack2(mul2(add2(pack2(x[j], x[j + 1]), nm), cc), d0, d1);
                d0 = floor_exponent(d0);
                d1 = floor_exponent(d1);
                const pair_t e = pack2(ex2(d0), ex2(d1));
                s = add2(s, e);
                u = fma2(e, pack2(d0, d1), u);
            }
        }
        return cm;
    }
    __device__ __forceinline__ void add_one(float x, float c) {
        // x - x is NaN for NaN and for +inf, as x - m is among vectors
        const Stats a = merge(total(), Stats{x != x ? kNegInf : x, x == kNegInf ? 0.f : 1.f + (x - x), 0.f}, c);
        m = a.m;
        s = pack2(a.s, 0.f);
        u = pack2(a.u, 0.f);
    }
    __device__ __forceinline__ Stats total() const {
        float a, b, x, y;
        unpack2(s, a, b);
        unpack2(u, x, y);
        return {m, a + b, x + y};
    }
};

// What a row's outputs and gradients are made of.
struct RowResult {
    float m;          // finite reference: the maximum, or 0 when every logit is -inf
    float log2s;      // log2 of the sum
    float H;
    bool empty;
};
__device__ __forceinline__ RowResult finish(const Stats& a) {
    RowResult r;
    r.empty = a.s == 0.f;
    r.m = a.m == kNegInf ? 0.f : a.m;
    r.log2s = r.empty ? kNegInf : log2f(a.s);
    r.H = r.empty ? 0.f : kLn2 * (r.log2s - a.u / a.s);
    return r;
}
// in natural units throughout: a logit of the type's lowest value keeps its finite log probability
__device__ __forceinline__ float log_prob(float x, const RowResult& r, float scale) {
    return r.empty ? kNegInf : fmaf(x - r.m, scale, -kLn2 * r.log2s);
}
// dx_j = p_j (a + b t_j) (+ at the token: `token`), t_j = log2 p_j = (x_j - m) c - log2s.  An empty row has a = b = 0 and
// log2s = 0 here, which makes every gradient 0.
struct GradCoef {
    float m, log2s, a, b, token;
    int32_t t;        // the token, -1 when it does not count
};
// What a row's coefficients need from memory; loaded before its statistics are there.
struct Upstream {
    int64_t t;
    float d_logprob, d_entropy;
};
__device__ __forceinline__ Upstream upstream(const LogprobsParams& p, int64_t row) {
    return {p.targets ? p.targets[row] : -1, p.d_logprob ? p.d_logprob[row] : 0.f, p.d_entropy ? p.d_entropy[row] : 0.f};
}
__device__ __forceinline__ GradCoef grad_coef(const LogprobsParams& p, const Upstream& u, const RowResult& r) {
    GradCoef g;
    const bool counts = u.t >= 0 && u.t < p.vocab && !r.empty;
    const float up = counts ? u.d_logprob : 0.f;
    const float h = r.empty ? 0.f : u.d_entropy;
    g.t = counts ? (int32_t)u.t : -1;
    g.m = r.m;
    g.log2s = r.empty ? 0.f : r.log2s;
    g.a = -p.scale * (up + h * r.H);
    g.b = -p.scale * h * kLn2;
    g.token = p.scale * up;
    return g;
}
__device__ __forceinline__ float grad_of(float x, float c, const GradCoef& g) {
    const float t = floor_exponent(fmaf(x - g.m, c, -g.log2s));
    return ex2(t) * fmaf(g.b, t, g.a);
}
// The gradients of a vector of logits whose first is element `first` of the row.
template <bool BF16>
__device__ __forceinline__ uint4 grad_vec(const uint4& w, int first, float c, const GradCoef& g) {
    constexpr int E = Elem<BF16>::kPerVec;
    float x[E];
    Elem<BF16>::widen(w, x);
    const pair_t nm = pack2(-g.m, -g.m), cc = pack2(c, c), nl = pack2(-g.log2s, -g.log2s), aa = pack2(g.a, g.a), bb = pack2(g.b, g.b);
#pragma unroll
    for (int j = 0; j < E; j += 2) {
        float t0, t1;
        unpack2(fma2(add2(pack2(x[j], x[j + 1]), nm), cc, nl), t0, t1);
        t0 = floor_exponent(t0);
        t1 = floor_exponent(t1);
        unpack2(mul2(pack2(ex2(t0), ex2(t1)), fma2(bb, pack2(t0, t1), aa)), x[j], x[j + 1]);
    }
    const int at = g.t - first;
    if (at >= 0 && at < E) {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j == at) x[j] += g.token;
    }
    return Elem<BF16>::narrow(x);
}
// Stores the vectors of a warp's lanes, lane l's at dst + 16 l for the first n lanes, where dst need not be a 16-byte boundary:
// whole vectors are put together from neighbouring lanes, only the run's two ends go by elements.
template <bool BF16>
__device__ __forceinline__ void store_run(char* dst, int n, const uint4& w, int lane) {
    const uint32_t off = (uint32_t)(uintptr_t)dst & 15;
    if (off == 0) {
        if (lane < n) *(uint4*)(dst + 16 * lane) = w;
        return;
    }
    const uint4 next = make_uint4(__shfl_down_sync(0xFFFFFFFFu, w.x, 1), __shfl_down_sync(0xFFFFFFFFu, w.y, 1), __shfl_down_sync(0xFFFFFFFFu, w.z, 1),
                                  __shfl_down_sync(0xFFFFFFFFu, w.w, 1));
    const uint32_t skip = 16 - off;                  // bytes of this vector that belong to the boundary before
    const uint32_t bits = 8 * (skip & 3);
    uint32_t a, b, c, d, e;                          // the words that hold the vector after the next boundary
    switch (skip >> 2) {
        case 0: a = w.x, b = w.y, c = w.z, d = w.w, e = next.x; break;
        case 1: a = w.y, b = w.z, c = w.w, d = next.x, e = next.y; break;
        case 2: a = w.z, b = w.w, c = next.x, d = next.y, e = next.z; break;
        default: a = w.w, b = next.x, c = next.y, d = next.z, e = next.w; break;
    }
    if (lane < n - 1)
        *(uint4*)(dst + 16 * lane + skip) = make_uint4(__funnelshift_r(a, b, bits), __funnelshift_r(b, c, bits), __funnelshift_r(c, d, bits), __funnelshift_r(d, e, bits));
    constexpr int S = Elem<BF16>::kBytes;
    auto element = [&](int i) {
        const uint32_t word = i * S < 4 ? w.x : i * S < 8 ? w.y : i * S < 12 ? w.z : w.w;
        if constexpr (BF16) ((uint16_t*)(dst + 16 * lane))[i] = (uint16_t)(word >> (16 * (i & 1)));
        else ((uint32_t*)(dst + 16 * lane))[i] = word;
    };
    if (lane == 0)
        for (int i = 0; i * S < (int)skip; ++i) element(i);
    if (lane == n - 1)
        for (int i = skip / S; i < 16 / S; ++i) element(i);
}

// Order of the alternatives as whole numbers: NaN, then the larger value, then the lower index.  0 is below every real key.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);   // -0 counts as 0
    if (x != x) return 0xFFFFFFFFu;                // whatever its sign
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ uint64_t make_key(float x, uint32_t index) { return ((uint64_t)ordered(x) << 32) | (0xFFFFFFFFu - index); }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xFFFFFFFFu - (uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) { return from_ordered((uint32_t)(k >> 32)); }

__device__ __forceinline__ void write_row(const LogprobsParams& p, int64_t row, const RowResult& r, float max, bool has_token, float token_x) {
    if (p.logprob) p.logprob[row] = has_token ? log_prob(token_x, r, p.scale) : 0.f;
    if (p.entropy) p.entropy[row] = r.H;
    if (p.row_stats) p.row_stats[row] = make_float4(max, r.log2s, r.H, r.empty ? kNegInf : fmaf(r.m, p.scale, r.log2s * kLn2));
}
__device__ __forceinline__ RowResult from_stats(const float4& st) { return {st.x == kNegInf ? 0.f : st.x, st.y, st.z, st.y == kNegInf}; }

// ------------------------------------------------------------------ a row in registers
// L lanes hold L * N logits.  Lane i of the group has elements i, i + L, ...
template <bool BF16, int L, int N>
__global__ void __launch_bounds__(256) small_vocab_kernel(const LogprobsParams p, const bool have_stats) {
    using E = Elem<BF16>;
    const int lane = threadIdx.x & (L - 1);
    const int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if (row >= p.rows) return;   // whole groups leave
    const unsigned mask = L == 32 ? 0xFFFFFFFFu : ((1u << L) - 1u) << ((threadIdx.x & 31) & ~(L - 1));
    const char* x_row = (const char*)p.logits + row * p.row_stride * E::kBytes;
    const float c = p.scale_log2e;
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = lane + i * L;
        x[i] = j < p.vocab ? E::load(x_row, j) : kNegInf;
    }
    Upstream up = {};
    if (p.d_logits) up = upstream(p, row);
    RowResult r;
    if (have_stats) {
        r = from_stats(p.row_stats[row]);
    } else {
        Stats a;
        a.m = x[0] != x[0] ? kNegInf : x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) a.m = fmaxf(a.m, x[i]);
#pragma unroll
        for (int o = L / 2; o; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(mask, a.m, o));
        const float base = a.m == kNegInf ? 0.f : a.m;
        a.s = a.u = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = floor_exponent((x[i] - base) * c), e = ex2(d);
            a.s += e;
            a.u += e * d;
        }
#pragma unroll
        for (int o = L / 2; o; o >>= 1) {
            a.s += __shfl_xor_sync(mask, a.s, o);
            a.u += __shfl_xor_sync(mask, a.u, o);
        }
        r = finish(a);
        if (lane == 0) {
            const int64_t t = p.logprob ? p.targets[row] : -1;
            const bool has_token = t >= 0 && t < p.vocab;
            write_row(p, row, r, a.m, has_token, has_token ? E::load(x_row, t) : 0.f);
        }
        // the gradient may go where the logits are: the token's has been read.  (Read with the row instead, ahead of the sums, it held up
        // the warp: 4096 x 1000 bf16 11.4 instead of 9.1 us.)
        if (p.d_logits) __syncwarp(mask);
        if (p.top_k) {
            // Whole numbers in the order of the logits; 0: taken, or none.  A lane's best is its first of the largest, and of
            // several lanes the one with the lowest index.
            uint32_t o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = lane + i * L < p.vocab ? ordered(x[i]) : 0u;
            for (int k = 0; k < p.top_k; ++k) {
                uint32_t best = o[0], at = 0;
#pragma unroll
                for (int i = 1; i < N; ++i)
                    if (o[i] > best) best = o[i], at = i;
                uint32_t most = best;
#pragma unroll
                for (int d = L / 2; d; d >>= 1) most = max(most, __shfl_xor_sync(mask, most, d));
                const uint32_t mine = best == most ? lane + at * L : 0xFFFFFFFFu;
                uint32_t index = mine;
#pragma unroll
                for (int d = L / 2; d; d >>= 1) index = min(index, __shfl_xor_sync(mask, index, d));
                if (index == mine) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i == (int)at) o[i] = 0u;
                    if (p.top_logprob) p.top_logprob[row * p.top_k + k] = log_prob(from_ordered(most), r, p.scale);
                    if (p.top_index) p.top_index[row * p.top_k + k] = index;
                }
            }
        }
    }
    if (p.d_logits) {
        const GradCoef g = grad_coef(p, up, r);
        char* d_row = (char*)p.d_logits + row * p.d_row_stride * E::kBytes;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = lane + i * L;
            if (j < p.vocab) E::store(d_row, j, grad_of(x[i], c, g) + (j == g.t ? g.token : 0.f));
        }
    }
}

// ------------------------------------------------------------------ a row in the shared memory of a cluster
// A row at any element alignment: `head` single elements up to the first 16-byte boundary, vectors, single elements.
struct RowShape {
    int32_t head, vecs, tail;
};
template <bool BF16>
__device__ __forceinline__ RowShape row_shape(const char* x_row, int32_t vocab) {
    using E = Elem<BF16>;
    RowShape s;
    s.head = min(vocab, (int32_t)((16 - ((uintptr_t)x_row & 15)) & 15) / E::kBytes);
    s.vecs = (vocab - s.head) / E::kPerVec;
    s.tail = vocab - s.head - s.vecs * E::kPerVec;
    return s;
}
struct TopScratch {
    uint64_t cand[kCandidates];
    uint64_t list[HPL_TOP_MAX];               // this CTA's alternatives, best first; read by rank 0
    uint64_t gathered[kMaxCluster * HPL_TOP_MAX];
    uint64_t bound;
    __align__(16) uint32_t group_max[kGroups];
    uint32_t winners[kGroups];                // groups that reach the bound
    uint32_t n, n_winners, bound_value;
};

// The top_k keys of this CTA's part of the row, best first, into t.list (0 where the part has fewer elements).
// Thread t has the vectors t, t + kThreads, ...; four neighbouring threads are a group.  The k-th largest of the 64 group
// maxima bounds the k-th largest element from below, so only groups that reach it are looked through, by all threads
// together (about top_k of the 64).  If more elements reach the bound than there is room for (ties), the k-th best gathered is the
// next bound: it is strictly better than the last one, so the loop ends.
template <bool BF16>
__device__ void top_of_segment(TopScratch& t, const uint4* seg, int nv, uint32_t first_index, float my_max, int top_k, bool has_single,
                               uint64_t single_key) {
    using E = Elem<BF16>;
    constexpr int kPer = kThreads / kGroups;
    const int tid = threadIdx.x;
    uint32_t gm = my_max == kNegInf ? 0u : ordered(my_max);   // NaN ranks above everything
#pragma unroll
    for (int o = 1; o < kPer; o <<= 1) gm = max(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, o));
    if (tid % kPer == 0) t.group_max[tid / kPer] = gm;
    if (tid < HPL_TOP_MAX) t.list[tid] = 0;
    if (tid == 0) t.n = 0, t.bound_value = 0xFFFFFFFFu;
    __syncthreads();
    if (tid < kGroups) {        // the k-th largest is the least that fewer than k exceed
        const uint32_t mine = t.group_max[tid];
        int above = 0;
#pragma unroll 4
        for (int i = 0; i < kGroups; i += 4) {
            const uint4 q = *(const uint4*)&t.group_max[i];
            above += (q.x > mine) + (q.y > mine) + (q.z > mine) + (q.w > mine);
        }
        const uint32_t least = __reduce_min_sync(0xFFFFFFFFu, above < top_k ? mine : 0xFFFFFFFFu);
        if (tid % 32 == 0) atomicMin(&t.bound_value, least);
    }
    __syncthreads();
    uint64_t bound = (uint64_t)t.bound_value << 32;
    if (tid < kGroups) {        // in order: among ties the first gathered are then low indices, which makes for a good next bound
        const uint32_t least = (uint32_t)(bound >> 32);
        const uint32_t first = __ballot_sync(0xFFFFFFFFu, t.group_max[tid % 32] >= least), second = __ballot_sync(0xFFFFFFFFu, t.group_max[32 + tid % 32] >= least);
        const uint32_t mine = tid < 32 ? first : second, bit = 1u << tid % 32;
        if (mine & bit) t.winners[__popc(mine & (bit - 1)) + (tid < 32 ? 0 : __popc(first))] = tid;
        if (tid == 0) t.n_winners = __popc(first) + __popc(second);
    }
    __syncthreads();
    const int per_group = kPer * ((nv + kThreads - 1) / kThreads), work = (int)t.n_winners * per_group;
    for (;;) {
        const float floor_v = bound >> 32 ? from_ordered((uint32_t)(bound >> 32)) : kNegInf;
        auto offer = [&](uint64_t key) {
            if (key >= bound) {
                const uint32_t at = atomicAdd(&t.n, 1u);
                if (at < kCandidates) t.cand[at] = key;
            }
        };
        if (has_single) offer(single_key);
        for (int i = tid; i < work; i += kThreads) {
            const int in = i % per_group, v = (int)t.winners[i / per_group] * kPer + in % kPer + in / kPer * kThreads;
            if (v >= nv) continue;
            float x[E::kPerVec];
            E::widen(seg[v], x);
#pragma unroll
            for (int j = 0; j < E::kPerVec; ++j)
                if (!(x[j] < floor_v)) offer(make_key(x[j], first_index + v * E::kPerVec + j));
        }
        __syncthreads();
        const int n = (int)min(t.n, (uint32_t)kCandidates);
        const bool over = t.n > kCandidates;
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t mine = t.cand[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += t.cand[j] > mine;
            if (over) {
                if (rank == top_k - 1) t.bound = mine;
            } else if (rank < top_k) {
                t.list[rank] = mine;
            }
        }
        __syncthreads();
        if (!over) return;
        bound = t.bound;
        if (tid == 0) t.n = 0;
        __syncthreads();
    }
}

// Merges the statistics of the first N lanes of a warp (N a power of two); every one of them has the result.
template <int N>
__device__ __forceinline__ Stats merge_lanes(Stats a, float c) {
    float M = a.m;
#pragma unroll
    for (int o = N / 2; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
    a = rebase(a, M, c);
#pragma unroll
    for (int o = N / 2; o; o >>= 1) {
        a.s += __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a.u += __shfl_xor_sync(0xFFFFFFFFu, a.u, o);
    }
    return a;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) row_kernel(const LogprobsParams p) {
    using E = Elem<BF16>;
    extern __shared__ __align__(16) uint4 seg[];
    __shared__ Stats warp_part[kThreads / 32];
    __shared__ Stats cta_part;
    __shared__ RowResult row_result;
    TopScratch& top = *(TopScratch*)(seg + p.seg_vecs);     // there is one if top_k > 0
    __shared__ uint64_t bars[kMaxChunks];
    __shared__ int abort_flag;

    cg::cluster_group cluster = cg::this_cluster();
    const unsigned n_ranks = cluster.num_blocks(), rank = cluster.block_rank();
    const int64_t row = blockIdx.x / n_ranks;
    const int tid = threadIdx.x, lane = tid & 31;
    const char* x_row = (const char*)p.logits + row * p.row_stride * E::kBytes;
    const float c = p.scale_log2e;
    const RowShape shape = row_shape<BF16>(x_row, p.vocab);
    const int v0 = (int)min((uint32_t)shape.vecs, rank * p.seg_vecs);
    const int nv = (int)min((uint32_t)shape.vecs - v0, p.seg_vecs);
    const uint32_t bar0 = smem_addr(bars);
    if (tid == 0) {
        const char* src = x_row + (int64_t)shape.head * E::kBytes + (int64_t)v0 * 16;
        const uint32_t dst = smem_addr(seg);
        const int chunks = (nv + kChunkVecs - 1) / kChunkVecs;
        abort_flag = 0;
        for (int i = 0; i < chunks; ++i) mbar_init(bar0 + 8 * i, 1);
        mbar_fence_init();
        for (int i = 0; i < chunks; ++i) {
            const uint32_t bytes = 16 * min(kChunkVecs, nv - i * kChunkVecs), at = i * kChunkVecs * 16;
            mbar_expect(bar0 + 8 * i, bytes);
            bulk_load(dst + at, src + at, bytes, bar0 + 8 * i);
        }
    }
    // single elements: the head belongs to rank 0, the tail to the last rank; one per thread
    int single = -1;
    if (rank == 0 && tid < shape.head) single = tid;
    if (rank == n_ranks - 1 && tid >= 32 && tid - 32 < shape.tail) single = shape.head + shape.vecs * E::kPerVec + tid - 32;
    float single_x = 0.f;
    if (single >= 0) single_x = E::load(x_row, single);
    Upstream up = {};
    if (p.d_logits) up = upstream(p, row);
    float token_x = 0.f;
    bool has_token = false;
    if (rank == 0 && tid == 0 && p.targets) {
        const int64_t t = p.targets[row];
        has_token = t >= 0 && t < p.vocab;
        if (has_token) token_x = E::load(x_row, t);
    }
    __syncthreads();

    Running run;
    bool ok = true;
    for (int i = 0, v = tid; v < nv; ++i, v += kChunkVecs) {
        if (!(ok = mbar_wait(bar0 + 8 * i, 0, &abort_flag, kResults))) {
            let_copies_land();       // what follows reads all of them: the alternatives' bound, the search, the gradient
            break;
        }
        if (v + (kBatch - 1) * kThreads < nv) {
            uint4 w[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) w[k] = seg[v + k * kThreads];
            run.add<BF16, kBatch>(w, c);
        } else {
            for (int q = v; q < nv; q += kThreads) {
                uint4 w[1] = {seg[q]};
                run.add<BF16, 1>(w, c);
            }
        }
    }
    if (single >= 0) run.add_one(single_x, c);
    Stats a = run.total();
    if (!ok) a.s = __int_as_float(0x7FC00000);
    float my_max = a.m;                      // of this thread's logits, NaN if there is one among them
    if (p.top_k && a.s != a.s) {             // NaN or +inf: the maximum has passed NaN over
        if (single >= 0) my_max = max_nan(my_max, single_x);
        for (int v = tid; v < nv; v += kThreads) my_max = max_nan(my_max, E::template max_of<1>({seg[v]}));
    }
    a = merge_lanes<32>(a, c);
    if (lane == 0) warp_part[tid / 32] = a;
    __syncthreads();
    if (p.top_k)
        top_of_segment<BF16>(top, seg, nv, (uint32_t)(shape.head + v0 * E::kPerVec), my_max, p.top_k, single >= 0,
                             make_key(single_x, (uint32_t)single));
    if (tid < 32) a = merge_lanes<kThreads / 32>(warp_part[lane % (kThreads / 32)], c);
    if (n_ranks > 1) {
        if (tid == 0) cta_part = a;
        cluster.sync();
        if (tid < 32) a = merge_lanes<kMaxCluster>(lane % kMaxCluster < n_ranks ? *cluster.map_shared_rank(&cta_part, lane % kMaxCluster) : Stats{kNegInf, 0.f, 0.f}, c);
        if (p.top_k && rank == 0)
            for (int i = tid; i < (int)n_ranks * p.top_k; i += kThreads)
                top.gathered[i] = cluster.map_shared_rank(&top, i / p.top_k)->list[i % p.top_k];
        // a CTA's shared memory stays until everyone has read it: the second half of this barrier is at the end
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    }
    if (tid == 0) {
        row_result = finish(a);
        if (rank == 0) write_row(p, row, row_result, a.m, has_token, token_x);
    }
    __syncthreads();
    const RowResult r = row_result;
    if (p.top_k && rank == 0) {
        const uint64_t* keys = n_ranks > 1 ? top.gathered : top.list;
        const int n = (int)n_ranks * p.top_k;
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t mine = keys[i];
            int place = 0;
            for (int j = 0; j < n; ++j) place += keys[j] > mine;
            if (mine && place < p.top_k) {
                if (p.top_logprob) p.top_logprob[row * p.top_k + place] = log_prob(key_value(mine), r, p.scale);
                if (p.top_index) p.top_index[row * p.top_k + place] = key_index(mine);
            }
        }
    }
    if (p.d_logits) {
        const GradCoef g = grad_coef(p, up, r);
        char* d_row = (char*)p.d_logits + row * p.d_row_stride * E::kBytes;
        const int first = shape.head + v0 * E::kPerVec;
        char* d_seg = d_row + (int64_t)first * E::kBytes;
        for (int v = tid - lane; v < nv; v += kThreads) {      // a warp's 32 neighbouring vectors
            const int n = min(32, nv - v);
            const uint4 w = grad_vec<BF16>(seg[v + min(lane, n - 1)], first + (v + lane) * E::kPerVec, c, g);
            store_run<BF16>(d_seg + (int64_t)v * 16, n, w, lane);
        }
        if (single >= 0) E::store(d_row, single, grad_of(single_x, c, g) + (single == g.t ? g.token : 0.f));
    }
    if (n_ranks > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// ------------------------------------------------------------------ many long rows
// A ring of 16 KiB slots that one warp keeps filled, across row ends, and eight warps empty.  Thread t of the eight has the
// vectors t, t + 256, ... of a slot; warp w's 128 vectors of a slot (or, for short rows, each of its four runs of 32)
// leave their maximum behind, which is what the search for alternatives starts from.
constexpr int kStreamSlots = 4, kStreamThreads = kThreads + 32;
constexpr int kMaxEntries = 1024;
constexpr int kAhead = 2;                  // vectors that a thread of the search has under way (4: 275 instead of 249 us for 4096 x 131072, top 8)
struct StreamShared {
    Stats part[2][kThreads / 32];
    uint64_t full[kStreamSlots], empty[kStreamSlots];
    int abort_flag;
    uint32_t n, n_winners, bound_value;
    uint64_t bound;
    __align__(16) uint32_t entry[kMaxEntries];
    uint16_t winners[kMaxEntries];
    uint64_t cand[kCandidates];
};
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <bool BF16>
__global__ void __launch_bounds__(kStreamThreads) stream_kernel(const LogprobsParams p, const int runs /* of a warp in a slot, with a maximum each: 1 or 4 */) {
    using E = Elem<BF16>;
    extern __shared__ __align__(16) uint4 slots[];
    __shared__ StreamShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const uint32_t full0 = smem_addr(sh.full), empty0 = smem_addr(sh.empty);
    if (tid == 0) {
        sh.abort_flag = 0;
        for (int i = 0; i < kStreamSlots; ++i) {
            mbar_init(full0 + 8 * i, 1);
            mbar_init(empty0 + 8 * i, kThreads / 32);
        }
        mbar_fence_init();
    }
    __syncthreads();
    int slot = 0;
    uint32_t phase = 0;
    auto advance = [&] {
        if (++slot == kStreamSlots) slot = 0, phase ^= 1;
    };
    if (warp == kThreads / 32) {
        if (lane) return;
        for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
            const char* x_row = (const char*)p.logits + row * p.row_stride * E::kBytes;
            const RowShape shape = row_shape<BF16>(x_row, p.vocab);
            const char* src = x_row + shape.head * E::kBytes;
            for (int v = 0; v < shape.vecs; v += kChunkVecs) {
                if (!mbar_wait(empty0 + 8 * slot, phase ^ 1, &sh.abort_flag, kLoads)) {
                    let_copies_land();
                    return;
                }
                const uint32_t bytes = 16 * min(kChunkVecs, shape.vecs - v);
                mbar_expect(full0 + 8 * slot, bytes);
                bulk_load(smem_addr(slots + slot * kChunkVecs), src + (int64_t)v * 16, bytes, full0 + 8 * slot);
                advance();
            }
        }
        if (*(volatile int*)&sh.abort_flag) let_copies_land();     // nobody may be waiting for them
        return;
    }
    const float c = p.scale_log2e;
    int parity = 0;
    bool ok = true;        // for good: once a wait has run out, this thread no longer knows which pass of the ring a slot holds
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, parity ^= 1) {
        const char* x_row = (const char*)p.logits + row * p.row_stride * E::kBytes;
        const RowShape shape = row_shape<BF16>(x_row, p.vocab);
        int single = -1;
        if (tid < shape.head) single = tid;
        if (tid >= 32 && tid - 32 < shape.tail) single = shape.head + shape.vecs * E::kPerVec + tid - 32;
        const float single_x = single >= 0 ? E::load(x_row, single) : 0.f;
        bool has_token = false;
        float token_x = 0.f;
        if (tid == 0 && p.logprob) {
            const int64_t t = p.targets[row];
            has_token = t >= 0 && t < p.vocab;
            if (has_token) token_x = E::load(x_row, t);
        }
        Running run;
        for (int v = 0, n = 0; v < shape.vecs; v += kChunkVecs, ++n) {
            if (ok) ok = mbar_wait(full0 + 8 * slot, phase, &sh.abort_flag, kResults);
            const uint4* in = slots + slot * kChunkVecs;
            const int left = shape.vecs - v - tid;       // this thread's vectors: those of 0, 256, 512, 768 below it
            float most[kBatch];
            if (shape.vecs - v - (tid | 31) > (kBatch - 1) * kThreads) {   // the whole warp has all four
                uint4 w[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) w[i] = in[tid + i * kThreads];
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(empty0 + 8 * slot);
                if (runs == 1) {
                    most[0] = run.add<BF16, kBatch>(w, c);
                } else {
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) most[i] = run.add<BF16, 1>({w[i]}, c);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    most[i] = kNegInf;
                    if (i * kThreads < left) most[i] = run.add<BF16, 1>({in[tid + i * kThreads]}, c);
                }
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(empty0 + 8 * slot);
                if (runs == 1) most[0] = max_nan(max_nan(most[0], most[1]), max_nan(most[2], most[3]));
            }
            if (p.top_k) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (i < runs) {
                        const uint32_t o = __reduce_max_sync(0xFFFFFFFFu, most[i] == kNegInf ? 0u : ordered(most[i]));
                        if (lane == 0) sh.entry[(n * runs + i) * (kThreads / 32) + warp] = o;
                    }
            }
            advance();
        }
        if (single >= 0) run.add_one(single_x, c);
        Stats a = run.total();
        if (!ok) a.s = __int_as_float(0x7FC00000);
        __syncwarp();
        a = merge_lanes<32>(a, c);
        if (lane == 0) sh.part[parity][warp] = a;
        if (tid == 0) sh.n = sh.n_winners = 0, sh.bound_value = 0xFFFFFFFFu;
        consumers_sync();
        a = merge_lanes<kThreads / 32>(sh.part[parity][lane % (kThreads / 32)], c);
        const RowResult r = finish(a);
        if (tid == 0) write_row(p, row, r, a.m, has_token, token_x);
        if (!p.top_k) continue;

        // alternatives: see top_of_segment; the entries stand for its group maxima, the logits come from L2 again
        const int slot_shift = runs == 1 ? 3 : 5, run_shift = runs == 1 ? 7 : 5;   // entries of a slot, vectors of an entry
        const int entries = (shape.vecs + kChunkVecs - 1) / kChunkVecs << slot_shift;
        if (entries >= p.top_k) {       // the k-th largest is the least that fewer than k exceed; entries come in eights
            uint32_t least = 0xFFFFFFFFu;
            for (int e = tid; e < entries; e += kThreads) {
                const uint32_t mine = sh.entry[e];
                int above = 0;
#pragma unroll 4
                for (int i = 0; i < entries; i += 4) {
                    const uint4 q = *(const uint4*)&sh.entry[i];
                    above += (q.x > mine) + (q.y > mine) + (q.z > mine) + (q.w > mine);
                }
                if (above < p.top_k) least = min(least, mine);
            }
            least = __reduce_min_sync(0xFFFFFFFFu, least);
            if (lane == 0) atomicMin(&sh.bound_value, least);
            consumers_sync();
        }
        // (after a wait that ran out the entries say nothing: all of the row is looked through)
        uint64_t bound = entries >= p.top_k && !*(volatile int*)&sh.abort_flag ? (uint64_t)sh.bound_value << 32 : 0;
        for (int e = tid; e < entries; e += kThreads)
            if (sh.entry[e] >= (uint32_t)(bound >> 32)) sh.winners[atomicAdd(&sh.n_winners, 1u)] = (uint16_t)e;
        consumers_sync();
        const int work = (int)sh.n_winners << run_shift;
        const uint4* vecs = (const uint4*)(x_row + shape.head * E::kBytes);
        bool over;
        do {
            const float floor_v = bound >> 32 ? from_ordered((uint32_t)(bound >> 32)) : kNegInf;
            auto offer = [&](uint64_t key) {
                if (key >= bound) {
                    const uint32_t at = atomicAdd(&sh.n, 1u);
                    if (at < kCandidates) sh.cand[at] = key;
                }
            };
            if (single >= 0) offer(make_key(single_x, (uint32_t)single));
            for (int i0 = tid; i0 < work; i0 += kAhead * kThreads) {
                uint4 w[kAhead];
                int at[kAhead];
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {      // under way together: each is a trip to L2
                    const int i = i0 + q * kThreads;
                    at[q] = -1;
                    if (i < work) {
                        const int e = sh.winners[i >> run_shift], in = i & ((1 << run_shift) - 1);
                        const int run_in_slot = runs == 1 ? in / 32 : e % 32 / 8;
                        const int v = (e >> slot_shift) * kChunkVecs + run_in_slot * kThreads + e % 8 * 32 + in % 32;
                        if (v < shape.vecs) {
                            at[q] = v;
                            w[q] = vecs[v];
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {
                    if (at[q] < 0) continue;
                    float x[E::kPerVec];
                    E::widen(w[q], x);
#pragma unroll
                    for (int j = 0; j < E::kPerVec; ++j)
                        if (!(x[j] < floor_v)) offer(make_key(x[j], (uint32_t)(shape.head + at[q] * E::kPerVec + j)));
                }
            }
            consumers_sync();
            const int n = (int)min(sh.n, (uint32_t)kCandidates);
            over = sh.n > kCandidates;
            for (int i = tid; i < n; i += kThreads) {
                const uint64_t mine = sh.cand[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += sh.cand[j] > mine;
                if (over) {
                    if (rank == p.top_k - 1) sh.bound = mine;
                } else if (rank < p.top_k) {
                    if (p.top_logprob) p.top_logprob[row * p.top_k + rank] = log_prob(key_value(mine), r, p.scale);
                    if (p.top_index) p.top_index[row * p.top_k + rank] = key_index(mine);
                }
            }
            consumers_sync();
            if (over) {
                bound = sh.bound;
                if (tid == 0) sh.n = 0;
                consumers_sync();
            }
        } while (over);
    }
    if (!ok) let_copies_land();
}

// ------------------------------------------------------------------ gradient from saved statistics
// Block i: part i % segs of row i / segs.  Eight vectors per thread, four loads in flight at a time.
constexpr int kGradVecs = 8;
template <bool BF16>
__global__ void __launch_bounds__(kThreads) grad_kernel(const LogprobsParams p, const uint32_t segs) {
    using E = Elem<BF16>;
    const int64_t row = blockIdx.x / segs;
    const int part = (int)(blockIdx.x - row * segs);
    const int tid = threadIdx.x, lane = tid & 31;
    const char* x_row = (const char*)p.logits + row * p.row_stride * E::kBytes;
    char* d_row = (char*)p.d_logits + row * p.d_row_stride * E::kBytes;
    const float c = p.scale_log2e;
    const RowShape shape = row_shape<BF16>(x_row, p.vocab);
    const int v0 = part * kGradVecs * kThreads;
    const int nv = min(shape.vecs - v0, kGradVecs * kThreads);
    const GradCoef g = grad_coef(p, upstream(p, row), from_stats(p.row_stats[row]));
    const int first = shape.head + v0 * E::kPerVec;
    const char* src = x_row + (int64_t)first * E::kBytes;
    char* dst = d_row + (int64_t)first * E::kBytes;
    constexpr int B = 4;
#pragma unroll
    for (int b = 0; b < kGradVecs; b += B) {
        uint4 w[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = tid + (b + i) * kThreads;
            w[i] = make_uint4(0, 0, 0, 0);
            if (v < nv) w[i] = *(const uint4*)(src + (int64_t)v * 16);
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = tid - lane + (b + i) * kThreads;     // the warp's first vector
            if (v >= nv) break;
            store_run<BF16>(dst + (int64_t)v * 16, min(32, nv - v), grad_vec<BF16>(w[i], first + (v + lane) * E::kPerVec, c, g), lane);
        }
    }
    if (part == 0) {
        int single = -1;
        if (tid < shape.head) single = tid;
        if (tid >= 32 && tid - 32 < shape.tail) single = shape.head + shape.vecs * E::kPerVec + tid - 32;
        if (single >= 0) E::store(d_row, single, grad_of(E::load(x_row, single), c, g) + (single == g.t ? g.token : 0.f));
    }
}

// ------------------------------------------------------------------ host side
template <bool BF16, int L, int N>
int launch_small(const LogprobsParams& p, bool have_stats, cudaStream_t stream) {
    const int64_t per_cta = 256 / L, grid = (p.rows + per_cta - 1) / per_cta;
    small_vocab_kernel<BF16, L, N><<<(unsigned)grid, 256, 0, stream>>>(p, have_stats);
    return cudaGetLastError() == cudaSuccess ? HPL_OK : HPL_ERR_CUDA;
}
template <bool BF16>
int launch_small_any(const LogprobsParams& p, bool have_stats, cudaStream_t stream) {
    if (p.vocab <= 16) return launch_small<BF16, 4, 4>(p, have_stats, stream);
    if (p.vocab <= 32) return launch_small<BF16, 8, 4>(p, have_stats, stream);
    if (p.vocab <= 128) return launch_small<BF16, 32, 4>(p, have_stats, stream);
    if (p.vocab <= 512) return launch_small<BF16, 32, 16>(p, have_stats, stream);
    return launch_small<BF16, 32, 32>(p, have_stats, stream);
}

// Lets a kernel take more than the default shared memory, once per device.
template <typename K>
bool allow_smem(K* kernel, size_t bytes, int dev, std::atomic<uint64_t>& done) {
    const uint64_t bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_relaxed) & bit) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}
template <typename... Args>
int launch_cluster(void (*kernel)(Args...), int64_t grid, int threads, size_t smem, int cluster, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? HPL_OK : HPL_ERR_CUDA;
}

template <bool BF16>
int launch_rows(LogprobsParams p, cudaStream_t stream) {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return HPL_ERR_CUDA;
    const int64_t vecs = p.vocab / Elem<BF16>::kPerVec;
    constexpr size_t kSlot = (size_t)kChunkVecs * 16;
    // Many rows of more than a CTA's segment are streamed, with alternatives (whose search stops the stream) from twice that on.
    // us for 4096 bf16 rows, streamed and not: V = 24576 51 and 46, 32768 62 and 77; with 8 alternatives V = 32768 110 and 105,
    // 65536 200 and 211, 131072 249 and 443.  Few rows leave SMs without a stream: 150 x 131072 18.4 and 17.2, 296 x 131072 19.5 and 25.7.
    if (!p.d_logits && vecs * 16 > (p.top_k ? 2 : 1) * kSegment && p.rows >= 2 * sms) {
        static std::atomic<uint64_t> done{0};
        if (!allow_smem(stream_kernel<BF16>, kStreamSlots * kSlot, dev, done)) return HPL_ERR_CUDA;
        const int64_t chunks = (vecs + kChunkVecs - 1) / kChunkVecs;
        const int runs = !p.top_k || chunks >= 16 ? 1 : kBatch;
        const int64_t grid = p.rows < 3 * sms ? p.rows : 3 * sms;
        stream_kernel<BF16><<<(unsigned)grid, kStreamThreads, kStreamSlots * kSlot, stream>>>(p, runs);
        return cudaGetLastError() == cudaSuccess ? HPL_OK : HPL_ERR_CUDA;
    }
    // 54 KiB of a row per CTA lets four CTAs share an SM, so that one's copies run under another's arithmetic (4096 x 131072
    // bf16 with gradient: 480 us, 496 us at 64 KiB, 555 us at 36 KiB); few rows are split further, to 8 KiB, so that more
    // SMs take part.
    int64_t n = (vecs * 16 + kSegment - 1) / kSegment;
    if (n < 1) n = 1;
    while (n < kMaxCluster && p.rows * n * 2 <= sms && vecs * 16 > n * (8 << 10)) ++n;
    if (n > kMaxCluster) n = kMaxCluster;
    p.seg_vecs = (uint32_t)((vecs + n - 1) / n);
    static_assert(kMaxSegment + sizeof(TopScratch) + 1024 <= (227 << 10), "fits an SM");
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(row_kernel<BF16>, kMaxSegment + sizeof(TopScratch), dev, done)) return HPL_ERR_CUDA;
    return launch_cluster(row_kernel<BF16>, p.rows * n, kThreads, (size_t)p.seg_vecs * 16 + (p.top_k ? sizeof(TopScratch) : 0), (int)n, stream, p);
}

template <bool BF16>
int launch_grad(const LogprobsParams& p, cudaStream_t stream) {
    const int64_t per = (int64_t)kGradVecs * kThreads * Elem<BF16>::kPerVec;
    const int64_t segs = (p.vocab + per - 1) / per;
    grad_kernel<BF16><<<(unsigned)(p.rows * segs), kThreads, 0, stream>>>(p, (uint32_t)segs);
    return cudaGetLastError() == cudaSuccess ? HPL_OK : HPL_ERR_CUDA;
}

enum Pass { kForward, kBackward, kBoth };

int run_pass(const hpl_logprobs_args* a, Pass pass, cudaStream_t stream) {
    if (!a || a->rows < 0 || a->vocab < 1) return HPL_ERR_INVALID;
    if (a->dtype != HPL_F32 && a->dtype != HPL_BF16) return HPL_ERR_INVALID;
    const int64_t esize = a->dtype == HPL_BF16 ? 2 : 4;
    if (a->vocab * esize > HPL_LOGPROBS_MAX_ROW_BYTES || a->rows > HPL_LOGPROBS_MAX_ROWS) return HPL_ERR_INVALID;
    const float scale = a->scale == 0.f ? 1.f : a->scale;
    if (!(scale > 0.f) || !std::isfinite(scale * kLog2e)) return HPL_ERR_INVALID;
    const int64_t stride = a->row_stride ? a->row_stride : a->vocab;
    const int64_t d_stride = a->d_row_stride ? a->d_row_stride : a->vocab;
    if (stride < a->vocab || stride > HPL_LOGPROBS_MAX_STRIDE) return HPL_ERR_INVALID;
    if (a->rows == 0) return HPL_OK;
    if (!a->logits || (uintptr_t)a->logits % esize || (uintptr_t)a->targets % 8 || (uintptr_t)a->row_stats % 16) return HPL_ERR_INVALID;
    const int top_k = pass == kBackward ? 0 : a->top_k;
    if (pass != kBackward) {
        if (a->top_k < 0 || a->top_k > HPL_TOP_MAX || a->top_k > a->vocab) return HPL_ERR_INVALID;
        if (a->top_k > 0 && !a->top_logprob && !a->top_index) return HPL_ERR_INVALID;
        if (a->logprob && !a->targets) return HPL_ERR_INVALID;
        if ((uintptr_t)a->logprob % 4 || (uintptr_t)a->entropy % 4 || (uintptr_t)a->top_logprob % 4 || (uintptr_t)a->top_index % 8) return HPL_ERR_INVALID;
    }
    if (pass != kForward) {
        if (!a->d_logits || (uintptr_t)a->d_logits % esize || d_stride < a->vocab || d_stride > HPL_LOGPROBS_MAX_STRIDE) return HPL_ERR_INVALID;
        if (a->d_logprob && !a->targets) return HPL_ERR_INVALID;
        if ((uintptr_t)a->d_logprob % 4 || (uintptr_t)a->d_entropy % 4) return HPL_ERR_INVALID;
        if (pass == kBackward && !a->row_stats) return HPL_ERR_INVALID;
        if (a->d_logits == a->logits && d_stride != stride) return HPL_ERR_INVALID;   // in place: element by element
    }

    LogprobsParams p = {};
    p.logits = a->logits;
    p.targets = a->targets;
    p.rows = a->rows;
    p.vocab = (int32_t)a->vocab;
    p.row_stride = stride;
    p.scale = scale;
    p.scale_log2e = scale * kLog2e;
    p.row_stats = (float4*)a->row_stats;
    if (pass != kBackward) {
        p.logprob = a->logprob;
        p.entropy = a->entropy;
        p.top_k = top_k;
        p.top_logprob = a->top_logprob;
        p.top_index = a->top_index;
    }
    if (pass != kForward) {
        p.d_logprob = a->d_logprob;
        p.d_entropy = a->d_entropy;
        p.d_logits = a->d_logits;
        p.d_row_stride = d_stride;
    }
    if (!arm_expiry(stream)) return HPL_ERR_CUDA;
    const bool bf16 = a->dtype == HPL_BF16;
    if (a->vocab <= kSmallVocab) return bf16 ? launch_small_any<true>(p, pass == kBackward, stream) : launch_small_any<false>(p, pass == kBackward, stream);
    if (pass == kBackward) return bf16 ? launch_grad<true>(p, stream) : launch_grad<false>(p, stream);
    return bf16 ? launch_rows<true>(p, stream) : launch_rows<false>(p, stream);
}

}  // namespace
}  // namespace hpl

extern "C" int hpl_token_logprobs(const hpl_logprobs_args* args, void* cuda_stream) {
    return hpl::run_pass(args, hpl::kForward, (cudaStream_t)cuda_stream);
}
extern "C" int hpl_token_logprobs_grad(const hpl_logprobs_args* args, void* cuda_stream) {
    return hpl::run_pass(args, hpl::kBackward, (cudaStream_t)cuda_stream);
}
extern "C" int hpl_token_logprobs_with_grad(const hpl_logprobs_args* args, void* cuda_stream) {
    return hpl::run_pass(args, hpl::kBoth, (cudaStream_t)cuda_stream);
}
