// Orthogonalisation of an update by Newton-Schulz products, and the momentum step around it.
//
//     M' = beta M + s G          U = s G + beta M' (Nesterov) or M'          X_0 = U / (|U|_F + eps)
//     per step:  A = X X^T,  P = b A + c A A,  X <- a X + P X                 (a, b, c) = (3.4445, -4.7750, 2.0315)
//     W' = W (1 - lr wd) - lr us X
// A is taken on the shorter side (X^T X and X P for a matrix taller than wide), so it is s x s with s = min(rows, cols).
//
// Number format.  The steps multiply small singular values by 3.4445 each time, so what rounding does to X early is seen
// 480-fold at the end: X in one 16-bit plane is not enough.  X, A and P are held as two fp16 planes, hi + lo, of the value
// times 2^14 (|X| <= 1.21, |A| <= 1.47, |P| <= 2.81 by the polynomial's range, so hi stays below 65504; the pair resolves
// 22 bits down to 2^-38).  A product of pairs is three tensor-core products, hi hi + hi lo + lo hi, in one fp32
// accumulator: 32-bit results, for a 16-bit result too, whose only rounding that counts is then the last one (1.7e-3 of its norm).  Products
// of the hi planes alone would take a third of the tensor cores' work, but their 11 bits are seen: 1.6e-3 of the norm over a Gaussian
// matrix after 5 steps, where roundings average out, 3e-3 to 6e-3 where they do not (few rows that are not zero, equal entries, a
// single entry), and more with every further step (300 x 500 Gaussian: 4.6e-3 after 8, 1.4e-2 after 64).
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>

#include "../../include/hpl.h"
#include "device_async.h"

namespace hpl {
namespace {

namespace cg = cooperative_groups;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr double kLeastNorm = 1e-34;         // |U| + eps at least, so that kPlane over it is finite in fp32
constexpr float kPlane = 16384.f;            // planes hold value * 2^14
constexpr float kUnplane = 1.f / 16384.f;
constexpr int kTileM = 128, kTileK = 64;
constexpr int kChunk = 2;                    // blocks of 64 k between two readings of the accumulator
constexpr int kBoxBytes = 64 * 128;          // a TMA box: 64 rows of 64 fp16, 128-byte swizzle
constexpr int kEpiWarps = 8;
constexpr int kGemmThreads = (kEpiWarps + 4) * 32;   // whole warpgroups: loads and products have one of their own
constexpr int kBlockWords = 32 * 32;         // an epilogue warp's transposition block
// Shared memory of an SM, and what each block takes beside its own.  A block that holds tensor memory while it waits for the others of its
// cluster takes so much that no further block fits on its SM: two clusters could else each hold the tensor memory that a block of the other
// waits for.  A block without a cluster waits for nothing that holds any: it may share its SM.
constexpr size_t kSmSmem = 228 << 10, kBlockReserve = 1024;
constexpr int kPartials = 1024;               // at most so many partial sums of squares per matrix

// The three products of a step; the last one of the last step makes the result.
enum Op { kGram, kPoly, kApply };
// What becomes of a product: planes, planes of a sum with an addend, the result.
enum Mode { kPlanes, kAddend, kFinal };

// What becomes of the result.
struct Output {
    void* dst;              // orthogonalize: the matrix; step: new weights
    const void* weight;     // null: orthogonalize
    __nv_bfloat16* copy;
    int64_t row_stride, batch_stride;
    int32_t bf16;
    int32_t vec;            // every row of dst, weight and copy starts on a boundary of four elements
    float keep, take;       // W' = keep W - take X
};

struct Planes {             // [2][batch][rows][ld] fp16
    __half* p;
    int64_t lo;             // elements from the hi to the lo plane
    int64_t batch_stride;
    int32_t ld;
};

struct NsParams {
    CUtensorMap maps[4];    // X, the other X, A, P
    Planes x[2], a, p;
    Output out;
    int32_t rows, cols, side, batch, steps;
    int32_t phase;          // 3 step + op
    int32_t split;          // CTAs (a cluster) that share the sum over k of a tile; then there is one tile for each cluster
};

// ------------------------------------------------------------------ PTX
// The same shared memory address in the first CTA of the pair.
__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
// Relaxed: what it tells is that this warp's reads of the accumulator are over, and those have been waited for.  (A release
// would wait for the warp's global stores too.)
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
// CTAS = 2: the bytes land here, the barrier is the pair's first CTA's
template <int CTAS>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if constexpr (CTAS == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
                     "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
}
template <int CTAS>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CTAS == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"((uint32_t)accumulate)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"((uint32_t)accumulate)
                     : "memory");
}
// arrives when the products so far are done, in both CTAs of a pair
template <int CTAS>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CTAS == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// All threads of the cluster (CTAS = 2), or of the block.
template <int CTAS>
__device__ __forceinline__ void meet() {
    if constexpr (CTAS == 2)
        asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    else
        __syncthreads();
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]),
          "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ uint64_t pair_of(float x, float y) { return (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x); }
// Two fp32 additions, rounded to nearest; not moved behind the next load, whose registers are needed.
__device__ __forceinline__ void add_pair(uint64_t& acc, uint32_t x, uint32_t y) {
    asm volatile("{\n.reg .b64 t;\nmov.b64 t, {%1, %2};\nadd.rn.f32x2 %0, %0, t;\n}" : "+l"(acc) : "r"(x), "r"(y));
}
// An operand tile in shared memory, 128-byte swizzle, rows of 128 bytes.  K contiguous: groups of 8 rows every 1024 bytes.
// M (N) contiguous: blocks of 64 x 64 every 8192 bytes along M (N), groups of 8 k every 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn) {
    const uint64_t lead = mn ? kBoxBytes >> 4 : 1, stride = 1024 >> 4;
    return (uint64_t)(addr >> 4 & 0x3FFF) | lead << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}

// ------------------------------------------------------------------ phases and tiles
struct Phase {
    const CUtensorMap *map_a, *map_b;
    const Planes *src, *dst;    // the addend (none: null); where planes go (the result: null)
    int32_t M, N, K;
    int32_t a_mn, b_mn;         // operand stored with its M (N) dimension contiguous instead of K
    int32_t symmetric;
    float alpha, beta;          // alpha D + beta addend
    int32_t tiles_m, tiles_n, tiles;   // of one matrix
};
struct Tile {
    int b, row, col;            // matrix, first row and column
};
constexpr int kGroupRows = 8;   // tile rows that run together: their operands stay in L2 while the columns go by
// A symmetric result: a tile row has the column tiles that reach the diagonal or lie below it.
__host__ __device__ __forceinline__ int row_tiles(int i, int bm, int bn, int tiles_n) {
    const int n = ((i + 1) * bm + bn - 1) / bn;
    return n < tiles_n ? n : tiles_n;
}
__host__ __device__ inline void count_tiles(Phase& f, int bm, int bn) {
    f.tiles_m = (f.M + bm - 1) / bm;
    f.tiles_n = (f.N + bn - 1) / bn;
    f.tiles = f.tiles_m * f.tiles_n;
    if (f.symmetric) {
        f.tiles = 0;
        for (int i = 0; i < f.tiles_m; ++i) f.tiles += row_tiles(i, bm, bn, f.tiles_n);
    }
}
__host__ __device__ inline Phase phase_at(const NsParams& g, int phase, int bm, int bn) {
    const int step = phase / 3, op = phase % 3, cur = step & 1;
    const bool wide = g.rows <= g.cols;
    Phase f = {};
    f.M = f.N = f.K = g.side;
    f.symmetric = op != kApply;
    if (op == kGram) {          // A = X X^T, or X^T X with both operands' M (N) contiguous
        f.K = wide ? g.cols : g.rows;
        f.map_a = f.map_b = &g.maps[cur];
        f.a_mn = f.b_mn = !wide;
        f.dst = &g.a;
        f.alpha = kUnplane;
    } else if (op == kPoly) {   // P = b A + c A A
        f.map_a = f.map_b = &g.maps[2];
        f.src = &g.a;
        f.dst = &g.p;
        f.alpha = kC * kUnplane;
        f.beta = kB;
    } else {                    // X = a X + P X, or a X + X P
        f.M = g.rows;
        f.N = g.cols;
        f.map_a = wide ? &g.maps[3] : &g.maps[cur];
        f.map_b = wide ? &g.maps[cur] : &g.maps[3];
        f.b_mn = wide;
        f.src = &g.x[cur];
        f.dst = step + 1 < g.steps ? &g.x[cur ^ 1] : nullptr;
        f.alpha = kUnplane;
        f.beta = kA;
    }
    count_tiles(f, bm, bn);
    return f;
}
template <int BM, int BN>
__device__ __forceinline__ Tile tile_at(const Phase& f, int t) {
    Tile r;
    r.b = t / f.tiles;
    int q = t % f.tiles;
    if (f.symmetric) {
        int i = 0;
        for (int n; (n = row_tiles(i, BM, BN, f.tiles_n)) <= q; ++i) q -= n;
        r.row = i * BM;
        r.col = q * BN;
    } else {
        const int group = kGroupRows * f.tiles_n, first = q / group * kGroupRows, in = q % group;
        const int rows = min(kGroupRows, f.tiles_m - first);
        r.row = (first + in % rows) * BM;
        r.col = in / rows * BN;
    }
    return r;
}
// The tiles of all matrices go round the grid, in the same order for every role.
template <int CTAS, int BN, typename Work>
__device__ __forceinline__ void walk(const NsParams& g, const Phase& f, Work&& work) {
    const int unit = CTAS * g.split;
    for (int t = blockIdx.x / unit; t < f.tiles * g.batch; t += gridDim.x / unit)
        if (!work(tile_at<CTAS * kTileM, BN>(f, t))) return;
}

// CTAS = 2: a pair of CTAs on one 256 x BN tile, each with its 128 rows of A and of the result and half of B.
template <int CTAS, int BN>
struct Config {
    static constexpr int kBRows = BN / CTAS;
    static constexpr int kABytes = kTileM * 128, kBBytes = kBRows * 128;    // of a plane, 64 k
    static constexpr int kScratch = kEpiWarps * kBlockWords * 4;
    static constexpr int kRing = (227 << 10) - 1024 - 512 - kScratch;
    static constexpr size_t kSmem = 1024 + (size_t)kRing + kScratch + 512;
    static_assert(kSmem + kBlockReserve <= kSmSmem && kSmem + 2 * kBlockReserve > kSmSmem, "a block of a cluster that takes tensor memory has the SM to itself");
    static constexpr int kStageBytes = (kABytes + kBBytes) * 2, kStages = kRing / kStageBytes;   // as many as fit: 3 or 4
};

// Two values as a word of hi parts and a word of lo parts.
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(y - h.y), "f"(x - h.x));
}
__device__ __forceinline__ float2 join(uint32_t hi, uint32_t lo) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hi)), b = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    return make_float2(a.x + b.x, a.y + b.y);
}
// A transposition block: 32 rows of 8 16-byte chunks.  Chunks are permuted so that a lane per row, a row's chunks over lanes,
// and the words of one column over rows (every eighth row in one access) all spread over the banks.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * 8 + (((chunk ^ (row & 7)) + 2 * (row >> 3)) & 7); }

// Four neighbouring weights as fp32; what lies at or beyond `n` is not touched.
__device__ __forceinline__ float4 read_weights(const Output& o, int64_t at, int n) {
    if (o.vec && n >= 4) {
        if (!o.bf16) return *(const float4*)((const float*)o.weight + at);
        const uint2 r = *(const uint2*)((const __nv_bfloat16*)o.weight + at);
        return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xFFFF0000u));
    }
    float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) w[i] = o.bf16 ? __bfloat162float(((const __nv_bfloat16*)o.weight)[at + i]) : ((const float*)o.weight)[at + i];
    return make_float4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void write_result(const Output& o, int64_t at, int n, float4 x) {
    uint2 b;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b.x) : "f"(x.y), "f"(x.x));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b.y) : "f"(x.w), "f"(x.z));
    if (o.vec && n >= 4) {
        if (o.bf16) *(uint2*)((uint16_t*)o.dst + at) = b;
        else *(float4*)((float*)o.dst + at) = x;
        if (o.copy) *(uint2*)(o.copy + at) = b;
        return;
    }
    const float v[4] = {x.x, x.y, x.z, x.w};
    const uint16_t h[4] = {(uint16_t)b.x, (uint16_t)(b.x >> 16), (uint16_t)b.y, (uint16_t)(b.y >> 16)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) {
            if (o.bf16) ((uint16_t*)o.dst)[at + i] = h[i];
            else ((float*)o.dst)[at + i] = v[i];
            if (o.copy) ((uint16_t*)o.copy)[at + i] = h[i];
        }
}

// Products, and what follows them.  Warps 0-7: epilogue; 8: loads; 9: tensor-core products.
template <int CTAS, int BN, int MODE>
__global__ void __launch_bounds__(kGemmThreads, 1) ns_kernel(const __grid_constant__ NsParams g) {
    using C = Config<CTAS, BN>;
    constexpr int kTmemCols = 2 * BN, kStageBytes = C::kStageBytes, kStages = C::kStages;
    extern __shared__ uint8_t raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);   // the swizzle repeats every 1024 bytes
    uint4* scratch = (uint4*)(base + C::kRing / 1024 * 1024);
    uint64_t* bars = (uint64_t*)(scratch + kEpiWarps * kBlockWords / 4);
    // full[stage], empty[stage], accumulator full[2], accumulator empty[2]
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](int s) { return bar0 + 8 * s; };
    auto empty = [&](int s) { return bar0 + 8 * (kStages + s); };
    auto acc_full = [&](int s) { return bar0 + 8 * (2 * kStages + s); };
    auto acc_empty = [&](int s) { return bar0 + 8 * (2 * kStages + 2 + s); };
    volatile int* abort = (volatile int*)(bars + 2 * kStages + 4);
    uint32_t* tmem_slot = (uint32_t*)(bars + 2 * kStages + 5);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t cta = 0;       // which of the pair
    int part = 0;           // which of those that share a sum
    if constexpr (CTAS == 2) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(cta));
    else if (g.split > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(part));

    if (threadIdx.x == 0) {
        *abort = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(acc_full(s), 1);
            mbar_init(acc_empty(s), kEpiWarps * CTAS);
        }
        mbar_fence_init();
    }
    if (warp == 8 && lane < 4) asm volatile("prefetch.tensormap [%0];" ::"l"(&g.maps[lane]) : "memory");
    if (warp == 9) {
        if constexpr (CTAS == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "n"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "n"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if constexpr (CTAS == 2) meet<2>();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");        // what earlier kernels wrote is read from here on

    // The tensor core's fp32 accumulator cuts off what does not fit, always towards zero: over 256 additions that is 1e-5 of a
    // sum of squares.  Products therefore leave it every 2 blocks (24 additions, 8 of them onto a sum that matters) and
    // are summed up in registers, rounded to nearest.
    const Phase f = phase_at(g, g.phase, CTAS * kTileM, BN);
    const int all_blocks = (f.K + kTileK - 1) / kTileK, per_part = (all_blocks + g.split - 1) / g.split;
    const int first_block = part * per_part, k_blocks = min(per_part, all_blocks - first_block);    // of 64 k, this CTA's
    struct Ring {
        int stage = 0;
        uint32_t phase = 0;
    } ring;
    if (warp >= kEpiWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");      // 128 * 88 + 256 * 208 = 384 * 168
        if (warp == 8 && lane == 0) {
            walk<CTAS, BN>(
                g, f, [&](const Tile& tile) {
                    const int row = tile.row + (int)cta * kTileM, col = tile.col + (int)cta * C::kBRows;
                    for (int kb = 0; kb < k_blocks; ++kb) {
                        const int k0 = (first_block + kb) * kTileK;
                        if (!mbar_wait(empty(ring.stage), ring.phase ^ 1, abort, kLoads)) return false;
                        const uint32_t dst = smem_addr(base) + ring.stage * kStageBytes;
                        const uint32_t bar = CTAS == 2 ? leader_addr(full(ring.stage)) : full(ring.stage);
                        if (cta == 0) mbar_expect(full(ring.stage), CTAS * kStageBytes);
                        for (int pl = 0; pl < 2; ++pl) {
                            const int z = pl * g.batch + tile.b;
                            const uint32_t da = dst + pl * C::kABytes, db = dst + 2 * C::kABytes + pl * C::kBBytes;
#pragma unroll
                            for (int i = 0; i < kTileM / 64; ++i) {
                                const int r = row + 64 * i;
                                tma_load<CTAS>(da + i * kBoxBytes, f.map_a, f.a_mn ? r : k0, f.a_mn ? k0 : r, z, bar);
                            }
#pragma unroll
                            for (int i = 0; i < C::kBRows / 64; ++i) {
                                const int c = col + 64 * i;
                                tma_load<CTAS>(db + i * kBoxBytes, f.map_b, f.b_mn ? c : k0, f.b_mn ? k0 : c, z, bar);
                            }
                        }
                        if (++ring.stage == kStages) ring.stage = 0, ring.phase ^= 1;
                    }
                    return true;
                });
        } else if (warp == 9 && lane == 0 && cta == 0) {
            int buf = 0;
            uint32_t acc_phase = 0;
            walk<CTAS, BN>(
                g, f, [&](const Tile&) {
                    const uint32_t idesc = 1u << 4 | (uint32_t)f.a_mn << 15 | (uint32_t)f.b_mn << 16 | (uint32_t)(BN >> 3) << 17 | (uint32_t)(CTAS * kTileM >> 4) << 24;
                    const uint32_t ka = f.a_mn ? 2048 >> 4 : 32 >> 4, kb16 = f.b_mn ? 2048 >> 4 : 32 >> 4;   // 16 k further
                    for (int kc = 0; kc < k_blocks; kc += kChunk) {
                        if (!mbar_wait(acc_empty(buf), acc_phase ^ 1, abort, kProducts)) return false;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t d = tmem + buf * BN;
                        for (int kb = kc; kb < min(kc + kChunk, k_blocks); ++kb) {
                            if (!mbar_wait(full(ring.stage), ring.phase, abort, kProducts)) return false;
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            const uint32_t sa = smem_addr(base) + ring.stage * kStageBytes, sb = sa + 2 * C::kABytes;
                            const uint64_t a_hi = operand_desc(sa, f.a_mn), b_hi = operand_desc(sb, f.b_mn);
                            const uint64_t a_lo = operand_desc(sa + C::kABytes, f.a_mn), b_lo = operand_desc(sb + C::kBBytes, f.b_mn);
#pragma unroll
                            for (int k = 0; k < kTileK / 16; ++k) {   // the small terms first, while the accumulator is small
                                mma_f16<CTAS>(d, a_hi + k * ka, b_lo + k * kb16, idesc, kb > kc || k > 0);
                                mma_f16<CTAS>(d, a_lo + k * ka, b_hi + k * kb16, idesc, true);
                            }
#pragma unroll
                            for (int k = 0; k < kTileK / 16; ++k) mma_f16<CTAS>(d, a_hi + k * ka, b_hi + k * kb16, idesc, true);
                            mma_commit<CTAS>(empty(ring.stage));
                            if (++ring.stage == kStages) ring.stage = 0, ring.phase ^= 1;
                        }
                        mma_commit<CTAS>(acc_full(buf));
                        buf ^= 1;
                        if (buf == 0) acc_phase ^= 1;
                    }
                    return true;
                });
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        uint4* block = scratch + warp * (kBlockWords / 4);
        const int quad = warp & 3;
        constexpr int kCols = BN / 2, kBlocks = kCols / 32;   // this warp: 32 rows, half of the columns
        int buf = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        walk<CTAS, BN>(
            g, f, [&](const Tile& tile) {
                const int row_block = tile.row / kTileM + (int)cta;
                const int r0 = row_block * kTileM + quad * 32, col0 = tile.col + (warp >> 2) * kCols;
                auto skipped = [&](int c0) { return r0 >= f.M || c0 >= f.N || (f.symmetric && c0 / kTileM > row_block); };
                if constexpr (MODE == kFinal)      // weights are read at the end: towards L2 with them
                    if (g.out.weight && r0 + lane < f.M) {
                        const int size = g.out.bf16 ? 2 : 4;
                        const char* w = (const char*)g.out.weight + ((int64_t)tile.b * g.out.batch_stride + (int64_t)(r0 + lane) * g.out.row_stride + col0) * size;
                        for (int c = 0; c < min(kCols, f.N - col0) * size; c += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(w + c));
                    }
                uint64_t acc[kCols / 2] = {};      // sums, pairs of fp32
                // They begin with the addend: afterwards there is no room for it in registers, nor time to wait for it.  8 rows of
                // 64 bytes per access, through the transposition block to a row per lane.
                if (MODE != kPlanes && part == 0) {
                    const float e = f.beta / f.alpha;
                    const __half* p = f.src->p + (int64_t)tile.b * f.src->batch_stride + (int64_t)(r0 + lane / 4) * f.src->ld + 8 * (lane % 4);
                    const int64_t row8 = 8ll * f.src->ld;
#pragma unroll
                    for (int q = 0; q < kBlocks; ++q) {
                        const int c0 = col0 + 32 * q;
                        if (skipped(c0)) continue;
                        uint4 hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            hi[i] = lo[i] = make_uint4(0, 0, 0, 0);
                            if (r0 + 8 * i + lane / 4 < f.M && c0 + 8 * (lane % 4) < f.N) {
                                hi[i] = *(const uint4*)(p + i * row8 + c0);
                                lo[i] = *(const uint4*)(p + i * row8 + c0 + f.src->lo);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            block[chunk_at(8 * i + lane / 4, lane % 4)] = hi[i];
                            block[chunk_at(8 * i + lane / 4, 4 + lane % 4)] = lo[i];
                        }
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint4 h = block[chunk_at(lane, j)], l = block[chunk_at(lane, 4 + j)];
                            const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float2 v = join(hw[i], lw[i]);
                                acc[q * 16 + 4 * j + i] = pair_of(e * v.x, e * v.y);
                            }
                        }
                        __syncwarp();
                    }
                }
                for (int kc = 0; kc < k_blocks; kc += kChunk) {
                    // A warp that has given up reads no more and frees no accumulator: what it has not read may not be overwritten, for
                    // the other CTA of a pair may still be right.  The warp as a whole: its loads are aligned ones.
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full(buf), acc_phase, abort, kResults));
                    if (ok) {
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                        for (int q = 0; q < kCols; q += 32) {
                            uint32_t v[32];
                            tmem_load32(tmem + (warp >> 2) * kCols + ((uint32_t)(quad * 32) << 16) + buf * BN + q, v);
#pragma unroll
                            for (int i = 0; i < 16; ++i) add_pair(acc[q / 2 + i], v[2 * i], v[2 * i + 1]);
                        }
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            if (CTAS == 2) mbar_arrive_remote(leader_addr(acc_empty(buf)));
                            else mbar_arrive(acc_empty(buf));
                        }
                    }
                    buf ^= 1;
                    if (buf == 0) acc_phase ^= 1;
                }
                if (CTAS == 1 && g.split > 1) {
                    // the parts come together in the first CTA, in order; the ring has been read to its end and holds them meanwhile
                    if (!ok) {                         // ... or loads may be on their way to it
                        let_copies_land();
#pragma unroll
                        for (int i = 0; i < kCols / 2; ++i) acc[i] = 0x7FC000007FC00000ull;     // the sum is to be NaN
                    }
                    ulonglong2* mine = (ulonglong2*)base + threadIdx.x;
                    if (part)
#pragma unroll
                        for (int i = 0; i < kCols / 4; ++i) mine[i * 256] = make_ulonglong2(acc[2 * i], acc[2 * i + 1]);
                    meet<2>();
                    if (part == 0)
                        for (int r = 1; r < g.split; ++r) {
                            const ulonglong2* theirs = cg::this_cluster().map_shared_rank(mine, r);
#pragma unroll
                            for (int i = 0; i < kCols / 4; ++i) {
                                const ulonglong2 v = theirs[i * 256];
                                add_pair(acc[2 * i], (uint32_t)v.x, (uint32_t)(v.x >> 32));
                                add_pair(acc[2 * i + 1], (uint32_t)v.y, (uint32_t)(v.y >> 32));
                            }
                        }
                    meet<2>();
                    if (part) return true;
                }
#pragma unroll 1
                for (int q = 0; q < kBlocks; ++q) {
                    const int c0 = col0 + q * 32;
                    if (skipped(c0)) continue;
                    float x[32];
#pragma unroll
                    for (int w = 0; w < kBlocks; ++w)      // registers have no index
                        if (w == q) {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                x[2 * i] = __uint_as_float((uint32_t)acc[w * 16 + i]), x[2 * i + 1] = __uint_as_float((uint32_t)(acc[w * 16 + i] >> 32));
                        }
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = ok ? x[i] * f.alpha : __int_as_float(0x7FC00000);
                    if constexpr (MODE == kFinal) {
                        const int c = c0 + 4 * (lane % 8);         // four rows of 32 columns per access
                        const int64_t at = (int64_t)tile.b * g.out.batch_stride + (int64_t)(r0 + lane / 8) * g.out.row_stride + c;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            *(float4*)&block[chunk_at(lane, j)] = make_float4(x[4 * j] * kUnplane, x[4 * j + 1] * kUnplane, x[4 * j + 2] * kUnplane, x[4 * j + 3] * kUnplane);
                        __syncwarp();
#pragma unroll
                        for (int h = 0; h < 8; h += 4) {           // the weights of four accesses under way together
                            float4 w[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                w[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (g.out.weight && r0 + 4 * (h + i) + lane / 8 < f.M && c < f.N) w[i] = read_weights(g.out, at + 4 * (h + i) * g.out.row_stride, f.N - c);
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float4 v = *(const float4*)&block[chunk_at(4 * (h + i) + lane / 8, lane % 8)];
                                if (g.out.weight)
                                    v = make_float4(fmaf(-g.out.take, v.x, g.out.keep * w[i].x), fmaf(-g.out.take, v.y, g.out.keep * w[i].y),
                                                    fmaf(-g.out.take, v.z, g.out.keep * w[i].z), fmaf(-g.out.take, v.w, g.out.keep * w[i].w));
                                if (r0 + 4 * (h + i) + lane / 8 < f.M && c < f.N) write_result(g.out, at + 4 * (h + i) * g.out.row_stride, f.N - c, v);
                            }
                        }
                    } else {
                    // chunks 0-3: hi parts, 4-7: lo parts
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split2(x[8 * j + 2 * i], x[8 * j + 2 * i + 1], hi[i], lo[i]);
                        block[chunk_at(lane, j)] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        block[chunk_at(lane, 4 + j)] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                    __syncwarp();
                    __half* dst = f.dst->p + (int64_t)tile.b * f.dst->batch_stride;
                    const int64_t to_lo = f.dst->lo, ld = f.dst->ld;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 8 + lane / 4, j = lane % 4;
                        if (r0 + r < f.M && c0 + 8 * j < f.N) {
                            __half* d = dst + (r0 + r) * ld + c0 + 8 * j;
                            *(uint4*)d = block[chunk_at(r, j)];
                            *(uint4*)(d + to_lo) = block[chunk_at(r, 4 + j)];
                        }
                    }
                    if (f.symmetric && row_block > c0 / kTileM) {   // the mirrored block: eight rows of two columns per lane
                        const int r = lane / 8 * 8, p = lane % 8;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int word = i * 8 + p, plane = i / 2, c = c0 + 2 * (word % 16);
                            uint32_t v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = ((const uint32_t*)&block[chunk_at(r + e, word / 4)])[word % 4];
                            if (r0 + r < f.M) {
                                __half* d = dst + plane * to_lo + c * ld + r0 + r;
                                if (c < f.N)
                                    *(uint4*)d = make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[4], v[5], 0x5410),
                                                            __byte_perm(v[6], v[7], 0x5410));
                                if (c + 1 < f.N)
                                    *(uint4*)(d + ld) = make_uint4(__byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632),
                                                                   __byte_perm(v[4], v[5], 0x7632), __byte_perm(v[6], v[7], 0x7632));
                            }
                        }
                    }
                    }
                    __syncwarp();
                }
                return true;
            });
    }
    __syncwarp();
    if (CTAS == 1 && g.split > 1 && warp >= kEpiWarps) {      // the two meetings of the cluster above
        meet<2>();
        meet<2>();
    }
    __syncthreads();
    if (*abort) let_copies_land();          // loads into the ring and products that nobody waited for
    if constexpr (CTAS == 2) meet<2>();     // neither leaves while the other may still signal it
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 9) {
        if constexpr (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols));
    }
}

// ------------------------------------------------------------------ momentum, norm, planes
// NaN stays
__device__ __forceinline__ double at_least(double norm) { return norm < kLeastNorm ? kLeastNorm : norm; }
struct UpdateParams {
    const void* grad;
    int32_t grad_bf16, nesterov;
    const float* momentum;      // null: orthogonalize, U is grad
    float* new_momentum;
    float grad_scale, beta, eps;
    int32_t rows, cols, batch, parts;
    int32_t vec;                // rows of all three start on boundaries of four elements
    int64_t row_stride, batch_stride;   // of grad, momentum, new_momentum
    double* partials;           // [batch][kPartials]
    Planes x;
};
// Four neighbouring elements; those at or beyond `n` are 0 and not touched.
__device__ __forceinline__ float4 load4(const float* p, int n, bool vec) {
    if (vec && n >= 4) return *(const float4*)p;
    float4 v = make_float4(p[0], 0.f, 0.f, 0.f);
    if (n > 1) v.y = p[1];
    if (n > 2) v.z = p[2];
    if (n > 3) v.w = p[3];
    return v;
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p, int n, bool vec) {
    if (vec && n >= 4) {
        const uint2 r = *(const uint2*)p;
        return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xFFFF0000u));
    }
    float4 v = make_float4(__bfloat162float(p[0]), 0.f, 0.f, 0.f);
    if (n > 1) v.y = __bfloat162float(p[1]);
    if (n > 2) v.z = __bfloat162float(p[2]);
    if (n > 3) v.w = __bfloat162float(p[3]);
    return v;
}
__device__ __forceinline__ void store4(float* p, int n, bool vec, float4 v) {
    if (vec && n >= 4) {
        *(float4*)p = v;
        return;
    }
    p[0] = v.x;
    if (n > 1) p[1] = v.y;
    if (n > 2) p[2] = v.z;
    if (n > 3) p[3] = v.w;
}
__device__ __forceinline__ float4 grad4(const UpdateParams& u, int64_t at, int n) {
    return u.grad_bf16 ? load4((const __nv_bfloat16*)u.grad + at, n, u.vec) : load4((const float*)u.grad + at, n, u.vec);
}
__device__ __forceinline__ float4 fma4(float a, float4 x, float4 y) { return make_float4(fmaf(a, x.x, y.x), fmaf(a, x.y, y.y), fmaf(a, x.z, y.z), fmaf(a, x.w, y.w)); }
__device__ __forceinline__ float4 scale4(float a, float4 x) { return make_float4(a * x.x, a * x.y, a * x.z, a * x.w); }

// Both kernels go over a matrix in groups of four columns; a thread has kInFlight of them in flight.
constexpr int kInFlight = 4;

// New momentum, and partial sums of the squares of U.  They are fp64: neither the squares of large nor of small updates leave
// the range.
__global__ void __launch_bounds__(256) update_kernel(const UpdateParams u) {
    __shared__ double part[8];
    const int b = blockIdx.y;
    const int64_t base = (int64_t)b * u.batch_stride;
    const uint32_t per_row = (u.cols + 3) / 4, total = per_row * u.rows, step = gridDim.x * 256;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0;
    for (uint64_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)kInFlight * step) {
        float4 g[kInFlight], m[kInFlight];
        int64_t at[kInFlight];
        int n[kInFlight];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            const uint64_t j = i + (uint64_t)k * step;
            n[k] = 0;
            if (j < total) {
                const uint32_t row = (uint32_t)j / per_row, col = ((uint32_t)j - row * per_row) * 4;
                at[k] = base + (int64_t)row * u.row_stride + col;
                n[k] = u.cols - col;
                g[k] = grad4(u, at[k], n[k]);
                if (u.momentum) m[k] = load4(u.momentum + at[k], n[k], u.vec);
            }
        }
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            if (n[k] <= 0) continue;
            float4 v = g[k];
            if (u.momentum) {
                v = scale4(u.grad_scale, v);
                const float4 nm = fma4(u.beta, m[k], v);
                store4(u.new_momentum + at[k], n[k], u.vec, nm);
                v = u.nesterov ? fma4(u.beta, nm, v) : nm;
                if (n[k] < 4) {                       // what is not there stays 0
                    if (n[k] < 2) v.y = 0.f;
                    if (n[k] < 3) v.z = 0.f;
                    v.w = 0.f;
                }
            }
            sum += (double)v.x * v.x + (double)v.y * v.y + (double)v.z * v.z + (double)v.w * v.w;
        }
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += part[i];
        u.partials[b * kPartials + blockIdx.x] = sum;
    }
}

// X_0 = U / (|U| + eps) as planes.  U is made again from the gradient and the new momentum.
__global__ void __launch_bounds__(256) planes_kernel(const UpdateParams u) {
    __shared__ float factor;
    const int b = blockIdx.y;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x < 32) {
        double sum = 0;
        for (int i = threadIdx.x; i < u.parts; i += 32) sum += u.partials[b * kPartials + i];
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (threadIdx.x == 0) factor = (float)((double)kPlane / at_least(sqrt(sum) + (double)u.eps));
    }
    __syncthreads();
    const float f = factor;
    const int64_t base = (int64_t)b * u.batch_stride;
    __half* planes = u.x.p + (int64_t)b * u.x.batch_stride;
    const uint32_t per_row = (u.cols + 3) / 4, total = per_row * u.rows, step = gridDim.x * 256;
    const bool need_grad = !u.momentum || u.nesterov;
    for (uint64_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)kInFlight * step) {
        float4 g[kInFlight], m[kInFlight];
        int64_t to[kInFlight];
        int n[kInFlight];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            const uint64_t j = i + (uint64_t)k * step;
            n[k] = 0;
            if (j < total) {
                const uint32_t row = (uint32_t)j / per_row, col = ((uint32_t)j - row * per_row) * 4;
                const int64_t at = base + (int64_t)row * u.row_stride + col;
                n[k] = u.cols - col;
                to[k] = (int64_t)row * u.x.ld + col;
                if (need_grad) g[k] = grad4(u, at, n[k]);
                if (u.momentum) m[k] = load4((const float*)u.new_momentum + at, n[k], u.vec);
            }
        }
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            if (n[k] <= 0) continue;
            float4 v = g[k];
            if (u.momentum) v = u.nesterov ? fma4(u.beta, m[k], scale4(u.grad_scale, v)) : m[k];
            v = scale4(f, v);
            uint2 hi, lo;                             // rows of the planes are whole groups of eight
            split2(v.x, v.y, hi.x, lo.x);
            split2(v.z, v.w, hi.y, lo.y);
            *(uint2*)(planes + to[k]) = hi;
            *(uint2*)(planes + u.x.lo + to[k]) = lo;
        }
    }
}

// ------------------------------------------------------------------ small matrices
// A matrix whose shorter side is at most 128 stays on the chip from the gradient to the result: a cluster of up to 8 CTAs holds X,
// 256 of its columns (of its longer side) per CTA, and A and P in shared memory, in the layout the tensor cores read, and the
// epilogues write the next product's operand there themselves.  What bounds it is the chain of 15 products and epilogues;
// as separate launches each took 5 us, most of it the way through L2 (64 x 128, 24 matrices: 80 us in all).
//   X: blocks of 64 columns x 128 rows, 128-byte rows, swizzled.  As an operand of X X^T it has K contiguous, as that of P X
//      its N; both read the same bytes.  A, P: likewise, 1 or 2 blocks.  Everything beyond the matrix is zero.
// With several CTAs, each has part of the sum X X^T; the parts are added through distributed shared memory, each word by one CTA and in
// one order, and all then carry A and P alike.
constexpr int kSmallSide = 128, kSmallCols = 256, kSmallCluster = 8, kSmallThreads = 256;
constexpr int kBlockBytes = 128 * 128;       // a block of 64 columns, one plane
struct SmallParams {
    UpdateParams u;
    Output out;
    int32_t side, length, tall, steps;       // tall: the side runs along the columns in memory
    int32_t cols;                            // columns of X per CTA, a multiple of 64
};

// Chunk (8 columns) j of row r in a block.
__device__ __forceinline__ uint4* chunk_of(uint8_t* block, int r, int j) { return (uint4*)(block + r * 128 + ((j ^ (r & 7)) << 4)); }
// Column c of row r as a 16-bit element
__device__ __forceinline__ __half* element_of(uint8_t* blocks, int r, int c) {
    return (__half*)(blocks + (c >> 6) * kBlockBytes + r * 128 + ((((c >> 3) & 7) ^ (r & 7)) << 4)) + (c & 7);
}

__global__ void __launch_bounds__(kSmallThreads, 1) small_kernel(const SmallParams p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t done_bar;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ double warp_sum[8], cta_sum;
    __shared__ float factor;
    uint8_t* base = (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const int blocks = p.cols / 64, x_plane = blocks * kBlockBytes;
    const int s_blocks = (p.side + 63) / 64, s_cols = s_blocks * 64, a_plane = s_blocks * kBlockBytes;
    uint8_t* const x = base;                               // two planes of X
    uint8_t* const a = base + 2 * x_plane;                 // two planes of A, then of P
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned n_ranks = cluster.num_blocks(), rank = cluster.block_rank();
    const int64_t matrix = blockIdx.x / n_ranks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const int col0 = (int)rank * p.cols, n_cols = min(p.cols, p.length - col0);   // this CTA's columns of X
    const uint32_t done = smem_addr(&done_bar);

    if (tid == 0) {
        abort_flag = 0;
        mbar_init(done, 1);
        mbar_fence_init();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    for (int i = tid; i < 2 * (x_plane + a_plane) / 16; i += kSmallThreads) ((uint4*)base)[i] = make_uint4(0, 0, 0, 0);
    // Only now may the next launch come: were its block to get tensor memory before this one has, this one would wait for it
    // and it for this grid.
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // U in registers, four elements at a time: along the row where that is X's row, else four rows of a column of X, so that
    // neighbouring lanes write neighbouring elements of X either way.
    const UpdateParams& u = p.u;
    const int per_row = (n_cols + 3) / 4, total = p.tall ? (p.side + 3) / 4 * n_cols : p.side * per_row;
    auto place = [&](int i, int& r, int& c) {              // first element in X (c: column of this CTA)
        if (p.tall) {
            r = i / n_cols * 4;
            c = i % n_cols;
        } else {
            r = i / per_row;
            c = i % per_row * 4;
        }
    };
    constexpr int kMost = kSmallSide * kSmallCols / 4 / kSmallThreads, kAtOnce = 8;
    float4 v[kMost];
    double sum = 0;
#pragma unroll
    for (int k0 = 0; k0 < kMost; k0 += kAtOnce) {
        if (k0 * kSmallThreads >= total) break;
        float4 m[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = (k0 + k) * kSmallThreads + tid;
            v[k0 + k] = m[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < total) {
                int r, c;
                place(i, r, c);
                const int64_t at = matrix * u.batch_stride + (p.tall ? (int64_t)(col0 + c) * u.row_stride + r : (int64_t)r * u.row_stride + col0 + c);
                const int n = p.tall ? p.side - r : n_cols - c;
                v[k0 + k] = grad4(u, at, n);
                if (u.momentum) m[k] = load4(u.momentum + at, n, u.vec);
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = (k0 + k) * kSmallThreads + tid;
            if (i < total) {
                float4& e = v[k0 + k];
                if (u.momentum) {
                    int r, c;
                    place(i, r, c);
                    const int64_t at = matrix * u.batch_stride + (p.tall ? (int64_t)(col0 + c) * u.row_stride + r : (int64_t)r * u.row_stride + col0 + c);
                    const int n = p.tall ? p.side - r : n_cols - c;
                    e = scale4(u.grad_scale, e);
                    const float4 nm = fma4(u.beta, m[k], e);
                    store4(u.new_momentum + at, n, u.vec, nm);
                    e = u.nesterov ? fma4(u.beta, nm, e) : nm;
                    if (n < 2) e.y = 0.f;                  // what is not there stays 0
                    if (n < 3) e.z = 0.f;
                    if (n < 4) e.w = 0.f;
                }
                sum += (double)e.x * e.x + (double)e.y * e.y + (double)e.z * e.z + (double)e.w * e.w;
            }
        }
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) warp_sum[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int i = 1; i < 8; ++i) sum += warp_sum[i];
        cta_sum = sum;
    }
    if (n_ranks > 1) cluster.sync();
    if (tid == 0) {
        sum = 0;
        for (unsigned r = 0; r < n_ranks; ++r) sum += n_ranks > 1 ? *cluster.map_shared_rank(&cta_sum, r) : cta_sum;
        factor = (float)((double)kPlane / at_least(sqrt(sum) + (double)u.eps));
    }
    __syncthreads();
    const float f0 = factor;
#pragma unroll
    for (int k = 0; k < kMost; ++k) {
        if (k * kSmallThreads >= total) break;
        const int i = k * kSmallThreads + tid;
        if (i < total) {
            int r, c;
            place(i, r, c);
            const float4 e = scale4(f0, v[k]);
            uint2 hi, lo;
            split2(e.x, e.y, hi.x, lo.x);
            split2(e.z, e.w, hi.y, lo.y);
            if (!p.tall) {
                *(uint2*)element_of(x, r, c) = hi;
                *(uint2*)element_of(x + x_plane, r, c) = lo;
            } else {
                const uint32_t h[2] = {hi.x, hi.y}, l[2] = {lo.x, lo.y};
#pragma unroll
                for (int q = 0; q < 4; ++q) {              // rows beyond the side get the zeros that are there
                    *(uint16_t*)element_of(x, r + q, c) = (uint16_t)(h[q / 2] >> (16 * (q & 1)));
                    *(uint16_t*)element_of(x + x_plane, r + q, c) = (uint16_t)(l[q / 2] >> (16 * (q & 1)));
                }
            }
        }
    }
    const uint32_t tmem = tmem_slot;
    const uint32_t x_addr = smem_addr(x), a_addr = smem_addr(a);
    const uint32_t idesc = 1u << 4 | (uint32_t)(kTileM >> 4) << 24;
    uint32_t phase = 0;
    bool ok = true;
    // The products that `issue` asks for; everyone goes on when they are done.
    auto multiply = [&](auto&& issue) {
        asm volatile("fence.proxy.async;" ::: "memory");            // operands were written by these threads
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            issue();
            mma_commit<1>(done);
        }
        if (!mbar_wait(done, phase, &abort_flag, kResults)) {
            ok = false;
            let_copies_land();                                      // its operands and its accumulators are used again
        }
        __syncwarp();                                               // the loads of accumulators are aligned ones
        phase ^= 1;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    // Accumulators of `width` columns: the first for the small terms, the others take turns with the large ones, as few
    // additions each as there is room for, two at least (see the note on what the tensor core's accumulator cuts off).
    // A 16-bit result takes one.
    auto per_region = [&](int steps, int width) { return p.out.bf16 ? steps : max(2, (steps + 512 / width - 2) / (512 / width - 1)); };
    const int gram_steps = (n_cols + 15) / 16, side_steps = (p.side + 15) / 16;            // of 16 k
    const int gram_per = per_region(gram_steps, s_cols), poly_per = per_region(side_steps, s_cols), apply_per = per_region(side_steps, p.cols);
    auto regions = [](int steps, int per) { return 1 + (steps + per - 1) / per; };
    // One 16-deep product of plane pairs: the small terms into an accumulator of their own, the large ones into `d`.
    auto triple = [&](uint32_t cross, uint32_t d, uint64_t a_hi, uint64_t a_lo, uint64_t b_hi, uint64_t b_lo, uint32_t desc, bool first_cross, bool first) {
        mma_f16<1>(cross, a_hi, b_lo, desc, !first_cross);
        mma_f16<1>(cross, a_lo, b_hi, desc, true);
        mma_f16<1>(d, a_hi, b_hi, desc, !first);
    };
    const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
    const bool rows_used = quad * 32 < p.side;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    // Sum of the accumulators, 32 columns from `c`.
    auto collect = [&](float (&d)[32], int c, int n, int width) {
        uint32_t t[32];
        tmem_load32(lanes + c, t);
#pragma unroll
        for (int i = 0; i < 32; ++i) d[i] = __uint_as_float(t[i]);
#pragma unroll 1
        for (int g = 1; g < n; ++g) {
            tmem_load32(lanes + g * width + c, t);
#pragma unroll
            for (int i = 0; i < 32; ++i) d[i] += __uint_as_float(t[i]);
        }
        if (!ok) {
#pragma unroll
            for (int i = 0; i < 32; ++i) d[i] = __int_as_float(0x7FC00000);
        }
    };
    auto put = [&](uint8_t* planes, int plane, const float (&d)[32], int c) {   // 32 columns of this thread's row
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) split2(d[8 * j + 2 * i], d[8 * j + 2 * i + 1], hi[i], lo[i]);
            uint8_t* block = planes + (c >> 6) * kBlockBytes;
            const int chunk = (c >> 3 & 7) + j;
            *chunk_of(block, row, chunk) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *chunk_of(block + plane, row, chunk) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
    };
    const int s_half = s_cols / 2, s_parts = s_half / 32;          // columns of A of this thread, in parts of 32
    for (int step = 0; step < p.steps; ++step) {
        // A = X X^T
        multiply([&] {
            const uint32_t desc = idesc | (uint32_t)(s_cols >> 3) << 17;
            for (int k = 0, d = tmem + s_cols, n = 0; k < gram_steps; ++k, ++n) {
                if (n == gram_per) d += s_cols, n = 0;
                const uint32_t at = x_addr + k / 4 * kBlockBytes;
                const uint64_t hi = operand_desc(at, false) + k % 4 * 2, lo = operand_desc(at + x_plane, false) + k % 4 * 2;
                triple(tmem, d, hi, lo, hi, lo, desc, k == 0, n == 0);
            }
        });
        float av[2][32];
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (q < s_parts && rows_used) {
                collect(av[q], half * s_half + 32 * q, regions(gram_steps, gram_per), s_cols);
#pragma unroll
                for (int i = 0; i < 32; ++i) av[q][i] *= kUnplane;
            }
        if (n_ranks > 1) {
            // A thread's values lie at the same place in every CTA, in words of four.  Each word is added up by one of the CTAs,
            // which puts the sum back in all of them: every CTA reads and writes each word once over the cluster, where adding
            // up all words everywhere reads them once per CTA (1 x 128 x 2048: 115 us, 204 us that way).
            float4* mine = (float4*)a + tid;
            if (rows_used)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (q < s_parts)
#pragma unroll
                        for (int i = 0; i < 8; ++i) mine[(q * 8 + i) * kSmallThreads] = make_float4(av[q][4 * i], av[q][4 * i + 1], av[q][4 * i + 2], av[q][4 * i + 3]);
            cluster.sync();
            if (rows_used)
                for (int word = (int)rank; word < 8 * s_parts; word += (int)n_ranks) {
                    float4 part[kSmallCluster];
#pragma unroll
                    for (int r = 0; r < kSmallCluster; ++r)
                        if (r < (int)n_ranks) part[r] = cluster.map_shared_rank(mine, r)[word * kSmallThreads];
                    float4 t = part[0];
#pragma unroll
                    for (int r = 1; r < kSmallCluster; ++r)
                        if (r < (int)n_ranks) t = make_float4(t.x + part[r].x, t.y + part[r].y, t.z + part[r].z, t.w + part[r].w);
#pragma unroll
                    for (int r = 0; r < kSmallCluster; ++r)
                        if (r < (int)n_ranks) cluster.map_shared_rank(mine, r)[word * kSmallThreads] = t;
                }
            cluster.sync();
            if (rows_used)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (q < s_parts)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 t = mine[(q * 8 + i) * kSmallThreads];
                            av[q][4 * i] = t.x;
                            av[q][4 * i + 1] = t.y;
                            av[q][4 * i + 2] = t.z;
                            av[q][4 * i + 3] = t.w;
                        }
            __syncthreads();                                       // all have read: the room is A's again
            if (!rows_used)                                        // the parts lay where rows beyond the side are
                for (int c = half * s_half; c < half * s_half + s_half; c += 8) {
                    *chunk_of(a + (c >> 6) * kBlockBytes, row, c >> 3 & 7) = make_uint4(0, 0, 0, 0);
                    *chunk_of(a + a_plane + (c >> 6) * kBlockBytes, row, c >> 3 & 7) = make_uint4(0, 0, 0, 0);
                }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (q < s_parts && rows_used) put(a, a_plane, av[q], half * s_half + 32 * q);
        // P = b A + c A A, in A's place
        multiply([&] {
            const uint32_t desc = idesc | (uint32_t)(s_cols >> 3) << 17;
            for (int k = 0, d = tmem + s_cols, n = 0; k < side_steps; ++k, ++n) {
                if (n == poly_per) d += s_cols, n = 0;
                const uint32_t at = a_addr + k / 4 * kBlockBytes;
                const uint64_t hi = operand_desc(at, false) + k % 4 * 2, lo = operand_desc(at + a_plane, false) + k % 4 * 2;
                triple(tmem, d, hi, lo, hi, lo, desc, k == 0, n == 0);
            }
        });
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (q < s_parts && rows_used) {
                float d[32];
                collect(d, half * s_half + 32 * q, regions(side_steps, poly_per), s_cols);
#pragma unroll
                for (int i = 0; i < 32; ++i) d[i] = fmaf(d[i], kC * kUnplane, kB * av[q][i]);
                put(a, a_plane, d, half * s_half + 32 * q);
            }
        // X = a X + P X, in X's place
        multiply([&] {
            const uint32_t desc = idesc | 1u << 16 | (uint32_t)(p.cols >> 3) << 17;
            const uint64_t lead = (uint64_t)(kBlockBytes >> 4) << 16, own = (uint64_t)(kBoxBytes >> 4) << 16;   // blocks of 64 columns lie 128 rows apart
            for (int k = 0, d = tmem + p.cols, n = 0; k < side_steps; ++k, ++n) {
                if (n == apply_per) d += p.cols, n = 0;
                const uint32_t at = a_addr + k / 4 * kBlockBytes;
                const uint64_t hi = operand_desc(at, false) + k % 4 * 2, lo = operand_desc(at + a_plane, false) + k % 4 * 2;
                const uint64_t x_hi = operand_desc(x_addr + k * 2048, true) - own + lead, x_lo = operand_desc(x_addr + x_plane + k * 2048, true) - own + lead;
                triple(tmem, d, hi, lo, x_hi, x_lo, desc, k == 0, n == 0);
            }
        });
        const bool last = step + 1 == p.steps;
        uint4* turn = (uint4*)a + warp * (kBlockWords / 4);        // P is not needed any more
        if (rows_used)
            for (int q = 0; q < blocks; ++q) {
                const int c = half * (p.cols / 2) + 32 * q;
                float d[32];
                collect(d, c, regions(side_steps, apply_per), p.cols);
                uint8_t* block = x + (c >> 6) * kBlockBytes;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 h = *chunk_of(block, row, (c >> 3 & 7) + j), l = *chunk_of(block + x_plane, row, (c >> 3 & 7) + j);
                    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 e = join(hw[i], lw[i]);
                        d[8 * j + 2 * i] = fmaf(d[8 * j + 2 * i], kUnplane, kA * e.x);
                        d[8 * j + 2 * i + 1] = fmaf(d[8 * j + 2 * i + 1], kUnplane, kA * e.y);
                    }
                }
                if (!last) {
                    put(x, x_plane, d, c);
                    continue;
                }
                const Output& o = p.out;
                const int64_t out0 = matrix * o.batch_stride;
                if (p.tall) {                                      // lanes run along memory
#pragma unroll
                    for (int i0 = 0; i0 < 32; i0 += 8) {
                        float w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int64_t at = out0 + (int64_t)(col0 + c + i0 + i) * o.row_stride + row;
                            w[i] = 0.f;
                            if (o.weight && row < p.side && c + i0 + i < n_cols) w[i] = o.bf16 ? __bfloat162float(((const __nv_bfloat16*)o.weight)[at]) : ((const float*)o.weight)[at];
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int64_t at = out0 + (int64_t)(col0 + c + i0 + i) * o.row_stride + row;
                            float e = d[i0 + i] * kUnplane;
                            if (o.weight) e = fmaf(-o.take, e, o.keep * w[i]);
                            if (row < p.side && c + i0 + i < n_cols) {
                                if (o.bf16) ((__nv_bfloat16*)o.dst)[at] = __float2bfloat16_rn(e);
                                else ((float*)o.dst)[at] = e;
                                if (o.copy) o.copy[at] = __float2bfloat16_rn(e);
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *(float4*)&turn[chunk_at(lane, j)] = make_float4(d[4 * j] * kUnplane, d[4 * j + 1] * kUnplane, d[4 * j + 2] * kUnplane, d[4 * j + 3] * kUnplane);
                    __syncwarp();
                    const int cc = c + 4 * (lane % 8);
                    const int64_t at = out0 + (int64_t)(quad * 32 + lane / 8) * o.row_stride + col0 + cc;
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        float4 w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (o.weight && quad * 32 + 4 * (h + i) + lane / 8 < p.side && cc < n_cols) w[i] = read_weights(o, at + 4 * (h + i) * o.row_stride, n_cols - cc);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float4 e = *(const float4*)&turn[chunk_at(4 * (h + i) + lane / 8, lane % 8)];
                            if (o.weight)
                                e = make_float4(fmaf(-o.take, e.x, o.keep * w[i].x), fmaf(-o.take, e.y, o.keep * w[i].y), fmaf(-o.take, e.z, o.keep * w[i].z),
                                                fmaf(-o.take, e.w, o.keep * w[i].w));
                            if (quad * 32 + 4 * (h + i) + lane / 8 < p.side && cc < n_cols) write_result(o, at + 4 * (h + i) * o.row_stride, n_cols - cc, e);
                        }
                    }
                    __syncwarp();
                }
            }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (n_ranks > 1) cluster.sync();                               // nobody's shared memory goes while others may read it
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// ------------------------------------------------------------------ host side
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static std::atomic<EncodeFn> fn{nullptr};
    EncodeFn f = fn.load(std::memory_order_relaxed);
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        f = (EncodeFn)p;
        fn.store(f, std::memory_order_relaxed);
    }
    return f;
}

constexpr int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// Workspace: X twice, A, P (two planes each), partial sums.
struct Layout {
    int64_t rows, cols, side, ldx, lds, batch;
    int64_t x_plane, s_plane;                       // elements
    uint64_t off_x[2], off_a, off_p, off_part, total;
    Layout(int64_t b, int64_t r, int64_t c) : rows(r), cols(c), side(r < c ? r : c), batch(b) {
        ldx = up(c, 8);
        lds = up(side, 8);
        x_plane = b * r * ldx;
        s_plane = b * side * lds;
        uint64_t at = 0;
        auto take = [&](uint64_t bytes) {
            const uint64_t o = at;
            at += up(bytes, 256);
            return o;
        };
        off_x[0] = take(4 * x_plane);
        off_x[1] = take(4 * x_plane);
        off_a = take(4 * s_plane);
        off_p = take(4 * s_plane);
        off_part = take(8ull * b * kPartials);
        total = at + 256;                           // room to align the start
    }
};

template <typename... Args>
int launch(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? HPL_OK : HPL_ERR_CUDA;
}

struct Device {
    int dev, sms;
    cudaStream_t stream;
};

template <int CTAS, int BN, int MODE>
int launch_ns(const NsParams& g, int units, const Device& d) {
    using C = Config<CTAS, BN>;
    static std::atomic<uint64_t> allowed{0};
    const uint64_t bit = 1ull << (d.dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(ns_kernel<CTAS, BN, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem) != cudaSuccess) return HPL_ERR_CUDA;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch(ns_kernel<CTAS, BN, MODE>, dim3(CTAS * g.split * units), kGemmThreads, C::kSmem, CTAS * g.split, d.stream, g);
}
template <int CTAS, int BN>
int launch_phase(const NsParams& g, int units, const Device& d) {
    const Phase f = phase_at(g, g.phase, CTAS * kTileM, BN);
    const int mode = !f.dst ? kFinal : f.src ? kAddend : kPlanes;
    return mode == kPlanes ? launch_ns<CTAS, BN, kPlanes>(g, units, d) : mode == kAddend ? launch_ns<CTAS, BN, kAddend>(g, units, d) : launch_ns<CTAS, BN, kFinal>(g, units, d);
}
// Tiles of 256 x 256 on pairs of CTAs keep the tensor cores busiest (operands from L2 once per 256 rows and columns); 128 x 128
// and 128 x 64 give more SMs work where the matrix is small.
struct Kind {
    int ctas, bn;
    int block, tile, once;     // measured clocks: 64 k; a tile beside its products; a launch's end
};
constexpr Kind kKinds[3] = {{2, 256, 1750, 20000, 4000}, {1, 128, 1250, 9000, 4000}, {1, 64, 1200, 6000, 4000}};
constexpr int kMeet = 9000, kMaxSplit = 8;       // what it takes to bring parts of a sum together; parts at most

int64_t rounds(int64_t work, int64_t by) { return (work + by - 1) / by; }
struct Plan {
    int kind, split;
    int64_t tiles, time;
};
// The tile, and for few tiles the parts of the sum over k, that are estimated to be fastest: rounds of tiles, each its blocks of
// 64 k and what a tile takes beside them.  Clusters of more than a pair do not fill every SM: seven eighths are counted on.
Plan plan_phase(const NsParams& g, int sms) {
    Plan best = {0, 1, 0, INT64_MAX};
    for (int i = 0; i < 3; ++i) {
        const Kind& k = kKinds[i];
        const Phase f = phase_at(g, g.phase, k.ctas * kTileM, k.bn);
        const int64_t tiles = (int64_t)f.tiles * g.batch, blocks = (f.K + kTileK - 1) / kTileK;
        for (int split = 1; split <= (k.ctas == 1 ? kMaxSplit : 1) && split <= blocks && (split == 1 || tiles * split <= (split == 2 ? sms : sms * 7 / 8)); ++split) {
            if (rounds(blocks, rounds(blocks, split)) != split) continue;       // the last part would be empty
            const int64_t t = rounds(tiles, sms / k.ctas) * (rounds(blocks, split) * k.block + k.tile) + k.once + (split > 1 ? kMeet : 0);
            if (t < best.time) best = {i, split, tiles, t};
        }
    }
    return best;
}
int run_steps(NsParams g, const Device& d) {
    for (g.phase = 0; g.phase < 3 * g.steps; ++g.phase) {
        const Plan p = plan_phase(g, d.sms);
        if (p.tiles > INT32_MAX) return HPL_ERR_INVALID;
        g.split = p.split;
        const int64_t slots = d.sms / kKinds[p.kind].ctas;
        const int units = (int)(p.tiles < slots ? p.tiles : slots);
        const int rc = p.kind == 0 ? launch_phase<2, 256>(g, units, d) : p.kind == 1 ? launch_phase<1, 128>(g, units, d) : launch_phase<1, 64>(g, units, d);
        if (rc) return rc;
    }
    return HPL_OK;
}

// z: the hi planes of all matrices, then the lo planes
bool encode(EncodeFn f, CUtensorMap* map, const Planes& m, int64_t inner, int64_t rows, int64_t batch) {
    const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)(2 * batch)};
    const cuuint64_t strides[2] = {(cuuint64_t)m.ld * 2, (cuuint64_t)m.batch_stride * 2};
    const cuuint32_t box[3] = {64, 64, 1}, step[3] = {1, 1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, m.p, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Problem {
    int64_t batch, rows, cols;
    int32_t steps;
    void* workspace;
    uint64_t workspace_bytes;
};
bool valid(const Problem& q) {
    return q.batch >= 0 && q.batch <= HPL_ORTHO_MAX_BATCH && q.rows >= 1 && q.rows <= HPL_ORTHO_MAX_SIDE && q.cols >= 1 && q.cols <= HPL_ORTHO_MAX_SIDE &&
           q.rows * q.cols <= HPL_ORTHO_MAX_ELEMENTS && q.steps >= 0 && q.steps <= HPL_ORTHO_MAX_STEPS;
}
// 0 stands for contiguous; matrices must not overlap
bool strides(const Problem& q, int64_t& row, int64_t& batch) {
    if (row == 0) row = q.cols;
    if (row < q.cols || row > HPL_ORTHO_MAX_STRIDE) return false;
    if (batch == 0) batch = q.rows * row;
    return q.batch <= 1 || (batch >= (q.rows - 1) * row + q.cols && batch <= HPL_ORTHO_MAX_STRIDE);
}

int launch_small(const UpdateParams& u, const Output& out, int side, int length, const Problem& q, const Device& d) {
    const int ranks = (length + kSmallCols - 1) / kSmallCols;
    SmallParams p = {};
    p.u = u;
    p.out = out;
    p.side = side;
    p.length = length;
    p.tall = q.rows > q.cols;
    p.steps = q.steps;
    p.cols = (int32_t)up((length + ranks - 1) / ranks, 64);
    constexpr size_t whole = kSmSmem - 2 * kBlockReserve;              // the static part is below kBlockReserve
    static_assert(1024 + 2 * kBlockBytes * (kSmallCols / 64 + kSmallSide / 64) <= whole, "the largest case fits");
    const size_t smem = ranks > 1 ? whole : 1024 + 2 * kBlockBytes * (size_t)(p.cols / 64 + (side + 63) / 64);
    static std::atomic<uint64_t> allowed{0};
    const uint64_t bit = 1ull << (d.dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)whole) != cudaSuccess) return HPL_ERR_CUDA;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch(small_kernel, dim3((unsigned)(q.batch * ranks)), kSmallThreads, smem, ranks, d.stream, p);
}

// u and out are complete but for the planes
int orthogonalize(const Problem& q, UpdateParams u, Output out, cudaStream_t stream) {
    const uintptr_t four = out.bf16 ? 8 : 16;
    out.vec = (uintptr_t)out.dst % four == 0 && (uintptr_t)out.weight % four == 0 && (uintptr_t)out.copy % 8 == 0 && out.row_stride % 4 == 0 &&
              (q.batch == 1 || out.batch_stride % 4 == 0);
    const Layout lay(q.batch, q.rows, q.cols);
    if (!q.workspace || q.workspace_bytes < lay.total) return HPL_ERR_INVALID;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return HPL_ERR_CUDA;
    EncodeFn f = encode_fn();
    if (!f || !arm_expiry(stream)) return HPL_ERR_CUDA;
    uint8_t* ws = (uint8_t*)up((int64_t)(uintptr_t)q.workspace, 256);
    Planes x[2], a, p;
    for (int i = 0; i < 2; ++i) x[i] = {(__half*)(ws + lay.off_x[i]), lay.x_plane, q.rows * lay.ldx, (int32_t)lay.ldx};
    a = {(__half*)(ws + lay.off_a), lay.s_plane, lay.side * lay.lds, (int32_t)lay.lds};
    p = {(__half*)(ws + lay.off_p), lay.s_plane, lay.side * lay.lds, (int32_t)lay.lds};
    u.rows = (int32_t)q.rows;
    u.cols = (int32_t)q.cols;
    u.batch = (int32_t)q.batch;
    const uintptr_t of_grad = u.grad_bf16 ? 8 : 16;
    u.vec = (uintptr_t)u.grad % of_grad == 0 && (uintptr_t)u.momentum % 16 == 0 && (uintptr_t)u.new_momentum % 16 == 0 && u.row_stride % 4 == 0 &&
            (q.batch == 1 || u.batch_stride % 4 == 0);
    const Device d{dev, sms, stream};
    const int64_t length = q.rows < q.cols ? q.cols : q.rows;
    // Several CTAs per matrix pay as long as they take few rounds, which are slower here than the tiles of many matrices are there
    // (fp32, 16 x 128 x 2048: 230 us, by tiles 290; 40 x 128 x 2048: 366, by tiles 323).
    const int64_t ranks = (length + kSmallCols - 1) / kSmallCols;
    if (lay.side <= kSmallSide && ranks <= kSmallCluster && (ranks == 1 || q.batch * ranks <= 2 * sms)) return launch_small(u, out, (int)lay.side, (int)length, q, d);
    u.partials = (double*)(ws + lay.off_part);
    // a block for each 4096 elements, up to eight per SM over the batch
    const int64_t most = q.batch < 8 * sms ? 8 * sms / q.batch : 1, blocks = (q.rows * up(q.cols, 4) + 4095) / 4096;
    u.parts = (int32_t)(blocks < most ? blocks : most);
    if (u.parts > kPartials) u.parts = kPartials;
    u.x = x[0];
    int rc = launch(update_kernel, dim3(u.parts, (unsigned)q.batch), 256, 0, 1, stream, u);
    if (rc) return rc;
    rc = launch(planes_kernel, dim3(u.parts, (unsigned)q.batch), 256, 0, 1, stream, u);
    if (rc) return rc;

    NsParams g = {};
    if (!encode(f, &g.maps[0], x[0], q.cols, q.rows, q.batch) || !encode(f, &g.maps[1], x[1], q.cols, q.rows, q.batch) ||
        !encode(f, &g.maps[2], a, lay.side, lay.side, q.batch) || !encode(f, &g.maps[3], p, lay.side, lay.side, q.batch))
        return HPL_ERR_CUDA;
    g.x[0] = x[0];
    g.x[1] = x[1];
    g.a = a;
    g.p = p;
    g.out = out;
    g.rows = (int32_t)q.rows;
    g.cols = (int32_t)q.cols;
    g.side = (int32_t)lay.side;
    g.batch = (int32_t)q.batch;
    g.steps = q.steps;
    return run_steps(g, d);
}

bool aligned_to(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }
uintptr_t element(int32_t dtype) { return dtype == HPL_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == HPL_F32 || dtype == HPL_BF16; }

}  // namespace
}  // namespace hpl

using namespace hpl;

extern "C" uint64_t hpl_orthogonalize_workspace(int32_t batch, int64_t rows, int64_t cols) {
    if (!valid(Problem{batch, rows, cols, 1, nullptr, 0})) return 0;
    return Layout(batch, rows, cols).total;
}

extern "C" int hpl_orthogonalize(const hpl_ortho_args* args, void* cuda_stream) {
    if (!args) return HPL_ERR_INVALID;
    const hpl_ortho_args& a = *args;
    const Problem q{a.batch, a.rows, a.cols, a.steps ? a.steps : 5, a.workspace, a.workspace_bytes};
    int64_t sr = a.src_row_stride, sb = a.src_batch_stride, dr = a.dst_row_stride, db = a.dst_batch_stride;
    if (!valid(q) || !known(a.src_dtype) || !known(a.dst_dtype) || !strides(q, sr, sb) || !strides(q, dr, db)) return HPL_ERR_INVALID;
    if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) return HPL_ERR_INVALID;
    if (a.batch == 0) return HPL_OK;
    if (!a.src || !a.dst || !aligned_to(a.src, element(a.src_dtype)) || !aligned_to(a.dst, element(a.dst_dtype))) return HPL_ERR_INVALID;
    UpdateParams u = {};
    u.grad = a.src;
    u.grad_bf16 = a.src_dtype == HPL_BF16;
    u.eps = a.eps == 0.f ? 1e-7f : a.eps;
    u.row_stride = sr;
    u.batch_stride = sb;
    Output o = {};
    o.dst = a.dst;
    o.bf16 = a.dst_dtype == HPL_BF16;
    o.row_stride = dr;
    o.batch_stride = db;
    return orthogonalize(q, u, o, (cudaStream_t)cuda_stream);
}

extern "C" int hpl_muon_step(const hpl_muon_args* args, void* cuda_stream) {
    if (!args) return HPL_ERR_INVALID;
    const hpl_muon_args& a = *args;
    const Problem q{a.batch, a.rows, a.cols, a.steps ? a.steps : 5, a.workspace, a.workspace_bytes};
    int64_t sr = a.row_stride, sb = a.batch_stride;
    if (!valid(q) || !known(a.grad_dtype) || !known(a.weight_dtype) || !strides(q, sr, sb)) return HPL_ERR_INVALID;
    if (!(a.eps >= 0.f) || !std::isfinite(a.eps) || !std::isfinite(a.grad_scale) || !std::isfinite(a.beta) || !std::isfinite(a.lr) ||
        !std::isfinite(a.weight_decay) || !std::isfinite(a.update_scale))
        return HPL_ERR_INVALID;
    if (a.batch == 0) return HPL_OK;
    if (!a.grad || !a.momentum || !a.new_momentum || !a.weight || !a.new_weight) return HPL_ERR_INVALID;
    if (!aligned_to(a.grad, element(a.grad_dtype)) || !aligned_to(a.momentum, 4) || !aligned_to(a.new_momentum, 4) ||
        !aligned_to(a.weight, element(a.weight_dtype)) || !aligned_to(a.new_weight, element(a.weight_dtype)) || !aligned_to(a.new_copy, 2))
        return HPL_ERR_INVALID;
    UpdateParams u = {};
    u.grad = a.grad;
    u.grad_bf16 = a.grad_dtype == HPL_BF16;
    u.nesterov = a.nesterov != 0;
    u.momentum = a.momentum;
    u.new_momentum = a.new_momentum;
    u.grad_scale = a.grad_scale == 0.f ? 1.f : a.grad_scale;
    u.beta = a.beta;
    u.eps = a.eps == 0.f ? 1e-7f : a.eps;
    u.row_stride = sr;
    u.batch_stride = sb;
    Output o = {};
    o.dst = a.new_weight;
    o.weight = a.weight;
    o.copy = (__nv_bfloat16*)a.new_copy;
    o.bf16 = a.weight_dtype == HPL_BF16;
    o.row_stride = sr;
    o.batch_stride = sb;
    o.keep = (float)(1.0 - (double)a.lr * a.weight_decay);
    o.take = (float)((double)a.lr * (a.update_scale == 0.f ? 1.f : a.update_scale));
    return orthogonalize(q, u, o, (cudaStream_t)cuda_stream);
}
