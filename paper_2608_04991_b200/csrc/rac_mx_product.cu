// Products of microscaled 4-bit records for sm_100a: Y = A * B^T, with one weight matrix or one per segment of rows.
//
// The tensor cores take the records' codes and block scales as they stand (tcgen05.mma with block scaling, 64 channels an
// instruction): codes travel by TMA from the records to shared memory in 128-byte swizzled tiles, 256 channels of a row at a
// time, scale bytes by TMA too; eight warps, two for each quarter of tensor memory's lanes, carry the scales from shared to
// tensor memory (tcgen05.st), where lane i holds beside one another the scales of rows i, i+32, i+64 and i+96.  The
// copy instruction made for this (tcgen05.cp) takes its turn between the matrix instructions and held them up: 384 us
// against 220 us without any scales for 16384 x 5120 x 5120 (tiles of single CTAs, no epilogue).  Sums stay in tensor memory
// in binary32.  The row exponents of block 16 are powers of two and commute with the sum: the epilogue applies them.
//
// Two shapes of work.
//   wide    many rows: a pair of CTAs makes a tile of 256 rows of A by 256 (128) of B with cta_group::2, so that each CTA loads
//           half of either operand (38 KB a stage, 54 KB for a tile of 128 x 256 by one CTA, whose loads alone took 214 us of the
//           size above).  Rows of A are the lanes of the accumulator: a thread holds consecutive values of a row of Y.
//           Persistent pairs.  213 us (4.0 PFLOP/s; blocks of 32: 187) in short bursts; in a sustained run the power limit holds it
//           at 250 us.
//   narrow  few rows (a decode step, a segment of a few tokens): a tile is 128 rows of B by up to 64 of A, so the weights
//           fill the 128 lanes and a handful of tokens costs a handful of columns.  What bounds it is the weights' way in, a
//           ring of copies whose round trips are 1.5 to 2.5 us, and for a single token the set-up and the sums' exchange;
//           where the tiles alone do not fill the SMs, clusters split the channels and add their partial sums through
//           distributed shared memory in a fixed order.  1 x 4096 x 4096: 6.6 us; 64 x 5120 x 5120: 10.7 us.  Two CTAs an SM leave 72
//           registers a thread; 92 to 112 bytes a thread go through local memory.
// Times in this file are of blocks of 16 unless stated otherwise, on the device: a call out of 20 in a captured graph that is replayed
// alone, operands in L2 where they fit.  Passes one behind the other through the binding: 6.9 us for one token of 4096 x 4096.
// Warps 0-3 of a CTA are the epilogue, 4-11 carry scales, the next issues TMA loads and the last the matrix
// instructions.  Every wait on an mbarrier is bounded: a copy that never lands ends the kernel with RAC_STATUS_TIMEOUT.
#include <cuda.h>

#include "rac_mx.cuh"

namespace rac {

constexpr int kStageK = 256;             // channels per pipeline stage: one 128-byte row of codes
constexpr int kRows = 128;               // lanes of an accumulator
constexpr int kThreads = 448;

struct MxProductParams {
    const uint8_t *A, *B;
    void *Y;
    const int32_t *seg_off;   // NULL: all rows, one matrix
    uint32_t *status;
    int64_t M, N;
    int n_seg;
    int d, rec, scale_off, nblk, y_type;
    int k_stages;             // ceil(d / 256)
    int n_tiles;              // tiles along N
    int split;                // narrow: CTAs of a cluster that share the channels of a tile, 1 = none
    int y_maps;               // wide: Y has rows that TMA can store
    int early;                // the next kernel on the stream may be set up from the start
    uint32_t test_extra_tx;   // rac_mx_selftest_bounded_wait: bytes announced beyond what a stage's copies deliver
};
struct MxMaps {
    CUtensorMap a, b;              // codes
    CUtensorMap a_scale, b_scale;
    CUtensorMap y;
};

// ------------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Arrival on the barrier at the same place in the cluster's CTA `rank`, and the wait for such arrivals.  What they announce is
// complete when they are made (copies that have landed, stores to tensor memory that were waited for, tensor memory that was
// read) and no ordinary memory passes between the CTAs by them, so they carry no ordering of the whole cluster's memory:
// with .release.cluster and .acquire.cluster 16384 x 5120 x 5120 took 411 us, without 220 us.
__device__ __forceinline__ void mbar_arrive_at(uint32_t bar, uint32_t rank) {
    asm volatile("{\n\t.reg .b32 far;\n\tmapa.shared::cluster.u32 far, %0, %1;\n\t"
                 "mbarrier.arrive.shared::cluster.b64 _, [far];\n\t}" ::"r"(bar), "r"(rank)
                 : "memory");
}
// all threads of the cluster, nothing ordered by it
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
// a place in the shared memory of the cluster's CTA `rank`
__device__ __forceinline__ uint32_t cluster_at(uint32_t addr, uint32_t rank) {
    uint32_t far;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(addr), "r"(rank));
    return far;
}
// copies `bytes` from this CTA's shared memory there, counted on that CTA's mbarrier
__device__ __forceinline__ void cluster_push(uint32_t far, uint32_t src, uint32_t bytes, uint32_t far_bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(far), "r"(src), "r"(bytes), "r"(far_bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// PAIR: instructions for two CTAs at once, issued by the cluster's first; what they commit arrives at both
template <bool PAIR>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
#define RAC_TC_MMA(group, kind)                                                                                    \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"                                               \
                 "tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"           \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(static_cast<uint32_t>(add))           \
                 : "memory")
template <int BLOCK, bool PAIR>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    if constexpr (BLOCK == 16) {
        if constexpr (PAIR) RAC_TC_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X");
        else RAC_TC_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X");
    } else {
        if constexpr (PAIR) RAC_TC_MMA("2", "mxf4.block_scale.scale_vec::2X");
        else RAC_TC_MMA("1", "mxf4.block_scale.scale_vec::2X");
    }
}
// Shared-memory descriptor of codes: rows of 128 bytes, 128-byte swizzle (2 in the top three bits), 1024 bytes from one group of
// eight rows to the next (addresses and offsets in units of 16 bytes, version 1 in bit 46).
__device__ __forceinline__ uint64_t desc_codes(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor: both operands e2m1 and K-major, m rows by n; scales e4m3 or e8m0; `half`: which two of the four
// scale bytes of a column (block 32).
template <int BLOCK>
__device__ __forceinline__ uint32_t instr_desc(int m, int n, int half) {
    return static_cast<uint32_t>(2 * half) << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(n >> 3) << 17 | (BLOCK == 32 ? 1u << 23 : 0u) |
           static_cast<uint32_t>(m >> 7) << 27 | static_cast<uint32_t>(2 * half) << 29;
}

// the matrix instructions of one stage: `n` (4, except at the end of a row) times 64 channels
template <int BLOCK, bool PAIR, int QROWS, int QCOLS>
__device__ __forceinline__ void tc_stage(int n, uint32_t d, uint64_t a, uint64_t b, uint32_t sa, uint32_t sb, bool add) {
    auto one = [&](int j) {
        const int word = BLOCK == 16 ? j : j / 2, half = BLOCK == 16 ? 0 : j & 1;
        tc_mma<BLOCK, PAIR>(d, a + 2 * j, b + 2 * j, instr_desc<BLOCK>(PAIR ? 256 : 128, QROWS, half), sa + 4 * word, sb + QCOLS * word, add || j > 0);
    };
    if (n == 4) {        // written out: this thread keeps the tensor cores busy, and a loop with its descriptors costs 160 cycles a stage
        one(0);
        one(1);
        one(2);
        one(3);
    } else {
        for (int j = 0; j < n; j++) one(j);
    }
}
template <bool PAIR, int COLUMNS>
__device__ __forceinline__ void tc_alloc(uint32_t at) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "n"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "n"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR, int COLUMNS>
__device__ __forceinline__ void tc_free(uint32_t tmem) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLUMNS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLUMNS) : "memory");
}
// 16 columns of this thread's lane; `wait` before they are looked at
__device__ __forceinline__ void tc_load16(uint32_t tmem, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(tmem));
}
__device__ __forceinline__ void tc_load_wait(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
template <int N>
__device__ __forceinline__ void tc_store(uint32_t tmem, const uint32_t *r) {
    static_assert(N == 8 || N == 16, "columns");
    if constexpr (N == 8)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"r"(tmem), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
    else
        asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                     ::"r"(tmem), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                       "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tc_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------ tiles
// The rows of tile `t` (all lanes of a warp call this together, with t never falling).
struct Tile {
    int64_t lo, hi;     // rows of A that are left of the segment, from the tile's first
    int64_t matrix;     // first row of B of the segment's matrix
    int64_t n0;         // first row of B within the matrix
    bool valid;
};
template <int MROWS, int NROWS>
struct TileWalk {
    // 32 segments at a time, one a lane: its rows and the tiles along M up to its end
    int s = -32, lo = 0, hi = 0;
    int64_t sum = 0;
    __device__ __forceinline__ void load(const MxProductParams &p, int64_t before) {
        const int at = s + (threadIdx.x & 31);
        lo = hi = 0;
        if (at < p.n_seg) {
            lo = max(p.seg_off[at], 0);
            hi = static_cast<int>(min(static_cast<int64_t>(p.seg_off[at + 1]), p.M));
        }
        sum = hi > lo ? (static_cast<int64_t>(hi) - lo + MROWS - 1) / MROWS : 0;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t v = __shfl_up_sync(0xffffffffu, sum, o);
            if ((threadIdx.x & 31) >= o) sum += v;
        }
        sum += before;
    }
    __device__ __forceinline__ Tile at(const MxProductParams &p, int64_t t) {
        Tile r;
        const int64_t mt = t <= INT32_MAX ? static_cast<int32_t>(t) / p.n_tiles : t / p.n_tiles;
        r.n0 = (t - mt * p.n_tiles) * NROWS;
        if (!p.seg_off) {
            r.lo = mt * MROWS;
            r.hi = p.M;
            r.matrix = 0;
            r.valid = r.lo < p.M;
            return r;
        }
        r.valid = false;
        r.lo = r.hi = r.matrix = 0;
        if (s < 0) {
            s = 0;
            load(p, 0);
        }
        for (;;) {
            const uint32_t behind = __ballot_sync(0xffffffffu, sum > mt);
            if (behind) {
                const int l = __ffs(behind) - 1;
                r.hi = __shfl_sync(0xffffffffu, hi, l);
                // tiles are counted from the segment's end: the last one is the one that may not be full
                const int first = __shfl_sync(0xffffffffu, lo, l);
                const int64_t tiles = (r.hi - first + MROWS - 1) / MROWS;
                r.lo = first + (tiles - (__shfl_sync(0xffffffffu, sum, l) - mt)) * MROWS;
                r.matrix = static_cast<int64_t>(s + l) * p.N;
                r.valid = true;
                return r;
            }
            if (s + 32 >= p.n_seg) return r;
            const int64_t before = __shfl_sync(0xffffffffu, sum, 31);
            s += 32;
            load(p, before);
        }
    }
};

// ------------------------------------------------------------------------------------------------ scales
template <int BLOCK>
struct Scales {
    static constexpr int kWords = BLOCK == 16 ? 4 : 2;     // words of a row per stage: four scales each
    static constexpr int kBytes = 4 * kWords;
};
// The scales of one stage and 128 rows to tensor memory: word j of row i + 32g to lane i, column 4j + g (times `stride` / 4).
// `at`: where this lane finds the words of row i; `next`: from there to row i + 32.  What lies behind a row's scales (`left`
// of them from the stage's first) counts as 0, and so does bit 7 of an e4m3 scale.
template <int BLOCK, int GROUPS>
__device__ __forceinline__ void load_scales(uint32_t (&w)[Scales<BLOCK>::kWords * 4], uint32_t at, uint32_t next, int left) {
    constexpr int kWords = Scales<BLOCK>::kWords;
#pragma unroll
    for (int g = 0; g < 4; g++) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (g < GROUPS) {
            if constexpr (BLOCK == 16) v = lds128(at + g * next);
            else asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at + g * next));
        }
        const uint32_t vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < kWords; j++) w[4 * j + g] = BLOCK == 16 ? vs[j] & 0x7f7f7f7fu : vs[j];
    }
    if (left < Scales<BLOCK>::kBytes) {
#pragma unroll
        for (int j = 0; j < kWords; j++) {
            const int n = left - 4 * j;
            const uint32_t mask = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
#pragma unroll
            for (int g = 0; g < 4; g++) w[4 * j + g] &= mask;
        }
    }
}

// ------------------------------------------------------------------------------------------------ results
__device__ __forceinline__ void store_y(const MxProductParams &p, int64_t at, float v) {
    if (p.y_type == RAC_MX_FP32) static_cast<float *>(p.Y)[at] = v;
    else if (p.y_type == RAC_MX_FP16) static_cast<__half *>(p.Y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p.Y)[at] = __float2bfloat16_rn(v);
}
// v times 2^e, rounded once (a factor of its own may be beyond binary32)
__device__ __forceinline__ float scaled(float v, int e) { return e >= -126 && e <= 126 ? v * mx_pow2(e) : ldexpf(v, e); }
__device__ __forceinline__ uint32_t pack16(int y_type, float lo, float hi) {
    if (y_type == RAC_MX_FP16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    return f2_to_bf16x2(lo, hi);
}

// ------------------------------------------------------------------------------------------------ narrow
template <int QROWS>
struct NarrowLayout {
    static constexpr int kP = kRows * 128, kQ = QROWS * 128, kPScale = kRows * 16, kQScale = QROWS * 16;   // bytes
    static constexpr int kTx = kP + kQ + kPScale + kQScale;
    static constexpr int kStage = (kTx + 1023) / 1024 * 1024;
    static constexpr int kStages = QROWS == 64 ? 3 : 4;
    // Two teams of four warps carry scales, a stage each in turn.  In an even ring a team has stages of its own and sees every phase
    // of them.  In an odd one the stages change hands: both teams see every copy land and say so, or the ring could go on by two
    // phases before a late warp of the other team has looked, and that warp would wait for a phase that is over.
    static constexpr bool kOwnStages = kStages % 2 == 0;
    static constexpr int kReady = kOwnStages ? 4 : 8;                        // warps that a stage waits for
    // split: what the other CTAs of the cluster push, [rank][token][128] (this CTA's own sums lie in the idle stages)
    static constexpr int kPart = (QROWS == 64 ? 60 : 18) * 512;              // the most that (s - 1) * ceil(QROWS / s) is, up to 8
    static constexpr int kPartAt = kStages * kStage, kCtrlAt = kPartAt + kPart;
    static constexpr int kBytes = 1024 + kCtrlAt + 256;                      // 1024: alignment of the tiles
    static constexpr int kMaxSplit = 8;
    static constexpr int part(int s) { return (s - 1) * ((QROWS + s - 1) / s) * 512; }
    static constexpr int kGroups = QROWS > 32 ? QROWS / 32 : 1;              // groups of 32 rows of Q
    static constexpr int kColumns = 256, kScaleBase = 64, kScaleCols = 32;
    static_assert(kScaleBase + kStages * kScaleCols <= kColumns, "tensor memory");
    static_assert(kBytes > 77 * 1024 && kBytes <= 113 * 1024, "two CTAs an SM and no third, whose columns would not fit");
};
struct NarrowCtrl {
    unsigned long long full[4], ready[4], empty[4], acc_full, acc_empty, parts;
    uint32_t tmem;
    int abort;
};

template <int BLOCK, int QROWS>
__global__ void __launch_bounds__(kThreads, 2) mx_narrow_kernel(const MxProductParams p, const __grid_constant__ MxMaps maps) {
    using L = NarrowLayout<QROWS>;
    constexpr int kWords = Scales<BLOCK>::kWords;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = raw + (base - smem_u32(raw));
    NarrowCtrl *ctrl = reinterpret_cast<NarrowCtrl *>(base_ptr + L::kCtrlAt);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [&](const unsigned long long *b) { return smem_u32(b); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; i++) {
            mbar_init(bar(&ctrl->full[i]), 1);
            mbar_init(bar(&ctrl->ready[i]), L::kReady);
            mbar_init(bar(&ctrl->empty[i]), 1);
        }
        mbar_init(bar(&ctrl->acc_full), 1);
        mbar_init(bar(&ctrl->acc_empty), 4);
        mbar_init(bar(&ctrl->parts), 1);
        ctrl->abort = 0;
        mbar_init_fence();
    }
    if (warp == 12 && lane < 4) tma_prefetch(&maps.a + lane);
    if (warp == 13) tc_alloc<false, L::kColumns>(smem_u32(&ctrl->tmem));
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // not before this CTA has its columns: one of the next kernel's might take them and wait for this grid's end
    if (p.early) grid_launch_dependents();
    const uint32_t tmem = ctrl->tmem;
    if (p.split > 1) cluster_arrive();         // this CTA's barriers are there

    // this CTA's tiles, and its share of the channels of each
    const int split = p.split;
    const int rank = split > 1 ? static_cast<int>(blockIdx.x % split) : 0;
    const int64_t first = blockIdx.x / split, step = gridDim.x / split;
    const int ks0 = rank * p.k_stages / split, ks1 = (rank + 1) * p.k_stages / split;
    auto give_up = [&]() {
        if (p.status) atomicOr(p.status, RAC_STATUS_TIMEOUT);
        *reinterpret_cast<volatile int *>(&ctrl->abort) = 1;
    };
    auto aborted = [&]() { return *reinterpret_cast<volatile int *>(&ctrl->abort) != 0; };
    TileWalk<QROWS, kRows> walk, walk_sum;
    Tile head;                  // the first tile, worked out before the wait where it takes no memory to know it
    if (!p.seg_off) head = walk.at(p, first);
    grid_dependency_wait();
    if (p.seg_off) head = walk.at(p, first);
    int it = 0, done = 0;       // stages and tiles that this role has gone through
    bool pushed = false;
    const int exp_off = p.scale_off + p.nblk;

    // Without split one pass of this loop, in which every role goes through all of the CTA's tiles; with split one per tile.
    for (int64_t t0 = first;; t0 += step) {
        if (warp == 12) {
            // ---- TMA
            bool ok = true;
            for (int64_t t = t0; ok; t += step) {
                const Tile tile = t == first ? head : walk.at(p, t);
                if (!tile.valid) break;
                if (lane == 0) {
                    const int row_a = static_cast<int>(tile.lo), row_b = static_cast<int>(tile.matrix + tile.n0);
                    for (int ks = ks0; ks < ks1; ks++, it++) {
                        const int st = it % L::kStages;
                        if (!mbar_wait_bounded(bar(&ctrl->empty[st]), (it / L::kStages & 1) ^ 1)) {
                            give_up();
                            ok = false;
                            break;
                        }
                        const uint32_t full = bar(&ctrl->full[st]), dst = base + st * L::kStage;
                        const int xs = BLOCK == 16 ? ks * 16 : ks / 2 * 16;       // block 32: 16 bytes are two stages' scales
                        mbar_arrive_expect_tx(full, L::kTx + p.test_extra_tx);
                        tma_load_2d(dst, &maps.b, ks * 128, row_b, full);
                        tma_load_2d(dst + L::kP, &maps.a, ks * 128, row_a, full);
                        tma_load_2d(dst + L::kP + L::kQ, &maps.b_scale, xs, row_b, full);
                        tma_load_2d(dst + L::kP + L::kQ + L::kPScale, &maps.a_scale, xs, row_a, full);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (split > 1) break;
            }
            if (!ok && lane == 0) {      // copies in flight must land before the CTA's memory is given back
                for (int i = max(0, it - L::kStages); i < it; i++) mbar_wait_bounded(bar(&ctrl->full[i % L::kStages]), i / L::kStages & 1);
            }
        } else if (warp == 13) {
            // ---- matrix instructions
            bool ok = true;
            for (int64_t t = t0; ok; t += step) {
                const Tile tile = t == first ? head : walk.at(p, t);
                if (!tile.valid) break;
                if (lane == 0) {
                    ok = split > 1 || mbar_wait_bounded(bar(&ctrl->acc_empty), (done & 1) ^ 1);
                    tc_fence_after();
                    for (int ks = ks0; ok && ks < ks1; ks++, it++) {
                        const int st = it % L::kStages;
                        const uint32_t phase = it / L::kStages & 1;
                        ok = mbar_wait_bounded(bar(&ctrl->full[st]), phase) && mbar_wait_bounded(bar(&ctrl->ready[st]), phase);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t sp = tmem + L::kScaleBase + st * L::kScaleCols, sq = sp + 16;
                        const uint64_t dp = desc_codes(base + st * L::kStage), dq = desc_codes(base + st * L::kStage + L::kP);
                        tc_stage<BLOCK, false, QROWS, 4>(min(4, (p.d - ks * kStageK + 63) / 64), tmem, dp, dq, sp, sq, ks > ks0);
                        tc_commit<false>(bar(&ctrl->empty[st]));
                    }
                    if (!ok) give_up();
                    tc_commit<false>(bar(&ctrl->acc_full));
                    // what was issued ends before its operands and sums are given back
                    if (!ok) mbar_wait_bounded(bar(&ctrl->acc_full), done & 1);
                }
                done++;
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (split > 1) break;
            }
        } else if (warp >= 4) {
            // ---- scales, a quarter of the lanes each; two teams of four warps take turns, a stage each
            const uint32_t quarter = static_cast<uint32_t>(32 * (warp & 3)) << 16;
            const int team = (warp - 4) >> 2;
            bool ok = true;
            for (int64_t t = t0; ok; t += step) {
                const Tile tile = t == first ? head : walk.at(p, t);
                if (!tile.valid) break;
                for (int ks = ks0; ks < ks1; ks++, it++) {
                    const int st = it % L::kStages;
                    const bool mine = (it & 1) == team;
                    if (L::kOwnStages && !mine) continue;
                    ok = mbar_wait_bounded(bar(&ctrl->full[st]), it / L::kStages & 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (!mine) {
                        if (lane == 0) mbar_arrive(bar(&ctrl->ready[st]));
                        continue;
                    }
                    tc_fence_after();
                    const uint32_t at = base + st * L::kStage + L::kP + L::kQ + (BLOCK == 32 ? 8 * (ks & 1) : 0);
                    const int left = p.nblk - ks * Scales<BLOCK>::kBytes;
                    uint32_t wp[kWords * 4], wq[kWords * 4];
                    load_scales<BLOCK, 4>(wp, at + lane * 16, 512, left);
                    load_scales<BLOCK, L::kGroups>(wq, at + L::kPScale + (lane & (QROWS - 1)) * 16, 512, left);
                    const uint32_t to = tmem + quarter + L::kScaleBase + st * L::kScaleCols;
                    tc_store<kWords * 4>(to, wp);
                    tc_store<kWords * 4>(to + 16, wq);
                    tc_store_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&ctrl->ready[st]));
                }
                if (split > 1) break;
            }
            if (!ok && lane == 0) give_up();
        } else if (split == 1) {
            // ---- epilogue, 32 lanes of the accumulator each: lanes are rows of B, 32 consecutive values of a row of Y per warp
            const uint32_t acc = tmem + (static_cast<uint32_t>(32 * warp) << 16);
            const int r = 32 * warp + lane;
            bool ok = true;
            for (int64_t t = t0; ok; t += step, done++) {
                const Tile tile = t == first ? head : walk.at(p, t);
                if (!tile.valid) break;
                const int rows = static_cast<int>(min(tile.hi - tile.lo, static_cast<int64_t>(QROWS)));
                const int cols = static_cast<int>(min(p.N - tile.n0, static_cast<int64_t>(kRows)));
                const uint8_t *a = p.A + tile.lo * p.rec, *b = p.B + (tile.matrix + tile.n0) * p.rec;
                const int eb = BLOCK == 16 && r < cols ? mx_row_exp(b + r * static_cast<int64_t>(p.rec), exp_off) : 0;
                ok = mbar_wait_bounded(bar(&ctrl->acc_full), done & 1) && !aborted();
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                for (int c = 0; c < rows; c += 16) {
                    uint32_t v[16];
                    tc_load16(acc + c, v);
                    const int m = c + (lane & 15);
                    const int ea = BLOCK == 16 && m < rows ? mx_row_exp(a + m * static_cast<int64_t>(p.rec), exp_off) : 0;
                    tc_load_wait(v);
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const int e = BLOCK == 16 ? eb + __shfl_sync(0xffffffffu, ea, i) : 0;
                        const float y = __uint_as_float(v[i]);
                        if (c + i < rows && r < cols) store_y(p, (tile.lo + c + i) * p.N + tile.n0 + r, BLOCK == 16 ? scaled(y, e) : y);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&ctrl->acc_empty));
            }
            if (!ok && lane == 0) give_up();
        }
        if (split == 1) break;

        // ---- one tile per cluster: every CTA lays its partial sums out in its own shared memory, copies to each other CTA those
        // of the tokens that are that one's, and adds up its own tokens in order of rank
        const Tile tile = walk_sum.at(p, t0);
        if (!tile.valid) break;                    // the same for the whole cluster
        const bool more = walk_sum.at(p, t0 + step).valid;             // only where segments overlap
        const int rows = static_cast<int>(min(tile.hi - tile.lo, static_cast<int64_t>(QROWS)));
        const int cols = static_cast<int>(min(p.N - tile.n0, static_cast<int64_t>(kRows)));
        const int each = (rows + split - 1) / split, mine = max(0, min(each, rows - rank * each));     // tokens per CTA, and here
        if (warp < 4) {
            const int n = 32 * warp + lane;        // row of B: this thread's lane of the accumulator
            const uint8_t *a = p.A + (tile.lo + rank * each) * p.rec, *b = p.B + (tile.matrix + tile.n0) * p.rec;
            const uint32_t parts = base + L::kPartAt, own = base;      // the stages: idle once all has been multiplied
            if (threadIdx.x == 0) mbar_arrive_expect_tx(bar(&ctrl->parts), static_cast<uint32_t>((split - 1) * mine * 512));
            const int eb = BLOCK == 16 && n < cols ? mx_row_exp(b + n * static_cast<int64_t>(p.rec), exp_off) : 0;
            int ea = BLOCK == 16 && lane < mine ? mx_row_exp(a + lane * static_cast<int64_t>(p.rec), exp_off) : 0;
            bool ok = mbar_wait_bounded(bar(&ctrl->acc_full), done & 1) && !aborted();
            ok = __all_sync(0xffffffffu, ok);          // one answer a warp, what it read of the flag included
            tc_fence_after();
            if (ok) {
                for (int c = 0; c < rows; c += 16) {
                    uint32_t v[16];
                    tc_load16(tmem + (static_cast<uint32_t>(32 * warp) << 16) + c, v);
                    tc_load_wait(v);
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(own + ((c + i) * 128 + n) * 4), "r"(v[i]) : "memory");
                }
                fence_async_smem();
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (!pushed) cluster_wait();           // all CTAs have their barriers
            if (ok && threadIdx.x < split && threadIdx.x != rank) {
                const int to = threadIdx.x, n_to = min(each, rows - to * each), from = rank < to ? rank : rank - 1;
                if (n_to > 0)
                    cluster_push(cluster_at(parts + from * each * 512, to), own + to * each * 512, n_to * 512, cluster_at(bar(&ctrl->parts), to));
            }
            tc_fence_before();
            if (!more) asm volatile("bar.arrive 2, 160;" ::: "memory");        // tensor memory may go
            if (ok && mine > 0) {
                ok = mbar_wait_bounded(bar(&ctrl->parts), done & 1);
                ok = __all_sync(0xffffffffu, ok);
            }
            const float *mine_at = reinterpret_cast<const float *>(base_ptr) + rank * each * 128 + n;
            const float *parts_at = reinterpret_cast<const float *>(base_ptr + L::kPartAt) + n;
            for (int k = 0; ok && k < mine; k += 4) {          // four tokens at a time: their loads overlap
                float sum[4] = {};
                for (int q = 0; q < split; q++) {
                    const float *src = q == rank ? mine_at + k * 128 : parts_at + ((q < rank ? q : q - 1) * each + k) * 128;
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[i] += k + i < mine ? src[i * 128] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int e = BLOCK == 16 ? eb + __shfl_sync(0xffffffffu, ea, k + i) : 0;
                    if (k + i < mine && n < cols) store_y(p, (tile.lo + rank * each + k + i) * p.N + tile.n0 + n, BLOCK == 16 ? scaled(sum[i], e) : sum[i]);
                }
            }
            if (!ok && lane == 0) give_up();
            done++;
        } else if (!pushed) {
            cluster_wait();
        }
        pushed = true;
        if (!more) break;
        fence_async_smem();       // the next tile's copies come after these reads, and its sums when all have read theirs
        asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
    }
    if (p.split > 1) {
        if (!pushed) {            // no tile for this cluster
            cluster_wait();
            if (warp < 4) asm volatile("bar.arrive 2, 160;" ::: "memory");
        }
        cluster_arrive();         // nobody leaves while another CTA may push to it
        if (warp == 13) {
            asm volatile("bar.sync 2, 160;" ::: "memory");
            tc_fence_after();
            tc_free<false, L::kColumns>(tmem);
        }
        cluster_wait();
    } else {
        tc_fence_before();
        __syncthreads();
        if (warp == 13) {
            tc_fence_after();
            tc_free<false, L::kColumns>(tmem);
        }
    }
}

// ------------------------------------------------------------------------------------------------ wide
template <int BLOCK, int QROWS>
struct WideLayout {
    static constexpr int kHalf = QROWS / 2;                                  // rows of B that one CTA of the pair loads
    static constexpr int kP = kRows * 128, kQ = kHalf * 128, kStage = kP + kQ;
    static constexpr int kStages = 4;
    static constexpr int kQGroups = QROWS / 128;                             // groups of 128 rows of scales of B
    static constexpr int kGroup = 64 / Scales<BLOCK>::kBytes;                // stages whose scales one copy of 64 bytes a row holds
    static constexpr int kScale = (1 + kQGroups) * kRows * 64, kScaleBufs = 2;
    static constexpr int kScaleAt = kStages * kStage, kTurnAt = kScaleAt + kScaleBufs * kScale;
    static constexpr int kTurn = 4096;                                       // 32 rows of 128 bytes of Y; two for each warp
    static constexpr int kFactorAt = kTurnAt + 4 * 2 * kTurn, kCtrlAt = kFactorAt + QROWS * 4;
    static constexpr int kBytes = 1024 + kCtrlAt + 256;
    static constexpr int kAccs = QROWS == 256 ? 1 : 2;                       // accumulators
    static constexpr int kScaleBase = kAccs * QROWS, kScaleCols = (1 + kQGroups) * 16;
    static constexpr int kColumns = 512;
    static_assert(kScaleBase + kStages * kScaleCols <= kColumns && kBytes <= 227 * 1024, "tensor or shared memory");
};
struct WideCtrl {
    unsigned long long full[4], scale_full[2], scale_empty[2], ready[4], empty[4], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort;
};

// whether all 128 threads of the epilogue say so; a barrier for them
__device__ __forceinline__ bool epilogue_all(bool mine) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"(static_cast<uint32_t>(mine)) : "memory");
    return all != 0;
}
// `rows` rows of 128 bytes of Y from shared memory (16-byte piece q of row r at q ^ (r mod 8)) to rows of `cols` values that start
// at `at` and are p.N values apart.
__device__ __forceinline__ void store_turn(const MxProductParams &p, uint32_t turn, int rows, int64_t at, int cols) {
    const int lane = threadIdx.x & 31;
    if (p.y_maps) {               // rows of whole 16-byte pieces: eight lanes a row
        const int esize = p.y_type == RAC_MX_FP32 ? 4 : 2, q = lane & 7;
        uint8_t *const y = static_cast<uint8_t *>(p.Y) + at * esize + 16 * q;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int r = 4 * i + (lane >> 3);
            if (r < rows && q * 16 < cols * esize) *reinterpret_cast<uint4 *>(y + r * p.N * esize) = lds128(turn + r * 128 + (q ^ (r & 7)) * 16);
        }
    } else if (p.y_type == RAC_MX_FP32) {
        float *const y = static_cast<float *>(p.Y) + at + lane;
#pragma unroll 8
        for (int r = 0; r < rows; r++)
            if (lane < cols) y[r * p.N] = __uint_as_float(lds32(turn + r * 128 + ((lane >> 2) ^ (r & 7)) * 16 + (lane & 3) * 4));
    } else {
        // Two values a store wherever a row starts: the words between its first and last even places a row at a time, then what
        // that leaves at either end, a lane for each row (2051 x 2887 x 4096, blocks of 32: 27.4 us; with the ends
        // within the rows' loop 42; 2888 features, which TMA stores, 20.5).
        uint16_t *const y = static_cast<uint16_t *>(p.Y);
        const int odd0 = static_cast<int>(at & 1), turns = static_cast<int>(p.N & 1);             // rows start at even and odd places in turn
        uint16_t *row = y + at + 2 * lane;
        for (int r0 = 0; r0 < rows; r0 += 8) {
            uint32_t w[8], before[8];                                                                // values 2 lane, 2 lane + 1
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = lds32(turn + (r0 + i) * 128 + ((lane >> 2) ^ i) * 16 + (lane & 3) * 4);
#pragma unroll
            for (int i = 0; i < 8; i++) before[i] = __shfl_up_sync(0xffffffffu, w[i], 1);
#pragma unroll
            for (int i = 0; i < 8; i++, row += p.N) {
                const int odd = odd0 ^ (i & turns), c = 2 * lane - odd;
                const uint32_t two = odd ? __funnelshift_l(before[i], w[i], 16) : w[i];              // values c, c + 1
                if (r0 + i < rows && c >= 0 && c + 1 < cols) *reinterpret_cast<uint32_t *>(row - odd) = two;
            }
        }
        auto value = [&](int c) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(turn + lane * 128 + ((c >> 3) ^ (lane & 7)) * 16 + (c & 7) * 2));
            return v;
        };
        const int64_t to = at + lane * p.N;
        const int odd = static_cast<int>(to & 1);
        if (lane < rows && odd) y[to] = value(0);
        if (lane < rows && ((cols - odd) & 1)) y[to + cols - 1] = value(cols - 1);
    }
}

template <int BLOCK, int QROWS>
__global__ void __launch_bounds__(kThreads, 1) mx_wide_kernel(const MxProductParams p, const __grid_constant__ MxMaps maps) {
    using L = WideLayout<BLOCK, QROWS>;
    constexpr int kWords = Scales<BLOCK>::kWords;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = raw + (base - smem_u32(raw));
    WideCtrl *ctrl = reinterpret_cast<WideCtrl *>(base_ptr + L::kCtrlAt);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x & 1;              // of the pair; the first issues the matrix instructions
    auto bar = [&](const unsigned long long *b) { return smem_u32(b); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; i++) {
            mbar_init(bar(&ctrl->full[i]), 1);
            mbar_init(bar(&ctrl->ready[i]), 8);          // four warps of either CTA
            mbar_init(bar(&ctrl->empty[i]), 1);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(bar(&ctrl->scale_full[i]), 1);
            mbar_init(bar(&ctrl->scale_empty[i]), 8);
            mbar_init(bar(&ctrl->acc_full[i]), 1);
            mbar_init(bar(&ctrl->acc_empty[i]), 8);
        }
        ctrl->abort = 0;
        mbar_init_fence();
    }
    if (warp == 12 && lane < 4 + p.y_maps) tma_prefetch(&maps.a + lane);
    if (warp == 13) tc_alloc<true, L::kColumns>(smem_u32(&ctrl->tmem));
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                    // this CTA's barriers are there, and the other's
    cluster_wait();
    tc_fence_after();
    // not before this CTA has its columns: one of the next kernel's might take them and wait for this grid's end
    if (p.early) grid_launch_dependents();
    const uint32_t tmem = ctrl->tmem;

    const int64_t first = blockIdx.x / 2, step = gridDim.x / 2;
    auto give_up = [&]() {
        if (p.status) atomicOr(p.status, RAC_STATUS_TIMEOUT);
        *reinterpret_cast<volatile int *>(&ctrl->abort) = 1;
    };
    auto aborted = [&]() { return *reinterpret_cast<volatile int *>(&ctrl->abort) != 0; };
    TileWalk<2 * kRows, QROWS> walk;
    Tile head;                  // the first tile, worked out before the wait where it takes no memory to know it
    if (!p.seg_off) head = walk.at(p, first);
    grid_dependency_wait();
    if (p.seg_off) head = walk.at(p, first);
    bool ok = true;
    int it = 0, done = 0, group = 0;       // stages, tiles and scale copies that this role has gone through

    if (warp == 12) {
        // ---- TMA
        for (int64_t t = first; ok; t += step) {
            const Tile tile = t == first ? head : walk.at(p, t);
            if (!tile.valid) break;
            if (lane == 0) {
                const int row_a = static_cast<int>(min(tile.lo + rank * kRows, p.M)), row_b = static_cast<int>(tile.matrix + tile.n0);
                for (int ks = 0; ks < p.k_stages; ks++, it++) {
                    if (ks % L::kGroup == 0) {
                        const int sb = group & 1;
                        ok = mbar_wait_bounded(bar(&ctrl->scale_empty[sb]), (group >> 1 & 1) ^ 1) && !aborted();
                        if (!ok) break;
                        const uint32_t full = bar(&ctrl->scale_full[sb]), dst = base + L::kScaleAt + sb * L::kScale;
                        mbar_arrive_expect_tx(full, L::kScale);
                        tma_load_2d(dst, &maps.a_scale, ks / L::kGroup * 64, row_a, full);
#pragma unroll
                        for (int g = 0; g < L::kQGroups; g++)
                            tma_load_2d(dst + (1 + g) * kRows * 64, &maps.b_scale, ks / L::kGroup * 64, row_b + g * kRows, full);
                        group++;
                    }
                    const int st = it % L::kStages;
                    ok = mbar_wait_bounded(bar(&ctrl->empty[st]), (it / L::kStages & 1) ^ 1);
                    if (!ok) break;
                    const uint32_t full = bar(&ctrl->full[st]), dst = base + st * L::kStage;
                    mbar_arrive_expect_tx(full, L::kStage + p.test_extra_tx);
                    tma_load_2d(dst, &maps.a, ks * 128, row_a, full);
                    tma_load_2d(dst + L::kP, &maps.b, ks * 128, row_b + rank * L::kHalf, full);
                }
                if (!ok) give_up();
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
        }
        // Before the CTA's memory is given back the last stages' arrivals have come (the first CTA's matrix instructions make them,
        // with no regard to the barriers at the end), or, where a wait ran out, the copies in flight have landed.
        if (lane == 0) {
            for (int i = max(0, it - L::kStages); i < it; i++)
                mbar_wait_bounded(bar(ok ? &ctrl->empty[i % L::kStages] : &ctrl->full[i % L::kStages]), i / L::kStages & 1);
            for (int i = max(0, group - 2); !ok && i < group; i++) mbar_wait_bounded(bar(&ctrl->scale_full[i & 1]), i >> 1 & 1);
        }
    } else if (warp == 13) {
        // ---- matrix instructions, for both CTAs
        for (int64_t t = first; ok && rank == 0; t += step, done++) {
            const Tile tile = t == first ? head : walk.at(p, t);
            if (!tile.valid) break;
            if (lane == 0) {
                const int ab = done % L::kAccs;
                const uint32_t acc = tmem + ab * QROWS;
                ok = mbar_wait_bounded(bar(&ctrl->acc_empty[ab]), (done / L::kAccs & 1) ^ 1) && !aborted();
                tc_fence_after();
                for (int ks = 0; ok && ks < p.k_stages; ks++, it++) {
                    const int st = it % L::kStages;
                    ok = mbar_wait_bounded(bar(&ctrl->ready[st]), it / L::kStages & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sp = tmem + L::kScaleBase + st * L::kScaleCols, sq = sp + 16;
                    const uint64_t dp = desc_codes(base + st * L::kStage), dq = desc_codes(base + st * L::kStage + L::kP);
                    tc_stage<BLOCK, true, QROWS, 4 * L::kQGroups>(min(4, (p.d - ks * kStageK + 63) / 64), acc, dp, dq, sp, sq, ks > 0);
                    tc_commit<true>(bar(&ctrl->empty[st]));
                }
                if (!ok) give_up();
                tc_commit<true>(bar(&ctrl->acc_full[ab]));
                // what was issued ends before its operands and sums are given back
                if (!ok) mbar_wait_bounded(bar(&ctrl->acc_full[ab]), done / L::kAccs & 1);
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
        }
        // the other CTA's last arrivals have come, or will not any more: the barrier at the end orders none of them
        if (lane == 0) {
            for (int i = max(0, done - L::kAccs); i < done; i++) mbar_wait_bounded(bar(&ctrl->acc_empty[i % L::kAccs]), i / L::kAccs & 1);
        }
    } else if (warp >= 4) {
        // ---- scales, a quarter of the lanes each; two teams of four warps take turns, a stage each
        const uint32_t quarter = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const int team = (warp - 4) >> 2;
        const int turn = lane >> 1 & 3;              // 64-byte swizzle: 16-byte piece c of row r lies at c ^ (r / 2 mod 4)
        for (int64_t t = first; ok; t += step) {
            const Tile tile = t == first ? head : walk.at(p, t);
            if (!tile.valid) break;
            for (int ks = 0; ks < p.k_stages; ks++, it++) {
                const int st = it % L::kStages, sub = ks % L::kGroup, sb = group & 1;
                const bool last = sub == L::kGroup - 1 || ks == p.k_stages - 1;
                // both teams wait for every copy of scales: one that left a copy out could take its phase for the next but one
                // (stages come in fours, so that each team sees every phase of its own)
                if (sub == 0) ok = mbar_wait_bounded(bar(&ctrl->scale_full[sb]), group >> 1 & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                group += last;
                if ((it & 1) != team) {
                    if (last && lane == 0) mbar_arrive(bar(&ctrl->scale_empty[sb]));
                    continue;
                }
                ok = mbar_wait_bounded(bar(&ctrl->full[st]), it / L::kStages & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = base + L::kScaleAt + sb * L::kScale + lane * 64 +
                                    (BLOCK == 16 ? (sub ^ turn) * 16 : (sub / 2 ^ turn) * 16 + 8 * (sub & 1));
                const int left = p.nblk - ks * Scales<BLOCK>::kBytes;
                const uint32_t to = tmem + quarter + L::kScaleBase + st * L::kScaleCols;
                uint32_t w[1 + L::kQGroups][kWords * 4];
#pragma unroll
                for (int g = 0; g < 1 + L::kQGroups; g++) load_scales<BLOCK, 4>(w[g], at + g * kRows * 64, 32 * 64, left);
                tc_store<kWords * 4>(to, w[0]);
                if constexpr (L::kQGroups == 1) {
                    tc_store<kWords * 4>(to + 16, w[1]);
                } else {      // the eight groups of 32 rows beside one another
                    uint32_t q[kWords * 8];
#pragma unroll
                    for (int j = 0; j < kWords; j++)
#pragma unroll
                        for (int g = 0; g < 8; g++) q[8 * j + g] = w[1 + g / 4][4 * j + g % 4];
#pragma unroll
                    for (int j = 0; j < kWords / 2; j++) tc_store<16>(to + 16 + 16 * j, q + 16 * j);
                }
                tc_store_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_at(bar(&ctrl->ready[st]), 0);
                    if (last) mbar_arrive(bar(&ctrl->scale_empty[sb]));
                }
            }
        }
        if (!ok && lane == 0) give_up();
    } else {
        // ---- epilogue: 32 lanes of the accumulator each, 128 bytes of a row of Y at a time, through shared memory
        float *const factor = reinterpret_cast<float *>(base_ptr + L::kFactorAt);
        const uint32_t turn0 = base + L::kTurnAt + warp * 2 * L::kTurn;
        const int exp_off = p.scale_off + p.nblk;
        const int r = 32 * warp + lane;            // this thread's lane of the accumulator
        const bool wide_y = p.y_type == RAC_MX_FP32;
        const int per = wide_y ? 32 : 64;          // values of a row of Y per turn
        int turns = 0;
        for (int64_t t = first;; t += step, done++) {
            const Tile tile = t == first ? head : walk.at(p, t);
            if (!tile.valid) break;
            const int64_t row0 = tile.lo + rank * kRows;
            const int rows = static_cast<int>(max(static_cast<int64_t>(0), min(tile.hi - row0, static_cast<int64_t>(kRows))));
            const int cols = static_cast<int>(min(p.N - tile.n0, static_cast<int64_t>(QROWS)));
            const int ab = done % L::kAccs;
            const uint32_t acc = tmem + ab * QROWS + (static_cast<uint32_t>(32 * warp) << 16);
            // a warp whose wait ran out takes the others with it: nobody is left behind at a barrier of four (block 16: the tile
            // before has read its factors, too)
            if (BLOCK == 16) ok = epilogue_all(ok);
            if (!ok) break;
            int e = 0;
            bool plain = true;                     // exponents so small that their factors multiply without loss
            if (BLOCK == 16) {
                const uint8_t *a = p.A + row0 * p.rec, *b = p.B + (tile.matrix + tile.n0) * p.rec;
                e = r < rows ? mx_row_exp(a + r * static_cast<int64_t>(p.rec), exp_off) : 0;
                plain = e >= -50 && e <= 50;
                for (int c = r; c < QROWS; c += 128) {
                    const int eb = c < cols ? mx_row_exp(b + c * static_cast<int64_t>(p.rec), exp_off) : 0;
                    factor[c] = __int_as_float(eb);
                    plain = plain && eb >= -50 && eb <= 50;
                }
                plain = epilogue_all(plain);
                if (plain) {
                    for (int c = r; c < QROWS; c += 128) factor[c] = mx_pow2(__float_as_int(factor[c]));
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                }
            }
            ok = mbar_wait_bounded(bar(&ctrl->acc_full[ab]), done / L::kAccs & 1) && !aborted();
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) continue;
            tc_fence_after();
            const float fa = plain ? mx_pow2(e) : 0.0f;
            const int mine = min(32, rows - 32 * warp);                  // rows of this warp
            for (int c0 = 0; c0 < cols && mine > 0; c0 += per, turns++) {
                const uint32_t turn = turn0 + (turns & 1) * L::kTurn;
                if (lane == 0) bulk_wait_read<1>();                      // the store before the last has left this buffer
                __syncwarp();
#pragma unroll 1
                for (int c = 0; c < per; c += 32) {
                    uint32_t v[2][16];
                    tc_load16(acc + c0 + c, v[0]);
                    tc_load16(acc + c0 + c + 16, v[1]);
                    tc_load_wait(v[0]);
                    tc_load_wait(v[1]);
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        float y[16];
#pragma unroll
                        for (int i = 0; i < 16; i++) y[i] = __uint_as_float(v[h][i]);
                        if (BLOCK == 16) {
                            const float4 *f = reinterpret_cast<const float4 *>(factor + c0 + c + 16 * h);
                            if (plain) {
#pragma unroll
                                for (int i = 0; i < 4; i++) {
                                    const float4 x = f[i];
                                    y[4 * i] *= fa * x.x;
                                    y[4 * i + 1] *= fa * x.y;
                                    y[4 * i + 2] *= fa * x.z;
                                    y[4 * i + 3] *= fa * x.w;
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; i++) y[i] = ldexpf(y[i], e + __float_as_int(factor[c0 + c + 16 * h + i]));
                            }
                        }
                        // piece q (16 bytes) of a row lies at q ^ (row mod 8): the 128-byte swizzle of the copy
                        if (wide_y) {
#pragma unroll
                            for (int i = 0; i < 4; i++)
                                sts128(turn + lane * 128 + ((4 * h + i) ^ (lane & 7)) * 16,
                                       make_uint4(__float_as_uint(y[4 * i]), __float_as_uint(y[4 * i + 1]), __float_as_uint(y[4 * i + 2]), __float_as_uint(y[4 * i + 3])));
                        } else {
#pragma unroll
                            for (int i = 0; i < 2; i++)
                                sts128(turn + lane * 128 + ((c / 8 + 2 * h + i) ^ (lane & 7)) * 16,
                                       make_uint4(pack16(p.y_type, y[8 * i], y[8 * i + 1]), pack16(p.y_type, y[8 * i + 2], y[8 * i + 3]),
                                                  pack16(p.y_type, y[8 * i + 4], y[8 * i + 5]), pack16(p.y_type, y[8 * i + 6], y[8 * i + 7])));
                        }
                    }
                }
                if (p.y_maps && mine == 32) {
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&maps.y, static_cast<int>(tile.n0) + c0, static_cast<int>(row0) + 32 * warp, turn);
                        bulk_commit();
                    }
                } else {
                    // rows that are not all this segment's, or that start where TMA cannot
                    __syncwarp();
                    store_turn(p, turn, mine, (row0 + 32 * warp) * p.N + tile.n0 + c0, min(per, cols - c0));
                    __syncwarp();
                    if (lane == 0) bulk_commit();      // a group a turn, here without a copy: the wait above counts turns
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(bar(&ctrl->acc_empty[ab]), 0);
        }
        if (lane == 0) bulk_wait_all();
        if (!ok && lane == 0) give_up();
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();           // nobody leaves while the other's instructions read its memory or arrive at its barriers
    if (warp == 13) {
        tc_fence_after();
        tc_free<true, L::kColumns>(tmem);
    }
}

// ------------------------------------------------------------------------------------------------ host
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}
static bool tensor_map(CUtensorMap *map, CUtensorMapDataType type, const void *at, int64_t width, int64_t rows, int64_t stride, int box_w, int box_h,
                       CUtensorMapSwizzle swizzle) {
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(stride)};
    const cuuint32_t boxes[2] = {static_cast<cuuint32_t>(box_w), static_cast<cuuint32_t>(box_h)}, one[2] = {1, 1};
    return fn(map, type, 2, const_cast<void *>(at), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The codes of records as a matrix of bytes, in boxes of 128 bytes by `box` rows, and their scales (with what lies behind them up
// to the next multiple of 16 bytes), in boxes of `width` bytes.  What lies outside reads as zero; every box starts at a
// multiple of its width.
static bool record_maps(CUtensorMap *codes, CUtensorMap *scales, const uint8_t *recs, int64_t rows, const MxProductParams &p, int box, int scale_width,
                        int scale_box) {
    return tensor_map(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, recs, p.d / 2, rows, p.rec, 128, box, CU_TENSOR_MAP_SWIZZLE_128B) &&
           tensor_map(scales, CU_TENSOR_MAP_DATA_TYPE_UINT8, recs + p.scale_off, (p.nblk + 15) / 16 * 16, rows, p.rec, scale_width, scale_box,
                      scale_width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE);
}

// Tiles of `rows` rows of A, at most: with segments the lengths are on the device, and each may end in a tile that is not full.
static int64_t row_tiles(const MxProductParams &p, int rows) {
    if (!p.seg_off) return (p.M + rows - 1) / rows;
    return p.M < p.n_seg ? p.M : (p.M - p.n_seg) / rows + p.n_seg;
}
static int64_t weight_rows(const MxProductParams &p) { return p.seg_off ? p.n_seg * p.N : p.N; }

template <int BLOCK, int QROWS>
static int launch_narrow(MxProductParams p, int sms, cudaStream_t s) {
    using L = NarrowLayout<QROWS>;
    static_assert(L::part(2) <= L::kPart && L::part(3) <= L::kPart && L::part(4) <= L::kPart && L::part(5) <= L::kPart && L::part(6) <= L::kPart &&
                  L::part(7) <= L::kPart && L::part(L::kMaxSplit) <= L::kPart && L::kPartAt >= QROWS * 512, "partial sums");
    MxMaps maps = {};
    if (!record_maps(&maps.a, &maps.a_scale, p.A, p.M, p, QROWS, 16, QROWS) ||
        !record_maps(&maps.b, &maps.b_scale, p.B, weight_rows(p), p, kRows, 16, kRows))
        return RAC_ECUDA;
    p.n_tiles = static_cast<int>((p.N + kRows - 1) / kRows);
    const int64_t tiles = row_tiles(p, QROWS) * p.n_tiles;
    // CTAs of clusters: one per SM where a tile is a few tokens (1 x 4096 x 4096: 128 CTAs 6.6 us, 256 6.8; 1 x 5120 x 5120: 120 and
    // 240 CTAs 7.8, 280, which do not all fit beside one another in clusters, 12.2), more where the tokens are work, too
    // (64 x 5120 x 5120: 120 CTAs 12.8, 240 10.7, 280 18.3).
    const int64_t together = QROWS == 16 ? sms : sms * 5 / 3, slots = 2 * sms;
    p.split = 1;
    while (p.split < L::kMaxSplit && tiles * (p.split + 1) <= together && p.split < p.k_stages) p.split++;
    const int64_t ctas = p.split > 1 ? tiles * p.split : (tiles < slots ? tiles : slots);
    p.early = p.split > 1;
    auto kernel = mx_narrow_kernel<BLOCK, QROWS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes) != cudaSuccess) return RAC_ECUDA;
    if (p.split > 1) launch_cluster_after(kernel, static_cast<unsigned>(ctas), p.split, kThreads, L::kBytes, s, p, maps);
    else launch_after(kernel, static_cast<unsigned>(ctas), kThreads, L::kBytes, s, p, maps);
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
}

template <int BLOCK, int QROWS>
static int launch_wide(MxProductParams p, int sms, cudaStream_t s) {
    using L = WideLayout<BLOCK, QROWS>;
    MxMaps maps = {};
    if (!record_maps(&maps.a, &maps.a_scale, p.A, p.M, p, kRows, 64, kRows) ||
        !record_maps(&maps.b, &maps.b_scale, p.B, weight_rows(p), p, L::kHalf, 64, kRows))
        return RAC_ECUDA;
    const int esize = p.y_type == RAC_MX_FP32 ? 4 : 2;
    p.y_maps = p.N * esize % 16 == 0;
    if (p.y_maps && !tensor_map(&maps.y, p.y_type == RAC_MX_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, p.Y, p.N, p.M,
                                p.N * esize, 128 / esize, 32, CU_TENSOR_MAP_SWIZZLE_128B))
        return RAC_ECUDA;
    p.n_tiles = static_cast<int>((p.N + QROWS - 1) / QROWS);
    const int64_t tiles = row_tiles(p, 2 * kRows) * p.n_tiles, pairs = sms / 2;
    p.early = tiles <= pairs;
    auto kernel = mx_wide_kernel<BLOCK, QROWS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes) != cudaSuccess) return RAC_ECUDA;
    launch_cluster_after(kernel, static_cast<unsigned>(2 * (tiles < pairs ? tiles : pairs)), 2, kThreads, L::kBytes, s, p, maps);
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
}

template <int BLOCK>
static int dispatch_mx_product(const MxProductParams &p, cudaStream_t s) {
    const int sms = mx_sm_count();
    if (sms <= 0) return RAC_ECUDA;
    // By the rows that a weight matrix has, on average.  Few: their own width.  More: the narrow form where its tiles are few
    // enough to be split among five CTAs or more (128 x 1024 x 4096: 8.8 us, wide 10.4), else tiles of 256 x 128 or 256 x 256,
    // whichever takes less time in rounds of all pairs, a stage of the former taking 0.8 times as long as the latter's
    // (256 x 5120 x 5120, one round of either: 12.4 and 14.2 us; 512 rows, two rounds and one: 21.3 and 14.9 us).
    // The lengths of segments are on the device, so uneven ones go by their mean.  32 matrices of 2880 x 2880 (blocks of 32), tiles of 16 /
    // 64 rows of A / 256 x 256: 16 rows each 30 / 32 / 58 us, 64 each 71 / 39 / 53, 65 each 85 / 50 / 57, 128 each 133 / 56 / 54; one segment
    // of 1550 and 31 of 16 (mean 64) 78 / 52 / 65, one of 300 and 31 of 4 (mean 14) 38 / 35 / 56; 16 matrices, one of 2000 rows and 15
    // of 8 (mean 133) 76 / 40 / 36.  2048 x 4096 in blocks of 16, 65 each: 94 / 66 / 57.  At its worst the choice costs an eighth.
    const int64_t rows = (p.M + p.n_seg - 1) / p.n_seg, pairs = sms / 2 > 0 ? sms / 2 : 1;
    if (rows <= 16) return launch_narrow<BLOCK, 16>(p, sms, s);
    if (rows <= 64 || row_tiles(p, 64) * ((p.N + kRows - 1) / kRows) <= sms / 3) return launch_narrow<BLOCK, 64>(p, sms, s);
    const int64_t tall = row_tiles(p, 2 * kRows);
    const int64_t rounds128 = (tall * ((p.N + 127) / 128) + pairs - 1) / pairs, rounds256 = (tall * ((p.N + 255) / 256) + pairs - 1) / pairs;
    if (4 * rounds128 < 5 * rounds256) return launch_wide<BLOCK, 128>(p, sms, s);
    return launch_wide<BLOCK, 256>(p, sms, s);
}

static int mx_product_impl(const rac_mx_cfg *cfg, const void *A, int64_t M, const int32_t *seg_off, int64_t n_seg, const void *B,
                           int64_t N, void *Y, uint32_t *dev_status, void *stream, uint32_t test_extra_tx = 0) {
    MxGeometry g;
    const int rc = mx_geometry(cfg, &g);
    if (rc != RAC_OK) return rc;
    if (M < 0 || N < 0 || n_seg < 0) return RAC_EINVAL;
    if (M > INT32_MAX || N > INT32_MAX || n_seg > 65535 || n_seg * N > INT32_MAX) return RAC_EUNSUPPORTED;
    if (M == 0 || N == 0 || n_seg == 0) return RAC_OK;
    if (!A || !B || !Y) return RAC_EINVAL;
    if (!mx_aligned(A) || !mx_aligned(B) || !mx_aligned(Y)) return RAC_EALIGN;
    const size_t ny = static_cast<size_t>(M) * N * (g.y_type == RAC_MX_FP32 ? 4 : 2);
    if (mx_overlap(Y, ny, A, static_cast<size_t>(M) * g.rec) || mx_overlap(Y, ny, B, static_cast<size_t>(n_seg) * N * g.rec)) return RAC_EINVAL;
    MxProductParams p = {};
    p.A = static_cast<const uint8_t *>(A);
    p.B = static_cast<const uint8_t *>(B);
    p.Y = Y;
    p.seg_off = seg_off;
    p.status = dev_status;
    p.M = M;
    p.N = N;
    p.n_seg = static_cast<int>(n_seg);
    p.d = g.d;
    p.rec = g.rec;
    p.scale_off = g.scale_off;
    p.nblk = g.nblk;
    p.y_type = g.y_type;
    p.test_extra_tx = test_extra_tx;
    p.k_stages = (g.d + kStageK - 1) / kStageK;
    auto s = static_cast<cudaStream_t>(stream);
    return g.block == 16 ? dispatch_mx_product<16>(p, s) : dispatch_mx_product<32>(p, s);
}

}  // namespace rac

using namespace rac;

extern "C" {

int rac_mx_product(const rac_mx_cfg *cfg, const void *A, int64_t M, const void *B, int64_t N, void *Y, uint32_t *dev_status,
                   void *stream) {
    return mx_product_impl(cfg, A, M, nullptr, 1, B, N, Y, dev_status, stream);
}

int rac_mx_product_segments(const rac_mx_cfg *cfg, const void *A, int64_t M, const int32_t *seg_off, int64_t n_seg, const void *B,
                            int64_t N, void *Y, uint32_t *dev_status, void *stream) {
    MxGeometry g;
    if (mx_geometry(cfg, &g) == RAC_OK && M > 0 && N > 0 && n_seg > 0) {
        if (!seg_off) return RAC_EINVAL;
        if (reinterpret_cast<uintptr_t>(seg_off) & 3) return RAC_EALIGN;
    }
    return mx_product_impl(cfg, A, M, seg_off, n_seg, B, N, Y, dev_status, stream);
}

int rac_mx_selftest_bounded_wait(const rac_mx_cfg *cfg, const void *A, int64_t M, const void *B, int64_t N, void *Y,
                                 uint32_t *dev_status, void *stream) {
    if (M > 4096 || N > 4096) return RAC_EUNSUPPORTED;
    return mx_product_impl(cfg, A, M, nullptr, 1, B, N, Y, dev_status, stream, 16);
}

}  // extern "C"
