// Products of microscaled 4-bit records for sm_100a: Y = A * B^T, with one weight matrix or one per segment of rows.
//
// The tensor cores take the records' codes and block scales as they stand (tcgen05.mma with block scaling, 64 channels an
// instruction): codes travel by TMA from the records to shared memory in 128-byte swizzled tiles, 256 channels of a row at a
// time; the scale bytes go through registers, because the tensor cores want the four scales of rows r, r+32, r+64 and r+96
// beside one another (512-byte atoms, copied to tensor memory by tcgen05.cp).  Sums stay in tensor memory in binary32.  The
// row exponents of block 16 are powers of two and commute with the sum: the epilogue applies them.
//
// One pipeline, two shapes of work.
//   wide    many rows: a tile is 128 rows of A by 256 of B; rows of A are the lanes of the accumulator, so a thread holds
//           consecutive values of a row of Y.  Persistent CTAs, one per SM.
//   narrow  few rows (a decode step, a segment of a few tokens): a tile is 128 rows of B by up to 128 of A, so the weights
//           fill the 128 lanes and a handful of tokens costs a handful of columns.  What bounds it is reading the weights;
//           where the tiles alone do not fill the SMs, clusters split the channels and add their partial sums through
//           distributed shared memory in a fixed order.
// Warps 0-3 of a CTA are the epilogue, 4 issues TMA loads, 5 the matrix instructions, 6 and up carry scales.  Every wait on
// an mbarrier is bounded: a copy that never lands ends the kernel with RAC_STATUS_TIMEOUT.
#include <cuda.h>

#include "rac_mx.cuh"

namespace rac {

constexpr int kStageK = 256;             // channels per pipeline stage: one 128-byte row of codes
constexpr int kPRows = 128;              // rows of the operand that fills the accumulator's lanes

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
    int split;                // CTAs of a cluster that share the channels of a tile (narrow), 1 = none
    uint32_t test_extra_tx;   // rac_mx_selftest_bounded_wait: bytes announced beyond what a stage's copies deliver
};

// ------------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 512 bytes of scales (32 rows of 16) to 4 columns of tensor memory, the same in all four groups of 32 lanes
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int BLOCK>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    if constexpr (BLOCK == 16) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(static_cast<uint32_t>(add))
                     : "memory");
    } else {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(static_cast<uint32_t>(add))
                     : "memory");
    }
}
// 16 columns of this thread's lane
__device__ __forceinline__ void tc_load16(uint32_t tmem, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r[i]);
}

// Shared-memory descriptors (address and offsets in units of 16 bytes, version 1 in bit 46).
// Codes: rows of 128 bytes, 128-byte swizzle (2 in the top three bits), 1024 bytes from one group of eight rows to the next.
__device__ __forceinline__ uint64_t desc_codes(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61;
}
// Scales: no swizzle, 128 bytes from one group of eight rows (of 16 bytes) to the next.
__device__ __forceinline__ uint64_t desc_scales(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | 8ull << 16 | 8ull << 32 | 1ull << 46;
}
// Instruction descriptor: both operands e2m1 and K-major, 128 rows by n; scales e4m3 or e8m0; `half`: which two of the four
// scale bytes of a column (block 32).
template <int BLOCK>
__device__ __forceinline__ uint32_t instr_desc(int n, int half) {
    return static_cast<uint32_t>(2 * half) << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(n >> 3) << 17 | (BLOCK == 32 ? 1u << 23 : 0u) |
           1u << 27 | static_cast<uint32_t>(2 * half) << 29;
}

// ------------------------------------------------------------------------------------------------ layout
template <int BLOCK, int QROWS>
struct MxLayout {
    static constexpr bool kWide = QROWS == 256;
    static constexpr int kAtoms = BLOCK == 16 ? 4 : 2;                 // scale atoms per stage and 128 rows
    static constexpr int kQGroups = kWide ? 2 : 1;                     // groups of 128 rows of Q
    static constexpr int kP = kPRows * 128, kQ = QROWS * 128;          // bytes of codes
    static constexpr int kScales = (1 + kQGroups) * kAtoms * 512;
    static constexpr int kStage = kP + kQ + kScales;
    static constexpr int kStages = QROWS == 128 || QROWS == 64 ? 3 : 4;
    static constexpr int kCtrl = 256;
    static constexpr int kExtra = kWide ? 1024 + 4 * 32 * 17 * 4 : 0;  // factors of Q's rows, transposition of odd rows of Y
    static constexpr int kBytes = 1024 + kCtrl + kStages * kStage + kExtra;      // 1024: alignment of the tiles
    static constexpr int kScaleCols = (1 + kQGroups) * kAtoms * 4;     // columns of tensor memory per stage
    static constexpr int kColumns = kWide ? 512 : 256;
    static constexpr int kScaleBase = kWide ? 256 : 128;
    static constexpr int kThreads = 32 * (6 + 1 + kQGroups);
    static_assert(kScaleBase + kStages * kScaleCols <= kColumns, "tensor memory");
    static_assert(kBytes <= 227 * 1024 && (kWide || (kBytes > 77 * 1024 && kBytes <= 113 * 1024)),
                  "narrow: two CTAs an SM and no third, whose columns would not fit");
};
struct MxCtrl {
    unsigned long long full_codes[4], full_scales[4], empty[4], acc_full, acc_empty;
    uint32_t tmem;
    int abort;
};

// ------------------------------------------------------------------------------------------------ tiles
// The rows of tile `t` (all the rows of a warp call this together, with t never falling).
struct Tile {
    int64_t lo, hi;     // rows of A that are left of the segment, from the tile's first
    int64_t matrix;     // first row of B of the segment's matrix
    int64_t n0;         // first row of B within the matrix
    bool valid;
};
template <int MROWS, int NROWS>
struct TileWalk {
    int64_t before = 0;   // tiles along M of the segments before `s`
    int s = 0;
    __device__ __forceinline__ Tile at(const MxProductParams &p, int64_t t) {
        Tile r;
        const int64_t mt = t / p.n_tiles;
        r.n0 = (t - mt * p.n_tiles) * NROWS;
        if (!p.seg_off) {
            r.lo = mt * MROWS;
            r.hi = p.M;
            r.matrix = 0;
            r.valid = r.lo < p.M;
            return r;
        }
        const int lane = threadIdx.x & 31;
        r.valid = false;
        r.lo = r.hi = r.matrix = 0;
        while (s < p.n_seg) {
            int64_t lo = 0, hi = 0;
            if (s + lane < p.n_seg) {
                lo = max(p.seg_off[s + lane], 0);
                hi = min(static_cast<int64_t>(p.seg_off[s + lane + 1]), p.M);
            }
            const int64_t n = hi > lo ? (hi - lo + MROWS - 1) / MROWS : 0;
            int64_t sum = n;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            const uint32_t behind = __ballot_sync(0xffffffffu, before + sum > mt);
            if (behind) {
                const int l = __ffs(behind) - 1;
                before += __shfl_sync(0xffffffffu, sum - n, l);
                s += l;
                r.lo = __shfl_sync(0xffffffffu, lo, l) + (mt - before) * MROWS;
                r.hi = __shfl_sync(0xffffffffu, hi, l);
                r.matrix = static_cast<int64_t>(s) * p.N;
                r.valid = true;
                return r;
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
            s += 32;
        }
        return r;
    }
};

// ------------------------------------------------------------------------------------------------ scales
// The scale bytes of 128 rows and one stage: lane i holds those of rows i, i+32, i+64, i+96.
template <int BLOCK>
struct ScaleChunk {
    uint4 v[4];
    __device__ __forceinline__ void load(const uint8_t *recs, int64_t row0, int64_t rows, int stage, const MxProductParams &p) {
        constexpr int kBytes = kStageK / BLOCK;
        const int left = p.nblk - stage * kBytes;          // what lies behind the scales is not one
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t row = row0 + (threadIdx.x & 31) + 32 * i;
            v[i] = make_uint4(0, 0, 0, 0);
            if (row < rows) {
                const uint8_t *src = recs + row * p.rec + p.scale_off + stage * kBytes;
                if (BLOCK == 16) {
                    v[i] = *reinterpret_cast<const uint4 *>(src);
                } else {
                    const uint2 w = *reinterpret_cast<const uint2 *>(src);
                    v[i].x = w.x;
                    v[i].y = w.y;
                }
                if (left < kBytes) {
                    uint32_t *w = &v[i].x;
#pragma unroll
                    for (int j = 0; j < kBytes / 4; j++) {
                        const int n = left - 4 * j;
                        w[j] &= n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
                    }
                }
                if (BLOCK == 16) {
                    v[i].x &= 0x7f7f7f7fu;
                    v[i].y &= 0x7f7f7f7fu;
                    v[i].z &= 0x7f7f7f7fu;
                    v[i].w &= 0x7f7f7f7fu;
                }
            }
        }
    }
    // atom j: 16 bytes per lane, the four scales of each of its four rows
    __device__ __forceinline__ void store(uint32_t smem) const {
        const uint32_t at = smem + (threadIdx.x & 31) * 16;
        sts128(at, make_uint4(v[0].x, v[1].x, v[2].x, v[3].x));
        sts128(at + 512, make_uint4(v[0].y, v[1].y, v[2].y, v[3].y));
        if (BLOCK == 16) {
            sts128(at + 1024, make_uint4(v[0].z, v[1].z, v[2].z, v[3].z));
            sts128(at + 1536, make_uint4(v[0].w, v[1].w, v[2].w, v[3].w));
        }
    }
};

// ------------------------------------------------------------------------------------------------ results
__device__ __forceinline__ void store_y(const MxProductParams &p, int64_t at, float v) {
    if (p.y_type == RAC_MX_FP32) static_cast<float *>(p.Y)[at] = v;
    else if (p.y_type == RAC_MX_FP16) static_cast<__half *>(p.Y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p.Y)[at] = __float2bfloat16_rn(v);
}
// 16 consecutive values of a row of Y, at an address that is a multiple of 16 bytes
__device__ __forceinline__ void store_y16(const MxProductParams &p, int64_t at, const float (&v)[16]) {
    if (p.y_type == RAC_MX_FP32) {
        float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(p.Y) + at);
#pragma unroll
        for (int i = 0; i < 4; i++) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        return;
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (p.y_type == RAC_MX_FP16) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            w[i] = f2_to_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.Y) + at);
    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// all threads of the cluster
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// a word of the shared memory of the cluster's CTA `rank`, at the place `addr` has in this one's
__device__ __forceinline__ uint32_t cluster_load(uint32_t addr, int rank) {
    uint32_t far, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(far) : "memory");
    return v;
}
__device__ __forceinline__ void epilogue_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------ the kernel
template <int BLOCK, int QROWS>
__global__ void __launch_bounds__(MxLayout<BLOCK, QROWS>::kThreads, MxLayout<BLOCK, QROWS>::kWide ? 1 : 2)
    mx_product_kernel(const MxProductParams p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    using L = MxLayout<BLOCK, QROWS>;
    constexpr bool kWide = L::kWide;
    constexpr int MROWS = kWide ? kPRows : QROWS, NROWS = kWide ? QROWS : kPRows;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = raw + (base - smem_u32(raw));
    const uint32_t stage0 = base, ctrl_at = base + L::kStages * L::kStage;
    MxCtrl *ctrl = reinterpret_cast<MxCtrl *>(base_ptr + L::kStages * L::kStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [&](const unsigned long long *b) { return ctrl_at + static_cast<uint32_t>(reinterpret_cast<const uint8_t *>(b) - reinterpret_cast<const uint8_t *>(ctrl)); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; i++) {
            mbar_init(bar(&ctrl->full_codes[i]), 1);
            mbar_init(bar(&ctrl->full_scales[i]), 1 + L::kQGroups);
            mbar_init(bar(&ctrl->empty[i]), 1);
        }
        mbar_init(bar(&ctrl->acc_full), 1);
        mbar_init(bar(&ctrl->acc_empty), 4);
        ctrl->abort = 0;
        mbar_init_fence();
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl->tmem)), "n"(L::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctrl->tmem;
    grid_dependency_wait();

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
    TileWalk<MROWS, NROWS> walk, walk_sum;
    int it = 0, done = 0;       // stages and tiles that this role has gone through

    // Without split one pass of this loop, in which every role goes through all of the CTA's tiles; with split one per tile.
    for (int64_t t0 = first;; t0 += step) {
        if (warp == 4) {
            // ---- codes: TMA
            bool ok = true;
            for (int64_t t = t0; ok; t += step) {
                const Tile tile = walk.at(p, t);
                if (!tile.valid) break;
                if (lane == 0) {
                    const int row_a = static_cast<int>(tile.lo), row_b = static_cast<int>(tile.matrix + tile.n0);
                    for (int ks = ks0; ks < ks1; ks++, it++) {
                        const int st = it % L::kStages;
                        if (!mbar_wait_bounded(bar(&ctrl->empty[st]), (it / L::kStages & 1) ^ 1) || aborted()) {
                            give_up();
                            ok = false;
                            break;
                        }
                        const uint32_t full = bar(&ctrl->full_codes[st]), dst = stage0 + st * L::kStage;
                        mbar_arrive_expect_tx(full, L::kP + L::kQ + p.test_extra_tx);
                        tma_load_2d(dst, kWide ? &map_a : &map_b, ks * 128, kWide ? row_a : row_b, full);
                        tma_load_2d(dst + L::kP, kWide ? &map_b : &map_a, ks * 128, kWide ? row_b : row_a, full);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (split > 1) break;
            }
            if (!ok && lane == 0) {      // copies in flight must land before the CTA's memory is given back
                for (int i = max(0, it - L::kStages); i < it; i++) mbar_wait_bounded(bar(&ctrl->full_codes[i % L::kStages]), i / L::kStages & 1);
            }
        } else if (warp == 5) {
            // ---- matrix instructions
            bool ok = true;
            for (int64_t t = t0; ok; t += step, done++) {
                const Tile tile = walk.at(p, t);
                if (!tile.valid) break;
                if (lane == 0) {
                    ok = split > 1 || mbar_wait_bounded(bar(&ctrl->acc_empty), (done & 1) ^ 1);
                    tc_fence_after();
                    for (int ks = ks0; ok && ks < ks1; ks++, it++) {
                        const int st = it % L::kStages;
                        const uint32_t phase = it / L::kStages & 1;
                        ok = mbar_wait_bounded(bar(&ctrl->full_codes[st]), phase) && mbar_wait_bounded(bar(&ctrl->full_scales[st]), phase) && !aborted();
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t at = stage0 + st * L::kStage;
                        const uint32_t sp = tmem + L::kScaleBase + st * L::kScaleCols, sq = sp + L::kAtoms * 4;
                        const int mmas = min(4, (p.d - ks * kStageK + 63) / 64), atoms = BLOCK == 16 ? mmas : (mmas + 1) / 2;
                        const uint64_t ds = desc_scales(at + L::kP + L::kQ);
                        for (int j = 0; j < atoms; j++) {
                            tc_copy_scales(sp + 4 * j, ds + j * 32);
#pragma unroll
                            for (int g = 0; g < L::kQGroups; g++)
                                tc_copy_scales(sq + (j * L::kQGroups + g) * 4, ds + ((1 + g) * L::kAtoms + j) * 32);
                        }
                        const uint64_t dp = desc_codes(at), dq = desc_codes(at + L::kP);
                        for (int j = 0; j < mmas; j++) {
                            const int atom = BLOCK == 16 ? j : j / 2, half = BLOCK == 16 ? 0 : j & 1;
                            tc_mma<BLOCK>(tmem, dp + 2 * j, dq + 2 * j, instr_desc<BLOCK>(QROWS, half), sp + 4 * atom,
                                          sq + 4 * L::kQGroups * atom, ks > ks0 || j > 0);
                        }
                        tc_commit(bar(&ctrl->empty[st]));
                    }
                    if (ok) tc_commit(bar(&ctrl->acc_full));
                    else {
                        give_up();                         // what was issued ends before its operands and sums are given back
                        tc_commit(bar(&ctrl->acc_full));
                        mbar_wait_bounded(bar(&ctrl->acc_full), done & 1);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (split > 1) {
                    done++;
                    break;
                }
            }
        } else if (warp >= 6) {
            // ---- scales: warp 6 those of P, the others those of Q, four stages ahead in registers
            const int part = warp - 6;
            const uint8_t *recs = (part == 0) == kWide ? p.A : p.B;
            ScaleChunk<BLOCK> chunk[4];
            int64_t t = t0;
            Tile tile = walk.at(p, t);
            int ks = ks0, loaded = 0, stored = 0;
            auto fetch = [&](ScaleChunk<BLOCK> &c) {
                if (!tile.valid) return;
                const bool of_a = (part == 0) == kWide;
                const int64_t row0 = of_a ? tile.lo : tile.matrix + tile.n0 + (part > 0 ? 128 * (part - 1) : 0);
                const int64_t rows = of_a ? min(tile.hi, tile.lo + MROWS) : tile.matrix + p.N;
                c.load(recs, row0, rows, ks, p);
                loaded++;
                if (++ks == ks1) {
                    ks = ks0;
                    t += step;
                    if (split > 1) tile.valid = false;
                    else tile = walk.at(p, t);
                }
            };
            bool ok = true;
#pragma unroll
            for (int j = 0; j < 3; j++) fetch(chunk[j]);
            while (ok && stored < loaded) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if (!ok || stored >= loaded) break;
                    fetch(chunk[(j + 3) & 3]);
                    const int st = it % L::kStages;
                    ok = mbar_wait_bounded(bar(&ctrl->empty[st]), (it / L::kStages & 1) ^ 1) && !aborted();
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    chunk[j].store(stage0 + st * L::kStage + L::kP + L::kQ + part * L::kAtoms * 512);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&ctrl->full_scales[st]));
                    it++;
                    stored++;
                }
            }
            if (!ok && lane == 0) give_up();
        } else if (split == 1) {
            // ---- epilogue: warps 0-3, 32 lanes of the accumulator each
            float *const factor = reinterpret_cast<float *>(base_ptr + L::kStages * L::kStage + L::kCtrl);
            const uint32_t acc = tmem + (static_cast<uint32_t>(32 * warp) << 16);
            const int exp_off = p.scale_off + p.nblk;
            bool ok = true;
            for (int64_t t = t0; ok; t += step, done++) {
                const Tile tile = walk.at(p, t);
                if (!tile.valid) break;
                const int64_t rows = min(tile.hi - tile.lo, static_cast<int64_t>(MROWS)), cols = min(p.N - tile.n0, static_cast<int64_t>(NROWS));
                const uint8_t *a = p.A + tile.lo * p.rec + exp_off, *b = p.B + (tile.matrix + tile.n0) * p.rec + exp_off;
                const int r = 32 * warp + lane;            // this thread's lane of the accumulator
                int e = 0;
                bool plain = true;                         // exponents so small that their factors multiply without loss
                if (kWide && BLOCK == 16) {
                    epilogue_barrier();                    // the tile before has read its factors
                    e = r < rows ? mx_row_exp(a + r * static_cast<int64_t>(p.rec), 0) : 0;
                    for (int c = r; c < NROWS; c += 128) {
                        const int eb = c < cols ? mx_row_exp(b + c * static_cast<int64_t>(p.rec), 0) : 0;
                        reinterpret_cast<int *>(factor)[c] = eb;
                        plain = plain && eb >= -50 && eb <= 50;
                    }
                    plain = plain && e >= -50 && e <= 50;
                    uint32_t all;
                    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                                 : "=r"(all) : "r"(static_cast<uint32_t>(plain)) : "memory");
                    plain = all != 0;
                } else if (BLOCK == 16) {
                    e = r < cols ? mx_row_exp(b + r * static_cast<int64_t>(p.rec), 0) : 0;
                }
                ok = mbar_wait_bounded(bar(&ctrl->acc_full), done & 1) && !aborted();
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if constexpr (kWide) {
                    const int esize = p.y_type == RAC_MX_FP32 ? 4 : 2;
                    const bool straight = p.N * esize % 16 == 0;
                    float *const turn = factor + 256 + warp * 32 * 17;
                    const float fa = plain ? mx_pow2(e) : 0.0f;
                    for (int c = 0; c < cols; c += 16) {
                        float v[16];
                        tc_load16(acc + c, v);
                        if (BLOCK == 16) {
                            const int4 *eb = reinterpret_cast<const int4 *>(factor + c);
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const int4 x = eb[i];
                                const int xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                for (int j = 0; j < 4; j++)
                                    v[4 * i + j] = plain ? v[4 * i + j] * fa * mx_pow2(xs[j]) : ldexpf(v[4 * i + j], e + xs[j]);
                            }
                        }
                        if (straight && c + 16 <= cols) {
                            if (r < rows) store_y16(p, (tile.lo + r) * p.N + tile.n0 + c, v);
                        } else {
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 16; i++) turn[lane * 17 + i] = v[i];
                            __syncwarp();
#pragma unroll 4
                            for (int i = 0; i < 16; i++) {           // two rows of 16 values at a time
                                const int rr = 2 * i + (lane >> 4), cc = lane & 15;
                                if (32 * warp + rr < rows && c + cc < cols)
                                    store_y(p, (tile.lo + 32 * warp + rr) * p.N + tile.n0 + c + cc, turn[rr * 17 + cc]);
                            }
                        }
                    }
                } else {
                    for (int c = 0; c < rows; c += 16) {      // lanes are rows of B: 32 consecutive values of a row of Y per warp
                        float v[16];
                        tc_load16(acc + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            if (c + i < rows) {
                                const int ea = BLOCK == 16 ? mx_row_exp(a + (c + i) * static_cast<int64_t>(p.rec), 0) : 0;
                                if (r < cols) store_y(p, (tile.lo + c + i) * p.N + tile.n0 + r, BLOCK == 16 ? ldexpf(v[i], e + ea) : v[i]);
                            }
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&ctrl->acc_empty));
            }
            if (!ok && lane == 0) give_up();
        }

        if (split == 1) break;
        if constexpr (!kWide) {
            // ---- one tile per cluster: every CTA lays its partial sums out in its own shared memory (the stages are idle by now:
            // all that was loaded has been multiplied), then each adds up its share of the tokens over all CTAs, in order of rank
            const Tile tile = walk_sum.at(p, t0);
            if (!tile.valid) break;                    // the same for the whole cluster
            float *const part = reinterpret_cast<float *>(base_ptr);       // [QROWS][128]
            const int rows = static_cast<int>(min(tile.hi - tile.lo, static_cast<int64_t>(MROWS)));
            if (warp < 4) {
                bool ok = mbar_wait_bounded(bar(&ctrl->acc_full), done & 1) && !aborted();
                done++;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok && lane == 0) give_up();
                tc_fence_after();
                if (ok) {
                    for (int c = 0; c < rows; c += 16) {
                        float v[16];
                        tc_load16(tmem + (static_cast<uint32_t>(32 * warp) << 16) + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i++) part[(c + i) * 128 + 32 * warp + lane] = v[i];
                    }
                }
                tc_fence_before();
            }
            cluster_barrier();
            bool failed = false;
            for (int q = 0; q < split; q++) failed = failed || cluster_load(smem_u32(&ctrl->abort), q) != 0;
            const int exp_off = p.scale_off + p.nblk;
            const uint8_t *a = p.A + tile.lo * p.rec + exp_off, *b = p.B + (tile.matrix + tile.n0) * p.rec + exp_off;
            const int cols = static_cast<int>(min(p.N - tile.n0, static_cast<int64_t>(NROWS)));
            const int share = (rows * 128 + split - 1) / split;
            for (int i = rank * share + threadIdx.x; !failed && i < min(rows * 128, (rank + 1) * share); i += blockDim.x) {
                const int m = i >> 7, n = i & 127;
                float sum = 0.0f;
                for (int q = 0; q < split; q++) sum += __uint_as_float(cluster_load(smem_u32(part) + 4 * i, q));
                if (n < cols) {
                    int e = 0;
                    if (BLOCK == 16)
                        e = mx_row_exp(a + m * static_cast<int64_t>(p.rec), 0) + mx_row_exp(b + n * static_cast<int64_t>(p.rec), 0);
                    store_y(p, (tile.lo + m) * p.N + tile.n0 + n, BLOCK == 16 ? ldexpf(sum, e) : sum);
                }
            }
            fence_async_smem();       // the next tile's copies come after these reads
            cluster_barrier();        // and nobody leaves while others read its memory
            if (failed) break;
        }
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kColumns) : "memory");
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
// The codes of `rows` records as a matrix of bytes, in boxes of 128 bytes by `box` rows; bytes beyond the codes and rows beyond
// the last read as zero.  Every box starts at a multiple of 128 bytes.
static bool codes_map(CUtensorMap *map, const uint8_t *recs, int64_t rows, const MxProductParams &p, int box) {
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(p.d / 2), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(p.rec)};
    const cuuint32_t boxes[2] = {128, static_cast<cuuint32_t>(box)}, one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(recs), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

template <int BLOCK, int QROWS>
static int launch_mx_product(MxProductParams p, cudaStream_t s) {
    using L = MxLayout<BLOCK, QROWS>;
    constexpr int MROWS = L::kWide ? kPRows : QROWS, NROWS = L::kWide ? QROWS : kPRows;
    const int sms = sm_count();
    if (sms <= 0) return RAC_ECUDA;
    CUtensorMap map_a, map_b;
    if (!codes_map(&map_a, p.A, p.M, p, MROWS) || !codes_map(&map_b, p.B, p.seg_off ? p.n_seg * p.N : p.N, p, NROWS)) return RAC_ECUDA;
    p.n_tiles = static_cast<int>((p.N + NROWS - 1) / NROWS);
    // with segments the lengths are on the device: each may end in a tile that is not full
    int64_t tiles = (p.M + MROWS - 1) / MROWS;
    if (p.seg_off) tiles = p.M < p.n_seg ? p.M : (p.M - p.n_seg) / MROWS + p.n_seg;
    tiles *= p.n_tiles;
    const int64_t slots = L::kWide ? sms : 2 * sms;
    p.split = 1;
    if (!L::kWide)
        while (p.split < 8 && tiles * p.split * 2 <= slots && p.split * 2 <= p.k_stages) p.split *= 2;
    const int64_t ctas = p.split > 1 ? tiles * p.split : (tiles < slots ? tiles : slots);
    auto kernel = mx_product_kernel<BLOCK, QROWS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes) != cudaSuccess) return RAC_ECUDA;
    if (p.split > 1) launch_cluster_after(kernel, static_cast<unsigned>(ctas), p.split, L::kThreads, L::kBytes, s, p, map_a, map_b);
    else launch_after(kernel, static_cast<unsigned>(ctas), L::kThreads, L::kBytes, s, p, map_a, map_b);
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
}

template <int BLOCK>
static int dispatch_mx_product(const MxProductParams &p, cudaStream_t s) {
    // rows per weight matrix, on average
    const int64_t rows = (p.M + p.n_seg - 1) / p.n_seg;
    if (rows > 128) return launch_mx_product<BLOCK, 256>(p, s);
    if (rows > 64) return launch_mx_product<BLOCK, 128>(p, s);
    if (rows > 16) return launch_mx_product<BLOCK, 64>(p, s);
    return launch_mx_product<BLOCK, 16>(p, s);
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
    if (M > 1024 || N > 1024) return RAC_EUNSUPPORTED;
    return mx_product_impl(cfg, A, M, nullptr, 1, B, N, Y, dev_status, stream, 16);
}

}  // extern "C"
