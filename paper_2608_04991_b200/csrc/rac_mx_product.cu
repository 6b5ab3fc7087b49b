// Products of microscaled 4-bit records for sm_100a: Y = A * B^T, with one weight matrix or one per segment of rows.
#include "rac_mx.cuh"

namespace rac {

struct MxProductParams {
    const uint8_t *A, *B;
    void *Y;
    const int32_t *seg_off;   // NULL: all rows, one matrix
    uint32_t *status;
    int64_t M, N;
    int n_seg;
    int d, rec, scale_off, nblk;
};

constexpr int kTile = 64, kSlab = 32;

// 32 channels of 64 rows of records, as code * block scale in binary32
template <int BLOCK>
__device__ __forceinline__ void mx_load_slab(float (*out)[kTile + 4], const uint8_t *recs, int64_t row0, int64_t rows, int k0,
                                             const MxProductParams &p) {
    const int r = threadIdx.x >> 2, q = threadIdx.x & 3;     // a row and 8 of its channels
    uint32_t w = 0;
    float s = 0.0f;
    if (row0 + r < rows) {
        const uint8_t *rec = recs + (row0 + r) * p.rec;
        w = *reinterpret_cast<const uint32_t *>(rec + k0 / 2 + 4 * q);
        const uint32_t b = rec[p.scale_off + (k0 + 8 * q) / BLOCK];
        if (BLOCK == 32) s = b == 255 ? __uint_as_float(0x7fc00000u) : mx_e8m0(b);
        else s = mx_e4m3(b);
    }
    uint32_t h[4];
    mx_e2m1_to_half(w, h);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 v = __half22float2(*reinterpret_cast<__half2 *>(&h[i]));
        out[8 * q + 2 * i][r] = v.x * s;
        out[8 * q + 2 * i + 1][r] = v.y * s;
    }
}

template <int BLOCK, typename Out>
__global__ void __launch_bounds__(256) mx_product_kernel(const MxProductParams p) {
    __shared__ __align__(16) float a[kSlab][kTile + 4], b[kSlab][kTile + 4];
    grid_dependency_wait();
    const uint8_t *B = p.B;
    int64_t m0 = static_cast<int64_t>(blockIdx.y) * kTile, m1 = p.M;
    if (p.seg_off) {                 // the blockIdx.y-th tile over all segments
        int64_t tiles = 0;
        int s = 0;
        for (; s < p.n_seg; s++) {
            const int64_t lo = max(p.seg_off[s], 0), hi = min(static_cast<int64_t>(p.seg_off[s + 1]), p.M);
            const int64_t n = hi > lo ? (hi - lo + kTile - 1) / kTile : 0;
            if (blockIdx.y < tiles + n) {
                m0 = lo + (blockIdx.y - tiles) * kTile;
                m1 = hi;
                break;
            }
            tiles += n;
        }
        if (s == p.n_seg) return;
        B += static_cast<int64_t>(s) * p.N * p.rec;
    }
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < p.d; k0 += kSlab) {
        mx_load_slab<BLOCK>(a, p.A, m0, m1, k0, p);
        mx_load_slab<BLOCK>(b, B, n0, p.N, k0, p);
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < kSlab; k++) {
            const float4 u = *reinterpret_cast<const float4 *>(&a[k][4 * ty]), v = *reinterpret_cast<const float4 *>(&b[k][4 * tx]);
            const float us[4] = {u.x, u.y, u.z, u.w}, vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] += us[i] * vs[j];
        }
        __syncthreads();
    }
    const int exp_off = p.scale_off + p.nblk;
    for (int i = 0; i < 4; i++) {
        const int64_t m = m0 + 4 * ty + i;
        if (m >= m1) break;
        const int em = BLOCK == 16 ? mx_row_exp(p.A + m * p.rec, exp_off) : 0;
        for (int j = 0; j < 4; j++) {
            const int64_t n = n0 + 4 * tx + j;
            if (n >= p.N) break;
            const float v = BLOCK == 16 ? ldexpf(acc[i][j], em + mx_row_exp(B + n * p.rec, exp_off)) : acc[i][j];
            Out *y = static_cast<Out *>(p.Y) + m * p.N + n;
            if constexpr (sizeof(Out) == 4) *y = v;
            else *y = Out(v);
        }
    }
}

template <int BLOCK>
static void launch_mx_product(const MxProductParams &p, int y_type, cudaStream_t s) {
    // segments: at most one tile more than the rows fill, for each of them (and no tile for more segments than rows)
    int64_t tiles = (p.M + kTile - 1) / kTile;
    if (p.seg_off) tiles += p.n_seg;
    const dim3 grid(static_cast<unsigned>((p.N + kTile - 1) / kTile), static_cast<unsigned>(tiles));
    if (y_type == RAC_MX_FP32) mx_product_kernel<BLOCK, float><<<grid, 256, 0, s>>>(p);
    else if (y_type == RAC_MX_FP16) mx_product_kernel<BLOCK, __half><<<grid, 256, 0, s>>>(p);
    else mx_product_kernel<BLOCK, __nv_bfloat16><<<grid, 256, 0, s>>>(p);
}

static int mx_product_impl(const rac_mx_cfg *cfg, const void *A, int64_t M, const int32_t *seg_off, int64_t n_seg, const void *B,
                           int64_t N, void *Y, uint32_t *dev_status, void *stream) {
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
    auto s = static_cast<cudaStream_t>(stream);
    if (g.block == 16) launch_mx_product<16>(p, g.y_type, s);
    else launch_mx_product<32>(p, g.y_type, s);
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
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

}  // extern "C"
