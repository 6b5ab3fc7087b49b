// What the kernels of the microscaled 4-bit records share: geometry (host) and the conversions between values and codes.
#pragma once

#include "rac_common.cuh"

namespace rac {

struct MxGeometry {
    int d, block, x_type, y_type;
    int nblk;        // blocks (scale bytes) of a row
    int scale_off;   // byte offset of the scales in a record: d/2
    int rec;         // record stride in bytes, a multiple of 32
};
constexpr int kMxMaxD = 32768;
constexpr int kMxMaxExp = 117;   // the largest exponent an encoder writes: 448 * 6 * 2^117 > 2^128

inline int mx_geometry(const rac_mx_cfg *cfg, MxGeometry *g) {
    if (!cfg || cfg->d <= 0) return RAC_EINVAL;
    if (cfg->flags != 0 || (cfg->block != 16 && cfg->block != 32)) return RAC_EUNSUPPORTED;
    if (cfg->d % 32 || cfg->d > kMxMaxD) return RAC_EUNSUPPORTED;
    if (cfg->x_type != RAC_MX_BF16 && cfg->x_type != RAC_MX_FP16) return RAC_EUNSUPPORTED;
    if (cfg->y_type != RAC_MX_BF16 && cfg->y_type != RAC_MX_FP16 && cfg->y_type != RAC_MX_FP32) return RAC_EUNSUPPORTED;
    g->d = cfg->d;
    g->block = cfg->block;
    g->x_type = cfg->x_type;
    g->y_type = cfg->y_type;
    g->nblk = cfg->d / cfg->block;
    g->scale_off = cfg->d / 2;
    g->rec = (g->scale_off + g->nblk + (cfg->block == 16 ? 1 : 0) + 31) / 32 * 32;
    return RAC_OK;
}
inline bool mx_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool mx_overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && a0 < b0 + nb && b0 < a0 + na;
}

inline int mx_sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

// 2^e for e in -126..127
__device__ __forceinline__ float mx_pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// an e8m0 byte below 255
__device__ __forceinline__ float mx_e8m0(uint32_t b) { return __uint_as_float(b ? b << 23 : 0x00400000u); }
// an e4m3 byte, bit 7 not read; 127 is NaN
__device__ __forceinline__ float mx_e4m3(uint32_t b) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(b & 127u)));
    return half_bits_to_float(h & 0xffffu);
}
// row exponent of a record: what a foreign record may hold above kMxMaxExp is taken for that
__device__ __forceinline__ int mx_row_exp(const uint8_t *rec, int off) {
    return min(static_cast<int>(static_cast<int8_t>(rec[off])), kMxMaxExp);
}
// the eight codes of a word as four pairs of binary16 (exact)
__device__ __forceinline__ void mx_e2m1_to_half(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
// eight values to the nearest codes (the even one of two that are equally near), the first in the low bits
__device__ __forceinline__ uint32_t mx_e2m1_from_float(const float2 (&y)[4]) {
    uint32_t w;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(w)
        : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
    return w;
}

}  // namespace rac
