// Microscaled 4-bit records for sm_100a: encode (values to e2m1 codes with block scales, optionally the values they stand
// for in the same pass) and decode.  The products of such records are in rac_mx_product.cu.
//
// Both kernels stream: a thread has 16 consecutive channels (one block of 16, half a block of 32), a CTA has as many whole
// rows as fit its threads.  What bounds them is memory: 2 bytes in and 0.57 (+ 2 with x_hat) out per value.  131072 x 5120, blocks
// of 16: encode with x_hat 477 us in short bursts (6.4 TB/s; 506 to 536 us in sustained runs, where power counts), without 333 us
// (there instruction issue bounds it), decode 293 us (5.9 TB/s).
#include "rac_mx.cuh"

namespace rac {

struct MxParams {
    const uint8_t *X;        // [T,d], two bytes a value
    uint8_t *payload;
    uint8_t *X_hat;
    uint32_t *status;
    int64_t T;
    int d, rec, scale_off, nblk;
    int tpr;                 // threads per row: d/16
    int wide;                // X and X_hat start at multiples of 32 bytes: a thread's values in one access
    int rows;                // rows per CTA and round
    int each;                // rounds of a CTA (encode)
    int early;               // the next kernel on the stream may be set up from the start
};

// A thread's 32 bytes: in one access where they start at a multiple of 32 (two halves of a sector each, stored by two
// instructions, cost decode a third of its rate), else in two.
struct Piece {
    uint32_t w[8];
};
__device__ __forceinline__ Piece load_piece(const uint8_t *src, bool wide) {
    Piece v;
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7])
                     : "l"(src));
    } else {
        const uint4 a = reinterpret_cast<const uint4 *>(src)[0], b = reinterpret_cast<const uint4 *>(src)[1];
        v = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    }
    return v;
}
__device__ __forceinline__ void store_piece(uint8_t *dst, uint4 a, uint4 b, bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(dst), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
    } else {
        reinterpret_cast<uint4 *>(dst)[0] = a;
        reinterpret_cast<uint4 *>(dst)[1] = b;
    }
}

// The eight values of a word of codes times s, in the type of X: four words.
//
// A code has two significant bits and a scale four, so the product is exact in bf16 and, where nothing underflows, in
// binary16.  `fast` (0 or 2^-14 <= s <= 2^13) says that s and every product are exact numbers of both types: then one packed
// multiplication does two values.  bf16: the bits of the binary16 code, shifted down by three, are the code times 2^-112 as
// bf16; the factor is made up for in the scale.  Otherwise binary32, rounded once, no further than the largest finite value.
template <bool HALF>
__device__ __forceinline__ uint4 mx_values(uint32_t w, float s, bool fast) {
    uint32_t h[4], o[4];
    mx_e2m1_to_half(w, h);
    if (fast) {
        if constexpr (HALF) {
            const __half2 f = __float2half2_rn(s);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const __half2 v = __hmul2(*reinterpret_cast<__half2 *>(&h[i]), f);
                o[i] = *reinterpret_cast<const uint32_t *>(&v);
            }
        } else {
            const __nv_bfloat162 f = __float2bfloat162_rn(s * 5.192296858534828e33f);   // 2^112
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t b = (h[i] & 0x80008000u) | ((h[i] >> 3) & 0x0fff0fffu);
                const __nv_bfloat162 v = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&b), f);
                o[i] = *reinterpret_cast<const uint32_t *>(&v);
            }
        }
    } else {
        const float top = HALF ? 65504.0f : __uint_as_float(0x7f7f0000u);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float2 v = __half22float2(*reinterpret_cast<__half2 *>(&h[i]));
            v.x *= s;
            v.y *= s;
            v.x = fabsf(v.x) > top ? copysignf(top, v.x) : v.x;   // a NaN stays one
            v.y = fabsf(v.y) > top ? copysignf(top, v.y) : v.y;
            if constexpr (HALF) {
                const __half2 r = __floats2half2_rn(v.x, v.y);
                o[i] = *reinterpret_cast<const uint32_t *>(&r);
            } else {
                o[i] = f2_to_bf16x2(v.x, v.y);
            }
        }
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ bool mx_fast_scale(float s) { return s == 0.0f || (s >= 6.103515625e-05f && s <= 8192.0f); }

// Codes, scales and exponent of a row, and with XHAT the values they stand for.
//
// The quotient x / s decides integers, so it must not be off where it lands on the middle between two codes.  The reciprocal
// of s is off by an ulp at most; x has at most 11 significant bits and a middle times s at most 7, so a quotient that is not a
// middle is at least 2^-13 away from it.  One fused multiply-add onto 192 = 1.5 * 2^7 rounds the quotient to a multiple of
// 2^-16, which puts a middle where it belongs and moves no other value across one; then the conversion rounds as specified.
//
// The row's exponent needs the whole row: with block 16 a CTA barrier stands between the largest magnitude and the codes.  CTAs
// stay and load their next rows before they work on these, so that the loads go on behind the barrier.
template <bool HALF, int BLOCK, bool XHAT, int CHUNKS, bool STAY>
__global__ void __launch_bounds__(512, CHUNKS > 1 ? 1 : STAY ? 3 : 4) mx_encode_kernel(const MxParams p) {
    extern __shared__ uint32_t row_max[];          // BLOCK 16: bits of the largest finite-block magnitude per row of the CTA, three times
    constexpr uint32_t kInf = HALF ? 0x7c00u : 0x7f80u;
    const int tid = threadIdx.x;
    const int r = tid / p.tpr;                     // row within the CTA (CHUNKS > 1: always 0)
    const int c0 = tid - r * p.tpr;
    const bool wide = p.wide;
    if (p.early) grid_launch_dependents();
    if (BLOCK == 16) {
        for (int i = tid; i < 3 * p.rows; i += blockDim.x) row_max[i] = 0;
    }
    grid_dependency_wait();
    if (BLOCK == 16) __syncthreads();

    // a CTA's rows lie behind one another
    const int64_t step = p.rows, begin = static_cast<int64_t>(blockIdx.x) * p.each * p.rows, end = min(p.T, begin + static_cast<int64_t>(p.each) * p.rows);
    int64_t row = begin + r;
    Piece next[CHUNKS];
    auto fetch = [&](int64_t at) {
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int c = c0 + k * blockDim.x;
            if (r < p.rows && at < end && (CHUNKS == 1 || c < p.tpr)) next[k] = load_piece(p.X + (at * p.d + 16 * static_cast<int64_t>(c)) * 2, wide);
            else next[k] = Piece{};
        }
    };
    fetch(row);
    int slot = 0;
    uint32_t any_bad = 0;
    for (int64_t row0 = begin; row0 < end; row0 = STAY ? row0 + step : end, row += step) {
        const bool live = r < p.rows && row < end;
        Piece x[CHUNKS];
        uint32_t amax[CHUNKS];
        uint32_t bad = 0, most = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) x[k] = next[k];
        if (STAY) fetch(row + step);
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            uint32_t m = x[k].w[0] & 0x7fff7fffu;
#pragma unroll
            for (int i = 1; i < 8; i++) m = __vmaxu2(m, x[k].w[i] & 0x7fff7fffu);
            amax[k] = max(m & 0xffffu, m >> 16);
            if (BLOCK == 32) amax[k] = max(amax[k], __shfl_xor_sync(0xffffffffu, amax[k], 1));
            if (amax[k] >= kInf) {
                bad |= 1u << k;
                amax[k] = 0;
            }
            most = max(most, amax[k]);
        }
        int rexp = 0;
        if (BLOCK == 16) {
            uint32_t *const now = row_max + slot * p.rows;
            slot = slot == 2 ? 0 : slot + 1;
            // the next round's slot: everybody has read it, one round ago
            for (int i = tid; i < p.rows; i += blockDim.x) row_max[slot * p.rows + i] = 0;
            const int first = __shfl_sync(0xffffffffu, r, 0);
            if (__all_sync(0xffffffffu, r == first)) {
                const uint32_t m = __reduce_max_sync(0xffffffffu, most);
                if ((tid & 31) == 0 && first < p.rows && m) atomicMax(&now[first], m);
            } else if (live && most) {
                atomicMax(&now[r], most);
            }
            __syncthreads();
            if (r < p.rows) {
                const uint32_t m16 = now[r];
                const uint32_t f = __float_as_uint(HALF ? half_bits_to_float(m16) : __uint_as_float(m16 << 16));
                // f = 1.m * 2^(e-127): 2688 = 1.3125 * 2^11
                if (f) rexp = max(-100, static_cast<int>(f >> 23) - 138 + ((f & 0x7fffffu) > 0x280000u));
            }
        }
        if (!live) {
            if (STAY) continue;
            break;
        }
        any_bad |= bad;
        uint8_t *rec = p.payload + row * p.rec;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int c = c0 + k * blockDim.x;
            if (CHUNKS > 1 && c >= p.tpr) break;
            const float a = HALF ? half_bits_to_float(amax[k]) : __uint_as_float(amax[k] << 16);
            uint32_t byte;
            float s, inv;
            if (BLOCK == 32) {
                const uint32_t f = __float_as_uint(a);
                const int e = static_cast<int>(f >> 23) - 2 + ((f & 0x7fffffu) > 0x400000u);     // 6 = 1.5 * 2^2
                byte = f ? max(0, e) : 0;
                s = f ? mx_e8m0(byte) : 0.0f;
                inv = __uint_as_float((254u - byte) << 23);
            } else {
                const float b = a * mx_pow2(-rexp);                  // exact, or so small that the first scale serves
                uint16_t q;                                          // nearest e4m3, then the next one where that is too small
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(0.0f), "f"(b * (1.0f / 6.0f)));
                byte = q & 127u;
                byte += mx_e4m3(byte) * (6.0f * mx_pow2(rexp)) < a;  // both exact; a itself, which is not 0 where b may be
                const float v = mx_e4m3(byte);
                s = v * mx_pow2(rexp);
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(v > 0.0f ? v : 1.0f));        // off by an ulp at most; v is no less than 2^-9
                inv *= mx_pow2(-rexp);
            }
            const bool none = bad >> k & 1u;
            if (none) {
                byte = BLOCK == 32 ? 255u : 127u;
                s = __uint_as_float(0x7fc00000u);
            }
            const uint32_t *w = x[k].w;
            const float2 inv2 = make_float2(inv, inv), snap = make_float2(192.0f, 192.0f);
            uint32_t codes[2];
#pragma unroll
            for (int half = 0; half < 2; half++) {
                float2 y[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t u = w[half * 4 + i];
                    const float2 v = HALF ? __half22float2(*reinterpret_cast<const __half2 *>(&u)) : bf16x2_to_f2(u);
                    y[i] = sub2(fma2(v, inv2, snap), snap);
                }
                codes[half] = mx_e2m1_from_float(y);
                // a magnitude of 0 has no sign
                const uint32_t c1 = codes[half] | codes[half] >> 1 | codes[half] >> 2;
                codes[half] &= 0x77777777u | (c1 & 0x11111111u) << 3;
                if (none) codes[half] = 0;
            }
            *reinterpret_cast<uint2 *>(rec + 8 * c) = make_uint2(codes[0], codes[1]);
            if (BLOCK == 16) rec[p.scale_off + c] = static_cast<uint8_t>(byte);
            else if ((c & 1) == 0) rec[p.scale_off + (c >> 1)] = static_cast<uint8_t>(byte);
            if (XHAT) {
                const bool fast = mx_fast_scale(s);
                store_piece(p.X_hat + (row * p.d + 16 * static_cast<int64_t>(c)) * 2, mx_values<HALF>(codes[0], s, fast),
                            mx_values<HALF>(codes[1], s, fast), wide);
            }
        }
        // behind the scales: the exponent, zeros
        const int skip = CHUNKS > 1 ? static_cast<int>(blockDim.x) : p.tpr;
        for (int i = p.scale_off + p.nblk + c0; i < p.rec; i += skip)
            rec[i] = BLOCK == 16 && i == p.scale_off + p.nblk ? static_cast<uint8_t>(rexp) : 0;
    }
    if (any_bad && p.status) atomicOr(p.status, RAC_STATUS_NONFINITE);
}

template <bool HALF, int BLOCK>
__global__ void __launch_bounds__(512) mx_decode_kernel(const MxParams p) {
    const int r = threadIdx.x / p.tpr;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * p.rows + r;
    if (p.early) grid_launch_dependents();
    grid_dependency_wait();
    if (r >= p.rows || row >= p.T) return;
    const uint8_t *rec = p.payload + row * p.rec;
    for (int c = threadIdx.x - r * p.tpr; c < p.tpr; c += blockDim.x) {
        const uint2 codes = *reinterpret_cast<const uint2 *>(rec + 8 * c);
        float s;
        if (BLOCK == 32) {
            const uint32_t b = rec[p.scale_off + (c >> 1)];
            s = b == 255 ? __uint_as_float(0x7fc00000u) : mx_e8m0(b);
        } else {
            const int e = mx_row_exp(rec, p.scale_off + p.nblk);
            s = mx_e4m3(rec[p.scale_off + c]) * mx_pow2(max(e, -126)) * (e < -126 ? mx_pow2(e + 126) : 1.0f);
        }
        const bool fast = mx_fast_scale(s);
        store_piece(p.X_hat + (row * p.d + 16 * static_cast<int64_t>(c)) * 2, mx_values<HALF>(codes.x, s, fast), mx_values<HALF>(codes.y, s, fast),
                    p.wide);
        if (p.tpr <= static_cast<int>(blockDim.x)) break;      // several rows of the CTA: one piece per thread
    }
}

// CTAs of whole rows, 256 threads or one row's; `rounds`: the most rows (groups of rows) that a CTA takes one after the other
static int mx_shape(const MxGeometry &g, int64_t T, const void *X, const void *X_hat, int rounds, MxParams *p, unsigned *grid, unsigned *threads) {
    const int sms = mx_sm_count();
    if (sms <= 0) return RAC_ECUDA;
    p->T = T;
    p->d = g.d;
    p->rec = g.rec;
    p->scale_off = g.scale_off;
    p->nblk = g.nblk;
    p->wide = ((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(X_hat)) & 31) == 0;
    p->tpr = g.d / 16;
    p->rows = p->tpr >= 256 ? 1 : 256 / p->tpr;
    if (p->rows > T) p->rows = static_cast<int>(T);
    const int t = p->rows * p->tpr;
    *threads = static_cast<unsigned>(t > 512 ? 512 : (t + 31) / 32 * 32);
    const int64_t groups = (T + p->rows - 1) / p->rows;
    int64_t each = groups * *threads / (static_cast<int64_t>(sms) * 2048 * 2);       // two full rounds of the SMs at least
    each = each < 3 ? 1 : each > rounds ? rounds : each;
    p->each = static_cast<int>(each);
    *grid = static_cast<unsigned>((groups + each - 1) / each);
    p->early = groups * *threads <= static_cast<int64_t>(sms) * 1024;
    return RAC_OK;
}

template <bool HALF, int BLOCK, bool XHAT>
static void launch_mx_encode(const MxParams &p, unsigned grid, unsigned threads, cudaStream_t s) {
    const size_t smem = BLOCK == 16 ? 3 * sizeof(uint32_t) * p.rows : 0;
    const bool stay = p.each > 1;
    if (p.tpr > 1024) stay ? launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 4, true>, grid, threads, smem, s, p)
                           : launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 4, false>, grid, threads, smem, s, p);
    else if (p.tpr > 512) stay ? launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 2, true>, grid, threads, smem, s, p)
                               : launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 2, false>, grid, threads, smem, s, p);
    else stay ? launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 1, true>, grid, threads, smem, s, p)
              : launch_after(mx_encode_kernel<HALF, BLOCK, XHAT, 1, false>, grid, threads, smem, s, p);
}

}  // namespace rac

using namespace rac;

extern "C" {

size_t rac_mx_record_bytes(const rac_mx_cfg *cfg) {
    MxGeometry g;
    return mx_geometry(cfg, &g) == RAC_OK ? static_cast<size_t>(g.rec) : 0;
}

size_t rac_mx_payload_bytes(const rac_mx_cfg *cfg, int64_t T) {
    return T < 0 ? 0 : rac_mx_record_bytes(cfg) * static_cast<size_t>(T);
}

int rac_mx_encode(const rac_mx_cfg *cfg, const void *X, int64_t T, void *payload, size_t payload_cap, void *X_hat,
                  uint32_t *dev_status, void *stream) {
    MxGeometry g;
    const int rc = mx_geometry(cfg, &g);
    if (rc != RAC_OK) return rc;
    if (T < 0) return RAC_EINVAL;
    if (T == 0) return RAC_OK;
    if (T > INT32_MAX) return RAC_EUNSUPPORTED;
    if (!X || !payload) return RAC_EINVAL;
    if (!mx_aligned(X) || !mx_aligned(payload) || !mx_aligned(X_hat)) return RAC_EALIGN;
    const size_t nx = static_cast<size_t>(T) * g.d * 2, np = static_cast<size_t>(T) * g.rec;
    if (payload_cap < np) return RAC_ESIZE;
    if (mx_overlap(X, nx, payload, np)) return RAC_EINVAL;
    if (X_hat && (mx_overlap(X_hat, nx, payload, np) || (X_hat != X && mx_overlap(X_hat, nx, X, nx)))) return RAC_EINVAL;
    MxParams p = {};
    unsigned grid, threads;
    const int shaped = mx_shape(g, T, X, X_hat, 8, &p, &grid, &threads);
    if (shaped != RAC_OK) return shaped;
    p.X = static_cast<const uint8_t *>(X);
    p.payload = static_cast<uint8_t *>(payload);
    p.X_hat = static_cast<uint8_t *>(X_hat);
    p.status = dev_status;
    auto s = static_cast<cudaStream_t>(stream);
    const bool half = g.x_type == RAC_MX_FP16;
    if (g.block == 16) {
        if (X_hat) half ? launch_mx_encode<true, 16, true>(p, grid, threads, s) : launch_mx_encode<false, 16, true>(p, grid, threads, s);
        else half ? launch_mx_encode<true, 16, false>(p, grid, threads, s) : launch_mx_encode<false, 16, false>(p, grid, threads, s);
    } else {
        if (X_hat) half ? launch_mx_encode<true, 32, true>(p, grid, threads, s) : launch_mx_encode<false, 32, true>(p, grid, threads, s);
        else half ? launch_mx_encode<true, 32, false>(p, grid, threads, s) : launch_mx_encode<false, 32, false>(p, grid, threads, s);
    }
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
}

int rac_mx_decode(const rac_mx_cfg *cfg, const void *payload, int64_t T, void *X_hat, uint32_t *dev_status, void *stream) {
    MxGeometry g;
    const int rc = mx_geometry(cfg, &g);
    if (rc != RAC_OK) return rc;
    if (T < 0) return RAC_EINVAL;
    if (T == 0) return RAC_OK;
    if (T > INT32_MAX) return RAC_EUNSUPPORTED;
    if (!payload || !X_hat) return RAC_EINVAL;
    if (!mx_aligned(payload) || !mx_aligned(X_hat)) return RAC_EALIGN;
    if (mx_overlap(X_hat, static_cast<size_t>(T) * g.d * 2, payload, static_cast<size_t>(T) * g.rec)) return RAC_EINVAL;
    (void)dev_status;      // nothing in a record is out of range; kept for the shape of the calls
    MxParams p = {};
    unsigned grid, threads;
    const int shaped = mx_shape(g, T, X_hat, X_hat, 1, &p, &grid, &threads);
    if (shaped != RAC_OK) return shaped;
    p.payload = const_cast<uint8_t *>(static_cast<const uint8_t *>(payload));
    p.X_hat = static_cast<uint8_t *>(X_hat);
    auto s = static_cast<cudaStream_t>(stream);
    const bool half = g.x_type == RAC_MX_FP16;
    if (g.block == 16) half ? launch_after(mx_decode_kernel<true, 16>, grid, threads, 0, s, p) : launch_after(mx_decode_kernel<false, 16>, grid, threads, 0, s, p);
    else half ? launch_after(mx_decode_kernel<true, 32>, grid, threads, 0, s, p) : launch_after(mx_decode_kernel<false, 32>, grid, threads, 0, s, p);
    return cudaGetLastError() == cudaSuccess ? RAC_OK : RAC_ECUDA;
}

}  // extern "C"
