// fw_cache8.cuh -- the 8-bit store as the kernels see it: its rows, its scales
// and the two code formats.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fw_internal.h"

namespace fw {
namespace cache8 {

struct Store {
    int cells;
    int64_t rows;
    uint8_t *k, *v;
    float *ks, *vs;
    uint16_t *kt, *vt;
    const int64_t *base;
    const int32_t *capacity;
    int32_t *counts;

    __device__ uint8_t *codes(int kv) const { return kv ? v : k; }
    __device__ float *scale(int kv) const { return kv ? vs : ks; }
    __device__ uint16_t *tail(int kv) const { return kv ? vt : kt; }
};

inline Store store(const fw_cache8 &c)
{
    return {c.cells,   c.rows, (uint8_t *)c.k,         (uint8_t *)c.v, c.k_scale, c.v_scale, (uint16_t *)c.k_tail,
            (uint16_t *)c.v_tail, c.base,         c.capacity, c.counts};
}

// The cell's rows, checked against the store.
__device__ __forceinline__ fw_status cell_rows(const Store &s, int h, int64_t &base, int &cap)
{
    base = s.base[h];
    cap = s.capacity[h];
    return base < 0 || base % FW_CACHE8_BLOCK != 0 || cap < 0 || base > s.rows || cap > s.rows - base ? FW_ERR_INVALID_ARG
                                                                                                      : FW_OK;
}

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The least e >= -120 with a <= M 2^e for the bf16 magnitude bits a (finite).
// 448 = 1.75 2^8 and 127 = 1.984375 2^6: e is a's exponent less 8 (6), one more
// where a's mantissa is above 0x60 (0x7e) of 0x80.  Subnormal a: -120.
template <int FMT> __device__ __forceinline__ int scale_exponent(uint32_t a)
{
    constexpr uint32_t mant = FMT == FW_CACHE8_E4M3 ? 0x60 : 0x7e;
    constexpr int up = FMT == FW_CACHE8_E4M3 ? 8 : 6;
    return max(-120, (int)(a >> 7) - 127 - up + ((a & 0x7f) > mant ? 1 : 0));
}

// bf16 bits of the largest code times 2^e, M 2^e (-120 <= e <= 119, or 121 for int8)
template <int FMT> __device__ __forceinline__ uint32_t top_code_bits(int e)
{
    return FMT == FW_CACHE8_E4M3 ? (uint32_t)(e + 8 + 127) << 7 | 0x60u : (uint32_t)(e + 6 + 127) << 7 | 0x7eu;
}

// Largest magnitudes (bf16 bits) of the even and the odd ones of 8 values into the halves of top;
// infinities and NaN are the largest (0x7f80 and above).
__device__ __forceinline__ uint32_t piece_top(const uint4 &x, uint32_t top)
{
    const uint32_t m = 0x7fff7fffu;
    return __vmaxu2(__vmaxu2(__vmaxu2(top, x.x & m), __vmaxu2(x.y & m, x.z & m)), x.w & m);
}
__device__ __forceinline__ uint32_t top_of(uint32_t pair) { return max(pair & 0xffffu, pair >> 16); }

// 8 values times 2^-down, with their NaN put to 0 and their infinities to the magnitude `lim` (bf16 bits).  What falls below
// bf16's range may come out as anything below 2^-126.
__device__ __forceinline__ uint4 finite_piece(const uint4 &x, uint32_t lim, int down)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int sh = 16 * (i & 1);
        const uint32_t b = (w[i >> 1] >> sh) & 0xffffu, mag = b & 0x7fffu;
        const uint32_t y = mag > 0x7f80u ? 0u : (b & 0x8000u) | (mag == 0x7f80u ? lim : (uint32_t)max((int)mag - (down << 7), 0));
        w[i >> 1] = (w[i >> 1] & ~(0xffffu << sh)) | y << sh;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Codes of 8 values times inv, whose magnitudes are at most the largest code.
template <int FMT> __device__ __forceinline__ uint2 encode8(const uint4 &x, float inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __uint_as_float(w[i] << 16), b = __uint_as_float(w[i] & 0xffff0000u);
        if constexpr (FMT == FW_CACHE8_E4M3) {
            uint16_t c;  // (the second operand is the low byte)
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(b * inv), "f"(a * inv));
            r[i] = c;
        } else {
            // the sum's one rounding is to the integer, whose low byte is the sum's
            const float up = 12582912.f;  // 1.5 * 2^23
            r[i] = __byte_perm(__float_as_uint(fmaf(a, inv, up)), __float_as_uint(fmaf(b, inv, up)), 0x0040);
        }
    }
    return make_uint2(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410));
}

}  // namespace cache8

// Dispatch on a store's width and format: binds D and FMT.
#define FW_CACHE8_DISPATCH(c, ...)                                \
    do {                                                          \
        if ((c).d == 128 && (c).format == FW_CACHE8_E4M3) {       \
            constexpr int D = 128, FMT = FW_CACHE8_E4M3;          \
            __VA_ARGS__;                                          \
        } else if ((c).d == 128) {                                \
            constexpr int D = 128, FMT = FW_CACHE8_INT8;          \
            __VA_ARGS__;                                          \
        } else if ((c).format == FW_CACHE8_E4M3) {                \
            constexpr int D = 64, FMT = FW_CACHE8_E4M3;           \
            __VA_ARGS__;                                          \
        } else {                                                  \
            constexpr int D = 64, FMT = FW_CACHE8_INT8;           \
            __VA_ARGS__;                                          \
        }                                                         \
    } while (0)

}  // namespace fw
