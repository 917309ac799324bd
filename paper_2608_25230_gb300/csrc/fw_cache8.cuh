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

// Largest finite magnitude (bf16 bits) of 8 values into top; true where one is not finite.
__device__ __forceinline__ bool piece_top(const uint4 &x, uint32_t &top)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = w[i] & 0x7fff, hi = (w[i] >> 16) & 0x7fff;
        odd |= lo >= 0x7f80 || hi >= 0x7f80;
        top = max(top, max(lo >= 0x7f80 ? 0u : lo, hi >= 0x7f80 ? 0u : hi));
    }
    return odd;
}

// Codes of two values already divided by the scale; infinities saturate, NaN is 0.
template <int FMT> __device__ __forceinline__ uint32_t encode2(float a, float b)
{
    a = a != a ? 0.f : a;
    b = b != b ? 0.f : b;
    if constexpr (FMT == FW_CACHE8_E4M3) {
        uint16_t r;  // (the second operand is the low byte)
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
        return r;
    } else {
        const int i = __float2int_rn(fminf(fmaxf(a, -127.f), 127.f)), j = __float2int_rn(fminf(fmaxf(b, -127.f), 127.f));
        return (uint32_t)(i & 0xff) | (uint32_t)(j & 0xff) << 8;
    }
}
template <int FMT> __device__ __forceinline__ uint2 encode8(const uint4 &x, float inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = encode2<FMT>(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
    return make_uint2(r[0] | r[1] << 16, r[2] | r[3] << 16);
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
