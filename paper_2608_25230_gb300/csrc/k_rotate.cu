// k_rotate.cu -- norms of queries and keys for each head, with the position rotation in
// the same pass:
//   y = x / sqrt(mean_c x_c^2 + eps) * w;  (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
// with t = pos * inv_freq[f] for the pair f of columns.
//
// Bound: memory, every row read and written once.  A lane holds 16 columns of a head, so chosen
// that a pair's two columns meet in it, and LPL lanes a head; a warp keeps one token's
// cosines and sines in registers and goes over its heads.
#include <algorithm>

#include <cuda_bf16.h>

#include "fw_internal.h"

namespace fw {
namespace {

constexpr int RW = 8;  // warps of a CTA

struct RotateArgs {
    int64_t rows;
    int q_heads, kv_heads, d, rot, interleaved, split;
    const uint16_t *q, *k;
    uint16_t *q_out, *k_out;
    const void *w[2];
    int w_bf16;
    const int32_t *pos;
    const float *inv_freq;
    int64_t q_row, q_head, k_row, k_head, q_out_row, q_out_head, k_out_row, k_out_head;
    float eps;
};

// Turns per token of a frequency in radians, modulo one, in units of 2^-64: x / 2 pi with x = M 2^e.  A
// product with a position then wraps as the angle does, whatever the position: fp32 would
// be off by whole radians at positions of a million.
__device__ __forceinline__ uint64_t turns_of(float x)
{
    const uint64_t C = 0x28BE60DB9391054Aull;  // 2^64 / (2 pi), rounded
    const uint32_t b = __float_as_uint(x);
    const int ex = (int)(b >> 23 & 255u);
    const uint64_t M = (b & 0x7fffffu) | (ex ? 0x800000u : 0u);
    const int e = max(ex, 1) - 150;
    const uint64_t lo = M * C, hi = __umul64hi(M, C);
    uint64_t t;
    if (e >= 0)
        t = e < 64 ? lo << e : 0;
    else if (e > -64)
        t = lo >> -e | hi << (64 + e);
    else
        t = e > -128 ? hi >> (-e - 64) : 0;
    return b >> 31 ? 0 - t : t;
}

template <int LPL> __global__ void __launch_bounds__(32 * RW) k_qk_rotate(const RotateArgs a)
{
    constexpr int HP = 32 / LPL, PER = 8 / HP > 0 ? 8 / HP : 1;  // heads at a time; frequencies that a lane works out
    __shared__ float s_w[2][256];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, p = lane % LPL, hl = lane / LPL;
    if (a.eps >= 0.f) {
        for (int i = tid; i < 2 * a.d; i += 32 * RW) {
            const int kv = i >= a.d, c = i - kv * a.d;
            s_w[kv][c] = !a.w[kv] ? 1.f
                         : a.w_bf16 ? bf16_to_f32(static_cast<const uint16_t *>(a.w[kv])[c])
                                    : static_cast<const float *>(a.w[kv])[c];
        }
        __syncthreads();
    }
    const int64_t id = (int64_t)blockIdx.x * RW + wid;
    const int64_t row = id / a.split;
    if (row >= a.rows) return;
    const int part = (int)(id - row * a.split);

    const bool rotated = 16 * p < a.rot, there = 16 * p < a.d;
    const int at0 = rotated && !a.interleaved ? 8 * p : 16 * p;
    const int at1 = rotated && !a.interleaved ? a.rot / 2 + 8 * p : 16 * p + 8;
    float cs[8], sn[8];
    if (a.rot > 0) {
        const int64_t pos = a.pos[row];
        float c[PER], s[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int f = 8 * p + (hl * PER + i) % 8;
            const float x = rotated ? a.inv_freq[f] : 0.f;
            // half turns in [-1, 1): the upper 32 bits of the product
            const float h = (float)(int32_t)((uint64_t)pos * turns_of(x) >> 32) * 0x1p-31f;
            sincospif(isfinite(x) ? h : NAN, &s[i], &c[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = __shfl_sync(FW_FULL, c[i % PER], (i / PER) * LPL + p);
            sn[i] = __shfl_sync(FW_FULL, s[i % PER], (i / PER) * LPL + p);
        }
    }
    const int chunks_q = (a.q_heads + HP - 1) / HP, chunks = chunks_q + (a.kv_heads + HP - 1) / HP;
    auto load = [&](int ch, uint4 (&x)[2]) {
        const bool kv = ch >= chunks_q;
        const int h = (kv ? ch - chunks_q : ch) * HP + hl;
        x[0] = x[1] = make_uint4(0, 0, 0, 0);
        if (ch < chunks && there && h < (kv ? a.kv_heads : a.q_heads)) {
            const uint16_t *src = kv ? a.k + row * a.k_row + h * a.k_head : a.q + row * a.q_row + h * a.q_head;
            x[0] = *reinterpret_cast<const uint4 *>(src + at0);
            x[1] = *reinterpret_cast<const uint4 *>(src + at1);
        }
    };
    uint4 next[2];
    load(part, next);
    for (int ch = part; ch < chunks; ch += a.split) {
        const bool kv = ch >= chunks_q;
        const int h = (kv ? ch - chunks_q : ch) * HP + hl;
        const uint32_t w[8] = {next[0].x, next[0].y, next[0].z, next[0].w, next[1].x, next[1].y, next[1].z, next[1].w};
        float y[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[2 * i] = __uint_as_float(w[i] << 16);
            y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
        load(ch + a.split, next);
        if (a.eps >= 0.f) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(y[i], y[i], sum);
#pragma unroll
            for (int o = LPL / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(FW_FULL, sum, o);
            const float inv = rsqrtf(sum / (float)a.d + a.eps);
            const float *wt = s_w[kv];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] *= inv * (there ? wt[(i < 8 ? at0 : at1 - 8) + i] : 0.f);
        }
        if (rotated) {
            if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = y[2 * i], v = y[2 * i + 1];
                    y[2 * i] = u * cs[i] - v * sn[i];
                    y[2 * i + 1] = v * cs[i] + u * sn[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = y[i], v = y[8 + i];
                    y[i] = u * cs[i] - v * sn[i];
                    y[8 + i] = v * cs[i] + u * sn[i];
                }
            }
        }
        if (there && h < (kv ? a.kv_heads : a.q_heads)) {
            uint32_t r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
                r[i] = *reinterpret_cast<const uint32_t *>(&b);
            }
            uint16_t *dst = kv ? a.k_out + row * a.k_out_row + h * a.k_out_head : a.q_out + row * a.q_out_row + h * a.q_out_head;
            *reinterpret_cast<uint4 *>(dst + at0) = make_uint4(r[0], r[1], r[2], r[3]);
            *reinterpret_cast<uint4 *>(dst + at1) = make_uint4(r[4], r[5], r[6], r[7]);
        }
    }
}

template <int LPL> fw_status launch(RotateArgs &a, int sms, cudaStream_t s)
{
    constexpr int HP = 32 / LPL;
    const int chunks = (a.q_heads + HP - 1) / HP + (a.kv_heads + HP - 1) / HP;
    a.split = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, (int64_t)sms * 32 / a.rows));
    FW_LAUNCH(k_qk_rotate<LPL>, (unsigned)((a.rows * a.split + RW - 1) / RW), 32 * RW, 0, s, a);
    return FW_OK;
}

}  // namespace

fw_status qk_rotate(const fw_rotation &r, cudaStream_t s)
{
    int sms = 0;
    const fw_status st = device_sms(&sms);
    if (st != FW_OK) return st;
    RotateArgs a{r.rows, r.q_heads, r.kv_heads, r.d, r.rot, r.interleaved, 1, (const uint16_t *)r.q, (const uint16_t *)r.k,
                 (uint16_t *)r.q_out, (uint16_t *)r.k_out, {r.q_weight, r.k_weight}, r.w_dtype == FW_BF16, r.pos, r.inv_freq,
                 r.q_row, r.q_head, r.k_row, r.k_head, r.q_out_row, r.q_out_head, r.k_out_row, r.k_out_head, r.eps};
    if (r.d <= 64) return launch<4>(a, sms, s);
    if (r.d <= 128) return launch<8>(a, sms, s);
    return launch<16>(a, sms, s);
}

}  // namespace fw
