// k_rotate.cu -- norms of queries and keys for each head, with the position rotation in
// the same pass:
//   y = x / sqrt(mean_c x_c^2 + eps) * w;  (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
// with t = pos * inv_freq[f] for the pair f of columns.
//
// Bound: memory, every row read and written once, and near it issue (58 % of all slots, 66 % of the cycles in which an SM has
// work): 170 instructions a chunk of heads, 700 a
// token.  A lane holds 16 columns of a head, so chosen that a pair's two columns meet in it, and LPL lanes a head; a warp keeps
// one token's cosines and sines, times the weights, in registers and goes over its heads, which it has asked for ahead into
// shared memory.  16,381 tokens x 40 heads of 128: 54.5 us, 6.2 TB/s (registers alone, one chunk ahead: 67 us); 30,001 x
// 40 of 64 58 us (a token's 700 instructions weigh twice); 40 tokens x 16 heads 3.3 us.  Three CTAs an SM leave 80 registers, and 24 to
// 32 of them go to memory and back once or twice a token; with two CTAs nothing does, but less is under way: 55.4 us against 54.9 and
// 61.6 against 58.2 for the two long ones, 2.9 against 3.3 for the short one.
#include <algorithm>

#include <cuda_bf16.h>

#include "fw_chain.cuh"

namespace fw {
namespace {

constexpr int RW = 8;      // warps of a CTA
constexpr int AHEAD = 4;   // chunks of heads that a warp has asked for ahead of the one that it works on (6: 65 us)

__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

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

// Two fp32 numbers side by side, and operations on both at once.
__device__ __forceinline__ uint64_t pack2(float x, float y)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t swap2(uint64_t v)
{
    float x, y;
    unpack2(v, x, y);
    return pack2(y, x);
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// (a product and -0, which changes nothing, are one instruction)
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { return fma2(a, b, 0x8000000080000000ull); }
__device__ __forceinline__ uint32_t to_bf16x2(uint64_t v)
{
    float x, y;
    unpack2(v, x, y);
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}

// 8 weights from `at` on, in pairs.
__device__ __forceinline__ void weights8(const RotateArgs &a, int kv, int at, uint64_t (&w)[4])
{
    if (!a.w[kv]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(1.f, 1.f);
    } else if (a.w_bf16) {
        const uint4 x = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.w[kv]) + at);
        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 x = reinterpret_cast<const float4 *>(static_cast<const float *>(a.w[kv]) + at)[i];
            w[2 * i] = pack2(x.x, x.y), w[2 * i + 1] = pack2(x.z, x.w);
        }
    }
}

template <int LPL, bool INTER, bool FULL> __global__ void __launch_bounds__(32 * RW, 3) k_qk_rotate(const RotateArgs a)
{
    constexpr int HP = 32 / LPL, PER = 8 / HP;  // heads at a time; frequencies that a lane works out
    __shared__ uint4 s_x[RW][AHEAD + 1][2][32];  // a lane's own pieces: no lane reads another's
    let_the_next_start();
    wait_for_the_one_before();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, p = lane % LPL, hl = lane / LPL;
    const int64_t id = (int64_t)blockIdx.x * RW + wid;
    const int64_t row = id / a.split;
    const int part = (int)(id - row * a.split);
    if (row >= a.rows) return;

    // A lane's two pieces of 8 columns.  Half apart, they are a pair's, in the rotated columns; neighbours are in one
    // piece, so any two do.  The lanes' first pieces lie side by side, and so do their second ones, for whole sectors.
    const bool there = 16 * p < a.d, pair = FULL || 16 * p < a.rot;
    const int rest = INTER || FULL ? 0 : a.rot, q = INTER || pair ? p : p - a.rot / 16;
    const int at0 = (INTER || pair ? 0 : rest) + 8 * q;
    const int at1 = at0 + (INTER ? a.d / 2 : pair ? a.rot / 2 : (a.d - rest) / 2);
    const bool turn0 = FULL || (INTER ? at0 < a.rot : pair), turn1 = FULL || (INTER ? at1 < a.rot : pair);
    // chunks of HP heads: the queries' heads, then the keys'
    const int chunks_q = (a.q_heads + HP - 1) / HP, chunks = chunks_q + (a.kv_heads + HP - 1) / HP;
    const uint32_t mem = (uint32_t)__cvta_generic_to_shared(&s_x[wid][0][0][lane]);
    constexpr int SLOT = sizeof(s_x[0][0]), HALF = SLOT / 2;
    if (!there) {
#pragma unroll
        for (int i = 0; i <= AHEAD; ++i) s_x[wid][i][0][lane] = s_x[wid][i][1][lane] = make_uint4(0, 0, 0, 0);
    }
    // The next chunk to be asked for: its head of this lane and where that lies.
    int next = part, next_slot = 0, head = 0, heads_of = 0;
    const uint16_t *src = nullptr;
    auto seek = [&](int kv) {
        head = (next - (kv ? chunks_q : 0)) * HP + hl;
        heads_of = !there ? 0 : kv ? a.kv_heads : a.q_heads;
        src = (kv ? a.k + row * a.k_row + head * a.k_head : a.q + row * a.q_row + head * a.q_head) + at0;
    };
    seek(part >= chunks_q);
    auto load = [&]() {
        if (next < chunks) {
            if (head < heads_of) {
                copy_async16(mem + next_slot, src);
                copy_async16(mem + next_slot + HALF, src + (at1 - at0));
            }
            const bool was_q = next < chunks_q;
            next += a.split;
            if (was_q && next >= chunks_q) {
                seek(1);
            } else {
                head += a.split * HP;
                src += a.split * HP * (was_q ? a.q_head : a.k_head);
            }
        }
        next_slot = next_slot == AHEAD * SLOT ? 0 : next_slot + SLOT;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // (a row's first heads are under way before its angles are worked out)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load();
    float cs[8], sn[8];
    if (a.rot > 0) {
        const int64_t pos = a.pos[row];
        float c[PER], s[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = (hl * PER + i) % 8, f = INTER ? (j < 4 ? at0 : at1) / 2 + j % 4 : 8 * p + j;
            const float x = f < a.rot / 2 ? a.inv_freq[f] : 0.f;
            // half turns in [-1, 1): the upper 32 bits of the product
            const float h = (float)(int32_t)((uint64_t)pos * turns_of(x) >> 32) * 0x1p-31f;
            sincospif(isfinite(x) ? h : NAN, &s[i], &c[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = __shfl_sync(FW_FULL, c[i % PER], (i / PER) * LPL + p);
            sn[i] = __shfl_sync(FW_FULL, s[i % PER], (i / PER) * LPL + p);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
    }
    const float inv_d = 1.f / (float)a.d;
    int slot = 0, ch = part;
    for (int kv = 0; kv < 2; ++kv) {
        const int first = kv ? chunks_q : 0, end = kv ? chunks : chunks_q, heads = kv ? a.kv_heads : a.q_heads;
        if (ch >= end) continue;
        // Factors of a pair's columns, the weights in them: with y the head's values (before its root mean square),
        // half apart: out_a = y_a A_a - y_b B_b, out_b = y_b A_b + y_a B_a; neighbours: (y_0, y_1) A + (y_1, y_0) B.
        uint64_t A[2][4], B[2][4];
        if (there) {
            weights8(a, kv, at0, A[0]);
            weights8(a, kv, at1, A[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) A[0][i] = A[1][i] = 0;
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            if (z ? turn1 : turn0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (INTER) {
                        const int f = 4 * z + i;
                        B[z][i] = mul2(swap2(A[z][i]), pack2(-sn[f], sn[f]));
                        A[z][i] = mul2(A[z][i], pack2(cs[f], cs[f]));
                    } else {
                        const uint64_t s = z ? pack2(-sn[2 * i], -sn[2 * i + 1]) : pack2(sn[2 * i], sn[2 * i + 1]);
                        B[z][i] = mul2(A[z][i], s);
                        A[z][i] = mul2(A[z][i], pack2(cs[2 * i], cs[2 * i + 1]));
                    }
                }
            }
        }
        int h = (ch - first) * HP + hl;
        uint16_t *dst = (kv ? a.k_out + row * a.k_out_row + h * a.k_out_head : a.q_out + row * a.q_out_row + h * a.q_out_head) + at0;
        const int64_t step = a.split * HP * (kv ? a.k_out_head : a.q_out_head);
        const int mine = there ? heads : 0;
        for (; ch < end; ch += a.split, h += a.split * HP, dst += step) {
            load();
            asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
            uint64_t y[2][4];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const uint4 x = s_x[wid][slot][z][lane];
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[z][i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
            }
            slot = slot == AHEAD ? 0 : slot + 1;
            uint64_t inv = pack2(1.f, 1.f);
            if (a.eps >= 0.f) {
                uint64_t sum2 = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum2 = fma2(y[i >> 2][i & 3], y[i >> 2][i & 3], sum2);
                float s0, s1;
                unpack2(sum2, s0, s1);
                s0 += s1;
#pragma unroll
                for (int o = LPL / 2; o > 0; o >>= 1) s0 += __shfl_xor_sync(FW_FULL, s0, o);
                const float r = rsqrtf(fmaf(s0, inv_d, a.eps));
                inv = pack2(r, r);
            }
            uint32_t out[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (what is not rotated takes no part of another column, be that no number)
                uint64_t u = mul2(y[0][i], A[0][i]), v = mul2(y[1][i], A[1][i]);
                if (turn0) u = fma2(INTER ? swap2(y[0][i]) : y[1][i], INTER ? B[0][i] : B[1][i], u);
                if (turn1) v = fma2(INTER ? swap2(y[1][i]) : y[0][i], INTER ? B[1][i] : B[0][i], v);
                out[0][i] = to_bf16x2(mul2(u, inv));
                out[1][i] = to_bf16x2(mul2(v, inv));
            }
            if (h < mine) {
                *reinterpret_cast<uint4 *>(dst) = make_uint4(out[0][0], out[0][1], out[0][2], out[0][3]);
                *reinterpret_cast<uint4 *>(dst + (at1 - at0)) = make_uint4(out[1][0], out[1][1], out[1][2], out[1][3]);
            }
        }
    }
}

template <int LPL> fw_status launch(RotateArgs &a, int sms, cudaStream_t s)
{
    constexpr int HP = 32 / LPL;
    const int chunks = (a.q_heads + HP - 1) / HP + (a.kv_heads + HP - 1) / HP;
    a.split = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, (int64_t)sms * 32 / a.rows));
    const unsigned grid = (unsigned)((a.rows * a.split + RW - 1) / RW);
    // (all columns rotated: every lane does the same)
    return launch_chained(a.interleaved ? a.rot == a.d ? k_qk_rotate<LPL, true, true> : k_qk_rotate<LPL, true, false>
                          : a.rot == a.d ? k_qk_rotate<LPL, false, true> : k_qk_rotate<LPL, false, false>,
                          dim3(grid), 32 * RW, 0, 0, s, a);
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
