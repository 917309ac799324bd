// k_cache8_attend.cu -- attention over the 8-bit ragged store: with a cell's n
// rows of codes kc, vc and block scales sk, sv, query token i of m sees the rows
// j < n - m + 1 + i:
//   x_j = scale (q . kc_j) sk,  o = sum_j softmax_j(x) vc_j sv,  lse = log sum_j e^x_j.
//
// A warp per (cell, query row) goes over the rows with a running maximum and sum.
#include "fw_cache8.cuh"

namespace fw {
namespace {

using namespace cache8;

struct AttendArgs {
    Store s;
    int kv_heads, group, m;
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
};

template <int FMT> __device__ __forceinline__ float decode(uint8_t c)
{
    if constexpr (FMT == FW_CACHE8_INT8) return (float)(int8_t)c;
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)c));
    return __half2float(__ushort_as_half((uint16_t)r));
}

template <int D, int FMT> __global__ void __launch_bounds__(128) k_cache8_attend(const AttendArgs a)
{
    constexpr int N = D / 32;
    const int h = blockIdx.x, lane = threadIdx.x & 31, rows = a.group * a.m;
    const int b = h / a.kv_heads, hk = h % a.kv_heads;
    int64_t base;
    int cap;
    fw_status st = cell_rows(a.s, h, base, cap);
    int n = a.s.counts[h];
    if (st == FW_OK && (n < 0 || n > cap)) st = FW_ERR_INVALID_ARG;
    if (st != FW_OK) n = 0;
    if (blockIdx.y == 0 && threadIdx.x == 0 && a.status) a.status[h] = st;
    for (int r = blockIdx.y * 4 + (threadIdx.x >> 5); r < rows; r += gridDim.y * 4) {
        const int i = r / a.group, head = hk * a.group + r % a.group;
        const uint16_t *q = a.q + b * a.q_seq + i * a.q_tok + head * a.q_head;
        float qv[N], acc[N], mx = -INFINITY;
        double l = 0.0;  // (thousands of terms one after another)
        for (int u = 0; u < N; ++u) qv[u] = bf16_to_f32(q[lane + 32 * u]), acc[u] = 0.f;
        const int seen = n - a.m + 1 + i;
        for (int j = 0; j < seen; ++j) {
            const int64_t row = base + j;
            float x = 0.f;
            for (int u = 0; u < N; ++u) x = fmaf(qv[u], decode<FMT>(a.s.k[row * D + lane + 32 * u]), x);
            x = warp_sum(x) * a.s.ks[row / 32] * a.scale2;
            const float mn = fmaxf(mx, x), f = exp2f(mx - mn), p = exp2f(x - mn);
            mx = mn;
            l = l * f + p;
            for (int u = 0; u < N; ++u)
                acc[u] = acc[u] * f + p * a.s.vs[row / 32] * decode<FMT>(a.s.v[row * D + lane + 32 * u]);
        }
        const int64_t out = ((int64_t)b * a.m + i) * a.kv_heads * a.group + head;
        for (int u = 0; u < N; ++u)
            a.o[out * D + lane + 32 * u] = __bfloat16_as_ushort(__float2bfloat16_rn(seen > 0 ? acc[u] / (float)l : 0.f));
        if (a.lse && lane == 0) a.lse[out] = seen > 0 ? (mx + log2f((float)l)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace

size_t cache8_attend_workspace(const fw_cache8 &, const fw_cache8_query &) { return 0; }

fw_status cache8_attend(const fw_cache8 &c, const fw_cache8_query &q, void *o, float *lse, int32_t *status, void *,
                        cudaStream_t s)
{
    const AttendArgs a{store(c), q.kv_heads, q.group, q.m, (const uint16_t *)q.q, q.q_seq, q.q_tok, q.q_head,
                       q.scale * 1.4426950408889634f, (uint16_t *)o, lse, status};
    const dim3 grid((unsigned)c.cells, (unsigned)((q.group * q.m + 3) / 4));
    FW_CACHE8_DISPATCH(c, FW_LAUNCH((k_cache8_attend<D, FMT>), grid, 128, 0, s, a));
    return FW_OK;
}

}  // namespace fw
