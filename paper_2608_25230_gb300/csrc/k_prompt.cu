// k_prompt.cu -- causal attention over packed prompts with grouped heads: query
// token i of a sequence with lq query and lk key rows sees its keys
// j <= lk - lq + i:
//   x_j = scale q_i . k_j,  o_i = sum_j softmax_j(x) v_j,  lse_i = log sum_j e^x_j.
//
// A warp per (query row, head) goes over the keys with a running maximum and sum.
#include <cuda_bf16.h>

#include "fw_internal.h"

namespace fw {
namespace {

struct PromptArgs {
    fw_prompt p;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
};

// sequence bounds within their ranges
__device__ __forceinline__ bool seq_ok(const fw_prompt &p, int s)
{
    const int q0 = p.cu_q[s], q1 = p.cu_q[s + 1], k0 = p.cu_k[s], k1 = p.cu_k[s + 1];
    return q0 >= 0 && q1 >= q0 && q1 <= p.total_q && k0 >= 0 && k1 >= k0 && k1 <= p.total_k;
}

template <int D> __global__ void __launch_bounds__(128) k_prompt(const PromptArgs a)
{
    constexpr int N = D / 32;
    const fw_prompt &p = a.p;
    const int lane = threadIdx.x & 31, head = blockIdx.y, hk = head / (p.q_heads / p.kv_heads);
    if (blockIdx.x == 0 && blockIdx.y == 0 && a.status)
        for (int s = threadIdx.x; s < p.num_seqs; s += 128) a.status[s] = seq_ok(p, s) ? FW_OK : FW_ERR_INVALID_ARG;
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.total_q) return;
    int lo = 0, hi = p.num_seqs;  // the last sequence that starts at or before the row
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.cu_q[mid] <= row) lo = mid; else hi = mid;
    }
    if (!seq_ok(p, lo) || row < p.cu_q[lo] || row >= p.cu_q[lo + 1]) return;
    const int k0 = p.cu_k[lo], lk = p.cu_k[lo + 1] - k0;
    const int seen = lk - (p.cu_q[lo + 1] - p.cu_q[lo]) + (row - p.cu_q[lo]) + 1;
    const uint16_t *q = (const uint16_t *)p.q + row * p.q_row + head * p.q_head;
    float qv[N], acc[N], mx = -INFINITY;
    double l = 0.0;  // (thousands of terms one after another)
    for (int u = 0; u < N; ++u) qv[u] = bf16_to_f32(q[lane + 32 * u]), acc[u] = 0.f;
    for (int j = 0; j < seen; ++j) {
        const uint16_t *k = (const uint16_t *)p.k + (int64_t)(k0 + j) * p.k_row + hk * p.k_head;
        const uint16_t *v = (const uint16_t *)p.v + (int64_t)(k0 + j) * p.v_row + hk * p.v_head;
        float x = 0.f;
        for (int u = 0; u < N; ++u) x = fmaf(qv[u], bf16_to_f32(k[lane + 32 * u]), x);
        x = warp_sum(x) * a.scale2;
        const float mn = fmaxf(mx, x), f = exp2f(mx - mn), e = exp2f(x - mn);
        mx = mn;
        l = l * f + e;
        for (int u = 0; u < N; ++u) acc[u] = acc[u] * f + e * bf16_to_f32(v[lane + 32 * u]);
    }
    const int64_t out = (int64_t)row * p.q_heads + head;
    for (int u = 0; u < N; ++u)
        a.o[out * D + lane + 32 * u] = __bfloat16_as_ushort(__float2bfloat16_rn(seen > 0 ? acc[u] / (float)l : 0.f));
    if (a.lse && lane == 0) a.lse[out] = seen > 0 ? (mx + log2f((float)l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

fw_status prompt_attention(const fw_prompt &p, void *o, float *lse, int32_t *status, cudaStream_t s)
{
    const PromptArgs a{p, p.scale * 1.4426950408889634f, (uint16_t *)o, lse, status};
    if (p.q_heads > 65535) return FW_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((p.total_q + 3) / 4), (unsigned)p.q_heads);
    if (p.d == 128)
        FW_LAUNCH(k_prompt<128>, grid, 128, 0, s, a);
    else
        FW_LAUNCH(k_prompt<64>, grid, 128, 0, s, a);
    return FW_OK;
}

}  // namespace fw
