// k_pages_attend.cu -- attention over a cache in pages: with a cell's n rows k, v, query token i
// of m sees the rows j < n - m + 1 + i:
//   x_j = scale (q . k_j),  o = sum_j softmax_j(x) v_j,  lse = log sum_j e^x_j.
//
// A CTA per cell and query row, a running maximum and sum per warp, joined at the end.
#include <algorithm>

#include <cuda_bf16.h>

#include "fw_pages.cuh"

namespace fw {
namespace {

using namespace pages;

constexpr int AW = 4;

struct AttendArgs {
    Pages s;
    int kv_heads, group, m;
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    float scale;
    uint16_t *o;
    float *lse;
    int32_t *status;
};

template <int D> __global__ void __launch_bounds__(32 * AW) k_pages_attend(const AttendArgs a)
{
    constexpr int E = D / 32;
    const Pages &s = a.s;
    __shared__ float s_m[AW], s_l[AW], s_o[AW][D];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, rows = a.group * a.m;
    const int h = blockIdx.x, r = blockIdx.y, i = r / a.group, g = r - i * a.group;
    const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
    int n, held;
    const fw_status st = cell_rows(s, h, n, held);
    if (st != FW_OK) n = 0;
    const int seen = max(0, n - a.m + 1 + i);
    const uint16_t *q = a.q + seq * a.q_seq + i * a.q_tok + (int64_t)(hk * a.group + g) * a.q_head;
    float qf[E], acc[E], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) qf[e] = bf16_to_f32(q[lane + 32 * e]), acc[e] = 0.f;
    bool bad = st != FW_OK;
    for (int j = wid; j < n; j += AW) {
        const int page = s.row(h)[j / s.P];
        if (!s.is_page(page)) {
            bad = true;
            continue;
        }
        if (j >= seen) continue;
        const int64_t at = ((int64_t)page * s.P + j % s.P) * D + lane;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(qf[e], bf16_to_f32(s.k[at + 32 * e]), x);
        x = warp_sum(x) * a.scale;
        const float now = fmaxf(M, x), ref = now == -INFINITY ? 0.f : now;
        const float old = expf(M - ref), w = expf(x - ref);
        L = L * old + w;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * old + w * bf16_to_f32(s.v[at + 32 * e]);
        M = now;
    }
    if (lane == 0) s_m[wid] = M, s_l[wid] = L;
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[wid][lane + 32 * e] = acc[e];
    bad = __syncthreads_or(bad);
    if (wid != 0) return;
    M = -INFINITY;
    for (int w = 0; w < AW; ++w) M = fmaxf(M, s_m[w]);
    L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int w = 0; w < AW; ++w) {
        const float f = M == -INFINITY ? 0.f : expf(s_m[w] - M);
        L += f * s_l[w];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f * s_o[w][lane + 32 * e];
    }
    const int64_t out = ((int64_t)seq * a.m + i) * a.kv_heads * a.group + hk * a.group + g;
#pragma unroll
    for (int e = 0; e < E; ++e)
        a.o[out * D + lane + 32 * e] = __bfloat16_as_ushort(__float2bfloat16_rn(L == 0.f ? 0.f : acc[e] / L));
    if (lane == 0 && a.lse) a.lse[out] = L == 0.f ? -INFINITY : M + logf(L);
    if (lane == 0 && a.status && r == rows - 1) a.status[h] = bad ? FW_ERR_INVALID_ARG : FW_OK;
}

}  // namespace

size_t pages_attend_workspace(const fw_pages &, const fw_pages_query &) { return 0; }

fw_status pages_attend(const fw_pages &p, const fw_pages_query &q, void *o, float *lse, int32_t *status, void *,
                       cudaStream_t s)
{
    const AttendArgs a{view(p), q.kv_heads, q.group, q.m, (const uint16_t *)q.q, q.q_seq, q.q_tok, q.q_head, q.scale,
                       (uint16_t *)o, lse, status};
    const dim3 grid((unsigned)p.cells, (unsigned)(q.group * q.m));
    if (p.d == 128)
        FW_LAUNCH(k_pages_attend<128>, grid, 32 * AW, 0, s, a);
    else
        FW_LAUNCH(k_pages_attend<64>, grid, 32 * AW, 0, s, a);
    return FW_OK;
}

}  // namespace fw
