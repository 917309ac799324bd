// k_cache8.cu -- the ragged per-head store in 8 bits: compaction of a bf16
// cache's kept rows into it, and appends.
//
// A block is 32 rows of a cell.  With a = the largest magnitude among its filled
// rows (a bf16 number, or 0), its scale is 2^e, e the least integer >= -120 with
// a <= M 2^e, M = 448 (e4m3) or 127 (int8), and a code is rne(x 2^-e).  e follows
// from a's exponent and mantissa bits alone; x 2^-e is exact in fp32 (|e| <= 120,
// and what falls below fp32's range is far below half the least code), so the one
// rounding is the conversion to 8 bits.
#include <algorithm>

#include "fw_cache8.cuh"

namespace fw {
namespace {

using namespace cache8;

constexpr int BR = FW_CACHE8_BLOCK, TL = FW_CACHE8_TAIL;

// Quantises the rows of one block, held as 16-byte pieces x[i] of row r0 + RS * i, column 8 * col:
// the block's scale from the CTA's largest magnitude, then codes.  Rows at or past nrow are not
// filled.  Every thread of the CTA calls it.
template <int D, int FMT, int THREADS>
__device__ __forceinline__ bool quantise_block(uint4 *x, int nrow, uint8_t *codes, float *scale, uint32_t *s_max)
{
    constexpr int LPR = D / 8, RS = THREADS / LPR, N = BR / RS;
    const int tid = threadIdx.x, col = tid % LPR, r0 = tid / LPR;
    uint32_t top = 0;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (r0 + RS * i < nrow) odd |= piece_top(x[i], top);
    top = __reduce_max_sync(FW_FULL, top);
    if ((tid & 31) == 0) s_max[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) top = max(top, s_max[w]);
    __syncthreads();
    const int e = scale_exponent<FMT>(top);
    if (tid == 0) *scale = pow2f(e);
    const float inv = pow2f(-e);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (r0 + RS * i < nrow)
            *reinterpret_cast<uint2 *>(codes + (size_t)(r0 + RS * i) * D + 8 * col) = encode8<FMT>(x[i], inv);
    return odd;
}

struct CompactArgs {
    Store s;
    const uint16_t *K, *V;
    int T;
    int64_t cell_stride, row_stride;
    const int64_t *offsets;
    const int32_t *kept_pos;
    int64_t total;
    int32_t *status;
};

// A CTA per cell.
template <int D, int FMT>
__global__ void __launch_bounds__(128) k_cache8_compact(const CompactArgs a)
{
    constexpr int LPR = D / 8, RS = 128 / LPR, N = BR / RS;
    __shared__ uint32_t s_max[4];
    __shared__ int s_odd;
    const int h = blockIdx.x, tid = threadIdx.x, col = tid % LPR, r0 = tid / LPR;
    const int64_t o0 = a.offsets[h], o1 = a.offsets[h + 1];
    int64_t base;
    int cap;
    fw_status st = cell_rows(a.s, h, base, cap);
    if (st == FW_OK && (o0 < 0 || o1 < o0 || o1 > a.total)) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && o1 - o0 > cap) st = FW_ERR_WORKSPACE;
    if (tid == 0) s_odd = 0;
    __syncthreads();
    const int n = st == FW_OK ? (int)(o1 - o0) : 0;
    int odd = 0;
    for (int b = 0; b < n; b += BR) {
        const int nrow = min(BR, n - b);
        for (int kv = 0; kv < 2; ++kv) {
            const uint16_t *src = (kv ? a.V : a.K) + (int64_t)h * a.cell_stride;
            uint4 x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = r0 + RS * i;
                x[i] = make_uint4(0, 0, 0, 0);
                if (r < nrow) {
                    const int p = a.kept_pos[o0 + b + r];
                    if (p >= 0 && p < a.T)
                        x[i] = *reinterpret_cast<const uint4 *>(src + (int64_t)p * a.row_stride + 8 * col);
                    else
                        odd |= 2;
                    if (nrow < BR)
                        *reinterpret_cast<uint4 *>(a.s.tail(kv) + ((int64_t)h * TL + (b + r) % TL) * D + 8 * col) = x[i];
                }
            }
            if (quantise_block<D, FMT, 128>(x, nrow, a.s.codes(kv) + (base + b) * D, a.s.scale(kv) + (base + b) / BR, s_max))
                odd |= 1;
        }
    }
    if (odd) atomicOr(&s_odd, odd);
    __syncthreads();
    if (tid == 0) {
        a.s.counts[h] = n;
        if (a.status) a.status[h] = st != FW_OK ? st : (s_odd & 2) ? FW_ERR_INVALID_ARG : s_odd ? FW_ERR_NONFINITE : FW_OK;
    }
}

struct AppendArgs {
    Store s;
    const uint16_t *K, *V;
    int m;
    int32_t *status;
};

// A CTA per cell: the blocks its m rows touch, one after another.
template <int D, int FMT>
__global__ void __launch_bounds__(128) k_cache8_append(const AppendArgs a)
{
    constexpr int LPR = D / 8, RS = 128 / LPR, N = BR / RS;
    __shared__ uint32_t s_max[4];
    __shared__ int s_odd;
    const int h = blockIdx.x, tid = threadIdx.x, col = tid % LPR, r0 = tid / LPR;
    int64_t base;
    int cap;
    fw_status st = cell_rows(a.s, h, base, cap);
    const int n = a.s.counts[h];
    if (st == FW_OK && (n < 0 || n > cap)) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && a.m > cap - n) st = FW_ERR_WORKSPACE;
    if (tid == 0) s_odd = 0;
    __syncthreads();  // every thread has read the count
    if (st != FW_OK) {
        if (tid == 0 && a.status) a.status[h] = st;
        return;
    }
    int odd = 0;
    const int end = n + a.m;
    for (int b = n / BR * BR; b < end; b += BR) {
        const int nrow = min(BR, end - b);
        for (int kv = 0; kv < 2; ++kv) {
            uint4 x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = b + r0 + RS * i;
                x[i] = make_uint4(0, 0, 0, 0);
                if (r >= end) continue;
                uint16_t *slot = a.s.tail(kv) + ((int64_t)h * TL + r % TL) * D + 8 * col;
                if (r < n) {
                    x[i] = *reinterpret_cast<const uint4 *>(slot);
                } else {
                    x[i] = *reinterpret_cast<const uint4 *>((kv ? a.V : a.K) + ((int64_t)h * a.m + (r - n)) * D + 8 * col);
                    *reinterpret_cast<uint4 *>(slot) = x[i];
                }
            }
            if (quantise_block<D, FMT, 128>(x, nrow, a.s.codes(kv) + (base + b) * D, a.s.scale(kv) + (base + b) / BR, s_max))
                odd = 1;
        }
    }
    if (odd) s_odd = 1;
    __syncthreads();
    if (tid == 0) {
        a.s.counts[h] = end;
        if (a.status) a.status[h] = s_odd ? FW_ERR_NONFINITE : FW_OK;
    }
}

}  // namespace

fw_status cache8_compact(const fw_cache8 &c, const void *K, const void *V, int T, int64_t cell_stride,
                         int64_t row_stride, const int64_t *offsets, const int32_t *kept_pos, int64_t total,
                         int32_t *status, cudaStream_t s)
{
    const CompactArgs a{store(c), (const uint16_t *)K, (const uint16_t *)V, T, cell_stride, row_stride,
                        offsets,  kept_pos,            total,               status};
    FW_CACHE8_DISPATCH(c, FW_LAUNCH((k_cache8_compact<D, FMT>), (unsigned)c.cells, 128, 0, s, a));
    return FW_OK;
}

fw_status cache8_append(const fw_cache8 &c, const void *new_K, const void *new_V, int m, int32_t *status,
                        cudaStream_t s)
{
    const AppendArgs a{store(c), (const uint16_t *)new_K, (const uint16_t *)new_V, m, status};
    FW_CACHE8_DISPATCH(c, FW_LAUNCH((k_cache8_append<D, FMT>), (unsigned)c.cells, 128, 0, s, a));
    return FW_OK;
}

}  // namespace fw
