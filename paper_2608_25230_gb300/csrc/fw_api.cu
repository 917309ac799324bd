// fw_api.cu -- the C ABI: host-side validation, workspace carving, dispatch.
#include <cstring>

#include "fw_internal.h"

namespace fw {
std::atomic<uint64_t> g_launches{0};

static bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled tma_encoder()
{
    static std::atomic<EncodeTiled> fn{nullptr};
    EncodeTiled f = fn.load(std::memory_order_acquire);
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
                cudaSuccess &&
            q == cudaDriverEntryPointSuccess) {
            f = reinterpret_cast<EncodeTiled>(p);
            fn.store(f, std::memory_order_release);
        }
    }
    return f;
}

bool make_tma_2d_bf16(CUtensorMap *m, const void *base, uint64_t rows, uint64_t cols, uint32_t box_rows)
{
    EncodeTiled enc = tma_encoder();
    if (!enc) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {cols * 2};
    const cuuint32_t box[2] = {64, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tma_2d_bytes(CUtensorMap *m, const void *base, uint64_t rows, uint64_t cols, uint32_t box_rows)
{
    EncodeTiled enc = tma_encoder();
    if (!enc) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {cols};
    const cuuint32_t box[2] = {(cuuint32_t)cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, cols == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tma_heads_bf16(CUtensorMap *m, const void *base, int d, int heads, int64_t rows, int64_t head_stride,
                         int64_t row_stride, int box_heads, int box_rows)
{
    EncodeTiled enc = tma_encoder();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)head_stride * 2, (cuuint64_t)row_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

fw_status device_sms(int *sms)
{
    static std::atomic<int> cache[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FW_ERR_CUDA;
    if (dev >= 0 && dev < 64) {
        const int c = cache[dev].load(std::memory_order_relaxed);
        if (c > 0) {
            *sms = c;
            return FW_OK;
        }
    }
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return FW_ERR_CUDA;
    if (dev >= 0 && dev < 64) cache[dev].store(n, std::memory_order_relaxed);
    *sms = n;
    return FW_OK;
}

fw_status big_smem(const void *kernel, size_t bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FW_ERR_CUDA;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return FW_OK;
    FW_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done.fetch_or(bit, std::memory_order_relaxed);
    return FW_OK;
}

static bool good_stride(int64_t x) { return x > 0 && x % 8 == 0 && x < ((int64_t)1 << 38); }

static fw_status check_prompt(const fw_prompt *p)
{
    if (!p || p->num_seqs < 1 || p->q_heads < 1 || p->kv_heads < 1 || p->q_heads % p->kv_heads != 0)
        return FW_ERR_INVALID_ARG;
    if (p->total_q < 0 || p->total_k < 0 || !p->cu_q || !p->cu_k || !(p->scale > 0.f) || !(p->scale < 1e30f))
        return FW_ERR_INVALID_ARG;
    if (p->d != 64 && p->d != 128) return FW_ERR_UNSUPPORTED;
    if (p->q_heads / p->kv_heads > 128) return FW_ERR_UNSUPPORTED;
    const int64_t lim = ((int64_t)1 << 31) - 256;
    if (p->total_q >= lim || p->total_k >= lim) return FW_ERR_UNSUPPORTED;
    if (p->total_q > 0 && (!p->q || !aligned(p->q, 16) || !good_stride(p->q_row) || !good_stride(p->q_head)))
        return FW_ERR_INVALID_ARG;
    if (p->total_k > 0 && (!p->k || !p->v || !aligned(p->k, 16) || !aligned(p->v, 16) || !good_stride(p->k_row) ||
                           !good_stride(p->k_head) || !good_stride(p->v_row) || !good_stride(p->v_head)))
        return FW_ERR_INVALID_ARG;
    return FW_OK;
}

static fw_status check_cache8(const fw_cache8 *c)
{
    if (!c || c->cells < 1 || c->rows < 0 || c->rows % FW_CACHE8_BLOCK != 0) return FW_ERR_INVALID_ARG;
    if (c->format != FW_CACHE8_E4M3 && c->format != FW_CACHE8_INT8) return FW_ERR_INVALID_ARG;
    if (c->d != 64 && c->d != 128) return FW_ERR_UNSUPPORTED;
    if (!c->base || !c->capacity || !c->counts || !c->k_tail || !c->v_tail) return FW_ERR_INVALID_ARG;
    if (c->rows > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return FW_ERR_INVALID_ARG;
    if (c->rows >= ((int64_t)1 << 31) || c->cells > (1 << 24)) return FW_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16))
        return FW_ERR_INVALID_ARG;
    return FW_OK;
}

static fw_status check_cache8_query(const fw_cache8 *c, const fw_cache8_query *q)
{
    const fw_status st = check_cache8(c);
    if (st != FW_OK) return st;
    if (!q || q->kv_heads < 1 || q->group < 1 || q->m < 1 || c->cells % q->kv_heads != 0 || !(q->scale > 0.f) ||
        !(q->scale < 1e30f))
        return FW_ERR_INVALID_ARG;
    if ((int64_t)q->group * q->m > 65535) return FW_ERR_UNSUPPORTED;
    if (!q->q || !aligned(q->q, 16) || q->q_seq % 8 != 0 || q->q_tok % 8 != 0 || q->q_head % 8 != 0)
        return FW_ERR_INVALID_ARG;
    return FW_OK;
}

static bool multiple_of_8(int64_t x) { return x % 8 == 0 && x > -((int64_t)1 << 38) && x < ((int64_t)1 << 38); }

static fw_status check_pages(const fw_pages *p)
{
    if (!p || p->cells < 1 || p->num_pages < 1 || p->max_pages < 1) return FW_ERR_INVALID_ARG;
    if (!p->k || !p->v || !p->table || !p->held || !p->counts || !p->refs || !p->free_bits || !p->next)
        return FW_ERR_INVALID_ARG;
    if (!aligned(p->k, 16) || !aligned(p->v, 16)) return FW_ERR_INVALID_ARG;
    if (p->d != 64 && p->d != 128) return FW_ERR_UNSUPPORTED;
    if (p->page_rows != 16 && p->page_rows != 32 && p->page_rows != 64 && p->page_rows != 128) return FW_ERR_UNSUPPORTED;
    if (p->cells > (1 << 24) || (int64_t)p->num_pages * p->page_rows >= ((int64_t)1 << 31) ||
        (int64_t)p->cells * p->max_pages >= ((int64_t)1 << 31) || (int64_t)p->max_pages * p->page_rows >= ((int64_t)1 << 31))
        return FW_ERR_UNSUPPORTED;
    return FW_OK;
}

static fw_status check_pages_append(const fw_pages *p, int m)
{
    const fw_status st = check_pages(p);
    if (st != FW_OK) return st;
    if (m < 1) return FW_ERR_INVALID_ARG;
    // (the rows of all cells are numbered in 32 bits)
    return ((int64_t)m + 2 * p->page_rows) * p->cells >= ((int64_t)1 << 31) ? FW_ERR_UNSUPPORTED : FW_OK;
}

static fw_status check_pages_compact(const fw_pages *p, int64_t total)
{
    const fw_status st = check_pages(p);
    if (st != FW_OK) return st;
    return total < 0 ? FW_ERR_INVALID_ARG : total >= ((int64_t)1 << 35) ? FW_ERR_UNSUPPORTED : FW_OK;
}

static fw_status check_pages_query(const fw_pages *p, const fw_pages_query *q)
{
    const fw_status st = check_pages(p);
    if (st != FW_OK) return st;
    if (!q || q->kv_heads < 1 || q->group < 1 || q->m < 1 || q->longest < 0 || p->cells % q->kv_heads != 0 ||
        !(q->scale > 0.f) || !(q->scale < 1e30f))
        return FW_ERR_INVALID_ARG;
    if ((int64_t)q->group * q->m > 65535) return FW_ERR_UNSUPPORTED;
    // (blocks of 16 rows are numbered over all cells)
    if ((int64_t)p->cells * p->max_pages * (p->page_rows / 16) >= ((int64_t)1 << 31)) return FW_ERR_UNSUPPORTED;
    if (!q->q || !aligned(q->q, 16) || !multiple_of_8(q->q_seq) || !multiple_of_8(q->q_tok) || !multiple_of_8(q->q_head))
        return FW_ERR_INVALID_ARG;
    return FW_OK;
}

static fw_status check_rotation(const fw_rotation *r)
{
    if (!r || r->rows < 0 || r->q_heads < 1 || r->kv_heads < 0 || r->d < 1 || r->rot < 0 || r->rot > r->d)
        return FW_ERR_INVALID_ARG;
    if (r->interleaved != 0 && r->interleaved != 1) return FW_ERR_INVALID_ARG;
    if (r->w_dtype != FW_F32 && r->w_dtype != FW_BF16) return FW_ERR_INVALID_ARG;
    if (r->d % 16 != 0 || r->d > 256 || r->rot % 16 != 0) return FW_ERR_UNSUPPORTED;
    if (r->rows >= ((int64_t)1 << 31) || r->q_heads > 65536 || r->kv_heads > 65536) return FW_ERR_UNSUPPORTED;
    if (!(r->eps < 1e30f) || (r->eps < 0.f && (r->q_weight || r->k_weight))) return FW_ERR_INVALID_ARG;
    if (!aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return FW_ERR_INVALID_ARG;
    if (r->rows == 0) return FW_OK;
    if (r->rot > 0 && (!r->pos || !r->inv_freq)) return FW_ERR_INVALID_ARG;
    // (an input may be repeated by a stride of 0, an output's rows may not be one)
    if (!r->q || !r->q_out || !aligned(r->q, 16) || !aligned(r->q_out, 16) || !multiple_of_8(r->q_row) ||
        !multiple_of_8(r->q_head) || !good_stride(r->q_out_row) || !good_stride(r->q_out_head))
        return FW_ERR_INVALID_ARG;
    if (r->kv_heads > 0 && (!r->k || !r->k_out || !aligned(r->k, 16) || !aligned(r->k_out, 16) || !multiple_of_8(r->k_row) ||
                            !multiple_of_8(r->k_head) || !good_stride(r->k_out_row) || !good_stride(r->k_out_head)))
        return FW_ERR_INVALID_ARG;
    return FW_OK;
}

static fw_status check_rows(const fw_rows *r, RowsDev &R)
{
    if (!r) return FW_ERR_INVALID_ARG;
    if (r->num_groups < 0 || r->rows_per_group < 1 || r->max_n < 1) return FW_ERR_INVALID_ARG;
    if (r->d != 32 && r->d != 64 && r->d != 128 && r->d != 256) return FW_ERR_UNSUPPORTED;
    if (r->v_dtype != FW_F32 && r->v_dtype != FW_BF16) return FW_ERR_INVALID_ARG;
    if (r->num_groups > 0 && (!r->logits || !r->logit_off || !r->n || !r->v || !r->v_off))
        return FW_ERR_INVALID_ARG;
    if (((uintptr_t)r->v & 15u) != 0) return FW_ERR_INVALID_ARG;  // rows are read in 16-byte vectors
    R.num_groups = r->num_groups;
    R.R = r->rows_per_group;
    R.rows = r->num_groups * (int64_t)r->rows_per_group;
    R.d = r->d;
    R.max_n = r->max_n;
    R.v_dtype = r->v_dtype;
    R.logits = r->logits;
    R.logit_off = r->logit_off;
    R.n = r->n;
    R.v = r->v;
    R.v_off = r->v_off;
    return FW_OK;
}

}  // namespace fw

using namespace fw;

extern "C" {

const char *fw_status_string(fw_status s)
{
    switch (s) {
    case FW_OK: return "ok";
    case FW_ERR_INVALID_ARG: return "invalid argument";
    case FW_ERR_UNSUPPORTED: return "unsupported configuration";
    case FW_ERR_CUDA: return "CUDA error";
    case FW_ERR_TIMEOUT: return "timeout";
    case FW_ERR_WORKSPACE: return "workspace missing, too small or misaligned";
    case FW_ERR_NONFINITE: return "non-finite logit";
    default: return "unknown status";
    }
}

uint64_t fw_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

size_t fw_dense_and_topk_gap_workspace(const fw_rows *rows, int32_t nb)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK || nb < 1 || nb > 4) return 0;
    if (R.max_n <= 32) return 0;
    return long_gap_workspace(R, nb);
}

fw_status fw_dense_and_topk_gap(const fw_rows *rows, const int32_t *k, int32_t nb, const fw_gap_out *out,
                                void *workspace, size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (nb < 1 || nb > 4 || !k || !out || !out->gap || !out->dropped) return FW_ERR_INVALID_ARG;
    if (out->kept_bits && out->kept_words < (R.max_n + 31) / 32) return FW_ERR_INVALID_ARG;
    if (R.rows == 0) return FW_OK;
    cudaStream_t s = (cudaStream_t)stream;
    if (R.max_n <= 32) return small_gap(R, k, nb, *out, s);
    if (workspace_bytes < long_gap_workspace(R, nb) || !workspace || !aligned(workspace, 256))
        return FW_ERR_WORKSPACE;
    return long_gap(R, k, nb, *out, workspace, workspace_bytes, s);
}

size_t fw_swap_refine_workspace(const fw_rows *rows, int32_t nb, const fw_swap_params *prm)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK || nb < 1 || nb > 4 || !prm) return 0;
    if (R.max_n <= 32) return 0;
    return long_swap_workspace(R, nb, prm->E, prm->max_swaps);
}

fw_status fw_swap_refine(const fw_rows *rows, const int32_t *k, int32_t nb, const fw_gap_out *topk,
                         const fw_swap_params *prm, int32_t *n_swaps, int32_t *swap_out, int32_t *swap_in,
                         float *refined_gap, float *topk_gap, int32_t *capped, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (nb < 1 || nb > 4 || !k || !topk || !prm || !n_swaps || !swap_out || !swap_in || !refined_gap)
        return FW_ERR_INVALID_ARG;
    if (!topk->thr_key || !topk->thr_idx || !topk->o || !topk->row_max || !topk->row_sum)
        return FW_ERR_INVALID_ARG;
    if (prm->E < 0 || prm->max_swaps < 1) return FW_ERR_INVALID_ARG;
    if (R.rows == 0) return FW_OK;
    cudaStream_t s = (cudaStream_t)stream;
    if (R.max_n <= 32)
        return small_swap(R, k, nb, *topk, prm->E, prm->max_swaps, n_swaps, swap_out, swap_in,
                          refined_gap, topk_gap, capped, s);
    if (prm->E > kLongSwapMaxE) return FW_ERR_UNSUPPORTED;
    if (workspace_bytes < long_swap_workspace(R, nb, prm->E, prm->max_swaps) || !workspace ||
        !aligned(workspace, 256))
        return FW_ERR_WORKSPACE;
    return long_swap(R, k, nb, *topk, prm->E, prm->max_swaps, n_swaps, swap_out, swap_in, refined_gap,
                     topk_gap, capped, workspace, workspace_bytes, s);
}

size_t fw_group_vote_workspace(const fw_rows *rows, int32_t nb)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK || nb < 1 || nb > 4) return 0;
    return group_vote_workspace(R, nb);
}

fw_status fw_group_vote(const fw_rows *rows, const int32_t *s, int32_t nb, const fw_gap_out *topk, float *vote_gap,
                        float *vote_dropped, uint32_t *vote_bits, int32_t kept_words, int32_t *row_status,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (nb < 1 || nb > 4 || !s || !topk || !vote_gap) return FW_ERR_INVALID_ARG;
    if (!topk->o || !topk->row_max || !topk->row_sum) return FW_ERR_INVALID_ARG;
    if (vote_bits && kept_words < (R.max_n + 31) / 32) return FW_ERR_INVALID_ARG;
    if (R.rows == 0) return FW_OK;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < group_vote_workspace(R, nb))
        return FW_ERR_WORKSPACE;
    return group_vote(R, s, nb, *topk, vote_gap, vote_dropped, vote_bits, kept_words, row_status, workspace,
                      workspace_bytes, (cudaStream_t)stream);
}

size_t fw_best_subset_workspace(const fw_rows *rows)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK) return 0;
    return enum_workspace(R);
}

fw_status fw_best_subset(const fw_rows *rows, const int32_t *k, uint64_t *best_rank, float *best_gap,
                         int32_t *best_idx, int32_t k_max, float *topk_gap, int32_t *row_status,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (R.max_n > 32) return FW_ERR_UNSUPPORTED;
    if (!k || !best_rank || !best_gap || !best_idx || k_max < 1 || k_max > 32) return FW_ERR_INVALID_ARG;
    if (R.rows == 0) return FW_OK;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < enum_workspace(R)) return FW_ERR_WORKSPACE;
    return best_subset(R, k, best_rank, best_gap, best_idx, k_max, topk_gap, row_status, workspace,
                       workspace_bytes, (cudaStream_t)stream);
}

size_t fw_pool_best_subset_workspace(const fw_rows *rows, int32_t nb)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK || nb < 1 || nb > 4) return 0;
    return pool_best_subset_workspace(R, nb);
}

fw_status fw_pool_best_subset(const fw_rows *rows, const int32_t *k, int32_t nb, const int32_t *E,
                              const fw_gap_out *topk, float *best_gap, int32_t *best_idx, int32_t k_max,
                              float *topk_gap, int64_t *n_cand, int32_t *row_status, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (nb < 1 || nb > 4 || !k || !E || !topk || !best_gap || !best_idx || k_max < 1 || k_max > 32)
        return FW_ERR_INVALID_ARG;
    for (int b = 0; b < nb; ++b)
        if (E[b] < 0) return FW_ERR_INVALID_ARG;
    if (!topk->thr_key || !topk->thr_idx || !topk->o || !topk->row_max || !topk->row_sum) return FW_ERR_INVALID_ARG;
    if (R.rows == 0) return FW_OK;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < pool_best_subset_workspace(R, nb))
        return FW_ERR_WORKSPACE;
    return pool_best_subset(R, k, nb, E, *topk, best_gap, best_idx, k_max, topk_gap, n_cand, row_status, workspace,
                            (cudaStream_t)stream);
}

fw_status fw_sync_status(const int32_t *row_status, int64_t rows, int64_t *first_row, void *stream)
{
    if (first_row) *first_row = -1;
    if (rows < 0 || (rows > 0 && !row_status)) return FW_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    if (cudaStreamSynchronize(s) != cudaSuccess) return FW_ERR_CUDA;
    int32_t buf[4096];
    for (int64_t r0 = 0; r0 < rows; r0 += 4096) {
        const int64_t cnt = rows - r0 < 4096 ? rows - r0 : 4096;
        if (cudaMemcpyAsync(buf, row_status + r0, (size_t)cnt * 4, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
            cudaStreamSynchronize(s) != cudaSuccess)
            return FW_ERR_CUDA;
        for (int64_t i = 0; i < cnt; ++i)
            if (buf[i] != FW_OK) {
                if (first_row) *first_row = r0 + i;
                return (fw_status)buf[i];
            }
    }
    return FW_OK;
}

fw_status fw_fp32_fma_probe(int32_t blocks, int32_t iters, float *out, void *stream)
{
    if (blocks < 1 || iters < 1 || !out) return FW_ERR_INVALID_ARG;
    return fp32_fma_probe(blocks, iters, out, (cudaStream_t)stream);
}

fw_status fw_best_subset_read_stats(const fw_rows *rows, const void *workspace, fw_best_subset_stats *stats,
                                    void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (!stats || !workspace || !aligned(workspace, 256)) return FW_ERR_INVALID_ARG;
    if (R.max_n > 32) return FW_ERR_UNSUPPORTED;
    return best_subset_stats(R, workspace, stats, (cudaStream_t)stream);
}

size_t fw_contour_alloc_workspace(int32_t cells, int32_t T)
{
    if (cells < 1 || T < 1) return 0;
    return contour_workspace(cells, T);
}

fw_status fw_contour_alloc(const float *scores, int32_t cells, int32_t T, int32_t floor_, int64_t total_budget,
                           int32_t uniform_s, int32_t *counts, int64_t *offsets, int32_t *kept_pos, float *tau,
                           float *dropped_uniform, float *dropped_alloc, void *workspace, size_t workspace_bytes,
                           void *stream)
{
    if (!scores || cells < 1 || T < 1 || floor_ < 0 || uniform_s < 0) return FW_ERR_INVALID_ARG;
    const int F = floor_ < T ? floor_ : T;
    if (total_budget < (int64_t)cells * F || total_budget > (int64_t)cells * T) return FW_ERR_INVALID_ARG;
    if (!counts || !offsets || !kept_pos || !tau) return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < contour_workspace(cells, T))
        return FW_ERR_WORKSPACE;
    return contour_alloc(scores, cells, T, floor_, total_budget, uniform_s, counts, offsets, kept_pos, tau,
                         dropped_uniform, dropped_alloc, workspace, workspace_bytes, (cudaStream_t)stream);
}

size_t fw_contour_alloc_capped_workspace(int32_t cells, int32_t T)
{
    if (cells < 1 || T < 1) return 0;
    return contour_capped_workspace(cells, T);
}

fw_status fw_contour_alloc_capped(const float *scores, int32_t cells, int32_t T, int32_t floor_, int64_t total_budget,
                                  int32_t uniform_s, int32_t cap, int32_t *counts, int64_t *offsets, int32_t *kept_pos,
                                  float *tau, float *dropped_uniform, float *dropped_alloc, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    if (!scores || cells < 1 || T < 1 || floor_ < 0 || uniform_s < 0) return FW_ERR_INVALID_ARG;
    const int F = floor_ < T ? floor_ : T;
    if (total_budget < (int64_t)cells * F || total_budget > (int64_t)cells * T) return FW_ERR_INVALID_ARG;
    if (cap < F) return FW_ERR_INVALID_ARG;
    if (!counts || !offsets || !kept_pos || !tau) return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < contour_capped_workspace(cells, T))
        return FW_ERR_WORKSPACE;
    return contour_alloc(scores, cells, T, floor_, total_budget, uniform_s, counts, offsets, kept_pos, tau,
                         dropped_uniform, dropped_alloc, workspace, workspace_bytes, (cudaStream_t)stream, cap);
}

fw_status fw_ragged_compact(const void *K, const void *V, int32_t cells, int32_t T, int32_t row_bytes,
                            const int64_t *offsets, const int32_t *kept_pos, int64_t total, void *K_out,
                            void *V_out, void *stream)
{
    if (!K || !V || !offsets || !kept_pos || cells < 1 || T < 1 || total < 0) return FW_ERR_INVALID_ARG;
    if (row_bytes <= 0 || row_bytes % 16 != 0) return FW_ERR_INVALID_ARG;
    if (total > 0 && (!K_out || !V_out)) return FW_ERR_INVALID_ARG;
    if (!aligned(K, 16) || !aligned(V, 16) || (total > 0 && (!aligned(K_out, 16) || !aligned(V_out, 16))))
        return FW_ERR_INVALID_ARG;
    return ragged_compact(K, V, cells, T, row_bytes, offsets, kept_pos, total, K_out, V_out,
                          (cudaStream_t)stream);
}

fw_status fw_ragged_compact_to(const void *K, const void *V, int32_t cells, int32_t T, int32_t row_bytes,
                               const int64_t *offsets, const int32_t *kept_pos, const int64_t *base,
                               const int32_t *capacity, void *K_store, void *V_store, int32_t *status, void *stream)
{
    if (!K || !V || !offsets || !kept_pos || !base || !capacity || !K_store || !V_store || cells < 1 || T < 1)
        return FW_ERR_INVALID_ARG;
    if (row_bytes <= 0 || row_bytes % 16 != 0) return FW_ERR_INVALID_ARG;
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(K_store, 16) || !aligned(V_store, 16)) return FW_ERR_INVALID_ARG;
    return ragged_compact_to(K, V, cells, T, row_bytes, offsets, kept_pos, base, capacity, K_store, V_store, status,
                             (cudaStream_t)stream);
}

fw_status fw_ragged_append(void *K_store, void *V_store, const int64_t *base, const int32_t *capacity, int32_t *counts,
                           const void *new_K, const void *new_V, int32_t cells, int32_t m, int32_t row_bytes,
                           int32_t *status, void *stream)
{
    if (!K_store || !V_store || !base || !capacity || !counts || !new_K || !new_V || cells < 1 || m < 1)
        return FW_ERR_INVALID_ARG;
    if (row_bytes <= 0 || row_bytes % 16 != 0) return FW_ERR_INVALID_ARG;
    if ((int64_t)m * (row_bytes / 16) >= ((int64_t)1 << 31)) return FW_ERR_INVALID_ARG;
    if (!aligned(K_store, 16) || !aligned(V_store, 16) || !aligned(new_K, 16) || !aligned(new_V, 16))
        return FW_ERR_INVALID_ARG;
    return ragged_append(K_store, V_store, base, capacity, counts, new_K, new_V, cells, m, row_bytes, status,
                         (cudaStream_t)stream);
}

size_t fw_window_score_workspace(int32_t cells, int32_t T)
{
    if (cells < 1 || T < 1) return 0;
    return window_score_workspace(cells, T);
}

fw_status fw_window_score(const void *Qw, const void *K, int32_t cells, int32_t T, int32_t d, int32_t w, float scale,
                          int32_t pool, float *scores, int32_t *status, void *workspace, size_t workspace_bytes,
                          void *stream)
{
    if (!Qw || !K || !scores || cells < 1 || T < 1 || w < 1 || w > 32 || w > T) return FW_ERR_INVALID_ARG;
    if (pool < 1 || pool % 2 == 0 || !(scale > 0.f) || !(scale < 1e30f)) return FW_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return FW_ERR_UNSUPPORTED;
    if ((int64_t)cells * T >= ((int64_t)1 << 31) - 256) return FW_ERR_UNSUPPORTED;
    if (!aligned(Qw, 16) || !aligned(K, 16)) return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < window_score_workspace(cells, T))
        return FW_ERR_WORKSPACE;
    return window_score(Qw, K, cells, T, d, w, scale, pool, scores, workspace, status, (cudaStream_t)stream);
}

size_t fw_selector_audit_workspace(const fw_rows *rows, int32_t nb)
{
    RowsDev R;
    if (check_rows(rows, R) != FW_OK || nb < 1 || nb > 4) return 0;
    return selector_audit_workspace(R, nb);
}

fw_status fw_selector_audit(const fw_rows *rows, const int32_t *s, int32_t nb, const fw_gap_out *topk, float *es,
                            uint32_t *bits, int32_t words, void *workspace, size_t workspace_bytes, void *stream)
{
    RowsDev R;
    fw_status st = check_rows(rows, R);
    if (st != FW_OK) return st;
    if (nb < 1 || nb > 4 || !s || !topk || !es) return FW_ERR_INVALID_ARG;
    for (int b = 0; b < nb; ++b)
        if (s[b] < 1 || s[b] > 4096) return FW_ERR_INVALID_ARG;
    if (!topk->o || !topk->row_max || !topk->row_sum) return FW_ERR_INVALID_ARG;
    if (bits && words != (R.max_n + 31) / 32) return FW_ERR_INVALID_ARG;
    if (R.max_n > 65536) return FW_ERR_UNSUPPORTED;
    if (R.rows == 0) return FW_OK;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < selector_audit_workspace(R, nb))
        return FW_ERR_WORKSPACE;
    return selector_audit(R, s, nb, *topk, es, bits, words, workspace, (cudaStream_t)stream);
}

fw_status fw_prompt_attention(const fw_prompt *p, void *o, float *lse, int32_t *status, void *stream)
{
    const fw_status st = check_prompt(p);
    if (st != FW_OK) return st;
    if (p->total_q > 0 && (!o || !aligned(o, 16))) return FW_ERR_INVALID_ARG;
    return prompt_attention(*p, o, lse, status, (cudaStream_t)stream);
}

fw_status fw_cache8_compact(const fw_cache8 *c, const void *K, const void *V, int32_t T, int64_t cell_stride,
                            int64_t row_stride, const int64_t *offsets, const int32_t *kept_pos, int64_t total,
                            int32_t *status, void *stream)
{
    const fw_status st = check_cache8(c);
    if (st != FW_OK) return st;
    if (T < 1 || total < 0 || !offsets || !K || !V || !aligned(K, 16) || !aligned(V, 16)) return FW_ERR_INVALID_ARG;
    if (!good_stride(cell_stride) || !good_stride(row_stride)) return FW_ERR_INVALID_ARG;
    if (total > 0 && !kept_pos) return FW_ERR_INVALID_ARG;
    if (total >= ((int64_t)1 << 35)) return FW_ERR_UNSUPPORTED;
    return cache8_compact(*c, K, V, T, cell_stride, row_stride, offsets, kept_pos, total, status, (cudaStream_t)stream);
}

fw_status fw_cache8_append(const fw_cache8 *c, const void *new_K, const void *new_V, int32_t m, int32_t *status,
                           void *stream)
{
    const fw_status st = check_cache8(c);
    if (st != FW_OK) return st;
    if (m < 1 || !new_K || !new_V || !aligned(new_K, 16) || !aligned(new_V, 16)) return FW_ERR_INVALID_ARG;
    return cache8_append(*c, new_K, new_V, m, status, (cudaStream_t)stream);
}

size_t fw_cache8_attend_workspace(const fw_cache8 *c, const fw_cache8_query *q)
{
    if (check_cache8_query(c, q) != FW_OK) return 0;
    return cache8_attend_workspace(*c, *q);
}

fw_status fw_cache8_attend(const fw_cache8 *c, const fw_cache8_query *q, void *o, float *lse, int32_t *status,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    const fw_status st = check_cache8_query(c, q);
    if (st != FW_OK) return st;
    if (!o || !aligned(o, 16)) return FW_ERR_INVALID_ARG;
    const size_t need = cache8_attend_workspace(*c, *q);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return FW_ERR_WORKSPACE;
    return cache8_attend(*c, *q, o, lse, status, workspace, (cudaStream_t)stream);
}

size_t fw_pages_append_workspace(const fw_pages *p, int32_t m)
{
    return check_pages_append(p, m) == FW_OK ? pages_append_workspace(*p, m) : 0;
}

fw_status fw_pages_append(const fw_pages *p, const fw_pages_new *r, int32_t *status, void *workspace,
                          size_t workspace_bytes, void *stream)
{
    if (!r) return FW_ERR_INVALID_ARG;
    const fw_status st = check_pages_append(p, r->m);
    if (st != FW_OK) return st;
    if (r->kv_heads < 1 || p->cells % r->kv_heads != 0 || !r->k || !r->v || !aligned(r->k, 16) || !aligned(r->v, 16))
        return FW_ERR_INVALID_ARG;
    for (const int64_t x : {r->k_seq, r->k_tok, r->k_head, r->v_seq, r->v_tok, r->v_head})
        if (!multiple_of_8(x)) return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < pages_append_workspace(*p, r->m)) return FW_ERR_WORKSPACE;
    return pages_append(*p, *r, status, workspace, (cudaStream_t)stream);
}

size_t fw_pages_compact_workspace(const fw_pages *p, int64_t total)
{
    return check_pages_compact(p, total) == FW_OK ? pages_compact_workspace(*p, total) : 0;
}

fw_status fw_pages_compact(const fw_pages *p, const void *K, const void *V, int32_t T, int64_t cell_stride,
                           int64_t row_stride, const int64_t *offsets, const int32_t *kept_pos, int64_t total,
                           int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    const fw_status st = check_pages_compact(p, total);
    if (st != FW_OK) return st;
    if (!offsets || (total > 0 && !kept_pos) || (!K) != (!V)) return FW_ERR_INVALID_ARG;
    if (K && (T < 1 || !aligned(K, 16) || !aligned(V, 16) || !good_stride(cell_stride) || !good_stride(row_stride)))
        return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < pages_compact_workspace(*p, total))
        return FW_ERR_WORKSPACE;
    return pages_compact(*p, K, V, T, cell_stride, row_stride, offsets, kept_pos, total, status, workspace,
                         (cudaStream_t)stream);
}

size_t fw_pages_fork_workspace(const fw_pages *p) { return check_pages(p) == FW_OK ? pages_fork_workspace(*p) : 0; }

fw_status fw_pages_fork(const fw_pages *p, const int32_t *src, int32_t *status, void *workspace, size_t workspace_bytes,
                        void *stream)
{
    const fw_status st = check_pages(p);
    if (st != FW_OK) return st;
    if (!src) return FW_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < pages_fork_workspace(*p)) return FW_ERR_WORKSPACE;
    return pages_fork(*p, src, status, workspace, (cudaStream_t)stream);
}

size_t fw_pages_attend_workspace(const fw_pages *p, const fw_pages_query *q)
{
    return check_pages_query(p, q) == FW_OK ? pages_attend_workspace(*p, *q, true) : 0;
}

fw_status fw_pages_attend(const fw_pages *p, const fw_pages_query *q, void *o, float *lse, int32_t *status,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    const fw_status st = check_pages_query(p, q);
    if (st != FW_OK) return st;
    if (!o || !aligned(o, 16)) return FW_ERR_INVALID_ARG;
    const size_t need = pages_attend_workspace(*p, *q, false);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return FW_ERR_WORKSPACE;
    return pages_attend(*p, *q, o, lse, status, workspace, (cudaStream_t)stream);
}

void fw_pages_attend_give_up(int32_t tile, int32_t warp) { pages_attend_give_up(tile, warp); }

fw_status fw_qk_rotate(const fw_rotation *r, void *stream)
{
    const fw_status st = check_rotation(r);
    if (st != FW_OK) return st;
    return r->rows == 0 ? FW_OK : qk_rotate(*r, (cudaStream_t)stream);
}

}  // extern "C"
