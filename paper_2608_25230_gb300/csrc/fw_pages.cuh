// fw_pages.cuh -- the cache in pages as the kernels see it.
#pragma once

#include "fw_internal.h"

namespace fw {
namespace pages {

struct Pages {
    int cells, P, lg, N, width;  // P = 2^lg rows of a page (shifts for divisions: the attention over 8 cells of
                                   // 4,096 rows 7.9 -> 7.4 us), N pages, `width` entries of a table
    uint16_t *k, *v;
    int32_t *table, *held, *counts, *refs;
    uint32_t *bits;
    int32_t *next;

    __device__ int32_t *row(int h) const { return table + (int64_t)h * width; }
    __device__ bool is_page(int p) const { return (unsigned)p < (unsigned)N; }
};

inline Pages view(const fw_pages &p)
{
    return {p.cells, p.page_rows, __builtin_ctz((unsigned)p.page_rows), p.num_pages, p.max_pages,
            (uint16_t *)p.k, (uint16_t *)p.v, p.table, p.held, p.counts, p.refs, p.free_bits, p.next};
}

// A cell's rows and entries, checked against its table.
__device__ __forceinline__ fw_status cell_rows_ok(const Pages &s, int n, int held)
{
    return held < 0 || held > s.width || n < 0 || n > (int64_t)held * s.P ? FW_ERR_INVALID_ARG : FW_OK;
}
__device__ __forceinline__ fw_status cell_rows(const Pages &s, int h, int &n, int &held)
{
    n = s.counts[h];
    held = s.held[h];
    return cell_rows_ok(s, n, held);
}

}  // namespace pages
}  // namespace fw
