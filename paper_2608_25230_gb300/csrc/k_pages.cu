// k_pages.cu -- a cache of bf16 rows in pages: appends, compaction, forks.
//
// Every call changes the books (tables, counts, how many entries name a page, which pages are
// free) so that the result depends on the books before it alone, not on the order in which CTAs
// run: pages are handed out by one CTA (k_pages_plan) by sums over the cells in their order, and
// what runs in parallel counts entries up or down by integer atomics, whose order changes
// nothing.  A page that comes back is free for the calls behind, so the pages of a call are never
// read and handed out at once.
//
// Bound: append: latency, one CTA's sums and searches (5 us) and the copies behind it (a token to 256 cells, a fourth of
// them just forked: 8.0 us; 509 rows to 32 cells 8.4 us); compaction: memory, every kept row read and written once (256 x 32,768
// rows of 128 to an eighth: 183 us, 5.9 TB/s, of which the copies take 165 us, 6.5 TB/s; 64 x 7,001 rows in pages to a half:
// 45 us, the copies 35); fork: the tables' entries and their pages' counts (2,048 cells of 256 pages: 9.8 us; 24 cells 3.0 us).
#include <algorithm>
#include <type_traits>

#include "fw_chain.cuh"
#include "fw_pages.cuh"

namespace fw {
namespace {

using namespace pages;

constexpr int UR = 16;           // (2^4) rows that a warp copies at a time; no page holds less
constexpr int MW = 8;            // warps of a CTA of the copying kernels
constexpr int PT = 1024;         // threads of the plan's CTA
constexpr int WORDS = 4;         // words of the free bits that one of them asks for at a time

// ------------------------------------------------------------------ the plan
struct AppendArgs {
    Pages s;
    int m, kv_heads;
    const uint16_t *k, *v;
    int64_t k_seq, k_tok, k_head, v_seq, v_tok, v_head;
    int32_t *status;
    int32_t *first;    // workspace: [cells + 1] where each cell's pages stand in the list
    int32_t *list;     // workspace: the pages that are handed out
    int32_t *was;      // workspace: the pages that they replace, or -1
    int2 *plan;        // workspace: [cells] (rows before, -1 where the cell takes none; page to copy from or -1)
    int32_t *granted;  // workspace: pages handed out
};

struct CompactArgs {
    Pages s;
    const uint16_t *K, *V;  // null: the cells' own rows
    int T;
    int64_t cell_stride, row_stride;
    const int64_t *offsets;
    const int32_t *kept_pos;
    int64_t total;
    int32_t *status;
    int32_t *first, *list;  // workspace, as above
    int32_t *granted;       // workspace: pages handed out
};

// Whether entry i of a cell's table, which new rows touch, needs a page: those behind the held ones, and
// those that another entry names too.
__device__ __forceinline__ bool append_needs(const Pages &s, const int32_t *row, int held, int i)
{
    return i >= held || s.refs[row[i]] > 1;
}
// Pages that a cell needs, with its status.
__device__ __forceinline__ int cell_need(const AppendArgs &a, int h, int n, int held, fw_status &st)
{
    st = cell_rows_ok(a.s, n, held);
    if (st != FW_OK) return 0;
    const int i0 = n >> a.s.lg;
    const int64_t i1 = ((int64_t)n + a.m - 1) >> a.s.lg;
    if (i1 >= a.s.width) {
        st = FW_ERR_WORKSPACE;
        return 0;
    }
    const int32_t *row = a.s.row(h);
    int need = 0;
    for (int i = i0; i <= (int)i1; ++i) {
        if (i < held && !a.s.is_page(row[i])) {
            st = FW_ERR_INVALID_ARG;
            return 0;
        }
        need += append_needs(a.s, row, held, i);
    }
    return need;
}
// The same by a warp, a lane per entry (a thread takes half a microsecond for each).
__device__ __forceinline__ int cell_need_warp(const AppendArgs &a, int h, fw_status &st)
{
    const int lane = threadIdx.x & 31;
    int n, held;
    st = cell_rows(a.s, h, n, held);
    if (st != FW_OK) return 0;
    const int i0 = n >> a.s.lg;
    const int64_t i1 = ((int64_t)n + a.m - 1) >> a.s.lg;
    if (i1 >= a.s.width) {
        st = FW_ERR_WORKSPACE;
        return 0;
    }
    const int32_t *row = a.s.row(h);
    int need = 0;
    bool bad = false;
#pragma unroll 4
    for (int i = i0 + lane; i <= (int)i1; i += 32) {
        if (i < held && !a.s.is_page(row[i]))
            bad = true;
        else
            need += append_needs(a.s, row, held, i);
    }
    if (__any_sync(FW_FULL, bad)) {
        st = FW_ERR_INVALID_ARG;
        return 0;
    }
    return __reduce_add_sync(FW_FULL, need);
}
__device__ __forceinline__ int cell_need(const CompactArgs &a, int h, int n, int held, fw_status &st)
{
    st = cell_rows_ok(a.s, n, held);
    const int64_t o0 = a.offsets[h], o1 = a.offsets[h + 1];
    if (o0 < 0 || o1 < o0 || o1 > a.total) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && (o1 - o0 + a.s.P - 1) >> a.s.lg > a.s.width) st = FW_ERR_WORKSPACE;
    return st == FW_OK ? (int)((o1 - o0 + a.s.P - 1) >> a.s.lg) : 0;
}
// Rows that a cell of the compaction gets, or -1 where it is left as it was.  (Reads what the plan read, and
// what it wrote: the books' first change comes behind the last reader.)
__device__ __forceinline__ int compact_rows(const CompactArgs &a, int h, fw_status &st)
{
    cell_need(a, h, a.s.counts[h], a.s.held[h], st);
    if (st != FW_OK || (a.first[h + 1] > a.first[h] && a.first[h + 1] > *a.granted)) return -1;
    return (int)(a.offsets[h + 1] - a.offsets[h]);
}

// A free page's first entry, and an entry that goes.
__device__ __forceinline__ void take(const Pages &s, int page)
{
    s.refs[page] = 1;
    atomicAnd(&s.bits[page / 32], ~(1u << (page % 32)));
}
__device__ __forceinline__ void give(const Pages &s, int page)
{
    if (atomicSub(&s.refs[page], 1) == 1) atomicOr(&s.bits[page / 32], 1u << (page % 32));
}

// Several entries that go, all of them under way at once (a thread waits a microsecond for each otherwise).
template <int N> __device__ __forceinline__ void give_all(const Pages &s, const int (&page)[N])
{
    int old[N];
#pragma unroll
    for (int k = 0; k < N; ++k) old[k] = s.is_page(page[k]) ? atomicSub(&s.refs[page[k]], 1) : 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (old[k] == 1) atomicOr(&s.bits[page[k] / 32], 1u << (page[k] % 32));
}

// Exclusive sum over the CTA's threads; `all`: the sum of all.
__device__ __forceinline__ int scan_cta(int x, int &all, int (&s_scan)[32])
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(FW_FULL, incl, o);
        if (lane >= o) incl += y;
    }
    __syncthreads();  // (s_scan is free again)
    if (lane == 31) s_scan[wid] = incl;
    __syncthreads();
    const int mine = s_scan[lane];
    const int before = __reduce_add_sync(FW_FULL, lane < wid ? mine : 0);
    all = __reduce_add_sync(FW_FULL, mine);
    return before + incl - x;
}

// One CTA: what every cell needs, the free pages for it, and for appends the books.  WIDE: a warp per cell instead of a
// thread, for appends that touch several pages of few cells each.
template <typename Args, bool WIDE> __global__ void __launch_bounds__(PT, 1) k_pages_plan(const Args a)
{
    constexpr bool APPEND = std::is_same<Args, AppendArgs>::value;
    __shared__ int s_scan[32], s_granted;
    const Pages &s = a.s;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    let_the_next_start();
    if (tid == 0) s_granted = 0;
    wait_for_the_one_before();

    int n0 = 0, held0 = 0;  // (of the first cells, asked for before anything is waited for)
    if (!WIDE && tid < s.cells) n0 = s.counts[tid], held0 = s.held[tid];
    // The free bits from *next on, in a circle, the first word's lower part last; the first ones are asked for before
    // the cells are looked at.
    const int words = (s.N + 31) / 32, next = *s.next, start = s.is_page(next) ? next : 0, w0 = start / 32;
    uint32_t x[WORDS];
    auto word_of = [&](int t) { return w0 + t < words ? w0 + t : w0 + t - words; };
    auto look = [&](int b) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int t = b + i * PT + tid, w = word_of(t);
            x[i] = 0;
            if (t <= words) {
                x[i] = s.bits[w];
                if (t == 0) x[i] &= ~0u << (start % 32);
                if (t == words) x[i] &= ~(~0u << (start % 32));
                if (w == words - 1 && s.N % 32 != 0) x[i] &= ~(~0u << (s.N % 32));
            }
        }
    };
    look(0);

    if constexpr (WIDE) {
        for (int h = wid; h < s.cells; h += PT / 32) {
            fw_status st = FW_OK;
            const int need = cell_need_warp(a, h, st);
            if (lane == 0) {
                a.first[h] = need;
                if (a.status) a.status[h] = st;
                a.plan[h] = make_int2(st == FW_OK ? s.counts[h] : -1, -1);
            }
        }
        __syncthreads();
    }
    int want = 0;
    for (int b = 0; b < s.cells; b += PT) {
        const int h = b + tid;
        fw_status st = FW_OK;
        int need = 0;
        if (h < s.cells) {
            if constexpr (WIDE)
                need = a.first[h];
            else
                need = b == 0 ? cell_need(a, h, n0, held0, st) : cell_need(a, h, s.counts[h], s.held[h], st);
        }
        int all;
        const int at = want + scan_cta(need, all, s_scan);
        if (h < s.cells) {
            a.first[h] = at;
            if constexpr (!WIDE) {
                if (a.status) a.status[h] = st;
                if constexpr (APPEND) a.plan[h] = make_int2(st == FW_OK ? s.counts[h] : -1, -1);
            }
        }
        want += all;
    }
    if (tid == 0) a.first[s.cells] = want;

    // The first `want` free pages: a word of the bits a thread.  It writes its pages one after another; where a warp's words
    // hold many, its lanes write the pages of a word side by side (32,889 pages: 37,000 clocks one after another, whose
    // stores meet on no line, 3,000 side by side; 131 among 6,000 in use: 1,500 and 7,700).
    const int got_most = min(want, s.N);
    int found = 0;
    for (int b = 0; b <= words && found < got_most; b += PT * WORDS) {
        if (b > 0) look(b);
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (b + i * PT > words || found >= got_most) break;
            int all, at = found + scan_cta(__popc(x[i]), all, s_scan);
            const int w = word_of(b + i * PT + tid) * 32;
            if (__reduce_add_sync(FW_FULL, at < got_most ? __popc(x[i]) : 0) < 128) {
                for (uint32_t y = x[i]; y && at < got_most; y &= y - 1) a.list[at++] = w + __ffs(y) - 1;
            } else {
#pragma unroll 4
                for (int from = 0; from < 32; ++from) {
                    const uint32_t y = __shfl_sync(FW_FULL, x[i], from);
                    const int to = __shfl_sync(FW_FULL, at, from) + __popc(y & ((1u << lane) - 1));
                    const int page = __shfl_sync(FW_FULL, w, from) + lane;
                    if ((y >> lane & 1) && to < got_most) a.list[to] = page;
                }
            }
            found = min(found + all, got_most);
        }
    }
    __syncthreads();

    // Which cells it is enough for.
    for (int h = tid; h < s.cells; h += PT) {
        const int to = a.first[h + 1];
        if (to == a.first[h]) continue;
        if (to <= found) {
            atomicMax(&s_granted, to);
        } else {
            if (a.status) a.status[h] = FW_ERR_WORKSPACE;
            if constexpr (APPEND) a.plan[h].x = -1;
        }
    }
    __syncthreads();
    const int granted = s_granted;
    if (tid == 0 && granted > 0) {
        const int last = a.list[granted - 1];
        *s.next = last + 1 < s.N ? last + 1 : 0;
    }
    if (tid == 0) *a.granted = granted;
    if constexpr (APPEND) {
        for (int h = WIDE ? wid : tid; h < s.cells; h += WIDE ? PT / 32 : PT) {
            const int n = a.plan[h].x;
            if (n < 0) continue;
            const int held = s.held[h], i0 = n >> s.lg, i1 = (n + a.m - 1) >> s.lg;
            int32_t *row = s.row(h);
            int at = a.first[h];
            for (int b = i0; b <= i1; b += WIDE ? 32 : 1) {
                const int i = WIDE ? b + lane : b;
                const bool needs = i <= i1 && append_needs(s, row, held, i);
                const unsigned some = WIDE ? __ballot_sync(FW_FULL, needs) : needs;
                if (needs) {
                    const int was = i < held ? row[i] : -1, to = at + (WIDE ? __popc(some & ((1u << lane) - 1)) : 0);
                    row[i] = a.list[to];
                    a.was[to] = was;
                    if (i == i0 && (n & (s.P - 1)) != 0) a.plan[h].y = was;
                }
                at += __popc(some);
            }
            if (!WIDE || lane == 0) {
                s.held[h] = max(held, i1 + 1);
                s.counts[h] = n + a.m;
            }
        }
    }
}

// ------------------------------------------------------------------- copying
// UR rows of keys and of values by a warp, all reads under way at once: row i of `rows` from
// k_of(i), v_of(i) (null: zeros) to the rows behind kd, vd.
template <int D, typename F>
__device__ __forceinline__ void copy_rows(uint16_t *kd, uint16_t *vd, int lo, int hi, int lane, F source)
{
    constexpr int LPR = D / 8, RS = 32 / LPR, N = UR / RS;
    const int col = lane % LPR * 8, r0 = lane / LPR;
    uint4 x[2][N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = r0 + RS * i;
        const uint16_t *k, *v;
        source(r, k, v);  // (every lane: it may shuffle)
        const bool in = r >= lo && r < hi && k;
        x[0][i] = in ? __ldcs(reinterpret_cast<const uint4 *>(k + col)) : make_uint4(0, 0, 0, 0);
        x[1][i] = in ? __ldcs(reinterpret_cast<const uint4 *>(v + col)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = r0 + RS * i;
        if (r >= lo && r < hi) {
            *reinterpret_cast<uint4 *>(kd + r * D + col) = x[0][i];
            *reinterpret_cast<uint4 *>(vd + r * D + col) = x[1][i];
        }
    }
}

// New rows to their pages, and those of a page that was shared to the cell's own: a warp per cell and UR rows.  The first
// BOOK CTAs count the entries that came and went (behind the plan, which goes by how many entries name a page).
constexpr int BOOK = 4;
template <int D> __global__ void __launch_bounds__(32 * MW) k_pages_append(const AppendArgs a, int units)
{
    const Pages &s = a.s;
    const int lane = threadIdx.x & 31, id = ((int)blockIdx.x - BOOK) * MW + (threadIdx.x >> 5);
    let_the_next_start();
    wait_for_the_one_before();
    if (id < 0) {
        for (int t = blockIdx.x * 32 * MW + threadIdx.x, n = *a.granted; t < n; t += BOOK * 32 * MW) {
            const int was = a.was[t];
            take(s, a.list[t]);
            if (was >= 0) give(s, was);
        }
        return;
    }
    const int h = id / units;
    if (h >= s.cells) return;
    const int n = a.plan[h].x, from = a.plan[h].y;
    if (n < 0) return;
    const int64_t begin = (from >= 0 ? n & -s.P : n / UR * UR) + (int64_t)(id - h * units) * UR;
    const int end = n + a.m;
    if (begin >= end) return;
    const int r0 = (int)begin;
    const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
    const int64_t to = (((int64_t)s.row(h)[r0 >> s.lg] << s.lg) + (r0 & (s.P - 1))) * D;
    const int64_t old = (((int64_t)from << s.lg) + (r0 & (s.P - 1))) * D;
    copy_rows<D>(s.k + to, s.v + to, max(0, from >= 0 ? 0 : n - r0), min(UR, end - r0), lane,
                 [&](int r, const uint16_t *&k, const uint16_t *&v) {
                     const int64_t i = (int64_t)r0 + r - n;
                     k = i >= 0 ? a.k + seq * a.k_seq + i * a.k_tok + hk * a.k_head : s.k + old + r * D;
                     v = i >= 0 ? a.v + seq * a.v_seq + i * a.v_tok + hk * a.v_head : s.v + old + r * D;
                 });
}

// Entries of a cell that go: their pages are named by one less.  (Thread t of T.)
__device__ __forceinline__ void give_back(const Pages &s, const int32_t *row, int held, int t, int T)
{
    for (int i = t; i < held; i += 4 * T) {
        int page[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) page[k] = i + k * T < held ? row[i + k * T] : -1;
        give_all(s, page);
    }
}

// The kept rows to the pages that were taken for them: the list's pages, UR rows a warp, consecutive ones to a warp.
template <int D, bool OWN> __global__ void __launch_bounds__(32 * MW) k_pages_move(const CompactArgs a)
{
    const Pages &s = a.s;
    const int lane = threadIdx.x & 31, warps = gridDim.x * MW, id = blockIdx.x * MW + (threadIdx.x >> 5);
    const int lp = s.lg - 4;  // 2^lp units of a page
    let_the_next_start();
    wait_for_the_one_before();
    const int64_t units = (int64_t)*a.granted << lp, run = (units + warps - 1) / warps;
    const int64_t u0 = id * run, u1 = min(u0 + run, units);
    if (u0 >= u1) return;
    // the cell of the first: the last one whose pages start at or before it, 32 probes at a time
    int lo = 0, hi = s.cells;
    do {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const unsigned hit = __ballot_sync(FW_FULL, i < hi && a.first[min(i, hi - 1)] <= u0 >> lp);
        lo += max(__popc(hit) - 1, 0) * step;
        hi = min(lo + step, hi);
    } while (hi - lo > 1);
    int h = lo;
    for (int64_t u = u0; u < u1; ++u) {
        const int g = (int)(u >> lp);
        while (a.first[h + 1] <= g) ++h;
        const int64_t o0 = a.offsets[h];
        const int j0 = (int)(u - ((int64_t)a.first[h] << lp)) * UR, n = (int)(a.offsets[h + 1] - o0);
        if (j0 >= n) continue;
        const int rows = min(UR, n - j0);
        int64_t at = -1;  // lane r: where row r comes from
        if (lane < rows) {
            const int pos = a.kept_pos[o0 + j0 + lane];
            if constexpr (OWN) {
                const int page = pos >= 0 && pos < s.counts[h] ? s.row(h)[pos >> s.lg] : -1;
                at = s.is_page(page) ? (((int64_t)page << s.lg) + (pos & (s.P - 1))) * D : -1;
            } else {
                at = pos >= 0 && pos < a.T ? h * a.cell_stride + pos * a.row_stride : -1;
            }
        }
        const bool off = __any_sync(FW_FULL, lane < rows && at < 0);
        if (off && lane == 0 && a.status) atomicMax(a.status + h, FW_ERR_INVALID_ARG);
        const int64_t to = (((int64_t)a.list[g] << s.lg) + (j0 & (s.P - 1))) * D;
        copy_rows<D>(s.k + to, s.v + to, 0, rows, lane, [&](int r, const uint16_t *&k, const uint16_t *&v) {
            const int64_t f = __shfl_sync(FW_FULL, at, r);
            k = f >= 0 ? (OWN ? s.k : a.K) + f : nullptr;
            v = f >= 0 ? (OWN ? s.v : a.V) + f : nullptr;
        });
    }
}

// The cells' new tables, and the pages that they held given back: a CTA per cell.
__global__ void __launch_bounds__(128) k_pages_swap(const CompactArgs a)
{
    const Pages &s = a.s;
    const int h = blockIdx.x;
    fw_status st;
    let_the_next_start();
    wait_for_the_one_before();
    const int n = compact_rows(a, h, st);
    if (n < 0) return;
    int32_t *row = s.row(h);
    give_back(s, row, s.held[h], threadIdx.x, blockDim.x);
    __syncthreads();  // every thread has read the books
    const int need = (n + s.P - 1) >> s.lg;
    for (int i = threadIdx.x; i < need; i += blockDim.x) {
        const int page = a.list[a.first[h] + i];
        row[i] = page;
        take(s, page);
    }
    if (threadIdx.x == 0) {
        s.held[h] = need;
        s.counts[h] = n;
    }
}

// --------------------------------------------------------------------- forks
struct ForkArgs {
    Pages s;
    const int32_t *src;
    int32_t *status;
    int32_t *rows;   // workspace: [cells][width] the new tables
    int32_t *count;  // workspace: [cells] the new counts, -1 where a cell stays as it is
};

// A thread's first entries of a table (thread t of T), asked for before it is known how many there are: all lie in the table.
template <int T, int N> __device__ __forceinline__ void early(const Pages &s, int h, int t, int (&e)[N])
{
    const int32_t *row = s.row(h);
#pragma unroll
    for (int k = 0; k < N; ++k) e[k] = t + T * k < s.width ? __ldcg(row + t + T * k) : -1;
}
// f(i, e) for all n entries of the table that e begins, N a thread at a time: e[k] is entry i + T k, or -1 behind the n-th.
template <int T, int N, typename F>
__device__ __forceinline__ void entries(const Pages &s, int h, int n, int t, const int (&first)[N], F f)
{
    for (int i = t; i - t < n; i += T * N) {
        int e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = i + T * k >= n ? -1 : i == t ? first[k] : s.row(h)[i + T * k];
        f(i, e);
    }
}
// Whether any thread of a cell's has found something, and their wait for one another: a warp or a CTA.
template <int T> __device__ __forceinline__ bool any_of(bool x) { return T == 32 ? __any_sync(FW_FULL, x) : __syncthreads_or(x); }

// The table that a cell takes over, whose pages one more entry names then.
template <int T, int N> __device__ __forceinline__ void take_over(const ForkArgs &a, int h, int t)
{
    const Pages &s = a.s;
    const int from = a.src[h];
    const bool other = from >= 0 && from < s.cells && from != h;
    int n, held, rows = 0, first[N];
    if (other) early<T>(s, from, t, first);
    fw_status st = cell_rows(s, h, n, held);
    if (from >= s.cells) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && other) {
        st = cell_rows(s, from, rows, held);
        const int need = st == FW_OK ? (rows + s.P - 1) >> s.lg : 0;
        int32_t *to = a.rows + (int64_t)h * s.width;
        bool bad = false;
        entries<T, N>(s, from, need, t, first, [&](int i, const int (&e)[N]) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (i + T * k < need) {
                    to[i + T * k] = e[k];
                    bad |= !s.is_page(e[k]);
                }
        });
        if (any_of<T>(bad))
            st = FW_ERR_INVALID_ARG;
        else
            entries<T, N>(s, from, need, t, first, [&](int, const int (&e)[N]) {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (e[k] >= 0) atomicAdd(&s.refs[e[k]], 1);
            });
    }
    if (t == 0) {
        a.count[h] = st == FW_OK && from != h ? rows : -1;
        if (a.status) a.status[h] = st;
    }
}
// Its old pages given back (`first` begins its table, of `held` entries), behind all that took some over.
template <int T, int N> __device__ __forceinline__ void hand_over(const ForkArgs &a, int h, int held, int t, const int (&first)[N])
{
    const Pages &s = a.s;
    const int n = a.count[h];
    if (n < 0) return;
    entries<T, N>(s, h, held, t, first, [&](int, const int (&e)[N]) { give_all(s, e); });
    any_of<T>(false);  // (every thread has read the old entries)
    const int need = (n + s.P - 1) >> s.lg;
    int32_t *row = s.row(h);
#pragma unroll 4
    for (int i = t; i < need; i += T) row[i] = a.rows[(int64_t)h * s.width + i];
    if (t == 0) {
        s.held[h] = need;
        s.counts[h] = n;
    }
}

// A CTA per cell (a warp per cell: 2,048 cells of 256 pages 24 us, 12 so).
constexpr int KT = 128, KE = 2;
__global__ void __launch_bounds__(KT) k_pages_fork(const ForkArgs a)
{
    wait_for_the_one_before();
    let_the_next_start();  // (which reads tables before its own wait)
    take_over<KT, KE>(a, blockIdx.x, threadIdx.x);
}
__global__ void __launch_bounds__(KT) k_pages_fork_end(const ForkArgs a)
{
    // (the kernel before, k_pages_fork, changes no table, and has waited for what came before it, which so is in memory; an SM's own
    // cache is up to date only behind the wait, so these reads go past it)
    let_the_next_start();
    const int h = blockIdx.x, held = __ldcg(a.s.held + h);
    int first[KE];
    early<KT>(a.s, h, threadIdx.x, first);
    wait_for_the_one_before();
    hand_over<KT, KE>(a, h, held, threadIdx.x, first);
}
// Few cells of short tables: both by one CTA, a warp per cell.  The host takes 2 us less (11.3 against 13.5, which is longer than the GPU
// takes either way); the GPU in a graph, in us, one launch against two: 32 cells of 20 pages 3.6 and 3.3, 24 of 40 4.0 and 3.6, 32 of 64
// 5.2 and 3.5, of 128 7.5 and 4.2, of 250 5.6 and 5.3.
constexpr int ONE_CELLS = 32, ONE_PAGES = 256;
__global__ void __launch_bounds__(1024, 1) k_pages_fork_one(const ForkArgs a)
{
    const int h = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool mine = h < a.s.cells;
    let_the_next_start();
    wait_for_the_one_before();
    int first[KE], held = 0;
    if (mine) {
        held = a.s.held[h];
        early<32>(a.s, h, lane, first);
        take_over<32, KE>(a, h, lane);
    }
    __syncthreads();
    if (mine) hand_over<32, KE>(a, h, held, lane, first);
}

// Entries of a cell's table that m new rows touch, at most.
int64_t touched(const fw_pages &p, int m) { return ((int64_t)m + p.page_rows - 2) / p.page_rows + 1; }
size_t append_list(const fw_pages &p, int m) { return (size_t)std::min<int64_t>(p.num_pages, touched(p, m) * p.cells); }
size_t compact_list(const fw_pages &p, int64_t total)
{
    // (offsets out of order may name the same positions for several cells)
    const int64_t each = std::min<int64_t>(p.max_pages, (total + p.page_rows - 1) / p.page_rows);
    return (size_t)std::min<int64_t>(p.num_pages, each * p.cells);
}

}  // namespace

size_t pages_append_workspace(const fw_pages &p, int m)
{
    return align256(((size_t)p.cells + 1) * 4) + align256((size_t)p.cells * 8) + 2 * align256(append_list(p, m) * 4) + 256;
}

fw_status pages_append(const fw_pages &p, const fw_pages_new &r, int32_t *status, void *ws, cudaStream_t st)
{
    uint8_t *w = (uint8_t *)ws;
    AppendArgs a{view(p), r.m, r.kv_heads, (const uint16_t *)r.k, (const uint16_t *)r.v, r.k_seq, r.k_tok, r.k_head,
                 r.v_seq, r.v_tok, r.v_head, status, (int32_t *)w, nullptr, nullptr, nullptr, nullptr};
    w += align256(((size_t)p.cells + 1) * 4);
    a.plan = (int2 *)w;
    w += align256((size_t)p.cells * 8);
    a.list = (int32_t *)w;
    w += align256(append_list(p, r.m) * 4);
    a.was = (int32_t *)w;
    a.granted = (int32_t *)(w + align256(append_list(p, r.m) * 4));
    const int units = (p.page_rows - 1 + r.m + UR - 1) / UR;
    const unsigned grid = BOOK + (unsigned)(((int64_t)p.cells * units + MW - 1) / MW);
    // A warp per cell, 32 cells at a time (about 2 us a turn), or a thread, an entry at a time (0.3 us each).  Whole calls in us, a warp
    // against a thread, d = 64, pages of 16: 8 cells 6.6 and 6.9 for 64 rows, 7.4 and 11.0 for 300; 32 cells 7.4 and 7.3 for 40, 8.2
    // and 12.6 for 300; 64 cells 9.1 and 7.4 for 64, 10.6 and 12.4 for 300; 256 cells 25 and 21 for 300; 2,048 cells 129 and 33 for 64.
    const bool wide = touched(p, r.m) > 3 * (((int64_t)p.cells + 31) / 32);
    const fw_status planned = launch_chained(wide ? k_pages_plan<AppendArgs, true> : k_pages_plan<AppendArgs, false>,
                                             dim3(1), PT, 0, 0, st, a);
    if (planned != FW_OK) return planned;
    return launch_chained(p.d == 128 ? k_pages_append<128> : k_pages_append<64>, dim3(grid), 32 * MW, 0, 0, st, a, units);
}

size_t pages_compact_workspace(const fw_pages &p, int64_t total)
{
    return align256(((size_t)p.cells + 1) * 4) + 256 + align256(compact_list(p, total) * 4);
}

fw_status pages_compact(const fw_pages &p, const void *K, const void *V, int T, int64_t cell_stride, int64_t row_stride,
                        const int64_t *offsets, const int32_t *kept_pos, int64_t total, int32_t *status, void *ws,
                        cudaStream_t s)
{
    int sms = 0;
    const fw_status st = device_sms(&sms);
    if (st != FW_OK) return st;
    uint8_t *w = (uint8_t *)ws;
    CompactArgs a{view(p), (const uint16_t *)K, (const uint16_t *)V, T, cell_stride, row_stride, offsets, kept_pos, total,
                  status, (int32_t *)w, nullptr, nullptr};
    w += align256(((size_t)p.cells + 1) * 4);
    a.granted = (int32_t *)w;
    a.list = (int32_t *)(w + 256);
    const unsigned grid = (unsigned)sms * 4;
    fw_status done = launch_chained(k_pages_plan<CompactArgs, false>, dim3(1), PT, 0, 0, s, a);
    if (done == FW_OK)
        done = launch_chained(K ? p.d == 128 ? k_pages_move<128, false> : k_pages_move<64, false>
                              : p.d == 128 ? k_pages_move<128, true> : k_pages_move<64, true>,
                              dim3(grid), 32 * MW, 0, 0, s, a);
    return done == FW_OK ? launch_chained(k_pages_swap, dim3((unsigned)p.cells), 128, 0, 0, s, a) : done;
}

size_t pages_fork_workspace(const fw_pages &p)
{
    return align256((size_t)p.cells * 4) + align256((size_t)p.cells * p.max_pages * 4);
}

fw_status pages_fork(const fw_pages &p, const int32_t *src, int32_t *status, void *ws, cudaStream_t s)
{
    uint8_t *w = (uint8_t *)ws;
    const ForkArgs a{view(p), src, status, (int32_t *)(w + align256((size_t)p.cells * 4)), (int32_t *)w};
    if (p.cells <= ONE_CELLS && p.max_pages <= ONE_PAGES) return launch_chained(k_pages_fork_one, dim3(1), 1024, 0, 0, s, a);
    const fw_status taken = launch_chained(k_pages_fork, dim3((unsigned)p.cells), KT, 0, 0, s, a);
    return taken == FW_OK ? launch_chained(k_pages_fork_end, dim3((unsigned)p.cells), KT, 0, 0, s, a) : taken;
}

}  // namespace fw
