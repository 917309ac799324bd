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

// Threads of a CTA: the compaction's hold four pieces of the keys and four of the values each (d = 64, 108 cells x 22,554
// rows to an eighth: 19.5 us, 28.6 with 128 threads of two); the appends, of one block, are faster with more (512 cells x 7
// rows: 4.7 us, 5.6 with 64).
__host__ __device__ constexpr int compact_threads(int d) { return d; }
constexpr int AT = 128;
constexpr int compact_ctas(int d) { return d == 128 ? 8 : 16; }  // CTAs of the compaction per SM
constexpr int CHECK = 512;                                       // cells that one of its CTAs looks over

// A block's rows as a CTA holds them: thread t has the 16-byte pieces of column 8 * (t % LPR) of
// rows t / LPR + RS * i.
template <int D, int T> struct Lay {
    static constexpr int THREADS = T;
    static constexpr int LPR = D / 8, RS = THREADS / LPR, N = BR / RS, WARPS = THREADS / 32;
};

// Quantises the keys x[0] and the values x[1] of one block: the scales from the CTA's largest
// magnitudes, then the codes.  Rows at or past nrow are not filled (and hold zeros).  Every thread of the
// CTA calls it; s_max is free again two barriers later, so calls alternate between two.  Returns whether
// the block holds values that are not finite (the same for every thread).
template <int D, int FMT, int T>
__device__ __forceinline__ bool quantise_block(const Store &s, int64_t row, int nrow, uint4 (&x)[2][Lay<D, T>::N],
                                               uint32_t (&s_max)[2][Lay<D, T>::WARPS])
{
    using L = Lay<D, T>;
    const int tid = threadIdx.x, col = tid % L::LPR, r0 = tid / L::LPR;
    uint32_t top[2];
    int down[2] = {0, 0};  // octaves by which x was brought down
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < L::N; ++i) t = piece_top(x[kv][i], t);
        t = __reduce_max_sync(FW_FULL, top_of(t));
        if ((tid & 31) == 0) s_max[kv][tid >> 5] = t;
    }
    __syncthreads();
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        top[kv] = 0;
#pragma unroll
        for (int w = 0; w < L::WARPS; ++w) top[kv] = max(top[kv], s_max[kv][w]);
    }
    const bool odd = max(top[0], top[1]) >= 0x7f80u;
    if (odd) {  // (rare, and uniform: the scale is that of the finite values)
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < L::N; ++i) t = piece_top(finite_piece(x[kv][i], 0u, 0), t);
            t = __reduce_max_sync(FW_FULL, top_of(t));
            __syncthreads();
            if ((tid & 31) == 0) s_max[kv][tid >> 5] = t;
            __syncthreads();
            top[kv] = 0;
#pragma unroll
            for (int w = 0; w < L::WARPS; ++w) top[kv] = max(top[kv], s_max[kv][w]);
            // (the largest code times the largest scales is no number: such a block is encoded some octaves lower)
            const int e = scale_exponent<FMT>(top[kv]);
            down[kv] = e > 100 ? 100 : 0;
#pragma unroll
            for (int i = 0; i < L::N; ++i) x[kv][i] = finite_piece(x[kv][i], top_code_bits<FMT>(e - down[kv]), down[kv]);
        }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        const int e = scale_exponent<FMT>(top[kv]);
        if (tid == 0) s.scale(kv)[row / BR] = pow2f(e);
        const float inv = pow2f(down[kv] - e);
        uint8_t *codes = s.codes(kv) + row * D;
#pragma unroll
        for (int i = 0; i < L::N; ++i)
            if (r0 + L::RS * i < nrow)
                *reinterpret_cast<uint2 *>(codes + (size_t)(r0 + L::RS * i) * D + 8 * col) = encode8<FMT>(x[kv][i], inv);
    }
    return odd;
}

struct CompactArgs {
    Store s;
    const uint16_t *K, *V;
    int T;
    int64_t cell_stride, row_stride;
    const int64_t *offsets;
    const int32_t *kept_pos;
    int64_t total, slots;
    int checks, walks;  // CTAs that look over the cells, and behind them those that walk the slots
    int32_t *status;
};

// Whether a cell's offsets are in order; if all cells' are, they ascend within [0, total].
__device__ __forceinline__ bool offsets_ok(const CompactArgs &a, int h)
{
    return a.offsets[h] >= 0 && a.offsets[h + 1] >= a.offsets[h] && a.offsets[h + 1] <= a.total;
}

// A cell's rows in the compaction: its count, or 0 and why.
__device__ __forceinline__ fw_status compact_cell(const CompactArgs &a, int h, int64_t &o0, int64_t &base, int &n)
{
    int cap;
    o0 = a.offsets[h];
    const int64_t o1 = a.offsets[h + 1];
    fw_status st = cell_rows(a.s, h, base, cap);
    if (st == FW_OK && !offsets_ok(a, h)) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && o1 - o0 > cap) st = FW_ERR_WORKSPACE;
    n = st == FW_OK ? (int)(o1 - o0) : 0;
    return st;
}

// The cells' statuses as their arguments give them (the compaction adds what it finds in the rows).
__global__ void __launch_bounds__(256) k_cache8_status(const CompactArgs a)
{
    const int h = blockIdx.x * 256 + threadIdx.x;
    int64_t o0, base;
    int n;
    if (h < a.s.cells) a.status[h] = compact_cell(a, h, o0, base, n);
}

// The kept rows of all cells, block by block.  Bound: memory, the kept rows read (scattered rows of 2 d bytes) and the
// codes written.  Cell h's blocks are the slots from offsets[h] / 32 + h on, room for all of them (and one at least)
// without a prefix sum; a CTA takes a run of consecutive slots, finds its first one's cell by a search over the offsets
// and goes on from there.  All of a block's reads, keys and values, are under way at once (16 KB at d = 128), and the
// next block's positions with them.  The first CTAs write the cells' counts and look at their offsets: the slots hold
// every cell's blocks only if all offsets ascend within [0, total].  Where they do not, the first of these CTAs that
// sees it takes every block of every cell that is in order itself, one after another (about a microsecond a block; what
// the walk writes of them is the same), so that a cell's offsets concern no other cell.  256 cells x 32,768 rows to an
// eighth, d = 128: 133 to 139 us, 5.8 to 6.1 TB/s of rows read and codes written, 86 to 90 % of the measured copy rate
// (3.4 ms a CTA per cell, 180 us with an unpacked search for the largest magnitude, which left the integer pipe at 65
// %).
template <int D, int FMT>
__global__ void __launch_bounds__(Lay<D, compact_threads(D)>::THREADS, compact_ctas(D)) k_cache8_compact(const CompactArgs a)
{
    using L = Lay<D, compact_threads(D)>;
    __shared__ uint32_t s_max[2][2][Lay<D, compact_threads(D)>::WARPS];
    __shared__ int s_cell;
    const int tid = threadIdx.x, lane = tid & 31, col = tid % L::LPR, r0 = tid / L::LPR;
    const bool all = (int)blockIdx.x < a.checks;  // cell after cell instead of a run of the slots
    if (all) {
        const int lo = blockIdx.x * CHECK, hi = min(lo + CHECK, a.s.cells);
        bool bad = false;
        for (int c = lo + tid; c < hi; c += L::THREADS) {
            int64_t o0, base;
            int n;
            compact_cell(a, c, o0, base, n);
            a.s.counts[c] = n;
            bad |= !offsets_ok(a, c);
        }
        if (!__syncthreads_or(bad)) return;
        for (int c = 0; c < lo; c += L::THREADS)  // (lo is a multiple of THREADS)
            if (__syncthreads_or(!offsets_ok(a, c + tid))) return;
    }
    const int64_t run = (a.slots + a.walks - 1) / a.walks;
    const int64_t s0 = all ? 0 : run * (blockIdx.x - a.checks), s1 = all ? INT64_MAX : min(s0 + run, a.slots);
    auto first_slot = [&](int h) { return a.offsets[h] / BR + h; };  // (h <= cells)
    if (tid < 32 && !all) {
        int lo = 0, hi = a.s.cells;  // the last cell whose slots start at or before s0: 32 probes at a time
        do {
            const int step = (hi - lo + 31) / 32, i = lo + lane * step;
            const unsigned hit = __ballot_sync(FW_FULL, i < hi && first_slot(min(i, hi - 1)) <= s0);
            lo += max(__popc(hit) - 1, 0) * step;
            hi = min(lo + step, hi);
        } while (hi - lo > 1);
        if (lane == 0) s_cell = lo;
    }
    __syncthreads();
    int h = all ? -1 : s_cell - 1, n = 0, flip = 0;
    int64_t o0 = 0, base = 0, f0 = 0, f1 = s0;  // the cell's first kept position, first row, slots
    int pos[L::N];
    int64_t ahead = -1;  // the index of the positions that pos holds
    auto load_pos = [&](int64_t p) {
        ahead = p;
#pragma unroll
        for (int i = 0; i < L::N; ++i) pos[i] = p + r0 + L::RS * i < a.total ? a.kept_pos[p + r0 + L::RS * i] : -1;
    };
    for (int64_t slot = s0; slot < s1; ++slot) {
        if (slot >= f1) {
            if (++h >= a.s.cells) break;
            compact_cell(a, h, o0, base, n);
            f0 = all ? slot : first_slot(h);
            f1 = all ? slot + max(1, (n + BR - 1) / BR) : first_slot(h + 1);
        }
        const int64_t b = (slot - f0) * BR;
        if (b < 0 || b >= n) continue;  // (uniform)
        const int nrow = min(BR, n - (int)b);
        uint4 x[2][L::N];
        if (ahead != o0 + b) load_pos(o0 + b);
        bool off = false;
#pragma unroll
        for (int i = 0; i < L::N; ++i) {
            const bool in = r0 + L::RS * i < nrow && pos[i] >= 0 && pos[i] < a.T;
            off |= !in && r0 + L::RS * i < nrow;
            const int64_t at = (int64_t)h * a.cell_stride + (int64_t)pos[i] * a.row_stride + 8 * col;
            x[0][i] = in ? __ldcs(reinterpret_cast<const uint4 *>(a.K + at)) : make_uint4(0, 0, 0, 0);
            x[1][i] = in ? __ldcs(reinterpret_cast<const uint4 *>(a.V + at)) : make_uint4(0, 0, 0, 0);
        }
        load_pos(o0 + min((int64_t)n, b + BR));  // the next block's, or the next cell's first
        if (nrow < BR) {  // the open block's rows stay in the ring
#pragma unroll
            for (int i = 0; i < L::N; ++i) {
                const int r = r0 + L::RS * i;
                if (r < nrow)
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv)
                        *reinterpret_cast<uint4 *>(a.s.tail(kv) + ((int64_t)h * TL + (b + r) % TL) * D + 8 * col) = x[kv][i];
            }
        }
        const bool odd = quantise_block<D, FMT, L::THREADS>(a.s, base + b, nrow, x, s_max[flip]);
        flip ^= 1;
        if (a.status) {
            if (off) atomicMax(a.status + h, FW_ERR_INVALID_ARG);
            if (odd && tid == 0) atomicMax(a.status + h, FW_ERR_NONFINITE);
        }
    }
}

struct AppendArgs {
    Store s;
    const uint16_t *K, *V;
    int m;
    int32_t *status;
};

__device__ __forceinline__ fw_status append_cell(const AppendArgs &a, int h, int64_t &base, int &n)
{
    int cap;
    fw_status st = cell_rows(a.s, h, base, cap);
    n = a.s.counts[h];
    if (st == FW_OK && (n < 0 || n > cap)) st = FW_ERR_INVALID_ARG;
    if (st == FW_OK && a.m > cap - n) st = FW_ERR_WORKSPACE;
    return st;
}

// Quantises the block of a cell's n + m rows that starts at row b: rows before n from the ring, the
// others from the new ones.
template <int D, int FMT, bool RING>
__device__ __forceinline__ bool append_block(const AppendArgs &a, int h, int64_t base, int n, int b,
                                             uint32_t (&s_max)[2][Lay<D, AT>::WARPS])
{
    using L = Lay<D, AT>;
    const int tid = threadIdx.x, col = tid % L::LPR, r0 = tid / L::LPR, end = n + a.m;
    uint4 x[2][L::N];
#pragma unroll
    for (int i = 0; i < L::N; ++i) {
        const int r = b + r0 + L::RS * i;
        const int64_t slot = ((int64_t)h * TL + r % TL) * D + 8 * col;
        const int64_t at = ((int64_t)h * a.m + (r - n)) * D + 8 * col;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const uint16_t *src = r < n ? a.s.tail(kv) + slot : (kv ? a.V : a.K) + at;
            x[kv][i] = r < end ? *reinterpret_cast<const uint4 *>(src) : make_uint4(0, 0, 0, 0);
            if (RING && r >= n && r < end) *reinterpret_cast<uint4 *>(a.s.tail(kv) + slot) = x[kv][i];
        }
    }
    return quantise_block<D, FMT, AT>(a.s, base + b, min(BR, end - b), x, s_max);
}

// Bound: latency, one read of the rows, a barrier and the write (256 cells x 1 row and 512 x 7: 4.6 to
// 5.0 us).
// Appends of up to ONE_CTA rows: a CTA per cell takes the one or two blocks they touch, writes the ring and
// the count.  (The rows of the ring that it reads are fewer than 32 before the new ones: no slot of
// theirs is written.)
constexpr int ONE_CTA = BR;
template <int D, int FMT> __global__ void __launch_bounds__(Lay<D, AT>::THREADS) k_cache8_append(const AppendArgs a)
{
    __shared__ uint32_t s_max[2][2][Lay<D, AT>::WARPS];
    const int h = blockIdx.x, tid = threadIdx.x;
    int64_t base;
    int n;
    const fw_status st = append_cell(a, h, base, n);
    bool odd = false;
    if (st == FW_OK) {
        int flip = 0;
        for (int b = n / BR * BR; b < n + a.m; b += BR, flip ^= 1) odd |= append_block<D, FMT, true>(a, h, base, n, b, s_max[flip]);
    }
    __syncthreads();  // every thread has read the count
    if (tid == 0) {
        if (st == FW_OK) a.s.counts[h] = n + a.m;
        if (a.status) a.status[h] = st != FW_OK ? st : odd ? FW_ERR_NONFINITE : FW_OK;
    }
}

// Longer appends: a CTA per cell and block, then the ring and the counts by a second launch (one
// CTA per cell would take its blocks one after another, about a microsecond each).  d = 128, no status: 256 cells x 64 rows
// 6.9 us, x 512 rows 17 us; 8 cells x 2,048 rows 5.6 us.
__global__ void __launch_bounds__(256) k_cache8_append_status(const AppendArgs a)
{
    const int h = blockIdx.x * 256 + threadIdx.x;
    int64_t base;
    int n;
    if (h < a.s.cells) a.status[h] = append_cell(a, h, base, n);
}
template <int D, int FMT> __global__ void __launch_bounds__(Lay<D, AT>::THREADS) k_cache8_append_blocks(const AppendArgs a, int blocks)
{
    __shared__ uint32_t s_max[2][Lay<D, AT>::WARPS];
    const int h = blockIdx.x / blocks, i = blockIdx.x - h * blocks;
    int64_t base;
    int n;
    if (append_cell(a, h, base, n) != FW_OK) return;
    const int b = n / BR * BR + i * BR;
    if (b >= n + a.m) return;
    if (append_block<D, FMT, false>(a, h, base, n, b, s_max) && a.status && threadIdx.x == 0) atomicMax(a.status + h, FW_ERR_NONFINITE);
}
template <int D> __global__ void __launch_bounds__(256) k_cache8_append_end(const AppendArgs a)
{
    const int h = blockIdx.x;
    int64_t base;
    int n;
    if (append_cell(a, h, base, n) != FW_OK) return;
    const int end = n + a.m, rows = min(a.m, TL);
    for (int p = threadIdx.x; p < rows * (D / 8); p += 256) {
        const int r = end - rows + p / (D / 8), col = p % (D / 8);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
            *reinterpret_cast<uint4 *>(a.s.tail(kv) + ((int64_t)h * TL + r % TL) * D + 8 * col) =
                *reinterpret_cast<const uint4 *>((kv ? a.V : a.K) + ((int64_t)h * a.m + (r - n)) * D + 8 * col);
    }
    __syncthreads();
    if (threadIdx.x == 0) a.s.counts[h] = end;
}

}  // namespace

fw_status cache8_compact(const fw_cache8 &c, const void *K, const void *V, int T, int64_t cell_stride,
                         int64_t row_stride, const int64_t *offsets, const int32_t *kept_pos, int64_t total,
                         int32_t *status, cudaStream_t s)
{
    int sms = 0;
    const fw_status st = device_sms(&sms);
    if (st != FW_OK) return st;
    const int64_t slots = total / BR + c.cells, wave = (int64_t)sms * compact_ctas(c.d);
    const int checks = (c.cells + CHECK - 1) / CHECK;
    const int walks = (int)std::min(slots, std::max(wave - checks, wave / 2));  // (one wave, the checks with it)
    const CompactArgs a{store(c), (const uint16_t *)K, (const uint16_t *)V, T, cell_stride, row_stride, offsets,
                        kept_pos, total, slots, checks, walks, status};
    if (status) FW_LAUNCH(k_cache8_status, (unsigned)((c.cells + 255) / 256), 256, 0, s, a);
    FW_CACHE8_DISPATCH(c, FW_LAUNCH((k_cache8_compact<D, FMT>), (unsigned)(checks + walks), compact_threads(D), 0, s, a));
    return FW_OK;
}

fw_status cache8_append(const fw_cache8 &c, const void *new_K, const void *new_V, int m, int32_t *status,
                        cudaStream_t s)
{
    const AppendArgs a{store(c), (const uint16_t *)new_K, (const uint16_t *)new_V, m, status};
    if (m <= ONE_CTA) {
        FW_CACHE8_DISPATCH(c, FW_LAUNCH((k_cache8_append<D, FMT>), (unsigned)c.cells, AT, 0, s, a));
        return FW_OK;
    }
    const int64_t blocks = ((int64_t)m + 2 * BR - 2) / BR;  // that m rows can touch
    if (blocks * c.cells >= ((int64_t)1 << 31)) return FW_ERR_UNSUPPORTED;
    if (status) FW_LAUNCH(k_cache8_append_status, (unsigned)((c.cells + 255) / 256), 256, 0, s, a);
    FW_CACHE8_DISPATCH(c, {
        FW_LAUNCH((k_cache8_append_blocks<D, FMT>), (unsigned)(blocks * c.cells), AT, 0, s, a, (int)blocks);
        FW_LAUNCH(k_cache8_append_end<D>, (unsigned)c.cells, 256, 0, s, a);
    });
    return FW_OK;
}

}  // namespace fw
