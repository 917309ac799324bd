// k_pages_attend.cu -- attention over a cache in pages: with a cell's n rows k, v, query token i
// of m sees the rows j < n - m + 1 + i:
//   x_j = scale (q . k_j),  o = sum_j softmax_j(x) v_j,  lse = log sum_j e^x_j.
//
// Bound: the rows' bytes.  A cell reads each of its rows once; rows in pages that cells share are read by each of them, from the
// cache where it still holds them (8 beams each over 2 prefixes of 16,384 rows, 8 heads, d = 128: 441 MB from memory where the
// cells' rows are 1,074 and the distinct ones 134, 127 us against 190 with pages of their own; 4 beams over 4 of 8,192: 136 MB, 53
// against 111).  Two ways over the cells:
//   few short cells (k_pages_attend_few): a cluster of up to 12 CTAs per cell, its blocks dealt out to all
//   their teams, whose states are joined in shared memory and sent to the CTA that joins a row's;
//   many (k_pages_attend): the blocks of all cells in a row are divided evenly over the teams of
//   the GPU, whatever the cells' lengths, so a team takes the end of one cell, whole cells and the
//   start of another, and waits for no other; the parts of cells that several teams share go to the
//   workspace, and a second kernel, launched behind the first one's tail, joins them in their order.
// A team is a warp for 8 query rows, or 2, 3, 4 or 6 warps, which read the same blocks against other query
// rows.  It fetches its blocks by TMA into a ring of its own, through page numbers that its warps
// have read 32 blocks ahead.  64 x 8 cells of about 16,384 rows, d = 128, 4 query rows: 593 to 601 us, 6.8 TB/s, the measured
// copy rate; 24 x 4 cells of 5,000, 7 query rows 44.5 us (4.8 TB/s: 3 us to the first blocks, the teams finish up to 8 us
// apart, 5 us to join); 8 cells of 4,096 7.5 us (latency: 2 us to the first block, 4 blocks a warp, 3 us to join).
// (Ranges of a CTA each, with its warps' states joined at the end of each cell's share and the parts by the last CTA to come,
// were faster for many long cells, 128 x 8 of 4,096 326 us against 338, and slower for others, 32 x 8 of 1,024 38 against 34, drafts
// of 20 rows 56 against 47.)
//
// A block is 16 rows, so it lies in one page whatever the pages' size.  Against 8 query rows, transposed on the
// warp-wide bf16 tensor instructions (a few query rows cannot fill a tcgen05 tile, and the stream
// of rows leaves the slower instructions mostly idle: 13 % of their time with 8 query rows): S^T = K Q^T, then O^T += V^T P^T.
// The weights enter as the sum of two bf16 numbers, the upper half of the fp32 weight's bits and what that leaves, so that 16
// bits of each count (they are summed for the divisor in 32): the instructions take bf16 beside bf16 values, a third number would
// add a third to the products, and what two leave out, at most 2^-16 of a weight, is below the 2^-8 of the output's own rounding by so
// much that the distance from 64 bits is the same to five digits (1.7438e-3 in the 2-norm, 2.2e-3 with one number).  Both are
// positive where the weight is, so that an infinite value stays one.  More query rows are bound
// by the reading of the blocks from shared memory and by issue: an SM takes about 12 tiles of 8 rows x 16 keys a us (64 cells x 4,096 rows: 20
// query rows 40 us, 32 45, 48 55, 64 73).
#include <algorithm>
#include <climits>

#include <cuda_bf16.h>

#include "fw_chain.cuh"
#include "fw_pages.cuh"
#include "tc_sm100.cuh"

namespace fw {
namespace {

using namespace pages;

constexpr int BR = 16;                 // rows of a block
constexpr uint32_t A_WAIT = 1u << 22;  // polls before a wait gives up

struct AttendArgs {
    Pages s;
    int kv_heads, group, m;
    uint32_t group_inv;  // 2^32 / group + 1 (0 for a group of 1)
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
    int G, teams;      // CTAs along the blocks, and their teams
    int cluster;       // CTAs of a cell (few cells)
    int tiles;         // of query rows
    int give_tile, give_warp;  // (tests) the warp of every team that is as if its waits had given up; -1: none
    int32_t *start;    // workspace: [cells] first block of each cell
    int32_t *plan;     // workspace: blocks per team
    int32_t *flags;    // workspace: [teams][2] statuses of parts, but for waits that gave up
    int32_t *failed;   // workspace: [tiles of rows][teams][warps of a team] the cell from which on a warp's waits gave up
    float2 *part_ml;   // workspace: [tiles of rows][teams][2][rows of a tile] (max, sum)
    float *part_o;     // workspace: the same with D columns, column 8 i + g at g D / 8 + i
};

// r / group for a query row r: both are below 2^16, so the product's upper half is exact
__device__ __forceinline__ int token_of(const AttendArgs &a, int r) { return a.group_inv ? __umulhi(r, a.group_inv) : r; }

// Blocks of a cell (0 where the cell is not valid), and its status.
__device__ __forceinline__ int cell_blocks(const Pages &s, int h, int &n, fw_status &st)
{
    int held;
    st = cell_rows(s, h, n, held);
    if (st != FW_OK) n = 0;
    return (n + BR - 1) / BR;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a float to what this CTA has at the shared address p, in CTA `rank` of the cluster
__device__ __forceinline__ void store_to(const void *p, int rank, float v)
{
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}" ::"r"(
                     tc::smem_u32(p)),
                 "r"(rank), "f"(v)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
        "%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS> __device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr));
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr));
}
// true for one lane of a warp that is there as a whole
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// A box of BR rows and both halves of their columns: [half][row][64], rows swizzled over 128 bytes.
__device__ __forceinline__ void tma_load_rows(void *dst, const void *tmap, int32_t row, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2}], "
        "[%4];" ::"r"(tc::smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(0), "r"(row), "r"(tc::smem_u32(bar))
        : "memory");
}

// CTAs of W warps in teams of TW.
template <int D, int TW, int W> struct Cfg {
    static constexpr int TEAMS = W / TW;
    static constexpr int TILE = BR * D * 2;  // bytes of a block's keys, or values
    static constexpr int STAGES = 196608 / (2 * TILE) / TEAMS;
    static_assert(STAGES % TW == 0 || W % TW != 0, "a stage is always filled by the same warp");
    static constexpr int RING = TEAMS * STAGES * 2 * TILE;
    static constexpr size_t SMEM = 1024 + RING;
    static constexpr int RT = TW * 8;  // query rows of a team
    // blocks under way: with more warps one less than there is room for, so that the warp that asks does not wait for the
    // others at every block
    static constexpr int AHEAD = STAGES - (TW > 1 ? 1 : 0);
};
__host__ __device__ constexpr int range_warps(int D, int TW) { return TW > 1 ? 12 : D == 64 ? 16 : 8; }
__host__ __device__ constexpr int few_warps(int TW) { return TW > 1 ? 12 : 8; }

// Byte offset of piece x (16 bytes, 8 columns) of row r in a tile.
__device__ __forceinline__ int piece(int r, int x) { return (x >> 3) * (BR * 128) + r * 128 + (((x ^ r) & 7) << 4); }

// A team's ring of blocks.  Its warps fetch them in turn (asking for a block takes a warp 0.3 us where many are under way: drafts of
// 20 rows over 64 cells of 1,537 19.6 us, 21.4 with one that asks for all); with more warps than one each says that it has read a block.
template <int D, int STAGES, int TW> struct Ring {
    static constexpr int TILE = BR * D * 2;
    uint8_t *mem;
    uint64_t *full, *empty;
    int32_t *page;  // of the stages' blocks, -1: none
    int mine, used = 0;  // blocks of the team: the next that this warp fetches, and that it reads
    bool ok = true;

    __device__ void init(int lane, int member)
    {
        mine = member;
        if (member == 0)
            for (int i = lane; i < STAGES; i += 32) {
                tc::mbar_init(&full[i], 1);
                if (TW > 1) tc::mbar_init(&empty[i], TW);
            }
        tc::mbar_init_fence();
    }
    // block of BR rows from row `at` of page `pg`
    __device__ void fetch(const CUtensorMap *tmK, const CUtensorMap *tmV, const Pages &s, int pg, int at)
    {
        const int st = mine % STAGES;
        if (TW > 1 && mine >= STAGES && ok) ok = tc::mbar_wait(&empty[st], (mine / STAGES - 1) & 1, A_WAIT);
        if (!ok) return;
        if (elect_one()) {  // (8 cells of 4,096 rows: 8.5 us, 8.8 where lane 0 asks)
            const bool is = s.is_page(pg);
            page[st] = is ? pg : -1;
            if (is) {
                const int row = (pg << s.lg) + at;
                tc::mbar_arrive_expect_tx(&full[st], 2 * TILE);
                tma_load_rows(mem + st * 2 * TILE, tmK, row, &full[st]);
                tma_load_rows(mem + st * 2 * TILE + TILE, tmV, row, &full[st]);
            } else {
                tc::mbar_arrive(&full[st]);
            }
        }
        mine += TW;
    }
    // the next block's stage, or -1 where the wait gave up
    __device__ int next()
    {
        const int st = used % STAGES;
        if (ok) ok = tc::mbar_wait(&full[st], (used / STAGES) & 1, A_WAIT);
        if (!ok) return -1;
        ++used;
        return st;
    }
    // a block has been read by every lane
    __device__ void release(int st, int lane)
    {
        __syncwarp();
        if (TW > 1 && lane == 0) tc::mbar_arrive(&empty[st]);
    }
    // copies still under way land before the CTA's memory goes
    __device__ void drain()
    {
        for (int b = mine - TW; b >= used; b -= TW) tc::mbar_wait(&full[b % STAGES], (b / STAGES) & 1, A_WAIT);
    }
};

// The pages of a walk over blocks first, first + step, ...: 32 of them at a time, one a lane.
struct Window {
    int from, pages;
    // (a block's entry lies in the table whatever its number, the pages are looked at when they are fetched)
    __device__ void load(const Pages &s, int h, int first, int step, int lane)
    {
        from = first;
        const int64_t e = ((int64_t)first + (int64_t)lane * step) * BR >> s.lg;
        pages = s.row(h)[e < s.width ? (int)e : s.width - 1];
    }
    __device__ int at(int i) const { return __shfl_sync(FW_FULL, pages, i); }
};

// A warp's 8 query rows and their running softmax over blocks of one cell.
template <int D> struct Rows {
    static constexpr int MT = D / 16;  // 16-column tiles of the output, and steps of the first product
    uint32_t qf[MT][2];            // row g of each 8, columns 2c, 2c + 1 (and 8 behind them) of each 16
    // The weights are 2^(x - ref), ref[e] a maximum of row 2c + e as it was at some block, 0 where nothing was
    // seen yet (mx has -inf there): it follows the maximum once a weight would pass 2^UP, so most blocks
    // need no maximum over the lanes and no rescaling.
    static constexpr float UP = 8.f;
    float O[MT][4], mx[2], ref[2], l[2];
    bool settled;  // every row has seen something

    __device__ __forceinline__ void read(const AttendArgs &a, int seq, int hk, int row0, int lane)
    {
        const int g = lane >> 2, c = lane & 3, rows = a.group * a.m;
        const int r = row0 + g, i = token_of(a, r);
        const uint16_t *src = a.q + seq * a.q_seq + i * a.q_tok + (int64_t)(hk * a.group + r - i * a.group) * a.q_head + 2 * c;
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                qf[k][e] = r < rows ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * e) : 0;
    }
    __device__ __forceinline__ void start()
    {
        settled = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) mx[e] = -INFINITY, ref[e] = l[e] = 0.f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) O[i][e] = 0.f;
    }

    // One block, rows BR blk .. of a cell of n, whose tile of keys lies at tk, the values' behind it.
    __device__ __forceinline__ void block(const AttendArgs &a, const uint8_t *tk, int blk, int n, int row0, int lane)
    {
        const int g = lane >> 2, c = lane & 3;
        const uint32_t ak = tc::smem_u32(tk), av = ak + BR * D * 2;
        // S^T: keys g, g + 8 of rows 2c, 2c + 1, in two sums, so that fewer products wait for one another
        float S[4], S2[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) S[z] = S2[z] = 0.f;
        const int lr = lane & 7, lm = lane >> 3;  // the row and the matrix that a lane's address is for
#pragma unroll
        for (int k = 0; k < MT; ++k) {
            uint32_t x[4];  // keys 0 .. 7, 8 .. 15 of the step's first 8 columns, then of the others
            ldmatrix4<false>(x, ak + piece(lr + 8 * (lm & 1), 2 * k + (lm >> 1)));
            mma(k & 1 ? S2 : S, x, qf[k][0], qf[k][1]);
        }
        uint32_t V[MT][4];  // keys 0 .. 7 of a tile's first 8 columns and of the others, then keys 8 .. 15
#pragma unroll
        for (int i = 0; i < MT; ++i) ldmatrix4<true>(V[i], av + piece(lr + 8 * (lm >> 1), 2 * i + (lm & 1)));
        const int j0 = blk * BR, all = n - a.m + 1;  // rows that every query sees
        const bool masked = j0 + BR > all;
        bool over = !settled;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int z = e; z < 4; z += 2) S[z] += S2[z];
            if (masked) {
                const int seen = min(all + token_of(a, row0 + 2 * c + e), n);
                if (j0 + g >= seen) S[e] = -INFINITY;
                if (j0 + 8 + g >= seen) S[2 + e] = -INFINITY;
            }
            over |= fmaf(fmaxf(S[e], S[2 + e]), a.scale2, -ref[e]) > UP;
        }
        if (__any_sync(FW_FULL, over)) {
            settled = true;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(S[e], S[2 + e]);
                top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 4));
                top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 8));
                top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 16)) * a.scale2;
                // (a row moves by its own scores alone, whatever the rows beside it do)
                const float old = mx[e], now = old == -INFINITY || top > old + UP ? top : old;
                const float al = now > old ? ex2(old - now) : 1.f;  // (0 where nothing was seen before)
                mx[e] = now;
                ref[e] = now == -INFINITY ? 0.f : now;
                settled = settled && now > -INFINITY;
                l[e] *= al;
#pragma unroll
                for (int i = 0; i < MT; ++i) O[i][e] *= al, O[i][2 + e] *= al;
            }
            settled = __all_sync(FW_FULL, settled);
        }
        // the weights' upper halves and what they leave, with 2^-22 of the weight more, so that it is 0 only where the
        // weight is
        uint32_t ph[2], pl[2];
        float r[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const float p = S[z] = ex2(fmaf(S[z], a.scale2, -ref[z & 1]));
            r[z] = fmaf(p, 0x1p-22f, p - __uint_as_float(__float_as_uint(p) & 0xffff0000u));
            l[z & 1] += p;
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            ph[z] = transpose8x8(__byte_perm(__float_as_uint(S[2 * z]), __float_as_uint(S[2 * z + 1]), 0x7632));
            pl[z] = transpose8x8(pack_bf16(r[2 * z], r[2 * z + 1]));
        }
        // O^T += V^T P^T: columns g, g + 8 of each 16, keys 2c, 2c + 1 and 8 behind them
        uint32_t in0 = ~0u, in1 = ~0u;
        bool odd = false;
        if (masked) {
            // rows behind the count hold anything
            in0 = (j0 + 2 * c < n ? 0xffffu : 0u) | (j0 + 2 * c + 1 < n ? 0xffff0000u : 0u);
            in1 = (j0 + 2 * c + 8 < n ? 0xffffu : 0u) | (j0 + 2 * c + 9 < n ? 0xffff0000u : 0u);
            if (a.m > 1) odd = unseen_odd(tk + BR * D * 2, max(0, all - j0), min(BR, n - j0), lane);
        }
        if (masked) {
            const int f = all - j0 - 2 * c;  // keys from here on are not seen by all
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                V[i][0] &= in0, V[i][1] &= in0, V[i][2] &= in1, V[i][3] &= in1;
                if (odd)
#pragma unroll
                    for (int z = 0; z < 4; ++z) V[i][z] = finite_from(V[i][z], f - 8 * (z >> 1));
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) mma(O[i], V[i], ph[0], ph[1]);
#pragma unroll
        for (int i = 0; i < MT; ++i) mma(O[i], V[i], pl[0], pl[1]);
        if (odd) add_odd(a, tk + BR * D * 2, S, j0, all, n, row0, lane);
    }

    // Whether rows [lo, hi) of a tile of values, which some queries do not see, hold any that are not finite: a
    // weight of 0 times one of those is NaN.  (The last m - 1 rows of a cell, so a block or a few.)
    __device__ static bool unseen_odd(const uint8_t *tv, int lo, int hi, int lane)
    {
        bool odd = false;
        for (int p = lo * (D / 8) + lane; p < hi * (D / 8); p += 32) {
            const uint4 x = *reinterpret_cast<const uint4 *>(tv + piece(p / (D / 8), p % (D / 8)));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
        }
        return __any_sync(FW_FULL, odd);
    }
    // A pair of keys' values with 0 in the place of those that are not finite, of the keys from `f` on.
    __device__ static uint32_t finite_from(uint32_t x, int f)
    {
        if (f <= 0 && (x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if (f <= 1 && (x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        return x;
    }
    // What they give the rows that do see them.
    __device__ void add_odd(const AttendArgs &a, const uint8_t *tv, const float (&P)[4], int j0, int all, int n, int row0,
                            int lane)
    {
        const int g = lane >> 2, c = lane & 3;
        for (int key = max(0, all - j0); key < min(BR, n - j0); ++key) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float p = __shfl_sync(FW_FULL, key < 8 ? P[e] : P[2 + e], (key & 7) * 4 + c);
                if (j0 + key >= all + token_of(a, row0 + 2 * c + e)) continue;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const float v = bf16_to_f32(*reinterpret_cast<const uint16_t *>(tv + piece(key, 2 * i + z) + 2 * g));
                        if (!isfinite(v)) O[i][2 * z + e] += p * v;
                    }
            }
        }
    }

    // The sums over all lanes of a row.
    __device__ __forceinline__ void close()
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[e];
            sum += __shfl_xor_sync(FW_FULL, sum, 4);
            sum += __shfl_xor_sync(FW_FULL, sum, 8);
            sum += __shfl_xor_sync(FW_FULL, sum, 16);
            l[e] = sum;
        }
    }
};

// Index of query row r of cell (seq, hk) in the outputs.
__device__ __forceinline__ int64_t out_row(const AttendArgs &a, int seq, int hk, int r)
{
    const int i = token_of(a, r);
    return ((int64_t)seq * a.m + i) * a.kv_heads * a.group + hk * a.group + (r - i * a.group);
}
// lse of a row with running maximum mx and sum l of 2^(x - mx)
__device__ __forceinline__ float lse_of(float mx, float l) { return l == 0.f ? -INFINITY : (mx + log2f(l)) * 0.6931471805599453f; }

template <int D, int TW>
__global__ void __launch_bounds__(32 * range_warps(D, TW), 1)
    k_pages_attend(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    constexpr int W = range_warps(D, TW), AT = 32 * W;
    using C = Cfg<D, TW, W>;
    constexpr int TEAMS = C::TEAMS, MT = D / 16, RT = C::RT;
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t full[TEAMS][C::STAGES], empty[TEAMS][C::STAGES];
    __shared__ int32_t s_page[TEAMS][C::STAGES];
    __shared__ int s_scan[W], s_h0[TEAMS], s_b0[TEAMS], s_n0[TEAMS];  // (s_*0: where each team's range begins)

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, c = lane & 3;
    const int team = wid / TW, member = wid % TW;
    const int cta = blockIdx.x, tile = blockIdx.y, row0 = tile * RT + member * 8, rows = a.group * a.m;
    const Pages &s = a.s;
    let_the_next_start();
    Ring<D, C::STAGES, TW> ring;
    ring.mem = sm + team * C::STAGES * 2 * C::TILE;
    ring.full = full[team];
    ring.empty = empty[team];
    ring.page = s_page[team];
    ring.init(lane, member);
    wait_for_the_one_before();

    // ---- the blocks of all cells, divided evenly over the teams of all CTAs
    const int per = (s.cells + AT - 1) / AT;
    const int h_lo = min(tid * per, s.cells), h_hi = min(h_lo + per, s.cells);
    int mine = 0, nb_lo = 0, n_lo = 0;
    for (int h = h_lo; h < h_hi; ++h) {
        int n;
        fw_status st;
        const int nb = cell_blocks(s, h, n, st);
        if (h == h_lo) nb_lo = nb, n_lo = n;
        mine += nb;
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(FW_FULL, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[wid] = incl;
    __syncthreads();
    int total = 0, before = incl - mine;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < wid) before += s_scan[w];
        total += s_scan[w];
    }
    // consecutive ranges go to different CTAs; at least four blocks each, so that there is less to join
    // (the blocks of all cells may be just below 2^31)
    const int quota = max((int)(((int64_t)total + a.G * TEAMS - 1) / (a.G * TEAMS)), 4);
    {
        int at = before;
        for (int h = h_lo; h < h_hi; ++h) {
            int n = n_lo;
            fw_status st;
            const int nb = h == h_lo ? nb_lo : cell_blocks(s, h, n, st);
            // the teams of this CTA whose ranges begin in the cell
            for (int w = 0; w < TEAMS; ++w) {
                const int64_t u = (int64_t)(w * a.G + cta) * quota;
                if (u >= at && u < (int64_t)at + nb) {
                    s_h0[w] = h;
                    s_b0[w] = (int)(u - at);
                    s_n0[w] = n;
                }
            }
            if (cta == 0 && tile == 0) a.start[h] = at;
            at += nb;
        }
        if (cta == 0 && tile == 0 && tid == 0) *a.plan = quota;
    }
    __syncthreads();
    const int gw = team * a.G + cta;
    const int64_t first = (int64_t)gw * quota;
    if (first >= total) return;
    int u = (int)first;
    const int u1 = (int)min(first + quota, (int64_t)total);

    // the warp's next block to fetch, by cell
    int left = u1 - u - member, ph = s_h0[team], pb = s_b0[team] + member, pn = s_n0[team], pnb = (pn + BR - 1) / BR;
    fw_status pst;
    Window win;
    win.from = -1;
    auto fetch = [&]() {
        if (left <= 0) return;
        while (pb >= pnb && ph + 1 < s.cells) {  // (a block is left, so a cell holds it)
            pb -= pnb;
            pnb = cell_blocks(s, ++ph, pn, pst);
            win.from = -1;
        }
        if (win.from < 0 || pb - win.from >= 32 * TW) win.load(s, ph, pb, TW, lane);
        ring.fetch(&tmK, &tmV, s, win.at((pb - win.from) / TW), pb * BR & (s.P - 1));
        left -= TW;
        pb += TW;
    };
    Rows<D> R;
    R.read(a, ph / a.kv_heads, ph % a.kv_heads, row0, lane);
#pragma unroll 1
    for (int i = member; i < C::AHEAD; i += TW) fetch();

    int h = s_h0[team], b = s_b0[team];  // the segment: blocks of one cell
    // the cell where the warp's waits give up: its rows are NaN there and in all cells behind
    auto gave = [&](int cell) {
        if (a.status && lane == 0) a.failed[((int64_t)tile * a.teams + gw) * TW + member] = row0 < rows ? cell : INT_MAX;
    };
    gave(INT_MAX);
    while (u < u1) {
        int n = s_n0[team];
        fw_status st;
        int nb = u == (int)first ? (n + BR - 1) / BR : cell_blocks(s, h, n, st);
        while (b >= nb && h + 1 < s.cells) {  // cells without rows, and the next cell
            b -= nb;
            nb = cell_blocks(s, ++h, n, st);
        }
        if (b >= nb) break;  // (never, unless the counts change under the call)
        const int bend = min(nb, b + (u1 - u));
        const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
        if (u != (int)first) R.read(a, seq, hk, row0, lane);
        R.start();
        bool bad = false;
        const bool was = ring.ok;
        if (tile == a.give_tile && member == a.give_warp) ring.ok = false;
#pragma unroll 1
        for (int blk = b; blk < bend; ++blk) {
            const int stage = ring.next();
            if (stage < 0) break;
            if (s_page[team][stage] < 0)
                bad = true;
            else if (row0 < rows)
                R.block(a, ring.mem + stage * 2 * C::TILE, blk, n, row0, lane);
            ring.release(stage, lane);
            if (ring.mine < ring.used + C::AHEAD) fetch();
        }
        R.close();
        const bool whole = b == 0 && bend == nb;
        const int seg = u == (int)first ? 0 : 1;
        float sum[2], inv[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            sum[e] = ring.ok ? R.l[e] : NAN;
            inv[e] = sum[e] == 0.f ? 0.f : 1.f / sum[e];
        }
        if (whole) {
            const int r = row0 + g;
            uint16_t *dst = a.o + out_row(a, seq, hk, r) * D + 2 * c;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint32_t x = transpose8x8(pack_bf16(R.O[i][2 * z] * inv[0], R.O[i][2 * z + 1] * inv[1]));
                    if (r < rows) *reinterpret_cast<uint32_t *>(dst + 16 * i + 8 * z) = x;
                }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = row0 + 2 * c + e;
            if (r >= rows) continue;
            if (whole) {
                if (a.lse && g == 0) a.lse[out_row(a, seq, hk, r)] = lse_of(R.mx[e], sum[e]);
            } else {
                const int64_t at = (((int64_t)tile * a.teams + gw) * 2 + seg) * RT + member * 8 + 2 * c + e;
                if (g == 0) a.part_ml[at] = make_float2(R.mx[e], sum[e]);
                float4 *dst = reinterpret_cast<float4 *>(a.part_o + at * D + g * (D / 8));
#pragma unroll
                for (int i = 0; i < MT; i += 2)
                    dst[i / 2] = make_float4(R.O[i][e], R.O[i][2 + e], R.O[i + 1][e], R.O[i + 1][2 + e]);
            }
        }
        if (was && !ring.ok) gave(h);
        if (tile == 0 && member == 0 && lane == 0) {
            const int code = bad ? FW_ERR_INVALID_ARG : FW_OK;
            if (!whole)
                a.flags[gw * 2 + seg] = code;
            else if (a.status)
                a.status[h] = code;
        }
        u += bend - b;
        b = bend;
    }
    ring.drain();
}

// The parts of a cell that several teams share, joined in their order; empty cells' outputs.  Each of a CTA's JW warps
// takes a row, or (SPREAD) all of them one row's parts, where there are few rows and so the parts may be many: the fewer
// the rows the more warps (8 cells x 4 rows of 150 parts each, 32,768 rows a cell: 35 us with 4 warps, 26 with 16; 64 cells x 20
// rows: 21.6 with 4, 27 with 8).  CTAs of 4 are small enough to wait beside the first kernel's.  Where statuses are asked for, a
// cell's last CTA sees to its.
template <int D, bool SPREAD, int JW> __global__ void __launch_bounds__(32 * JW, JW == 4 ? 5 : 1) k_pages_join(const AttendArgs a, int RT)
{
    constexpr int E = D / 32;
    __shared__ float s_o[SPREAD ? JW : 1][D];
    __shared__ float2 s_ml[JW];
    let_the_next_start();
    wait_for_the_one_before();
    const int h = blockIdx.x, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int r = SPREAD ? blockIdx.y : blockIdx.y * JW + wid;
    int n;
    fw_status st;
    const int nb = cell_blocks(a.s, h, n, st), quota = *a.plan, s = a.start[h];
    const int w0 = s / quota, w1 = nb > 0 ? (s + nb - 1) / quota + 1 : w0;  // the cell's teams
    const bool whole = w1 == w0 + 1;
    auto seg_of = [&](int p) { return p == w0 && s > p * quota ? 1 : 0; };
    if (a.status && blockIdx.y == gridDim.y - 1) {
        // the cell's status: whether any warp of any tile gave up in it, and where it has parts, theirs
        if (wid != 0) return;
        int code = st;
        if (!whole)
#pragma unroll 4
            for (int p = w0 + lane; p < w1; p += 32) code = max(code, a.flags[p * 2 + seg_of(p)]);
        const int each = (w1 - w0) * (RT / 8);
#pragma unroll 4
        for (int i = lane; i < each * a.tiles; i += 32)
            if (a.failed[((int64_t)(i / each) * a.teams + w0) * (RT / 8) + i % each] <= h) code = max(code, FW_ERR_TIMEOUT);
        code = __reduce_max_sync(FW_FULL, code);
        if (lane == 0 && (!whole || code != FW_OK)) a.status[h] = code;
        return;
    }
    if (whole) return;
    if (r >= a.group * a.m) return;  // (SPREAD: none is)
    const int64_t tile0 = (int64_t)(r / RT) * a.teams;
    auto part_at = [&](int p) { return ((tile0 + p) * 2 + seg_of(p)) * RT + r % RT; };
    // this warp's parts: 32 maxima and sums at a time, then their columns
    const int all = w1 - w0, each = SPREAD ? (all + JW - 1) / JW : all;
    const int p0 = SPREAD ? w0 + min(wid * each, all) : w0, p1 = min(p0 + each, w1);
    float M = -INFINITY, L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int q = p0; q < p1; q += 32) {
        // (the columns of B parts are asked for before the maxima are looked at, and B at a time after that)
        constexpr int B = 32 / E;
        const int cnt = min(32, p1 - q);
        const float2 ml = lane < cnt ? a.part_ml[part_at(q + lane)] : make_float2(-INFINITY, 0.f);
        float f = 0.f;
        for (int i = 0; i < cnt; i += B) {
            float x[B][E];
#pragma unroll
            for (int u = 0; u < B; ++u) {
#pragma unroll
                for (int e = 0; e < E; ++e) x[u][e] = 0.f;
                if (i + u < cnt) {
                    const float *src = a.part_o + part_at(q + i + u) * D + lane * E;
                    if constexpr (E == 4) {
                        const float4 y = *reinterpret_cast<const float4 *>(src);
                        x[u][0] = y.x, x[u][1] = y.y, x[u][2] = y.z, x[u][3] = y.w;
                    } else {
                        const float2 y = *reinterpret_cast<const float2 *>(src);
                        x[u][0] = y.x, x[u][1] = y.y;
                    }
                }
            }
            if (i == 0) {
                const float now = fmaxf(M, warp_max(ml.x)), old = M == now ? 1.f : ex2(M - now);
                f = ml.x == now ? 1.f : ex2(ml.x - now);
                M = now;
                L = fmaf(L, old, warp_sum(f * ml.y));
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= old;
            }
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const float g = __shfl_sync(FW_FULL, f, i + u);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(g, x[u][e], acc[e]);  // (a part that is not there is 0, its factor 0 or 1)
            }
        }
    }
    if constexpr (SPREAD) {
        if (lane == 0) s_ml[wid] = make_float2(M, L);
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[wid][lane * E + e] = acc[e];
        __syncthreads();
        if (wid != 0) return;
        const float2 ml = lane < JW ? s_ml[lane] : make_float2(-INFINITY, 0.f);
        M = warp_max(ml.x);
        const float f = ml.x == M ? 1.f : ex2(ml.x - M);
        L = warp_sum(f * ml.y);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < JW; ++w) {
            const float g = __shfl_sync(FW_FULL, f, w);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(g, s_o[w][lane * E + e], acc[e]);
        }
    }
    const int seq = h / a.kv_heads;
    const int64_t out = out_row(a, seq, h - seq * a.kv_heads, r);
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int at = lane * E + e, col = at % (D / 8) * 8 + at / (D / 8);
        a.o[out * D + col] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e] * inv));
    }
    if (a.lse && lane == 0) a.lse[out] = lse_of(M, L);
}

// Up to N states of a row joined: their (maximum, sum) and E of a lane's columns.
template <int N, int E, typename FM, typename FO>
__device__ __forceinline__ void join(int n, FM ml_of, FO o_of, float &M, float &L, float (&acc)[E])
{
    float2 ml[N];
    M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < N; ++w) ml[w] = w < n ? ml_of(w) : make_float2(-INFINITY, 0.f), M = fmaxf(M, ml[w].x);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < N; ++w) {
        if (w >= n) break;
        const float f = ml[w].x == M ? 1.f : ex2(ml[w].x - M);
        L = fmaf(f, ml[w].y, L);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(f, o_of(w, e), acc[e]);
    }
}

// A cluster of up to FEW CTAs per cell and tile of rows, its blocks dealt out to their teams one by one.
constexpr int FEW = 12;
template <int D, int TW> constexpr size_t few_smem() { return Cfg<D, TW, few_warps(TW)>::SMEM + (TW * 8 + FEW) * (D + 4) * 4; }
template <int D, int TW>
__global__ void __launch_bounds__(32 * few_warps(TW), 1)
    k_pages_attend_few(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    constexpr int W = few_warps(TW);
    using C = Cfg<D, TW, W>;
    constexpr int MT = D / 16, RT = C::RT, E = D / 32, LDO = D + 4, TEAMS = C::TEAMS, STAGES = C::STAGES;
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    float *s_o = reinterpret_cast<float *>(sm);               // [W][8][LDO], in the rings' place when these are done
    float *s_in = reinterpret_cast<float *>(sm + C::RING);    // [rows of this CTA][cluster][LDO]: the CTAs' states of them
    static_assert(W * 8 * LDO * 4 <= C::RING, "the states fit the rings");
    __shared__ __align__(8) uint64_t full[TEAMS][STAGES], empty[TEAMS][STAGES];
    __shared__ int32_t s_page[TEAMS][STAGES];
    __shared__ float2 s_ml[W][8];
    __shared__ float2 s_mlin[TW * 8 + FEW];
    __shared__ int s_code, s_codes[FEW];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, c = lane & 3;
    const int team = wid / TW, member = wid % TW;
    const int h = blockIdx.x / a.cluster, rank = blockIdx.x % a.cluster, rows = a.group * a.m;
    const int tile0 = blockIdx.y * RT, row0 = tile0 + member * 8;
    const Pages &s = a.s;
    const int first = rank + a.cluster * team, step = a.cluster * TEAMS;  // (the first blocks go to different CTAs)
    let_the_next_start();
    cluster_arrive();  // (waited for before anything is sent: every CTA of the cluster runs then)
    Ring<D, STAGES, TW> ring;
    ring.mem = sm + team * STAGES * 2 * C::TILE;
    ring.full = full[team];
    ring.empty = empty[team];
    ring.page = s_page[team];
    ring.init(lane, member);
    wait_for_the_one_before();
    Window win;
    win.load(s, h, first + member * step, step * TW, lane);  // (beside the counts)
    int n;
    fw_status st;
    const int nb = cell_blocks(s, h, n, st);
    if (tid == 0) s_code = st;
    __syncthreads();
    int pb = first + member * step;  // the warp's next block to fetch
    auto fetch = [&]() {
        if (pb >= nb) return;
        int i = (pb - win.from) / (step * TW);
        if (i >= 32) win.load(s, h, pb, step * TW, lane), i = 0;
        ring.fetch(&tmK, &tmV, s, win.at(i), pb * BR & (s.P - 1));
        pb += step * TW;
    };
    const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
    Rows<D> R;
    R.read(a, seq, hk, row0, lane);
#pragma unroll 1
    for (int i = member; i < C::AHEAD; i += TW) fetch();
    R.start();
    bool bad = false;
    if ((int)blockIdx.y == a.give_tile && member == a.give_warp && first < nb) ring.ok = false;
#pragma unroll 1
    for (int blk = first; blk < nb; blk += step) {
        const int stage = ring.next();
        if (stage < 0) break;
        if (s_page[team][stage] < 0)
            bad = true;
        else if (row0 < rows)
            R.block(a, ring.mem + stage * 2 * C::TILE, blk, n, row0, lane);
        ring.release(stage, lane);
        if (ring.mine < ring.used + C::AHEAD) fetch();
    }
    R.close();
    ring.drain();
    const int code = !ring.ok ? FW_ERR_TIMEOUT : bad ? FW_ERR_INVALID_ARG : FW_OK;
    if (lane == 0 && code != FW_OK) atomicMax(&s_code, code);
    // ---- the teams' rows joined in the CTA
    __syncthreads();  // (the rings have been read)
    if (g == 0) {
#pragma unroll
        for (int e = 0; e < 2; ++e) s_ml[wid][2 * c + e] = make_float2(R.mx[e], ring.ok ? R.l[e] : NAN);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) s_o[(wid * 8 + 2 * c + (f & 1)) * LDO + 16 * i + 8 * (f >> 1) + g] = R.O[i][f];
    __syncthreads();
    // ---- and sent to the CTA of the cluster that joins the row's: rows in turn to the CTAs
    cluster_wait();
    float M, L, acc[E];
    for (int x = wid; x < TW * 8; x += W) {  // row x & 7 of member x >> 3
        if (tile0 + x >= rows) break;
        join<TEAMS, E>(TEAMS, [&](int w) { return s_ml[w * TW + (x >> 3)][x & 7]; },
                       [&](int w, int e) { return s_o[(w * TW * 8 + x) * LDO + lane + 32 * e]; }, M, L, acc);
        const int to = x % a.cluster, slot = x - to + rank;
#pragma unroll
        for (int e = 0; e < E; ++e) store_to(&s_in[slot * LDO + lane + 32 * e], to, acc[e]);
        if (lane < 2) store_to(lane ? &s_mlin[slot].y : &s_mlin[slot].x, to, lane ? L : M);
    }
    if (tid == 0) store_to(&s_codes[rank], 0, __int_as_float(s_code));
    cluster_arrive();
    cluster_wait();
    for (int x = rank + a.cluster * wid; x < TW * 8; x += a.cluster * W) {
        const int r = tile0 + x, slot = x - rank;
        if (r >= rows) break;
        join<FEW, E>(a.cluster, [&](int w) { return s_mlin[slot + w]; }, [&](int w, int e) { return s_in[(slot + w) * LDO + lane + 32 * e]; },
                     M, L, acc);
        const int64_t out = out_row(a, seq, hk, r);
        const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
        for (int e = 0; e < E; ++e)
            a.o[out * D + lane + 32 * e] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e] * inv));
        if (a.lse && lane == 0) a.lse[out] = lse_of(M, L);
    }
    if (rank == 0 && wid == W - 1 && a.status) {
        const int codes = __reduce_max_sync(FW_FULL, lane < a.cluster ? s_codes[lane] : 0);
        if (lane == 0 && gridDim.y == 1) a.status[h] = codes;
        if (lane == 0 && gridDim.y > 1 && codes != FW_OK) atomicMax(a.status + h, codes);
    }
}

// The statuses that the clusters of several tiles raise (0.65 us in front of them; a single tile's cluster writes its cell's status).
__global__ void __launch_bounds__(128) k_pages_clear_status(const AttendArgs a)
{
    const int h = blockIdx.x * 128 + threadIdx.x;
    let_the_next_start();
    wait_for_the_one_before();
    if (h < a.s.cells) a.status[h] = FW_OK;
}

// How many clusters of each size find room on the GPU at once, a CTA an SM (GPUs differ in the SMs of their parts), and the
// sizes.  Sizes above 8 are let in for these kernels.
constexpr int SIZES = 6, SIZE[SIZES] = {12, 10, 8, 4, 2, 1};
void clusters_at_once(int (&room)[SIZES])
{
    static std::atomic<int> cache[64][SIZES];
    const int known[SIZES] = {9, 14, 16, 37, 77, 153};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) dev = -1;
    for (int i = 0; i < SIZES; ++i) {
        int n = dev >= 0 ? cache[dev][i].load(std::memory_order_relaxed) : known[i];  // (one more than it is)
        if (n == 0) {
            const auto kernel = k_pages_attend_few<128, 1>;
            constexpr size_t smem = few_smem<128, 1>();
            cudaLaunchAttribute at[1];
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = (unsigned)SIZE[i];
            at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)SIZE[i]);
            cfg.blockDim = dim3(32 * few_warps(1));
            cfg.dynamicSmemBytes = smem;
            cfg.attrs = at;
            cfg.numAttrs = 1;
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
                cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
                cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
                cudaGetLastError();  // (sizes that the GPU has no room for are not taken)
                n = 0;
            }
            cache[dev][i].store(++n, std::memory_order_relaxed);
        }
        room[i] = n - 1;
    }
}

// CTAs of a cell's cluster where that is the faster way, else 0 (ranges).  Both ways' times in us, from sweeps of cells of
// unlike lengths (the longest about twice the mean, which the host does not know).  Ranges: two launches, the sums
// over the cells, the joining, and the blocks of all over the GPU.  Clusters: a launch, and the longest cell's blocks over
// its CTAs, which share the memory with all others at first and have their SMs' whole rate at the end.  (Of 57 shapes, 8 to 128
// cells of 300 to 3,000 rows on average, 4 to 64 query rows, it takes the slower way for 2, by 1 to 3 us.  d = 128, 4 query rows,
// clusters against ranges: 8 cells of 3,000 9.6 us against 12.8, 64 of 300 6.6 against 11.3, of 1,000 14.6 against 15.4, 128 of 3,000 62
// against 39; 20 query rows, 64 of 3,000: 61 against 34.  A bound 2 or 4 times the longest cell asks for ranges earlier and costs at most
// what no bound costs: of 14 shapes, 2 times changed the way of 2, by 2 us, 4 times of 5, by 2 to 5: 8 cells of 4,000 7.6 to 12.0.)
int cluster_of(const fw_pages &p, const fw_pages_query &q, int TW, int tiles, int sms)
{
    if (q.longest == 0) return 0;
    // an SM's time for a block of 16 rows
    const double per = (p.d == 128 ? 1.0 : 0.5) * std::max(0.12, 0.08 * TW);
    const double memory = BR * p.d * 4 / 6.7e6;  // and the memory's
    // (no cell has more rows than its table)
    const int64_t longest = std::min<int64_t>(q.longest, (int64_t)p.max_pages * p.page_rows);
    const double blocks = (double)((longest + BR - 1) / BR), all = 0.5 * blocks * p.cells * tiles;
    int best = 0, room[SIZES];
    double least = 11.0 + std::max(all * per / sms, all * memory / tiles);
    clusters_at_once(room);
    for (int i = SIZES - 1; i >= 0; --i) {
        if (room[i] < 1) continue;
        const int64_t clusters = (int64_t)p.cells * tiles, waves = (clusters + room[i] - 1) / room[i];
        const double at_once = (double)std::min<int64_t>(clusters, room[i]) * SIZE[i] * memory / tiles;
        const double t = waves * (5.4 + 0.05 * SIZE[i] + blocks / SIZE[i] * 0.5 * (per + std::max(per, at_once)));
        if (t < least - 0.1) best = SIZE[i], least = t;
    }
    return best;
}

struct Plan {
    int few;  // CTAs of a cell's cluster, or 0
    int G, TW, teams, RT, tiles;
    size_t start, plan, flags, failed, ml, o, bytes;  // (of ranges, whichever way is taken: a workspace serves both)
};
void plan_of(const fw_pages &p, const fw_pages_query &q, Plan &x)
{
    int sms = 0;
    if (device_sms(&sms) != FW_OK) sms = 152;  // no device: the size query still answers
    const int rows = q.group * q.m;
    // as many warps a team as hold the rows; beyond 48 rows, tiles of 48 or 32, whichever leave fewer warps without rows
    // (64 x 4,096 rows, d = 128, 64 query rows: two tiles of 32 73 us, one of 96 90)
    const int need = (rows + 7) / 8;
    x.TW = need > 6 && (need + 5) / 6 * 6 > (need + 3) / 4 * 4 ? 4 : 6;
    for (const int tw : {4, 3, 2, 1})
        if (need <= tw) x.TW = tw;
    x.start = 0;
    x.RT = x.TW * 8;
    x.tiles = (rows + x.RT - 1) / x.RT;
    x.few = cluster_of(p, q, x.TW, x.tiles, sms);
    x.G = std::max(1, sms / x.tiles);  // one wave
    x.teams = x.G * (range_warps(p.d, x.TW) / x.TW);
    x.plan = align256((size_t)p.cells * 4);
    x.flags = x.plan + 256;
    x.failed = x.flags + align256((size_t)x.teams * 8);
    x.ml = x.failed + align256((size_t)x.tiles * x.teams * x.TW * 4);
    const size_t parts = (size_t)x.tiles * x.teams * 2 * x.RT;
    x.o = x.ml + align256(parts * 8);
    x.bytes = x.o + align256(parts * p.d * 4);
}

// Lets a kernel have clusters of more than 8 CTAs on the current device, once per device (a bit each).
fw_status wide_clusters(const void *kernel, std::atomic<uint64_t> &done)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FW_ERR_CUDA;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return FW_OK;
    FW_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    done.fetch_or(bit, std::memory_order_relaxed);
    return FW_OK;
}

template <typename K>
fw_status launch(K kernel, int grid, int tiles, int cluster, int threads, size_t smem, const CUtensorMap &mk,
                 const CUtensorMap &mv, const AttendArgs &a, std::atomic<uint64_t> &done, cudaStream_t s)
{
    const fw_status st = big_smem((const void *)kernel, smem, done);
    if (st != FW_OK) return st;
    return launch_chained(kernel, dim3((unsigned)grid, (unsigned)tiles), threads, smem, cluster, s, mk, mv, a);
}
template <int D, int TW>
fw_status launch_ranges(const Plan &x, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a, cudaStream_t s)
{
    constexpr int W = range_warps(D, TW);
    static std::atomic<uint64_t> done{0};
    return launch(k_pages_attend<D, TW>, x.G, x.tiles, 0, 32 * W, Cfg<D, TW, W>::SMEM, mk, mv, a, done, s);
}
template <int D, int TW>
fw_status launch_few(const Plan &x, int cells, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a, cudaStream_t s)
{
    constexpr int W = few_warps(TW);
    static std::atomic<uint64_t> done{0}, wide{0};
    if (x.few > 8) {
        const fw_status st = wide_clusters((const void *)k_pages_attend_few<D, TW>, wide);
        if (st != FW_OK) return st;
    }
    if (x.tiles > 1 && a.status) {
        const fw_status st = launch_chained(k_pages_clear_status, dim3((unsigned)((cells + 127) / 128)), 128, 0, 0, s, a);
        if (st != FW_OK) return st;
    }
    return launch(k_pages_attend_few<D, TW>, cells * x.few, x.tiles, x.few, 32 * W, few_smem<D, TW>(), mk, mv, a, done, s);
}
template <int D, int TW>
fw_status launch_one(const Plan &x, int cells, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a, cudaStream_t s)
{
    return x.few ? launch_few<D, TW>(x, cells, mk, mv, a, s) : launch_ranges<D, TW>(x, mk, mv, a, s);
}
template <int D>
fw_status attend(const Plan &x, int cells, int rows, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a,
                 cudaStream_t s)
{
    const fw_status st = x.TW == 1   ? launch_one<D, 1>(x, cells, mk, mv, a, s)
                         : x.TW == 2 ? launch_one<D, 2>(x, cells, mk, mv, a, s)
                         : x.TW == 3 ? launch_one<D, 3>(x, cells, mk, mv, a, s)
                         : x.TW == 4 ? launch_one<D, 4>(x, cells, mk, mv, a, s)
                                     : launch_one<D, 6>(x, cells, mk, mv, a, s);
    if (x.few) return st;
    if (st != FW_OK) return st;
    // the joining kernel starts as the first one's CTAs leave
    const bool spread = x.teams >= 4 * cells && (int64_t)cells * rows <= 16 * x.G;
    const int JW = !spread ? 4 : cells * rows <= 64 ? 16 : cells * rows <= 2 * x.G ? 8 : 4;
    const dim3 grid((unsigned)cells, (unsigned)(spread ? rows : (rows + JW - 1) / JW) + (a.status ? 1 : 0));
    return launch_chained(JW == 16 ? k_pages_join<D, true, 16> : JW == 8 ? k_pages_join<D, true, 8>
                          : spread ? k_pages_join<D, true, 4> : k_pages_join<D, false, 4>,
                          grid, 32 * JW, 0, 0, s, a, x.RT);
}

std::atomic<int64_t> g_give_up{-1};  // tile << 32 | warp

}  // namespace

void pages_attend_give_up(int tile, int warp) { g_give_up.store(tile < 0 || warp < 0 ? -1 : (int64_t)tile << 32 | warp); }

size_t pages_attend_workspace(const fw_pages &p, const fw_pages_query &q, bool any_longest)
{
    Plan x;
    plan_of(p, q, x);
    return any_longest || !x.few ? x.bytes : 0;
}

fw_status pages_attend(const fw_pages &p, const fw_pages_query &q, void *o, float *lse, int32_t *status, void *ws,
                       cudaStream_t s)
{
    Plan x;
    plan_of(p, q, x);
    // (rows of the pool as the second axis, the halves of their columns as the third)
    const int rows = p.num_pages * p.page_rows, halves = p.d / 64;
    CUtensorMap mk, mv;
    if (!make_tma_heads_bf16(&mk, p.k, 64, rows, halves, p.d, 64, BR, halves) ||
        !make_tma_heads_bf16(&mv, p.v, 64, rows, halves, p.d, 64, BR, halves))
        return FW_ERR_CUDA;
    uint8_t *w = (uint8_t *)ws;
    const uint32_t inv = q.group > 1 ? (uint32_t)(((uint64_t)1 << 32) / q.group + 1) : 0;
    const int64_t give = g_give_up.load(std::memory_order_relaxed);
    const AttendArgs a{view(p), q.kv_heads, q.group, q.m, inv, (const uint16_t *)q.q, q.q_seq, q.q_tok, q.q_head,
                       q.scale * 1.4426950408889634f, (uint16_t *)o, lse, status, x.G, x.teams, x.few,
                       x.tiles, (int)(give >> 32), (int)give, (int32_t *)(w + x.start), (int32_t *)(w + x.plan),
                       (int32_t *)(w + x.flags), (int32_t *)(w + x.failed), (float2 *)(w + x.ml), (float *)(w + x.o)};
    return p.d == 128 ? attend<128>(x, p.cells, q.group * q.m, mk, mv, a, s) : attend<64>(x, p.cells, q.group * q.m, mk, mv, a, s);
}

}  // namespace fw
