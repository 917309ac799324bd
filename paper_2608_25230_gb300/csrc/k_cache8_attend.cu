// k_cache8_attend.cu -- attention over the 8-bit ragged store: with a cell's n
// rows of codes kc, vc and block scales sk, sv, query token i of m sees the rows
// j < n - m + 1 + i:
//   x_j = scale (q . kc_j) sk,  o = sum_j softmax_j(x) vc_j sv,  lse = log sum_j e^x_j.
//
// Bound: the codes' bytes, each read once from memory.  The blocks of all cells
// in a row are divided evenly over one CTA per SM, whatever the cells' lengths, so
// a CTA takes the end of one cell, whole cells and the start of another; its eight
// warps take every eighth block each and fetch them by TMA into a ring of their
// own, so no warp waits for another before a cell's end.  There the warps' states
// (running maximum, sum, output) are joined through shared memory; a cell within
// one CTA is done with that, the parts of the others go to the workspace and a
// second kernel, launched behind the first one's tail, joins them in their order.
//
// A block of 32 rows against 8 query rows, transposed on the warp-wide fp16 tensor
// instructions (a few rows of queries cannot fill a tcgen05 tile, and the stream of
// codes leaves the slower instructions mostly idle): S^T = K Q^T with the codes as
// the 16-row operand, then O^T += V^T P^T.  Codes of both formats are exact in
// fp16; a scale multiplies its block's products in fp32.  The queries of a row are
// brought below 2^15 by a power of two; the weights are 2^(x - max + 14), so that
// fp16 keeps 11 bits of every weight above 2^-28 of the largest.  The order of a
// contraction is free: a thread takes 16 consecutive bytes of a row where the
// instruction's layout asks for scattered ones, and the operand on the other side
// follows.
#include <algorithm>

#include "fw_cache8.cuh"
#include "tc_sm100.cuh"

namespace fw {
namespace {

using namespace cache8;

constexpr int BR = FW_CACHE8_BLOCK;
constexpr int AW = 8;                   // warps of a CTA
constexpr int AT = 32 * AW;
constexpr uint32_t A_WAIT = 1u << 22;   // polls before a wait gives up
constexpr float P_UP = 14.f;            // weights are 2^(x - max + P_UP)

struct AttendArgs {
    Store s;
    int kv_heads, group, m;
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
    int G;               // CTAs along the blocks
    int32_t *start;      // workspace: [cells] first unit of each cell
    int32_t *plan;       // workspace: units per CTA
    float2 *part_ml;     // workspace: [tiles of rows][G][2][rows of a tile] (max, sum)
    float *part_o;       // workspace: the same with D columns
};

// Blocks of a cell (0 where the cell is not valid), and its status.
__device__ __forceinline__ int cell_blocks(const Store &s, int h, int64_t &base, int &n, fw_status &st)
{
    int cap;
    st = cell_rows(s, h, base, cap);
    n = s.counts[h];
    if (st == FW_OK && (n < 0 || n > cap)) st = FW_ERR_INVALID_ARG;
    if (st != FW_OK) n = 0;
    return (n + BR - 1) / BR;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
        "%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// four codes of a word, in order, as two pairs of fp16
template <int FMT> __device__ __forceinline__ void decode4(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if constexpr (FMT == FW_CACHE8_E4M3) {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    } else {
        // a byte b with 0x64 above it is 1024 + b; with the sign bit flipped, 1152 + the signed value
        w ^= 0x80808080u;
        const __half2 off = __half2half2(__ushort_as_half(0x6480));  // 1152
        const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off);
        const __half2 y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}

template <int D> struct Cfg {
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int BLK = BR * D;                       // bytes of a block's codes
    static constexpr int RING = AW * STAGES * 2 * BLK;       // 192 KB
    static constexpr int LDO = D + 4;                        // floats of a row in the joining buffer
    static constexpr int JOIN = AW * 8 * LDO * 4;
    static constexpr size_t SMEM = 1024 + RING + JOIN;
};

// Position of a cell's row among the MMA's: row g of each 8 is key kappa(g).  It keeps
// the 16-byte reads of K (8 lanes: rows kappa(g), kappa(g + 1), four pieces) and of V (rows
// kappa(2c) or kappa(2c + 1), two pieces) on different banks of the swizzled tile.
__device__ __forceinline__ int kappa(int g) { return (g & 1) ? (((g - 1) ^ 4) | 1) : g; }

// Byte offset of piece x (16 bytes) of row r in a tile that TMA wrote swizzled over its row length.
template <int D> __device__ __forceinline__ int piece(int r, int x)
{
    return D == 128 ? r * 128 + ((x ^ (r & 7)) << 4) : r * 64 + ((x ^ ((r >> 1) & 3)) << 4);
}

template <int D, int FMT, int NT>
__global__ void __launch_bounds__(AT, 1) k_cache8_attend(const __grid_constant__ CUtensorMap tmK,
                                                         const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    using C = Cfg<D>;
    constexpr int MT = D / 16;        // 16-column tiles of the output
    constexpr int RT = 8 * NT;        // query rows of a CTA
    constexpr int H = D / 64;         // 64-byte halves of a row
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    float *s_o = reinterpret_cast<float *>(sm + C::RING);
    __shared__ __align__(8) uint64_t full[AW][C::STAGES];
    __shared__ float2 s_ml[AW][8];
    __shared__ int s_scan[AW], s_h0, s_b0, s_err;

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, c = lane & 3;
    const int cta = blockIdx.x, tile = blockIdx.y, row0 = tile * RT, rows = a.group * a.m;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0)
        for (int s = 0; s < C::STAGES; ++s) tc::mbar_init(&full[wid][s], 1);
    tc::mbar_init_fence();
    if (tid == 0) s_err = 0;

    // ---- the units (blocks) of all cells, divided evenly over the CTAs
    const int per = (a.s.cells + AT - 1) / AT;
    const int h_lo = min(tid * per, a.s.cells), h_hi = min(h_lo + per, a.s.cells);
    int mine = 0;
    for (int h = h_lo; h < h_hi; ++h) {
        int64_t base;
        int n;
        fw_status st;
        mine += cell_blocks(a.s, h, base, n, st);
        if (cta == 0 && tile == 0 && a.status) a.status[h] = st;
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
    for (int w = 0; w < AW; ++w) {
        if (w < wid) before += s_scan[w];
        total += s_scan[w];
    }
    // at least a block for every warp of a CTA: fewer parts to join
    const int quota = max((total + a.G - 1) / a.G, AW);
    const int u0 = min(cta * quota, total), u1 = min(u0 + quota, total);
    if (u0 >= before && u0 < before + mine) {  // the cell of the CTA's first unit
        int at = before;
        for (int h = h_lo; h < h_hi; ++h) {
            int64_t base;
            int n;
            fw_status st;
            const int nb = cell_blocks(a.s, h, base, n, st);
            if (u0 < at + nb) {
                s_h0 = h;
                s_b0 = u0 - at;
                break;
            }
            at += nb;
        }
    }
    if (cta == 0 && tile == 0) {
        int at = before;
        for (int h = h_lo; h < h_hi; ++h) {
            int64_t base;
            int n;
            fw_status st;
            a.start[h] = at;
            at += cell_blocks(a.s, h, base, n, st);
        }
        if (tid == 0) *a.plan = quota;
    }
    __syncthreads();
    if (u0 >= u1) return;

    // ---- queries: rows of 8, permuted like the codes, below 2^15
    uint8_t *ring = sm + wid * C::STAGES * 2 * C::BLK;
    // the warp's producer: its next unit to fetch, by cell
    int pu = u0 + wid, ph = s_h0, pb = s_b0 + wid, pn, pnb;
    int64_t pbase;
    fw_status pst;
    uint32_t pphase = 0;  // fetches so far
    pnb = cell_blocks(a.s, ph, pbase, pn, pst);
    auto fetch = [&]() {
        if (pu >= u1) return;
        while (pb >= pnb && ph + 1 < a.s.cells) {  // (a unit is left, so a cell holds it)
            pb -= pnb;
            pnb = cell_blocks(a.s, ++ph, pbase, pn, pst);
        }
        const int s = pphase % C::STAGES;
        if (lane == 0) {
            tc::mbar_arrive_expect_tx(&full[wid][s], 2 * C::BLK);
            const int32_t r = (int32_t)(pbase / BR) + pb;
            tc::tma_load_2d(ring + s * 2 * C::BLK, &tmK, 0, r * BR, &full[wid][s]);
            tc::tma_load_2d(ring + s * 2 * C::BLK + C::BLK, &tmV, 0, r * BR, &full[wid][s]);
        }
        ++pphase;
        pu += AW;
        pb += AW;
    };
#pragma unroll 1
    for (int s = 0; s < C::STAGES; ++s) fetch();

    int h = s_h0, b = s_b0, u = u0;  // the segment: blocks of one cell
    uint32_t cphase = 0;             // blocks consumed by this warp
    bool ok = true;
    while (u < u1) {
        int64_t base;
        int n;
        fw_status st;
        int nb = cell_blocks(a.s, h, base, n, st);
        while (b >= nb && h + 1 < a.s.cells) {  // cells without rows, and the next cell
            b -= nb;
            nb = cell_blocks(a.s, ++h, base, n, st);
        }
        if (b >= nb) break;  // (never, unless the counts change under the call)
        const int bend = min(nb, b + (u1 - u));
        const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;

        // this thread's part of the queries: row g of each 8, 16 consecutive columns of each half
        uint32_t qf[NT][H][8];
        float rf[NT][2];     // logits' factor of rows 2c, 2c + 1
        int seen[NT][2];     // rows of the cell they see
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + 8 * t + g;
            uint4 x[H][2];
            uint32_t top = 0;
            const int i = r / a.group;
            const uint16_t *src = a.q + seq * a.q_seq + i * a.q_tok + (int64_t)(hk * a.group + r - i * a.group) * a.q_head;
#pragma unroll
            for (int e = 0; e < H; ++e)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    x[e][f] = r < rows ? *reinterpret_cast<const uint4 *>(src + 64 * e + 16 * c + 8 * f) : make_uint4(0, 0, 0, 0);
                    top = piece_top(x[e][f], top);
                }
            top = top_of(top);
            top = max(top, __shfl_xor_sync(FW_FULL, top, 1));
            top = max(top, __shfl_xor_sync(FW_FULL, top, 2));
            // the largest magnitude's exponent to 14 (2^14 .. 2^15)
            const int k = min(max((int)(top >> 7) - 127 - 14, -126), 126);
            const float down = pow2f(-k);
#pragma unroll
            for (int e = 0; e < H; ++e)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const uint32_t w[4] = {x[e][f].x, x[e][f].y, x[e][f].z, x[e][f].w};
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        qf[t][e][4 * f + z] = pack_f16(__uint_as_float(w[z] << 16) * down, __uint_as_float(w[z] & 0xffff0000u) * down);
                }
            const float fac = a.scale2 * pow2f(k);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                rf[t][e] = __shfl_sync(FW_FULL, fac, (2 * c + e) * 4);
                seen[t][e] = n - a.m + 1 + (row0 + 8 * t + 2 * c + e) / a.group;
            }
        }
        const int all = n - a.m + 1;  // rows that every query sees

        float O[NT][MT][4], mx[NT][2], l[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            mx[t][0] = mx[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[t][i][e] = 0.f;
        }
        // the warp's first block at or behind b: units u0 + wid + 8 i
        const int first = b + ((wid - (u - u0)) & (AW - 1));
#pragma unroll 1
        for (int blk = first; blk < bend; blk += AW) {
            const int s = cphase % C::STAGES;
            const float sk = a.s.ks[base / BR + blk], sv = a.s.vs[base / BR + blk];
            if (ok) ok = tc::mbar_wait(&full[wid][s], (cphase / C::STAGES) & 1u, A_WAIT);
            if (!ok) break;
            ++cphase;
            const uint8_t *tk = ring + s * 2 * C::BLK, *tv = tk + C::BLK;
            // S^T: two tiles of 16 keys
            float S[NT][2][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int z = 0; z < 8; ++z) S[t][z >> 2][z & 3] = 0.f;
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int e = 0; e < H; ++e) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(tk + piece<D>(16 * z + kappa(g), 4 * e + c));
                    const uint4 y = *reinterpret_cast<const uint4 *>(tk + piece<D>(16 * z + 8 + kappa(g), 4 * e + c));
                    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t a0, a1, a2, a3;
                        decode4<FMT>(xw[k], a0, a2);
                        decode4<FMT>(yw[k], a1, a3);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma(S[t][z], a0, a1, a2, a3, qf[t][e][2 * k], qf[t][e][2 * k + 1]);
                    }
                }
            // weights: keys kappa(g) + 8 i of rows 2c, 2c + 1
            const int j0 = blk * BR + kappa(g);
            const bool masked = blk * BR + BR > all;
            uint32_t pb4[NT][4];
            bool grew = false;
            float al[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float f = rf[t][e] * sk;
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &x = S[t][i >> 1][2 * (i & 1) + e];
                        x *= f;
                        if (masked && j0 + 8 * i >= seen[t][e]) x = -INFINITY;
                        top = fmaxf(top, x);
                    }
                    top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(FW_FULL, top, 16));
                    const float old = mx[t][e], now = fmaxf(old, top);
                    grew |= now > old;
                    al[t][e] = now > old ? ex2(old - now) : 1.f;  // (0 where nothing was seen before)
                    mx[t][e] = now;
                    const float ref = now == -INFINITY ? 0.f : now - P_UP;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &x = S[t][i >> 1][2 * (i & 1) + e];
                        x = ex2(x - ref);
                        sum += x;
                    }
                    l[t][e] = fmaf(l[t][e], al[t][e], sum);
                }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    pb4[t][i] = transpose8x8(pack_f16(S[t][i >> 1][2 * (i & 1)], S[t][i >> 1][2 * (i & 1) + 1]));
            if (__any_sync(FW_FULL, grew)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) O[t][i][e] *= al[t][e & 1];
            }
            // O^T += sv V^T P^T: keys kappa(2c), kappa(2c + 1), 8 behind them, then 16
            const bool stale = blk * BR + BR > n;
            constexpr int VW = D / 32;  // words of a row's D / 8 columns
            uint32_t v[8][VW];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = 8 * (i >> 1) + kappa(2 * c + (i & 1));
                if constexpr (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(tv + piece<D>(key, g));
                    v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(tv + piece<D>(key, g >> 1) + 8 * (g & 1));
                    v[i][0] = x.x, v[i][1] = x.y;
                }
                if (stale && blk * BR + key >= n) {  // rows behind the count hold anything
#pragma unroll
                    for (int w = 0; w < VW; ++w) v[i][w] = 0;
                }
            }
            __syncwarp();
            fetch();  // every lane has read the stage
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                // columns 4w .. 4w + 3 of the thread's: pairs of keys side by side
                uint32_t p[4][4];  // [pair of keys][column]
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    decode4<FMT>(__byte_perm(v[2 * i][w], v[2 * i + 1][w], 0x5140), p[i][0], p[i][1]);
                    decode4<FMT>(__byte_perm(v[2 * i][w], v[2 * i + 1][w], 0x7362), p[i][2], p[i][3]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        float x[4] = {0.f, 0.f, 0.f, 0.f};
                        mma(x, p[0][2 * f], p[0][2 * f + 1], p[1][2 * f], p[1][2 * f + 1], pb4[t][0], pb4[t][1]);
                        mma(x, p[2][2 * f], p[2][2 * f + 1], p[3][2 * f], p[3][2 * f + 1], pb4[t][2], pb4[t][3]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) O[t][2 * w + f][e] = fmaf(sv, x[e], O[t][2 * w + f][e]);
                    }
            }
        }
        if (!ok) s_err = 1;
        // ---- the warps' states joined, 8 rows at a time
        const bool whole = b == 0 && bend == nb;
        const int part = cta * 2 + (u == u0 ? 0 : 1);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (row0 + 8 * t >= rows) break;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[t][e];
                sum += __shfl_xor_sync(FW_FULL, sum, 4);
                sum += __shfl_xor_sync(FW_FULL, sum, 8);
                sum += __shfl_xor_sync(FW_FULL, sum, 16);
                l[t][e] = sum;
            }
            __syncthreads();
            if (g == 0) {
                s_ml[wid][2 * c] = make_float2(mx[t][0], l[t][0]);
                s_ml[wid][2 * c + 1] = make_float2(mx[t][1], l[t][1]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < MT; i += 2)
                    *reinterpret_cast<float4 *>(s_o + (wid * 8 + 2 * c + e) * C::LDO + g * (D / 8) + 2 * i) =
                        make_float4(O[t][i][e], O[t][i][2 + e], O[t][i + 1][e], O[t][i + 1][2 + e]);
            __syncthreads();
            const int r = row0 + 8 * t + wid;  // a warp per row
            if (r < rows) {
                float M = -INFINITY, L = 0.f, acc[D / 32];
#pragma unroll
                for (int w = 0; w < AW; ++w) M = fmaxf(M, s_ml[w][wid].x);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) acc[i] = 0.f;
#pragma unroll
                for (int w = 0; w < AW; ++w) {
                    const float2 ml = s_ml[w][wid];
                    const float f = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2(ml.x - M);
                    L = fmaf(f, ml.y, L);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(f, s_o[(w * 8 + wid) * C::LDO + lane + 32 * i], acc[i]);
                }
                if (s_err) L = NAN;
                if (whole) {
                    const int i = r / a.group;
                    const int64_t out = ((int64_t)seq * a.m + i) * a.kv_heads * a.group + hk * a.group + (r - i * a.group);
                    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
                    for (int e = 0; e < D / 32; ++e)
                        a.o[out * D + lane + 32 * e] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e] * inv));
                    if (a.lse && lane == 0) a.lse[out] = L == 0.f ? -INFINITY : (M - P_UP + log2f(L)) * 0.6931471805599453f;
                } else {
                    const int64_t at = ((int64_t)tile * a.G * 2 + part) * RT + 8 * t + wid;
                    if (lane == 0) a.part_ml[at] = make_float2(M, L);
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) a.part_o[at * D + lane + 32 * e] = acc[e];
                }
            }
        }
        if (s_err && tid == 0 && a.status) a.status[h] = FW_ERR_TIMEOUT;
        u += bend - b;
        b = bend;
    }
    // copies of this warp that are still under way land before the CTA's memory goes
    for (; cphase < pphase; ++cphase) tc::mbar_wait(&full[wid][cphase % C::STAGES], (cphase / C::STAGES) & 1u, A_WAIT);
}

// The parts of a cell that spans several CTAs, joined in their order; empty cells' outputs.
// A CTA per (cell, query row): four warps take every fourth part each.
template <int D> __global__ void __launch_bounds__(128) k_cache8_join(const AttendArgs a, int RT)
{
    constexpr int E = D / 32;
    __shared__ float s_o[4][D];
    __shared__ float2 s_ml[4];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int h = blockIdx.x, r = blockIdx.y, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int64_t base;
    int n;
    fw_status st;
    const int nb = cell_blocks(a.s, h, base, n, st), quota = *a.plan, s = a.start[h];
    const int c0 = s / quota, c1 = nb > 0 ? (s + nb - 1) / quota : c0;
    if (nb > 0 && c0 == c1) return;
    float M = -INFINITY, L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    if (nb > 0)
        for (int p = c0 + wid; p <= c1; p += 4) {
            const int seg = p == c0 && s > p * quota ? 1 : 0;
            const int64_t at = ((int64_t)(r / RT) * a.G * 2 + 2 * p + seg) * RT + r % RT;
            const float2 ml = a.part_ml[at];
            const float now = fmaxf(M, ml.x);
            const float f = M == now ? 1.f : ex2(M - now), y = ml.x == now ? 1.f : ex2(ml.x - now);
            M = now;
            L = fmaf(L, f, ml.y * y);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(acc[e], f, a.part_o[at * D + lane + 32 * e] * y);
        }
    if (lane == 0) s_ml[wid] = make_float2(M, L);
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[wid][lane + 32 * e] = acc[e];
    __syncthreads();
    if (wid != 0) return;
    M = fmaxf(fmaxf(s_ml[0].x, s_ml[1].x), fmaxf(s_ml[2].x, s_ml[3].x));
    L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = s_ml[w].x == M ? 1.f : ex2(s_ml[w].x - M);
        L = fmaf(f, s_ml[w].y, L);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(f, s_o[w][lane + 32 * e], acc[e]);
    }
    const int seq = h / a.kv_heads, i = r / a.group;
    const int64_t out = ((int64_t)seq * a.m + i) * a.kv_heads * a.group + (h - seq * a.kv_heads) * a.group + (r - i * a.group);
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int e = 0; e < E; ++e)
        a.o[out * D + lane + 32 * e] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e] * inv));
    if (a.lse && lane == 0) a.lse[out] = L == 0.f ? -INFINITY : (M - P_UP + log2f(L)) * 0.6931471805599453f;
}

// Query rows of a CTA: 8 where they suffice (a row more costs the second product's and
// the statistics' work again), else 16 and as many rounds over the store as that takes.
int row_tile(const fw_cache8_query &q) { return q.group * q.m <= 8 ? 8 : 16; }

struct Plan {
    int G, RT, tiles;
    size_t start, plan, ml, o, bytes;
};
fw_status plan_of(const fw_cache8 &c, const fw_cache8_query &q, Plan &p)
{
    if (device_sms(&p.G) != FW_OK) p.G = 152;  // no device: the size query still answers
    p.RT = row_tile(q);
    p.tiles = (q.group * q.m + p.RT - 1) / p.RT;
    p.start = 0;
    p.plan = align256((size_t)c.cells * 4);
    p.ml = p.plan + 256;
    const size_t parts = (size_t)p.tiles * p.G * 2 * p.RT;
    p.o = p.ml + align256(parts * 8);
    p.bytes = p.o + align256(parts * c.d * 4);
    return FW_OK;
}

}  // namespace

size_t cache8_attend_workspace(const fw_cache8 &c, const fw_cache8_query &q)
{
    Plan p;
    return plan_of(c, q, p) == FW_OK ? p.bytes : 0;
}

fw_status cache8_attend(const fw_cache8 &c, const fw_cache8_query &q, void *o, float *lse, int32_t *status, void *ws,
                        cudaStream_t s)
{
    Plan p;
    plan_of(c, q, p);
    CUtensorMap mk, mv;
    // (a store without rows has no blocks to fetch: any valid map does)
    const uint64_t rows = std::max<int64_t>(c.rows, BR);
    if (!make_tma_2d_bytes(&mk, c.rows ? c.k : ws, rows, (uint64_t)c.d, BR) ||
        !make_tma_2d_bytes(&mv, c.rows ? c.v : ws, rows, (uint64_t)c.d, BR))
        return FW_ERR_CUDA;
    uint8_t *w = (uint8_t *)ws;
    const AttendArgs a{store(c),  q.kv_heads, q.group, q.m, (const uint16_t *)q.q, q.q_seq, q.q_tok, q.q_head,
                       q.scale * 1.4426950408889634f, (uint16_t *)o, lse, status, p.G, (int32_t *)(w + p.start),
                       (int32_t *)(w + p.plan), (float2 *)(w + p.ml), (float *)(w + p.o)};
    auto attend = [&](auto kernel, size_t smem) -> fw_status {
        FW_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        FW_LAUNCH(kernel, dim3((unsigned)p.G, (unsigned)p.tiles), AT, smem, s, mk, mv, a);
        return FW_OK;
    };
    fw_status st = FW_OK;
    FW_CACHE8_DISPATCH(c, st = p.RT == 8 ? attend(k_cache8_attend<D, FMT, 1>, Cfg<D>::SMEM)
                                         : attend(k_cache8_attend<D, FMT, 2>, Cfg<D>::SMEM));
    if (st != FW_OK) return st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)c.cells, (unsigned)(q.group * q.m));
    cfg.blockDim = dim3(128);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = c.d == 128 ? cudaLaunchKernelEx(&cfg, k_cache8_join<128>, a, p.RT)
                                     : cudaLaunchKernelEx(&cfg, k_cache8_join<64>, a, p.RT);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? FW_OK : FW_ERR_CUDA;
}

}  // namespace fw
