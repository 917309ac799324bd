// k_cache8_attend.cu -- attention over the 8-bit ragged store: with a cell's n
// rows of codes kc, vc and block scales sk, sv, query token i of m sees the rows
// j < n - m + 1 + i:
//   x_j = scale (q . kc_j) sk,  o = sum_j softmax_j(x) vc_j sv,  lse = log sum_j e^x_j.
//
// Bound: the codes' bytes, each read once from memory.  Two ways over the cells:
//   few short cells (k_cache8_attend_few): a cluster of 2 to 8 CTAs per cell, its blocks dealt out
//   to all their warps, whose states are joined through (distributed) shared memory;
//   many (k_cache8_attend): the blocks of all cells in a row are divided evenly over the
//   warps of the GPU, whatever the cells' lengths, so a warp takes the end of one cell,
//   whole cells and the start of another, and waits for no other warp; the parts of
//   cells that several warps share go to the workspace, and a second kernel, launched
//   behind the first one's tail, joins them in their order.
// Every warp fetches its blocks by TMA into a ring of its own.  64 x 8 cells of about 16,384 rows, d = 128:
// 306 us, 6.9 TB/s, the measured copy rate; 32 x 8 cells of 4,096 48 us (5.3 TB/s: the warps finish
// 14 us apart, and the joining follows them); 8 cells of 4,096 7.2 us (latency).
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
#include <type_traits>
#include <utility>

#include "fw_cache8.cuh"
#include "tc_sm100.cuh"

namespace fw {
namespace {

using namespace cache8;

constexpr int BR = FW_CACHE8_BLOCK;
constexpr int AW = 8;                   // warps of a CTA of the few-cells kernel
constexpr int AT = 32 * AW;
constexpr uint32_t A_WAIT = 1u << 22;   // polls before a wait gives up
constexpr float P_UP = 14.f;            // weights are 2^(x - max + P_UP)

struct AttendArgs {
    Store s;
    int kv_heads, group, m;
    uint32_t group_inv;  // 2^32 / group + 1 (0 for a group of 1)
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
    int G, warps;        // CTAs along the blocks, and their warps
    int cluster;         // CTAs of a cell (few cells)
    int32_t *start;      // workspace: [cells] first unit of each cell
    int32_t *plan;       // workspace: units per warp
    float2 *part_ml;     // workspace: [tiles of rows][warps][2][rows of a tile] (max, sum)
    float *part_o;       // workspace: the same with D columns
};

// r / group for a query row r: both are below 2^16, so the product's upper half is exact
__device__ __forceinline__ int token_of(const AttendArgs &a, int r) { return a.group_inv ? __umulhi(r, a.group_inv) : r; }

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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a float at this CTA's shared address p, as CTA `rank` of the cluster has it
__device__ __forceinline__ float remote(const float *p, int rank)
{
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}"
                 : "=f"(v)
                 : "r"(tc::smem_u32(p)), "r"(rank)
                 : "memory");
    return v;
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

// W warps of a CTA with rings of STAGES blocks.  Two blocks a warp keep the memory busy (128 KB an SM); with three, each
// waits longer in the queue and the GPU's warps finish further apart (64 x 8 cells of 16,384 rows, d = 128: 309 us, 329
// with three).
template <int D, int W> struct Cfg {
    static constexpr int STAGES = D == 128 ? 2 : 3;
    static constexpr int BLK = BR * D;                       // bytes of a block's codes
    static constexpr int RING = W * STAGES * 2 * BLK;
    static constexpr size_t SMEM = 1024 + RING;
};
// The few-cells kernel's: the warps' rows of 8 behind the rings.
template <int D> struct CfgFew : Cfg<D, AW> {
    static constexpr int LDO = D + 4;  // floats of a row
    static constexpr size_t SMEM = Cfg<D, AW>::SMEM + AW * 8 * LDO * 4;
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

// A warp's ring of blocks.
template <int D, int STAGES> struct Ring {
    static constexpr int BLK = BR * D;
    uint8_t *mem;
    uint64_t *full;
    uint32_t issued = 0, used = 0;
    bool ok = true;

    __device__ void fetch(const CUtensorMap *tmK, const CUtensorMap *tmV, int64_t row, int lane)
    {
        const int s = issued % STAGES;
        if (lane == 0) {
            tc::mbar_arrive_expect_tx(&full[s], 2 * BLK);
            tc::tma_load_2d(mem + s * 2 * BLK, tmK, 0, (int32_t)row, &full[s]);
            tc::tma_load_2d(mem + s * 2 * BLK + BLK, tmV, 0, (int32_t)row, &full[s]);
        }
        ++issued;
    }
    // the next block, or null where the wait gave up
    __device__ const uint8_t *next()
    {
        const int s = used % STAGES;
        if (ok) ok = tc::mbar_wait(&full[s], (used / STAGES) & 1u, A_WAIT);
        if (!ok) return nullptr;
        ++used;
        return mem + s * 2 * BLK;
    }
    // copies still under way land before the CTA's memory goes
    __device__ void drain()
    {
        for (; used < issued; ++used) tc::mbar_wait(&full[used % STAGES], (used / STAGES) & 1u, A_WAIT);
    }
};

// A warp's queries and running softmax over blocks of one cell, NT tiles of 8 query rows.
template <int D, int FMT, int NT> struct Rows {
    static constexpr int MT = D / 16;  // 16-column tiles of the output
    static constexpr int H = D / 64;   // 64-byte halves of a row
    uint32_t qf[NT][H][8];             // row g of each 8, 16 consecutive columns of each half
    float rf[NT][2];                   // logits' factor of rows 2c, 2c + 1
    float O[NT][MT][4], mx[NT][2], l[NT][2];

    // The queries' raw rows, in two steps, so that their reads are under way before a kernel's first blocks are asked
    // for: behind those (29 MB over the GPU) they took 3.5 us.
    struct Raw {
        uint4 x[NT][H][2];
    };
    __device__ __forceinline__ static void read(Raw &q, const AttendArgs &a, int seq, int hk, int row0, int lane)
    {
        const int g = lane >> 2, c = lane & 3, rows = a.group * a.m;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + 8 * t + g, i = token_of(a, r);
            const uint16_t *src = a.q + seq * a.q_seq + i * a.q_tok + (int64_t)(hk * a.group + r - i * a.group) * a.q_head;
#pragma unroll
            for (int e = 0; e < H; ++e)
#pragma unroll
                for (int f = 0; f < 2; ++f)
                    q.x[t][e][f] = r < rows ? *reinterpret_cast<const uint4 *>(src + 64 * e + 16 * c + 8 * f) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void start(const Raw &q, const AttendArgs &a, int lane)
    {
        const int c = lane & 3;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < H; ++e) top = piece_top(q.x[t][e][1], piece_top(q.x[t][e][0], top));
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
                    const uint4 x = q.x[t][e][f];
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        qf[t][e][4 * f + z] = pack_f16(__uint_as_float(w[z] << 16) * down, __uint_as_float(w[z] & 0xffff0000u) * down);
                }
            const float fac = a.scale2 * pow2f(k);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                rf[t][e] = __shfl_sync(FW_FULL, fac, (2 * c + e) * 4);
                mx[t][e] = -INFINITY;
                l[t][e] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[t][i][e] = 0.f;
        }
    }

    // One block, rows 32 blk .. of a cell of n; `read` is called once the tile has been read.
    template <typename F>
    __device__ __forceinline__ void block(const AttendArgs &a, const uint8_t *tk, float sk, float sv, int blk, int n, int row0,
                                          int lane, F read)
    {
        const int g = lane >> 2, c = lane & 3;
        const uint8_t *tv = tk + BR * D;
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
        const int j0 = blk * BR + kappa(g), all = n - a.m + 1;  // rows that every query sees
        const bool masked = blk * BR + BR > all;
        uint32_t p4[NT][4];
        bool grew = false;
        float al[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float f = rf[t][e] * sk;
#pragma unroll
                for (int i = 0; i < 4; ++i) S[t][i >> 1][2 * (i & 1) + e] *= f;
                if (masked) {
                    const int seen = all + token_of(a, row0 + 8 * t + 2 * c + e);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (j0 + 8 * i >= seen) S[t][i >> 1][2 * (i & 1) + e] = -INFINITY;
                }
                float top = fmaxf(fmaxf(S[t][0][e], S[t][0][2 + e]), fmaxf(S[t][1][e], S[t][1][2 + e]));
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
                p4[t][i] = transpose8x8(pack_f16(S[t][i >> 1][2 * (i & 1)], S[t][i >> 1][2 * (i & 1) + 1]));
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
        read();  // every lane has read the tile
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
                    mma(x, p[0][2 * f], p[0][2 * f + 1], p[1][2 * f], p[1][2 * f + 1], p4[t][0], p4[t][1]);
                    mma(x, p[2][2 * f], p[2][2 * f + 1], p[3][2 * f], p[3][2 * f + 1], p4[t][2], p4[t][3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[t][2 * w + f][e] = fmaf(sv, x[e], O[t][2 * w + f][e]);
                }
        }
    }

    // The sums over all lanes of a row.
    __device__ __forceinline__ void close()
    {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[t][e];
                sum += __shfl_xor_sync(FW_FULL, sum, 4);
                sum += __shfl_xor_sync(FW_FULL, sum, 8);
                sum += __shfl_xor_sync(FW_FULL, sum, 16);
                l[t][e] = sum;
            }
    }
};

// Index of query row r of cell (seq, hk) in the outputs.
__device__ __forceinline__ int64_t out_row(const AttendArgs &a, int seq, int hk, int r)
{
    const int i = token_of(a, r);
    return ((int64_t)seq * a.m + i) * a.kv_heads * a.group + hk * a.group + (r - i * a.group);
}
// lse of a row with running maximum mx and sum l of 2^(x - mx + P_UP)
__device__ __forceinline__ float lse_of(float mx, float l)
{
    return l == 0.f ? -INFINITY : (mx - P_UP + log2f(l)) * 0.6931471805599453f;
}

template <int D, int FMT, int NT, int W>
__global__ void __launch_bounds__(32 * W, 1) k_cache8_attend(const __grid_constant__ CUtensorMap tmK,
                                                         const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    using C = Cfg<D, W>;
    constexpr int AT = 32 * W;
    constexpr int MT = D / 16, RT = 8 * NT;  // RT: query rows of a CTA
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t full[W][C::STAGES];
    __shared__ int s_scan[W], s_h0[W], s_b0[W], s_n0[W];  // (s_*0: where each warp's range begins)
    __shared__ int64_t s_base0[W];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, c = lane & 3;
    const int cta = blockIdx.x, tile = blockIdx.y, row0 = tile * RT, rows = a.group * a.m;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane < C::STAGES) tc::mbar_init(&full[wid][lane], 1);
    tc::mbar_init_fence();

    // ---- the units (blocks) of all cells, divided evenly over the warps of all CTAs
    const int per = (a.s.cells + AT - 1) / AT;
    const int h_lo = min(tid * per, a.s.cells), h_hi = min(h_lo + per, a.s.cells);
    int mine = 0, nb_lo = 0, n_lo = 0;
    int64_t base_lo = 0;
    for (int h = h_lo; h < h_hi; ++h) {
        int64_t base;
        int n;
        fw_status st;
        const int nb = cell_blocks(a.s, h, base, n, st);
        if (h == h_lo) nb_lo = nb, n_lo = n, base_lo = base;
        mine += nb;
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
    for (int w = 0; w < W; ++w) {
        if (w < wid) before += s_scan[w];
        total += s_scan[w];
    }
    // consecutive ranges go to different CTAs; at least two blocks each, so that there is less to join
    const int quota = max((total + a.G * W - 1) / (a.G * W), 2);
    {
        int at = before;
        for (int h = h_lo; h < h_hi; ++h) {
            int64_t base = base_lo;
            int n = n_lo;
            fw_status st;
            const int nb = h == h_lo ? nb_lo : cell_blocks(a.s, h, base, n, st);
            // the warps of this CTA whose ranges begin in the cell
            for (int w = 0; w < W; ++w) {
                const int64_t u = (int64_t)(w * a.G + cta) * quota;
                if (u >= at && u < at + nb) {
                    s_h0[w] = h;
                    s_b0[w] = (int)(u - at);
                    s_n0[w] = n;
                    s_base0[w] = base;
                }
            }
            if (cta == 0 && tile == 0) a.start[h] = at;
            at += nb;
        }
        if (cta == 0 && tile == 0 && tid == 0) *a.plan = quota;
    }
    __syncthreads();
    const int gw = wid * a.G + cta;
    const int64_t first = (int64_t)gw * quota;
    if (first >= total) return;
    int u = (int)first;
    const int u1 = min(u + quota, total);

    Ring<D, C::STAGES> ring;
    ring.mem = sm + wid * C::STAGES * 2 * C::BLK;
    ring.full = full[wid];
    // the warp's producer: its next unit to fetch, by cell
    int pu = u, ph = s_h0[wid], pb = s_b0[wid], pn = s_n0[wid], pnb = (pn + BR - 1) / BR;
    int64_t pbase = s_base0[wid];
    fw_status pst;
    auto fetch = [&]() {
        if (pu >= u1) return;
        while (pb >= pnb && ph + 1 < a.s.cells) {  // (a unit is left, so a cell holds it)
            pb -= pnb;
            pnb = cell_blocks(a.s, ++ph, pbase, pn, pst);
        }
        ring.fetch(&tmK, &tmV, pbase + (int64_t)pb * BR, lane);
        ++pu;
        ++pb;
    };
    Rows<D, FMT, NT> R;
    typename Rows<D, FMT, NT>::Raw raw;
    R.read(raw, a, ph / a.kv_heads, ph % a.kv_heads, row0, lane);
#pragma unroll 1
    for (int s = 0; s < C::STAGES; ++s) fetch();

    int h = s_h0[wid], b = s_b0[wid];  // the segment: blocks of one cell
    while (u < u1) {
        int64_t base = s_base0[wid];
        int n = s_n0[wid];
        fw_status st;
        int nb = u == (int)first ? (n + BR - 1) / BR : cell_blocks(a.s, h, base, n, st);
        while (b >= nb && h + 1 < a.s.cells) {  // cells without rows, and the next cell
            b -= nb;
            nb = cell_blocks(a.s, ++h, base, n, st);
        }
        if (b >= nb) break;  // (never, unless the counts change under the call)
        const int bend = min(nb, b + (u1 - u));
        const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
        if (u != (int)first) R.read(raw, a, seq, hk, row0, lane);
        R.start(raw, a, lane);
        const float *ks = a.s.ks + base / BR, *vs = a.s.vs + base / BR;
        float sk = ks[b], sv = vs[b];
#pragma unroll 1
        for (int blk = b; blk < bend; ++blk) {
            const float k = sk, v = sv;
            if (blk + 1 < bend) sk = ks[blk + 1], sv = vs[blk + 1];
            const uint8_t *tk = ring.next();
            if (!tk) break;
            R.block(a, tk, k, v, blk, n, row0, lane, fetch);
        }
        R.close();
        const bool whole = b == 0 && bend == nb;
        const int seg = u == (int)first ? 0 : 1;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = row0 + 8 * t + 2 * c + e;
                if (r >= rows) continue;
                const float sum = ring.ok ? R.l[t][e] : NAN;
                if (whole) {
                    const int64_t out = out_row(a, seq, hk, r);
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    uint32_t w[MT];
#pragma unroll
                    for (int i = 0; i < MT; ++i) w[i] = pack_bf16(R.O[t][i][e] * inv, R.O[t][i][2 + e] * inv);
                    uint4 *dst = reinterpret_cast<uint4 *>(a.o + out * D + g * (D / 8));
#pragma unroll
                    for (int i = 0; i < MT; i += 4) dst[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                    if (a.lse && g == 0) a.lse[out] = lse_of(R.mx[t][e], sum);
                } else {
                    const int64_t at = (((int64_t)tile * a.warps + gw) * 2 + seg) * RT + 8 * t + 2 * c + e;
                    if (g == 0) a.part_ml[at] = make_float2(R.mx[t][e], sum);
                    float4 *dst = reinterpret_cast<float4 *>(a.part_o + at * D + g * (D / 8));
#pragma unroll
                    for (int i = 0; i < MT; i += 2)
                        dst[i / 2] = make_float4(R.O[t][i][e], R.O[t][i][2 + e], R.O[t][i + 1][e], R.O[t][i + 1][2 + e]);
                }
            }
        if (!ring.ok && lane == 0 && a.status) a.status[h] = FW_ERR_TIMEOUT;
        u += bend - b;
        b = bend;
    }
    ring.drain();
}

// The parts of a cell that several warps share, joined in their order; empty cells' outputs.  Each of a CTA's W warps
// takes a row, or (SPREAD) all of them one row's parts, where there are few rows and so the parts may be many:
// a CTA per row of 64 cells x 20 rows came in 8 waves of small CTAs behind the first kernel, 7 us.
template <int D, int W, bool SPREAD> __global__ void __launch_bounds__(32 * W) k_cache8_join(const AttendArgs a, int RT)
{
    constexpr int E = D / 32;
    using Vec = typename std::conditional<D == 128, float4, float2>::type;
    __shared__ float s_o[SPREAD ? W : 1][D];
    __shared__ float2 s_ml[W];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int h = blockIdx.x, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int r = SPREAD ? blockIdx.y : blockIdx.y * W + wid;
    int64_t base;
    int n;
    fw_status st;
    const int nb = cell_blocks(a.s, h, base, n, st), quota = *a.plan, s = a.start[h];
    const int w0 = s / quota, w1 = nb > 0 ? (s + nb - 1) / quota + 1 : w0;  // the cell's warps
    if (w1 == w0 + 1) return;
    if (r >= a.group * a.m) return;  // (SPREAD: no row of the grid is)
    const int64_t tile0 = (int64_t)(r / RT) * a.warps;
    auto part_at = [&](int p) {
        const int seg = p == w0 && s > p * quota ? 1 : 0;
        return ((tile0 + p) * 2 + seg) * RT + r % RT;
    };
    // this warp's parts: 32 maxima and sums at a time, then their columns
    const int all = w1 - w0, each = SPREAD ? (all + W - 1) / W : all;
    const int p0 = SPREAD ? w0 + min(wid * each, all) : w0, p1 = min(p0 + each, w1);
    float M = -INFINITY, L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int q = p0; q < p1; q += 32) {
        // (the columns of B parts are asked for before the maxima are looked at, and B at a time after that)
        constexpr int B = 64 / E;
        const int cnt = min(32, p1 - q);
        const float2 ml = lane < cnt ? a.part_ml[part_at(q + lane)] : make_float2(-INFINITY, 0.f);
        float f = 0.f;
        for (int i = 0; i < cnt; i += B) {
            Vec x[B];
#pragma unroll
            for (int u = 0; u < B; ++u) {
                x[u] = Vec{};
                if (i + u < cnt) x[u] = *reinterpret_cast<const Vec *>(a.part_o + part_at(q + i + u) * D + lane * E);
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
                for (int e = 0; e < E; ++e)  // (a part that is not there is 0, its factor 0 or 1)
                    acc[e] = fmaf(g, reinterpret_cast<const float *>(&x[u])[e], acc[e]);
            }
        }
    }
    if constexpr (SPREAD) {
        if (lane == 0) s_ml[wid] = make_float2(M, L);
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[wid][lane * E + e] = acc[e];
        __syncthreads();
        if (wid != 0) return;
        const float2 ml = lane < W ? s_ml[lane] : make_float2(-INFINITY, 0.f);
        M = warp_max(ml.x);
        const float f = ml.x == M ? 1.f : ex2(ml.x - M);
        L = warp_sum(f * ml.y);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float g = __shfl_sync(FW_FULL, f, w);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(g, s_o[w][lane * E + e], acc[e]);
        }
    }
    const int seq = h / a.kv_heads;
    const int64_t out = out_row(a, seq, h - seq * a.kv_heads, r);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    uint32_t *dst = reinterpret_cast<uint32_t *>(a.o + out * D + lane * E);
#pragma unroll
    for (int e = 0; e < E; e += 2) dst[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
    if (a.lse && lane == 0) a.lse[out] = lse_of(M, L);
}

// Eight states of a row joined: their (maximum, sum) and E of a lane's columns.
template <int E, typename FM, typename FO>
__device__ __forceinline__ void join8(FM ml_of, FO o_of, float &M, float &L, float (&acc)[E])
{
    float2 ml[8];
    M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) ml[w] = ml_of(w), M = fmaxf(M, ml[w].x);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const float f = ml[w].x == M ? 1.f : ex2(ml[w].x - M);
        L = fmaf(f, ml[w].y, L);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(f, o_of(w, e), acc[e]);
    }
}

// A cluster of up to FEW CTAs per cell and tile of rows, its blocks dealt out to their warps one by one.
constexpr int FEW = 8;
template <int D, int FMT, int NT>
__global__ void __launch_bounds__(AT, 1)
    k_cache8_attend_few(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    using C = CfgFew<D>;
    constexpr int MT = D / 16, RT = 8 * NT, E = D / 32;
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    float *s_o = reinterpret_cast<float *>(sm + C::RING);  // [AW][8][LDO]
    __shared__ __align__(8) uint64_t full[AW][C::STAGES];
    __shared__ float2 s_ml[AW][8];
    __shared__ float2 s_pml[8];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, c = lane & 3;
    const int h = blockIdx.x / a.cluster, rank = blockIdx.x % a.cluster, row0 = blockIdx.y * RT, rows = a.group * a.m;
    if (lane < C::STAGES) tc::mbar_init(&full[wid][lane], 1);
    tc::mbar_init_fence();
    __syncwarp();
    int64_t base;
    int n;
    fw_status st;
    const int nb = cell_blocks(a.s, h, base, n, st);
    if (rank == 0 && blockIdx.y == 0 && tid == 0 && a.status) a.status[h] = st;
    Ring<D, C::STAGES> ring;
    ring.mem = sm + wid * C::STAGES * 2 * C::BLK;
    ring.full = full[wid];
    int pb = rank + a.cluster * wid;  // (the first blocks go to different CTAs)
    auto fetch = [&]() {
        if (pb >= nb) return;
        ring.fetch(&tmK, &tmV, base + (int64_t)pb * BR, lane);
        pb += a.cluster * AW;
    };
    const int seq = h / a.kv_heads, hk = h - seq * a.kv_heads;
    Rows<D, FMT, NT> R;
    typename Rows<D, FMT, NT>::Raw raw;
    R.read(raw, a, seq, hk, row0, lane);
#pragma unroll 1
    for (int s = 0; s < C::STAGES; ++s) fetch();
    R.start(raw, a, lane);
    const float *ks = a.s.ks + base / BR, *vs = a.s.vs + base / BR;
#pragma unroll 1
    for (int blk = rank + a.cluster * wid; blk < nb; blk += a.cluster * AW) {
        const float sk = ks[blk], sv = vs[blk];
        const uint8_t *tk = ring.next();
        if (!tk) break;
        R.block(a, tk, sk, sv, blk, n, row0, lane, fetch);
    }
    R.close();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (row0 + 8 * t >= rows) break;
        // ---- the warps' rows joined in the CTA, a warp per row
        if (t > 0) cluster_sync();  // (the rows before have been read)
        if (g == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) s_ml[wid][2 * c + e] = make_float2(R.mx[t][e], ring.ok ? R.l[t][e] : NAN);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < MT; i += 2)
                *reinterpret_cast<float4 *>(s_o + (wid * 8 + 2 * c + e) * C::LDO + g * (D / 8) + 2 * i) =
                    make_float4(R.O[t][i][e], R.O[t][i][2 + e], R.O[t][i + 1][e], R.O[t][i + 1][2 + e]);
        __syncthreads();
        float M, L, acc[E];
        join8<E>([&](int w) { return s_ml[w][wid]; }, [&](int w, int e) { return s_o[(w * 8 + wid) * C::LDO + lane + 32 * e]; },
                 M, L, acc);
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[wid * C::LDO + lane + 32 * e] = acc[e];  // (its row in the first warp's place)
        if (lane == 0) s_pml[wid] = make_float2(M, L);
        cluster_sync();
        // ---- and over the cluster's CTAs: rows dealt out to them and their warps
        const int r8 = rank + a.cluster * wid, r = row0 + 8 * t + r8;
        if (r8 < 8 && r < rows) {
            join8<E>([&](int w) { return w < a.cluster ? make_float2(remote(&s_pml[r8].x, w), remote(&s_pml[r8].y, w))
                                                      : make_float2(-INFINITY, 0.f); },
                     [&](int w, int e) { return w < a.cluster ? remote(&s_o[r8 * C::LDO + lane + 32 * e], w) : 0.f; }, M, L, acc);
            const int64_t out = out_row(a, seq, hk, r);
            const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
            for (int e = 0; e < E; ++e)
                a.o[out * D + lane + 32 * e] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e] * inv));
            if (a.lse && lane == 0) a.lse[out] = lse_of(M, L);
        }
    }
    ring.drain();
    if (!ring.ok && lane == 0 && a.status) a.status[h] = FW_ERR_TIMEOUT;
    cluster_sync();  // no CTA leaves while another reads its rows
}
static_assert(FEW == 8 && AW == 8, "a warp per row of 8, eight states to join");

// Query rows of a CTA: as few tiles of 8 as hold them, as far as registers go (a second round over
// the store costs its fetches and products again: 64 cells of 4,096 rows, d = 128, 4 query rows 20 us, 20 in two rounds 34,
// 40 in three 48, 128 in eight 105).
int row_tile(const fw_cache8 &c, const fw_cache8_query &q)
{
    const int rows = q.group * q.m;
    return rows <= 8 ? 8 : rows <= 16 || c.d == 128 ? 16 : rows <= 24 ? 24 : 32;
}

// Warps of a CTA of the many-cells kernel: 16 where a warp's registers allow it (d = 64, 8 rows: 32 x 8 cells of 4,096 rows
// 31 us, 36 with 8), else 8 (d = 64, 24 rows: 64 cells of 1,537 18.4 us, 19.7 with 12, which spill).
constexpr int warps_of(int d, int RT) { return d == 64 && RT == 8 ? 16 : 8; }

// CTAs of a cell where the cells are few and hold little at most, so that a cluster each is faster, else 0.  (Per-layer
// calls, d = 128, clusters against ranges: 8 cells of 4,096 rows 7.2 us against 10.7; 16 cells in 8 each, whose clusters of
// whole SMs do not all find them at once, 12.9 against 11.9, of 1,000 rows in 4 each 7.1 against 10.3, of 3,300 13.6 against
// 11.6; 48 cells of 500 in 2 each 7.4 against 13.2, of 2,000 16.8 against 15.4: the longest cell decides.)  What the host
// knows of the lengths is the store's rows over the call's cells: the mean where the store holds nothing else, more where
// the cells are a part of a larger one.  A layer of a large store therefore takes ranges: 8 cells of 4,096 rows of 256,
// 10.6 us (7.9 in a store of their own; codes from memory in both).
int cluster_of(const fw_cache8 &c, int tiles)
{
    struct Rule {
        int ctas;
        int64_t cells, rows;
    };
    for (const Rule &r : {Rule{8, 14, 8192}, Rule{4, 36, 2560}, Rule{2, 72, 1280}})
        if ((int64_t)c.cells * tiles <= r.cells && c.rows <= r.rows * c.cells) return r.ctas;
    return 0;
}

struct Plan {
    int few;  // CTAs of a cell's cluster, or 0
    int G, W, RT, tiles;
    size_t start, plan, ml, o, bytes;
};
void plan_of(const fw_cache8 &c, const fw_cache8_query &q, Plan &p)
{
    int sms = 0;
    if (device_sms(&sms) != FW_OK) sms = 152;  // no device: the size query still answers
    p.RT = row_tile(c, q);
    p.tiles = (q.group * q.m + p.RT - 1) / p.RT;
    p.few = cluster_of(c, p.tiles);
    p.G = std::max(1, sms / p.tiles);  // one wave
    p.W = warps_of(c.d, p.RT);
    p.start = p.plan = p.ml = p.o = p.bytes = 0;
    if (p.few) return;
    p.plan = align256((size_t)c.cells * 4);
    p.ml = p.plan + 256;
    const size_t parts = (size_t)p.tiles * p.G * p.W * 2 * p.RT;
    p.o = p.ml + align256(parts * 8);
    p.bytes = p.o + align256(parts * c.d * 4);
}

template <typename K>
fw_status launch(K kernel, int grid, int tiles, int cluster, int threads, size_t smem, const CUtensorMap &mk,
                 const CUtensorMap &mv, const AttendArgs &a, std::atomic<uint64_t> &done, cudaStream_t s)
{
    const fw_status st = big_smem((const void *)kernel, smem, done);
    if (st != FW_OK) return st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, (unsigned)tiles);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = cluster ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, mk, mv, a);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? FW_OK : FW_ERR_CUDA;
}
template <int D, int FMT, int NT>
fw_status launch_tiles(const Plan &p, int cells, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a, cudaStream_t s)
{
    constexpr int W = warps_of(D, 8 * NT);
    static std::atomic<uint64_t> few{0}, many{0};
    return p.few ? launch(k_cache8_attend_few<D, FMT, NT>, cells * p.few, p.tiles, p.few, AT, CfgFew<D>::SMEM, mk, mv, a, few, s)
                 : launch(k_cache8_attend<D, FMT, NT, W>, p.G, p.tiles, 0, 32 * W, Cfg<D, W>::SMEM, mk, mv, a, many, s);
}
template <int D, int FMT>
fw_status attend(const Plan &p, int cells, const CUtensorMap &mk, const CUtensorMap &mv, const AttendArgs &a, cudaStream_t s)
{
    if (p.RT == 8) return launch_tiles<D, FMT, 1>(p, cells, mk, mv, a, s);
    if (p.RT == 16) return launch_tiles<D, FMT, 2>(p, cells, mk, mv, a, s);
    if constexpr (D == 64) {  // (with d = 128 two tiles of 8 rows at most)
        if (p.RT == 24) return launch_tiles<D, FMT, 3>(p, cells, mk, mv, a, s);
        return launch_tiles<D, FMT, 4>(p, cells, mk, mv, a, s);
    }
    return FW_ERR_UNSUPPORTED;
}

}  // namespace

size_t cache8_attend_workspace(const fw_cache8 &c, const fw_cache8_query &q)
{
    Plan p;
    plan_of(c, q, p);
    return p.bytes;
}

fw_status cache8_attend(const fw_cache8 &c, const fw_cache8_query &q, void *o, float *lse, int32_t *status, void *ws,
                        cudaStream_t s)
{
    Plan p;
    plan_of(c, q, p);
    CUtensorMap mk, mv;
    // (a store without rows has no blocks to fetch: any valid map does)
    const uint64_t rows = std::max<int64_t>(c.rows, BR);
    if (!make_tma_2d_bytes(&mk, c.rows ? c.k : o, rows, (uint64_t)c.d, BR) ||
        !make_tma_2d_bytes(&mv, c.rows ? c.v : o, rows, (uint64_t)c.d, BR))
        return FW_ERR_CUDA;
    uint8_t *w = (uint8_t *)ws;
    const uint32_t inv = q.group > 1 ? (uint32_t)(((uint64_t)1 << 32) / q.group + 1) : 0;
    const AttendArgs a{store(c), q.kv_heads, q.group, q.m, inv, (const uint16_t *)q.q, q.q_seq, q.q_tok, q.q_head,
                       q.scale * 1.4426950408889634f, (uint16_t *)o, lse, status, p.G, p.G * p.W, p.few, (int32_t *)(w + p.start),
                       (int32_t *)(w + p.plan), (float2 *)(w + p.ml), (float *)(w + p.o)};
    fw_status st = FW_OK;
    FW_CACHE8_DISPATCH(c, st = attend<D, FMT>(p, c.cells, mk, mv, a, s));
    if (st != FW_OK || p.few) return st;
    const int qrows = q.group * q.m;
    // rows so few that they would not keep the GPU's warps busy: every row's parts over a CTA
    const bool spread = (int64_t)c.cells * qrows <= 4 * p.G * p.tiles;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)c.cells, (unsigned)(spread ? qrows : (qrows + 7) / 8));
    cfg.blockDim = dim3(spread ? 512 : 256);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const auto join = c.d == 128 ? (spread ? k_cache8_join<128, 16, true> : k_cache8_join<128, 8, false>)
                                 : (spread ? k_cache8_join<64, 16, true> : k_cache8_join<64, 8, false>);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, join, a, p.RT);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? FW_OK : FW_ERR_CUDA;
}

}  // namespace fw
