// k_prompt.cu -- causal attention over packed prompts with grouped heads: query
// token i of a sequence with lq query and lk key rows sees its keys
// j <= lk - lq + i:
//   x_j = scale q_i . k_j,  o_i = sum_j softmax_j(x) v_j,  lse_i = log sum_j e^x_j.
//
// Bound: the tensor cores (two products of 128 x 128 x d per block of 128 keys): 16,384 tokens x 32 heads
// (8 KV heads), d = 128: 1.33 to 1.44 ms from box to box, 1.53 to 1.65 PFLOP/s, 89 to 96 % of what the card sustains in
// bf16 products under its power limit.  With d = 64 the exponentials and the hand-overs between the warps weigh twice as much: 8,192 tokens x 32 heads
// 291 us, 0.94 PFLOP/s.  The weights are rounded to bf16 for the second product, which wants both its operands of one
// type; sums and statistics are of the unrounded ones.
// The query heads of a KV head are rows of the same product, so a tile of 128 rows
// is floor(128 / group) tokens with all their heads, and a CTA holds one tile or two of
// consecutive tokens against one stream of keys and values (TMA, 128-byte swizzle,
// a ring of tiles).  On tcgen05, S = Q K^T goes to TMEM; the tile's four softmax
// warps, a thread per row, read it, write the weights over it in bf16, and O += P V
// takes them from there: while one tile's rows are in the softmax the other tile's
// products (another CTA's, where a CTA holds one) run.  A weight is 2^(x - ref): ref is the row's maximum as of the last
// time that it had grown by more than 2^8, so the rescaling of O in TMEM, which the
// softmax threads do themselves, is rare; sum and output are of the same ref, so the
// quotient is exact.  Behind the softmax's warps one issues the copies, one per tile its
// products (the first owns the TMEM), and one looks over the values of blocks that some row does not see in full:
// a weight of 0 does not make 0 of a NaN or an infinity, so it puts 0 in their place,
// and the rows that do see them add them when they are written.
//
// Slots are the tokens of a CTA's tiles: sequence i's are numbered from
// floor(cu_q[i] / slot) + i on, which leaves room for all of them without a prefix
// sum; a CTA finds its sequence by a search over cu_q.  Where there are few slots, a cluster of CTAs takes the
// blocks of one, and its rows' parts are joined through distributed shared memory.  Slots are taken from the last
// to the first: a sequence's last rows, which see the most keys, come first (of packed sequences the last one does, however
// short it is).
#include <cuda_bf16.h>

#include "fw_internal.h"
#include "tc_sm100.cuh"

namespace fw {
namespace {

constexpr int PK = 128;                  // keys of a block
// blocks that some row of a slot does not see in full: the first and the last row's ends are
// at most 255 keys apart
constexpr int PG = 3;
constexpr int MAX_PARTS = 8;             // CTAs of a cluster
constexpr int SPLIT = 12, MIN_PART = 4;  // blocks of keys a slot is split from, and of a part at least
constexpr uint32_t P_WAIT = 1u << 20;    // polls before a wait gives up (seconds)
constexpr float GROW = 8.f;              // octaves a row's maximum may be above its reference

struct PromptArgs {
    const int32_t *cu_q, *cu_k;
    int64_t total_q, total_k;
    int num_seqs, q_heads, kv_heads, group, slots;
    int TT, parts;  // tokens of a tile; CTAs (of a cluster) that a slot's keys are split over
    const uint16_t *v;
    int64_t v_row, v_head;
    float scale2;  // scale * log2(e)
    uint16_t *o;
    float *lse;
    int32_t *status;
};

template <int D, int TILES> struct PCfg {
    static_assert(D == 128 || TILES == 1, "two tiles a CTA: d = 128 only");
    static constexpr int NB = D / 64;              // 128-byte boxes across d
    static constexpr int QT = 128 * D * 2;         // bytes of a tile of queries
    static constexpr int KT = PK * D * 2;          // bytes of a tile of keys or values
    static constexpr int STAGES = 5;
    static constexpr size_t SMEM = 1024 + TILES * QT + (size_t)STAGES * KT;
    // Parts of a block of scores: with two, the next part's product runs under the softmax of this one (d = 128,
    // 16,384 tokens x 32 heads: 1.46 ms in one part, 1.37 in two).
    static constexpr int NS = 2;
    static constexpr int SK = PK / NS;             // keys of a part
    static constexpr uint32_t COLS = 256 * TILES;  // TMEM columns
    static constexpr uint32_t O_COL = PK * TILES;  // S of the tiles first, O behind them
    // the softmax's warps, then those of the copies, the products, the guard, and of the other tile's products
    static constexpr int W_COPY = 4 * TILES, W_MMA = W_COPY + 1, W_GUARD = W_COPY + 2, W_MMA1 = W_COPY + 3;
    static constexpr int THREADS = 32 * (W_COPY + 4);
    static constexpr int CTAS = D == 64 ? 2 : 1;   // per SM
};

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
__device__ __forceinline__ void tma_load_3d(void *dst, const void *tmap, int x, int y, int z, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(tc::smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(bar))
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_bf16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, bool acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
                 "r"(a), "l"(bdesc), "r"(idesc), "r"((uint32_t)acc)
                 : "memory");
}
// 64 consecutive fp32 columns of this warp's 32 TMEM lanes, waited on in the same statement
__device__ __forceinline__ void ld_scores(uint32_t taddr, float (&v)[64])
{
    uint32_t r[64];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, "
        "%34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, "
        "%54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 w, x, y;\n\t"
        "mov.b64 {%0, %1}, w;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the floats at this CTA's shared address p (aligned to their size), as CTA `rank` of the cluster has them
__device__ __forceinline__ void remote(const float *p, int rank, float (&v)[2])
{
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %2, %3;\n\tld.shared::cluster.v2.f32 {%0, %1}, [a];\n\t}"
                 : "=f"(v[0]), "=f"(v[1])
                 : "r"(tc::smem_u32(p)), "r"(rank)
                 : "memory");
}
__device__ __forceinline__ void remote(const float *p, int rank, float (&v)[4])
{
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                 : "r"(tc::smem_u32(p)), "r"(rank)
                 : "memory");
}
// true for one lane of a warp that is there as a whole
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// each lane waits for a phase of a barrier of its own, the warp for all of them
__device__ __forceinline__ bool wait_lanes(uint64_t *bar, uint32_t parity, uint32_t limit)
{
    bool done = false;
    for (uint32_t it = 0; it < limit; ++it) {
        done = done || tc::mbar_wait(bar, parity, 1);
        if (__all_sync(FW_FULL, done)) return true;
    }
    return false;
}

// a warp's stores to TMEM are complete and known to the products' warp
__device__ __forceinline__ void hand_over(uint64_t *bar, int lane)
{
    wait_st();
    tc::fence_before_sync();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar);
}

// sequence bounds within their ranges
__device__ __forceinline__ bool seq_ok(const PromptArgs &a, int s)
{
    const int q0 = a.cu_q[s], q1 = a.cu_q[s + 1], k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
    return q0 >= 0 && q1 >= q0 && q1 <= a.total_q && k0 >= 0 && k1 >= k0 && k1 <= a.total_k;
}

// The sequences' statuses where there are no query rows, and so nothing else to do.
__global__ void __launch_bounds__(256) k_prompt_status(const PromptArgs a)
{
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s < a.num_seqs) a.status[s] = seq_ok(a, s) ? FW_OK : FW_ERR_INVALID_ARG;
}

template <int D, int TILES>
__global__ void __launch_bounds__(PCfg<D, TILES>::THREADS, PCfg<D, TILES>::CTAS)
    k_prompt(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
             const __grid_constant__ CUtensorMap tmV, const PromptArgs a)
{
    using C = PCfg<D, TILES>;
    constexpr int PT = C::THREADS;
    extern __shared__ uint8_t smraw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~(uintptr_t)1023);
    uint8_t *sQ = sm, *sKV = sm + TILES * C::QT;
    __shared__ __align__(8) uint64_t full[C::STAGES], empty[C::STAGES], q_full;
    __shared__ __align__(8) uint64_t s_full[2][C::NS], p_full[2][C::NS], o_done[2], drained[2], v_in[PG], v_ok[PG];
    __shared__ uint32_t s_taddr;
    __shared__ int s_seq[5], s_err, s_odd;  // (s_seq: the sequence, its query and key rows)

    // (by a shuffle, so that the compiler knows the warp's role for the same in all lanes)
    const int tid = threadIdx.x, lane = tid & 31, wid = __shfl_sync(FW_FULL, tid >> 5, 0);
    const bool split = TILES == 1 && a.parts > 1;  // (a CTA of two tiles has all their keys)
    const int part = split ? blockIdx.x % a.parts : 0, item = split ? blockIdx.x / a.parts : blockIdx.x;
    const int slot = a.slots - 1 - item / a.kv_heads, hk = item % a.kv_heads;
    const int TT = a.TT, ST = TILES * TT;  // tokens of a tile and of a slot

    if (blockIdx.x == 0 && a.status)  // (before any wait can have given up)
        for (int s = tid; s < a.num_seqs; s += PT) a.status[s] = seq_ok(a, s) ? FW_OK : FW_ERR_INVALID_ARG;
    if (wid == 0) {
        // the last sequence whose slots start at or before this one: 32 probes at a time
        int lo = 0, hi = a.num_seqs;
        bool any = true;
        do {
            const int step = (hi - lo + 31) / 32, i = lo + lane * step;
            const unsigned hit = __ballot_sync(FW_FULL, i < hi && a.cu_q[min(i, hi - 1)] / ST + i <= slot);
            if (hit == 0) {
                any = false;
                break;
            }
            lo += (__popc(hit) - 1) * step;
            hi = min(lo + step, hi);
        } while (hi - lo > 1);
        if (lane < 4) s_seq[1 + lane] = (lane < 2 ? a.cu_q : a.cu_k)[lo + (lane & 1)];
        if (lane == 0) s_seq[0] = any ? lo : -1;
    } else if (wid == C::W_COPY) {
        if (lane < C::STAGES) {
            tc::mbar_init(&full[lane], 1);
            tc::mbar_init(&empty[lane], 2);
        } else if (lane < C::STAGES + PG) {
            tc::mbar_init(&v_in[lane - C::STAGES], 1);
            tc::mbar_init(&v_ok[lane - C::STAGES], 1);
        } else if (lane < C::STAGES + PG + 2) {
            const int t = lane - C::STAGES - PG;
            for (int u = 0; u < C::NS; ++u) {
                tc::mbar_init(&s_full[t][u], 1);
                tc::mbar_init(&p_full[t][u], 4);
            }
            tc::mbar_init(&o_done[t], 1);
            tc::mbar_init(&drained[t], 1);
        } else if (lane == 31) {
            tc::mbar_init(&q_full, 1);
            s_err = 0;
            s_odd = 0;
        }
        tc::mbar_init_fence();
    } else if (wid == C::W_MMA) {
        tc::tmem_alloc(&s_taddr, C::COLS);
    } else if (wid == C::W_GUARD && lane == 0) {
        tc::tma_prefetch_desc(&tmQ);
        tc::tma_prefetch_desc(&tmK);
        tc::tma_prefetch_desc(&tmV);
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t taddr = __shfl_sync(FW_FULL, s_taddr, 0);
    const int seq = s_seq[0], q0 = s_seq[1], q1 = s_seq[2], k0 = s_seq[3], k1 = s_seq[4];
    const bool valid = seq >= 0 && q0 >= 0 && q1 >= q0 && q1 <= a.total_q && k0 >= 0 && k1 >= k0 && k1 <= a.total_k;
    const int lq = valid ? q1 - q0 : 0, lk = valid ? k1 - k0 : 0;
    const int t0 = (slot - (q0 / ST + seq)) * ST;  // the slot's first token in the sequence
    if (!valid || t0 < 0 || t0 >= lq) {  // (a sequence out of range, or a slot behind its last token)
        if (wid == C::W_MMA) tc::tmem_dealloc(taddr, C::COLS);
        return;
    }
    const int tiles = TILES == 2 && t0 + TT < lq ? 2 : 1;
    // keys that the first token sees, and blocks of keys that each tile's last one does
    const int seen0 = max(0, lk - lq + t0 + 1);
    int nb[2];
    nb[0] = (max(0, lk - lq + min(t0 + TT, lq)) + PK - 1) / PK;
    nb[1] = TILES == 2 && tiles == 2 ? (max(0, lk - lq + min(t0 + ST, lq)) + PK - 1) / PK : 0;
    int J = max(nb[0], nb[1]), jm = seen0 / PK;  // blocks from jm on are not seen in full by every row
    int j0 = 0;                                  // this CTA's part: blocks j0 .. j0 + J, counted from j0 below
    if (split) {
        j0 = J * part / a.parts;
        J = nb[0] = J * (part + 1) / a.parts - j0;
        jm = min(max(jm - j0, 0), J);
    }
    const int kb = k0 + j0 * PK;  // the part's first key row

    // Copy i of the ring (K of block 0, V of block 0, K of block 1, ...) arrives on its stage's barrier;
    // the values that the guard looks over on one of their own, which the guard can wait for without
    // following the stage's phases (no stage of theirs is used again: at most five copies come behind the first).
    static_assert(C::STAGES >= 2 * PG - 1, "stages of guarded values");
    auto arrival = [&](int i) { return (i & 1) && (i >> 1) >= jm ? &v_in[min((i >> 1) - jm, PG - 1)] : &full[i % C::STAGES]; };
    auto arrival_phase = [&](int i) { return (i & 1) && (i >> 1) >= jm ? 0u : (uint32_t)(i / C::STAGES) & 1u; };

    if (wid == C::W_COPY) {
        // ------------------------------------------------------------ copies
        if (lane == 0 && J > 0) {
            const uint32_t qbytes = (uint32_t)(128 * a.group * TT);  // (one box: 64 columns of a tile's rows)
            tc::mbar_arrive_expect_tx(&q_full, qbytes * C::NB * tiles);
            for (int t = 0; t < tiles; ++t)
                for (int h = 0; h < C::NB; ++h)
                    tma_load_3d(sQ + t * C::QT + h * (128 * 128), &tmQ, 64 * h, hk * a.group, q0 + t0 + t * TT, &q_full);
            int issued = 0;
            bool ok = true;
            for (int i = 0; i < 2 * J; ++i) {
                const int s = i % C::STAGES;
                if (i >= C::STAGES && !tc::mbar_wait(&empty[s], (uint32_t)(i / C::STAGES - 1) & 1u, P_WAIT)) {
                    ok = false;
                    break;
                }
                uint64_t *bar = arrival(i);
                tc::mbar_arrive_expect_tx(bar, C::KT);
                for (int h = 0; h < C::NB; ++h)
                    tma_load_3d(sKV + s * C::KT + h * (PK * 128), (i & 1) ? &tmV : &tmK, 64 * h, hk, kb + (i >> 1) * PK, bar);
                ++issued;
            }
            if (!ok) atomicOr(&s_err, 1);
            // every copy has landed before the CTA's memory goes
            for (int i = max(0, issued - C::STAGES); i < issued; ++i)
                if (!tc::mbar_wait(arrival(i), arrival_phase(i), P_WAIT)) atomicOr(&s_err, 1);
            if (!tc::mbar_wait(&q_full, 0, P_WAIT)) atomicOr(&s_err, 1);
        }
        __syncwarp();
    } else if (wid == C::W_MMA || (TILES == 2 && wid == C::W_MMA1)) {
        // ---------------------------------------------------------- products
        // A warp per tile: what issuing costs (waits, commits) hides behind the other tile's products.  The
        // whole warp waits and an elected lane issues: with the waits inside the one lane's branch the
        // operands are not kept in uniform registers, and an instruction took 100 clocks to issue.
        const int t = wid == C::W_MMA1;
        if (t < tiles && J > 0) {
            constexpr uint32_t id_s = tc::idesc_bf16_f32(128, C::SK, false, false);
            constexpr uint32_t id_o = tc::idesc_bf16_f32(128, D, false, true);
            const uint64_t qd = tc::sdesc_sw128(tc::smem_u32(sQ) + t * C::QT, 16, 1024);
            const uint64_t kd = tc::sdesc_sw128(tc::smem_u32(sKV), 16, 1024);
            const uint64_t vd = tc::sdesc_sw128(tc::smem_u32(sKV), PK * 128, 1024);
            const uint32_t tS = taddr + t * PK, tO = taddr + C::O_COL + t * D;
            const int n = nb[t];
            bool ok = tc::mbar_wait(&q_full, 0, P_WAIT);
            int st = 0;         // stage of the next copy of the ring
            uint32_t ph = 0;    // and its phase
            // the barrier and parity that the next copy arrives with, and its stage
            auto next_copy = [&](bool guarded, int j, uint64_t *&bar, uint32_t &parity) {
                bar = guarded ? &v_ok[min(j - jm, PG - 1)] : &full[st];
                parity = guarded ? 0u : ph;
                const int s = st;
                if (++st == C::STAGES) st = 0, ph ^= 1u;
                return s;
            };
            uint64_t *bar;
            uint32_t parity;
            auto free_stage = [&](int s) {  // once the products so far have read it; a tile alone arrives for both
                tc::commit(&empty[s]);
                if (tiles == 1) tc::commit(&empty[s]);
            };
            auto qk = [&](int s, int u) {  // a part of S = Q K^T
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = (ks >> 2) * (128 * 128) + (ks & 3) * 32;
                    tc::mma_bf16(tS + u * C::SK, qd + (off >> 4), kd + ((s * C::KT + u * (C::SK * 128) + off) >> 4), id_s,
                                 ks > 0);
                }
                tc::commit(&s_full[t][u]);
                if (u == C::NS - 1) free_stage(s);
            };
            const int s0 = next_copy(false, 0, bar, parity);
            ok = __all_sync(FW_FULL, ok && tc::mbar_wait(bar, parity, P_WAIT));
            if (ok && n > 0) {
                tc::fence_after_sync();
                if (elect_one())
                    for (int u = 0; u < C::NS; ++u) qk(s0, u);
                __syncwarp();
            }
            for (int j = 0; ok && j < n; ++j) {
                // The weights, V of this block and K of the next are waited for together, a lane each: a wait takes
                // 200 clocks even where nothing is left to wait for, in a queue that the softmax's exponentials fill.
                uint64_t *pb = &p_full[t][0];
                uint32_t pp = (uint32_t)j & 1u;
                const int sv = next_copy(j >= jm, j, bar, parity);
                if (lane == 1) pb = bar, pp = parity;
                if (lane == 2 && j >= jm) pb = &v_in[min(j - jm, PG - 1)], pp = 0u;
                int sk = 0;
                if (j + 1 < n) {
                    sk = next_copy(false, 0, bar, parity);
                    if (lane == 3) pb = bar, pp = parity;
                }
#pragma unroll
                for (int u = 0; u < C::NS; ++u) {
                    ok = wait_lanes(u == 0 ? pb : &p_full[t][u], u == 0 ? pp : (uint32_t)j & 1u, P_WAIT);
                    if (!ok) break;
                    tc::fence_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < C::SK / 16; ++ks)  // O += P V
                            mma_bf16_ts(tO, tS + u * C::SK + ks * 8,
                                        vd + ((sv * C::KT + (u * (C::SK / 16) + ks) * 2048) >> 4), id_o, j > 0 || u > 0 || ks > 0);
                        tc::commit(&o_done[t]);
                        if (u == C::NS - 1) free_stage(sv);
                        if (j + 1 < n) qk(sk, u);
                    }
                    __syncwarp();
                }
            }
            // The products have completed before O is read and the TMEM freed.  (A barrier of its own: o_done
            // may be one or two phases behind here, and its parity does not tell which.)
            if (elect_one()) tc::commit(&drained[t]);
            __syncwarp();
            // blocks that only the other tile's rows see: their stages are free as far as this tile goes
            if (n == 0 && ok && lane == 0) tc::mbar_arrive(&empty[s0]);
            for (int i = max(2 * n, 1); ok && i < 2 * J; ++i) {
                const int s = next_copy((i & 1) && (i >> 1) >= jm, i >> 1, bar, parity);
                ok = tc::mbar_wait(bar, parity, P_WAIT);
                if (ok && lane == 0) tc::mbar_arrive(&empty[s]);
            }
            if (!__all_sync(FW_FULL, ok)) atomicOr(&s_err, 1);
            if (!tc::mbar_wait(&drained[t], 0, P_WAIT)) atomicOr(&s_err, 1);
        }
        __syncwarp();
    } else if (wid == C::W_GUARD) {
        // ------------------------------------------------------------- guard
        bool ok = true;
        for (int j = jm; ok && j < J; ++j) {
            const int s = (2 * j + 1) % C::STAGES;
            ok = tc::mbar_wait(&v_in[min(j - jm, PG - 1)], 0, P_WAIT);
            if (!ok) break;
            uint4 *v = reinterpret_cast<uint4 *>(sKV + s * C::KT) + lane;
            bool odd = false;
#pragma unroll 1
            for (int p = 0; p < C::KT / 512; p += 8) {
                uint4 x[8];
                uint32_t top = 0;  // the largest magnitudes of the even and the odd columns
#pragma unroll
                for (int z = 0; z < 8; ++z) x[z] = v[32 * (p + z)];
#pragma unroll
                for (int z = 0; z < 8; ++z)
                    top = __vmaxu2(__vmaxu2(__vmaxu2(top, x[z].x & 0x7fff7fffu), __vmaxu2(x[z].y & 0x7fff7fffu, x[z].z & 0x7fff7fffu)),
                                   x[z].w & 0x7fff7fffu);
                if (max(top & 0xffffu, top >> 16) >= 0x7f80u) {
                    odd = true;
                    for (int z = 0; z < 8; ++z) {
                        uint32_t *w = reinterpret_cast<uint32_t *>(v + 32 * (p + z));
                        for (int e = 0; e < 4; ++e)
                            w[e] = ((w[e] & 0x7f80u) == 0x7f80u ? 0u : w[e] & 0xffffu) |
                                   ((w[e] & 0x7f800000u) == 0x7f800000u ? 0u : w[e] & 0xffff0000u);
                    }
                }
            }
            if (__any_sync(FW_FULL, odd)) {
                tc::fence_async_smem();
                s_odd = 1;
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&v_ok[min(j - jm, PG - 1)]);
        }
        if (!ok && lane == 0) atomicOr(&s_err, 1);
    } else if (wid < 4 * TILES) {
        // ----------------------------------------------------------- softmax
        const int t = wid >> 2, r = tid & 127;
        if (t < tiles) {
            const int tok = min(t0 + t * TT + r / a.group, lq - 1);
            const bool live = r < TT * a.group && t0 + t * TT + r / a.group < lq;
            const int seen = min(max(0, lk - lq + tok + 1 - j0 * PK), J * PK), n = nb[t];
            const uint32_t lanes = (uint32_t)((wid & 3) * 32) << 16;
            const uint32_t sS = taddr + lanes + t * PK, sO = taddr + lanes + C::O_COL + t * D;
            const float c2 = a.scale2;
            float ref = -INFINITY, l = 0.f;
            bool ok = true;
            for (int i = 0; i < n * C::NS; ++i) {  // part i: keys i SK ..
                const int u = i % C::NS;
                const uint32_t sP = sS + u * C::SK;
                if (ok) ok = tc::mbar_wait(&s_full[t][u], (uint32_t)(i / C::NS) & 1u, P_WAIT);
                if (!__all_sync(FW_FULL, ok)) {
                    ok = false;
                    break;
                }
                tc::fence_after_sync();
                float x[C::SK];
                ld_scores(sP, x);
                if (__any_sync(FW_FULL, (i + 1) * C::SK > seen)) {
                    const int lim = seen - i * C::SK;
#pragma unroll
                    for (int e = 0; e < C::SK; ++e) x[e] = e < lim ? x[e] : -INFINITY;
                }
                float top[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = max3(x[3 * e], x[3 * e + 1], x[3 * e + 2]);
#pragma unroll
                for (int e = 12; e + 1 < C::SK; e += 2) top[(e >> 1) & 3] = max3(top[(e >> 1) & 3], x[e], x[e + 1]);
                const float xm = fmaxf(max3(top[0], top[1], top[2]), top[3]) * c2;
                const bool need = xm > ref + GROW;
                if (__any_sync(FW_FULL, need)) {
                    const float now = need ? xm : ref;  // (a row's result does not depend on its neighbours)
                    const float f = now == ref ? 1.f : ex2(ref - now);
                    l *= f;
                    ref = now;
                    if (i > 0) {
                        ok = tc::mbar_wait(&o_done[t], (uint32_t)(i - 1) & 1u, P_WAIT);
                        if (!__all_sync(FW_FULL, ok)) {
                            ok = false;
                            break;
                        }
                        tc::fence_after_sync();
#pragma unroll 1
                        for (int h = 0; h < D; h += 16) {
                            float y[16];
                            tc::ld16(sO + h, y);
                            uint32_t z[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(y[e] * f);
                            st16(sO + h, z);
                        }
                    }
                }
                const float off = ref == -INFINITY ? 0.f : -ref;
                const float2 cc = make_float2(c2, c2), oo = make_float2(off, off);
                float2 sum[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = make_float2(0.f, 0.f);
#pragma unroll
                for (int c = 0; c < C::SK / 32; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 w = fma2(make_float2(x[32 * c + e], x[32 * c + e + 1]), cc, oo);
                        w.x = ex2(w.x);
                        w.y = ex2(w.y);
                        sum[(e >> 1) & 3] = add2(sum[(e >> 1) & 3], w);
                        p[e >> 1] = pack_bf16(w.x, w.y);
                    }
                    st16(sP + 16 * c, p);
                }
                hand_over(&p_full[t][u], lane);
                sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
                l += sum[0].x + sum[0].y;
            }
            // ------------------------------------------------------ epilogue
            // (its queries' memory is written below: without products, the copy has to have landed)
            if (ok && J > 0) ok = n > 0 ? tc::mbar_wait(&drained[t], 0, P_WAIT) : tc::mbar_wait(&q_full, 0, P_WAIT);
            if (ok && J > jm) ok = tc::mbar_wait(&v_ok[min(J - 1 - jm, PG - 1)], 0, P_WAIT);  // (the guard is done)
            ok = __all_sync(FW_FULL, ok);
            if (!ok && lane == 0) atomicOr(&s_err, 1);
            tc::fence_after_sync();
            const bool odd = *(volatile int *)&s_odd != 0;
            const int64_t row = (int64_t)(q0 + tok) * a.q_heads + hk * a.group + r % a.group;
            // (of a part: as it is, the parts' sums come later)
            const float inv = !ok ? NAN : split ? 1.f : l == 0.f ? 0.f : 1.f / l;
            // The rows go out by way of the tile's queries' memory (the products have read them), a warp's 32 rows its
            // own: whole rows a store.  (A row a lane: 32 lines an instruction, 6,200 clocks for a CTA's rows.)
            constexpr int PCS = D / 8;  // 16-byte pieces of a row
            uint4 *stage = reinterpret_cast<uint4 *>(sQ + t * C::QT) + (r & ~31) * PCS;
#pragma unroll 1
            for (int i = 0; i < D; i += 64) {
                float y[64];
                if (ok && n > 0) {
                    ld_scores(sO + i, y);
                } else {
#pragma unroll
                    for (int e = 0; e < 64; ++e) y[e] = 0.f;
                }
                // (a row that sees nothing has no O where its tile saw nothing: its sum is 0 and so is it)
#pragma unroll
                for (int e = 0; e < 64; ++e) y[e] = l == 0.f && ok ? 0.f : y[e] * inv;
                if (odd && live) {  // the values the guard took out, for the rows that see them
#pragma unroll 1
                    for (int j = jm * PK; j < seen; ++j) {
                        const uint16_t *src = a.v + (int64_t)(kb + j) * a.v_row + hk * a.v_head + i;
#pragma unroll
                        for (int e = 0; e < 64; ++e) {
                            const uint16_t b = src[e];
                            if ((b & 0x7f80u) == 0x7f80u) y[e] += bf16_to_f32(b);
                        }
                    }
                }
                if (split) {  // (the products are done with the ring's memory)
                    float4 *dst = reinterpret_cast<float4 *>(sKV) + r * (D / 4);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        dst[(i / 4 + e) ^ (r & 7)] = make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    stage[lane * PCS + ((i / 8 + e) ^ (lane & 7))] =
                        make_uint4(pack_bf16(y[8 * e], y[8 * e + 1]), pack_bf16(y[8 * e + 2], y[8 * e + 3]),
                                   pack_bf16(y[8 * e + 4], y[8 * e + 5]), pack_bf16(y[8 * e + 6], y[8 * e + 7]));
            }
            __syncwarp();
            if (split) reinterpret_cast<float2 *>(sQ)[r] = make_float2(ref, ok ? l : NAN);
#pragma unroll 8
            for (int p = 0; !split && p < 32; p += 32 / PCS) {
                const int k = p + lane / PCS, c = lane % PCS;
                const int64_t to = __shfl_sync(FW_FULL, live ? row : -1, k);
                if (to >= 0) reinterpret_cast<uint4 *>(a.o + to * D)[c] = stage[k * PCS + (c ^ (k & 7))];
            }
            if (live && a.lse && !split)
                a.lse[row] = !ok ? NAN : l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (split) {
        // The parts of every row joined over the cluster: a CTA takes every parts-th row, a warp a row at a time.
        cluster_sync();
        for (int r = part + a.parts * wid; r < 128; r += a.parts * (PT / 32)) {
            const int tok = t0 + r / a.group;
            if (r >= TT * a.group || tok >= lq) continue;
            // (columns 4 lane .. of 32 lanes, or 2 lane ..: one piece of 16 bytes, or half of one)
            const float *src = reinterpret_cast<float *>(sKV) + r * D +
                               (D == 128 ? 4 * (lane ^ (r & 7)) : 4 * ((lane >> 1) ^ (r & 7)) + 2 * (lane & 1));
            float m[MAX_PARTS], l[MAX_PARTS], x[MAX_PARTS][D / 32];
#pragma unroll
            for (int p = 0; p < MAX_PARTS; ++p) {  // (all reads under way at once)
                const bool in = p < a.parts;
                float ml[2] = {-INFINITY, 0.f};
                if (in) remote(reinterpret_cast<float *>(sQ) + 2 * r, p, ml);
                m[p] = ml[0];
                l[p] = ml[1];
#pragma unroll
                for (int e = 0; e < D / 32; ++e) x[p][e] = 0.f;
                if (in) remote(src, p, x[p]);
            }
            float M = -INFINITY, L = 0.f, y[D / 32];
#pragma unroll
            for (int p = 0; p < MAX_PARTS; ++p) M = fmaxf(M, m[p]);
#pragma unroll
            for (int e = 0; e < D / 32; ++e) y[e] = 0.f;
#pragma unroll
            for (int p = 0; p < MAX_PARTS; ++p) {
                const float f = m[p] == M ? 1.f : ex2(m[p] - M);
                L = fmaf(f, l[p], L);
#pragma unroll
                for (int e = 0; e < D / 32; ++e) y[e] = fmaf(f, x[p][e], y[e]);
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const int64_t row = (int64_t)(q0 + tok) * a.q_heads + hk * a.group + r % a.group;
            uint32_t *dst = reinterpret_cast<uint32_t *>(a.o + row * D + lane * (D / 32));
#pragma unroll
            for (int e = 0; e < D / 32; e += 2) dst[e / 2] = pack_bf16(L == 0.f ? 0.f : y[e] * inv, L == 0.f ? 0.f : y[e + 1] * inv);
            if (a.lse && lane == 0) a.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
        }
        cluster_sync();  // no CTA leaves while another reads its rows
    }
    if (tid == 0 && s_err && a.status) a.status[seq] = FW_ERR_TIMEOUT;
    if (wid == C::W_MMA) {
        tc::fence_after_sync();
        tc::tmem_dealloc(taddr, C::COLS);
    }
}

// Whether a CTA takes one tile instead of two: where the CTAs of two would not fill half of the SMs (512 tokens, 8 x 4
// heads, d = 128: 10.9 us against 13.6), and for d = 64, where two such CTAs fit an SM and one starts and ends while the
// other computes (16 prompts of 300 tokens 32.3 us against 35.1, 8,192 tokens 291 against 302).
bool one_tile(int d, int64_t ctas_of_two, int sms)
{
    return d == 64 || ctas_of_two * 2 <= sms;
}

template <int D, int TILES>
fw_status launch(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PromptArgs &a, cudaStream_t s)
{
    using C = PCfg<D, TILES>;
    const auto kernel = k_prompt<D, TILES>;
    static std::atomic<uint64_t> done{0};
    const fw_status st = big_smem((const void *)kernel, C::SMEM, done);
    if (st != FW_OK) return st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)a.parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.slots * a.kv_heads * a.parts));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = a.parts > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, mq, mk, mv, a);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? FW_OK : FW_ERR_CUDA;
}

}  // namespace

fw_status prompt_attention(const fw_prompt &p, void *o, float *lse, int32_t *status, cudaStream_t s)
{
    if (p.total_q == 0) {
        PromptArgs a{};
        a.cu_q = p.cu_q, a.cu_k = p.cu_k, a.total_k = p.total_k, a.num_seqs = p.num_seqs, a.status = status;
        if (status) FW_LAUNCH(k_prompt_status, ((unsigned)p.num_seqs + 255u) / 256u, 256, 0, s, a);
        return FW_OK;
    }
    const int group = p.q_heads / p.kv_heads, TT = 128 / group;
    int sms = 0;
    const fw_status st = device_sms(&sms);
    if (st != FW_OK) return st;
    auto slots_of = [&](int tiles) { return p.total_q / (tiles * TT) + p.num_seqs; };
    const int tiles = one_tile(p.d, slots_of(2) * p.kv_heads, sms) ? 1 : 2;
    const int64_t slots = slots_of(tiles);
    if (slots * p.kv_heads >= ((int64_t)1 << 31)) return FW_ERR_UNSUPPORTED;  // (parts only where this is small)
    // Few rows against long keys: the keys of a slot split over a cluster, as long as the CTAs fit the SMs once.  The
    // joining costs several blocks' time, so only from SPLIT blocks on average on, and MIN_PART or more to a part
    // (one sequence, 8 x 4 heads, d = 128: 17 rows against 16,384 keys 130 us whole, 24 in 8 parts; 256 against 2,048
    // 28.4 whole, 26.3 in 2; d = 64, 128 against 1,024 16.2 whole, 19.1 in 2).  The host knows the lengths' mean alone: a long
    // sequence among short ones is not split (16 of one token on 8 KV heads, 128 keys each but one with 16,384: 127 us).
    // (Of two tiles a CTA there are more than half as many CTAs as SMs, so that their keys are never split.)
    const int64_t blocks = p.total_k / ((int64_t)p.num_seqs * PK);
    int parts = 1;
    while (blocks >= SPLIT && parts < MAX_PARTS && slots * p.kv_heads * parts * 2 <= sms && blocks >= MIN_PART * parts * 2)
        parts *= 2;
    CUtensorMap mq, mk, mv;
    // (without keys no copy is issued: any valid map does)
    const bool keys = p.total_k > 0;
    if (!make_tma_heads_bf16(&mq, p.q, p.d, p.q_heads, p.total_q, p.q_head, p.q_row, group, TT) ||
        !make_tma_heads_bf16(&mk, keys ? p.k : p.q, p.d, p.kv_heads, keys ? p.total_k : 1, keys ? p.k_head : p.d,
                             keys ? p.k_row : (int64_t)p.d * p.kv_heads, 1, PK) ||
        !make_tma_heads_bf16(&mv, keys ? p.v : p.q, p.d, p.kv_heads, keys ? p.total_k : 1, keys ? p.v_head : p.d,
                             keys ? p.v_row : (int64_t)p.d * p.kv_heads, 1, PK))
        return FW_ERR_CUDA;
    const PromptArgs a{p.cu_q,  p.cu_k,     p.total_q, p.total_k, p.num_seqs, p.q_heads, p.kv_heads,
                       group,   (int)slots, TT, parts, (const uint16_t *)p.v, p.v_row,   p.v_head,
                       p.scale * 1.4426950408889634f, (uint16_t *)o, lse,  status};
    if (p.d == 64) return launch<64, 1>(mq, mk, mv, a, s);
    return tiles == 1 ? launch<128, 1>(mq, mk, mv, a, s) : launch<128, 2>(mq, mk, mv, a, s);
}

}  // namespace fw
