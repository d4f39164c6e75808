// y[p] = W x[row(p)] for 4-bit weights with a scale for every group of inputs (gs4 layers, layout in rmsmp.h), on tcgen05: what the few-token
// kernel (gs4_product.cu) would read the weights more than once or twice for.
//   y[p][m] = sum_u s[m][u] * (sum_{k in u} (code[m][k] - zero[m][u]) * x[k]),   u: runs of 32, 64 or 128 inputs
// A CTA takes 128 rows and kBN tokens.  For every 128 inputs its sixteen working warps turn the packed codes into exact 16-bit floats of the activations'
// type in shared memory (operand A, 128-byte swizzle), the tokens' inputs come beside them (operand B), and one warp issues the matrix instructions, a run's
// into one of two accumulators in tensor memory.  While they run, the working warps take the accumulators of the 128 inputs before, multiply each
// by its row's scale and add it to fp32 sums in registers.  Scales never touch the operands: a code times a scale, rounded to 16 bits, was tried (one accumulator
// for all inputs) and has 1.3 to 1.4 times the error.
// An fp32 activation is three bf16 numbers (its bits cut 8 at a time: exact down to 2^-133) that the same accumulator adds up, with three times the instructions.
// Packed codes come through a ring of bulk copies.  x comes by tensor copies where its rows follow each other, else in the workers' hands.
// A cluster of `split` CTAs shares the inputs where there are few tiles; its sums meet in distributed shared memory, in a fixed order.
// 4096 x 4096 for 1024 bf16 tokens: 42 us, 813 TFLOP/s, half of the measured 1679; 4096 x 1024 for 2048 in groups of 64: 31.9 us, 538.  What bounds it there is
// the hand-over between the roles: 2060 cycles for 128 inputs, of which the instructions need 1024; with no expansion, no instructions and no sums at all 1400 are
// left (29 us), as many for 192 tokens a tile as for 256; without expansion and sums it is 40 us, without the instructions 37.  No unit is busy (tensor pipe 34 %,
// shared memory and copies 26 %, L2 14 %).  Tried against that: pairs of CTAs that share operand B (cta_group::2, 256 rows: every block waits for the other CTA,
// 63 us); operand A in tensor memory (no room for two accumulators of 256 tokens; 192: 39 us for 768 tokens, 41 this way); a warp of its own for the copies of
// codes, and their slots free before the sums are taken (46 us); blocks of inputs in another order for every CTA (48 us: CTAs that read the same x at the same time
// share their reads).  With few tokens a tile it is the expansion, some 600 cycles a block whatever their number: 8192 x 8192, 9 to 64 tokens 31 to 36 us (floor 5.4), 4096 x 4096, 64 tokens
// 12 to 13 (1.5).  fp32: tiles of 64 tokens at most, whose x every row tile's CTAs split again: 4096 x 4096, 512 tokens 123 us, 140 TFLOP/s; 4096 x 1024, 2048 tokens 129.
#include <algorithm>
#include "gs4.cuh"
#include "ptx.cuh"
#include "tmap.cuh"

namespace rmsmp {

namespace {

constexpr int kWorkers = 512, kWorkWarps = kWorkers / 32;
constexpr int kIssuer = kWorkWarps, kCopier = kWorkWarps + 1;         // the warp that issues matrix instructions; the one that issues copies of x
constexpr int kBytesA = 128 * 128 * 2;                    // operand A of 128 inputs: two tiles of 128 rows x 64 inputs
constexpr int kOutPad = 4;                                // floats behind a token's 128 sums in shared memory

struct Plan {
    Gs4Args a;
    int ring;                            // blocks of 128 inputs in the ring of packed codes
    int split, units;                    // CTAs of a cluster; blocks of 128 inputs of each
    int mtiles, ntiles;                  // row tiles; token tiles (experts: as many as there can be)
    int y_vec;                           // four sums can be stored at once
    CUtensorMap x_map;                   // of x: boxes of 64 inputs x kBN tokens (kBulk only)
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, uint64_t src, uint32_t bytes)      // 16 bytes, of which the first `bytes` (0 or 16) are read and the others zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void store16(uint32_t dst, const uint32_t (&w)[4])
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
__device__ __forceinline__ void cluster_arrive_wait()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster(uint32_t addr, int rank)
{
    uint32_t r;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(r) : "memory");
    return v;
}
// kSteps matrix instructions of 16 inputs, 32 bytes further on in both operands' rows each; the whole warp takes part, the elected lane issues (see
// mma_i8_step in ptx.cuh).  The descriptors' halves: `hi` is the same for both.
template <int kSteps>
__device__ __forceinline__ void mma_f16_steps(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate)
{
#define RMSMP_F16_HEAD "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
#define RMSMP_F16_MMA "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t"
#define RMSMP_F16_NEXT "setp.eq.u32 p, 0, 0;\n\tadd.s64 da, da, 2;\n\tadd.s64 db, db, 2;\n\t" RMSMP_F16_MMA
    static_assert(kSteps == 2 || kSteps == 4, "");
    if (kSteps == 2)
        asm volatile(RMSMP_F16_HEAD RMSMP_F16_MMA RMSMP_F16_NEXT "}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(RMSMP_F16_HEAD RMSMP_F16_MMA RMSMP_F16_NEXT RMSMP_F16_NEXT RMSMP_F16_NEXT "}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) : "memory");
#undef RMSMP_F16_HEAD
#undef RMSMP_F16_MMA
#undef RMSMP_F16_NEXT
}
// two sums at once: t += s * v
__device__ __forceinline__ void fma2(float2& t, float2 s, float2 v)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(reinterpret_cast<uint64_t&>(t)) : "l"(reinterpret_cast<uint64_t&>(s)), "l"(reinterpret_cast<uint64_t&>(v)));
}
// kN consecutive columns of this lane's row.
template <int kN> struct Columns;
template <> struct Columns<4> {
    static __device__ __forceinline__ void load(uint32_t at, float (&v)[4])
    {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at) : "memory");
        asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]) :: "memory");
    }
};
template <> struct Columns<8> {
    static __device__ __forceinline__ void load(uint32_t at, float (&v)[8])
    {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(at) : "memory");
        asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]) :: "memory");
    }
};
template <> struct Columns<16> {
    static __device__ __forceinline__ void load(uint32_t at, float (&v)[16])
    {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
                       "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(at) : "memory");
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
                       "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]) :: "memory");
    }
};

// Eight codes of rows g (lo) and g + 8 (hi), four consecutive inputs each, to code - zero as pairs of 16-bit floats.  r[0], r[2]: row g; r[1], r[3]: row g + 8.
// (As in gs4_product.cu: in fp16 a code adds itself to 1024 or, four bits up, 16 times itself; in bf16 it has to be in the low bits of 128.)
template <bool kBf>
__device__ __forceinline__ void expand(uint32_t w, uint32_t lo, uint32_t hi, uint32_t (&r)[4])
{
    if (kBf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v;
            asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w >> (4 * i)), "n"(0x000F000F), "r"(0x43004300u));
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(i & 1 ? hi : lo));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t u, v;
            asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w >> (8 * i)), "n"(0x000F000F), "r"(0x64006400u));
            asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w >> (8 * i)), "n"(0x00F000F0), "r"(0x64006400u));
            asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r[2 * i]) : "r"(u), "r"(lo));
            asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[2 * i + 1]) : "r"(v), "r"(0x2C002C00u), "r"(hi));
        }
    }
}

// (four deep as long as a stage has at most 32 KB)
template <int kBN, int kX>
constexpr int kStagesB = kBN * (kX == RMSMP_F32 ? 3 : 1) <= 128 ? 4 : 2;
template <int kBN, int kX>
constexpr int kBytesB = kBN * 256 * (kX == RMSMP_F32 ? 3 : 1);      // operand B of 128 inputs: two tiles of kBN tokens x 64 inputs, three times in parts

template <bool kBulk> constexpr int kThreads = kWorkers + (kBulk ? 64 : 32);

// kBulk: x comes by tensor copies (16-bit rows that start on 16 bytes and follow each other), else in the workers' hands.  (Gathered rows by tensor copies of
// four rows: sixteen experts of 4096 x 1024 over 8192 rows 398 us, 174 by the workers.)  Eighteen warps leave 96 registers a thread; at that ptxas spills three to six words (and
// reads two to eleven back) in the forms of 192 tokens with tensor copies and those of 256.
template <int kBN, int kX, bool kBulk>
__global__ void __launch_bounds__(kThreads<kBulk>, 1) gs4_tensor_kernel(const __grid_constant__ Plan p)
{
    constexpr bool kBf = kX != RMSMP_F16;
    constexpr int kParts = kX == RMSMP_F32 ? 3 : 1, kSB = kStagesB<kBN, kX>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const smem = smem_raw + (-smem_u32(smem_raw) & 1023u);
    __shared__ __align__(8) uint64_t s_full[16], s_empty[16], s_ready[2], s_done[2], s_free[2], s_xfull[kSB], s_xempty[kSB];
    __shared__ uint64_t s_row[kBN];                                 // address of a token's inputs, 0: zeros
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_tile[3];
    constexpr int kCols = kBN / 4;                                  // tokens of a warp's sums
    constexpr int kLd = kCols < 16 ? kCols : 16;
    const Gs4Args& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int sums = a.sums;
    constexpr uint32_t kRunCols = kBN < 32 ? 32 : kBN, kTmemCols = kBN == 192 ? 512 : 2 * kRunCols;      // two accumulators; a power of two
    auto allocate = [&]() {
        // (in front of the trigger: a kernel that is placed early must not hold tensor memory that this one still has to get)
        if (warp == kIssuer) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "n"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    };
    if (!a.offsets) allocate();
    if (tid == 0) {
        s_abort = 0;
        for (int i = 0; i < p.ring; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_empty[i]), kWorkWarps);
        }
        for (int i = 0; i < kSB; ++i) {
            mbar_init(smem_u32(&s_xfull[i]), 1);
            mbar_init(smem_u32(&s_xempty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s_ready[i]), kWorkWarps);
            mbar_init(smem_u32(&s_done[i]), 1);
            mbar_init(smem_u32(&s_free[i]), kWorkWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    }
    pdl_wait();
    // which tile: token tiles of experts follow from the offsets
    const int rank = blockIdx.x % p.split, mt = blockIdx.x / p.split % p.mtiles, nt = blockIdx.x / p.split / p.mtiles;
    if (a.offsets) {
        if (tid == 0) s_tile[0] = -1;
        __syncthreads();
        if (warp == 0) {
            int before = 0;
            for (int e0 = 0; e0 < a.E && before <= nt; e0 += 32) {
                const int e = e0 + lane;
                int64_t lo = 0, hi = 0;
                if (e < a.E) {
                    lo = min(max((int64_t)a.offsets[e], (int64_t)0), a.R);
                    hi = min((int64_t)a.offsets[e + 1], a.R);
                }
                const int mine = hi > lo ? (int)((hi - lo + kBN - 1) / kBN) : 0;
                int upto = mine;
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                const int start = before + upto - mine;
                if (nt >= start && nt < start + mine) {
                    const int64_t b = lo + (int64_t)(nt - start) * kBN;
                    s_tile[0] = e; s_tile[1] = (int)b; s_tile[2] = (int)min((int64_t)kBN, hi - b);
                }
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
        }
        __syncthreads();
        if (s_tile[0] < 0) return;                                  // (fewer tiles than there could be; the same for a whole cluster)
        allocate();
    }
    const int expert = a.offsets ? s_tile[0] : 0;
    const int64_t p0 = a.offsets ? s_tile[1] : (int64_t)nt * kBN;
    const int n = a.offsets ? s_tile[2] : (int)min((int64_t)kBN, a.R - p0);
    for (int t = tid; t < kBN; t += kThreads<kBulk>) {
        uint64_t at = 0;
        if (t < n) {
            const int64_t row = a.rows ? a.rows[p0 + t] : p0 + t;
            if (row >= 0 && row < a.x_rows) at = reinterpret_cast<uint64_t>(a.x) + row * a.ld_x * (kX == RMSMP_F32 ? 4 : 2);
        }
        s_row[t] = at;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = s_tmem;
    volatile int* abort_flag = &s_abort;
    bool alive = true;

    const uint32_t units_k = (uint32_t)a.Kp >> 7;
    const int unit0 = rank * p.units, units = max(0, min(p.units, (int)units_k - unit0));
    uint8_t* const smem_a = smem;                                   // [2][kBytesA]
    uint8_t* const smem_b = smem + 2 * kBytesA;                     // [kSB][kBytesB]
    uint8_t* const ring = smem_b + kSB * kBytesB<kBN, kX>;          // [p.ring][4][block_bytes]
    const uint8_t* const blocks = a.blocks + ((int64_t)expert * a.tiles + mt * 4) * units_k * a.block_bytes;
    const int row_blocks = min(4, a.tiles - mt * 4);

    const uint32_t slot_bytes = 4u * a.block_bytes;
    constexpr uint32_t idesc = (1u << 4) | (kBf ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(kBN >> 3) << 17) | (8u << 24);
    float2 tot[kCols / 2];
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) tot[i] = make_float2(0.0f, 0.0f);
    const int quarter = warp & 3, group = warp >> 2;                // a worker's rows (of the accumulators; its share of the codes' block `group`), and tokens

    if (warp == kIssuer) {
        // ---- the issuing warp: packed codes come in, matrix instructions go out
        int fetched = 0, fetch_slot = 0;
        const uint8_t* fetch_from = blocks + ((uint64_t)min(lane, row_blocks - 1) * units_k + unit0) * a.block_bytes;
        uint32_t fetch_parity = 1;                                  // (the first round waits for nobody)
        auto fetch = [&]() {                                        // the next block
            const uint32_t bar = smem_u32(&s_full[fetch_slot]);
            alive = mbar_wait_step(smem_u32(&s_empty[fetch_slot]), fetch_parity, abort_flag) && alive;
            if (lane == 0) mbar_arrive_expect_tx(bar, row_blocks * a.block_bytes);
            __syncwarp();
            if (lane < row_blocks) bulk_load(smem_u32(ring + fetch_slot * slot_bytes + lane * a.block_bytes), fetch_from, a.block_bytes, bar);
            fetch_from += a.block_bytes;
            ++fetched;
            if (++fetch_slot == p.ring) { fetch_slot = 0; fetch_parity ^= 1; }
        };
        for (int u = 0; u < units && u < p.ring - 2; ++u) fetch();
        const uint32_t hi32 = (uint32_t)(smem_desc_kmajor(0, 128) >> 32), a0 = (smem_u32(smem_a) >> 4) | (1u << 16), b0 = (smem_u32(smem_b) >> 4) | (1u << 16);
        uint32_t run = 0, x_parity = 0;
        int stage = 0;
        for (int u = 0; u < units; ++u) {
            // The block after next at the latest, into the slot of block u - 2, and in front of this block's instructions: with four runs the third waits
            // until the first has been taken, which the workers do behind the operands of block u + 1.
            if (fetched < units) fetch();
            if (kBulk) alive = mbar_wait_step(smem_u32(&s_xfull[stage]), x_parity, abort_flag) && alive;
            alive = mbar_wait_step(smem_u32(&s_ready[u & 1]), (u >> 1) & 1, abort_flag) && alive;
            tc_fence_after();
            const uint32_t a_lo = a0 + (u & 1) * (kBytesA / 16), b_lo = b0 + stage * (kBytesB<kBN, kX> / 16);
            for (int r = 0; r < sums; ++r, ++run) {
                if (run >= 2) {
                    alive = mbar_wait_step(smem_u32(&s_free[run & 1]), ((run >> 1) & 1) ^ 1, abort_flag) && alive;
                    tc_fence_after();
                }
                const uint32_t d = tmem + (run & 1) * kRunCols;
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const uint32_t bq = b_lo + q * (kBN * 256 / 16);
                    if (sums == 4) {
                        mma_f16_steps<2>(d, a_lo + (r >> 1) * 1024 + (r & 1) * 4, bq + (r >> 1) * (kBN * 8) + (r & 1) * 4, hi32, idesc, q);
                    } else if (sums == 2) {
                        mma_f16_steps<4>(d, a_lo + r * 1024, bq + r * (kBN * 8), hi32, idesc, q);
                    } else {
                        mma_f16_steps<4>(d, a_lo, bq, hi32, idesc, q);
                        mma_f16_steps<4>(d, a_lo + 1024, bq + kBN * 8, hi32, idesc, 1);
                    }
                }
                mma_commit_step(smem_u32(&s_done[run & 1]));
            }
            if (kBulk) mma_commit_step(smem_u32(&s_xempty[stage]));
            if (++stage == kSB) { stage = 0; x_parity ^= 1; }
        }
    } else if (kBulk && warp == kCopier) {
        // ---- the copying warp: the tokens' inputs; K's end and rows that are not there read as zeros
        int stage = 0;
        uint32_t parity = 1;                                        // (the first round waits for nobody)
        for (int u = 0; u < units; ++u) {
            alive = mbar_wait_step(smem_u32(&s_xempty[stage]), parity, abort_flag) && alive;
            const uint32_t bar = smem_u32(&s_xfull[stage]), to = smem_u32(smem_b) + stage * kBytesB<kBN, kX>;
            const int k = (unit0 + u) * 128;
            if (lane == 0) mbar_arrive_expect_tx(bar, kBN * 256);
            __syncwarp();
            if (lane < 2) tma_load_2d(to + lane * (kBN * 128), &p.x_map, bar, k + lane * 64, (int)p0);
            if (++stage == kSB) { stage = 0; parity ^= 1; }
        }
    } else {
        // ---- the working warps
        // A thread copies inputs 8c .. 8c + 7 of every 32nd token.
        constexpr int kEach = (kBN * 16 + kWorkers - 1) / kWorkers;
        const int xc = tid & 15, xt = tid >> 4;
        const uint32_t x_dst = (xc >> 3) * (kBN * 128) + xt * 128 + (((xc & 7) ^ (xt & 7)) << 4);
        int stage_k = unit0 * 128;
        uint32_t stage_at = smem_u32(smem_b);
        const uint32_t stage_end = stage_at + kSB * kBytesB<kBN, kX>;
        auto copy_x = [&](int j) {                                  // one token's part of the next block
            const uint64_t at = s_row[min(xt + 32 * j, kBN - 1)];
            if (kBN * 16 >= kWorkers || xt < kBN)
                copy16(stage_at + x_dst + j * 4096, at != 0 ? at + (stage_k + xc * 8) * 2 : reinterpret_cast<uint64_t>(a.x), at != 0 ? 16u : 0u);
        };
        auto staged = [&]() {
            asm volatile("cp.async.commit_group;" ::: "memory");
            stage_k += 128;
            stage_at += kBytesB<kBN, kX>;
            if (stage_at == stage_end) stage_at = smem_u32(smem_b);
        };
        auto stage_x = [&]() {                                      // the tokens' inputs of the next block
            if (kX != RMSMP_F32 && a.x_vec && stage_k + 128 <= a.K) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) copy_x(j);
            } else {
                const int k = stage_k + xc * 8;
                for (int j = 0; j < kEach; ++j) {
                    if (kBN * 16 < kWorkers && xt >= kBN) break;
                    const uint64_t at = s_row[xt + 32 * j];
                    const uint32_t dst = stage_at + x_dst + j * 4096;
                    const int have = at ? min(8, a.K - k) : 0;      // may be negative
                    if (kX != RMSMP_F32) {
                        const uint16_t* src = reinterpret_cast<const uint16_t*>(at) + k;
                        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < have) w[i >> 1] |= (uint32_t)src[i] << (16 * (i & 1));
                        store16(dst, w);
                        continue;
                    }
                    const uint32_t* src = reinterpret_cast<const uint32_t*>(at) + k;
                    uint32_t b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (have == 8 && a.x_vec) {
                        *reinterpret_cast<uint4*>(b) = *reinterpret_cast<const uint4*>(src);
                        *reinterpret_cast<uint4*>(b + 4) = *reinterpret_cast<const uint4*>(src + 4);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < have) b[i] = src[i];
                    }
                    // cut off, not rounded: no part overflows
                    uint32_t part[3][4];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const bool finite = (b[i] & 0x7f800000u) != 0x7f800000u;
                        uint32_t h = b[i] >> 16;
                        if (!finite && (b[i] & 0x7fffffu)) h |= 0x40u;                    // (a NaN whose bits are all in the lower half)
                        const float r1 = finite ? __uint_as_float(b[i]) - __uint_as_float(b[i] & 0xffff0000u) : 0.0f;
                        const uint32_t m = __float_as_uint(r1);
                        const uint32_t l = __float_as_uint(r1 - __uint_as_float(m & 0xffff0000u));
                        if (i & 1) {
                            part[0][i >> 1] |= h << 16;
                            part[1][i >> 1] |= m & 0xffff0000u;
                            part[2][i >> 1] |= l & 0xffff0000u;
                        } else {
                            part[0][i >> 1] = h;
                            part[1][i >> 1] = m >> 16;
                            part[2][i >> 1] = l >> 16;
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 3; ++q) store16(dst + q * (kBN * 256), part[q]);
                }
            }
            staged();
        };

        const uint8_t* const my_scales = ring + min(quarter, row_blocks - 1) * a.block_bytes + kCodeBytes + ((lane & 7) * sums * 4 + (lane >> 3)) * 2;
        const uint32_t my_tmem = tmem + ((uint32_t)quarter << 21) + group * kCols;
        const bool scale_bf16 = a.scale_bf16;
        uint32_t run = 0;
        // The accumulators of a block's runs, in turn.  `with_x`: the copies of the next block's inputs, into what the last run's instructions have read, go out
        // between the loads from tensor memory, whose latency they fill.
        auto flush = [&](uint32_t slot_at, int slot, bool with_x) {
            for (int r = 0; r < sums; ++r, ++run) {
                const float f = scale_value(*reinterpret_cast<const uint16_t*>(my_scales + slot_at + r * 8), scale_bf16);
                const float2 s = make_float2(f, f);
                alive = mbar_wait_step(smem_u32(&s_done[run & 1]), (run >> 1) & 1, abort_flag) && alive;
                tc_fence_after();
                const uint32_t at = my_tmem + (run & 1) * kRunCols;
#pragma unroll
                for (int c = 0; c < kCols; c += kLd) {
                    float v[kLd];
                    Columns<kLd>::load(at + c, v);
#pragma unroll
                    for (int i = 0; i < kLd; i += 2) fma2(tot[(c + i) / 2], s, make_float2(v[i], v[i + 1]));
                    if (!kBulk && with_x && r == sums - 1) {
                        constexpr int kSteps = kCols / kLd;
#pragma unroll
                        for (int j = c / kLd * kEach / kSteps; j < (c / kLd + 1) * kEach / kSteps; ++j) copy_x(j);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_free[run & 1]));
            }
            if (lane == 0) mbar_arrive(smem_u32(&s_empty[slot]));
        };
        // operand A: this warp's 16 rows x 64 inputs of block `group`
        const int half = quarter >> 1, part = quarter & 1, g = lane >> 2, odd = g & 1;      // (odd rows take their halves the other way round: rows 128 bytes apart would meet in the same banks)
        const uint8_t* const my_codes = ring + min(group, row_blocks - 1) * a.block_bytes + quarter * 512 + lane * 16;
        const uint8_t* const my_zeros = ring + min(group, row_blocks - 1) * a.block_bytes + kCodeBytes + 64 * sums + g * sums * 2;
        uint8_t* const my_a = smem_a + part * (128 * 128) + (group * 32 + half * 16 + g) * 128;
        const int chunk0 = ((4 * odd + (lane & 3)) ^ g) << 4, chunk1 = ((4 * (1 - odd) + (lane & 3)) ^ g) << 4;
        const int zero0 = (2 * part + odd) * sums / 4 * 2, zero1 = (2 * part + 1 - odd) * sums / 4 * 2;

#pragma unroll
        for (int u = 0; u < kSB - 1 && !kBulk; ++u) {
            if (u < units) stage_x();
            else asm volatile("cp.async.commit_group;" ::: "memory");
        }
        int slot = 0, last_slot = 0;
        uint32_t slot_at = 0, last_at = 0, slot_parity = 0;
        for (int u = 0; u < units; ++u) {
            const uint32_t buf = u & 1;
            alive = mbar_wait_step(smem_u32(&s_full[slot]), slot_parity, abort_flag) && alive;
            {
                const uint4 q = *reinterpret_cast<const uint4*>(my_codes + slot_at);
                uint8_t* const to = my_a + buf * kBytesA;
                uint32_t zz0 = 0x88u, zz1 = 0x88u;
                if (a.has_zeros) {
                    zz0 = (uint32_t)*reinterpret_cast<const uint16_t*>(my_zeros + slot_at + zero0) >> (8 * half);
                    zz1 = (uint32_t)*reinterpret_cast<const uint16_t*>(my_zeros + slot_at + zero1) >> (8 * half);
                }
                const uint32_t w[4] = {odd ? q.z : q.x, odd ? q.w : q.y, odd ? q.x : q.z, odd ? q.y : q.w};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t zz = i ? zz1 : zz0;
                    const uint32_t lo = kBf ? (0x4300u + (zz & 15u)) * 0x10001u : (0x6400u + (zz & 15u)) * 0x10001u;
                    const uint32_t hi = kBf ? (0x4300u + (zz >> 4 & 15u)) * 0x10001u : (0xD400u + (zz & 0xF0u)) * 0x10001u;
                    uint32_t r0[4], r1[4];
                    expand<kBf>(w[2 * i], lo, hi, r0);
                    expand<kBf>(w[2 * i + 1], lo, hi, r1);
                    uint8_t* const at = to + (i ? chunk1 : chunk0);
                    *reinterpret_cast<uint4*>(at) = make_uint4(r0[0], r0[2], r1[0], r1[2]);
                    *reinterpret_cast<uint4*>(at + 8 * 128) = make_uint4(r0[1], r0[3], r1[1], r1[3]);
                }
            }
            if (!kBulk) asm volatile("cp.async.wait_group %0;" ::"n"(kSB - 2) : "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s_ready[buf]));
            // (block u - 1's matrix instructions are over behind its last run: its operands may go)
            const bool more = !kBulk && u + kSB - 1 < units, with_x = more && u > 0 && kX != RMSMP_F32 && a.x_vec && stage_k + 128 <= a.K;
            if (u > 0) flush(last_at, last_slot, with_x);
            if (with_x) staged();
            else if (more) stage_x();
            else if (!kBulk) asm volatile("cp.async.commit_group;" ::: "memory");
            last_at = slot_at;
            last_slot = slot;
            slot_at += slot_bytes;
            if (++slot == p.ring) { slot = 0; slot_at = 0; slot_parity ^= 1; }
        }
        if (units > 0) flush(last_at, last_slot, false);
    }

    // sums to shared memory (operands and ring are done with), [token][128 rows]
    float* const out = reinterpret_cast<float*>(smem);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        if (warp < kWorkWarps) out[(group * kCols + i) * (128 + kOutPad) + quarter * 32 + lane] = i & 1 ? tot[i / 2].y : tot[i / 2].x;
    if (p.split > 1) cluster_arrive_wait(); else __syncthreads();
    const int m_left = a.M - mt * 128;
    for (int i = tid + rank * kThreads<kBulk>; i < n * 32; i += kThreads<kBulk> * p.split) {
        const int t = i >> 5, m = (i & 31) * 4;
        float v[4];
        const float* from = out + t * (128 + kOutPad) + m;
        if (p.split == 1) {
            *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(from);
        } else {
            v[0] = v[1] = v[2] = v[3] = 0.0f;
            for (int k = 0; k < p.split; ++k) {
                const float4 q = ld_cluster(smem_u32(from), k);
                v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
            }
        }
        const int64_t to = (p0 + t) * a.ld_y + mt * 128 + m;
        if (p.y_vec && m + 4 <= m_left) {
            if (a.y_type == RMSMP_F32) {
                *reinterpret_cast<float4*>(static_cast<float*>(a.y) + to) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                uint32_t w[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (a.y_type == RMSMP_F16) {
                        const __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
                        w[j] = reinterpret_cast<const uint32_t&>(h);
                    } else {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                        w[j] = reinterpret_cast<const uint32_t&>(h);
                    }
                }
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + to) = make_uint2(w[0], w[1]);
            }
        } else {
            for (int j = 0; j < 4 && m + j < m_left; ++j) store_as(a.y, to + j, a.y_type, v[j]);
        }
    }
    if (p.split > 1) cluster_arrive_wait(); else __syncthreads();
    if (!alive) {
        // a wait ran out: what is still under way is given the same time once more
        if (lane == 0 && warp == 0) {
            volatile int again = 0;
            for (int i = 0; i < 2 && units > 0; ++i) {
                const int last = units * sums - 1 - i;
                if (last >= 0) mbar_wait(smem_u32(&s_done[last & 1]), (last >> 1) & 1, &again);
            }
            for (int u = max(0, units - p.ring); u < units && !again; ++u) mbar_wait(smem_u32(&s_full[u % p.ring]), (u / p.ring) & 1, &again);
        }
        for (int i = 0; i < 200; ++i) __nanosleep(1000);            // (copies of x in flight land)
        if (lane == 0) atomicMax(a.status, (uint32_t)RMSMP_ERR_TIMEOUT);
    }
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols) : "memory");
    }
}

template <int kBN, int kX, bool kBulk>
cudaError_t launch_one(Plan& p, cudaStream_t st)
{
    static bool attr_set[kMaxDevices] = {};
    constexpr int kRoom = kGs4MostSmem - 12 * kBN - 768;               // beside the static shared memory
    auto* const kernel = gs4_tensor_kernel<kBN, kX, kBulk>;
    if (!ensure_smem_attr(reinterpret_cast<const void*>(kernel), kRoom, attr_set)) return cudaErrorInvalidValue;
    const size_t fixed = 1024 + 2 * kBytesA + (size_t)kStagesB<kBN, kX> * kBytesB<kBN, kX>, slot = 4 * (size_t)p.a.block_bytes;
    p.ring = (int)std::min<size_t>(std::min<size_t>(16, (kRoom - fixed) / slot), std::max(3, p.units + 2));
    if (p.ring < 3) return cudaErrorInvalidValue;
    const size_t smem = std::max<size_t>(fixed + p.ring * slot, 1024 + (size_t)kBN * (128 + kOutPad) * sizeof(float));
    const int64_t grid = (int64_t)p.mtiles * p.ntiles * p.split;
    if (grid > (1ll << 31) - 1) return cudaErrorInvalidValue;
    if (kBulk) {
        const cuuint64_t dim[2] = {(cuuint64_t)p.a.K, (cuuint64_t)p.a.x_rows}, pitch[1] = {(cuuint64_t)p.a.ld_x * 2};
        const cuuint32_t box[2] = {64, (cuuint32_t)kBN}, step[2] = {1, 1};
        if (tensor_map_encoder()(&p.x_map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(p.a.x), dim, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    if (p.split == 1) return launch_dependent(kernel, (unsigned)grid, kThreads<kBulk>, smem, st, p);
    return launch_dependent_cluster(kernel, p.split, (unsigned)grid, kThreads<kBulk>, smem, st, p);
}
template <int kX>
cudaError_t launch_tokens(Plan& p, int bn, cudaStream_t st)
{
    constexpr bool kHalf = kX != RMSMP_F32;
    // What the copy engine can address: 16-bit rows, one after the other, that start on 16 bytes.
    const bool bulk = kHalf && !p.a.rows && p.a.x_vec && p.a.x_rows > 0 && (uint64_t)p.a.ld_x * 2 < (1ull << 40) && tensor_map_encoder();
    switch (bn) {
        case 16: return bulk ? launch_one<16, kX, kHalf>(p, st) : launch_one<16, kX, false>(p, st);
        case 32: return bulk ? launch_one<32, kX, kHalf>(p, st) : launch_one<32, kX, false>(p, st);
        case 64: return bulk ? launch_one<64, kX, kHalf>(p, st) : launch_one<64, kX, false>(p, st);
        case 128: return bulk ? launch_one<kHalf ? 128 : 64, kX, kHalf>(p, st) : launch_one<kHalf ? 128 : 64, kX, false>(p, st);
        case 192: return bulk ? launch_one<kHalf ? 192 : 64, kX, kHalf>(p, st) : launch_one<kHalf ? 192 : 64, kX, false>(p, st);
        default: return bulk ? launch_one<kHalf ? 256 : 64, kX, kHalf>(p, st) : launch_one<kHalf ? 256 : 64, kX, false>(p, st);
    }
}

}  // namespace

cudaError_t launch_gs4_tensor(const Gs4Args& a, cudaStream_t st)
{
    const Gs4ManyPlan of = gs4_plan_many(sizes_of(a));
    if (of.ntiles > (1 << 30)) return cudaErrorInvalidValue;
    Plan p;
    p.a = a;
    p.split = of.split; p.units = of.units; p.mtiles = of.mtiles; p.ntiles = (int)of.ntiles;
    p.y_vec = (reinterpret_cast<uintptr_t>(a.y) % (4 * dtype_size(a.y_type))) == 0 && a.ld_y % 4 == 0;
    return a.x_type == RMSMP_F16    ? launch_tokens<RMSMP_F16>(p, of.bn, st)
           : a.x_type == RMSMP_BF16 ? launch_tokens<RMSMP_BF16>(p, of.bn, st)
                                    : launch_tokens<RMSMP_F32>(p, of.bn, st);
}

}  // namespace rmsmp
