// y[p] = W x[row(p)] for 4-bit weights with a scale for every group of inputs (gs4 layers, layout in rmsmp.h), few tokens a matrix.
//   y[p][m] = sum_u s[m][u] * (sum_{k in u} (code[m][k] - zero[m][u]) * x[k]),   u: runs of 32, 64 or 128 inputs
// The inner sums are warp-level matrix instructions of 16 rows x 8 columns x 16 inputs on fp16 numbers with fp32 sums: a code becomes its exact
// fp16 integer by five logic operations and four half2 additions for eight codes, and the CUDA cores have no multiply-add of their own but those
// by the scale.  (fp16 whatever the activations' type: in bf16, whose last place is 1 at 128 where fp16's is 1 at 1024, every pair of codes
// needs a shift of its own, 7 logic operations for eight, which go at half rate.)  Columns are tokens; bf16 and fp32
// activations come to fp16 by a power of two for every run and token, an fp32 one as two columns (see stage_x).
// A warp streams blocks of 32 rows x 128 inputs (2 KB of codes) through a ring of its own in shared memory, filled by bulk copies; a CTA's warps are
// `wr` row blocks x `wk` shares of the inputs, each CTA has `per` row blocks, and a cluster of `split` CTAs shares the inputs further where there are
// few rows.  Partial sums meet in shared memory, and across the cluster in distributed shared memory, in a fixed order; no scratch memory, no atomics.
// Weights in turn from more than the L2 holds (ranges: several cards): 8192 x 8192, one bf16 token 12.4 to 13.1 us, eight fp16 tokens 14.6 to 15.9 (34.9 MB: 2.2 to 2.4 TB/s, a
// third of the measured copy), eight bf16 16 to 17.4, one fp32 16, four 17; 65536 x 8192, one token 55 to 59 (4.7 to 5.0 TB/s, 73 to 77 %).  4096 x 4096, one token 5.7 to 6.4;
// 1024 x 1024 3.5 to 4.4.  What bounds them is latency: for eight tokens of 8192 x 8192 an SM issues 1.24 instructions a cycle of four, the tensor pipe is busy for 10 % and
// DRAM for 23 %.  An SM reads 234 KB of its codes, under four fills of its rings, so the start, staging x (all of a CTA's inputs, ahead of its first block: some 3 of the 15 us by the rate in gs4_plan.h) and the join are
// what is measured.  Experts, 64 of 1408 x 2048, 256 pairs: 33 to 36 us, 2.7 to 2.9 TB/s: their CTAs do not fill whole waves.
#include "gs4.cuh"
#include "ptx.cuh"

namespace rmsmp {

namespace {

constexpr int kWarps = kGs4FewWarps, kThreads = kWarps * 32, kRing = kGs4FewRing, kRed = kGs4FewRed;

struct Operands { Gs4Args a; };
struct Plan : Operands, Gs4FewPlan {};

// c = a * b + (kFirst ? 0 : c)
template <bool kFirst>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (kFirst)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// (w & mask) | magic in one instruction; the mask is part of it
template <uint32_t kMask>
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t magic)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "n"(kMask), "r"(magic));
    return d;
}
__device__ __forceinline__ uint32_t constant(uint32_t v)                             // in a register, and kept there
{
    uint32_t r;
    asm volatile("mov.u32 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// Eight codes to four pairs code - zero, exactly.  A code in the low bits of the fp16 number 1024 adds itself to it, four bits further up
// 16 times itself.
struct Expander {
    uint32_t magic = constant(0x64006400u), sixteenth = constant(0x2C002C00u);
    uint32_t lo[2], hi[2];                                                           // 1024 + z and -(64 + z): rows g and g + 8 of each 16
    __device__ __forceinline__ void set(uint32_t word)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            lo[h] = (0x6400u + (word >> (8 * h) & 15u)) * 0x10001u;
            hi[h] = (0xD400u + (word >> (8 * h) & 0xF0u)) * 0x10001u;
        }
    }
    __device__ __forceinline__ void operator()(uint32_t w, int h, uint32_t (&r)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t s = w >> (8 * i);
            asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r[2 * i]) : "r"(and_or<0x000F000Fu>(s, magic)), "r"(lo[h]));
            asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[2 * i + 1]) : "r"(and_or<0x00F000F0u>(s, magic)), "r"(sixteenth), "r"(hi[h]));
        }
    }
};

// Adds a block, 32 rows x 128 inputs, to the sums of the first kUsed of kNT times eight columns.  `codes`, `scales`, `zeros`: this lane's; `x`: this lane's places in the staged activations, at the block's first input; `f`: its columns' factors.
template <int kNT, int kUsed, int kSums, bool kZeros, bool kFactor>
__device__ __forceinline__ void use_block(const uint8_t* codes, const uint8_t* scales, const uint8_t* zeros, Expander& expand, int scale_bf16, const uint8_t* const (&x)[kNT], const float* f, float (&tot)[2][kNT][4])
{
    uint4 q[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) q[h][i] = *reinterpret_cast<const uint4*>(codes + (2 * h + i) * 512);
    float acc[2][kUsed][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int run = b * kSums / 4;
        const bool first = b * kSums % 4 == 0, last = (b + 1) * kSums % 4 == 0;
        if (kZeros && first) expand.set(*reinterpret_cast<const uint16_t*>(zeros + run * 2));
        uint32_t xb[kUsed][4];
#pragma unroll
        for (int t = 0; t < kUsed; ++t) *reinterpret_cast<uint4*>(xb[t]) = *reinterpret_cast<const uint4*>(x[t] + b * 64);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w[2] = {b & 1 ? q[h][b >> 1].z : q[h][b >> 1].x, b & 1 ? q[h][b >> 1].w : q[h][b >> 1].y};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t r[4];
                expand(w[j], h, r);
#pragma unroll
                for (int t = 0; t < kUsed; ++t) {
                    if (first && j == 0) mma16816<true>(acc[h][t], r, xb[t][0], xb[t][1]);
                    else mma16816<false>(acc[h][t], r, xb[t][2 * j], xb[t][2 * j + 1]);
                }
            }
        }
        if (last) {
            const uint2 s4 = *reinterpret_cast<const uint2*>(scales + run * 8);
            const uint32_t pair[2] = {s4.x, s4.y};
            float s[2][2];
            if (scale_bf16) {
#pragma unroll
                for (int h = 0; h < 2; ++h) { s[h][0] = __uint_as_float(pair[h] << 16); s[h][1] = __uint_as_float(pair[h] & 0xffff0000u); }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h][0] = __half2float(__ushort_as_half((unsigned short)(pair[h] & 0xffffu)));
                    s[h][1] = __half2float(__ushort_as_half((unsigned short)(pair[h] >> 16)));
                }
            }
#pragma unroll
            for (int t = 0; t < kUsed; ++t) {
                float2 factor;
                if (kFactor) factor = *reinterpret_cast<const float2*>(f + run * (8 * kNT) + 8 * t);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = kFactor ? acc[h][t][i] * (i & 1 ? factor.y : factor.x) : acc[h][t][i];
                        tot[h][t][i] = __fmaf_rn(s[h][i >> 1], v, tot[h][t][i]);
                    }
            }
        }
    }
}

// 2^e, e in -149..127
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << (e + 149)); }

// Inputs k0 .. k0 + slab of `n` rows of x (-1: zeros) into shared memory, a column of `col_bytes` for each part of each token, and the factors
// ([run][column]).  fp16 goes as it is.  The others are scaled by 2^-e, 2^e <= 2^-14 max|x| < 2^(e+1) over the finite numbers of the run, so that the
// largest is in 2^14..2^15: a bf16 number's 8 bits are then exact down to 2^-31 of that, where fp16's last place has become fixed; what is smaller is off by
// half of that place, 2^-25, at most: 2^-39 of the largest.  An fp32 number is the sum of two fp16 ones, each rounded to nearest.  The first leaves up to
// 2^-11 of it, to a unit of its last place; of 11 bits, the second is off by one such unit at most, 2^-23 of the number.  (A third part would make it
// exact, for half as many columns again.)
template <int kSums, int kX>
__device__ __forceinline__ void stage_x(const Plan& p, uint8_t* xs, float* factors, int columns, uint32_t col_bytes, const int* rows, int n, int k0, int slab)
{
    constexpr int kParts = kX == RMSMP_F32 ? 2 : 1;
    const Gs4Args& a = p.a;
    const int vecs = slab >> 3;
    const int lg = min(32 - __clz(vecs - 1), 31 - __clz(kThreads));             // 2^lg threads a token; 16 vectors a block, so 16 lanes go through this together
    const int v0 = threadIdx.x & ((1 << lg) - 1);
    int t_next = v0 < vecs ? threadIdx.x >> lg : n, v_next = v0;
    constexpr int kAhead = 2;                                 // vectors that a thread has under way (4096 x 4096, eight tokens: 9.1 us, one by one 9.5)
    while (t_next < n) {
        int ts[kAhead], vs[kAhead];
        uint32_t ws[kAhead][4 * kParts];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            ts[q] = t_next; vs[q] = v_next;
#pragma unroll
            for (int j = 0; j < 4 * kParts; ++j) ws[q][j] = 0;
            if (t_next >= n) continue;
            const int row = rows[t_next], k = k0 + v_next * 8;
            const int have = row >= 0 ? min(8, a.K - k) : 0;                    // may be negative
            const int64_t at = row * a.ld_x + k;
            if (have == 8 && a.x_vec) {
#pragma unroll
                for (int j = 0; j < kParts; ++j) *reinterpret_cast<uint4*>(ws[q] + 4 * j) = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.x) + at * (2 * kParts) + 16 * j);
            } else if (kX == RMSMP_F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < have) ws[q][j & (4 * kParts - 1)] = static_cast<const uint32_t*>(a.x)[at + j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < have) ws[q][j >> 1] |= (uint32_t)static_cast<const uint16_t*>(a.x)[at + j] << (16 * (j & 1));
            }
            v_next += 1 << lg;
            if (v_next >= vecs) { v_next = v0; t_next += kThreads >> lg; }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int t = ts[q], v = vs[q];
            if (t >= n) continue;
            const uint32_t (&w)[4 * kParts] = ws[q];
            uint8_t* const dst = xs + (uint32_t)(t * kParts) * col_bytes + v * 16;
            if (kX == RMSMP_F16) {
                *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                continue;
            }
            float f[8];
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[j] = __uint_as_float(kX == RMSMP_F32 ? w[j & (4 * kParts - 1)] : j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
                most = fmaxf(most, fabsf(f[j]));                                // (NaN is passed over)
            }
            if (most == INFINITY) {
                most = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(f[j]) < INFINITY ? fabsf(f[j]) : 0.0f);
            }
            constexpr int kLanes = 16 / kSums;                                  // of a run
            const uint32_t bits = __reduce_max_sync(((1u << kLanes) - 1) << (threadIdx.x & 31 & ~(kLanes - 1)), __float_as_uint(most));
            const int e = max((int)(bits >> 23), 1) - 127 - 14;
            if (e >= -126) {
                const float up = power_of_two(-e);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] *= up;
            } else {                                                            // (2^140 is no fp32 number)
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = f[j] * power_of_two(126) * power_of_two(-e - 126);
            }
            __half2 hi[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) hi[j] = __floats2half2_rn(f[2 * j], f[2 * j + 1]);
            *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(hi);
            if (kParts == 2) {
                __half2 lo[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = fabsf(f[j]) < 65504.0f ? f[j] - (j & 1 ? __high2float(hi[j >> 1]) : __low2float(hi[j >> 1])) : 0.0f;      // (infinities and NaN: nothing)
#pragma unroll
                for (int j = 0; j < 4; ++j) lo[j] = __floats2half2_rn(f[2 * j], f[2 * j + 1]);
                *reinterpret_cast<uint4*>(dst + col_bytes) = *reinterpret_cast<const uint4*>(lo);
            }
            if (v % kLanes == 0) {
                float* const to = factors + v / kLanes * columns + t * kParts;
                to[0] = power_of_two(e);
                if (kParts == 2) to[kParts - 1] = to[0];
            }
        }
    }
}

// `bytes` (a multiple of 16) from global memory; the barrier counts them.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_arrive_wait()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank)
{
    uint32_t r;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(r) : "memory");
    return v;
}

// (At these bounds, 128 registers with sixteen columns and 80 with eight, ptxas spills two words in ten forms: those of fp32 and bf16 with sixteen columns and two or four runs, and with
// eight columns, four runs and no zeros.)
template <int kNT, int kSums, bool kZeros, int kX>
__global__ void __launch_bounds__(kThreads, kNT == 2 ? 2 : 3) gs4_mma_kernel(const __grid_constant__ Plan p)
{
    constexpr int kCols = 8 * kNT, kChunk = gs4_few_chunk(kNT);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kRing];
    __shared__ int s_abort, s_found[3];
    __shared__ int s_passes[kWarps], s_rows[kCols];
    constexpr bool kFactor = kX != RMSMP_F16;
    constexpr int kBlockBytes = kCodeBytes + 64 * kSums + (kZeros ? 16 * kSums : 0);
    const Gs4Args& a = p.a;
    const bool scale_bf16 = a.scale_bf16;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);      // (the same for the whole warp to the compiler too)
    Expander expand;
    expand.set(0x8888u);
    const uint32_t full = smem_u32(s_full[warp]);
    if (lane == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(full + i * 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    }
    if (threadIdx.x == 0) s_abort = 0;
    __syncthreads();
    volatile int* abort_flag = &s_abort;
    bool alive = true;
    if (!a.offsets && p.split == 1 && lane == 0) {
        // The first blocks on their way into the L2, which is where later writes go too: nothing is read ahead of the wait.  (4096 x 4096, one token: 6.0 us
        // against 6.4; not for clusters, 4096 x 4096 for eight 10.2 against 9.2.)
        const int tile = (int)(blockIdx.x % p.groups) * p.per + warp % p.wr, units = p.slab / 128, u0 = units * (warp / p.wr) / p.wk, run = units * (warp / p.wr + 1) / p.wk - u0;
        if (run > 0 && tile < a.tiles)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.blocks + ((uint64_t)tile * ((uint32_t)a.Kp >> 7) + u0) * kBlockBytes),
                         "r"(min(run, kRing * kChunk) * kBlockBytes) : "memory");
    }
    pdl_wait();
    pdl_trigger();
    int block = blockIdx.x;
    asm volatile("" : "+r"(block));                                             // (nothing of the above kept in registers)
    const int rank = block % p.split;
    const int rg = block / p.split % p.groups;
    const int which = block / p.split / p.groups;                          // number of a pass over some expert's weights
    const int wr = warp % p.wr, wk = warp / p.wr;
    const uint32_t units_k = (uint32_t)a.Kp >> 7;                               // blocks of a whole row
    const int slice0 = rank * p.slice, slice1 = min(a.Kp, slice0 + p.slice);
    const int tile0 = rg * p.per, tiles = min(p.per, a.tiles - tile0);          // this CTA's row blocks
    uint8_t* const ring = smem + warp * (kRing * kChunk * kBlockBytes);
    uint8_t* const xs = smem + kWarps * (kRing * kChunk * kBlockBytes);
    const uint8_t *const codes = ring + lane * 16, *const scales = ring + kCodeBytes + (lane >> 2) * (8 * kSums);
    const uint8_t* const zeros = ring + kCodeBytes + 64 * kSums + (lane >> 2) * (2 * kSums);
    const uint32_t col_bytes = (uint32_t)p.slab * 2 + 64;                       // (columns 64 bytes apart modulo 128: a lane group's eight loads touch every bank once)
    float* const factors = reinterpret_cast<float*>(xs + min(kCols, p.tokens * p.parts) * col_bytes);      // [run][column]
    float* const red = factors + (kFactor ? p.slab / 128 * kSums * kCols : 0);                             // [row block][share][column][kRed]

    int64_t p0 = 0, end = a.R, matrix = 0;                                      // rows of y
    if (a.offsets) {
        // pass number `which` of `tokens` rows, counted over the matrices that have rows (there are CTAs for no more than there can be)
        int before = 0;
        for (int e0 = 0; e0 < a.E && before <= which; e0 += kThreads) {
            const int e = e0 + (int)threadIdx.x;
            int lo = 0, hi = 0;
            if (e < a.E) {
                lo = max(a.offsets[e], 0);
                hi = (int)min((int64_t)a.offsets[e + 1], a.R);
            }
            const int passes = hi > lo ? (hi - lo + p.tokens - 1) / p.tokens : 0;
            int at = passes;
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, at, o);
                if (lane >= o) at += v;
            }
            __syncthreads();
            if (lane == 31) s_passes[warp] = at;
            __syncthreads();
            at += before - passes;                                              // this matrix's first
            for (int w = 0; w < kWarps; ++w) {
                if (w < warp) at += s_passes[w];
                before += s_passes[w];
            }
            if (which >= at && which < at + passes) {
                lo += (which - at) * p.tokens;
                s_found[0] = e; s_found[1] = lo; s_found[2] = min(hi, lo + p.tokens);
            }
        }
        __syncthreads();
        if (before <= which) return;                                            // (the whole cluster)
        matrix = s_found[0]; p0 = s_found[1]; end = s_found[2];
    }
    const uint8_t* const blocks = a.blocks + matrix * a.tiles * units_k * kBlockBytes;
    const int mine = tiles > wr ? (tiles - wr + p.wr - 1) / p.wr : 0;           // this warp's
    const bool alone = p.alone;                                                 // a warp has all inputs of its row blocks, in one stage
    int slot = 0;                                                               // of the ring, and the phase that its barrier is in
    uint32_t phase = 0;

    const int n = (int)(end - p0), cols = n * p.parts;
    if ((int)threadIdx.x < n) {
        const int64_t row = a.rows ? a.rows[p0 + threadIdx.x] : p0 + threadIdx.x;
        s_rows[threadIdx.x] = row >= 0 && row < a.x_rows ? (int)row : -1;
    }
    // columns behind the last read the last one's inputs (their sums are dropped)
    const uint8_t* x_lane[kNT];
#pragma unroll
    for (int t = 0; t < kNT; ++t) x_lane[t] = xs + min(8 * t + (lane >> 2), cols - 1) * col_bytes + (lane & 3) * 16;
    for (int s0 = slice0; s0 < slice1 || s0 == slice0; s0 += p.slab) {
        const int units = max(0, min(p.slab, slice1 - s0)) / 128;
        const int u0 = units * wk / p.wk, run = units * (wk + 1) / p.wk - u0;               // this warp's of every row block
        // the block to fetch next, how many of its row are left, and row blocks
        uint32_t next = (uint32_t)(tile0 + wr) * units_k + s0 / 128 + u0;
        const uint32_t jump = (uint32_t)p.wr * units_k - run;
        int left_next = run, rows_next = run > 0 ? mine : 0;
        auto fetch = [&](int to) {
            const int blocks_n = min(left_next, kChunk);
            if (lane == 0) {
                mbar_arrive_expect_tx(full + to * 8, blocks_n * kBlockBytes);
                bulk_load(smem_u32(ring + to * (kChunk * kBlockBytes)), blocks + (uint64_t)next * (uint32_t)kBlockBytes, blocks_n * kBlockBytes, full + to * 8);
            }
            next += blocks_n;
            left_next -= blocks_n;
            if (left_next == 0) { next += jump; left_next = run; --rows_next; }
        };
        for (int d = 0; d < kRing && rows_next > 0 && alive; ++d) fetch((slot + d) % kRing);
        __syncthreads();                                                    // the rows are there; the last stage is read
        stage_x<kSums, kX>(p, xs, factors, kCols, col_bytes, s_rows, n, s0, units * 128);
        __syncthreads();
        float* const first = kNT == 2 && p.single ? reinterpret_cast<float*>(ring) : red + (wr * p.wk + wk) * kCols * kRed;
        float* sums = first + (lane & 3) * 2 * kRed + (lane >> 2);       // of the row block at hand
        for (int r = run > 0 ? mine : 0; r > 0 && alive; --r) {
            const uint8_t* x[kNT];
            float tot[2][kNT][4];
#pragma unroll
            for (int t = 0; t < kNT; ++t) {
                x[t] = x_lane[t] + u0 * 256;
#pragma unroll
                for (int i = 0; i < 4; ++i) tot[0][t][i] = tot[1][t][i] = 0.0f;
            }
            const float* f = factors + u0 * (kSums * kCols) + (lane & 3) * 2;
            for (int left = run; left > 0; left -= kChunk) {
                alive = mbar_wait_step(full + slot * 8, phase, abort_flag);
                if (!alive) break;
                const int at = slot * (kChunk * kBlockBytes);
#pragma unroll
                for (int c = 0; c < kChunk; ++c) {
                    if (c > 0 && c >= left) break;
                    const int o = at + c * kBlockBytes;
                    if (kNT == 1 || cols <= 8) use_block<kNT, 1, kSums, kZeros, kFactor>(codes + o, scales + o, zeros + o, expand, scale_bf16, x, f, tot);
                    else use_block<kNT, kNT, kSums, kZeros, kFactor>(codes + o, scales + o, zeros + o, expand, scale_bf16, x, f, tot);
#pragma unroll
                    for (int t = 0; t < kNT; ++t) x[t] += 256;
                    f += kSums * kCols;
                }
                __syncwarp();
                if (rows_next > 0) fetch(slot);
                if (++slot == kRing) { slot = 0; phase ^= 1; }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < kNT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float* to = sums + (8 * t + (i & 1)) * kRed + 8 * (i >> 1) + 16 * h;
                        if (8 * t + (lane & 3) * 2 + (i & 1) < cols) *to = s0 == slice0 ? tot[h][t][i] : *to + tot[h][t][i];
                    }
            if (alone) {
                // nobody else adds to these rows
                __syncwarp();
                const int m = (tile0 + wr + (mine - r) * p.wr) * 32 + lane;
                for (int t = 0; t < n; ++t) {
                    const float* from = first + t * p.parts * kRed + lane;
                    const float v = p.parts == 2 ? from[0] + from[kRed] : from[0];
                    if (m < a.M) store_as(a.y, (p0 + t) * a.ld_y + m, a.y_type, v);
                }
                __syncwarp();
            } else {
                sums += p.wr * p.wk * kCols * kRed;
            }
        }
        if (run == 0 && s0 == slice0)                                       // no inputs for this warp: its share is zero
            for (int r = 0; r < mine; ++r, sums += p.wr * p.wk * kCols * kRed)
                for (int i = 0; i < kCols; i += 8)
                    for (int j = 0; j < 4; ++j) sums[i * kRed + 8 * j] = sums[(i + 1) * kRed + 8 * j] = 0.0f;
    }
    if (!alone) {
        __syncthreads();
        // 2^lg threads a column of the CTA's rows
        const int rows = tiles * 32, lg = min(32 - __clz(rows - 1), 31 - __clz(kThreads)), step = kThreads >> lg;
        const int r0 = threadIdx.x & ((1 << lg) - 1), t0 = threadIdx.x >> lg;
        const int tile_floats = p.wk * kCols * kRed;
        if (p.split > 1) {
            // the CTA's own sum, over its warps' shares, in place of the first share's
            for (int col = t0; col < cols; col += step)
                for (int r = r0; r < rows; r += 1 << lg) {
                    float* const of = &red[(r >> 5) * tile_floats + col * kRed + (r & 31)];
                    float v = 0.0f;
                    for (int k = 0; k < p.wk; ++k) v += of[k * kCols * kRed];
                    *of = v;
                }
            cluster_arrive_wait();
        }
        const int shares = p.split > 1 ? p.split : p.wk;
        for (int t = t0 * p.split + rank; t < n; t += step * p.split)
            for (int r = r0; r < rows; r += 1 << lg) {
                const int m = tile0 * 32 + r;
                if (m >= a.M) break;
                float v = 0.0f;
                for (int q = 0; q < p.parts; ++q) {
                    const float* from = &red[(r >> 5) * tile_floats + (t * p.parts + q) * kRed + (r & 31)];
                    for (int k = 0; k < shares; ++k) v += p.split > 1 ? ld_cluster(smem_u32(from), k) : from[k * kCols * kRed];
                }
                store_as(a.y, (p0 + t) * a.ld_y + m, a.y_type, v);
            }
        if (p.split > 1) cluster_arrive_wait();                                 // the others have read this CTA's sums
    }
    if (!alive) {
        // a wait ran out: copies that are still under way are given the same time once more
        volatile int again = 0;
        for (int i = 0; i < kRing; ++i) mbar_wait(full + (slot + i) % kRing * 8, slot + i < kRing ? phase : phase ^ 1, &again);
        if (lane == 0) atomicMax(a.status, (uint32_t)RMSMP_ERR_TIMEOUT);
    }
}

template <int kNT, int kSums, bool kZeros, int kX>
cudaError_t launch_one(const Plan& p, cudaStream_t st)
{
    static bool attr_set[kMaxDevices] = {};
    auto* const kernel = gs4_mma_kernel<kNT, kSums, kZeros, kX>;
    if (!ensure_smem_attr(reinterpret_cast<const void*>(kernel), kGs4MostSmem, attr_set)) return cudaErrorInvalidValue;
    if (p.split == 1) return launch_dependent(kernel, (unsigned)p.grid, kThreads, p.smem, st, p);
    return launch_dependent_cluster(kernel, p.split, (unsigned)p.grid, kThreads, p.smem, st, p);
}
template <int kNT, int kSums, bool kZeros>
cudaError_t launch_type(const Plan& p, cudaStream_t st)
{
    return p.a.x_type == RMSMP_F16    ? launch_one<kNT, kSums, kZeros, RMSMP_F16>(p, st)
           : p.a.x_type == RMSMP_BF16 ? launch_one<kNT, kSums, kZeros, RMSMP_BF16>(p, st)
                                      : launch_one<kNT, kSums, kZeros, RMSMP_F32>(p, st);
}
template <int kNT, int kSums>
cudaError_t launch_kind(const Plan& p, cudaStream_t st)
{
    return p.a.has_zeros ? launch_type<kNT, kSums, true>(p, st) : launch_type<kNT, kSums, false>(p, st);
}
template <int kNT>
cudaError_t launch_sums(const Plan& p, cudaStream_t st)
{
    return p.a.sums == 1 ? launch_kind<kNT, 1>(p, st) : p.a.sums == 2 ? launch_kind<kNT, 2>(p, st) : launch_kind<kNT, 4>(p, st);
}

}  // namespace

cudaError_t launch_gs4_product(const Gs4Args& a, cudaStream_t st)
{
    Plan p;
    static_cast<Gs4FewPlan&>(p) = gs4_plan_few(sizes_of(a));
    p.a = a;
    if (p.grid > (1ll << 31) - 1) return cudaErrorInvalidValue;
    return p.nt == 1 ? launch_sums<1>(p, st) : launch_sums<2>(p, st);
}

}  // namespace rmsmp
