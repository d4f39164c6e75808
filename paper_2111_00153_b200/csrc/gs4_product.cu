// y[p] = W x[row(p)] for 4-bit weights with a scale for every group of inputs (gs4 layers, layout in rmsmp.h), few tokens a matrix.
//   y[p][m] = sum_u s[m][u] * (sum_{k in u} (code[m][k] - zero[m][u]) * x[k]),   u: runs of 32, 64 or 128 inputs
// The inner sums are warp-level matrix instructions of 16 rows x 8 columns x 16 inputs: a code is turned into its exact fp16 or bf16 integer by
// two or three logic operations and one subtraction for two codes, and no multiply-add is left for the CUDA cores but the one by the
// scale, 4 for 16 x 8 x (32..128).  (One multiply-add and one conversion for each code would take 3 instructions a code; at the rate at which
// memory delivers codes an SM has 2.7.)  Columns are tokens.  An fp32 token takes three: its bf16 parts, cut off 8 bits at a time, add up to it exactly.
// A warp streams blocks of 16 rows x 128 inputs (1 KB of codes, one 16-byte load a lane and 64 inputs, all of a warp's next to each
// other) kDepth blocks ahead in registers; a CTA's warps are `wr` row blocks x `wk` shares of the inputs, and a cluster of `split` CTAs shares the inputs
// further where there are few rows.  Partial sums meet in shared memory, and across the cluster in distributed shared memory, in
// a fixed order; no scratch memory, no atomics.
#include <algorithm>
#include "gs4.cuh"
#include "ptx.cuh"

namespace rmsmp {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kDepth = 4;
constexpr int kRed = 20;                 // floats between columns of a warp's 16-row partial sums (16, padded against bank conflicts)

struct Plan {
    Gs4Args a;
    int wr, wk, split;                   // row blocks x input shares of a CTA's warps; CTAs of a cluster
    int slice, slab;                     // inputs of a CTA, and of one stage of x in shared memory (multiples of 128)
    int groups;                          // groups of wr row blocks
    int tokens;                          // tokens of one pass over the weights
    int parts;                           // columns of a token
};

template <bool kBf>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (kBf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What is subtracted from the codes of rows g and g + 8 (see expand).
struct Zeros { uint32_t lo, hi; };
template <bool kBf>
__device__ __forceinline__ Zeros zeros_of(uint32_t byte)
{
    const uint32_t zl = byte & 15u, zh = byte >> 4 & 15u;
    if (kBf) return {(0x4300u + zl) * 0x10001u, (0x4300u + zh) * 0x10001u};          // 128 + z
    return {(0x6400u + zl) * 0x10001u, (0xD400u + (zh << 4)) * 0x10001u};            // 1024 + z; -(64 + z)
}
// Eight codes to four pairs code - zero, exactly.  A code in the low bits of the fp16 number 1024 adds itself to it, four bits further up
// 16 times itself; in bf16, whose last place is 1 at 128, it has to be in the low bits.
template <bool kBf>
__device__ __forceinline__ void expand(uint32_t w, const Zeros& z, uint32_t (&r)[4])
{
    if (kBf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
            const uint32_t zz = i & 1 ? z.hi : z.lo;
            __nv_bfloat162 d = __hsub2(reinterpret_cast<__nv_bfloat162&>(v), reinterpret_cast<const __nv_bfloat162&>(zz));
            r[i] = reinterpret_cast<uint32_t&>(d);
        }
    } else {
        const uint32_t sixteenth = 0x2C002C00u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t s = w >> (8 * i);
            uint32_t lo = (s & 0x000F000Fu) | 0x64006400u, hi = (s & 0x00F000F0u) | 0x64006400u;
            __half2 a = __hsub2(reinterpret_cast<__half2&>(lo), reinterpret_cast<const __half2&>(z.lo));
            __half2 b = __hfma2(reinterpret_cast<__half2&>(hi), reinterpret_cast<const __half2&>(sixteenth), reinterpret_cast<const __half2&>(z.hi));
            r[2 * i] = reinterpret_cast<uint32_t&>(a);
            r[2 * i + 1] = reinterpret_cast<uint32_t&>(b);
        }
    }
}

// 16 rows x 128 inputs as one lane holds them.
template <int kSums>
struct Unit {
    uint4 q[2];
    uint32_t s[kSums];
    uint32_t z;              // a byte a sum
};
template <int kSums>
__device__ __forceinline__ void load_unit(Unit<kSums>& u, const Gs4Args& a, int64_t block, int lane)
{
    const uint4* q = reinterpret_cast<const uint4*>(a.codes) + block * 64 + lane;
    u.q[0] = __ldg(q);
    u.q[1] = __ldg(q + 32);
    const int64_t at = block * 8 + (lane >> 2);
    if (kSums == 1) {
        u.s[0] = __ldg(reinterpret_cast<const uint32_t*>(a.scales) + at);
        if (a.zeros) u.z = __ldg(a.zeros + at);
    } else if (kSums == 2) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(a.scales) + at);
        u.s[0] = v.x; u.s[kSums - 1] = v.y;
        if (a.zeros) u.z = __ldg(reinterpret_cast<const uint16_t*>(a.zeros) + at);
    } else {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(a.scales) + at);
        u.s[0] = v.x; u.s[kSums / 4] = v.y; u.s[kSums / 2] = v.z; u.s[kSums - 1] = v.w;
        if (a.zeros) u.z = __ldg(reinterpret_cast<const uint32_t*>(a.zeros) + at);
    }
}

// `x`: this lane's place in the staged activations, at the unit's first input.
template <bool kBf, int kNT, int kSums>
__device__ __forceinline__ void use_unit(const Unit<kSums>& u, const Gs4Args& a, uint32_t x, uint32_t col_bytes, float (&tot)[kNT][4])
{
    float acc[kNT][4];
    Zeros z = zeros_of<kBf>(0x88u);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int sum = b * kSums / 4;
        if (b * kSums % 4 == 0) {
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] = 0.0f;
            if (a.zeros) z = zeros_of<kBf>(u.z >> (8 * sum));
        }
        uint32_t xb[kNT][4];
#pragma unroll
        for (int t = 0; t < kNT; ++t)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(xb[t][0]), "=r"(xb[t][1]), "=r"(xb[t][2]), "=r"(xb[t][3])
                         : "r"(x + t * 8 * col_bytes + b * 64));
        const uint4& q = u.q[b >> 1];
        const uint32_t w[2] = {b & 1 ? q.z : q.x, b & 1 ? q.w : q.y};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t r[4];
            expand<kBf>(w[j], z, r);
#pragma unroll
            for (int t = 0; t < kNT; ++t) mma16816<kBf>(acc[t], r[0], r[1], r[2], r[3], xb[t][2 * j], xb[t][2 * j + 1]);
        }
        if ((b + 1) * kSums % 4 == 0) {
            const float s0 = scale_value(u.s[sum] & 0xffffu, a.scale_bf16), s1 = scale_value(u.s[sum] >> 16, a.scale_bf16);
#pragma unroll
            for (int t = 0; t < kNT; ++t) {
                tot[t][0] = __fmaf_rn(s0, acc[t][0], tot[t][0]);
                tot[t][1] = __fmaf_rn(s0, acc[t][1], tot[t][1]);
                tot[t][2] = __fmaf_rn(s1, acc[t][2], tot[t][2]);
                tot[t][3] = __fmaf_rn(s1, acc[t][3], tot[t][3]);
            }
        }
    }
}

// The three bf16 numbers, eight significant bits each, that add up to an fp32 number.  Cut off, not rounded: no part overflows.
__device__ __forceinline__ void split3(float v, uint32_t (&h)[3])
{
    const uint32_t b = __float_as_uint(v);
    h[0] = b >> 16;
    const float hi = __uint_as_float(b & 0xffff0000u);
    const bool finite = (b & 0x7f800000u) != 0x7f800000u;
    if (!finite && (b & 0x7fffffu)) h[0] |= 0x40u;               // (a NaN whose bits are all in the lower half)
    const float r1 = finite ? v - hi : 0.0f;
    h[1] = __float_as_uint(r1) >> 16;
    const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
    h[2] = __float_as_uint(r2) >> 16;
}

// Inputs k0 .. k0 + slab of `n` rows of x, from row p0 on, into shared memory: a column of `col_bytes` for each part of each token.
__device__ __forceinline__ void stage_x(const Plan& p, uint8_t* xs, uint32_t col_bytes, int64_t p0, int n, int k0, int slab)
{
    const Gs4Args& a = p.a;
    const int vecs = slab >> 3;
    for (int i = threadIdx.x; i < n * vecs; i += kThreads) {
        const int t = i / vecs, v = i - t * vecs, k = k0 + v * 8;
        int64_t row = p0 + t;
        if (a.rows) row = a.rows[row];
        const int have = row < 0 || row >= a.x_rows ? 0 : min(8, a.K - k);     // may be negative
        uint8_t* dst = xs + (uint32_t)t * p.parts * col_bytes + v * 16;
        if (a.x_type != RMSMP_F32) {
            const uint16_t* src = static_cast<const uint16_t*>(a.x) + row * a.ld_x + k;
            uint32_t o[4] = {0, 0, 0, 0};
            if (have == 8 && a.x_vec) {
                *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(src);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < have) o[j >> 1] |= (uint32_t)src[j] << (16 * (j & 1));
            }
            *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
            const float* src = static_cast<const float*>(a.x) + row * a.ld_x + k;
            float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (have == 8 && a.x_vec) {
                *reinterpret_cast<float4*>(f) = *reinterpret_cast<const float4*>(src);
                *reinterpret_cast<float4*>(f + 4) = *reinterpret_cast<const float4*>(src + 4);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < have) f[j] = src[j];
            }
            uint32_t o[3][4] = {};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t h[3];
                split3(f[j], h);
                for (int q = 0; q < 3; ++q) o[q][j >> 1] |= h[q] << (16 * (j & 1));
            }
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(dst + q * col_bytes) = make_uint4(o[q][0], o[q][1], o[q][2], o[q][3]);
        }
    }
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

template <bool kBf, int kNT, int kSums>
__global__ void __launch_bounds__(kThreads, 2) gs4_mma_kernel(const __grid_constant__ Plan p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_wait();
    pdl_trigger();
    constexpr int kCols = 8 * kNT;
    Gs4Args a = p.a;
    a.codes = pdl_ordered(a.codes); a.scales = pdl_ordered(a.scales); a.zeros = pdl_ordered(a.zeros);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t col_bytes = (uint32_t)p.slab * 2 + 64;                       // (columns 64 bytes apart modulo 128: a lane group's eight loads touch every bank once)
    float* red = reinterpret_cast<float*>(smem + kCols * col_bytes);            // [warp][column][kRed]

    const int rank = blockIdx.x % p.split;
    const int rg = blockIdx.x / p.split % p.groups;
    const int which = blockIdx.x / p.split / p.groups;                          // expert, or piece of the rows of y
    int64_t begin, end;
    int64_t matrix = 0;
    if (a.offsets) {
        matrix = which;
        begin = min(max((int64_t)a.offsets[which], (int64_t)0), a.R);
        end = min((int64_t)a.offsets[which + 1], a.R);
    } else {
        begin = (int64_t)which * p.tokens;
        end = min(begin + p.tokens, a.R);
    }
    const int wr = warp % p.wr, wk = warp / p.wr;
    const int tile = rg * p.wr + wr;
    const int units_k = a.Kp >> 7;                                              // of a whole row
    const int64_t block0 = (matrix * a.tiles + min(tile, a.tiles - 1)) * units_k;
    const int slice0 = rank * p.slice, slice1 = min(a.Kp, slice0 + p.slice);
    const uint32_t x_lane = smem_u32(smem) + (lane >> 2) * col_bytes + (lane & 3) * 16;

    for (int64_t p0 = begin; p0 < end; p0 += p.tokens) {
        const int n = (int)min((int64_t)p.tokens, end - p0);
        float tot[kNT][4];
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[t][i] = 0.0f;
        for (int s0 = slice0; s0 < slice1; s0 += p.slab) {
            const int slab = min(p.slab, slice1 - s0);
            const int count = tile < a.tiles ? (slab / 128 - wk + p.wk - 1) / p.wk : 0;         // this warp's units
            const int64_t first = block0 + s0 / 128 + wk;
            Unit<kSums> u[kDepth];
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                u[d].z = 0;
                if (d < count) load_unit(u[d], a, first + (int64_t)d * p.wk, lane);
            }
            __syncthreads();                                                    // the last stage, and the last tokens' sums, are read
            stage_x(p, smem, col_bytes, p0, n, s0, slab);
            __syncthreads();
            for (int i = 0; i < count; i += kDepth) {
#pragma unroll
                for (int d = 0; d < kDepth; ++d)
                    if (i + d < count) {
                        use_unit<kBf, kNT, kSums>(u[d], a, x_lane + (uint32_t)((i + d) * p.wk + wk) * 256, col_bytes, tot);
                        if (i + d + kDepth < count) load_unit(u[d], a, first + (int64_t)(i + d + kDepth) * p.wk, lane);
                    }
            }
        }
        float* mine = red + warp * kCols * kRed;
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(8 * t + (lane & 3) * 2 + (i & 1)) * kRed + (lane >> 2) + 8 * (i >> 1)] = tot[t][i];
        __syncthreads();
        if (p.split > 1) {
            // the CTA's own sum, over its warps' shares, in place of the first share's
            for (int i = threadIdx.x; i < p.wr * 16 * n * p.parts; i += kThreads) {
                const int r = i & 15, tile_of = (i >> 4) % p.wr, col = (i >> 4) / p.wr;
                float v = 0.0f;
                for (int k = 0; k < p.wk; ++k) v += red[((k * p.wr + tile_of) * kCols + col) * kRed + r];
                red[(tile_of * kCols + col) * kRed + r] = v;
            }
            cluster_arrive_wait();
        }
        const int shares = p.split > 1 ? p.split : p.wk;
        for (int i = threadIdx.x + rank * kThreads; i < p.wr * 16 * n; i += kThreads * p.split) {
            const int r = i & 15, tile_of = (i >> 4) % p.wr, t = (i >> 4) / p.wr;
            const int m = (rg * p.wr + tile_of) * 16 + r;
            float v = 0.0f;
            for (int q = 0; q < p.parts; ++q) {
                const int col = t * p.parts + q;
                for (int k = 0; k < shares; ++k)
                    v += p.split > 1 ? ld_cluster(smem_u32(&red[(tile_of * kCols + col) * kRed + r]), k)
                                     : red[((k * p.wr + tile_of) * kCols + col) * kRed + r];
            }
            if (m < a.M) store_as(a.y, (p0 + t) * a.ld_y + m, a.y_type, v);
        }
        if (p.split > 1) cluster_arrive_wait();                                 // the others have read this CTA's sums
    }
}

template <bool kBf, int kNT, int kSums>
cudaError_t launch_one(const Plan& p, int64_t grid, size_t smem, cudaStream_t st)
{
    static bool attr_set[kMaxDevices] = {};
    if (!ensure_smem_attr(reinterpret_cast<const void*>(gs4_mma_kernel<kBf, kNT, kSums>), 227 * 1024, attr_set)) return cudaErrorInvalidValue;
    if (p.split == 1) return launch_dependent(gs4_mma_kernel<kBf, kNT, kSums>, (unsigned)grid, kThreads, smem, st, p);
    return launch_dependent_cluster(gs4_mma_kernel<kBf, kNT, kSums>, p.split, (unsigned)grid, kThreads, smem, st, p);
}
template <bool kBf, int kNT>
cudaError_t launch_sums(const Plan& p, int64_t grid, size_t smem, cudaStream_t st)
{
    return p.a.sums == 1 ? launch_one<kBf, kNT, 1>(p, grid, smem, st) : p.a.sums == 2 ? launch_one<kBf, kNT, 2>(p, grid, smem, st) : launch_one<kBf, kNT, 4>(p, grid, smem, st);
}
template <bool kBf>
cudaError_t launch_columns(const Plan& p, int nt, int64_t grid, size_t smem, cudaStream_t st)
{
    return nt == 1 ? launch_sums<kBf, 1>(p, grid, smem, st) : nt == 2 ? launch_sums<kBf, 2>(p, grid, smem, st) : launch_sums<kBf, 4>(p, grid, smem, st);
}

}  // namespace

cudaError_t launch_gs4_product(const Gs4Args& a, cudaStream_t st)
{
    Plan p;
    p.a = a;
    p.parts = a.x_type == RMSMP_F32 ? 3 : 1;
    const int64_t expect = a.offsets ? std::max<int64_t>(1, (a.R + a.E - 1) / a.E) : a.R;      // tokens of a matrix
    const int nt = expect * p.parts <= 8 ? 1 : expect * p.parts <= 16 ? 2 : 4;
    p.tokens = 8 * nt / p.parts;
    const int64_t many = a.offsets ? a.E : (a.R + p.tokens - 1) / p.tokens;
    p.wr = 1;
    while (p.wr < kWarps && a.tiles * many / (p.wr * 2) >= 2 * sm_count()) p.wr *= 2;
    p.wk = kWarps / p.wr;
    p.groups = (a.tiles + p.wr - 1) / p.wr;
    p.split = 1;
    while (p.split < 8 && p.groups * many * p.split * 2 <= 2 * sm_count() && a.Kp / 128 >= p.wk * p.split * 2) p.split *= 2;
    p.slice = (a.Kp / 128 + p.split - 1) / p.split * 128;
    const int most = (96 * 1024 / (8 * nt) - 64) / 2 / 128 * 128;
    p.slab = std::min(p.slice, most);
    const size_t smem = (size_t)8 * nt * (p.slab * 2 + 64) + (size_t)kWarps * 8 * nt * kRed * sizeof(float);
    const int64_t grid = many * p.groups * p.split;
    if (grid > (1ll << 31) - 1) return cudaErrorInvalidValue;
    return a.x_type == RMSMP_F16 ? launch_columns<false>(p, nt, grid, smem, st) : launch_columns<true>(p, nt, grid, smem, st);
}

}  // namespace rmsmp
