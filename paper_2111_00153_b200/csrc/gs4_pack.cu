// Packing of 4-bit weights with a scale for every group of inputs (layout: rmsmp.h), from fp32/fp16/bf16 weights or from codes and
// scales that are there already.  Set-up work: one pass for the scales (a warp per row and group: a maximum), one for the codes (a thread
// per word of eight), a few times off that bound (8192 x 8192 bf16 weights: quantize 267 us, from codes 176, unpack 410; their bytes 40, 15 and 15): done once, and kept simple.  Launched the ordinary way and without letting dependents start early, as every
// writer of packed buffers is.
#include <algorithm>
#include "gs4.cuh"

namespace rmsmp {

namespace {

constexpr int kThreads = 256;

struct PackArgs {
    const void* w;               // weights (quantize) or null
    const uint8_t* codes_in;     // codes, scales, zeros (pack)
    const void* scale_in;
    const uint8_t* zero_in;
    uint8_t* blocks;
    int M, K, Kp, tiles, E, group, sums, scale_bf16, w_type, G, block_bytes, has_zeros;
};

// The scales and zero points of rows g, g + 8, g + 16, g + 24 for run number `run` of a row.
struct Quad { uint2* scale; uint16_t* zero; };
__device__ __forceinline__ Quad quad_of(const PackArgs& a, int64_t et, int g, int run)
{
    uint8_t* b = a.blocks + (et * (a.Kp / 128) + run / a.sums) * a.block_bytes + kCodeBytes;
    const int i = g * a.sums + run % a.sums;
    return {reinterpret_cast<uint2*>(b) + i, reinterpret_cast<uint16_t*>(b + 64 * a.sums) + i};
}

__device__ __forceinline__ float warp_max(float v)
{
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// one warp: rows g, g + 8, g + 16, g + 24 of a block, one group
__global__ void __launch_bounds__(kThreads) gs4_scales_kernel(const PackArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t items = (int64_t)a.E * a.tiles * 8 * a.G;
    for (int64_t it = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); it < items; it += (int64_t)gridDim.x * (kThreads / 32)) {
        const int grp = (int)(it % a.G);
        const int g = (int)(it / a.G % 8);
        const int64_t et = it / a.G / 8;
        const int64_t e = et / a.tiles;
        const int m0 = (int)(et % a.tiles) * 32 + g;
        uint32_t s2[4] = {}, z2[4] = {};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int m = m0 + 8 * h;
            if (m >= a.M) continue;
            const int64_t row = e * a.M + m;
            if (!a.w) {
                s2[h] = static_cast<const uint16_t*>(a.scale_in)[row * a.G + grp];
                if (a.has_zeros) z2[h] = a.zero_in[row * a.G + grp] & 15u;
                continue;
            }
            const int k1 = min((int64_t)a.K, ((int64_t)grp + 1) * a.group);
            float lo = 0.0f, hi = 0.0f;
            for (int k = grp * a.group + lane; k < k1; k += 32) {
                const float v = load_as(a.w, row * a.K + k, a.w_type);
                lo = fmaxf(lo, -v);
                hi = fmaxf(hi, v);
            }
            lo = warp_max(lo);
            hi = warp_max(hi);
            const float s = a.has_zeros ? (hi + lo) / 15.0f : fmaxf(hi, lo) / 7.0f;
            float sr;
            if (a.scale_bf16) {
                const __nv_bfloat16 b = __float2bfloat16_rn(fminf(s, 3.3895313892515355e38f));
                s2[h] = __bfloat16_as_ushort(b);
                sr = __bfloat162float(b);
            } else {
                const __half b = __float2half_rn(fminf(s, 65504.0f));
                s2[h] = __half_as_ushort(b);
                sr = __half2float(b);
            }
            if (a.has_zeros && sr > 0.0f) z2[h] = (uint32_t)fminf(fmaxf(rintf(lo / sr), 0.0f), 15.0f);
        }
        const int size = 128 / a.sums;
        const int64_t c1 = min((int64_t)a.Kp, ((int64_t)grp + 1) * a.group) / size;
        for (int64_t c = (int64_t)grp * a.group / size + lane; c < c1; c += 32) {
            const Quad to = quad_of(a, et, g, (int)c);
            *to.scale = make_uint2(s2[0] | s2[1] << 16, s2[2] | s2[3] << 16);
            if (a.has_zeros) *to.zero = (uint16_t)(z2[0] | z2[1] << 4 | z2[2] << 8 | z2[3] << 12);
        }
    }
}

// one thread: a word, rows g and g + 8 x four consecutive inputs (behind gs4_scales_kernel)
__global__ void __launch_bounds__(kThreads) gs4_codes_kernel(const PackArgs a)
{
    const int64_t words = (int64_t)a.E * a.tiles * (a.Kp / 128) * 512;
    for (int64_t it = (int64_t)blockIdx.x * kThreads + threadIdx.x; it < words; it += (int64_t)gridDim.x * kThreads) {
        const int w = (int)(it & 3), lane = (int)(it >> 2) & 31, part = (int)(it >> 7) & 1, half = (int)(it >> 8) & 1;
        const int64_t blk = it >> 9;
        const int kb = (int)(blk % (a.Kp / 128));
        const int64_t et = blk / (a.Kp / 128);
        const int64_t e = et / a.tiles;
        const int m0 = (int)(et % a.tiles) * 32 + half * 16 + (lane >> 2);
        const int k0 = kb * 128 + part * 64 + (w >> 1) * 32 + (lane & 3) * 8 + (w & 1) * 4;
        const Quad of = quad_of(a, et, lane >> 2, k0 / (128 / a.sums));
        const uint32_t pair = half ? of.scale->y : of.scale->x;
        const uint32_t zz = a.has_zeros ? (uint32_t)*of.zero >> (8 * half) : 0x88u;
        uint32_t out = 0;
        for (int h = 0; h < 2; ++h) {
            const int m = m0 + 8 * h;
            const uint32_t z = (zz >> (4 * h)) & 15u;
            const float s = scale_value((pair >> (16 * h)) & 0xffffu, a.scale_bf16);
            for (int i = 0; i < 4; ++i) {
                uint32_t u = z;                                            // beyond the matrix: zero
                if (m < a.M && k0 + i < a.K) {
                    const int64_t at = (e * a.M + m) * a.K + k0 + i;
                    if (!a.w) {
                        u = a.codes_in[at] & 15u;
                    } else if (s > 0.0f) {
                        const float q = rintf(load_as(a.w, at, a.w_type) / s);
                        u = a.has_zeros ? (uint32_t)fminf(fmaxf(q + (float)z, 0.0f), 15.0f) : (uint32_t)(8.0f + fminf(fmaxf(q, -7.0f), 7.0f));
                    }
                }
                out |= u << (4 * ((i >> 1) * 2 + h + 4 * (i & 1)));
            }
        }
        reinterpret_cast<uint32_t*>(a.blocks + blk * a.block_bytes)[it & 511] = out;
    }
}

__global__ void __launch_bounds__(kThreads) gs4_unpack_kernel(const PackArgs a, uint8_t* codes, uint16_t* scale, uint8_t* zero)
{
    const int64_t count = (int64_t)a.E * a.M * a.K;
    for (int64_t it = (int64_t)blockIdx.x * kThreads + threadIdx.x; it < count; it += (int64_t)gridDim.x * kThreads) {
        const int k = (int)(it % a.K);
        const int64_t row = it / a.K;
        const int m = (int)(row % a.M);
        const int64_t et = row / a.M * a.tiles + m / 32;
        const int g = m & 7, h = (m >> 3) & 1, quarter = (m >> 3) & 3, o = k & 31, i = o & 3;
        const uint8_t* block = a.blocks + (et * (a.Kp / 128) + k / 128) * a.block_bytes;
        const int word = ((((m >> 4) & 1) * 2 + ((k >> 6) & 1)) * 32 + g * 4 + (o >> 3)) * 4 + ((k >> 5) & 1) * 2 + ((o >> 2) & 1);
        codes[it] = (uint8_t)(reinterpret_cast<const uint32_t*>(block)[word] >> (4 * ((i >> 1) * 2 + h + 4 * (i & 1))) & 15u);
        if (k % a.group == 0) {
            const Quad of = quad_of(a, et, g, k / (128 / a.sums));
            const int64_t to = row * a.G + k / a.group;
            if (scale) scale[to] = (uint16_t)((quarter & 2 ? of.scale->y : of.scale->x) >> (16 * (quarter & 1)));
            if (zero) zero[to] = a.has_zeros ? (uint8_t)(*of.zero >> (4 * quarter) & 15u) : (uint8_t)8;
        }
    }
}

struct HeaderWords { uint32_t w[8]; };
__global__ void gs4_header_kernel(uint32_t* blob, const HeaderWords h) { blob[threadIdx.x] = h.w[threadIdx.x]; }

PackArgs args_of(const rmsmp_gs4_layer& L, uint8_t* blob)
{
    PackArgs a = {};
    a.blocks = blob + L.off_blocks; a.block_bytes = L.block_bytes; a.has_zeros = L.mode == RMSMP_GS4_ZERO;
    a.M = L.M; a.K = L.K; a.Kp = L.Kp; a.tiles = L.tiles; a.E = L.E; a.group = L.group; a.sums = L.sums;
    a.scale_bf16 = L.scale_type == RMSMP_BF16;
    a.G = (int)(((int64_t)L.K + L.group - 1) / L.group);
    return a;
}

unsigned blocks_for(int64_t items, int per_block)
{
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + per_block - 1) / per_block, (int64_t)sm_count() * 32));
}

cudaError_t launch_all(const rmsmp_gs4_layer& L, const PackArgs& a, uint8_t* blob, cudaStream_t st)
{
    // the header's rest with its status word, and the scales behind a row's last group, are zeros
    const cudaError_t e = cudaMemsetAsync(blob, 0, (size_t)L.packed_bytes, st);
    if (e != cudaSuccess) return e;
    HeaderWords h = {{kGs4Magic, 1u, (uint32_t)L.E, (uint32_t)L.M, (uint32_t)L.K, (uint32_t)L.group, (uint32_t)L.mode, (uint32_t)L.scale_type}};
    gs4_header_kernel<<<1, 8, 0, st>>>(reinterpret_cast<uint32_t*>(blob), h);
    gs4_scales_kernel<<<blocks_for((int64_t)a.E * a.tiles * 8 * a.G, kThreads / 32), kThreads, 0, st>>>(a);
    gs4_codes_kernel<<<blocks_for((int64_t)a.E * a.tiles * (a.Kp / 128) * 512, kThreads), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gs4_quantize(const rmsmp_gs4_layer& L, const void* dW, int w_type, uint8_t* blob, cudaStream_t st)
{
    PackArgs a = args_of(L, blob);
    a.w = dW; a.w_type = w_type;
    return launch_all(L, a, blob, st);
}

cudaError_t launch_gs4_pack(const rmsmp_gs4_layer& L, const uint8_t* codes, const void* scale, const uint8_t* zero, uint8_t* blob, cudaStream_t st)
{
    PackArgs a = args_of(L, blob);
    a.codes_in = codes; a.scale_in = scale; a.zero_in = zero;
    return launch_all(L, a, blob, st);
}

cudaError_t launch_gs4_unpack(const rmsmp_gs4_layer& L, const uint8_t* blob, uint8_t* codes, void* scale, uint8_t* zero, cudaStream_t st)
{
    const PackArgs a = args_of(L, const_cast<uint8_t*>(blob));
    gs4_unpack_kernel<<<blocks_for((int64_t)a.E * a.M * a.K, kThreads), kThreads, 0, st>>>(a, codes, static_cast<uint16_t*>(scale), zero);
    return cudaGetLastError();
}

}  // namespace rmsmp
