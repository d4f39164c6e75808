// Internal declarations of the group-scaled 4-bit layers and of the operators on tokens sorted by expert (not part of the ABI).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"
#include "gs4_plan.h"

namespace rmsmp {

constexpr uint32_t kGs4Magic = 0x47533452u;      // "GS4R"

// The product y[p] = W x[row(p)]; passed by value.
struct Gs4Args {
    const uint8_t* blocks;                       // of 32 rows and 128 inputs: codes, scales, zeros
    const void* x;
    void* y;
    const int32_t *rows, *offsets;               // null: row p itself; one matrix and all R rows
    uint32_t* status;
    int64_t x_rows, ld_x, ld_y, R;
    int M, K, Kp, tiles, E, sums;
    int sms;                                     // of the device
    int block_bytes, has_zeros;                  // (no zeros: 8 everywhere)
    int scale_bf16, x_type, y_type, x_vec;       // x_vec: rows of x are 16-byte aligned
};
inline Gs4Sizes sizes_of(const Gs4Args& a)
{
    return {a.R, a.E, a.tiles, a.Kp, a.sums, a.block_bytes, a.x_type, a.offsets != nullptr, !a.rows, a.x_vec != 0, a.sms};
}

cudaError_t launch_gs4_quantize(const rmsmp_gs4_layer& L, const void* dW, int w_type, uint8_t* blob, cudaStream_t st);
cudaError_t launch_gs4_pack(const rmsmp_gs4_layer& L, const uint8_t* codes, const void* scale, const uint8_t* zero, uint8_t* blob, cudaStream_t st);
cudaError_t launch_gs4_unpack(const rmsmp_gs4_layer& L, const uint8_t* blob, uint8_t* codes, void* scale, uint8_t* zero, cudaStream_t st);
cudaError_t launch_gs4_product(const Gs4Args& a, cudaStream_t st);
cudaError_t launch_gs4_tensor(const Gs4Args& a, cudaStream_t st);

cudaError_t launch_expert_sort(const int32_t* ids, int64_t P, int k, int E, int32_t* offsets, int32_t* rows, int32_t* place, cudaStream_t st);
cudaError_t launch_expert_gather(const void* x, int size, int64_t x_rows, int64_t H, int64_t ld_x, const int32_t* rows, int64_t R, void* xs,
                                 int64_t ld_xs, cudaStream_t st);
cudaError_t launch_expert_combine(const void* ys, int type, int64_t R, int64_t H, int64_t ld_ys, const int32_t* place, const float* w, int64_t T, int k,
                                  void* y, int64_t ld_y, cudaStream_t st);
cudaError_t launch_expert_combine_backward(const void* dy, int type, int64_t T, int k, int64_t H, int64_t ld_dy, const void* ys, int64_t R, int64_t ld_ys,
                                           const int32_t* place, const float* w, void* dys, int64_t ld_dys, float* dw, cudaStream_t st);

constexpr int kCodeBytes = 2048;                  // of a block

__host__ __device__ inline int dtype_size(int t) { return t == RMSMP_F32 ? 4 : 2; }

__device__ __forceinline__ float scale_value(uint32_t bits16, int is_bf16)
{
    return is_bf16 ? __uint_as_float(bits16 << 16) : __half2float(__ushort_as_half((unsigned short)bits16));
}
// One value, rounded once to the type.
__device__ __forceinline__ void store_as(void* p, int64_t i, int type, float v)
{
    if (type == RMSMP_F32) static_cast<float*>(p)[i] = v;
    else if (type == RMSMP_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ float load_as(const void* p, int64_t i, int type)
{
    if (type == RMSMP_F32) return static_cast<const float*>(p)[i];
    if (type == RMSMP_F16) return __half2float(static_cast<const __half*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

}  // namespace rmsmp
