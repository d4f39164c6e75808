// Host side of the group-scaled 4-bit layers and of the operators on tokens sorted by expert: validation, description, dispatch.
#include "gs4.cuh"
#include "nvtx.cuh"

using namespace rmsmp;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;

inline uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
inline bool type_ok(int t) { return t == RMSMP_F32 || t == RMSMP_F16 || t == RMSMP_BF16; }
inline bool aligned(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) == 0; }
inline rmsmp_status done(cudaError_t e)
{
    if (e == cudaSuccess) return RMSMP_OK;
    cudaGetLastError();
    return RMSMP_ERR_CUDA;
}

// Everything that follows from E, M, K, group, mode and scale_type.
void lay_out(rmsmp_gs4_layer* L)
{
    L->Kp = (int32_t)up((uint64_t)L->K, 128);
    L->tiles = (L->M + 31) / 32;
    L->sums = L->group % 128 == 0 ? 1 : L->group % 64 == 0 ? 2 : 4;
    L->block_bytes = kCodeBytes + 64 * L->sums + (L->mode == RMSMP_GS4_ZERO ? 16 * L->sums : 0);
    L->reserved = 0;
    L->off_blocks = 256;
    L->packed_bytes = up(L->off_blocks + (uint64_t)L->E * L->tiles * (L->Kp / 128) * L->block_bytes, 256);
    L->magic = kGs4Magic;
}

bool describable(int E, int M, int K, int group)
{
    constexpr int kMost = 1 << 20;
    return E >= 1 && E <= 4096 && M >= 1 && M <= kMost && K >= 1 && K <= kMost && group >= 32 && group <= kMost && group % 32 == 0;
}

// A descriptor is taken only if it is exactly what rmsmp_gs4_layer_init makes of its sizes: every address follows from it.
bool gs4_ok(const rmsmp_gs4_layer* L)
{
    if (!L || L->magic != kGs4Magic || !describable(L->E, L->M, L->K, L->group)) return false;
    if (L->mode != RMSMP_GS4_SYM && L->mode != RMSMP_GS4_ZERO) return false;
    if (L->scale_type != RMSMP_F16 && L->scale_type != RMSMP_BF16) return false;
    rmsmp_gs4_layer want = *L;
    lay_out(&want);
    return want.Kp == L->Kp && want.tiles == L->tiles && want.sums == L->sums && want.block_bytes == L->block_bytes &&
           want.off_blocks == L->off_blocks && want.packed_bytes == L->packed_bytes;
}

rmsmp_status product(const rmsmp_gs4_layer* L, const void* d_packed, const void* d_x, rmsmp_dtype x_type, int64_t x_rows, int64_t ld_x,
                     const int32_t* d_rows, const int32_t* d_offsets, int64_t R, void* d_y, rmsmp_dtype y_type, int64_t ld_y, bool experts, void* stream)
{
    if (!L || !d_packed || (experts && !d_offsets)) return RMSMP_ERR_NULL;
    if (!gs4_ok(L)) return RMSMP_ERR_BAD_LAYER;
    if (!type_ok(x_type) || !type_ok(y_type)) return RMSMP_ERR_SCHEME;
    if ((!experts && L->E != 1) || R < 0 || R > kMostRows || x_rows < 0 || x_rows > kMostRows || ld_x < L->K || ld_y < L->M) return RMSMP_ERR_SHAPE;
    if ((!d_x && x_rows) || (!d_y && R)) return RMSMP_ERR_NULL;
    if (!aligned(d_packed, 256) || !aligned(d_x, dtype_size(x_type)) || !aligned(d_y, dtype_size(y_type)) || !aligned(d_rows, 4) || !aligned(d_offsets, 4))
        return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK || R == 0) return arch;
    const uint8_t* blob = static_cast<const uint8_t*>(d_packed);
    Gs4Args a = {};
    a.blocks = blob + L->off_blocks; a.block_bytes = L->block_bytes; a.has_zeros = L->mode == RMSMP_GS4_ZERO;
    a.status = reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(blob) + kStatusOffset);
    a.x = x_rows ? d_x : d_packed;               // (no rows: a copy of no bytes still names an address, and that of d_x may be null)
    a.y = d_y; a.rows = d_rows; a.offsets = d_offsets;
    a.x_rows = x_rows; a.ld_x = ld_x; a.ld_y = ld_y; a.R = R;
    a.M = L->M; a.K = L->K; a.Kp = L->Kp; a.tiles = L->tiles; a.E = L->E; a.sums = L->sums;
    a.scale_bf16 = L->scale_type == RMSMP_BF16; a.x_type = x_type; a.y_type = y_type;
    a.x_vec = aligned(d_x, 16) && ld_x * dtype_size(x_type) % 16 == 0;
    a.sms = sm_count();
    const bool many = gs4_many_tokens(R, L->E, x_type, experts);
    return done(many ? launch_gs4_tensor(a, static_cast<cudaStream_t>(stream)) : launch_gs4_product(a, static_cast<cudaStream_t>(stream)));
}

// What the row operators have in common: a type, H columns, and matrices of `rows` rows that are that wide.
struct Matrix { const void* p; int64_t rows, ld; };
template <int n>
rmsmp_status rows_ok(rmsmp_dtype type, int64_t H, const Matrix (&m)[n])
{
    if (!type_ok(type)) return RMSMP_ERR_SCHEME;
    if (H < 1 || H > kMostRows) return RMSMP_ERR_SHAPE;
    for (const Matrix& x : m)
        if (x.rows < 0 || x.rows > kMostRows || x.ld < H) return RMSMP_ERR_SHAPE;
    for (const Matrix& x : m)
        if (!aligned(x.p, dtype_size(type))) return RMSMP_ERR_ALIGN;
    return RMSMP_OK;
}

}  // namespace

extern "C" {

rmsmp_status rmsmp_gs4_layer_init(rmsmp_gs4_layer* L, int E, int M, int K, int group, rmsmp_gs4_mode mode, rmsmp_dtype scale_type)
{
    if (!L) return RMSMP_ERR_NULL;
    if (!describable(E, M, K, group)) return RMSMP_ERR_SHAPE;
    if ((mode != RMSMP_GS4_SYM && mode != RMSMP_GS4_ZERO) || (scale_type != RMSMP_F16 && scale_type != RMSMP_BF16)) return RMSMP_ERR_SCHEME;
    *L = rmsmp_gs4_layer{};
    L->E = E; L->M = M; L->K = K; L->group = group; L->mode = mode; L->scale_type = scale_type;
    lay_out(L);
    return RMSMP_OK;
}

rmsmp_status rmsmp_gs4_quantize_pack(const rmsmp_gs4_layer* L, const void* d_W, rmsmp_dtype w_type, void* d_packed, size_t packed_bytes, void* stream)
{
    NvtxRange nvtx_range("rmsmp_gs4_quantize_pack");
    if (!L || !d_W || !d_packed) return RMSMP_ERR_NULL;
    if (!gs4_ok(L)) return RMSMP_ERR_BAD_LAYER;
    if (!type_ok(w_type)) return RMSMP_ERR_SCHEME;
    if (packed_bytes < L->packed_bytes) return RMSMP_ERR_BUFFER_TOO_SMALL;
    if (!aligned(d_packed, 256) || !aligned(d_W, dtype_size(w_type))) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK) return arch;
    return done(launch_gs4_quantize(*L, d_W, w_type, static_cast<uint8_t*>(d_packed), static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_gs4_pack_codes(const rmsmp_gs4_layer* L, const uint8_t* d_codes, const void* d_scale, const uint8_t* d_zero, void* d_packed,
                                  size_t packed_bytes, void* stream)
{
    NvtxRange nvtx_range("rmsmp_gs4_pack_codes");
    if (!L || !d_codes || !d_scale || !d_packed) return RMSMP_ERR_NULL;
    if (!gs4_ok(L)) return RMSMP_ERR_BAD_LAYER;
    if (L->mode == RMSMP_GS4_ZERO && !d_zero) return RMSMP_ERR_NULL;
    if (packed_bytes < L->packed_bytes) return RMSMP_ERR_BUFFER_TOO_SMALL;
    if (!aligned(d_packed, 256) || !aligned(d_scale, 2)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK) return arch;
    return done(launch_gs4_pack(*L, d_codes, d_scale, d_zero, static_cast<uint8_t*>(d_packed), static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_gs4_unpack(const rmsmp_gs4_layer* L, const void* d_packed, uint8_t* d_codes, void* d_scale, uint8_t* d_zero, void* stream)
{
    NvtxRange nvtx_range("rmsmp_gs4_unpack");
    if (!L || !d_packed || !d_codes) return RMSMP_ERR_NULL;
    if (!gs4_ok(L)) return RMSMP_ERR_BAD_LAYER;
    if (!aligned(d_packed, 256) || !aligned(d_scale, 2)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK) return arch;
    return done(launch_gs4_unpack(*L, static_cast<const uint8_t*>(d_packed), d_codes, d_scale, d_zero, static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_gs4_gemm(const rmsmp_gs4_layer* L, const void* d_packed, const void* d_x, rmsmp_dtype x_type, int64_t N, int64_t ld_x, void* d_y,
                            rmsmp_dtype y_type, int64_t ld_y, void* stream)
{
    NvtxRange nvtx_range("rmsmp_gs4_gemm");
    return product(L, d_packed, d_x, x_type, N, ld_x, nullptr, nullptr, N, d_y, y_type, ld_y, false, stream);
}

rmsmp_status rmsmp_gs4_gemm_experts(const rmsmp_gs4_layer* L, const void* d_packed, const void* d_x, rmsmp_dtype x_type, int64_t x_rows, int64_t ld_x,
                                    const int32_t* d_rows, const int32_t* d_offsets, int64_t R, void* d_y, rmsmp_dtype y_type, int64_t ld_y, void* stream)
{
    NvtxRange nvtx_range("rmsmp_gs4_gemm_experts");
    return product(L, d_packed, d_x, x_type, x_rows, ld_x, d_rows, d_offsets, R, d_y, y_type, ld_y, true, stream);
}

rmsmp_status rmsmp_expert_sort(const int32_t* d_ids, int64_t T, int k, int E, int32_t* d_offsets, int32_t* d_rows, int32_t* d_place, void* stream)
{
    NvtxRange nvtx_range("rmsmp_expert_sort");
    if (!d_offsets || (T && (!d_ids || !d_rows || !d_place))) return RMSMP_ERR_NULL;
    if (T < 0 || T > kMostRows || k < 1 || k > 1024 || E < 1 || E > 1024 || T * k > kMostRows) return RMSMP_ERR_SHAPE;
    if (!aligned(d_ids, 4) || !aligned(d_offsets, 4) || !aligned(d_rows, 4) || !aligned(d_place, 4)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK) return arch;
    return done(launch_expert_sort(d_ids, T * k, k, E, d_offsets, d_rows, d_place, static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_expert_gather(const void* d_x, rmsmp_dtype type, int64_t x_rows, int64_t H, int64_t ld_x, const int32_t* d_rows, int64_t R, void* d_xs,
                                 int64_t ld_xs, void* stream)
{
    NvtxRange nvtx_range("rmsmp_expert_gather");
    if ((x_rows && !d_x) || (R && (!d_rows || !d_xs))) return RMSMP_ERR_NULL;
    const rmsmp_status ok = rows_ok(type, H, {{d_x, x_rows, ld_x}, {d_xs, R, ld_xs}});
    if (ok != RMSMP_OK) return ok;
    if (!aligned(d_rows, 4)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK || R == 0 || x_rows == 0) return arch;
    return done(launch_expert_gather(d_x, dtype_size(type), x_rows, H, ld_x, d_rows, R, d_xs, ld_xs, static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_expert_combine(const void* d_ys, rmsmp_dtype type, int64_t R, int64_t H, int64_t ld_ys, const int32_t* d_place, const float* d_w,
                                  int64_t T, int k, void* d_y, int64_t ld_y, void* stream)
{
    NvtxRange nvtx_range("rmsmp_expert_combine");
    if ((R && !d_ys) || (T && (!d_place || !d_y))) return RMSMP_ERR_NULL;
    const rmsmp_status ok = rows_ok(type, H, {{d_ys, R, ld_ys}, {d_y, T, ld_y}});
    if (ok != RMSMP_OK) return ok;
    if (k < 1 || k > 1024) return RMSMP_ERR_SHAPE;
    if (!aligned(d_place, 4) || !aligned(d_w, 4)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK || T == 0) return arch;
    return done(launch_expert_combine(d_ys, type, R, H, ld_ys, d_place, d_w, T, k, d_y, ld_y, static_cast<cudaStream_t>(stream)));
}

rmsmp_status rmsmp_expert_combine_backward(const void* d_dy, rmsmp_dtype type, int64_t T, int k, int64_t H, int64_t ld_dy, const void* d_ys, int64_t R,
                                           int64_t ld_ys, const int32_t* d_place, const float* d_w, void* d_dys, int64_t ld_dys, float* d_dw, void* stream)
{
    NvtxRange nvtx_range("rmsmp_expert_combine_backward");
    if (T && (!d_dy || !d_place || (R && !d_dys && !d_dw) || (d_dw && R && !d_ys))) return RMSMP_ERR_NULL;      // (no rows: a gradient of none may have no address)
    const rmsmp_status ok = rows_ok(type, H, {{d_dy, T, ld_dy}, {d_ys, R, d_ys ? ld_ys : H}, {d_dys, R, d_dys ? ld_dys : H}});
    if (ok != RMSMP_OK) return ok;
    if (k < 1 || k > 1024) return RMSMP_ERR_SHAPE;
    if (!aligned(d_place, 4) || !aligned(d_w, 4) || !aligned(d_dw, 4)) return RMSMP_ERR_ALIGN;
    const rmsmp_status arch = arch_status();
    if (arch != RMSMP_OK || T == 0 || (!d_dys && !d_dw)) return arch;
    return done(launch_expert_combine_backward(d_dy, type, T, k, H, ld_dy, d_ys, R, ld_ys, d_place, d_w, d_dys, ld_dys, d_dw,
                                               static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
