// Operators on tokens sorted by expert: the order (a stable counting sort of the (token, choice) pairs by expert), the rows copied in that
// order, the weighted sum back, and its gradient.  The row operators are bound by memory: every row is read and written once.
#include <algorithm>
#include "gs4.cuh"
#include "ptx.cuh"

namespace rmsmp {

namespace {

// ------------------------------------------------------------------ order
// One cluster.  Every warp owns a run of consecutive pairs.  First each warp counts its pairs by expert (lanes of the same expert find
// each other by a match; the lowest adds their number); the counts are summed over warps, over the cluster's CTAs through
// distributed shared memory, and over the experts; then each warp walks its run again and hands out positions in order.  Nothing
// depends on timing: counts have one writer each, and no atomics are used.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

struct SortArgs {
    const int32_t* ids;
    int32_t *offsets, *rows, *place;
    int64_t P;
    int k, E, ctas;
    int per_warp;                // pairs of a warp, a multiple of 32
};

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr, int rank)
{
    uint32_t r, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
    return v;
}

__global__ void __launch_bounds__(kSortThreads) expert_sort_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) uint32_t count[];            // [warp][E], then [E]: the CTA's
    __shared__ uint32_t s_warp[kSortWarps];
    pdl_wait();
    pdl_trigger();
    const int32_t* ids = a.ids;
    uint32_t* total = count + kSortWarps * a.E;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = a.ctas > 1 ? (int)blockIdx.x : 0;
    for (int i = tid; i < kSortWarps * a.E; i += kSortThreads) count[i] = 0;
    __syncthreads();
    const int64_t first = ((int64_t)rank * kSortWarps + warp) * a.per_warp, last = min(a.P, first + a.per_warp);
    uint32_t* mine = count + warp * a.E;
    for (int64_t i0 = first; i0 < last; i0 += 32) {
        const int64_t i = i0 + lane;
        const uint32_t id = i < last ? (uint32_t)ids[i] : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, id);
        if (id < (uint32_t)a.E && (same & ((1u << lane) - 1)) == 0) mine[id] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    // thread e: pairs of expert e in front of each warp of this CTA
    uint32_t all = 0;
    if (tid < a.E) {
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t n = count[w * a.E + tid];
            count[w * a.E + tid] = all;
            all += n;
        }
        total[tid] = all;
    }
    uint32_t before = 0;
    if (a.ctas > 1) {
        cluster_sync();
        all = 0;
        if (tid < a.E)
            for (int r = 0; r < a.ctas; ++r) {
                const uint32_t n = ld_cluster_u32(smem_u32(total + tid), r);
                if (r < rank) before += n;
                all += n;
            }
        cluster_sync();
    }
    // exclusive sums over the experts
    uint32_t run = all;
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t n = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += n;
    }
    if (lane == 31) s_warp[warp] = run;
    __syncthreads();
    uint32_t base = 0, pairs = 0;
    for (int w = 0; w < kSortWarps; ++w) {
        if (w < warp) base += s_warp[w];
        pairs += s_warp[w];
    }
    const uint32_t start = base + run - all;
    if (tid < a.E) {
        for (int w = 0; w < kSortWarps; ++w) count[w * a.E + tid] += start + before;
        if (rank == 0) a.offsets[tid] = (int32_t)start;
    }
    if (rank == 0 && tid == 0) a.offsets[a.E] = (int32_t)pairs;
    __syncthreads();
    for (int64_t i0 = first; i0 < last; i0 += 32) {
        const int64_t i = i0 + lane;
        const uint32_t id = i < last ? (uint32_t)ids[i] : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, id);
        const uint32_t lower = same & ((1u << lane) - 1);
        const bool kept = id < (uint32_t)a.E;
        uint32_t at = 0;
        if (kept) at = mine[id] + __popc(lower);
        __syncwarp();
        if (kept && lower == 0) mine[id] += __popc(same);
        __syncwarp();
        if (i < last) a.place[i] = kept ? (int32_t)at : -1;
        if (kept) a.rows[at] = (int32_t)(i / a.k);
    }
    for (int64_t p = pairs + (int64_t)rank * kSortThreads + tid; p < a.P; p += (int64_t)a.ctas * kSortThreads) a.rows[p] = -1;
}

// ------------------------------------------------------------------ rows
constexpr int kRowThreads = 256;

// Rows are cut into pieces of kBytes; a block's threads are `rows` rows x `lanes` pieces.
struct Shape { int lanes, rows; };
Shape shape_of(int64_t pieces)
{
    int lanes = 1;
    while (lanes < kRowThreads && lanes < pieces) lanes *= 2;
    return {lanes, kRowThreads / lanes};
}
bool whole(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0; }

template <typename T>
__global__ void __launch_bounds__(kRowThreads) expert_gather_kernel(const T* x, T* xs, const int32_t* rows, int64_t x_rows, int64_t R, int64_t pieces,
                                                                    int64_t ld_x, int64_t ld_xs, int lanes)
{
    pdl_wait();
    pdl_trigger();
    const int per = kRowThreads / lanes;
    const int c0 = threadIdx.x % lanes;
    for (int64_t p = (int64_t)blockIdx.x * per + threadIdx.x / lanes; p < R; p += (int64_t)gridDim.x * per) {
        const int64_t r = rows[p];
        if (r < 0 || r >= x_rows) continue;
        for (int64_t c = c0; c < pieces; c += lanes) xs[p * ld_xs + c] = x[r * ld_x + c];
    }
}

// Values of one 16-byte piece (kVec), or a single value.
template <int kType, bool kVec> struct Piece {
    static constexpr int kSize = kType == RMSMP_F32 ? 4 : 2;
    static constexpr int kN = kVec ? 16 / kSize : 1;
    __device__ static void load(const void* p, int64_t i, float (&v)[kN])      // i: in values
    {
        if (!kVec) {
            v[0] = load_as(p, i, kType);
        } else {
            const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p) + i * kSize);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                if (kType == RMSMP_F32) v[j] = __uint_as_float(w[j]);
                else v[j] = scale_value((w[j >> 1] >> (16 * (j & 1))) & 0xffffu, kType == RMSMP_BF16);
            }
        }
    }
    __device__ static void store(void* p, int64_t i, const float (&v)[kN])
    {
        if (!kVec) {
            store_as(p, i, kType, v[0]);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                if (kType == RMSMP_F32) w[j] = __float_as_uint(v[j]);
                else w[j >> 1] |= (uint32_t)(kType == RMSMP_F16 ? __half_as_ushort(__float2half_rn(v[j])) : __bfloat16_as_ushort(__float2bfloat16_rn(v[j]))) << (16 * (j & 1));
            }
            *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p) + i * kSize) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

struct CombineArgs {
    const void *ys, *dy;
    void *y, *dys;
    const int32_t* place;
    const float* w;
    float* dw;
    int64_t R, T, H, ld_ys, ld_y, ld_dy, ld_dys;
    int k, lanes;
};

template <int kType, bool kVec>
__global__ void __launch_bounds__(kRowThreads) expert_combine_kernel(const CombineArgs a)
{
    using P = Piece<kType, kVec>;
    pdl_wait();
    pdl_trigger();
    const int per = kRowThreads / a.lanes;
    const int64_t step = (int64_t)a.lanes * P::kN;
    for (int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / a.lanes; t < a.T; t += (int64_t)gridDim.x * per) {
        for (int64_t c = (int64_t)(threadIdx.x % a.lanes) * P::kN; c < a.H; c += step) {
            float sum[P::kN];
#pragma unroll
            for (int i = 0; i < P::kN; ++i) sum[i] = 0.0f;
            for (int j = 0; j < a.k; ++j) {
                const int64_t p = a.place[t * a.k + j];
                if (p < 0 || p >= a.R) continue;
                const float w = a.w ? a.w[t * a.k + j] : 1.0f;
                float v[P::kN];
                P::load(a.ys, p * a.ld_ys + c, v);
#pragma unroll
                for (int i = 0; i < P::kN; ++i) sum[i] = __fmaf_rn(w, v[i], sum[i]);
            }
            P::store(a.y, t * a.ld_y + c, sum);
        }
    }
}

// a block: one pair (token, choice)
template <int kType, bool kVec>
__global__ void __launch_bounds__(kRowThreads) expert_combine_backward_kernel(const CombineArgs a)
{
    using P = Piece<kType, kVec>;
    __shared__ float s_sum[kRowThreads / 32];
    pdl_wait();
    pdl_trigger();
    for (int64_t i = blockIdx.x; i < a.T * a.k; i += gridDim.x) {
        const int64_t t = i / a.k, p = a.place[i];
        const bool kept = p >= 0 && p < a.R;
        float dot = 0.0f;
        if (kept) {
            const float w = a.w ? a.w[i] : 1.0f;
            for (int64_t c = (int64_t)threadIdx.x * P::kN; c < a.H; c += kRowThreads * P::kN) {
                float g[P::kN], v[P::kN];
                P::load(a.dy, t * a.ld_dy + c, g);
                if (a.dw) {
                    P::load(a.ys, p * a.ld_ys + c, v);
#pragma unroll
                    for (int j = 0; j < P::kN; ++j) dot = __fmaf_rn(g[j], v[j], dot);
                }
                if (a.dys) {
#pragma unroll
                    for (int j = 0; j < P::kN; ++j) v[j] = w * g[j];
                    P::store(a.dys, p * a.ld_dys + c, v);
                }
            }
        }
        if (a.dw) {
            for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
            __syncthreads();
            if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = dot;
            __syncthreads();
            if (threadIdx.x == 0) {
                float v = 0.0f;
                for (int j = 0; j < kRowThreads / 32; ++j) v += s_sum[j];
                a.dw[i] = v;
            }
        }
    }
}

unsigned grid_for(int64_t items, int per) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + per - 1) / per, (int64_t)sm_count() * 16)); }

template <template <int, bool> class F, typename... A>
cudaError_t by_type(int type, bool vec, A... args)
{
    if (vec) return type == RMSMP_F32 ? F<RMSMP_F32, true>::run(args...) : type == RMSMP_F16 ? F<RMSMP_F16, true>::run(args...) : F<RMSMP_BF16, true>::run(args...);
    return type == RMSMP_F32 ? F<RMSMP_F32, false>::run(args...) : type == RMSMP_F16 ? F<RMSMP_F16, false>::run(args...) : F<RMSMP_BF16, false>::run(args...);
}
template <int kType, bool kVec> struct Combine {
    static cudaError_t run(CombineArgs a, cudaStream_t st)
    {
        const Shape s = shape_of((a.H + Piece<kType, kVec>::kN - 1) / Piece<kType, kVec>::kN);
        a.lanes = s.lanes;
        return launch_dependent(expert_combine_kernel<kType, kVec>, grid_for(a.T, s.rows), kRowThreads, 0, st, a);
    }
};
template <int kType, bool kVec> struct Backward {
    static cudaError_t run(CombineArgs a, cudaStream_t st)
    {
        return launch_dependent(expert_combine_backward_kernel<kType, kVec>, grid_for(a.T * a.k, 1), kRowThreads, 0, st, a);
    }
};

}  // namespace

cudaError_t launch_expert_sort(const int32_t* ids, int64_t P, int k, int E, int32_t* offsets, int32_t* rows, int32_t* place, cudaStream_t st)
{
    static bool attr_set[kMaxDevices] = {};
    SortArgs a = {ids, offsets, rows, place, P, k, E, 1, 0};
    while (a.ctas < 8 && P > (int64_t)a.ctas * kSortThreads * 2) a.ctas *= 2;
    const int64_t warps = (int64_t)a.ctas * kSortWarps;
    a.per_warp = (int)(((P + warps - 1) / warps + 31) / 32 * 32);
    const size_t smem = sizeof(uint32_t) * (kSortWarps + 1) * (size_t)E;
    if (!ensure_smem_attr(reinterpret_cast<const void*>(expert_sort_kernel), (kSortWarps + 1) * 1024 * 4, attr_set)) return cudaErrorInvalidValue;
    if (a.ctas == 1) return launch_dependent(expert_sort_kernel, 1, kSortThreads, smem, st, a);
    return launch_dependent_cluster(expert_sort_kernel, a.ctas, a.ctas, kSortThreads, smem, st, a);
}

cudaError_t launch_expert_gather(const void* x, int size, int64_t x_rows, int64_t H, int64_t ld_x, const int32_t* rows, int64_t R, void* xs,
                                 int64_t ld_xs, cudaStream_t st)
{
    if (whole(x, ld_x, size) && whole(xs, ld_xs, size) && H * size % 16 == 0) {
        const int n = 16 / size;
        const Shape s = shape_of(H / n);
        return launch_dependent(expert_gather_kernel<uint4>, grid_for(R, s.rows), kRowThreads, 0, st, static_cast<const uint4*>(x), static_cast<uint4*>(xs), rows,
                                x_rows, R, H / n, ld_x / n, ld_xs / n, s.lanes);
    }
    const Shape s = shape_of(H);
    if (size == 4)
        return launch_dependent(expert_gather_kernel<uint32_t>, grid_for(R, s.rows), kRowThreads, 0, st, static_cast<const uint32_t*>(x), static_cast<uint32_t*>(xs),
                                rows, x_rows, R, H, ld_x, ld_xs, s.lanes);
    return launch_dependent(expert_gather_kernel<uint16_t>, grid_for(R, s.rows), kRowThreads, 0, st, static_cast<const uint16_t*>(x), static_cast<uint16_t*>(xs), rows,
                            x_rows, R, H, ld_x, ld_xs, s.lanes);
}

cudaError_t launch_expert_combine(const void* ys, int type, int64_t R, int64_t H, int64_t ld_ys, const int32_t* place, const float* w, int64_t T, int k,
                                  void* y, int64_t ld_y, cudaStream_t st)
{
    CombineArgs a = {};
    a.ys = ys; a.y = y; a.place = place; a.w = w; a.R = R; a.T = T; a.H = H; a.ld_ys = ld_ys; a.ld_y = ld_y; a.k = k;
    const int size = dtype_size(type);
    return by_type<Combine>(type, whole(ys, ld_ys, size) && whole(y, ld_y, size) && H * size % 16 == 0, a, st);
}

cudaError_t launch_expert_combine_backward(const void* dy, int type, int64_t T, int k, int64_t H, int64_t ld_dy, const void* ys, int64_t R, int64_t ld_ys,
                                           const int32_t* place, const float* w, void* dys, int64_t ld_dys, float* dw, cudaStream_t st)
{
    CombineArgs a = {};
    a.dy = dy; a.ys = ys; a.dys = dys; a.dw = dw; a.place = place; a.w = w;
    a.R = R; a.T = T; a.H = H; a.ld_dy = ld_dy; a.ld_ys = ld_ys; a.ld_dys = ld_dys; a.k = k;
    const int size = dtype_size(type);
    return by_type<Backward>(type, whole(dy, ld_dy, size) && (!dw || whole(ys, ld_ys, size)) && (!dys || whole(dys, ld_dys, size)) && H * size % 16 == 0, a, st);
}

}  // namespace rmsmp
