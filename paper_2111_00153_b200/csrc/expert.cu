// Operators on tokens sorted by expert: the order (a stable counting sort of the (token, choice) pairs by expert), the rows copied in that
// order, the weighted sum back, and its gradient.  The row operators are bound by memory: every row is read and written once.
#include <algorithm>
#include <atomic>
#include "gs4.cuh"
#include "ptx.cuh"

namespace rmsmp {

namespace {

// ------------------------------------------------------------------ order
// One cluster.  Every warp owns a run of consecutive pairs.  First each warp counts its pairs by expert (lanes of the same expert find
// each other by a match; the lowest adds their number); the counts are summed over warps, over the cluster's CTAs through
// distributed shared memory, and over the experts; then each warp walks its run again and hands out positions in order.  Nothing
// depends on timing: counts have one writer each, and no atomics are used.  A warp reads kAhead times 32 ids at once.  What bounds it is latency: two loads
// of the ids, the counts' way through the cluster and the ordered walk; 65536 pairs of 64 experts 11 us on sixteen CTAs (0.8 MB), two pairs 2.7.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kAhead = 8;

struct SortArgs {
    const int32_t* ids;
    int32_t *offsets, *rows, *place;
    uint32_t P, k;
    int E, ctas;
    int warps;                   // of a CTA that have pairs
    uint32_t per_warp;           // pairs of a warp, a multiple of 32
    int bits;                    // of 0..E
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

// Lanes with the same id, of those below 2^bits.  (A ballot for each bit; the match instruction, which takes any word, kept an SM busy for some 80
// cycles a warp: 65536 pairs of 64 experts 21.8 us with it.)
__device__ __forceinline__ uint32_t same_id(uint32_t id, int bits)
{
    uint32_t same = 0xffffffffu;
    for (int b = 0; b < bits; ++b) {
        const bool one = id >> b & 1u;
        const uint32_t ones = __ballot_sync(0xffffffffu, one);
        same &= one ? ones : ~ones;
    }
    return same;
}

__global__ void __launch_bounds__(kSortThreads) expert_sort_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) uint32_t count[];            // [warp][E], then [E]: the CTA's
    __shared__ uint32_t s_warp[kSortWarps];
    pdl_wait();
    pdl_trigger();
    const int32_t* ids = a.ids;
    uint32_t* total = count + a.warps * a.E;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = a.ctas > 1 ? (int)blockIdx.x : 0;
    const uint32_t first = min(a.P, ((uint32_t)rank * a.warps + warp) * a.per_warp), last = warp < a.warps ? min(a.P, first + a.per_warp) : first;
    uint32_t id[kAhead];
    auto read = [&](uint32_t i0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t i = i0 + 32 * j + lane;
            id[j] = min(i < last ? (uint32_t)ids[i] : 0xffffffffu, (uint32_t)a.E);      // (E: nowhere)
        }
    };
    read(first);                                                 // (kept for the second walk where it is all)
    for (int i = tid; i < a.warps * a.E; i += (int)blockDim.x) count[i] = 0;
    __syncthreads();
    uint32_t* mine = count + warp * a.E;
    for (uint32_t i0 = first; i0 < last; i0 += 32 * kAhead) {
        if (i0 != first) read(i0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + 32 * j >= last) break;
            const uint32_t same = same_id(id[j], a.bits);
            if (id[j] < (uint32_t)a.E && (same & ((1u << lane) - 1)) == 0) mine[id[j]] += __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    // thread e: pairs of expert e in front of each warp of this CTA
    uint32_t all = 0;
    if (tid < a.E) {
        for (int w = 0; w < a.warps; ++w) {
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
    for (int w = 0; w < (int)blockDim.x / 32; ++w) {
        if (w < warp) base += s_warp[w];
        pairs += s_warp[w];
    }
    const uint32_t start = base + run - all;
    if (tid < a.E) {
        for (int w = 0; w < a.warps; ++w) count[w * a.E + tid] += start + before;
        if (rank == 0) a.offsets[tid] = (int32_t)start;
    }
    if (rank == 0 && tid == 0) a.offsets[a.E] = (int32_t)pairs;
    __syncthreads();
    for (uint32_t i0 = first; i0 < last; i0 += 32 * kAhead) {
        if (last - first > 32 * kAhead) read(i0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + 32 * j >= last) break;
            const uint32_t i = i0 + 32 * j + lane;
            const uint32_t same = same_id(id[j], a.bits);
            const uint32_t lower = same & ((1u << lane) - 1);
            const bool kept = id[j] < (uint32_t)a.E;
            uint32_t at = 0;
            if (kept) at = mine[id[j]] + __popc(lower);
            __syncwarp();
            if (kept && lower == 0) mine[id[j]] += __popc(same);
            __syncwarp();
            if (i < last) a.place[i] = kept ? (int32_t)at : -1;
            if (kept) a.rows[at] = (int32_t)(i / a.k);
        }
    }
    for (uint32_t p = pairs + (uint32_t)rank * blockDim.x + tid; p < a.P; p += (uint32_t)a.ctas * blockDim.x) a.rows[p] = -1;
}

// ------------------------------------------------------------------ rows
// Rows whose pieces of 16 bytes are aligned everywhere are read and written in those; others value by value (8192 tokens of two choices, 1001 fp16 columns: gather 24 us
// for 66 MB, combine 35, on another card 27 and 38; 1024 columns 10 and 11).
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

// xs[p] = x[rows[p]].  8192 tokens of eight choices, a tenth without a place, 2048 bf16 columns: 50 us, 273 MB at 5.5 TB/s; x comes from the L2 seven times of eight.
constexpr int kRowsAhead = 4;               // rows that a thread copies at once: their loads wait together
template <typename T>
__global__ void __launch_bounds__(kRowThreads) expert_gather_kernel(const T* x, T* xs, const int32_t* rows, int64_t x_rows, int64_t R, int64_t pieces,
                                                                    int64_t ld_x, int64_t ld_xs, int lanes)
{
    pdl_wait();
    pdl_trigger();
    const int per = kRowThreads / lanes;
    const int c0 = threadIdx.x % lanes;
    for (int64_t p0 = (int64_t)blockIdx.x * per * kRowsAhead + threadIdx.x / lanes; p0 < R; p0 += (int64_t)gridDim.x * per * kRowsAhead) {
        int64_t r[kRowsAhead];
#pragma unroll
        for (int j = 0; j < kRowsAhead; ++j) {
            r[j] = p0 + j * per < R ? rows[p0 + j * per] : -1;
            if (r[j] >= x_rows) r[j] = -1;
        }
        for (int64_t c = c0; c < pieces; c += lanes) {
            T v[kRowsAhead];
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j)
                if (r[j] >= 0) v[j] = x[r[j] * ld_x + c];
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j)
                if (r[j] >= 0) __stcs(xs + (p0 + j * per) * ld_xs + c, v[j]);       // (x stays in the L2, not what is written)
        }
    }
}

// One 16-byte piece (kVec), or a single value, as it lies in memory (kept so until it is used: as fp32, the rows that a thread has under way take twice
// the registers), and its values.
template <int kType, bool kVec> struct Piece {
    static constexpr int kSize = kType == RMSMP_F32 ? 4 : 2;
    static constexpr int kN = kVec ? 16 / kSize : 1, kWords = kVec ? 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* p, int64_t i)      // i: in values
    {
        const uint8_t* at = static_cast<const uint8_t*>(p) + i * kSize;
        if (kVec) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
        else w[0] = kType == RMSMP_F32 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
    }
    __device__ __forceinline__ float value(int j) const
    {
        if (kType == RMSMP_F32) return __uint_as_float(w[kVec ? j : 0]);
        const uint32_t u = w[kVec ? j >> 1 : 0];
        if (kType == RMSMP_BF16) return __uint_as_float(j & 1 ? u & 0xffff0000u : u << 16);
        return __half2float(__ushort_as_half((unsigned short)(j & 1 ? u >> 16 : u & 0xffffu)));
    }
    __device__ static __forceinline__ void store(void* p, int64_t i, const float (&v)[kN])
    {
        if (!kVec) {
            store_as(p, i, kType, v[0]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (kType == RMSMP_F32) {
                    w[j] = __float_as_uint(v[j & (kN - 1)]);
                } else if (kType == RMSMP_F16) {
                    const __half2 h = __floats2half2_rn(v[2 * j & (kN - 1)], v[(2 * j + 1) & (kN - 1)]);
                    w[j] = reinterpret_cast<const uint32_t&>(h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j & (kN - 1)], v[(2 * j + 1) & (kN - 1)]);
                    w[j] = reinterpret_cast<const uint32_t&>(h);
                }
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

// y[t] = sum_j w[t][j] ys[place[t][j]].  `lanes` threads a token, a piece each; kTerms: choices whose rows a thread reads at once.  Bound by memory: 8192 tokens of eight
// choices and 2048 bf16 columns, a tenth without a place: 45 us, 6.1 TB/s, 93 % of the measured copy.  As many blocks an SM as leave each thread the registers for its rows
// (16384 tokens of four choices: 57 us with five, 87 with eight; of two 39 with six, 56 with eight; 4096 of eight, eight rows at once 26 us, four 26, two 28, one 31;
// at these bounds ptxas spills one to six words of the 16-bit forms of one, two and eight).
template <int kType, bool kVec, int kTerms>
__global__ void __launch_bounds__(kRowThreads, kTerms == 8 ? 4 : kTerms == 4 ? 5 : kTerms == 2 ? 6 : 8) expert_combine_kernel(const CombineArgs a)
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
            const int32_t* place = a.place + t * a.k;
            for (int j0 = 0; j0 < a.k; j0 += kTerms, place += kTerms) {
                int p[kTerms];
                P v[kTerms];
#pragma unroll
                for (int j = 0; j < kTerms; ++j) {
                    p[j] = j0 + j < a.k ? place[j] : -1;
                    if (p[j] >= a.R) p[j] = -1;
                }
#pragma unroll
                for (int j = 0; j < kTerms; ++j)
                    if (a.R > 0) v[j].load(a.ys, (int64_t)max(p[j], 0) * a.ld_ys + c);      // (a pair without a place: any row, not used)
#pragma unroll
                for (int j = 0; j < kTerms; ++j)
                    if (p[j] >= 0) {
                        const float w = a.w ? a.w[t * a.k + j0 + j] : 1.0f;
#pragma unroll
                        for (int i = 0; i < P::kN; ++i) sum[i] = __fmaf_rn(w, v[j].value(i), sum[i]);
                    }
            }
            P::store(a.y, t * a.ld_y + c, sum);
        }
    }
}

// dys[place[t][j]] = w[t][j] dy[t], dw[t][j] = <dy[t], ys[place[t][j]]>.  `lanes` threads a token, at most a warp's (kBlock: all of a block's): dy is read once for kTerms
// choices, whose rows are read together; the dot products meet by shuffles, and in shared memory, in a fixed order.  Bound by memory: 4096 tokens of eight
// choices and 2048 bf16 columns 51 us, 5.6 TB/s, 86 % of the measured copy (choices one by one 63 us, two at once 51, four 49).
// (ptxas spills one to six words of the forms in whole pieces with less than a block a token: of one choice, and of two in fp32.)
template <int kType, bool kVec, bool kBlock, int kTerms>
__global__ void __launch_bounds__(kRowThreads, !kVec ? 3 : kTerms >= 4 ? 4 : 6) expert_combine_backward_kernel(const CombineArgs a)
{
    using P = Piece<kType, kVec>;
    __shared__ float s_sum[kTerms][kRowThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int lanes = kBlock ? kRowThreads : a.lanes, per = kRowThreads / lanes, c0 = threadIdx.x % lanes;
    const int64_t step = (int64_t)lanes * P::kN;
    const int64_t rounds = (a.T + per - 1) / per;                // (whole rounds: a warp's shuffles take all its lanes)
    for (int64_t t0 = blockIdx.x; t0 < rounds; t0 += gridDim.x) {
        const int64_t t = t0 * per + threadIdx.x / lanes;
        for (int j0 = 0; j0 < a.k; j0 += kTerms) {
            int p[kTerms];
            float dot[kTerms];
#pragma unroll
            for (int j = 0; j < kTerms; ++j) {
                const bool there = t < a.T && j0 + j < a.k;
                p[j] = there ? a.place[t * a.k + j0 + j] : -1;
                if (p[j] >= a.R) p[j] = -1;
                dot[j] = 0.0f;
            }
            for (int64_t c = (int64_t)c0 * P::kN; c < a.H && t < a.T; c += step) {
                P g, v[kTerms];
                g.load(a.dy, t * a.ld_dy + c);
                if (a.dw) {
#pragma unroll
                    for (int j = 0; j < kTerms; ++j)
                        if (a.R > 0) v[j].load(a.ys, (int64_t)max(p[j], 0) * a.ld_ys + c);
#pragma unroll
                    for (int j = 0; j < kTerms; ++j)
                        if (p[j] >= 0) {
#pragma unroll
                            for (int i = 0; i < P::kN; ++i) dot[j] = __fmaf_rn(g.value(i), v[j].value(i), dot[j]);
                        }
                }
                if (a.dys) {
#pragma unroll
                    for (int j = 0; j < kTerms; ++j)
                        if (p[j] >= 0) {
                            const float w = a.w ? a.w[t * a.k + j0 + j] : 1.0f;
                            float o[P::kN];
#pragma unroll
                            for (int i = 0; i < P::kN; ++i) o[i] = w * g.value(i);
                            P::store(a.dys, (int64_t)p[j] * a.ld_dys + c, o);
                        }
                }
            }
            if (!a.dw) continue;
#pragma unroll
            for (int j = 0; j < kTerms; ++j)
                for (int o = kBlock ? 16 : lanes / 2; o; o >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
            if (kBlock) {
                __syncthreads();
                if ((threadIdx.x & 31) == 0)
#pragma unroll
                    for (int j = 0; j < kTerms; ++j) s_sum[j][threadIdx.x >> 5] = dot[j];
                __syncthreads();
                if (threadIdx.x < kTerms && j0 + (int)threadIdx.x < a.k) {
                    float v = 0.0f;
                    for (int i = 0; i < kRowThreads / 32; ++i) v += s_sum[threadIdx.x][i];
                    a.dw[t * a.k + j0 + threadIdx.x] = v;
                }
            } else if (c0 == 0 && t < a.T) {
#pragma unroll
                for (int j = 0; j < kTerms; ++j)
                    if (j0 + j < a.k) a.dw[t * a.k + j0 + j] = dot[j];
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
    template <int kTerms> static cudaError_t go(const CombineArgs& a, int rows, cudaStream_t st)
    {
        return launch_dependent(expert_combine_kernel<kType, kVec, kTerms>, grid_for(a.T, rows), kRowThreads, 0, st, a);
    }
    static cudaError_t run(CombineArgs a, cudaStream_t st)
    {
        const Shape s = shape_of((a.H + Piece<kType, kVec>::kN - 1) / Piece<kType, kVec>::kN);
        a.lanes = s.lanes;
        return a.k == 1 ? go<1>(a, s.rows, st) : a.k == 2 ? go<2>(a, s.rows, st) : a.k <= 4 ? go<4>(a, s.rows, st) : go<8>(a, s.rows, st);
    }
};
template <int kType, bool kVec> struct Backward {
    template <int kTerms> static cudaError_t go(CombineArgs a, cudaStream_t st)
    {
        // A block a token where rows are wide, or tokens few; else up to a warp.  (Both: 4096 tokens of eight choices, 256 pieces: 50 us and 56, 64 pieces: 24 and 12.5; 300 of
        // two, 64 pieces: 2.8 and 3.7; 1024 of two: 4.4 and 3.8.)
        const int64_t pieces = (a.H + Piece<kType, kVec>::kN - 1) / Piece<kType, kVec>::kN;
        if (pieces >= 128 || (pieces > 32 && a.T < (int64_t)sm_count() * 4))
            return launch_dependent(expert_combine_backward_kernel<kType, kVec, true, kTerms>, grid_for(a.T, 1), kRowThreads, 0, st, a);
        a.lanes = std::min(32, shape_of(pieces).lanes);
        return launch_dependent(expert_combine_backward_kernel<kType, kVec, false, kTerms>, grid_for(a.T, kRowThreads / a.lanes), kRowThreads, 0, st, a);
    }
    static cudaError_t run(CombineArgs a, cudaStream_t st)
    {
        return a.k == 1 ? go<1>(a, st) : a.k == 2 ? go<2>(a, st) : go<4>(a, st);
    }
};

constexpr int kSortSmem = (kSortWarps + 1) * 1024 * (int)sizeof(uint32_t);      // the most that a CTA takes

// CTAs of the largest cluster that the current device places, asked once: a cluster of sixteen is more than every device promises.  (Threads that
// ask at the same time each set the attribute before they use it, and store the same answer.)
int most_sort_ctas()
{
    static std::atomic<int> known[kMaxDevices] = {};
    const int dev = device_ordinal();
    if (dev < 0) return 8;
    int most = known[dev].load(std::memory_order_acquire);
    if (most) return most;
    most = 8;
    if (cudaFuncSetAttribute(expert_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 16; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(16); lc.blockDim = dim3(kSortThreads); lc.dynamicSmemBytes = kSortSmem;
        lc.attrs = at; lc.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, expert_sort_kernel, &lc) == cudaSuccess && clusters > 0) most = 16;
    }
    if (most == 8) cudaGetLastError();
    known[dev].store(most, std::memory_order_release);
    return most;
}

}  // namespace

cudaError_t launch_expert_sort(const int32_t* ids, int64_t P, int k, int E, int32_t* offsets, int32_t* rows, int32_t* place, cudaStream_t st)
{
    static bool attr_set[kMaxDevices] = {};
    if (!ensure_smem_attr(reinterpret_cast<const void*>(expert_sort_kernel), kSortSmem, attr_set)) return cudaErrorInvalidValue;
    SortArgs a = {ids, offsets, rows, place, (uint32_t)P, (uint32_t)k, E, 1, 1, 32, 32 - __builtin_clz((unsigned)E)};
    while (a.ctas < 16 && P > (int64_t)a.ctas * kSortThreads * 2) a.ctas *= 2;
    if (a.ctas > 8) a.ctas = most_sort_ctas();
    a.warps = (int)std::max<uint32_t>(1, std::min<uint32_t>(kSortWarps, (a.P + 32 * a.ctas - 1) / (32 * a.ctas)));
    const uint32_t warps = (uint32_t)(a.ctas * a.warps);
    a.per_warp = std::max(1u, (a.P + warps * 32 - 1) / (warps * 32)) * 32;
    const size_t smem = sizeof(uint32_t) * (a.warps + 1) * (size_t)a.E;
    const int threads = std::max(a.warps, (a.E + 31) / 32) * 32;           // a thread an expert, and the warps that have pairs
    if (a.ctas == 1) return launch_dependent(expert_sort_kernel, 1, threads, smem, st, a);
    return launch_dependent_cluster(expert_sort_kernel, a.ctas, a.ctas, threads, smem, st, a);
}

cudaError_t launch_expert_gather(const void* x, int size, int64_t x_rows, int64_t H, int64_t ld_x, const int32_t* rows, int64_t R, void* xs,
                                 int64_t ld_xs, cudaStream_t st)
{
    if (whole(x, ld_x, size) && whole(xs, ld_xs, size) && H * size % 16 == 0) {
        const int n = 16 / size;
        const Shape s = shape_of(H / n);
        return launch_dependent(expert_gather_kernel<uint4>, grid_for(R, s.rows * kRowsAhead), kRowThreads, 0, st, static_cast<const uint4*>(x), static_cast<uint4*>(xs), rows,
                                x_rows, R, H / n, ld_x / n, ld_xs / n, s.lanes);
    }
    const Shape s = shape_of(H);
    if (size == 4)
        return launch_dependent(expert_gather_kernel<uint32_t>, grid_for(R, s.rows * kRowsAhead), kRowThreads, 0, st, static_cast<const uint32_t*>(x), static_cast<uint32_t*>(xs),
                                rows, x_rows, R, H, ld_x, ld_xs, s.lanes);
    return launch_dependent(expert_gather_kernel<uint16_t>, grid_for(R, s.rows * kRowsAhead), kRowThreads, 0, st, static_cast<const uint16_t*>(x), static_cast<uint16_t*>(xs), rows,
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
