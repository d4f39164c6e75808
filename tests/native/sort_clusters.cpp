// Stands in for the CUDA runtime under expert.cu, to see which clusters its sort asks for: prints the launches that were refused, those of
// sixteen CTAs and those of eight.  Argument: what the device does with clusters of sixteen.
//   slow     places them once an attribute call, which takes a while, has returned; four threads sort for the first time
//   never    refuses the attribute; three sorts, one after the other
//   no_room  takes the attribute and has no room for them; three sorts
#include <atomic>
#include <chrono>
#include <cstdio>
#include <cstring>
#include <thread>
#include <vector>
#include <cuda_runtime_api.h>

namespace {
const char* device_does = "";
std::atomic<bool> allowed{false};
std::atomic<int> refused{0}, sixteen{0}, eight{0};
void wait_ms(int ms) { std::this_thread::sleep_for(std::chrono::milliseconds(ms)); }
bool placed() { return allowed && std::strcmp(device_does, "slow") == 0; }
}  // namespace

namespace rmsmp {
int device_ordinal() { return 0; }
int sm_count() { return 148; }
bool ensure_smem_attr(const void*, int, bool*) { return true; }
cudaError_t launch_expert_sort(const int32_t* ids, int64_t P, int k, int E, int32_t* offsets, int32_t* rows, int32_t* place, cudaStream_t st);
}  // namespace rmsmp

extern "C" {
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute what, int)
{
    if (what != cudaFuncAttributeNonPortableClusterSizeAllowed) return cudaSuccess;
    if (std::strcmp(device_does, "never") == 0) return cudaErrorNotSupported;
    wait_ms(200);
    allowed = true;
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int* clusters, const void*, const cudaLaunchConfig_t*)
{
    *clusters = placed() ? 9 : 0;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* config, const void*, void**)
{
    unsigned cluster = 1;
    for (unsigned i = 0; i < config->numAttrs; ++i)
        if (config->attrs[i].id == cudaLaunchAttributeClusterDimension) cluster = config->attrs[i].val.clusterDim.x;
    if (cluster > 8 && !placed()) {
        ++refused;
        return cudaErrorLaunchOutOfResources;
    }
    ++(cluster == 16 ? sixteen : eight);
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
char __cudaInitModule(void**) { return 0; }
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
}

int main(int, char** argv)
{
    device_does = argv[1];
    static int32_t words[1];                                     // (nothing is run: no address is looked at)
    auto sort = []() {
        if (rmsmp::launch_expert_sort(words, 65536, 8, 64, words, words, words, nullptr) != cudaSuccess) std::printf("failed ");
    };
    if (std::strcmp(device_does, "slow") == 0) {
        std::vector<std::thread> threads;
        for (int i = 0; i < 4; ++i) {
            threads.emplace_back(sort);
            wait_ms(20);
        }
        for (auto& t : threads) t.join();
    } else {
        for (int i = 0; i < 3; ++i) sort();
    }
    std::printf("%d %d %d\n", refused.load(), sixteen.load(), eight.load());
    return 0;
}
