// What the entry points of the attention block's layers share: argument checks, the context's device, kernel attributes.
#pragma once

#include <atomic>
#include <initializer_list>

#include "common.cuh"

namespace small {

static inline int check_pointers(std::initializer_list<const void *> required, std::initializer_list<const void *> optional = {}) {
    for (const void *p : required) {
        if (!p) return SMALL_ERR_INVALID_ARG;
        if (!aligned16(p)) return SMALL_ERR_ALIGN;
    }
    for (const void *p : optional)
        if (p && !aligned16(p)) return SMALL_ERR_ALIGN;
    return SMALL_OK;
}

static inline bool one_math_mode(unsigned flags) { return (flags & SMALL_MATH_MASK) != SMALL_MATH_MASK; }

// The call runs on the context's device, whichever is current: its tensors live there.  A context that small_init has not filled has none: the rules
// that plan a launch divide by its SMs.
struct OnDevice {
    int before = -1;
    cudaError_t error;
    explicit OnDevice(const small_ctx *ctx) {
        int now = 0;
        error = ctx->sm_count > 0 ? cudaGetDevice(&now) : cudaErrorInvalidDevice;
        if (error == cudaSuccess && now != ctx->device) {
            before = now;
            error = cudaSetDevice(ctx->device);
        }
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
};

// Gives a kernel the device's whole shared memory, once for each device; `done` is that kernel's own (a bit for each device).
template <typename K>
static inline int allow_shared_memory(small_ctx *ctx, K *kern, std::atomic<unsigned long long> &done, size_t bytes) {
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (done.load(std::memory_order_relaxed) & bit) return SMALL_OK;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, 100);       // several blocks a SM where they fit
    if (e != cudaSuccess) { ctx->last_cuda = (int)e; return SMALL_ERR_CUDA; }
    done.fetch_or(bit, std::memory_order_relaxed);
    return SMALL_OK;
}

#ifdef __CUDACC__
// launch_kernel for thread-block clusters of `cluster` blocks along x.
template <typename... KArgs, typename... Args>
static inline void launch_clusters(small_ctx *ctx, void (*kern)(KArgs...), dim3 grid, dim3 block, int cluster, size_t smem, cudaStream_t st, Args &&...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctx->dependent ? 2 : 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
    (void)e;   // picked up by check_launch through cudaGetLastError
}

// The other blocks of a cluster: barrier and a float of block `rank`'s shared memory.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }       // orders no memory
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float cluster_read(const float *p, int rank) {
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(r) : "memory");
    return v;
}

__device__ __forceinline__ void copy16_async(void *smem, const void *global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
#endif

}  // namespace small
