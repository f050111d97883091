// Launches of the expert layer's kernels. Every one is a dependent launch: it starts while the kernel before
// it on the stream still runs (once all of that one's CTAs have started, where it says so), sets up what
// needs no global memory, and then waits for it to finish. That hides a microsecond or so of launch latency
// behind each kernel. And the shared-memory limit of a kernel, set once.
#pragma once

#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>

namespace esp_moe_impl {

namespace {

// In a kernel launched with after_launch_before(): waits until the launch before it has finished and its
// writes are visible. No global memory is touched before.
__device__ __forceinline__ void wait_for_launch_before()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The launch after may start once every CTA has called this or ended.
__device__ __forceinline__ void let_next_launch_start()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

inline cudaLaunchAttribute after_launch_before()
{
    cudaLaunchAttribute a = {};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}

// Launches a kernel that calls wait_for_launch_before().
template <typename... P, typename... A>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1] = {after_launch_before()};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Lets a kernel use up to Most bytes of dynamic shared memory on `device`: the most that any of its launches asks for,
// whatever this one does, so that handles of several threads set the same limit. The default limit counts static
// memory too. Done once per kernel and device (the call takes about a microsecond).
template <auto Kernel, size_t Most>
inline cudaError_t allow_smem(int device)
{
    constexpr int kDevices = 64;
    static std::atomic<bool> done[kDevices];
    if (device < kDevices && done[device].load())
        return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(Kernel),
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Most);
    if (e == cudaSuccess && device < kDevices)
        done[device].store(true);
    return e;
}

}  // namespace

}  // namespace esp_moe_impl
