// Launches of the expert layer's kernels. Every one is a dependent launch: it starts while the kernel before
// it on the stream still runs (once all of that one's CTAs have started, where it says so), sets up what
// needs no global memory, and then waits for it to finish. That hides a microsecond or so of launch latency
// behind each kernel. And the shared-memory limit of a kernel, raised once.
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

// Lets a kernel use `bytes` of dynamic shared memory on `device` (the call takes about a microsecond, so the
// largest amount allowed so far is kept per kernel and device).
template <auto Kernel>
inline cudaError_t allow_smem(size_t bytes, int device)
{
    constexpr int kDevices = 64;
    static std::atomic<size_t> allowed[kDevices];
    if (bytes <= 48 * 1024 || (device < kDevices && allowed[device].load() >= bytes))
        return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && device < kDevices)
        allowed[device].store(bytes);
    return e;
}

}  // namespace

}  // namespace esp_moe_impl
