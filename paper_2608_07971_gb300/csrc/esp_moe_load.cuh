// Element types of the expert layer's kernels: loads to fp32 and rounded stores, single and vectors.
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace esp_moe_impl {

namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V elements that move as one load or store (at most 16 bytes), aligned to their size.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
    static_assert(sizeof(T) * V <= 16, "one load");
};

template <typename T, int V>
__device__ __forceinline__ void load_pack(const T *p, float *out)
{
    const Pack<T, V> r = *reinterpret_cast<const Pack<T, V> *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i)
        out[i] = to_f32(r.v[i]);
}

template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const float *in)
{
    Pack<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i)
        r.v[i] = from_f32<T>(in[i]);
    *reinterpret_cast<Pack<T, V> *>(p) = r;
}

}  // namespace

// Host: every row of a matrix starts at a multiple of `bytes`.
inline bool rows_aligned(const void *p, int64_t ld, size_t size, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ((uint64_t)ld * size) % bytes == 0;
}

// Calls f(T()) for the element type of dtype.
template <typename F>
inline cudaError_t with_dtype(int32_t dtype, F &&f)
{
    if (dtype == 0)
        return f(float());
    if (dtype == 1)
        return f(__nv_bfloat16());
    return f(__half());
}

}  // namespace esp_moe_impl
