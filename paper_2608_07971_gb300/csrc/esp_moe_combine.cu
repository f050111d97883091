// The experts' rows back into their tokens (include/esp_moe.h: esp_moe_combine and its gradients): one
// CTA per token, a thread owns V consecutive columns (16 bytes where the rows allow it) of all the
// token's rows, KT of them in flight at once. Bound by HBM: for 8192 tokens x 8 rows of 4096 bf16 the sum
// takes 92 us (604 MB, 6.5 TB/s), both gradients 175 us (1.14 GB, 6.5 TB/s).

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "esp_moe_impl.h"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kMaxThreads = 256;

// A token's rows and weights in shared memory; rows outside [0, M) become -1.
struct Picks {
    int32_t pos[ESP_MOE_MAX_CHOICES];
    float weight[ESP_MOE_MAX_CHOICES];
};

__device__ __forceinline__ void load_picks(const CombineArgs &a, int64_t t, Picks &s)
{
    let_next_launch_start();
    wait_for_launch_before();
    if (threadIdx.x < ESP_MOE_MAX_CHOICES) {
        int32_t p = -1;
        float w = 0.0f;
        if ((int)threadIdx.x < a.k) {
            p = a.pos[t * a.k + threadIdx.x];
            w = a.weight ? a.weight[t * a.k + threadIdx.x] : 1.0f;
        }
        s.pos[threadIdx.x] = p >= 0 && p < a.M ? p : -1;
        s.weight[threadIdx.x] = w;
    }
    __syncthreads();
}

// V elements as loaded, for a load that may be left out (a row that does not exist: zeros).
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_if(bool on, const T *p)
{
    Pack<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i)
        r.v[i] = from_f32<T>(0.0f);
    if (on) {
        if constexpr (sizeof(r) == 16) {
            // read once: evicted first
            const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(p));
            memcpy(&r, &w, 16);
        } else {
            r = *reinterpret_cast<const Pack<T, V> *>(p);
        }
    }
    return r;
}

template <typename T, int V, int KT>
__global__ void __launch_bounds__(kMaxThreads) k_combine(const CombineArgs a)
{
    __shared__ Picks s;
    const int64_t t = blockIdx.x;
    load_picks(a, t, s);
    const T *y = static_cast<const T *>(a.y);
    T *out = static_cast<T *>(a.out) + t * a.ldo;
    for (int h = threadIdx.x * V; h < a.H; h += blockDim.x * V) {
        float acc[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            acc[i] = 0.0f;
        for (int j0 = 0; j0 < a.k; j0 += KT) {
            Pack<T, V> v[KT];
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const int32_t p = s.pos[j0 + j];   // -1 past k
                v[j] = load_if<T, V>(p >= 0, y + p * a.ldy + h);
            }
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const float w = s.weight[j0 + j];
                if (s.pos[j0 + j] >= 0)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        acc[i] = fmaf(w, to_f32(v[j].v[i]), acc[i]);
            }
        }
        store_pack<T, V>(out + h, acc);
    }
}

template <typename T, int V, int KT>
__global__ void __launch_bounds__(kMaxThreads) k_combine_backward(const CombineArgs a)
{
    __shared__ Picks s;
    __shared__ float part[ESP_MOE_MAX_CHOICES][kMaxThreads / 32];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    load_picks(a, t, s);
    const T *y = static_cast<const T *>(a.y), *dout = static_cast<const T *>(a.dout) + t * a.lddo;
    T *dy = static_cast<T *>(a.dy);
    for (int j0 = 0; j0 < a.k; j0 += KT) {
        float dot[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j)
            dot[j] = 0.0f;
        for (int h = threadIdx.x * V; h < a.H; h += blockDim.x * V) {
            float d[V];
            Pack<T, V> v[KT];
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const int32_t p = s.pos[j0 + j];
                v[j] = load_if<T, V>(a.dweight && p >= 0, y + p * a.ldy + h);
            }
            load_pack<T, V>(dout + h, d);
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const int32_t p = s.pos[j0 + j];
                if (p < 0)
                    continue;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    dot[j] = fmaf(d[i], to_f32(v[j].v[i]), dot[j]);
                if (dy) {
                    const float w = s.weight[j0 + j];
                    float g[V];
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        g[i] = w * d[i];
                    store_pack<T, V>(dy + p * a.lddy + h, g);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            float x = dot[j];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                x += __shfl_xor_sync(0xffffffffu, x, o);
            if (lane == 0 && j0 + j < ESP_MOE_MAX_CHOICES)
                part[j0 + j][warp] = x;
        }
    }
    if (!a.dweight)
        return;
    __syncthreads();
    if ((int)threadIdx.x < a.k) {
        float x = 0.0f;
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w)
            x += part[threadIdx.x][w];
        a.dweight[t * a.k + threadIdx.x] = x;
    }
}

// Threads of a CTA: enough for a row, whole warps, at least one.
int threads_for(int64_t H, int V)
{
    return (int)std::min<int64_t>(kMaxThreads, std::max<int64_t>(32, ceil_div(ceil_div(H, V), 32) * 32));
}

// Calls f(V): the widest load, or single elements where not every row allows it.
template <typename T, typename F>
cudaError_t with_load(bool wide, F &&f)
{
    return wide ? f(std::integral_constant<int, 16 / (int)sizeof(T)>()) : f(std::integral_constant<int, 1>());
}

template <typename T, int V, int KT>
cudaError_t start_combine(esp_moe *m, const CombineArgs &a)
{
    m->launches += 1;
    return launch_after(k_combine<T, V, KT>, dim3((unsigned)a.T), threads_for(a.H, V), 0, m->stream, a);
}

}  // namespace

cudaError_t launch_combine(esp_moe *m, int32_t dtype, const CombineArgs &a)
{
    if (a.T == 0 || a.H == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) {
        using T = decltype(elem);
        const bool wide = rows_aligned(a.y, a.ldy, sizeof(T), 16) && rows_aligned(a.out, a.ldo, sizeof(T), 16) &&
                          a.H * sizeof(T) % 16 == 0;
        return with_load<T>(wide, [&](auto v) -> cudaError_t {
            constexpr int V = decltype(v)::value;
            if constexpr (V > 1)   // rows in flight
                if (a.k <= 4)
                    return start_combine<T, V, 4>(m, a);
            return start_combine<T, V, 8>(m, a);
        });
    });
}

cudaError_t launch_combine_backward(esp_moe *m, int32_t dtype, const CombineArgs &a)
{
    if (a.T == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) {
        using T = decltype(elem);
        const bool wide = (!a.dweight || rows_aligned(a.y, a.ldy, sizeof(T), 16)) &&
                          (!a.dy || rows_aligned(a.dy, a.lddy, sizeof(T), 16)) &&
                          rows_aligned(a.dout, a.lddo, sizeof(T), 16) && a.H * sizeof(T) % 16 == 0;
        // four rows in flight: eight take 97 registers and halve the CTAs of an SM (8192 x 8 rows of 4096 bf16:
        // 186 us, 175 with four)
        return with_load<T>(wide, [&](auto v) -> cudaError_t {
            constexpr int V = decltype(v)::value, KT = V > 1 ? 4 : 8;
            m->launches += 1;
            return launch_after(k_combine_backward<T, V, KT>, dim3((unsigned)a.T), threads_for(a.H, V), 0, m->stream, a);
        });
    });
}

}  // namespace esp_moe_impl
