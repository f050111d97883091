// Norm of many gradient tensors together and their clipping (include/esp_moe.h: esp_moe_clip).
//
// norm = |scale| sqrt(sum g^2) over all elements of all tensors; out = g * factor, factor = scale min(1, max_norm / norm)
// (scale where the norm is not finite). Two passes, as the factor needs every element: k_norm reads all, k_scale reads
// again and writes. Bound by HBM. The tensors are cut into chunks of 16-byte groups that the CTAs take in turn; k_scale
// takes them from the last to the first, so that it begins with what k_norm left in L2. k_norm leaves a sum for each of
// its CTAs; every CTA of k_scale adds them up for itself, and loads its first chunk while k_norm still runs. 1.4e9 elements
// (2.8 GB) take 1222 us, three times their bytes at the copy rate 1229; 300,000 elements of 7 tensors 13 to 17 us.
//
// A thread sums the squares of a chunk's groups in fp32 (at most 64 of them), then adds that to its sum in fp64; the
// threads', CTAs' and launches' sums are joined in a fixed order in fp64. Squares of values that fp32 does not hold
// (above 2^60, or all below 2^-50) are summed again in fp64.

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "esp_moe_impl.h"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 256;
constexpr int kCtasPerSm = 4;      // k_norm's, each with many chunks and eight loads of a thread in flight
// k_scale's, with four: more than run at once, so that they end together (1.4e9 elements, 2.8 GB: 1325 us with 8,
// 1246 with 16, 1222 with 32)
constexpr int kScaleCtas = 32, kScaleCtasOfFew = 8;   // few bytes: less often the sum of k_norm's CTAs

constexpr int kFewTensors = 16, kManyTensors = 144;   // tensors of a launch, in its parameters
constexpr int64_t kMostBytes = (int64_t)1 << 44;   // of all tensors; keeps a launch's chunks in int32
constexpr int kGroupsOfMany = 4;                   // the least that a thread has in a chunk where there are many bytes
// besides, a chunk of each tensor is not full, and the last step of a CTA goes past the end
static_assert(kMostBytes / (16 * kThreads * kGroupsOfMany) + 2 * kManyTensors + kScaleCtas * 1024 < ((int64_t)1 << 31), "int32");

struct ClipTensor {
    const void *grad;
    void *out;
    int64_t n;
};

template <int N>
struct ClipArgs {
    ClipTensor t[N];
    int32_t first[N];             // first chunk of each tensor
    uint8_t dtype[N];
    int32_t count, chunks;
};

struct SumArgs {
    const double *partial;        // one for each CTA of k_norm
    int32_t count;
    double max_norm, scale;
    float *norm;
};

// Elements before the first of a tensor in its first 16-byte group.
template <typename T>
__device__ __forceinline__ int lead(const void *p)
{
    return (int)(reinterpret_cast<uintptr_t>(p) % 16) / (int)sizeof(T);
}

template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);

// The tensor whose chunks hold `chunk`.
template <int N>
__device__ __forceinline__ int tensor_of(const ClipArgs<N> &a, int chunk)
{
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Group g of a tensor (groups are aligned in memory; the first and last may hold fewer elements): zeros where it has none.
template <typename T>
__device__ __forceinline__ uint4 load_group(const ClipTensor &t, int64_t g, int skip)
{
    uint4 r = make_uint4(0, 0, 0, 0);
    const int64_t i = g * kPer<T> - skip;   // element
    const T *p = static_cast<const T *>(t.grad) + i;
    if (i >= 0 && i + kPer<T> <= t.n) {
        r = *reinterpret_cast<const uint4 *>(p);
    } else if (i < t.n) {
        T v[kPer<T>];
        memcpy(v, &r, 16);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j)
            if (i + j >= 0 && i + j < t.n)
                v[j] = p[j];
        memcpy(&r, v, 16);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4 &r, float (&f)[kPer<T>])
{
    T v[kPer<T>];
    memcpy(v, &r, 16);
#pragma unroll
    for (int j = 0; j < kPer<T>; ++j)
        f[j] = to_f32(v[j]);
}

// This thread's squares in U groups from g0 + threadIdx.x on, kThreads apart.
template <typename T, int U>
__device__ __forceinline__ double square_chunk(const ClipTensor &t, int64_t g0)
{
    const int skip = lead<T>(t.grad);
    uint4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        r[u] = load_group<T>(t, g0 + u * kThreads + threadIdx.x, skip);
    float s = 0.0f;
    uint32_t bits = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[kPer<T>];
        unpack<T>(r[u], f);
        float q = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j)
            q = fmaf(f[j], f[j], q);
        s += q;
        bits |= r[u].x | r[u].y | r[u].z | r[u].w;
    }
    bits &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    if (s < 0x1p120f && (s > 0x1p-90f || bits == 0))
        return (double)s;
    double d = 0.0;
    for (int u = 0; u < U; ++u) {
        float f[kPer<T>];
        unpack<T>(load_group<T>(t, g0 + u * kThreads + threadIdx.x, skip), f);
        for (int j = 0; j < kPer<T>; ++j)
            d += (double)f[j] * (double)f[j];
    }
    return d;
}

// Sum over the CTA, in thread 0. One warp adds up: an fp64 addition of a warp keeps an SM's fp64 units for about 16
// cycles, so that few of them is what counts.
__device__ __forceinline__ double sum_of_cta(double v, double *all)
{
    all[threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        for (int i = 32; i < kThreads; i += 32)
            v += all[threadIdx.x + i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            v += __shfl_down_sync(0xffffffffu, v, o);
    }
    return v;
}

template <int U, int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_norm(const __grid_constant__ ClipArgs<N> a, double *partial)
{
    __shared__ double all[kThreads];
    wait_for_launch_before();
    let_next_launch_start();
    double sum = 0.0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(a, c);
        const ClipTensor &t = a.t[i];
        const int64_t g0 = (int64_t)(c - a.first[i]) * (U * kThreads);
        sum += a.dtype[i] == ESP_MOE_F32    ? square_chunk<float, U>(t, g0)
               : a.dtype[i] == ESP_MOE_BF16 ? square_chunk<__nv_bfloat16, U>(t, g0)
                                            : square_chunk<__half, U>(t, g0);
    }
    sum = sum_of_cta(sum, all);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = sum;
}

// 2^e of a normal number.
__device__ __forceinline__ double power_of_two(int e)
{
    return __longlong_as_double((long long)(1023 + e) << 52);
}

// This thread's groups of a chunk that is to be written.
template <typename T, int U>
__device__ __forceinline__ void load_chunk(const ClipTensor &t, int64_t g0, uint4 (&r)[U])
{
    if (!t.out)
        return;
    const int skip = lead<T>(t.grad);
#pragma unroll
    for (int u = 0; u < U; ++u)
        r[u] = load_group<T>(t, g0 + u * kThreads + threadIdx.x, skip);
}

// What the gradients are multiplied by. Where fp32 would hold it in fewer bits (a small limit of large gradients), `wide`
// is not 0 and is it.
struct Factor {
    float by;
    double wide;
};

template <typename T, int U>
__device__ __forceinline__ void scale_chunk(const ClipTensor &t, int64_t g0, const Factor &k, const uint4 (&r)[U])
{
    if (!t.out || (k.by == 1.0f && t.out == t.grad))
        return;
    const int skip = lead<T>(t.grad);
    const bool same = lead<T>(t.out) == skip;   // groups of `out` are aligned too
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = (g0 + u * kThreads + threadIdx.x) * kPer<T> - skip;
        if (i >= t.n)
            break;
        T *out = static_cast<T *>(t.out) + i;
        float f[kPer<T>];
        unpack<T>(r[u], f);
        if (k.wide == 0.0) {
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j)
                f[j] *= k.by;
        } else {
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j)
                f[j] = (float)((double)f[j] * k.wide);
        }
        T v[kPer<T>];
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j)
            v[j] = from_f32<T>(f[j]);
        if (same && i >= 0 && i + kPer<T> <= t.n) {
            uint4 w;
            memcpy(&w, v, 16);
            *reinterpret_cast<uint4 *>(out) = w;
        } else {
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j)
                if (i + j >= 0 && i + j < t.n)
                    out[j] = v[j];
        }
    }
}

// Calls f(T()) for a tensor's type.
template <typename F>
__device__ __forceinline__ void by_dtype(uint8_t dtype, F &&f)
{
    if (dtype == ESP_MOE_F32)
        f(float());
    else if (dtype == ESP_MOE_BF16)
        f(__nv_bfloat16());
    else
        f(__half());
}

template <int U, int N>
__global__ void __launch_bounds__(kThreads) k_scale(const __grid_constant__ ClipArgs<N> a, const SumArgs n)
{
    __shared__ double all[kThreads];
    __shared__ Factor factor;
    uint4 r[U];
    int c = a.chunks - 1 - (int)blockIdx.x, i = 0;
    int64_t g0 = 0;
    const auto load = [&] {
        if (c < 0)
            return;
        i = tensor_of(a, c);
        g0 = (int64_t)(c - a.first[i]) * (U * kThreads);
        by_dtype(a.dtype[i], [&](auto elem) { load_chunk<decltype(elem), U>(a.t[i], g0, r); });
    };
    // the launch before is k_norm (or an earlier k_scale, of other tensors), which let this one start after all work before
    // it was done: the gradients are there
    load();
    wait_for_launch_before();
    let_next_launch_start();
    double sum = 0.0;
    for (int j = threadIdx.x; j < n.count; j += kThreads)
        sum += __ldcg(n.partial + j);
    sum = sum_of_cta(sum, all);
    if (threadIdx.x == 0) {
        // sum = m 4^e with m in [1, 4): fp32's reciprocal root of m (2 ulp) and one Newton step in fp64 leave it exact to
        // 2^-40; fp64's own root and division take several microseconds here
        float norm = (float)sum;
        double by = n.scale;
        if (sum > 0.0 && sum < (double)INFINITY) {
            const int e = ((int)(__double_as_longlong(sum) >> 52) - 1023) >> 1;
            const double m = sum * power_of_two(-2 * e);
            double r = (double)rsqrtf((float)m);
            r = r * (1.5 - 0.5 * m * r * r);
            norm = (float)(n.scale * m * r * power_of_two(e));
            if (norm < INFINITY)
                by = fmin(n.scale, n.max_norm * r * power_of_two(-e));
        }
        factor = Factor{(float)by, by < (double)FLT_MIN ? by : 0.0};
        if (blockIdx.x == 0)
            *n.norm = norm;
    }
    __syncthreads();
    const Factor by = factor;
    while (c >= 0) {
        by_dtype(a.dtype[i], [&](auto elem) { scale_chunk<decltype(elem), U>(a.t[i], g0, by, r); });
        c -= gridDim.x;
        load();
    }
}

int size_of(int32_t dtype)
{
    return dtype == ESP_MOE_F32 ? 4 : 2;
}

// Chunks of a tensor, U groups for each of a CTA's threads.
int64_t chunks_of(const esp_moe_tensor &t, int U)
{
    const int size = size_of(t.dtype);
    const int64_t skip = (int64_t)(reinterpret_cast<uintptr_t>(t.grad) % 16) / size;
    return ceil_div(ceil_div(t.n + skip, 16 / size), (int64_t)U * kThreads);
}

bool good_tensor(const esp_moe_tensor &t)
{
    if (t.dtype != ESP_MOE_F32 && t.dtype != ESP_MOE_BF16 && t.dtype != ESP_MOE_F16)
        return false;
    const int size = size_of(t.dtype);
    return t.n >= 0 && t.n <= (int64_t)1 << 40 && (t.n == 0 || t.grad) &&
           reinterpret_cast<uintptr_t>(t.grad) % size == 0 && reinterpret_cast<uintptr_t>(t.out) % size == 0;
}

// Whether some memory is written for one tensor, or for the norm, and read or written for another.
bool overlapping(int32_t count, const esp_moe_tensor *tensors, const float *norm)
{
    struct Range {
        uintptr_t lo, hi;
        bool written;
    };
    std::vector<Range> all;
    all.reserve(2 * (size_t)count + 1);
    const uintptr_t at = reinterpret_cast<uintptr_t>(norm);
    all.push_back(Range{at, at + sizeof(float), true});
    for (int32_t i = 0; i < count; ++i) {
        const esp_moe_tensor &t = tensors[i];
        if (t.n == 0)
            continue;
        const uintptr_t bytes = (uintptr_t)t.n * size_of(t.dtype);
        const uintptr_t g = reinterpret_cast<uintptr_t>(t.grad), o = reinterpret_cast<uintptr_t>(t.out);
        all.push_back(Range{g, g + bytes, g == o});
        if (o && o != g)
            all.push_back(Range{o, o + bytes, true});
    }
    std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.lo < b.lo; });
    // ends of what came before: of all of it, and of what is written
    uintptr_t end = 0, end_written = 0;
    for (const Range &r : all) {
        if (r.lo < end_written || (r.written && r.lo < end))
            return true;
        end = std::max(end, r.hi);
        if (r.written)
            end_written = std::max(end_written, r.hi);
    }
    return false;
}

// U, V: groups in flight of a thread of k_norm and of k_scale. N: tensors of a launch.
template <int U, int V, int N>
cudaError_t launch_clip(esp_moe *m, int32_t count, const esp_moe_tensor *tensors, double *partial, SumArgs n)
{
    const int most = kCtasPerSm * m->sm_count;
    ClipArgs<N> a;
    for (int pass = 0; pass < 2; ++pass) {
        int32_t at = 0;
        for (bool more = true; more;) {
            a.count = a.chunks = 0;
            for (; at < count && a.count < N; ++at) {
                const esp_moe_tensor &t = tensors[at];
                const int64_t chunks = t.n == 0 || (pass == 1 && !t.out) ? 0 : chunks_of(t, pass == 0 ? U : V);
                if (chunks == 0)
                    continue;
                a.t[a.count] = ClipTensor{t.grad, t.out, t.n};
                a.first[a.count] = a.chunks;
                a.dtype[a.count] = (uint8_t)t.dtype;
                a.chunks += (int32_t)chunks;
                a.count += 1;
            }
            more = at < count;
            if (pass == 0 && a.chunks == 0)
                continue;
            // k_scale writes the norm too, so that one of it runs even where there is nothing to write
            const int grid = std::max(1, std::min(pass == 0 ? most : (U == 8 ? kScaleCtas : kScaleCtasOfFew) * m->sm_count, a.chunks));
            n.partial = partial;
            m->launches += 1;
            const cudaError_t e =
                pass == 0 ? launch_after(k_norm<U, N>, dim3(grid), kThreads, 0, m->stream, a, partial + n.count)
                          : launch_after(k_scale<V, N>, dim3(grid), kThreads, 0, m->stream, a, n);
            if (e != cudaSuccess)
                return e;
            if (pass == 0)
                n.count += grid;
        }
    }
    return cudaSuccess;
}

}  // namespace

}  // namespace esp_moe_impl

using namespace esp_moe_impl;

extern "C" esp_status esp_moe_clip(esp_moe *m, int32_t count, const esp_moe_tensor *tensors, double max_norm, double scale,
                                   float *norm)
{
    esp_status st = begin_call(m);
    if (st != ESP_OK)
        return st;
    if (count < 0 || (count > 0 && !tensors) || !norm || reinterpret_cast<uintptr_t>(norm) % sizeof(float) != 0 ||
        !(max_norm > 0.0) || !(scale > 0.0) || !std::isnormal((float)scale))
        return ESP_ERR_INVALID_ARG;
    int64_t bytes = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!good_tensor(tensors[i]))
            return ESP_ERR_INVALID_ARG;
        bytes += tensors[i].n * size_of(tensors[i].dtype);
        if (bytes > kMostBytes)
            return ESP_ERR_INVALID_ARG;
    }
    try {
        if (overlapping(count, tensors, norm))
            return ESP_ERR_INVALID_ARG;
    } catch (const std::bad_alloc &) {
        return ESP_ERR_OOM;
    }
    SumArgs n{};
    double *partial = nullptr;
    const size_t launches = (size_t)count / kManyTensors + 1;
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        partial = c.take<double>((size_t)kCtasPerSm * m->sm_count * launches);
        if (pass == 0 && (st = reserve_space(m, c.used())) != ESP_OK)
            return st;
    }
    n.max_norm = max_norm;
    n.scale = scale;
    n.norm = norm;
    // eight loads of a thread in flight where every CTA of k_norm has such a chunk, else fewer and more CTAs
    const int64_t chunk = (int64_t)kThreads * 16, ctas = (int64_t)m->sm_count * kCtasPerSm;
    const auto launch = [&](auto tensors_per_launch) {
        constexpr int N = decltype(tensors_per_launch)::value;
        return bytes >= 16 * ctas * chunk   ? launch_clip<8, kGroupsOfMany, N>(m, count, tensors, partial, n)
               : bytes >= 2 * ctas * chunk ? launch_clip<4, 4, N>(m, count, tensors, partial, n)
                                           : launch_clip<2, 2, N>(m, count, tensors, partial, n);
    };
    const cudaError_t e = count <= kFewTensors ? launch(std::integral_constant<int, kFewTensors>())
                                               : launch(std::integral_constant<int, kManyTensors>());
    return e == cudaSuccess ? ESP_OK : fail_call(m);
}
