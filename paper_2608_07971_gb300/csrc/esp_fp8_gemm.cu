// Products of 8-bit codes with a scale per block of 128 (include/esp_moe.h): each block's products are
// summed in fp32, scaled and added to the result.

#include <algorithm>

#include <cuda_fp8.h>

#include "esp_moe_impl.h"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kTile = 64, kStep = 32, kGemmThreads = 256;

__device__ __forceinline__ float code_value(uint8_t c)
{
    const __half_raw h = __nv_cvt_fp8_to_halfraw(c, __NV_E4M3);
    return __half2float(__half(h));
}

// acc[4][4] += the block's products of A rows a0.. and B rows b0.. (columns k0 .. k0 + 127 below K).
__device__ void block_product(const uint8_t *A, int64_t lda, int rows_a, const uint8_t *B, int64_t ldb, int rows_b,
                              int klen, float (&sa)[kTile][kStep + 1], float (&sb)[kTile][kStep + 1],
                              float (&acc)[4][4])
{
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int ks = 0; ks < klen; ks += kStep) {
        __syncthreads();
        for (int i = threadIdx.x; i < kTile * kStep; i += kGemmThreads) {
            const int r = i / kStep, k = ks + i % kStep;
            sa[r][i % kStep] = r < rows_a && k < klen ? code_value(A[r * lda + k]) : 0.0f;
            sb[r][i % kStep] = r < rows_b && k < klen ? code_value(B[r * ldb + k]) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < kStep; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(sa[ty * 4 + i][k], sb[tx * 4 + j][k], acc[i][j]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kGemmThreads) k_gemm_rows(const GemmRowsArgs a)
{
    __shared__ float sa[kTile][kStep + 1], sb[kTile][kStep + 1];
    int64_t base = 0, m0 = 0;
    int rows = 0, e = 0;
    for (; e < a.E; ++e) {
        const int64_t lo = a.offsets ? max((int64_t)0, min(a.M, (int64_t)a.offsets[e])) : 0;
        const int64_t hi = a.offsets ? max(lo, min(a.M, (int64_t)a.offsets[e + 1])) : a.M;
        const int64_t tiles = (hi - lo + kTile - 1) / kTile;
        if (blockIdx.x < base + tiles) {
            m0 = lo + (blockIdx.x - base) * kTile;
            rows = (int)min((int64_t)kTile, hi - m0);
            break;
        }
        base += tiles;
    }
    if (e == a.E)
        return;
    const int n0 = blockIdx.y * kTile, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float out[4][4] = {};
    for (int kb = 0; kb * kBlock < a.K; ++kb) {
        float acc[4][4] = {};
        block_product(a.A + m0 * a.lda + kb * kBlock, a.lda, rows, a.B + ((int64_t)e * a.N + n0) * a.ldb + kb * kBlock,
                      a.ldb, min(kTile, a.N - n0), min(kBlock, a.K - kb * kBlock), sa, sb, acc);
        const float s_b = a.scale_b[e * a.sb_e + (n0 / kBlock) * a.sb_n + kb * a.sb_k];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = ty * 4 + i < rows ? a.scale_a[(m0 + ty * 4 + i) * a.lds + kb] * s_b : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                out[i][j] = fmaf(acc[i][j], s, out[i][j]);
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (ty * 4 + i < rows && n0 + tx * 4 + j < a.N)
                static_cast<T *>(a.out)[(m0 + ty * 4 + i) * a.ldo + n0 + tx * 4 + j] = from_f32<T>(out[i][j]);
}

__global__ void __launch_bounds__(kGemmThreads) k_gemm_cols(const GemmColsArgs a)
{
    __shared__ float sa[kTile][kStep + 1], sb[kTile][kStep + 1];
    const int e = blockIdx.z, k0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int64_t run0 = 0, run1 = 0;
    for (int i = 0; i <= e; ++i) {
        const int64_t lo = a.offsets ? max((int64_t)0, min(a.M, (int64_t)a.offsets[i])) : 0;
        const int64_t hi = a.offsets ? max(lo, min(a.M, (int64_t)a.offsets[i + 1])) : a.M;
        run0 = run1;
        run1 += (hi - lo + kBlock - 1) / kBlock;
    }
    float out[4][4] = {};
    for (int64_t r = run0; r < run1; ++r) {
        float acc[4][4] = {};
        block_product(a.A + n0 * a.lda + r * kBlock, a.lda, min(kTile, a.N - n0), a.B + k0 * a.ldb + r * kBlock, a.ldb,
                      min(kTile, a.K - k0), kBlock, sa, sb, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n0 + ty * 4 + i < a.N && k0 + tx * 4 + j < a.K)
                    out[i][j] = fmaf(acc[i][j] * a.scale_a[r * a.lds_a + n0 + ty * 4 + i],
                                     a.scale_b[r * a.lds_b + k0 + tx * 4 + j], out[i][j]);
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (n0 + ty * 4 + i < a.N && k0 + tx * 4 + j < a.K)
                a.out[((int64_t)e * a.N + n0 + ty * 4 + i) * a.ldo + k0 + tx * 4 + j] = out[i][j];
}

}  // namespace

cudaError_t launch_gemm_rows(esp_moe *m, int32_t dtype, const GemmRowsArgs &a)
{
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        const dim3 grid((unsigned)(a.M / kTile + a.E), (unsigned)ceil_div(a.N, kTile));
        k_gemm_rows<T><<<grid, kGemmThreads, 0, m->stream>>>(a);
        m->launches += 1;
        return cudaGetLastError();
    });
}

cudaError_t launch_gemm_cols(esp_moe *m, const GemmColsArgs &a)
{
    const dim3 grid((unsigned)ceil_div(a.K, kTile), (unsigned)ceil_div(a.N, kTile), (unsigned)a.E);
    k_gemm_cols<<<grid, kGemmThreads, 0, m->stream>>>(a);
    m->launches += 1;
    return cudaGetLastError();
}

}  // namespace esp_moe_impl
