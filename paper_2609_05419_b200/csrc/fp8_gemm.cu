// Product of two 8-bit floating-point matrices with block scales,
//   D[i, j] = C[i, j] + sum_b SA[i / block, b] SB[j / block, b] sum_{p in block b} A[i, p] B[j, p],
// blocks of 128 along k.  Every block's sum is accumulated in 32 bits, scaled, and added to a 32-bit total; D is rounded once.
#include "layer_ops.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

namespace gemm2m {

namespace {

__device__ __forceinline__ float fp8_value(uint8_t q, int fmt) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(q, fmt == kE4M3 ? __NV_E4M3 : __NV_E5M2)));
}

// One block of 256 threads per 64 x 64 tile, 4 x 4 entries per thread, operands unpacked into shared memory 32 columns at a time.
__global__ void __launch_bounds__(256) fp8_gemm_simple_kernel(const Fp8GemmArgs a, int col_tiles) {
    __shared__ float sa[32][68], sb[32][68];
    const int64_t i0 = (int64_t)(blockIdx.x / (unsigned)col_tiles) * 64, j0 = (int64_t)(blockIdx.x % (unsigned)col_tiles) * 64;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    wait_for_prior_kernels();
    float total[4][4] = {};
    for (int64_t kb = 0; kb * 128 < a.k; ++kb) {
        float part[4][4] = {};
        for (int64_t k0 = kb * 128; k0 < a.k && k0 < kb * 128 + 128; k0 += 32) {
            for (int t = threadIdx.x; t < 64 * 32; t += 256) {
                const int r = t >> 5, p = t & 31;
                sa[p][r] = i0 + r < a.m && k0 + p < a.k ? fp8_value(a.A.Q[(i0 + r) * a.A.ld + k0 + p], a.A.fmt) : 0.f;
                sb[p][r] = j0 + r < a.n && k0 + p < a.k ? fp8_value(a.B.Q[(j0 + r) * a.B.ld + k0 + p], a.B.fmt) : 0.f;
            }
            __syncthreads();
            for (int p = 0; p < 32; ++p)
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int v = 0; v < 4; ++v) part[u][v] += sa[p][ty * 4 + u] * sb[p][tx * 4 + v];
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t i = i0 + ty * 4 + u, j = j0 + tx * 4 + v;
                if (i < a.m && j < a.n)
                    total[u][v] += a.A.S[kb * a.A.lds + i / a.A.block] * a.B.S[kb * a.B.lds + j / a.B.block] * part[u][v];
            }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ty * 4 + u, j = j0 + tx * 4 + v;
            if (i >= a.m || j >= a.n) continue;
            const int64_t at = i * a.ldd + j, ct = i * a.ldc + j;
            if (a.type == kF32) ((float*)a.D)[at] = total[u][v] + (a.C ? ((const float*)a.C)[ct] : 0.f);
            else if (a.type == kF16) ((__half*)a.D)[at] = __float2half_rn(total[u][v] + (a.C ? __half2float(((const __half*)a.C)[ct]) : 0.f));
            else ((__nv_bfloat16*)a.D)[at] = __float2bfloat16_rn(total[u][v] + (a.C ? __bfloat162float(((const __nv_bfloat16*)a.C)[ct]) : 0.f));
        }
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    (void)sm_count;
    const int64_t tr = (a.m + 63) / 64, tc = (a.n + 63) / 64;
    if (tr * tc > INT32_MAX) return cudaErrorInvalidValue;
    cudaError_t err = launch_chained(fp8_gemm_simple_kernel, dim3((unsigned)(tr * tc)), dim3(256), 0, st, a, (int)tc);
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace gemm2m
