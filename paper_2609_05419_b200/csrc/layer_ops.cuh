// Operators of a layer's training step next to the products of common.cuh: quantisation to 8-bit floating point with block
// scales (fp8_quantise.cu), the product of two such matrices (fp8_gemm.cu) and Newton-Schulz orthogonalisation
// (newton_schulz.cu).  Matrices are row-major here: rows contiguous, leading dimension = elements between rows.
#pragma once
#include "common.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace gemm2m {

constexpr int kScaleBlock = 128;          // entries along k that share a scale
constexpr float kLeastMax = 0x1p-100f;    // smallest block maximum: keeps MAX / maximum finite, and gives a block of zeros a scale

// Element types, numbered as in gemm2m_type.
enum ElemType { kF32 = 0, kF16 = 1, kBF16 = 2, kE4M3 = 3, kE5M2 = 4 };

struct QuantiseArgs {
    int64_t rows, cols;
    const void* X; int type; int64_t ldx;
    int fmt, block_rows;                  // kE4M3 / kE5M2; 1 or 128 rows per scale
    uint8_t* Q; int64_t ldq; float* S; int64_t lds;
    uint8_t* Qt; int64_t ldqt; float* St; int64_t ldst;      // transposed form, or null
};
cudaError_t launch_fp8_quantise(const QuantiseArgs& a, cudaStream_t st, int* launches);

// One operand of the scaled product: rows x k bytes, k contiguous; scale of (row r, block b) at S[b lds + r / block].
struct Fp8Operand { const uint8_t* Q; int fmt; int64_t ld; const float* S; int64_t lds; int block; };
struct Fp8GemmArgs {
    int64_t m, n, k;
    Fp8Operand A, B;
    const void* C; int64_t ldc;           // added to the product, or null; same type as D
    void* D; int type; int64_t ldd;
    int* dev_status;
};
cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches);

// Newton-Schulz iteration on `batch` matrices (see newton_schulz.cu for the arithmetic and the workspace).
struct NewtonSchulzLayout {
    int64_t ldx, lds;                     // leading dimensions of the iterate and of the short-side squares, in elements
    int64_t off_norm, off_count, off_shift, off_trace[2], off_hi[2], off_lo[2], off_gram, off_poly, off_part, off_part_count, total;      // bytes from the start of the workspace
    int64_t norm_parts, trace_parts;      // partial sums per matrix
    int splits; int64_t part_counts;      // pieces of the first product's inner dimension, and counters of finished ones
};
NewtonSchulzLayout newton_schulz_layout(int64_t batch, int64_t m, int64_t n, int64_t offset);
struct NewtonSchulzArgs {
    int64_t batch, m, n;
    const void* G; int type; int64_t ldg, stride_g;
    void* O; int64_t ldo, stride_o;       // bf16
    int steps; const float* coeffs;       // host, (a, b, c) per step
    float eps;
    char* ws; NewtonSchulzLayout lay;
    int* dev_status;
};
cudaError_t launch_newton_schulz(const NewtonSchulzArgs& a, int sm_count, cudaStream_t st, int launches[2]);
unsigned long long newton_schulz_wait_ns(int64_t batch, int64_t m, int64_t n);      // limit of its device-side waits

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// Eight consecutive entries of a row as they are in memory: a whole aligned group, or entry by entry with those at or beyond `valid`
// zero.  Loads that are to be in flight together must not sit in branches of their own (each would be waited for at its
// branch's end: 96 against 36 us for 8192 x 8192 bf16 entries), so callers choose once for all of them.  Converted later, by to_floats8.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> load8_part(const T* p, int64_t valid) {
    Raw8<T> r;
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t[i] = T(0.f);
        if (i < valid) t[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4*>(t)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void to_floats8(const Raw8<T>& r, float (&v)[8]) {
    const T* t = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float<T>(t[i]);
}

#endif

}  // namespace gemm2m
