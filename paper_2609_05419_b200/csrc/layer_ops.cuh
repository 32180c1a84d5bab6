// Operators of a layer's training step next to the products of common.cuh: quantisation to 8-bit floating point with block
// scales (fp8_quantise.cu), the product of two such matrices (fp8_gemm.cu), Newton-Schulz orthogonalisation
// (newton_schulz.cu), the root-mean-square norm and its gradients (rms_norm*.cu), clipping of gradients (clip_gradients.cu) and low-rank
// updates of many adapters (adapters*.cu).  Matrices are row-major here: rows contiguous, leading dimension = elements between rows.
#pragma once
#include "common.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace gemm2m {

constexpr int kScaleBlock = 128;          // entries along k that share a scale
constexpr int kSms = 148;                  // of a B200: grids that decide how sums are cut go by this, not by the device at hand
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

// Root-mean-square norm of the rows of H = X + R (rms_norm.cu); any of the outputs may be null.
constexpr int64_t kMaxNormCols = 32768;   // a row is held in the registers of one block
struct RmsNormArgs {
    int64_t rows, cols;
    const void* X; int type; int64_t ldx;                    // X, R, H, Y: the same type
    const void* R; int64_t ldr;
    const void* W; int w_type; float eps;                    // null: ones
    void* H; int64_t ldh;
    void* Y; int64_t ldy;
    int fmt;
    uint8_t* Q; int64_t ldq; float* S; int64_t lds;
    uint8_t* Qt; int64_t ldqt; float* St; int64_t ldst;
    float* rstd;                                             // needed for Qt
};
cudaError_t launch_rms_norm(const RmsNormArgs& a, cudaStream_t st, int* launches);
struct RmsNormBackwardArgs {
    int64_t rows, cols;
    const void* dY; int type; int64_t lddy;                  // dY, H, dR, dX: the same type
    const void* H; int64_t ldh;
    const void* W; int w_type;
    const float* rstd;
    const void* dR; int64_t lddr;
    void* dX; int64_t lddx;
    float* dW; int add;
    float* part;                                             // workspace: partial sums of dW
};
int64_t rms_norm_backward_partials(int64_t rows, int64_t cols);      // partial sums of dW of a call of these sizes, or smaller ones, at the most
cudaError_t launch_rms_norm_backward(const RmsNormBackwardArgs& a, cudaStream_t st, int* launches);

// Common 2-norm of many tensors, and the tensors scaled down where it is above a limit (clip_gradients.cu).
struct GradTensor {
    const void* g; void* o;               // o == g: in place
    int64_t rows, cols, ldg, ldo;         // row-major; rows = 1 where the entries are contiguous
    int type;
};
int64_t clip_partials(int64_t count);     // doubles of workspace for that many tensors
// norm: device float or null.  scale = false: the norm alone, no tensor is written.
cudaError_t launch_clip_gradients(const GradTensor* t, int64_t count, bool scale, float max_norm, float eps, float* norm, double* partials, cudaStream_t st,
                                  int launches[2]);

// Low-rank updates of many adapters, added to what a shared projection wrote (adapters.cu).
constexpr int kMaxRank = 128, kMaxAdapters = 16384;
struct AdapterArgs {
    int64_t tokens, n, k;
    int adapters, rank;
    const void* X; int type; int64_t ldx;                    // X, A, B: the same 16-bit type
    const void* A; int64_t lda, stride_a;                    // adapter a: rank x k
    const void* B; int64_t ldb, stride_b;                    // adapter a: n x rank
    const int32_t* index; const float* scales; const int32_t* ranks;
    const void* C; int64_t ldc;
    void* D; int d_type; int64_t ldd;
    char* ws;
    int* dev_status;
};
int64_t adapter_bytes(int64_t tokens, int rank, int adapters);      // workspace of a call of these sizes, or smaller ones
cudaError_t launch_adapter_add(const AdapterArgs& a, cudaStream_t st, int launches[2]);

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
// The same of memory that the kernel also writes (an output in the place of an input): not through the read-only path.
template <typename T>
__device__ __forceinline__ Raw8<T> load8_rw(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4*>(p)[i];
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
// Two 16-bit numbers of a word, the first in the low half.  (bf16: one shift and one mask; taken out of memory one by one they cost twice the instructions.)
template <typename T> __device__ __forceinline__ void unpack_as(uint32_t w, float* a, float* b);
template <> __device__ __forceinline__ void unpack_as<__nv_bfloat16>(uint32_t w, float* a, float* b) {
    *a = __uint_as_float(w << 16);
    *b = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack_as<__half>(uint32_t w, float* a, float* b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    *a = f.x;
    *b = f.y;
}
template <typename T>
__device__ __forceinline__ void to_floats8(const Raw8<T>& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        unpack_as<T>(r.w[0].x, &v[0], &v[1]);
        unpack_as<T>(r.w[0].y, &v[2], &v[3]);
        unpack_as<T>(r.w[0].z, &v[4], &v[5]);
        unpack_as<T>(r.w[0].w, &v[6], &v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i] = __uint_as_float(r.w[i].x);
            v[4 * i + 1] = __uint_as_float(r.w[i].y);
            v[4 * i + 2] = __uint_as_float(r.w[i].z);
            v[4 * i + 3] = __uint_as_float(r.w[i].w);
        }
    }
}
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
// Two values rounded to a 16-bit type, the first in the low half (one instruction).
template <typename T> __device__ __forceinline__ uint32_t pack_as(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_as<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack_as<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Eight values rounded to T; a whole aligned group, or the first `valid` entries one by one.
template <typename T>
__device__ __forceinline__ void store8_as(T* p, const float (&v)[8], bool whole, int64_t valid) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 2) {
        r.w[0] = make_uint4(pack_as<T>(v[0], v[1]), pack_as<T>(v[2], v[3]), pack_as<T>(v[4], v[5]), pack_as<T>(v[6], v[7]));
    } else {
        r.w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        r.w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
    const T* t = reinterpret_cast<const T*>(&r);
    if (whole) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = r.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = t[i];
    }
}
// Eight entries of a vector of any floating type (type code known at run time).
__device__ __forceinline__ void load8_any(const void* p, int type, int64_t at, int64_t valid, bool whole, float (&v)[8]) {
    if (type == kF32) to_floats8<float>(whole ? load8<float>((const float*)p + at) : load8_part<float>((const float*)p + at, valid), v);
    else if (type == kF16) to_floats8<__half>(whole ? load8<__half>((const __half*)p + at) : load8_part<__half>((const __half*)p + at, valid), v);
    else to_floats8<__nv_bfloat16>(whole ? load8<__nv_bfloat16>((const __nv_bfloat16*)p + at) : load8_part<__nv_bfloat16>((const __nv_bfloat16*)p + at, valid), v);
}

#endif

}  // namespace gemm2m
