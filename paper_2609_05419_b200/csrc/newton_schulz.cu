// Newton-Schulz iteration of an update matrix G (m x n, s = min(m, n), l = max(m, n)), as the Muon optimiser applies it:
//   X_0 = G / (|G|_F + eps),   X <- a X + (b A + c A^2) X,   A = X X^T  (m <= n; for m > n the same with A = X^T X on the right).
//
// Numbers.  Products take 16-bit floating-point operands (11 bits) and accumulate in 32 bits.  Rounding the iterate itself to 11 bits in
// every step is not enough: the iteration multiplies small singular directions by about a per step, and what was rounded off
// with them.  So the iterate is held as hi + lo (two 16-bit planes, 22 bits); products read hi, the linear term reads both.
// In the last two steps the linear term also takes over what it can from the products: with any g,
//   A' = A - g I,   a X + (b A + c A^2) X = (a + b g + c g^2) X + ((b + 2 c g) A' + c A'^2) X,
// exactly, and g = trace(A) / s makes A' (what is rounded) smallest.  trace(A) = |X|_F^2 comes from the step before, as one
// partial sum per tile, added in a fixed order by every reader.  (Earlier steps keep g = 0: there P = b A + c A^2 vanishes on the
// directions where X does, so that it lets none of hi's rounding into them, which a shift would, to be multiplied by a in every
// later step.)  All planes are scaled by powers of two into the middle of the 16-bit range.  Against 64 bits the result is off
// by 4e-4 .. 1.1e-3 of its norm for sides from 64 up (flat, k^-1/2 and k^-1 spectra, full rank and a third of it; up to 4e-3 for sides
// below 20), before its rounding to bf16 (1.7e-3); rounding the iterate to 16 bits instead costs up to 2e-2, all planes in bf16 up to 2e-1.
//
// Work.  A and A^2 are symmetric: only tiles on and below the diagonal are computed, and written twice.  Per step
// s^2 l + s^3 + 2 s^2 l operations.
#include "layer_ops.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace gemm2m {

namespace {

constexpr int kXExp = 8;              // hi = rn16(2^8 X): entries of X are at most about 1.2
constexpr int kLoExp = 11;            // lo = rn16(2^11 (2^8 X - hi))
constexpr int kSExp = 4;              // A' and the polynomial are held times 2^4
constexpr int kNormParts = 256;       // partial sums of |G|_F^2 per matrix
constexpr int kRowThreads = 256;

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// Sum over the block in a fixed order; every thread gets it.
__device__ __forceinline__ double block_sum(double v, double* scratch) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += scratch[w];
    return s;
}

// |G|_F^2, one partial sum per block, in 64 bits (a square of a 32-bit number always fits).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_kernel(const T* G, int64_t m, int64_t n, int64_t ldg, int64_t stride_g, double* parts) {
    __shared__ double scratch[kRowThreads / 32];
    wait_for_prior_kernels();
    const T* g = G + (int64_t)blockIdx.y * stride_g;
    double s = 0.0;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < n; c += kRowThreads) {
            const double v = (double)to_float<T>(g[r * ldg + c]);
            s += v * v;
        }
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// X_0 in two planes.  The first block of each matrix also leaves |X_0|_F^2 as the first of the trace's partial sums.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) start_kernel(const T* G, int64_t m, int64_t n, int64_t ldg, int64_t stride_g, const double* parts,
                                                            int nparts, float eps, __half* hi, __half* lo, int64_t ldx, float* trace, int trace_parts) {
    __shared__ double scratch[kRowThreads / 32];
    wait_for_prior_kernels();
    const int64_t b = blockIdx.y;
    double sq = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kRowThreads) sq += parts[b * nparts + i];
    sq = block_sum(sq, scratch);
    const double norm = sqrt(sq) + (double)eps;
    const double inv = norm > 0.0 ? (double)(1 << kXExp) / norm : 0.0;       // in 64 bits: 1 / norm of a tiny matrix overflows 32
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < trace_parts; i += kRowThreads) trace[b * trace_parts + i] = i == 0 && norm > 0.0 ? (float)(sq / (norm * norm)) : 0.f;
    const T* g = G + b * stride_g;
    for (int64_t r = blockIdx.x; r < m; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < n; c += kRowThreads) {
            const float x = (float)((double)to_float<T>(g[r * ldg + c]) * inv);
            const __half h = __float2half_rn(x);
            hi[(b * m + r) * ldx + c] = h;
            lo[(b * m + r) * ldx + c] = __float2half_rn((x - __half2float(h)) * (float)(1 << kLoExp));
        }
}

enum Mode { kGram, kPoly, kUpdate, kLast };

// One operand of a product: element (row r, inner p) of matrix b at p[b stride + r ld + p], or p[b stride + p ld + r] if `turned`.
struct Operand { const __half* p; int64_t ld, stride; int turned; };
struct NsGemm {
    int mode;
    int64_t M, N, K;
    Operand A, B;
    int64_t short_side;
    float a, b, c;
    const float* trace; int trace_parts;                           // partial sums of |X|_F^2, or null for g = 0
    __half* out; int64_t ldo, stride_o;                            // kGram, kPoly: symmetric square, scaled by 2^kSExp
    const __half* gram;                                             // kPoly: A', laid out as out
    const __half *hi, *lo; __half *hi_out, *lo_out; float* trace_out;   // kUpdate, kLast
    __nv_bfloat16* last; int64_t ld_last, stride_last;              // kLast
};

// g = trace(A) / s from the partial sums of matrix b, or zero.
__device__ __forceinline__ float shift_of(const NsGemm& q, int64_t b, double* scratch) {
    if (!q.trace) return 0.f;
    double t = 0.0;
    for (int i = threadIdx.x; i < q.trace_parts; i += blockDim.x) t += (double)q.trace[b * q.trace_parts + i];
    return (float)(block_sum(t, scratch) / (double)q.short_side);
}

// One block of 256 threads per 64 x 64 tile, 4 x 4 entries per thread.
__global__ void __launch_bounds__(256) ns_gemm_simple_kernel(const NsGemm q, int tiles_r, int tiles_c) {
    __shared__ float sa[32][68], sb[32][68];
    __shared__ double scratch[8];
    const int tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int64_t b = blockIdx.y;
    const bool square = q.mode == kGram || q.mode == kPoly;
    if (square && tc > tr) return;
    wait_for_prior_kernels();
    const float g = shift_of(q, b, scratch);
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const int64_t i0 = (int64_t)tr * 64, j0 = (int64_t)tc * 64;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < q.K; k0 += 32) {
        for (int t = threadIdx.x; t < 64 * 32; t += 256) {
            const int ra = q.A.turned ? t & 63 : t >> 5, pa = q.A.turned ? t >> 6 : t & 31;
            const int rb = q.B.turned ? t & 63 : t >> 5, pb = q.B.turned ? t >> 6 : t & 31;
            sa[pa][ra] = i0 + ra < q.M && k0 + pa < q.K ? __half2float(q.A.p[b * q.A.stride + (q.A.turned ? (k0 + pa) * q.A.ld + i0 + ra : (i0 + ra) * q.A.ld + k0 + pa)]) : 0.f;
            sb[pb][rb] = j0 + rb < q.N && k0 + pb < q.K ? __half2float(q.B.p[b * q.B.stride + (q.B.turned ? (k0 + pb) * q.B.ld + j0 + rb : (j0 + rb) * q.B.ld + k0 + pb)]) : 0.f;
        }
        __syncthreads();
        for (int p = 0; p < 32; ++p)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] += sa[p][ty * 4 + u] * sb[p][tx * 4 + v];
        __syncthreads();
    }
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ty * 4 + u, j = j0 + tx * 4 + v;
            if (i >= q.M || j >= q.N) continue;
            if (square) {
                float w;
                if (q.mode == kGram) w = acc[u][v] * exp2f(kSExp - 2 * kXExp) - (i == j ? g * exp2f(kSExp) : 0.f);
                else w = (q.b + 2.f * q.c * g) * __half2float(q.gram[b * q.stride_o + i * q.ldo + j]) + q.c * exp2f(-kSExp) * acc[u][v];
                q.out[b * q.stride_o + i * q.ldo + j] = __float2half_rn(w);
                if (tr != tc) q.out[b * q.stride_o + j * q.ldo + i] = __float2half_rn(w);
            } else {
                const int64_t at = (b * q.M + i) * q.ldo + j;
                const float x = __half2float(q.hi[at]) + __half2float(q.lo[at]) * exp2f(-kLoExp);
                const float w = (q.a + g * (q.b + q.c * g)) * x + acc[u][v] * exp2f(-kSExp);
                if (q.mode == kLast) {
                    q.last[b * q.stride_last + i * q.ld_last + j] = __float2bfloat16_rn(w * exp2f(-kXExp));
                } else {
                    const __half h = __float2half_rn(w);
                    q.hi_out[at] = h;
                    q.lo_out[at] = __float2half_rn((w - __half2float(h)) * exp2f(kLoExp));
                    sum += w * w;
                }
            }
        }
    if (q.mode == kUpdate) {
        const double s = block_sum((double)sum, scratch);
        if (threadIdx.x == 0) q.trace_out[b * q.trace_parts + blockIdx.x] = (float)(s * exp2(-2.0 * kXExp));
    }
}

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

cudaError_t run_gemm(const NsGemm& q, int64_t batch, cudaStream_t st, int* launches) {
    const int64_t tr = (q.M + 63) / 64, tc = (q.N + 63) / 64;
    cudaError_t err = launch_chained(ns_gemm_simple_kernel, dim3((unsigned)(tr * tc), (unsigned)batch), dim3(256), 0, st, q, (int)tr, (int)tc);
    if (err == cudaSuccess) ++*launches;
    return err;
}

template <typename T>
cudaError_t launch_start(const NewtonSchulzArgs& a, cudaStream_t st, int* launches) {
    const NewtonSchulzLayout& l = a.lay;
    double* parts = (double*)(a.ws + l.off_norm);
    const int blocks = (int)(a.m < kNormParts ? a.m : kNormParts);
    cudaError_t err = launch_chained(norm_kernel<T>, dim3(blocks, (unsigned)a.batch), dim3(kRowThreads), 0, st, (const T*)a.G, a.m, a.n, a.ldg, a.stride_g, parts);
    if (err != cudaSuccess) return err;
    err = launch_chained(start_kernel<T>, dim3((unsigned)(a.m < 1024 ? a.m : 1024), (unsigned)a.batch), dim3(kRowThreads), 0, st, (const T*)a.G, a.m, a.n, a.ldg,
                         a.stride_g, parts, blocks, a.eps, (__half*)(a.ws + l.off_hi[0]), (__half*)(a.ws + l.off_lo[0]), l.ldx,
                         (float*)(a.ws + l.off_trace[0]), l.trace_parts);
    if (err == cudaSuccess) *launches += 2;
    return err;
}

}  // namespace

NewtonSchulzLayout newton_schulz_layout(int64_t batch, int64_t m, int64_t n, int64_t offset) {
    NewtonSchulzLayout l = {};
    const int64_t s = m < n ? m : n;
    l.ldx = round_up(n, 64);
    l.lds = round_up(s, 64);
    l.norm_parts = kNormParts;
    l.trace_parts = (int)(((m + 63) / 64) * ((n + 63) / 64));
    int64_t off = round_up(offset, 256);
    auto take = [&](int64_t bytes) { int64_t o = off; off = round_up(off + bytes, 256); return o; };
    l.off_norm = take(8 * batch * l.norm_parts);
    for (int i = 0; i < 2; ++i) l.off_trace[i] = take(4 * batch * l.trace_parts);
    for (int i = 0; i < 2; ++i) {
        l.off_hi[i] = take(2 * batch * m * l.ldx);
        l.off_lo[i] = take(2 * batch * m * l.ldx);
    }
    l.off_gram = take(2 * batch * s * l.lds);
    l.off_poly = take(2 * batch * s * l.lds);
    l.total = off;
    return l;
}

cudaError_t launch_newton_schulz(const NewtonSchulzArgs& a, int sm_count, cudaStream_t st, int launches[2]) {
    (void)sm_count;
    cudaError_t err = a.type == kF32 ? launch_start<float>(a, st, &launches[0])
                      : a.type == kF16 ? launch_start<__half>(a, st, &launches[0]) : launch_start<__nv_bfloat16>(a, st, &launches[0]);
    if (err != cudaSuccess) return err;
    const NewtonSchulzLayout& l = a.lay;
    const bool tall = a.m > a.n;
    const int64_t s = tall ? a.n : a.m, L = tall ? a.m : a.n;
    __half* gram = (__half*)(a.ws + l.off_gram);
    __half* poly = (__half*)(a.ws + l.off_poly);
    for (int k = 0; k < a.steps; ++k) {
        const __half* hi = (const __half*)(a.ws + l.off_hi[k & 1]);
        const Operand x_rows = {hi, l.ldx, a.m * l.ldx, 0}, x_cols = {hi, l.ldx, a.m * l.ldx, 1};
        NsGemm q = {};
        q.short_side = s;
        q.a = a.coeffs[3 * k]; q.b = a.coeffs[3 * k + 1]; q.c = a.coeffs[3 * k + 2];
        q.trace = k + 2 >= a.steps ? (const float*)(a.ws + l.off_trace[k & 1]) : nullptr; q.trace_parts = l.trace_parts;
        q.ldo = l.lds; q.stride_o = s * l.lds;
        // A' = X X^T - g I  (X^T X for a tall matrix)
        q.mode = kGram; q.M = q.N = s; q.K = L;
        q.A = q.B = tall ? x_cols : x_rows;
        q.out = gram;
        if ((err = run_gemm(q, a.batch, st, &launches[1])) != cudaSuccess) return err;
        // P = (b + 2 c g) A' + c A'^2
        q.mode = kPoly; q.K = s;
        q.A = q.B = Operand{gram, l.lds, s * l.lds, 0};
        q.gram = gram; q.out = poly;
        if ((err = run_gemm(q, a.batch, st, &launches[1])) != cudaSuccess) return err;
        // X <- (a + b g + c g^2) X + P X  (X P for a tall matrix; P is symmetric)
        q.mode = k + 1 == a.steps ? kLast : kUpdate;
        q.M = a.m; q.N = a.n; q.K = s;
        const Operand p = {poly, l.lds, s * l.lds, 0};
        q.A = tall ? x_rows : p;
        q.B = tall ? p : x_cols;
        q.ldo = l.ldx;
        q.hi = hi; q.lo = (const __half*)(a.ws + l.off_lo[k & 1]);
        q.hi_out = (__half*)(a.ws + l.off_hi[(k + 1) & 1]);
        q.lo_out = (__half*)(a.ws + l.off_lo[(k + 1) & 1]);
        q.trace_out = (float*)(a.ws + l.off_trace[(k + 1) & 1]);
        q.last = (__nv_bfloat16*)a.O; q.ld_last = a.ldo; q.stride_last = a.stride_o;
        if ((err = run_gemm(q, a.batch, st, &launches[1])) != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace gemm2m
