// Quantisation to 8-bit floating point with block scales.
//
// A block is 1 x 128 entries of a row (block_rows = 1; 128 x 1 entries of a column for the transposed form) or 128 x 128.
// With u = max(max |x| over the block, 2^-100) and MAX the largest finite 8-bit value: scale s = u / MAX, q = rn(x (MAX / u)),
// saturating.  Both forms come from one read of X.  The maximum is taken over bit patterns with the sign cleared, where
// NaN > Inf > every finite number, so a block with a non-finite entry is seen as such and gets the scale NaN.
//
// One block of 256 threads per 128 x 128 tile, held in registers: thread = 8 x 8 entries, 16 threads across a row, so a load of
// 8 entries per thread is 256 (bf16) or 512 (f32) contiguous bytes of two rows per warp.  Row maxima are a butterfly over the 16 threads of a
// row; column maxima are the thread's own 8 rows, one exchange with the other half-warp and a combination of the 8 warps through
// shared memory.  The transposed form turns in shared memory, in 8-byte pieces (8 rows of a column) whose position is XORed with
// the column's group of 8 so that neither side has bank conflicts.
//
// Bound by HBM where a tile has one scale (8192^2 f32, both forms: 62.9 us, 6.4 TB/s).  Where every row and column has one, neither HBM
// (62 % of its rate) nor the issue slots (55 %) are full: a block's loads, arithmetic and stores follow one another, and 16 warps per SM do not
// cover the waits for the loads (8192 x 4096 bf16, both forms: 33.5 us, 4.1 TB/s; 8192^2 bf16, rows only, 24 warps: 35.4 us, 5.7 TB/s).
#include "layer_ops.cuh"

#include <cuda_fp8.h>

namespace gemm2m {

namespace {

constexpr int kThreads = 256;

template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    constexpr __nv_fp8_interpretation_t kind = FMT == kE4M3 ? __NV_E4M3 : __NV_E5M2;
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, kind);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, kind);
    return lo | (hi << 16);
}

// Scale and inverse scale of a block from the bit pattern of its largest magnitude.
template <int FMT>
__device__ __forceinline__ void scales(uint32_t top, float* s, float* inv) {
    constexpr float kMax = FMT == kE4M3 ? 448.f : 57344.f;
    const float u = fmaxf(__uint_as_float(top), kLeastMax);
    const bool finite = top < 0x7f800000u;
    *s = finite ? __fdiv_rn(u, kMax) : __uint_as_float(0x7fffffffu);
    *inv = finite ? __fdiv_rn(kMax, u) : 0.f;
}

__device__ __forceinline__ void store8(uint8_t* p, uint2 v, int64_t valid) {
    if (valid >= 8) {
        *reinterpret_cast<uint2*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
    }
}

template <typename T, int FMT, bool TILE, bool BOTH>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 || (BOTH && !TILE) ? 2 : 3) fp8_quantise_kernel(const QuantiseArgs a, int col_tiles, int vec) {
    __shared__ uint32_t warp_top[8][128];
    __shared__ __align__(16) uint2 turned[BOTH ? 128 : 1][16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile_r = blockIdx.x / (unsigned)col_tiles, tile_c = blockIdx.x - tile_r * col_tiles;
    const int group = lane & 15;                         // columns 8 group .. 8 group + 7 of the tile
    const int rows8 = warp * 2 + (lane >> 4);            // rows 8 rows8 .. of the tile
    const int64_t row0 = tile_r * 128 + rows8 * 8, col0 = tile_c * 128 + group * 8;
    const int64_t valid = a.cols - col0;
    wait_for_prior_kernels();

    Raw8<T> raw[8];
    const T* src = (const T*)a.X + row0 * a.ldx + col0;
    if (vec && (tile_r + 1) * 128 <= a.rows && (tile_c + 1) * 128 <= a.cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = load8<T>(src + i * a.ldx);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = load8_part<T>(src + i * a.ldx, row0 + i < a.rows ? valid : 0);
    }
    float x[8][8];
    uint32_t top_row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) to_floats8<T>(raw[i], x[i]);
    uint32_t top_col[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top_col[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top_row[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t size = __float_as_uint(x[i][j]) & 0x7fffffffu;
            top_row[i] = max(top_row[i], size);
            if (BOTH && !TILE) top_col[j] = max(top_col[j], size);
        }
    }
    float inv_row[8];
    if (TILE) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, top_row[i]);
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) warp_top[warp][0] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, warp_top[w][0]);
        float s, inv;
        scales<FMT>(top, &s, &inv);
#pragma unroll
        for (int i = 0; i < 8; ++i) inv_row[i] = inv;
        if (threadIdx.x == 0) {
            if (a.Q) a.S[tile_c * a.lds + tile_r] = s;
            if (BOTH) a.St[tile_r * a.ldst + tile_c] = s;
        }
    } else if (a.Q) {
        // Row maxima over 16 lanes, halving the rows that a lane keeps with every exchange: lane g of the 16 ends with row g / 2, forms
        // its scale (two divisions, not sixteen) and hands the inverse back.
#pragma unroll
        for (int d = 8, keep = 4; d > 1; d >>= 1, keep >>= 1) {
            const bool upper = (lane & d) != 0;
#pragma unroll
            for (int i = 0; i < keep; ++i) {
                const uint32_t mine = upper ? top_row[i + keep] : top_row[i], theirs = upper ? top_row[i] : top_row[i + keep];
                top_row[i] = max(mine, __shfl_xor_sync(0xffffffffu, theirs, d));
            }
        }
        top_row[0] = max(top_row[0], __shfl_xor_sync(0xffffffffu, top_row[0], 1));
        float s, inv;
        scales<FMT>(top_row[0], &s, &inv);
        const int64_t row = row0 + (group >> 1);
        if (!(lane & 1) && row < a.rows) a.S[tile_c * a.lds + row] = s;
#pragma unroll
        for (int i = 0; i < 8; ++i) inv_row[i] = __shfl_sync(0xffffffffu, inv, (lane & 16) | (2 * i));
    }
    if (a.Q && valid > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 q = make_uint2(pack4<FMT>(x[i][0] * inv_row[i], x[i][1] * inv_row[i], x[i][2] * inv_row[i], x[i][3] * inv_row[i]),
                                       pack4<FMT>(x[i][4] * inv_row[i], x[i][5] * inv_row[i], x[i][6] * inv_row[i], x[i][7] * inv_row[i]));
            if (row0 + i < a.rows) store8(a.Q + (row0 + i) * a.ldq + col0, q, valid);
        }
    }
    if (BOTH) {
        float inv_col[8];
        if (TILE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) inv_col[j] = inv_row[0];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) top_col[j] = max(top_col[j], __shfl_xor_sync(0xffffffffu, top_col[j], 16));
            if (lane < 16) {
                *reinterpret_cast<uint4*>(&warp_top[warp][group * 8]) = make_uint4(top_col[0], top_col[1], top_col[2], top_col[3]);
                *reinterpret_cast<uint4*>(&warp_top[warp][group * 8 + 4]) = make_uint4(top_col[4], top_col[5], top_col[6], top_col[7]);
            }
            __syncthreads();
            // one thread per column forms the scale and leaves the inverse in row 0 of the table
            float inv = 0.f;
            if (threadIdx.x < 128) {
                uint32_t t = 0;
#pragma unroll
                for (int w = 0; w < 8; ++w) t = max(t, warp_top[w][threadIdx.x]);
                float s;
                scales<FMT>(t, &s, &inv);
                const int64_t col = tile_c * 128 + threadIdx.x;
                if (col < a.cols) a.St[tile_r * a.ldst + col] = s;
                warp_top[0][threadIdx.x] = __float_as_uint(inv);      // only this thread reads column threadIdx.x before the barrier
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) inv_col[j] = __uint_as_float(warp_top[0][group * 8 + j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            turned[group * 8 + j][rows8 ^ group] =
                make_uint2(pack4<FMT>(x[0][j] * inv_col[j], x[1][j] * inv_col[j], x[2][j] * inv_col[j], x[3][j] * inv_col[j]),
                           pack4<FMT>(x[4][j] * inv_col[j], x[5][j] * inv_col[j], x[6][j] * inv_col[j], x[7][j] * inv_col[j]));
        __syncthreads();
        const int64_t out_row = tile_r * 128 + group * 8;              // here `group` is a group of 8 rows, warp and half-warp a column
        const int64_t valid_rows = a.rows - out_row;
        if (valid_rows > 0) {
#pragma unroll
            for (int it = 0; it < 8; ++it) {
                const int c = it * 16 + rows8;
                const int64_t col = tile_c * 128 + c;
                if (col < a.cols) store8(a.Qt + col * a.ldqt + out_row, turned[c][group ^ (c >> 3)], valid_rows);
            }
        }
    }
}

template <typename T, int FMT, bool TILE>
cudaError_t launch_typed(const QuantiseArgs& a, cudaStream_t st, int* launches) {
    const int64_t tr = (a.rows + 127) / 128, tc = (a.cols + 127) / 128;
    if (tr * tc > INT32_MAX) return cudaErrorInvalidValue;
    const int vec = ((uintptr_t)a.X & 15) == 0 && (a.ldx * sizeof(T)) % 16 == 0;
    cudaError_t err = a.Qt ? launch_chained(fp8_quantise_kernel<T, FMT, TILE, true>, dim3((unsigned)(tr * tc)), dim3(kThreads), 0, st, a, (int)tc, vec)
                           : launch_chained(fp8_quantise_kernel<T, FMT, TILE, false>, dim3((unsigned)(tr * tc)), dim3(kThreads), 0, st, a, (int)tc, vec);
    if (err == cudaSuccess) ++*launches;
    return err;
}
template <typename T>
cudaError_t launch_fmt(const QuantiseArgs& a, cudaStream_t st, int* launches) {
    if (a.block_rows == 1) return a.fmt == kE4M3 ? launch_typed<T, kE4M3, false>(a, st, launches) : launch_typed<T, kE5M2, false>(a, st, launches);
    return a.fmt == kE4M3 ? launch_typed<T, kE4M3, true>(a, st, launches) : launch_typed<T, kE5M2, true>(a, st, launches);
}

}  // namespace

cudaError_t launch_fp8_quantise(const QuantiseArgs& a, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_fmt<float>(a, st, launches);
    if (a.type == kF16) return launch_fmt<__half>(a, st, launches);
    return launch_fmt<__nv_bfloat16>(a, st, launches);
}

}  // namespace gemm2m
