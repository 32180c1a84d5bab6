// Root-mean-square norm with the residual's addition, written as 8-bit operands with block scales, and its gradients.
//
// Forward: H = rn(X + R), rstd = 1 / sqrt(mean_j H_ij^2 + eps), N = (H rstd) W, held in 32 bits; Y = rn(N); Q, S = N in 1 x 128 blocks
// along the rows, Qt, St = N in blocks along the columns, both as the quantiser forms them (fp8_quantise.cu).  The norm is that of H as it is stored,
// so that the backward pass, which reads H, differentiates what was computed.
// Backward: with n = H rstd and dN = dY W: dX = rn(rstd (dN - n mean_j(dN n)) + dR), dW = (dW) + sum_i dY n.
//
// A row is held in the registers of 32 to 1024 threads, 8 consecutive entries in each of NV places per thread, so every operand is
// read once; 16 neighbouring threads hold a block of 128.
#include "fp8_pack.cuh"

namespace gemm2m {

namespace {

constexpr int kNormThreads = 256;         // per block, unless a row needs more

// Sum over the `width` threads (a power of two, 32 to 1024) that share a row; every thread of the block takes part.
__device__ __forceinline__ float row_sum(float v, int width, float* warps) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (width == 32) return v;
    const int warp = threadIdx.x >> 5, first = (threadIdx.x & ~(width - 1)) >> 5;
    if ((threadIdx.x & 31) == 0) warps[warp] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < width >> 5; ++w) v += warps[first + w];
    return v;
}

// Blocks of 128 along a row from a thread's 8 values: the maximum over 16 neighbouring threads, then as the quantiser.
template <int FMT>
__device__ __forceinline__ void quantise8(const float (&y)[8], uint8_t* q, int64_t valid, float* s) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
#pragma unroll
    for (int d = 8; d; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    float scale, inv;
    scales<FMT>(top, &scale, &inv);
    if (valid <= 0) return;
    if ((threadIdx.x & 15) == 0) *s = scale;
    store8(q, make_uint2(pack4<FMT>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), pack4<FMT>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)), valid);
}

template <typename T, int NV>
__global__ void __launch_bounds__(1024) rms_norm_rows_kernel(const RmsNormArgs a, int width, int vec, int w_vec) {
    __shared__ float warps[32];
    const int lane = threadIdx.x & (width - 1);
    const int64_t row = blockIdx.x * (int64_t)(blockDim.x / width) + threadIdx.x / width;
    const bool active = row < a.rows;
    const T* X = (const T*)a.X + row * a.ldx;
    const T* R = (const T*)a.R + row * a.ldr;
    wait_for_prior_kernels();
    Raw8<T> x[NV], r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (lane + (int64_t)i * width) * 8, valid = active ? a.cols - col : 0;
        if (vec && valid >= 8) {
            x[i] = load8_rw<T>(X + col);
            if (a.R) r[i] = load8_rw<T>(R + col);
        } else {
            x[i] = load8_part<T>(X + col, valid);
            if (a.R) r[i] = load8_part<T>(R + col, valid);
        }
    }
    float h[NV][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (lane + (int64_t)i * width) * 8, valid = active ? a.cols - col : 0;
        to_floats8<T>(x[i], h[i]);
        if (a.R) {
            float t[8];
            to_floats8<T>(r[i], t);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = to_float<T>(from_float<T>(h[i][j] + t[j]));
        }
        if (a.H && valid > 0) store8_as<T>((T*)a.H + row * a.ldh + col, h[i], vec && valid >= 8, valid);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += h[i][j] * h[i][j];
    }
    const float rstd = __frsqrt_rn(row_sum(sum, width, warps) / (float)a.cols + a.eps);
    if (a.rstd && active && lane == 0) a.rstd[row] = rstd;
    if (!a.Y && !a.Q) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (lane + (int64_t)i * width) * 8, valid = active ? a.cols - col : 0;
        float y[8], w[8];
        if (a.W) load8_any(a.W, a.w_type, col, a.cols - col, w_vec && a.cols - col >= 8, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = a.W ? h[i][j] * rstd * w[j] : h[i][j] * rstd;
        if (a.Y && valid > 0) store8_as<T>((T*)a.Y + row * a.ldy + col, y, vec && valid >= 8, valid);
        if (a.Q) {
            uint8_t* q = a.Q + row * a.ldq + col;
            float* s = a.S + (col >> 7) * a.lds + row;
            if (a.fmt == kE4M3) quantise8<kE4M3>(y, q, valid, s);
            else quantise8<kE5M2>(y, q, valid, s);
        }
    }
}

// Qt, St from H (or X + R) and rstd: one block per 128 x 128 tile, thread = 8 x 8 entries, as in the quantiser.
template <typename T, int FMT>
__global__ void __launch_bounds__(256, 2) rms_norm_turned_kernel(const RmsNormArgs a, int col_tiles, int vec, int w_vec) {
    __shared__ uint32_t warp_top[8][128];
    __shared__ __align__(16) uint2 turned[128][16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile_r = blockIdx.x / (unsigned)col_tiles, tile_c = blockIdx.x - tile_r * col_tiles;
    const int group = lane & 15;
    const int rows8 = warp * 2 + (lane >> 4);
    const int64_t row0 = tile_r * 128 + rows8 * 8, col0 = tile_c * 128 + group * 8;
    const int64_t valid = a.cols - col0;
    wait_for_prior_kernels();

    float y[8][8], w[8];
    const bool add = a.R && !a.H, full = vec && (tile_r + 1) * 128 <= a.rows && (tile_c + 1) * 128 <= a.cols;
    const T* src = a.H ? (const T*)a.H + row0 * a.ldh + col0 : (const T*)a.X + row0 * a.ldx + col0;
    const int64_t ld = a.H ? a.ldh : a.ldx;
    {
        Raw8<T> raw[8];
        if (full) {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i] = load8<T>(src + i * ld);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[i] = load8_part<T>(src + i * ld, row0 + i < a.rows ? valid : 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) to_floats8<T>(raw[i], y[i]);
    }
    if (add) {
        const T* res = (const T*)a.R + row0 * a.ldr + col0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float t[8];
            to_floats8<T>(full ? load8<T>(res + i * a.ldr) : load8_part<T>(res + i * a.ldr, row0 + i < a.rows ? valid : 0), t);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i][j] = to_float<T>(from_float<T>(y[i][j] + t[j]));
        }
    }
    if (a.W) load8_any(a.W, a.w_type, col0, valid, w_vec && valid >= 8, w);
    uint32_t top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float rstd = row0 + i < a.rows ? __ldg(a.rstd + row0 + i) : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[i][j] = a.W ? y[i][j] * rstd * w[j] : y[i][j] * rstd;
            top[j] = max(top[j], __float_as_uint(y[i][j]) & 0x7fffffffu);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = max(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
    if (lane < 16) {
        *reinterpret_cast<uint4*>(&warp_top[warp][group * 8]) = make_uint4(top[0], top[1], top[2], top[3]);
        *reinterpret_cast<uint4*>(&warp_top[warp][group * 8 + 4]) = make_uint4(top[4], top[5], top[6], top[7]);
    }
    __syncthreads();
    // one thread per column forms the scale and leaves the inverse in row 0 of the table
    if (threadIdx.x < 128) {
        uint32_t t = 0;
#pragma unroll
        for (int v = 0; v < 8; ++v) t = max(t, warp_top[v][threadIdx.x]);
        float s, inv;
        scales<FMT>(t, &s, &inv);
        const int64_t col = tile_c * 128 + threadIdx.x;
        if (col < a.cols) a.St[tile_r * a.ldst + col] = s;
        warp_top[0][threadIdx.x] = __float_as_uint(inv);      // only this thread reads column threadIdx.x before the barrier
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = __uint_as_float(warp_top[0][group * 8 + j]);
        turned[group * 8 + j][rows8 ^ group] = make_uint2(pack4<FMT>(y[0][j] * inv, y[1][j] * inv, y[2][j] * inv, y[3][j] * inv),
                                                          pack4<FMT>(y[4][j] * inv, y[5][j] * inv, y[6][j] * inv, y[7][j] * inv));
    }
    __syncthreads();
    const int64_t out_row = tile_r * 128 + group * 8;              // here `group` is a group of 8 rows, warp and half-warp a column
    const int64_t valid_rows = a.rows - out_row;
    if (valid_rows <= 0) return;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
        const int c = it * 16 + rows8;
        const int64_t col = tile_c * 128 + c;
        if (col < a.cols) store8(a.Qt + col * a.ldqt + out_row, turned[c][group ^ (c >> 3)], valid_rows);
    }
}

// Rows blockIdx, blockIdx + grid, ...; the sums of dW over them go to row blockIdx of `part`.
template <typename T, int NV>
__global__ void __launch_bounds__(1024) rms_norm_backward_kernel(const RmsNormBackwardArgs a, int width, int vec, int w_vec) {
    __shared__ float warps[2][32];
    const int lane = threadIdx.x & (width - 1);
    const int per_block = blockDim.x / width;
    float acc[NV][8], w[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f, w[i][j] = 1.f;
    wait_for_prior_kernels();
    if (a.W) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = (lane + (int64_t)i * width) * 8;
            load8_any(a.W, a.w_type, col, a.cols - col, w_vec && a.cols - col >= 8, w[i]);
        }
    }
    int turn = 0;
    for (int64_t first = blockIdx.x * (int64_t)per_block; first < a.rows; first += gridDim.x * (int64_t)per_block, turn ^= 1) {
        const int64_t row = first + threadIdx.x / width;
        const bool active = row < a.rows;
        const T* G = (const T*)a.dY + row * a.lddy;
        const T* H = (const T*)a.H + row * a.ldh;
        const T* R = (const T*)a.dR + row * a.lddr;
        Raw8<T> g[NV], h[NV], r[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = (lane + (int64_t)i * width) * 8, valid = active ? a.cols - col : 0;
            if (vec && valid >= 8) {
                g[i] = load8_rw<T>(G + col);
                h[i] = load8_rw<T>(H + col);
                if (a.dR) r[i] = load8_rw<T>(R + col);
            } else {
                g[i] = load8_part<T>(G + col, valid);
                h[i] = load8_part<T>(H + col, valid);
                if (a.dR) r[i] = load8_part<T>(R + col, valid);
            }
        }
        const float rstd = active ? a.rstd[row] : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float dy[8], n[8];
            to_floats8<T>(g[i], dy);
            to_floats8<T>(h[i], n);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = dy[j] * (n[j] * rstd);
                acc[i][j] += t;
                sum += t * w[i][j];
            }
        }
        // (two tables in turn: a warp may be a row ahead of one that still reads)
        const float mean = row_sum(sum, width, warps[turn]) / (float)a.cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = (lane + (int64_t)i * width) * 8, valid = active ? a.cols - col : 0;
            if (valid <= 0) continue;
            float dy[8], n[8], t[8], out[8];
            to_floats8<T>(g[i], dy);
            to_floats8<T>(h[i], n);
            if (a.dR) to_floats8<T>(r[i], t);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                out[j] = rstd * (dy[j] * w[i][j] - n[j] * rstd * mean);
                if (a.dR) out[j] += t[j];
            }
            store8_as<T>((T*)a.dX + row * a.lddx + col, out, vec && valid >= 8, valid);
        }
    }
    if (!a.dW) return;
    float* part = a.part + (blockIdx.x * (int64_t)per_block + threadIdx.x / width) * a.cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (lane + (int64_t)i * width) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < a.cols) part[col + j] = acc[i][j];
    }
}

// dW = (dW) + the sum of the `parts` rows of partial sums: 32 columns per block, 32 threads deep, in a fixed order.
__global__ void __launch_bounds__(1024) rms_norm_dw_kernel(const float* __restrict__ part, int64_t parts, int64_t cols, float* dW, int add) {
    __shared__ float sums[32][33];
    const int64_t col = blockIdx.x * 32LL + threadIdx.x;
    wait_for_prior_kernels();
    float s = 0.f;
    if (col < cols)
        for (int64_t p = threadIdx.y; p < parts; p += 32) s += part[p * cols + col];
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    float t = sums[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int d = 16; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    const int64_t out = blockIdx.x * 32LL + threadIdx.y;
    if (threadIdx.x == 0 && out < cols) dW[out] = add ? dW[out] + t : t;
}

template <typename T>
bool aligned8(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * sizeof(T)) % 16 == 0; }

// Threads per row: the fewest powers of two that hold it with `places` groups of 8 per thread.
int row_width(int64_t cols, int places) {
    int width = 32;
    while (width < 1024 && (int64_t)width * places * 8 < cols) width *= 2;
    return width;
}

template <typename T>
cudaError_t launch_typed(const RmsNormArgs& a, cudaStream_t st, int* launches) {
    const int vec = aligned8<T>(a.X, a.ldx) && (!a.R || aligned8<T>(a.R, a.ldr)) && (!a.H || aligned8<T>(a.H, a.ldh)) && (!a.Y || aligned8<T>(a.Y, a.ldy));
    const int w_vec = ((uintptr_t)a.W & 15) == 0;
    const int width = row_width(a.cols, 2);
    const int places = (int)((a.cols + width * 8 - 1) / (width * 8));
    const int threads = width > kNormThreads ? width : kNormThreads;
    const int64_t blocks = (a.rows + threads / width - 1) / (threads / width);
    const dim3 grid((unsigned)blocks), block(threads);
    cudaError_t err = places <= 1 ? launch_chained(rms_norm_rows_kernel<T, 1>, grid, block, 0, st, a, width, vec, w_vec)
                    : places <= 2 ? launch_chained(rms_norm_rows_kernel<T, 2>, grid, block, 0, st, a, width, vec, w_vec)
                                  : launch_chained(rms_norm_rows_kernel<T, 4>, grid, block, 0, st, a, width, vec, w_vec);
    if (err != cudaSuccess) return err;
    ++*launches;
    if (!a.Qt) return cudaSuccess;
    const int64_t tr = (a.rows + 127) / 128, tc = (a.cols + 127) / 128;
    err = a.fmt == kE4M3 ? launch_chained(rms_norm_turned_kernel<T, kE4M3>, dim3((unsigned)(tr * tc)), dim3(256), 0, st, a, (int)tc, vec, w_vec)
                         : launch_chained(rms_norm_turned_kernel<T, kE5M2>, dim3((unsigned)(tr * tc)), dim3(256), 0, st, a, (int)tc, vec, w_vec);
    if (err == cudaSuccess) ++*launches;
    return err;
}

struct BackwardShape { int width, places, threads; int64_t blocks; };
BackwardShape backward_shape(int64_t rows, int64_t cols) {
    BackwardShape s;
    s.width = row_width(cols, 2);
    s.places = (int)((cols + s.width * 8 - 1) / (s.width * 8));
    s.threads = s.width > kNormThreads ? s.width : kNormThreads;
    const int64_t need = (rows + s.threads / s.width - 1) / (s.threads / s.width), most = 1024 / s.threads * (int64_t)kSms;
    s.blocks = need < most ? need : most;
    return s;
}

template <typename T>
cudaError_t launch_backward_typed(const RmsNormBackwardArgs& a, cudaStream_t st, int* launches) {
    const BackwardShape s = backward_shape(a.rows, a.cols);
    const int vec = aligned8<T>(a.dY, a.lddy) && aligned8<T>(a.H, a.ldh) && aligned8<T>(a.dX, a.lddx) && (!a.dR || aligned8<T>(a.dR, a.lddr));
    const int w_vec = ((uintptr_t)a.W & 15) == 0;
    const dim3 grid((unsigned)s.blocks), block(s.threads);
    cudaError_t err = s.places <= 1 ? launch_chained(rms_norm_backward_kernel<T, 1>, grid, block, 0, st, a, s.width, vec, w_vec)
                    : s.places <= 2 ? launch_chained(rms_norm_backward_kernel<T, 2>, grid, block, 0, st, a, s.width, vec, w_vec)
                                    : launch_chained(rms_norm_backward_kernel<T, 4>, grid, block, 0, st, a, s.width, vec, w_vec);
    if (err != cudaSuccess) return err;
    ++*launches;
    if (!a.dW) return cudaSuccess;
    err = launch_chained(rms_norm_dw_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(32, 32), 0, st, (const float*)a.part, a.parts, a.cols, a.dW, a.add);
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace

cudaError_t launch_rms_norm(const RmsNormArgs& a, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_typed<float>(a, st, launches);
    if (a.type == kF16) return launch_typed<__half>(a, st, launches);
    return launch_typed<__nv_bfloat16>(a, st, launches);
}

int64_t rms_norm_backward_parts(int64_t rows, int64_t cols) {
    const BackwardShape s = backward_shape(rows, cols);
    return s.blocks * (s.threads / s.width);
}

cudaError_t launch_rms_norm_backward(const RmsNormBackwardArgs& a, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_backward_typed<float>(a, st, launches);
    if (a.type == kF16) return launch_backward_typed<__half>(a, st, launches);
    return launch_backward_typed<__nv_bfloat16>(a, st, launches);
}

}  // namespace gemm2m
