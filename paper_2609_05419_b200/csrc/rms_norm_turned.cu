// The 8-bit form of a root-mean-square norm with blocks along the columns (rms_norm.cuh).
#include "rms_norm.cuh"

namespace gemm2m {

namespace {

// Qt, St from H (or X + R) and rstd: one block of 128 threads per tile of 128 rows x 64 columns, thread = 8 x 8 entries, otherwise as in the quantiser.  (Half a
// tile of the quantiser's: with four blocks on an SM their loads, arithmetic and stores overlap better than with two.)  It waits for its loads
// (8192 x 4096 bf16: 25 us; 67 of the 134 MB of H are still in the on-chip cache, since the tiles go from the last rows to the first).
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(128, 4) rms_norm_turned_kernel(const RmsNormArgs a, int col_tiles, int w_vec) {
    __shared__ uint32_t warp_top[4][64];
    __shared__ __align__(16) uint2 turned[64][16];
    __shared__ __align__(16) float turns[VEC ? 1 : 4][VEC ? 4 : kSegment];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned tile = gridDim.x - 1 - blockIdx.x;
    const int64_t tile_r = tile / (unsigned)col_tiles, tile_c = tile - tile_r * col_tiles;
    const int group = lane & 7;                          // columns 8 group .. of the tile
    const int rows8 = warp * 4 + (lane >> 3);            // rows 8 rows8 .. of the tile
    const int64_t row0 = tile_r * 128 + rows8 * 8, col0 = tile_c * 64 + group * 8;
    const int64_t valid = a.cols - col0;
    wait_for_prior_kernels();

    float y[8][8], w[8], rstd[8];
    // y = rows 8 rows8 + i of M, this thread's 8 columns; or these added to y, rounded to T
    auto read = [&](const T* M, int64_t ld, auto add) {
        auto take = [&](int i, const float (&v)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i][j] = decltype(add)::value ? to_float<T>(from_float<T>(y[i][j] + v[j])) : v[j];
        };
        if constexpr (VEC) {
            Raw8<T> raw[8];
            const T* src = M + row0 * ld + col0;
            if ((tile_r + 1) * 128 <= a.rows && (tile_c + 1) * 64 <= a.cols) {
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[i] = load8<T>(src + i * ld);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[i] = load8_part<T>(src + i * ld, row0 + i < a.rows ? valid : 0);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v[8];
                to_floats8<T>(raw[i], v);
                take(i, v);
            }
        } else {
            // four rows of 64 columns at a time: entry e = 32 j + lane is column e & 63 of the warp's row 8 (e >> 6) + i
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += 4) {
                T raw[4][8];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int64_t row = tile_r * 128 + warp * 32 + 8 * (j >> 1) + i0 + i, col = tile_c * 64 + (j & 1) * 32 + lane;
                        raw[i][j] = M[min(row, a.rows - 1) * ld + min(col, a.cols - 1)];
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int64_t row = tile_r * 128 + warp * 32 + 8 * (j >> 1) + i0 + i, col = tile_c * 64 + (j & 1) * 32 + lane;
                        v[j] = row < a.rows && col < a.cols ? to_float<T>(raw[i][j]) : 0.f;
                    }
                    to_groups(v, turns[warp]);
                    take(i0 + i, v);
                }
            }
        }
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) rstd[i] = __ldg(a.rstd + min(row0 + i, a.rows - 1));
    // (rows beyond the last: their entries are zero, and stay so)
    if (row0 + 8 > a.rows)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (row0 + i >= a.rows) rstd[i] = 0.f;
    read(a.H ? (const T*)a.H : (const T*)a.X, a.H ? a.ldh : a.ldx, std::false_type());
    if (a.R && !a.H) read((const T*)a.R, a.ldr, std::true_type());
    if (a.W) load8_any(a.W, a.w_type, col0, valid, w_vec && valid >= 8, w);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.f;
    float top[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] = y[i][j] * rstd[i] * w[j];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        top[j] = top3(top3(top3(y[0][j], y[1][j], y[2][j]), y[3][j], y[4][j]), top3(y[5][j], y[6][j], y[7][j]), 0.f);
    }
    // over the four lanes of a group of columns, which keep half of the columns after every exchange
#pragma unroll
    for (int d = 16, keep = 4; d >= 8; d >>= 1, keep >>= 1) {
        const bool upper = (lane & d) != 0;
#pragma unroll
        for (int j = 0; j < keep; ++j) {
            const float mine = upper ? top[j + keep] : top[j], theirs = upper ? top[j] : top[j + keep];
            top[j] = top3(mine, __shfl_xor_sync(0xffffffffu, theirs, d), 0.f);
        }
    }
    *reinterpret_cast<float2*>(&warp_top[warp][group * 8 + (lane >> 4) * 4 + (lane >> 3 & 1) * 2]) = make_float2(top[0], top[1]);
    __syncthreads();
    // one thread per column forms the scale and leaves the inverse in row 0 of the table
    if (threadIdx.x < 64) {
        uint32_t t = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) t = max(t, warp_top[v][threadIdx.x]);
        float s, inv;
        scales<FMT>(t, &s, &inv);
        const int64_t col = tile_c * 64 + threadIdx.x;
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
    const int eight = lane & 15;                             // here a lane has a group of 8 rows, a half-warp a column
    const int64_t out_row = tile_r * 128 + eight * 8, valid_rows = a.rows - out_row;
    if (valid_rows <= 0) return;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
        const int c = it * 8 + warp * 2 + (lane >> 4);
        const int64_t col = tile_c * 64 + c;
        if (col < a.cols) store8(a.Qt + col * a.ldqt + out_row, turned[c][eight ^ (c >> 3)], valid_rows);
    }
}

template <typename T, bool VEC>
cudaError_t launch_turned(const RmsNormArgs& a, int w_vec, cudaStream_t st) {
    const int64_t tr = (a.rows + 127) / 128, tc = (a.cols + 63) / 64;
    const dim3 grid((unsigned)(tr * tc)), block(128);
    return a.fmt == kE4M3 ? launch_chained(rms_norm_turned_kernel<T, kE4M3, VEC>, grid, block, 0, st, a, (int)tc, w_vec)
                          : launch_chained(rms_norm_turned_kernel<T, kE5M2, VEC>, grid, block, 0, st, a, (int)tc, w_vec);
}

template <typename T>
cudaError_t launch_typed(const RmsNormArgs& a, bool vec, int w_vec, cudaStream_t st) {
    return vec ? launch_turned<T, true>(a, w_vec, st) : launch_turned<T, false>(a, w_vec, st);
}

}  // namespace

cudaError_t launch_rms_norm_turned(const RmsNormArgs& a, bool vec, int w_vec, cudaStream_t st) {
    if (a.type == kF32) return launch_typed<float>(a, vec, w_vec, st);
    if (a.type == kF16) return launch_typed<__half>(a, vec, w_vec, st);
    return launch_typed<__nv_bfloat16>(a, vec, w_vec, st);
}

}  // namespace gemm2m
