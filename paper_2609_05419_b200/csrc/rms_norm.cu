// Root-mean-square norm with the residual's addition, written as 8-bit operands with block scales.
//
// H = rn(X + R), rstd = 1 / sqrt(mean_j H_ij^2 + eps), N = (H rstd) W, held in 32 bits; Y = rn(N); Q, S = N in 1 x 128 blocks along the rows (here), Qt, St = N in
// blocks along the columns (rms_norm_turned.cu), both as the quantiser forms them (fp8_quantise.cu).  The norm is that of H as it is stored, so that the
// backward pass (rms_norm_backward.cu), which reads H, differentiates what was computed.
#include "rms_norm.cuh"

namespace gemm2m {

namespace {

// One row for every `warps` warps of a block, held in registers: read once, all outputs from there.  Bound by memory (8192 x 4096 bf16 with residual, H and 8-bit rows: 45 us,
// 5.2 TB/s; blocks of one wave each, whose loads, sums and stores overlap with the other blocks' of the SM).
template <typename T, int NV, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 1 : (VEC ? 1024 : 512) / THREADS) rms_norm_rows_kernel(const RmsNormArgs a, int warps, Two inv_cols, int w_vec) {
    __shared__ float sums[THREADS / 32 * NV];
    __shared__ __align__(16) float turns[VEC ? 1 : THREADS / 32][VEC ? 4 : kSegment];
    const Position at(warps, a.cols);
    float* turn = turns[VEC ? 0 : at.warp];
    const int lane = at.lane, cols = at.cols;
    const int64_t my_row = blockIdx.x * (int64_t)at.rows() + at.row_in, row = min(my_row, a.rows - 1);
    const bool write = my_row < a.rows;                  // a row beyond the last does the last one's work again, for itself
    wait_for_prior_kernels();
    Place<T, VEC> x[NV], r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i].load((const T*)a.X + row * a.ldx, at.first(i), cols);
    if (a.R)
#pragma unroll
        for (int i = 0; i < NV; ++i) r[i].load((const T*)a.R + row * a.ldr, at.first(i), cols);
    float h[NV][8], sum[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        x[i].get(h[i], turn);
        if (a.R) {
            float t[8];
            r[i].get(t, turn);
            if constexpr (sizeof(T) == 2) {
                // rounded two at a time
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    unpack_as<T>(pack_as<T>(h[i][j] + t[j], h[i][j + 1] + t[j + 1]), &h[i][j], &h[i][j + 1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += t[j];
            }
        }
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += h[i][j] * h[i][j];
        sum[i] = at.there(i) ? s : 0.f;
    }
    if (a.H)
#pragma unroll
        for (int i = 0; i < NV; ++i) store_place<T, VEC>((T*)a.H + row * a.ldh, at.first(i), cols, write, h[i], turn);
    float* segments = sums + at.row_in * warps * NV;
    const float mine = segment_sums<NV>(sum, segments, at.warp_in_row, warps, at.segments);
    // The barrier tells all threads of the block whether squares of any of its rows may leave the range in which 32 bits hold them and their sum (of up to 128 segments).  (8192 x 4096:
    // 44.9 us, 44.0 without this; with sums in 64 bits instead 50, in a function of their own 60.)
    const bool some = __syncthreads_or(!(mine < 0x1p120f) || (a.eps < 0x1p-99f && mine < 0x1p-80f));
    Two total = over_segments(segments, at.segments);
    float power = 1.f;
    if (some) {
        // Once more, of H 2^-72 where the sum is infinite (some entry is above 2^56), of H 2^75 where mean + eps is below 2^-99 (none is above 2^-41, and squares below 2^-126 have lost bits);
        // other rows get the number that they had.
        const float about = fmaf(total.hi, inv_cols.hi, a.eps);
        power = !(about < INFINITY) ? 0x1p-72f : about < 0x1p-99f ? 0x1p75f : 1.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += h[i][j] * power * (h[i][j] * power);
            sum[i] = at.there(i) ? s : 0.f;
        }
        __syncthreads();
        segment_sums<NV>(sum, segments, at.warp_in_row, warps, at.segments);
        __syncthreads();
        total = over_segments(segments, at.segments);
    }
    const float rstd = inverse_root(total, inv_cols, a.eps * power * power) * power;
    if (a.rstd && write && at.warp_in_row == 0 && lane == 0) a.rstd[row] = rstd;
    if (!a.Y && !a.Q) return;
    float top[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float w[1][8];
        load_weights<1>(a.W, a.w_type, w_vec, cols, [&](int) { return at.first(i); }, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * rstd * w[0][j];
        const float t = top8(h[i]);
        top[i] = at.there(i) ? t : 0.f;
    }
    if (a.Y)
#pragma unroll
        for (int i = 0; i < NV; ++i) store_place<T, VEC>((T*)a.Y + row * a.ldy, at.first(i), cols, write, h[i], turn);
    if (!a.Q) return;
    // Blocks of 128 columns are 16 lanes: maxima over these, halving the places that a lane keeps; it ends with place (lane & 15) / 4 (four places) or 0 (one),
    // forms its scale in even lanes and the inverse in odd ones, one division for both, and hands the inverse back.
    constexpr int kLanes = 16 / NV;
    int keep = NV;
#pragma unroll
    for (int d = 8; d; d >>= 1) {
        if (keep > 1) {
            keep >>= 1;
            const bool upper = (lane & d) != 0;
#pragma unroll
            for (int i = 0; i < keep; ++i) {
                const float mine = upper ? top[i + keep] : top[i], theirs = upper ? top[i] : top[i + keep];
                top[i] = top3(mine, __shfl_xor_sync(0xffffffffu, theirs, d), 0.f);
            }
        } else {
            top[0] = top3(top[0], __shfl_xor_sync(0xffffffffu, top[0], d), 0.f);
        }
    }
    const float largest = a.fmt == kE4M3 ? 448.f : 57344.f, u = fmaxf(top[0], kLeastMax);
    const bool finite = __float_as_uint(top[0]) < 0x7f800000u, inverse = (lane & 1) != 0;
    const float ratio = finite ? __fdiv_rn(inverse ? largest : u, inverse ? u : largest) : inverse ? 0.f : __uint_as_float(0x7fffffffu);
    {
        const int col = at.first((lane & 15) / kLanes) + (lane & 16) * 8;
        if ((lane & (kLanes - 1)) == 0 && write && col < cols) a.S[(col >> 7) * a.lds + row] = ratio;
    }
    uint8_t* Q = a.Q + row * a.ldq;
    auto quantise = [&](auto fmt) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint2 q = to_fp8<decltype(fmt)::value>(h[i], __shfl_sync(0xffffffffu, ratio, (lane & 16) + i * kLanes + 1));
            const int col = at.first(i) + lane * 8;
            if (write && col + 8 <= cols) __stcs(reinterpret_cast<uint2*>(Q + col), q);
            else if (write) store8(Q + col, q, cols - col);
        }
    };
    if (a.fmt == kE4M3) quantise(std::integral_constant<int, kE4M3>());
    else quantise(std::integral_constant<int, kE5M2>());
}

template <typename T, int NV, bool VEC, int THREADS>
cudaError_t launch_rows(const RmsNormArgs& a, int warps, int threads, int w_vec, cudaStream_t st) {
    const int here = threads / (32 * warps);
    const double inv_cols = 1.0 / (double)a.cols;
    const Two inv = {(float)inv_cols, (float)(inv_cols - (float)inv_cols)};
    return launch_chained(rms_norm_rows_kernel<T, NV, VEC, THREADS>, dim3((unsigned)((a.rows + here - 1) / here)), dim3(threads), 0, st, a, warps, inv, w_vec);
}

template <typename T, bool VEC>
cudaError_t launch_shape(const RmsNormArgs& a, int w_vec, cudaStream_t st) {
    // Few rows: as many warps to a row as it has segments, for the shortest way through it (16 x 4096 in a graph: 2.7 us; with four segments per warp 3.3 us, when this took 2.9).
    // Many: four segments per warp, whose places share exchanges and divisions.
    const bool few = (a.rows <= 2 * kSms && a.cols <= 32 * kSegment) || a.cols <= 2 * kSegment;
    const int warps = row_warps(a.cols, few ? 1 : 4), threads = few && a.cols > 2 * kSegment ? warps * 32 : block_threads(warps);
    if (few) return launch_rows<T, 1, VEC, 1024>(a, warps, threads, w_vec, st);
    if (threads <= 256) return launch_rows<T, 4, VEC, 256>(a, warps, threads, w_vec, st);
    if (threads <= 512) return launch_rows<T, 4, VEC, 512>(a, warps, threads, w_vec, st);
    return launch_rows<T, 4, VEC, 1024>(a, warps, threads, w_vec, st);
}

template <typename T>
cudaError_t launch_typed(const RmsNormArgs& a, cudaStream_t st, int* launches) {
    const bool vec = aligned8<T>(a.X, a.ldx) && (!a.R || aligned8<T>(a.R, a.ldr)) && (!a.H || aligned8<T>(a.H, a.ldh)) && (!a.Y || aligned8<T>(a.Y, a.ldy)) &&
                     a.cols * sizeof(T) % 16 == 0;
    const int w_vec = ((uintptr_t)a.W & 15) == 0 && a.cols % 8 == 0;
    cudaError_t err = vec ? launch_shape<T, true>(a, w_vec, st) : launch_shape<T, false>(a, w_vec, st);
    if (err != cudaSuccess) return err;
    ++*launches;
    if (!a.Qt) return cudaSuccess;
    err = launch_rms_norm_turned(a, vec, w_vec, st);
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace

cudaError_t launch_rms_norm(const RmsNormArgs& a, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_typed<float>(a, st, launches);
    if (a.type == kF16) return launch_typed<__half>(a, st, launches);
    return launch_typed<__nv_bfloat16>(a, st, launches);
}

}  // namespace gemm2m
