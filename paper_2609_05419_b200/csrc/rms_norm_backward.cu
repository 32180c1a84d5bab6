// Gradients of the root-mean-square norm (rms_norm.cu): with n = H rstd and dN = dY W,
// dX = rn(rstd (dN - n mean_j(dN n)) + dR), dW = (dW) + sum_i dY n.
#include "gemm_ptx.cuh"
#include "rms_norm.cuh"

namespace gemm2m {

namespace {

constexpr int NV = 2;                     // segments of 256 columns per warp
constexpr int64_t kWholeCols = 8192, kSliceCols = 4096;      // columns up to which one block holds a row; those that each of several has

// Blocks of a kernel for so many threads that an SM is to hold.
constexpr int backward_blocks(int threads) { return threads <= 320 ? 2 : 1; }

// Groups of rows, dealt out to the blocks in turn; the sums of dW over a block's rows go to its row of `part`.  SPLIT: a row is shared by the blocks of a cluster, each of which
// has `slice` segments of it; they hand each other their sums (2048 x 16384: 78 us, and 51 for as many
// bytes in 8192 x 4096; in one block with four segments per warp, or in twice the threads, 112).
template <typename T, bool VEC, bool SPLIT, int THREADS>
__global__ void __launch_bounds__(THREADS, backward_blocks(THREADS)) rms_norm_backward_kernel(const RmsNormBackwardArgs a, int warps, int slice, double inv_cols, int w_vec) {
    __shared__ float sums[2][THREADS / 32 * NV];
    __shared__ float slices[2][8];
    __shared__ __align__(16) float turns[VEC ? 1 : THREADS / 32][VEC ? 4 : kSegment];
    extern __shared__ float columns[];                       // rows of a block beyond one: [rows - 1][cols], to add their sums up
    const int shares = SPLIT ? (int)((a.cols + kSegment * slice - 1) / (kSegment * slice)) : 1, share = SPLIT ? (int)cluster_ctarank() : 0;
    const unsigned block = blockIdx.x / shares, blocks = gridDim.x / shares;       // (the cluster's, where a row is shared)
    const Position at(warps, SPLIT ? min(a.cols, (int64_t)(share + 1) * slice * kSegment) : a.cols, SPLIT ? share * slice * kSegment : 0);
    const int lane = at.lane, row_in = at.row_in, warp_in_row = at.warp_in_row, rows_here = at.rows(), cols = at.cols, segments = at.segments;
    float* turn = turns[VEC ? 0 : at.warp];
    auto first_of = [&](int i) { return at.first(i); };
    // Aligned 16-bit numbers: dY and n are held as they came from memory and formed again behind the sum, and what that saves holds the next row, which is on its way meanwhile
    // (8192 x 4096: 51 us; without it 60; with three blocks on an SM instead, whose registers do not suffice, 85).
    constexpr bool kAhead = VEC && sizeof(T) == 2;
    float acc[NV][8], w[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    wait_for_prior_kernels();
    if (SPLIT) cluster_sync_all();                           // (every block of it runs before another writes to its tables)
    load_weights<NV>(a.W, a.w_type, w_vec, cols, first_of, w);
    const int64_t stride = blocks * (int64_t)rows_here;
    struct Row { Place<T, VEC> g[NV], h[NV], r[NV]; float rstd; };
    auto fetch = [&](Row& o, int64_t row) {
        row = min(row, a.rows - 1);
        o.rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) o.g[i].load((const T*)a.dY + row * a.lddy, first_of(i), cols);
#pragma unroll
        for (int i = 0; i < NV; ++i) o.h[i].load((const T*)a.H + row * a.ldh, first_of(i), cols);
        if (a.dR)
#pragma unroll
            for (int i = 0; i < NV; ++i) o.r[i].load((const T*)a.dR + row * a.lddr, first_of(i), cols);
    };
    Row o, ahead;
    if (kAhead) fetch(ahead, block * (int64_t)rows_here + row_in);
    int turn_of = 0;
    for (int64_t first = block * (int64_t)rows_here; first < a.rows; first += stride, turn_of ^= 1) {
        const bool write = first + row_in < a.rows;          // a row beyond the last does the last one's work again, for nothing
        const int64_t row = min(first + row_in, a.rows - 1);
        if (kAhead) {
            o = ahead;
            if (first + stride < a.rows) fetch(ahead, first + stride + row_in);
        } else {
            fetch(o, row);
        }
        auto numbers = [&](int i, float (&dy)[8], float (&n)[8]) {
            o.g[i].get(dy, turn);
            o.h[i].get(n, turn);
#pragma unroll
            for (int j = 0; j < 8; ++j) n[j] *= o.rstd;
        };
        float sum[NV], all_dy[kAhead ? 1 : NV][8], all_n[kAhead ? 1 : NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float new_dy[8], new_n[8], s = 0.f;
            float (&dy)[8] = kAhead ? new_dy : all_dy[kAhead ? 0 : i], (&n)[8] = kAhead ? new_n : all_n[kAhead ? 0 : i];
            numbers(i, dy, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = dy[j] * n[j];
                acc[i][j] += write ? t : 0.f;
                s += t * w[i][j];
            }
            sum[i] = at.there(i) ? s : 0.f;
        }
        // (two tables in turn: a warp may be a row ahead of one that still reads)
        float total = row_sum<NV>(sum, sums[turn_of] + row_in * warps * NV, warp_in_row, warps, segments);
        if constexpr (SPLIT) {
            // every block of the cluster gets every block's sum (two tables in turn, again: a block writes the one of row k + 2 when all have passed the barrier of row k + 1)
            if (threadIdx.x < (unsigned)shares) st_cluster_u32(map_to_cta(smem_u32(&slices[turn_of][share]), threadIdx.x), __float_as_uint(total));
            __syncwarp();
            cluster_sync_all();
            total = 0.f;
            for (int i = 0; i < shares; ++i) total += slices[turn_of][i];
        }
        const float mean = (float)((double)total * inv_cols);
        if constexpr (kAhead) {
            // (the compiler would rather keep the numbers than form them again)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                asm volatile("" : "+r"(o.g[i].raw.w[0].x), "+r"(o.g[i].raw.w[0].y), "+r"(o.g[i].raw.w[0].z), "+r"(o.g[i].raw.w[0].w));
                asm volatile("" : "+r"(o.h[i].raw.w[0].x), "+r"(o.h[i].raw.w[0].y), "+r"(o.h[i].raw.w[0].z), "+r"(o.h[i].raw.w[0].w));
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float new_dy[8], new_n[8], t[8], out[8];
            float (&dy)[8] = kAhead ? new_dy : all_dy[kAhead ? 0 : i], (&n)[8] = kAhead ? new_n : all_n[kAhead ? 0 : i];
            if (kAhead) numbers(i, dy, n);
            if (a.dR) o.r[i].get(t, turn);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                out[j] = o.rstd * (dy[j] * w[i][j] - n[j] * mean);
                if (a.dR) out[j] += t[j];
            }
            store_place<T, VEC>((T*)a.dX + row * a.lddx, first_of(i), cols, write, out, turn);
        }
    }
    if (!a.dW) return;
    // the rows of a block first, in their order
    if (row_in > 0)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (first_of(i) + lane * 8 + j < cols) columns[(row_in - 1) * cols + first_of(i) + lane * 8 + j] = acc[i][j];
    __syncthreads();
    if (row_in > 0) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = first_of(i) + lane * 8 + j;
            if (col >= cols) continue;
            float v = acc[i][j];
            for (int k = 1; k < rows_here; ++k) v += columns[(k - 1) * cols + col];
            a.part[block * a.cols + col] = v;
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

struct BackwardShape { int shares, slice, warps, threads, here, bound; int64_t blocks; };      // blocks: clusters of `shares` blocks
BackwardShape backward_shape(int64_t rows, int64_t cols) {
    BackwardShape s;
    const int segments = (int)((cols + kSegment - 1) / kSegment);
    s.shares = cols <= kWholeCols ? 1 : (int)((cols + kSliceCols - 1) / kSliceCols);
    s.slice = (segments + s.shares - 1) / s.shares;
    s.warps = (s.slice + NV - 1) / NV;
    s.threads = block_threads(s.warps);
    s.here = s.threads / (32 * s.warps);
    s.bound = s.threads <= 256 ? 256 : s.threads <= 320 ? 320 : 512;
    // Clusters: 7/8 of the places, for some of an SM group are left over where its number is no multiple of the cluster's (512 x 32768 in 32
    // bits: 76 us; with 15/16 a second round, 110; with 3/4 86)
    const int64_t places = backward_blocks(s.bound) * (int64_t)kSms, need = (rows + s.here - 1) / s.here, most = s.shares > 1 ? places * 7 / 8 / s.shares : places;
    s.blocks = need < most ? need : most;
    return s;
}

template <typename T, bool VEC, bool SPLIT, int THREADS>
cudaError_t launch_rows(const RmsNormBackwardArgs& a, const BackwardShape& s, int w_vec, cudaStream_t st) {
    const size_t smem = a.dW ? (size_t)(s.here - 1) * a.cols * 4 : 0;      // (at most 7 x 512 columns)
    const dim3 grid((unsigned)(s.blocks * s.shares)), block(s.threads);
    const double inv_cols = 1.0 / (double)a.cols;
    if (SPLIT) return launch_chained_cluster(rms_norm_backward_kernel<T, VEC, SPLIT, THREADS>, grid, block, smem, s.shares, st, a, s.warps, s.slice, inv_cols, w_vec);
    return launch_chained(rms_norm_backward_kernel<T, VEC, SPLIT, THREADS>, grid, block, smem, st, a, s.warps, s.slice, inv_cols, w_vec);
}

template <typename T, bool VEC>
cudaError_t launch_shape(const RmsNormBackwardArgs& a, const BackwardShape& s, int w_vec, cudaStream_t st) {
    if (s.shares > 1) return launch_rows<T, VEC, true, 256>(a, s, w_vec, st);
    if (s.bound == 256) return launch_rows<T, VEC, false, 256>(a, s, w_vec, st);
    return s.bound == 320 ? launch_rows<T, VEC, false, 320>(a, s, w_vec, st) : launch_rows<T, VEC, false, 512>(a, s, w_vec, st);
}

template <typename T>
cudaError_t launch_typed(const RmsNormBackwardArgs& a, cudaStream_t st, int* launches) {
    const BackwardShape s = backward_shape(a.rows, a.cols);
    const bool vec = aligned8<T>(a.dY, a.lddy) && aligned8<T>(a.H, a.ldh) && aligned8<T>(a.dX, a.lddx) && (!a.dR || aligned8<T>(a.dR, a.lddr)) && a.cols * sizeof(T) % 16 == 0;
    const int w_vec = ((uintptr_t)a.W & 15) == 0 && a.cols % 8 == 0;
    cudaError_t err = vec ? launch_shape<T, true>(a, s, w_vec, st) : launch_shape<T, false>(a, s, w_vec, st);
    if (err != cudaSuccess) return err;
    ++*launches;
    if (!a.dW) return cudaSuccess;
    err = launch_chained(rms_norm_dw_kernel, dim3((unsigned)((a.cols + 31) / 32)), dim3(32, 32), 0, st, (const float*)a.part, s.blocks, a.cols, a.dW, a.add);
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace

// Up to the width at which an SM still holds two blocks, what is used grows with both sizes.  Wider rows have fewer blocks; there a bound that does not fall stands in for it: a part for
// each row, and as many entries as at that width (8192 columns in 148 blocks, or up to 4096 times the blocks of a cluster in 259 / that many clusters, are fewer).
int64_t rms_norm_backward_partials(int64_t rows, int64_t cols) {
    constexpr int64_t kTwoBlocks = 320 / 32 * NV * kSegment, kMost = kTwoBlocks * backward_blocks(320) * kSms;
    if (cols <= kTwoBlocks) return backward_shape(rows, cols).blocks * cols;
    return rows < kMost / cols ? rows * cols : kMost;
}

cudaError_t launch_rms_norm_backward(const RmsNormBackwardArgs& a, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_typed<float>(a, st, launches);
    if (a.type == kF16) return launch_typed<__half>(a, st, launches);
    return launch_typed<__nv_bfloat16>(a, st, launches);
}

}  // namespace gemm2m
