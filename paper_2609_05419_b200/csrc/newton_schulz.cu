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
#include "pair_pipeline.cuh"

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

// X_0 in two planes.  The first block of each matrix also leaves |X_0|_F^2, the trace of the first step.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) start_kernel(const T* G, int64_t m, int64_t n, int64_t ldg, int64_t stride_g, const double* parts,
                                                            int nparts, float eps, __half* hi, __half* lo, int64_t ldx, float* trace) {
    __shared__ double scratch[kRowThreads / 32];
    wait_for_prior_kernels();
    const int64_t b = blockIdx.y;
    double sq = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kRowThreads) sq += parts[b * nparts + i];
    sq = block_sum(sq, scratch);
    const double norm = sqrt(sq) + (double)eps;
    const double inv = norm > 0.0 ? (double)(1 << kXExp) / norm : 0.0;       // in 64 bits: 1 / norm of a tiny matrix overflows 32
    if (blockIdx.x == 0)
        if (threadIdx.x == 0) trace[b] = norm > 0.0 ? (float)(sq / (norm * norm)) : 0.f;
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

constexpr int kBM = 128;                  // rows of the first operand per CTA
constexpr int kBK = 64;                   // 16-bit entries of the inner dimension per stage: one 128-byte swizzle row
constexpr int kEpilogueWarps = 8;
constexpr int kGemmThreads = 64 + 32 * kEpilogueWarps;

template <int BN>
struct Cfg {
    static constexpr int kHalfRows = BN / 2;              // rows of the second operand per CTA
    static constexpr int kStageBytes = (kBM + kHalfRows) * 128;
    static constexpr int kStages = BN == 256 ? 6 : 8;
    static constexpr int kCols = BN / 2;                  // columns per epilogue warp
    static constexpr uint32_t kTmemCols = 2 * BN;
    static constexpr size_t kPipeBytes = (PairPipe<kStages>::kBytes + 15) / 16 * 16;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 + kPipeBytes + kEpilogueWarps * 4096;
};

struct NsGemm {
    int mode;
    int M, N, kblocks, batch;
    int tiles_r, tiles_c, tiles;                          // row and column tiles of a matrix, and how many of them are computed
    float a, b, c, short_side;
    const float* trace; int64_t trace_parts;              // kGram: partial sums of |X|_F^2, or null for g = 0
    float* shift;                                         // g of every matrix: written by kGram, read by the others
    __half* out; int64_t ldo, stride_o;                   // kGram, kPoly: symmetric square, times 2^kSExp
    const __half* gram;                                   // kPoly: A', laid out as out
    const __half *hi, *lo; __half *hi_out, *lo_out; float* trace_out; int64_t ldx, stride_x;      // kUpdate, kLast
    __nv_bfloat16* last; int64_t ld_last, stride_last; int last_vec;                              // kLast
    uint32_t idesc;
    int* dev_status;
    unsigned long long wait_ns;
};

__device__ __forceinline__ void umma_f16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor of kind::f16: half-precision operands, 32-bit accumulator; turned = the operand's rows are contiguous.
uint32_t make_idesc_f16(bool turned_a, bool turned_b, int M, int N) {
    return (1u << 4) | ((uint32_t)turned_a << 15) | ((uint32_t)turned_b << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Shared-memory descriptor of an operand whose rows are contiguous (128-byte swizzle): pieces of 64 rows x 8 inner entries are
// 1024 bytes; the next 8 inner entries follow 1024 bytes on, the next 64 rows 64 x 128 bytes on.
__device__ __forceinline__ uint64_t make_smem_desc_turned(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(8192 >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// This CTA's `rows` rows from row0 and one stage of the inner dimension.
template <bool TURNED>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, uint32_t bar, int kb, int row0, int rows, int b) {
    if (!TURNED) {
        tma_load_3d_pair(dst, map, bar, kb * kBK, row0, b);
    } else {
        for (int r = 0; r < rows; r += 64) tma_load_3d_pair(dst + r * 128, map, bar, row0 + r, kb * kBK, b);
    }
}

// Tile `t` of a launch: matrix, row tile, column tile.  A symmetric square has the tiles up to and including the diagonal block's:
// row tile r has q (r + 1) of them, q = column tiles per row tile.
template <int BN>
__device__ __forceinline__ void tile_at(const NsGemm& p, int t, int* b, int* tr, int* tc) {
    constexpr int q = 2 * kBM / BN;
    *b = t / p.tiles;
    const int i = t - *b * p.tiles;
    if (p.mode == kGram || p.mode == kPoly) {
        int r = (int)((sqrtf(8.f * (float)(i / q) + 1.f) - 1.f) * 0.5f);
        while (q * r * (r + 1) / 2 > i) --r;              // (rounding of the root)
        while (q * (r + 1) * (r + 2) / 2 <= i) ++r;
        *tr = r;
        *tc = i - q * r * (r + 1) / 2;
    } else {                                              // bands of 8 row tiles, column by column: operands are shared through L2
        const int band = i / (8 * p.tiles_c), in_band = i - band * 8 * p.tiles_c, rows = min(8, p.tiles_r - 8 * band);
        *tc = in_band / rows;
        *tr = 8 * band + in_band - *tc * rows;
    }
}

struct alignas(8) Half4 { __half h[4]; };
struct alignas(8) Bf4 { __nv_bfloat16 h[4]; };

// 32 columns of 32 rows (v: this lane's row), at (row0, col0) of matrix b.  The values turn in shared memory (16-byte pieces XORed
// with the row) so that eight lanes have four columns each of one row, and what is read and written beside them is whole
// sectors.  Planes have padded rows, so that four columns can always be touched; what lies in the padding is not used.
__device__ __forceinline__ float finish_block(const NsGemm& p, const uint32_t (&v)[32], uint32_t turn, int b, int row0, int col0, bool mirror, float g) {
    const int lane = threadIdx.x & 31, piece = lane & 7;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (uint32_t)(lane * 128 + ((q ^ (lane & 7)) << 4))), "r"(v[4 * q]), "r"(v[4 * q + 1]),
                     "r"(v[4 * q + 2]), "r"(v[4 * q + 3]) : "memory");
    __syncwarp();
    const int col = col0 + piece * 4;
    const int rows = col < p.N ? min(32, p.M - row0) : 0;
    const float gram_scale = exp2f(kSExp - 2 * kXExp), g_scaled = g * exp2f(kSExp);
    const float poly_lin = p.b + 2.f * p.c * g, poly_sq = p.c * exp2f(-kSExp);
    const float x_lin = p.a + g * (p.b + p.c * g);
    float sum = 0.f;
#pragma unroll 2
    for (int r = lane >> 3; r < rows; r += 4) {
        float x[4];
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3])
                     : "r"(turn + (uint32_t)(r * 128 + ((piece ^ (r & 7)) << 4))) : "memory");
        const int row = row0 + r;
        if (p.mode == kGram || p.mode == kPoly) {
            const int64_t at = (int64_t)b * p.stride_o + (int64_t)row * p.ldo + col;
            Half4 o;
            if (p.mode == kGram) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o.h[j] = __float2half_rn(x[j] * gram_scale - (row == col + j ? g_scaled : 0.f));
            } else {
                const Half4 s = *reinterpret_cast<const Half4*>(p.gram + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) o.h[j] = __float2half_rn(poly_lin * __half2float(s.h[j]) + poly_sq * x[j]);
            }
            *reinterpret_cast<Half4*>(p.out + at) = o;
        } else {
            const int64_t at = (int64_t)b * p.stride_x + (int64_t)row * p.ldx + col;
            const Half4 h = *reinterpret_cast<const Half4*>(p.hi + at), l = *reinterpret_cast<const Half4*>(p.lo + at);
            float w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = x_lin * (__half2float(h.h[j]) + __half2float(l.h[j]) * exp2f(-kLoExp)) + x[j] * exp2f(-kSExp);
            if (p.mode == kUpdate) {
                Half4 ho, lo;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    ho.h[j] = __float2half_rn(w[j]);
                    lo.h[j] = __float2half_rn((w[j] - __half2float(ho.h[j])) * exp2f(kLoExp));
                    if (col + j < p.N) sum += w[j] * w[j];
                }
                *reinterpret_cast<Half4*>(p.hi_out + at) = ho;
                *reinterpret_cast<Half4*>(p.lo_out + at) = lo;
            } else {
                __nv_bfloat16* d = p.last + (int64_t)b * p.stride_last + (int64_t)row * p.ld_last + col;
                Bf4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o.h[j] = __float2bfloat16_rn(w[j] * exp2f(-kXExp));
                if (p.last_vec && col + 4 <= p.N) *reinterpret_cast<Bf4*>(d) = o;
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col + j < p.N) d[j] = o.h[j];
            }
        }
    }
    if (mirror && row0 + lane < p.M) {                    // the same numbers at (column, row): 32 lanes are 32 neighbours there
        const int64_t base = (int64_t)b * p.stride_o + row0 + lane;
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            if (col0 + c >= p.N) break;
            const int64_t at = base + (int64_t)(col0 + c) * p.ldo;
            const float x = __uint_as_float(v[c]);
            p.out[at] = __float2half_rn(p.mode == kGram ? x * gram_scale : poly_lin * __half2float(p.gram[at]) + poly_sq * x);
        }
    }
    return sum;
}

// g = trace(A) / s of matrix b, by one warp, from the partial sums in their order.
__device__ __forceinline__ float shift_of(const NsGemm& p, int b) {
    if (p.mode != kGram) return p.shift[b];
    if (!p.trace) return 0.f;
    double t = 0.0;
    for (int64_t i = threadIdx.x & 31; i < p.trace_parts; i += 32) t += (double)p.trace[(int64_t)b * p.trace_parts + i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    return (float)(t / (double)p.short_side);
}

template <int BN, bool TURNED_A, bool TURNED_B>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
ns_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ NsGemm p) {
    using cfg = Cfg<BN>;
    constexpr int STAGES = cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles_base = (raw + 1023u) & ~1023u;
    unsigned char* behind = smem_raw + (tiles_base - raw) + (size_t)STAGES * cfg::kStageBytes;
    PairPipe<STAGES> pipe;
    pipe.open(behind, kEpilogueWarps, 1, cfg::kTmemCols, p.dev_status, p.wait_ns);
    wait_for_prior_kernels();

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    const int total_tiles = p.tiles * p.batch;

    if (warp == 0) {
        if (lane == 0) {                                  // copies, both CTAs
            const uint32_t leader_full = map_to_cta(pipe.full, 0);
            RingPos<STAGES> at;
            uint32_t fills = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
                int b, tr, tc;
                tile_at<BN>(p, tile, &b, &tr, &tc);
                const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM, col0 = tc * BN + (int)pipe.rank * cfg::kHalfRows;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!(ok = pipe.wait(pipe.empty + 8 * at.stage, at.phase ^ 1u, kDevTimeoutProducer))) break;
                    const uint32_t dst = tiles_base + at.stage * cfg::kStageBytes;
                    if (pipe.rank == 0) mbar_arrive_expect_tx(pipe.full + 8 * at.stage, 2 * cfg::kStageBytes);
                    load_operand<TURNED_A>(dst, &map_a, leader_full + 8 * at.stage, kb, row0, kBM, b);
                    load_operand<TURNED_B>(dst + kBM * 128, &map_b, leader_full + 8 * at.stage, kb, col0, cfg::kHalfRows, b);
                    ++fills;
                    at.next();
                }
            }
            *pipe.fills_issued = fills;
            if (!ok) pipe.tell_peer();
        }
    } else if (warp == 1) {
        if (lane == 0 && pipe.rank == 0) {                // MMAs, leader
            RingPos<STAGES> at;
            uint32_t it = 0;                              // tile counter: buffer it & 1, its use number it >> 1
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs, ++it) {
                const uint32_t buf = it & 1u;
                if (!(ok = pipe.wait(pipe.tempty + 8 * buf, ((it >> 1) & 1u) ^ 1u, kDevTimeoutMma))) break;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!(ok = pipe.wait(pipe.full + 8 * at.stage, at.phase, kDevTimeoutMma))) break;
                    tcgen05_fence_after();
                    const uint32_t a_addr = tiles_base + at.stage * cfg::kStageBytes, b_addr = a_addr + kBM * 128;
                    const uint64_t adesc = TURNED_A ? make_smem_desc_turned(a_addr) : make_smem_desc(a_addr);
                    const uint64_t bdesc = TURNED_B ? make_smem_desc_turned(b_addr) : make_smem_desc(b_addr);
                    // 16 inner entries: 32 bytes along a swizzle row, or 16 rows of 128 bytes
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4)
                        umma_f16_pair(pipe.tmem + buf * BN, adesc + (uint64_t)(k4 * (TURNED_A ? 128 : 2)), bdesc + (uint64_t)(k4 * (TURNED_B ? 128 : 2)), p.idesc,
                                      (uint32_t)((kb | k4) != 0));
                    umma_commit_pair(pipe.empty + 8 * at.stage, 3);
                    at.next();
                }
                if (ok) umma_commit_pair(pipe.tfull + 8 * buf, 3);
            }
            if (!ok) pipe.tell_peer();
        }
    } else {
        // Epilogue: warp w reads lanes 32 (w & 3) .. of TMEM (rows), columns of half (w - 2) / 4.
        const int half = (warp - 2) >> 2, quarter = warp & 3;
        constexpr int NC = cfg::kCols;
        const uint32_t turn = smem_u32(behind) + (uint32_t)cfg::kPipeBytes + (uint32_t)(warp - 2) * 4096;
        const uint32_t leader_tempty = map_to_cta(pipe.tempty, 0);
        uint32_t it = 0;
        int shift_for = -1;
        float g = 0.f;
        bool ok = true;
        for (int tile = pair; ok && tile < total_tiles; tile += npairs, ++it) {
            int b, tr, tc;
            tile_at<BN>(p, tile, &b, &tr, &tc);
            const uint32_t buf = it & 1u;
            if (b != shift_for) {
                g = shift_of(p, b);
                shift_for = b;
            }
            if (p.mode == kGram && tr == 0 && tc == 0 && pipe.rank == 0 && warp == 2 && lane == 0) p.shift[b] = g;
            ok = __all_sync(0xffffffffu, pipe.wait(pipe.tfull + 8 * buf, (it >> 1) & 1u, kDevTimeoutEpilogue));
            if (!ok) break;
            tcgen05_fence_after();
            const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM + quarter * 32, col0 = tc * BN + half * NC;
            const bool mirror = (p.mode == kGram || p.mode == kPoly) && (tc + 1) * BN <= tr * 2 * kBM;      // below the diagonal block
            const uint32_t taddr = pipe.tmem + ((uint32_t)(quarter * 32) << 16) + buf * BN + (uint32_t)(half * NC);
            float sum = 0.f;
#pragma unroll 1
            for (int c = 0; c < NC; c += 32) {
                uint32_t v[32];
                tmem_ld32(taddr + c, v);
                tmem_ld_wait();
                if (c + 32 == NC) pipe.release_at(leader_tempty + 8 * buf);
                if (row0 < p.M && col0 + c < p.N) sum += finish_block(p, v, turn, b, row0, col0 + c, mirror, g);
                // one partial sum per 32 rows and 64 columns, whatever the tile width: results do not depend on that choice
                if (p.mode == kUpdate && (c & 32)) {
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    const int part_row = row0 >> 5, part_col = (col0 + c) >> 6, cols = (p.N + 63) >> 6;
                    if (lane == 0 && row0 < p.M && part_col < cols) p.trace_out[(int64_t)b * p.trace_parts + (int64_t)part_row * cols + part_col] = sum * exp2f(-2 * kXExp);
                    sum = 0.f;
                }
            }
        }
        if (!ok && lane == 0) pipe.tell_peer();
    }
    pipe.close(cfg::kTmemCols, cfg::kStageBytes);
}

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Partial sums of the trace that an update of m x n matrices leaves.
inline int64_t update_trace_parts(int64_t m, int64_t n) { return (m + 31) / 32 * ((n + 63) / 64); }

// One operand of a product, rows x inner entries of `batch` matrices `stride` apart: element (r, k) at r ld + k, or at k ld + r if turned.
struct Operand { const __half* p; int64_t rows, inner, ld, stride; bool turned; };

bool make_half_map(CUtensorMap* map, const Operand& o, int64_t batch, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)(o.turned ? o.rows : o.inner), (cuuint64_t)(o.turned ? o.inner : o.rows), (cuuint64_t)batch};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)(o.turned ? kBK : box_rows), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(o.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool TURNED_A, bool TURNED_B>
cudaError_t launch_tiles(NsGemm& q, const Operand& A, const Operand& B, int sm_count, cudaStream_t st, int* launches) {
    using cfg = Cfg<BN>;
    static int pairs_dev[kMaxDevices] = {};
    int& max_pairs = pairs_dev[current_device_slot()];
    if (!max_pairs) {
        int pairs = 0;
        cudaError_t err = resident_pairs(ns_gemm_pair_kernel<BN, TURNED_A, TURNED_B>, kGemmThreads, cfg::kSmem, sm_count, &pairs);
        if (err != cudaSuccess) return err;
        max_pairs = pairs;
    }
    CUtensorMap map_a, map_b;
    if (!make_half_map(&map_a, A, q.batch, kBM) || !make_half_map(&map_b, B, q.batch, cfg::kHalfRows)) return cudaErrorInvalidValue;
    q.tiles_r = (q.M + 2 * kBM - 1) / (2 * kBM);
    q.tiles_c = (q.N + BN - 1) / BN;
    constexpr int per = 2 * kBM / BN;
    // (a square's last row tile has all of its column tiles, the others those up to the diagonal block)
    const int64_t all = q.mode == kGram || q.mode == kPoly ? (int64_t)per * q.tiles_r * (q.tiles_r - 1) / 2 + q.tiles_c : (int64_t)q.tiles_r * q.tiles_c;
    if (all * q.batch > INT32_MAX / 4) return cudaErrorInvalidValue;
    q.tiles = (int)all;
    q.idesc = make_idesc_f16(TURNED_A, TURNED_B, 2 * kBM, BN);
    const int pairs = (int)(all * q.batch < max_pairs ? all * q.batch : max_pairs);
    cudaError_t err = launch_chained(ns_gemm_pair_kernel<BN, TURNED_A, TURNED_B>, dim3(2 * pairs), dim3(kGemmThreads), cfg::kSmem, st, map_a, map_b, q);
    if (err == cudaSuccess) ++*launches;
    return err;
}

template <int BN>
cudaError_t launch_width(NsGemm& q, const Operand& A, const Operand& B, int sm_count, cudaStream_t st, int* launches) {
    if (A.turned) return launch_tiles<BN, true, true>(q, A, B, sm_count, st, launches);        // X^T X
    if (B.turned) return launch_tiles<BN, false, true>(q, A, B, sm_count, st, launches);       // P X
    return launch_tiles<BN, false, false>(q, A, B, sm_count, st, launches);
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
                         (float*)(a.ws + l.off_trace[0]));
    if (err == cudaSuccess) *launches += 2;
    return err;
}

// Whether a product's tiles are 256 or 128 columns wide: whichever makes the last pair finish first, a narrow tile counted as
// 0.55 of a wide one (half the MMAs, three quarters of the operand bytes).
bool wide_tiles(int64_t wide, int64_t narrow, int64_t pairs) {
    return (double)((wide + pairs - 1) / pairs) <= 0.55 * (double)((narrow + pairs - 1) / pairs);
}

}  // namespace

NewtonSchulzLayout newton_schulz_layout(int64_t batch, int64_t m, int64_t n, int64_t offset) {
    NewtonSchulzLayout l = {};
    const int64_t s = m < n ? m : n;
    l.ldx = round_up(n, 64);
    l.lds = round_up(s, 64);
    l.norm_parts = kNormParts;
    l.trace_parts = update_trace_parts(m, n);
    int64_t off = round_up(offset, 256);
    auto take = [&](int64_t bytes) { int64_t o = off; off = round_up(off + bytes, 256); return o; };
    l.off_norm = take(8 * batch * l.norm_parts);
    l.off_shift = take(4 * batch);
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
    cudaError_t err = a.type == kF32 ? launch_start<float>(a, st, &launches[0])
                      : a.type == kF16 ? launch_start<__half>(a, st, &launches[0]) : launch_start<__nv_bfloat16>(a, st, &launches[0]);
    if (err != cudaSuccess) return err;
    const NewtonSchulzLayout& l = a.lay;
    const bool tall = a.m > a.n;
    const int64_t s = tall ? a.n : a.m, L = tall ? a.m : a.n;
    __half* gram = (__half*)(a.ws + l.off_gram);
    __half* poly = (__half*)(a.ws + l.off_poly);
    // Tile width of every product (see wide_tiles)
    const int64_t rt = (s + 255) / 256, pairs = sm_count / 2;
    auto width = [&](int64_t wide, int64_t narrow) { return wide_tiles(wide * a.batch, narrow * a.batch, pairs); };
    const bool wide_square = width(rt * (rt - 1) / 2 + (s + 255) / 256, rt * (rt - 1) + (s + 127) / 128);
    const int64_t mt = (a.m + 255) / 256;
    const bool wide_update = width(mt * ((a.n + 255) / 256), mt * ((a.n + 127) / 128));
    for (int k = 0; k < a.steps; ++k) {
        const __half* hi = (const __half*)(a.ws + l.off_hi[k & 1]);
        const int64_t sx = a.m * l.ldx, ss = s * l.lds;
        const Operand x_rows = {hi, a.m, a.n, l.ldx, sx, false}, x_cols = {hi, a.n, a.m, l.ldx, sx, true};
        NsGemm q = {};
        q.batch = (int)a.batch;
        q.short_side = (float)s;
        q.a = a.coeffs[3 * k]; q.b = a.coeffs[3 * k + 1]; q.c = a.coeffs[3 * k + 2];
        q.trace = k + 2 >= a.steps ? (const float*)(a.ws + l.off_trace[k & 1]) : nullptr;
        q.trace_parts = k == 0 ? 1 : l.trace_parts;
        q.shift = (float*)(a.ws + l.off_shift);
        q.ldo = l.lds; q.stride_o = ss;
        q.ldx = l.ldx; q.stride_x = sx;
        q.dev_status = a.dev_status;
        q.wait_ns = kWaitLimitNs;
        auto run = [&](const Operand& A, const Operand& B, int64_t K, bool wide) {
            q.M = (int)A.rows; q.N = (int)B.rows;
            q.kblocks = (int)((K + kBK - 1) / kBK);
            return wide ? launch_width<256>(q, A, B, sm_count, st, &launches[1]) : launch_width<128>(q, A, B, sm_count, st, &launches[1]);
        };
        // A' = X X^T - g I  (X^T X for a tall matrix)
        q.mode = kGram;
        q.out = gram;
        if ((err = run(tall ? x_cols : x_rows, tall ? x_cols : x_rows, L, wide_square)) != cudaSuccess) return err;
        // P = (b + 2 c g) A' + c A'^2
        const Operand sq = {gram, s, s, l.lds, ss, false}, p = {poly, s, s, l.lds, ss, false};
        q.mode = kPoly;
        q.gram = gram; q.out = poly;
        if ((err = run(sq, sq, s, wide_square)) != cudaSuccess) return err;
        // X <- (a + b g + c g^2) X + P X  (X P for a tall matrix; P is symmetric)
        q.mode = k + 1 == a.steps ? kLast : kUpdate;
        q.hi = hi; q.lo = (const __half*)(a.ws + l.off_lo[k & 1]);
        q.hi_out = (__half*)(a.ws + l.off_hi[(k + 1) & 1]);
        q.lo_out = (__half*)(a.ws + l.off_lo[(k + 1) & 1]);
        q.trace_out = (float*)(a.ws + l.off_trace[(k + 1) & 1]);
        q.trace_parts = l.trace_parts;
        q.last = (__nv_bfloat16*)a.O; q.ld_last = a.ldo; q.stride_last = a.stride_o;
        q.last_vec = ((uintptr_t)a.O & 7) == 0 && a.ldo % 4 == 0 && a.stride_o % 4 == 0;
        if ((err = run(tall ? x_rows : p, tall ? p : x_cols, s, wide_update)) != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace gemm2m
