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
// later step.)  All planes are scaled by powers of two into the middle of the 16-bit range.  Against 64 bits the result of five
// default steps (this arithmetic on the CPU, before the rounding to bf16, which is 1.7e-3) is off by 4e-4 .. 2.4e-3 of its norm for sides from 64 up
// (flat, k^-1/2 and k^-1 spectra, full rank and a third of it; rows and singular values down to 1e-3 of the largest), by up to 5e-3 between 20 and
// 64 and 9e-3 below; rounding the iterate to 16 bits instead costs up to 2e-2, all planes in bf16 up to 2e-1.  More steps, or coefficients
// with steeper slopes, multiply the rounding of the steps before: ten default steps 8e-3, 1 % damped steep sets 5e-3, undamped ones 4e-2 and more.
//
// Work.  A and A^2 are symmetric: only tiles on and below the diagonal are computed, and written twice.  Per step
// s^2 l + s^3 + 2 s^2 l operations.  One cooperative launch runs all steps (ns_steps_kernel).  4096^2, five steps: 1.16 to 1.21 ms in a short run, tensor
// pipe 63 % active, 1.18 PFLOP/s of the operations above, and 1.41 ms in a steady stream of calls at the board's power limit; 16384 x 4096 in 32 bits:
// 3.8 and 4.4 ms; 16 x 1024^2: 553 and 637 us.  Small
// matrices are bound by the chain of each of the 15 products (counter, first copies, MMAs, epilogue, fence: about 5 us).
#include "layer_ops.cuh"
#include "pair_pipeline.cuh"

namespace gemm2m {

namespace {

constexpr int kXExp = 8;              // hi = rn16(2^8 X): entries of X are at most about 1.2; 255 fit
constexpr int kLoExp = 11;            // lo = rn16(2^11 (2^8 X - hi))
constexpr int kSExp = 4;              // A' and the polynomial are held times 2^4: entries up to 4094 fit, so singular values below 64
constexpr int kNormParts = 592;       // partial sums of |G|_F^2 per matrix
constexpr int kRowThreads = 256;

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

// The matrix is walked in groups of eight entries of a row, kUnroll groups per thread in flight (rows that are not 16-byte aligned are
// read entry by entry).  HBM-bound: 16384 x 4096 f32, norm 45 us (268 MB, 5.9 TB/s), start 89 us (537 MB, 6.0 TB/s).
constexpr int kUnroll = 4;

// Groups i, i + stride, ..: their entries, and (at) where they go in a plane with rows of ldx, -1 behind the last group.
template <typename T>
__device__ __forceinline__ void load_groups(Raw8<T> (&raw)[kUnroll], int64_t* at, const T* g, int64_t i, int64_t stride, int64_t groups, uint32_t per_row, int64_t n,
                                            int64_t ldg, int vec, int64_t ldx) {
    if (vec && i + (kUnroll - 1) * stride < groups) {      // vec: every group is whole and aligned
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t k = i + u * stride, row = k / per_row, col = (k - row * per_row) * 8;
            raw[u] = load8<T>(g + row * ldg + col);
            if (at) at[u] = row * ldx + col;
        }
    } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t k = i + u * stride, row = k / per_row, col = (k - row * per_row) * 8;
            raw[u] = load8_part<T>(g + row * ldg + col, k < groups ? n - col : 0);
            if (at) at[u] = k < groups ? row * ldx + col : -1;
        }
    }
}

// |G|_F^2, one partial sum per block, in 64 bits (a square of a 32-bit number always fits).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_kernel(const T* G, int64_t groups, uint32_t per_row, int64_t n, int64_t ldg, int64_t stride_g, int vec, double* parts) {
    __shared__ double scratch[kRowThreads / 32];
    wait_for_prior_kernels();
    const T* g = G + (int64_t)blockIdx.y * stride_g;
    const int64_t stride = (int64_t)gridDim.x * kRowThreads;
    double s = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; i < groups; i += kUnroll * stride) {
        Raw8<T> raw[kUnroll];
        load_groups<T>(raw, nullptr, g, i, stride, groups, per_row, n, ldg, vec, 0);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float v[8];
            to_floats8<T>(raw[u], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (double)v[j] * (double)v[j];
        }
    }
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// X_0 in two planes.  The first block of each matrix also leaves |X_0|_F^2, the trace of the first step.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) start_kernel(const T* G, int64_t groups, uint32_t per_row, int64_t m, int64_t n, int64_t ldg, int64_t stride_g, int vec,
                                                            const double* parts, int nparts, float eps, __half* hi, __half* lo, int64_t ldx, float* trace, uint32_t* phase_count, uint32_t* part_count,
                                                            int64_t part_counts) {
    __shared__ double scratch[kRowThreads / 32];
    wait_for_prior_kernels();
    const int64_t b = blockIdx.y;
    double sq = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kRowThreads) sq += parts[b * nparts + i];
    sq = block_sum(sq, scratch);
    const double norm = sqrt(sq) + (double)eps;
    const double inv = norm > 0.0 ? (double)(1 << kXExp) / norm : 0.0;
    const bool in32 = inv > 1e-30 && inv < 1e30;           // 1 / norm of a tiny matrix overflows 32 bits
    const float inv32 = (float)inv;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (b == 0) *phase_count = 0;
        trace[b] = norm > 0.0 ? (float)(sq / (norm * norm)) : 0.f;
    }
    if (b == 0)
        for (int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; i < part_counts; i += (int64_t)gridDim.x * kRowThreads) part_count[i] = 0;
    const T* g = G + b * stride_g;
    const int64_t stride = (int64_t)gridDim.x * kRowThreads;
    for (int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; i < groups; i += kUnroll * stride) {
        Raw8<T> raw[kUnroll];
        int64_t at[kUnroll];
        load_groups<T>(raw, at, g, i, stride, groups, per_row, n, ldg, vec, ldx);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (at[u] < 0) continue;
            float v[8];
            to_floats8<T>(raw[u], v);
            __half h[8], l[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = in32 ? v[j] * inv32 : (float)((double)v[j] * inv);
                h[j] = __float2half_rn(x);
                l[j] = __float2half_rn((x - __half2float(h[j])) * (float)(1 << kLoExp));
            }
            *reinterpret_cast<uint4*>(hi + b * m * ldx + at[u]) = *reinterpret_cast<const uint4*>(h);      // (rows of the planes are padded)
            *reinterpret_cast<uint4*>(lo + b * m * ldx + at[u]) = *reinterpret_cast<const uint4*>(l);
        }
    }
}

constexpr int kBM = 128;                  // rows of the first operand per CTA
constexpr int kBK = 64;                   // 16-bit entries of the inner dimension per stage: one 128-byte swizzle row
constexpr int kStages = 5;
constexpr int kBoxBytes = 64 * 128;       // a copy: 64 rows x 64 inner entries, in either order
constexpr int kStageBytes = 4 * kBoxBytes;
constexpr int kEpilogueWarps = 8;
// Warps 0 and 1 copy operands and issue MMAs, 2 and 3 do nothing, 4 .. 11 are the epilogue, which holds a block's operands ahead and
// needs more registers than an equal share (168): 128 x 40 + 256 x 232 = 384 x 168.
constexpr int kFirstEpilogueWarp = 4;
constexpr int kGemmThreads = 32 * (kFirstEpilogueWarp + kEpilogueWarps);
constexpr int kLaunchRegs = 168, kPipeRegs = 40, kEpilogueRegs = 232;
static_assert(128 * kPipeRegs + 32 * kEpilogueWarps * kEpilogueRegs <= kGemmThreads * kLaunchRegs, "register shares exceed what the block is launched with");
constexpr int kMaxSteps = 64;
constexpr size_t kPipeBytes = (PairPipe<kStages>::kBytes + 15) / 16 * 16;
constexpr size_t kGemmSmem = (size_t)kStages * kStageBytes + 1024 + kPipeBytes;

enum Mode { kGram, kPoly, kUpdate, kLast };

struct NsParams {
    // The iterate's hi planes, A' and the polynomial in boxes of 64 and 128 rows by 64 inner entries; the iterate turned, in boxes of 64
    // inner entries (rows of the matrix) by one and two groups of 64 of its columns.
    CUtensorMap x[2][2], gram_map[2], poly_map[2], x_turned[2][2];
    int m, n, s, batch, steps;
    int square_width, update_width;                       // columns of a tile: 256, 128 or 64
    float coeffs[3 * kMaxSteps];
    float* trace[2]; int64_t trace_parts;           // partial sums of |X|_F^2 (one in front of the first step)
    int splits; float* part; uint32_t* part_count;        // A' in pieces along its inner dimension (see kGram's epilogue)
    float* shift;                                         // g of every matrix: written with A', read by the rest of the step
    __half *gram, *poly; int64_t lds;                     // s x s, times 2^kSExp
    __half *hi[2], *lo[2]; int64_t ldx;                   // m x n
    __nv_bfloat16* out; int64_t ld_out, stride_out; int out_vec;
    uint32_t* phase_count;                                // CTAs that have finished a phase, over all phases so far
    int* dev_status;
    unsigned long long wait_ns;
};

// One product of a step: kind 0 A' = X X^T - g I, 1 P = (b + 2 c g) A' + c A'^2, 2 X <- (a + b g + c g^2) X + P X.
struct Phase {
    int mode, M, N, kblocks, bn, tiles_r, tiles_c, tiles;
    int splits, items;                                    // pieces of the inner dimension per tile; tiles and pieces of all matrices
    bool turned_a, turned_b;
    const CUtensorMap *map_a, *map_b;
};
__host__ __device__ inline int square_tiles(int tiles_r, int tiles_c, int per) { return per * tiles_r * (tiles_r - 1) / 2 + tiles_c; }
template <bool PIECES>
__device__ __forceinline__ Phase phase_at(const NsParams& p, int step, int kind) {
    Phase q;
    const bool tall = p.m > p.n;
    q.mode = kind == 0 ? kGram : kind == 1 ? kPoly : step + 1 == p.steps ? kLast : kUpdate;
    q.bn = kind == 2 ? p.update_width : p.square_width;
    q.M = kind == 2 ? p.m : p.s;
    q.N = kind == 2 ? p.n : p.s;
    q.kblocks = ((kind == 0 ? (tall ? p.m : p.n) : p.s) + kBK - 1) / kBK;
    q.tiles_r = (q.M + 2 * kBM - 1) / (2 * kBM);
    q.tiles_c = (q.N + q.bn - 1) / q.bn;
    q.tiles = kind == 2 ? q.tiles_r * q.tiles_c : square_tiles(q.tiles_r, q.tiles_c, 2 * kBM / q.bn);
    q.splits = PIECES && kind == 0 ? p.splits : 1;
    q.items = q.tiles * p.batch * q.splits;
    q.turned_a = kind == 0 && tall;                       // X^T X contracts along the rows of X
    q.turned_b = (kind == 0 && tall) || (kind == 2 && !tall);
    const CUtensorMap* x = p.x[step & 1];
    const CUtensorMap* x_turned = p.x_turned[step & 1];
    q.map_a = kind == 0 ? (tall ? x_turned : x) : kind == 1 ? p.gram_map : tall ? x : p.poly_map;
    q.map_b = kind == 0 ? (tall ? x_turned : x) : kind == 1 ? p.gram_map : tall ? p.poly_map : x_turned;
    return q;
}

__device__ __forceinline__ void umma_f16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor of kind::f16: half-precision operands, 32-bit accumulator; turned = the operand's rows are contiguous.
__device__ __forceinline__ uint32_t make_idesc_f16(bool turned_a, bool turned_b, int M, int N) {
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
// `rows` (32, 64 or 128) rows from row0 and one stage of the inner dimension, in one copy (a copy is 64 rows at least).  One copy per
// operand and stage instead of one per 64 rows: 4096 x 4096, five steps, 1270 against 1376 us.
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, uint32_t bar, bool turned, int kb, int row0, int rows, int b) {
    if (!turned) {
        tma_load_3d_pair(dst, map + (rows == 128), bar, kb * kBK, row0, b);
    } else {
        asm volatile(
            "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
            ::"r"(dst), "l"(map + (rows == 128)), "r"(bar), "r"(row0 & 63), "r"(kb * kBK), "r"(row0 >> 6), "r"(b)
            : "memory");
    }
}

// Tile `t` of a phase: matrix, row tile, column tile.  A symmetric square has the tiles up to and including the diagonal block's:
// row tile r has per (r + 1) of them, per = column tiles per row tile.
__device__ __forceinline__ void tile_at(const Phase& q, int t, int* b, int* tr, int* tc) {
    *b = t / q.tiles;
    const int i = t - *b * q.tiles;
    if (q.mode == kGram || q.mode == kPoly) {
        const int per = 2 * kBM / q.bn;
        int r = (int)((sqrtf(8.f * (float)(i / per) + 1.f) - 1.f) * 0.5f);
        while (per * r * (r + 1) / 2 > i) --r;            // (rounding of the root)
        while (per * (r + 1) * (r + 2) / 2 <= i) ++r;
        *tr = r;
        *tc = i - per * r * (r + 1) / 2;
    } else {                                              // bands of 8 row tiles, column by column: operands are shared through L2
        const int band = i / (8 * q.tiles_c), in_band = i - band * 8 * q.tiles_c, rows = min(8, q.tiles_r - 8 * band);
        *tc = in_band / rows;
        *tr = 8 * band + in_band - *tc * rows;
    }
}

// Waits (bounded) until `target` CTAs in all have finished their phases, and sees what they wrote.  (The look itself is relaxed: an
// acquire every time would empty the SM's L1 under the warps that still work.)
__device__ __forceinline__ bool wait_for_phase(const NsParams& p, uint32_t target, volatile int* abort_flag, bool patient) {
    const unsigned long long t0 = global_timer_ns();
    for (uint32_t spins = 1;; ++spins) {
        uint32_t seen;
        asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(p.phase_count) : "memory");
        if (seen >= target) break;
        if (patient) __nanosleep(100);                    // (the epilogue warps have the first tile's products to wait for; the copies have not)
        if ((spins & 63u) == 0) {
            if (*abort_flag) return false;
            if (global_timer_ns() - t0 > p.wait_ns) {
                *abort_flag = 1;
                atomicCAS(p.dev_status, kDevOk, kDevTimeoutProducer);
                return false;
            }
        }
    }
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    return true;
}

// Blocks of the inner dimension of piece `split`.
__device__ __forceinline__ void piece_of(const Phase& q, int split, int* from, int* to) {
    *from = (int)((int64_t)q.kblocks * split / q.splits);
    *to = (int)((int64_t)q.kblocks * (split + 1) / q.splits);
}

// A block of 32 x 32 accumulators is finished row by row: a lane has one row's 32 columns, 64 bytes of a half-precision plane, which it
// reads and writes as two whole sectors.  (Planes have padded rows, so that 32 columns can always be touched; what lies in the padding
// is not used.  Turning the block in shared memory so that eight lanes share a row takes as many sectors and twice the
// instructions.)
struct Row32 { uint32_t w[16]; };                         // 32 halves
__device__ __forceinline__ void load_row(const __half* p, Row32& r) {
#pragma unroll
    for (int i = 0; i < 16; i += 8)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r.w[i]), "=r"(r.w[i + 1]), "=r"(r.w[i + 2]), "=r"(r.w[i + 3]), "=r"(r.w[i + 4]), "=r"(r.w[i + 5]), "=r"(r.w[i + 6]), "=r"(r.w[i + 7])
                     : "l"(p + 2 * i) : "memory");
}
__device__ __forceinline__ void store_row(__half* p, const Row32& r) {
#pragma unroll
    for (int i = 0; i < 16; i += 8)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + 2 * i), "r"(r.w[i]), "r"(r.w[i + 1]), "r"(r.w[i + 2]), "r"(r.w[i + 3]),
                     "r"(r.w[i + 4]), "r"(r.w[i + 5]), "r"(r.w[i + 6]), "r"(r.w[i + 7]) : "memory");
}
__device__ __forceinline__ float2 to_floats(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t to_halves(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// What a row reads beside its accumulators: hi and lo (update), or A' (polynomial); `at`: its element offset in the planes.
struct Beside { Row32 a, b; };
__device__ __forceinline__ int64_t place_of(const NsParams& p, const Phase& q, int b, int row, int col) {
    const bool square = q.mode == kGram || q.mode == kPoly;
    return ((int64_t)b * (square ? p.s : p.m) + row) * (square ? p.lds : p.ldx) + col;
}
__device__ __forceinline__ void load_beside(const NsParams& p, const Phase& q, int step, int64_t at, Beside& in) {
    if (q.mode == kGram) return;
    load_row((q.mode == kPoly ? p.gram : p.hi[step & 1]) + at, in.a);
    if (q.mode != kPoly) load_row(p.lo[step & 1] + at, in.b);
}

// Row `row` and columns [col0, col0 + 32) of a phase's accumulators (v) of matrix b.  `in` was read ahead; `next`, called between the
// arithmetic and the stores, reads ahead for the block after this one (the compiler cannot move loads over stores that might
// alias them, and a round trip costs more than a block's arithmetic).  Whole warps: a lane whose row does not exist takes part in
// the exchange.  Returns the row's sum of squares where the next step needs it.
template <typename Next>
__device__ __forceinline__ float finish_row(const NsParams& p, const Phase& q, int step, const uint32_t (&v)[32], int64_t at, Beside& in, int b, int row, int col0, bool mirror,
                                            float g, Next next) {
    const float ca = p.coeffs[3 * step], cb = p.coeffs[3 * step + 1], cc = p.coeffs[3 * step + 2];
    const bool have = row < q.M;
    float sum = 0.f;
    Row32 o;
    if (q.mode == kGram || q.mode == kPoly) {
        __half* out = q.mode == kGram ? p.gram : p.poly;
        if (q.mode == kGram) {
            constexpr float kScale = 1.f / (float)(1 << (2 * kXExp - kSExp));
            const float diagonal = g * (float)(1 << kSExp);
            const int on = row - col0;                    // which of the 32 columns is the diagonal's
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o.w[i] = to_halves(__uint_as_float(v[2 * i]) * kScale - (on == 2 * i ? diagonal : 0.f), __uint_as_float(v[2 * i + 1]) * kScale - (on == 2 * i + 1 ? diagonal : 0.f));
        } else {
            const float lin = cb + 2.f * cc * g, sq = cc * (1.f / (float)(1 << kSExp));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 s = to_floats(in.a.w[i]);
                o.w[i] = to_halves(lin * s.x + sq * __uint_as_float(v[2 * i]), lin * s.y + sq * __uint_as_float(v[2 * i + 1]));
            }
        }
        next();
        if (have) store_row(out + at, o);
        if (mirror) {                                     // the same numbers at (column, row): neighbouring lanes trade, so that each stores two rows of a column
            const bool odd = threadIdx.x & 1;             // (the second row may lie in the padding)
            __half* to = out + ((int64_t)b * p.s + col0 + odd) * p.lds + (row & ~1);
            const bool pair = (row & ~1) < q.M;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t theirs = __shfl_xor_sync(0xffffffffu, o.w[i], 1);
                const uint32_t w = odd ? __byte_perm(theirs, o.w[i], 0x7632) : __byte_perm(o.w[i], theirs, 0x5410);
                if (pair && col0 + 2 * i + odd < q.N) *reinterpret_cast<uint32_t*>(to + (int64_t)(2 * i) * p.lds) = w;
            }
        }
    } else {
        const float lin = ca + g * (cb + cc * g), lin_lo = lin * (1.f / (float)(1 << kLoExp));
        const bool traced = step + 3 >= p.steps;          // the next step is one of the last two, which shift
        Row32 ol;
        float f[32];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 h = to_floats(in.a.w[i]), l = to_floats(in.b.w[i]);
            f[2 * i] = lin * h.x + (lin_lo * l.x + __uint_as_float(v[2 * i]) * (1.f / (float)(1 << kSExp)));
            f[2 * i + 1] = lin * h.y + (lin_lo * l.y + __uint_as_float(v[2 * i + 1]) * (1.f / (float)(1 << kSExp)));
        }
        if (q.mode == kUpdate) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                o.w[i] = to_halves(f[2 * i], f[2 * i + 1]);
                const float2 h = to_floats(o.w[i]);
                ol.w[i] = to_halves((f[2 * i] - h.x) * (float)(1 << kLoExp), (f[2 * i + 1] - h.y) * (float)(1 << kLoExp));
            }
            if (traced && have)
#pragma unroll
                for (int i = 0; i < 32; ++i) sum += col0 + i < q.N ? f[i] * f[i] : 0.f;
        }
        next();
        if (q.mode == kUpdate && have) {
            store_row(p.hi[(step + 1) & 1] + at, o);
            store_row(p.lo[(step + 1) & 1] + at, ol);
        } else if (have) {
            __nv_bfloat16* d = p.out + (int64_t)b * p.stride_out + (int64_t)row * p.ld_out + col0;
            constexpr float kScale = 1.f / (float)(1 << kXExp);
            if (p.out_vec && col0 + 32 <= q.N) {
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    __nv_bfloat162 w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __floats2bfloat162_rn(f[i + 2 * j] * kScale, f[i + 2 * j + 1] * kScale);
                    *reinterpret_cast<uint4*>(d + i) = *reinterpret_cast<const uint4*>(w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (col0 + i < q.N) d[i] = __float2bfloat16_rn(f[i] * kScale);
            }
        }
    }
    return sum;
}

// g of matrix b, by one warp: with A', trace(A) / s from the partial sums in their order (in the last two steps), or zero.
__device__ __forceinline__ float shift_of(const NsParams& p, int step, int mode, int b) {
    if (mode != kGram) return p.shift[b];
    if (step + 2 < p.steps) return 0.f;
    const int64_t parts = step == 0 ? 1 : p.trace_parts;
    double t = 0.0;
    for (int64_t i = threadIdx.x & 31; i < parts; i += 32) t += (double)p.trace[step & 1][b * parts + i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    return (float)(t / (double)p.s);
}

// All steps in one launch.  The CTA pairs share a phase's tiles; a phase begins when every CTA has finished the one before (a counter
// in the workspace, which every CTA adds to; the launch is cooperative).  Without launches in between, what is left between
// two phases is the counter's round trip and the filling of the pipeline.
// PIECES: the first product's inner dimension is split (a kernel of its own, for the others are 4 % slower with that path in it).
template <bool PIECES>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1) ns_steps_kernel(const __grid_constant__ NsParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles_base = (raw + 1023u) & ~1023u;
    unsigned char* behind = smem_raw + (tiles_base - raw) + (size_t)kStages * kStageBytes;
    PairPipe<kStages> pipe;
    pipe.open(behind, kEpilogueWarps, 1, 512, p.dev_status, p.wait_ns);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    const int phases = 3 * p.steps;

    if (warp < kFirstEpilogueWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPipeRegs));
        if (warp == 0) {                                  // copies, both CTAs
            const uint32_t leader_full = map_to_cta(pipe.full, 0);
            RingPos<kStages> at;
            uint32_t fills = 0;
            bool ok = true;
            for (int ph = 0; ok && ph < phases; ++ph) {
                const Phase q = phase_at<PIECES>(p, ph / 3, ph % 3);
                if (pair >= q.items) continue;
                const int half_rows = q.bn / 2;
                int b, tr, tc, from, to;
                tile_at(q, pair / q.splits, &b, &tr, &tc);
                piece_of(q, pair % q.splits, &from, &to);
                asm volatile("prefetch.tensormap [%0];" ::"l"(q.map_a) : "memory");
                asm volatile("prefetch.tensormap [%0];" ::"l"(q.map_b) : "memory");
                if (!(ok = __all_sync(0xffffffffu, wait_for_phase(p, (uint32_t)ph * gridDim.x, pipe.abort_flag, false)))) break;
                asm volatile("fence.proxy.async.global;" ::: "memory");       // the other CTAs' stores, then this thread's bulk copies
                for (int item = pair; ok && item < q.items; item += npairs) {
                    if (item != pair) {
                        tile_at(q, item / q.splits, &b, &tr, &tc);
                        piece_of(q, item % q.splits, &from, &to);
                    }
                    const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM, col0 = tc * q.bn + (int)pipe.rank * half_rows;
                    for (int kb = from; kb < to; ++kb) {
                        if (!(ok = pipe.wait_warp(pipe.empty + 8 * at.stage, at.phase ^ 1u, kDevTimeoutProducer))) break;
                        const uint32_t dst = tiles_base + at.stage * kStageBytes;
                        if (elect_one()) {
                            pipe.announce(at.stage, (uint32_t)(kBM + max(half_rows, 64)) * 128u);      // (a copy is 64 rows, also where half of them are used)
                            load_operand(dst, q.map_a, leader_full + 8 * at.stage, q.turned_a, kb, row0, kBM, b);
                            load_operand(dst + kBM * 128, q.map_b, leader_full + 8 * at.stage, q.turned_b, kb, col0, half_rows, b);
                        }
                        __syncwarp();
                        ++fills;
                        at.next();
                    }
                }
            }
            if (lane == 0) *pipe.fills_issued = fills;
            if (!ok && lane == 0) pipe.tell_peer();
        } else if (warp == 1 && pipe.rank == 0) {         // MMAs, leader
            RingPos<kStages> at;
            uint32_t it = 0;                              // tile counter: buffer it & 1, its use number it >> 1
            bool ok = true;
            for (int ph = 0; ok && ph < phases; ++ph) {
                const Phase q = phase_at<PIECES>(p, ph / 3, ph % 3);
                const uint32_t idesc = make_idesc_f16(q.turned_a, q.turned_b, 2 * kBM, q.bn);
                // 16 inner entries: 32 bytes along a swizzle row, or 16 rows of 128 bytes
                const uint64_t step_a = q.turned_a ? 128 : 2, step_b = q.turned_b ? 128 : 2;
                for (int item = pair; ok && item < q.items; item += npairs, ++it) {
                    const uint32_t buf = it & 1u;
                    int from, to;
                    piece_of(q, item % q.splits, &from, &to);
                    if (!(ok = pipe.wait_warp(pipe.tempty + 8 * buf, ((it >> 1) & 1u) ^ 1u, kDevTimeoutMma))) break;
                    for (int kb = from; kb < to; ++kb) {
                        if (!(ok = pipe.wait_warp(pipe.full + 8 * at.stage, at.phase, kDevTimeoutMma))) break;
                        tcgen05_fence_after();
                        const uint32_t a_addr = tiles_base + at.stage * kStageBytes, b_addr = a_addr + kBM * 128;
                        const uint64_t adesc = q.turned_a ? make_smem_desc_turned(a_addr) : make_smem_desc(a_addr);
                        const uint64_t bdesc = q.turned_b ? make_smem_desc_turned(b_addr) : make_smem_desc(b_addr);
                        if (elect_one()) {
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4)
                                umma_f16_pair(pipe.tmem + buf * 256, adesc + k4 * step_a, bdesc + k4 * step_b, idesc, (uint32_t)(kb != from || k4 != 0));
                            umma_commit_pair(pipe.empty + 8 * at.stage, 3);
                        }
                        __syncwarp();
                        at.next();
                    }
                    if (ok && elect_one()) umma_commit_pair(pipe.tfull + 8 * buf, 3);
                    __syncwarp();
                }
            }
            if (!ok && lane == 0) pipe.tell_peer();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegs));
        // Epilogue: warp w reads lanes 32 (w & 3) .. of TMEM (rows), columns of half (w - 4) / 4.
        const int half = (warp - kFirstEpilogueWarp) >> 2, quarter = warp & 3;
        const uint32_t leader_tempty = map_to_cta(pipe.tempty, 0);
        uint32_t it = 0;
        bool ok = true;
        for (int ph = 0; ph < phases; ++ph) {
            const int step = ph / 3;
            const Phase q = phase_at<PIECES>(p, step, ph % 3);
            if (ok) {                                     // (without tiles too: a CTA is counted for a phase only after the phases before it)
                ok = lane != 0 || wait_for_phase(p, (uint32_t)ph * gridDim.x, pipe.abort_flag, true);
                ok = __all_sync(0xffffffffu, ok);
                __syncwarp();                             // lane 0 has acquired the other CTAs' stores; this orders the other lanes' reads behind it (a vote does not)
            }
            const int nc = q.bn / 2;
            int shift_for = -1;
            float g = 0.f;
            for (int item = pair; ok && item < q.items; item += npairs, ++it) {
                int b, tr, tc;
                tile_at(q, item / q.splits, &b, &tr, &tc);
                const uint32_t buf = it & 1u;
                if (b != shift_for) {
                    g = shift_of(p, step, q.mode, b);
                    shift_for = b;
                }
                if (q.mode == kGram && tr == 0 && tc == 0 && item % q.splits == 0 && pipe.rank == 0 && warp == kFirstEpilogueWarp && lane == 0) p.shift[b] = g;
                const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM + quarter * 32, col0 = tc * q.bn + half * nc;
                const bool mirror = (q.mode == kGram || q.mode == kPoly) && (tc + 1) * q.bn <= tr * 2 * kBM;      // below the diagonal block
                const uint32_t taddr = pipe.tmem + ((uint32_t)(quarter * 32) << 16) + buf * 256 + (uint32_t)(half * nc);
                const int row = row0 + lane;
                Beside in;
                int64_t at = place_of(p, q, b, row, col0);
                if (row < q.M && col0 < q.N) load_beside(p, q, step, at, in);      // on its way while the tile's last MMAs run
                ok = __all_sync(0xffffffffu, pipe.wait(pipe.tfull + 8 * buf, (it >> 1) & 1u, kDevTimeoutEpilogue));
                if (!ok) break;
                tcgen05_fence_after();
                // A tile in pieces: every warp leaves its rows' sums of a piece in memory and counts itself; the last one of a tile's
                // pieces adds them all, in the order of the pieces whoever is last, and finishes the rows.
                const int64_t rows_id = ((int64_t)(item / q.splits) * 2 + pipe.rank) * kEpilogueWarps + (warp - kFirstEpilogueWarp);
                float* part = p.part + rows_id * q.splits * 32 * nc + lane;
                if (PIECES && q.splits > 1) {
#pragma unroll 1
                    for (int c = 0; c < nc; c += 32) {
                        uint32_t v[32];
                        tmem_ld32(taddr + c, v);
                        tmem_ld_wait();
                        float* to = part + (item % q.splits * nc + c) * 32;
#pragma unroll
                        for (int j = 0; j < 32; ++j) to[j * 32] = __uint_as_float(v[j]);
                    }
                    pipe.release_at(leader_tempty + 8 * buf);
                    __threadfence();
                    __syncwarp();
                    uint32_t before = 0;
                    if (lane == 0) before = atomicAdd(p.part_count + rows_id, 1u);
                    before = __shfl_sync(0xffffffffu, before, 0);
                    if (before + 1 != (uint32_t)q.splits) continue;
                    __threadfence();
                    __syncwarp();                         // lane 0 has seen the other pieces counted; its fence orders the other lanes' reads too
                    if (lane == 0) p.part_count[rows_id] = 0;      // for the next step, which begins behind a phase's end
                }
#pragma unroll 1
                for (int c = 0; c < nc; c += 32, at += 32) {
                    float sum = 0.f;
                    uint32_t v[32];
                    if (PIECES && q.splits > 1) {
                        const float* from = part + c * 32;
                        float f[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[j] = from[j * 32];
                        for (int s = 1; s < q.splits; ++s) {
                            from += nc * 32;
#pragma unroll
                            for (int j = 0; j < 32; ++j) f[j] += from[j * 32];
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(f[j]);
                    } else {
                        tmem_ld32(taddr + c, v);
                        tmem_ld_wait();
                        if (c + 32 == nc) pipe.release_at(leader_tempty + 8 * buf);
                    }
                    if (row0 < q.M && col0 + c < q.N)
                        sum = finish_row(p, q, step, v, at, in, b, row, col0 + c, mirror, g, [&]() {
                            if (c + 32 < nc && col0 + c + 32 < q.N && row < q.M) load_beside(p, q, step, at + 32, in);
                        });
                    // one partial sum per block, whatever the tile width: results do not depend on that choice
                    if (q.mode == kUpdate && step + 3 >= p.steps) {
#pragma unroll
                        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                        const int part_row = row0 >> 5, part_col = (col0 + c) >> 5, cols = (q.N + 31) >> 5;
                        if (lane == 0 && row0 < q.M && part_col < cols)
                            p.trace[(step + 1) & 1][(int64_t)b * p.trace_parts + (int64_t)part_row * cols + part_col] = sum * (1.f / (float)(1 << (2 * kXExp)));
                    }
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpilogueWarps) : "memory");
            if (warp == kFirstEpilogueWarp && lane == 0) {      // what the barrier has collected is published as a whole, to bulk copies too
                asm volatile("fence.proxy.async.global;" ::: "memory");
                __threadfence();
                asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p.phase_count) : "memory");
            }
        }
        if (!ok && lane == 0) pipe.tell_peer();
    }
    pipe.close(512);
}

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Partial sums of the trace that an update of m x n matrices leaves.
inline int64_t update_trace_parts(int64_t m, int64_t n) { return (m + 31) / 32 * ((n + 31) / 32); }

// rows x cols of `batch` matrices, padded rows; box = box_rows x 64 of one matrix (64 x 64 serves as rows x inner entries in either order).
bool make_half_map(CUtensorMap* map, const __half* base, int64_t rows, int64_t cols, int64_t ld, int64_t batch, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(rows * ld) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same matrix turned: its columns in groups of 64, so that a copy of 64 matrix rows by `groups` groups lands as 64 x groups operand
// rows.  Columns between the last one and the end of the padded row are read as operand rows that no result is kept of.
bool make_turned_map(CUtensorMap* map, const __half* base, int64_t rows, int64_t ld, int64_t batch, int groups) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(ld / 64), (cuuint64_t)batch};
    const cuuint64_t strides[3] = {(cuuint64_t)ld * 2, 128, (cuuint64_t)(rows * ld) * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)kBK, (cuuint32_t)groups, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<__half*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
cudaError_t launch_start(const NewtonSchulzArgs& a, cudaStream_t st, int* launches) {
    const NewtonSchulzLayout& l = a.lay;
    double* parts = (double*)(a.ws + l.off_norm);
    const uint32_t per_row = (uint32_t)((a.n + 7) / 8);
    const int64_t groups = a.m * per_row, needed = (groups + kRowThreads - 1) / kRowThreads;
    const int vec = a.n % 8 == 0 && ((uintptr_t)a.G & 15) == 0 && a.ldg * sizeof(T) % 16 == 0 && a.stride_g * sizeof(T) % 16 == 0;
    // (by the matrix alone, so that its sums do not depend on the batch it is in; eight groups or more per thread)
    const int blocks = (int)((needed + 7) / 8 < kNormParts ? (needed + 7) / 8 : kNormParts);
    cudaError_t err = launch_chained(norm_kernel<T>, dim3(blocks, (unsigned)a.batch), dim3(kRowThreads), 0, st, (const T*)a.G, groups, per_row, a.n, a.ldg, a.stride_g, vec, parts);
    if (err != cudaSuccess) return err;
    const int start_blocks = (int)((needed + kUnroll - 1) / kUnroll < 1024 ? (needed + kUnroll - 1) / kUnroll : 1024);
    err = launch_chained(start_kernel<T>, dim3(start_blocks, (unsigned)a.batch), dim3(kRowThreads), 0, st, (const T*)a.G, groups, per_row, a.m, a.n, a.ldg, a.stride_g, vec,
                         parts, blocks, a.eps, (__half*)(a.ws + l.off_hi[0]), (__half*)(a.ws + l.off_lo[0]), l.ldx, (float*)(a.ws + l.off_trace[0]),
                         (uint32_t*)(a.ws + l.off_count), (uint32_t*)(a.ws + l.off_part_count), l.part_counts);
    if (err == cudaSuccess) *launches += 2;
    return err;
}

// Columns of a product's tiles (index 0, 1, 2: 64, 128, 256), by the time of the pair that finishes last.  A tile's copies and MMAs take,
// per 64 inner entries, about 370, 400 or 560 cycles (1000 x 4096: 370 for 64 columns; 4096^2, all SMs: 560 for 256), its epilogue
// 1500 per 32 columns of a warp.  The longer of the two counts for every tile, the shorter once.
int best_width(const int64_t (&tiles)[3], int64_t kblocks, int64_t pairs) {
    int best = 0;
    double least = 0.0;
    for (int w = 0; w < 3; ++w) {
        const double rounds = (double)((tiles[w] + pairs - 1) / pairs), feed = (double)kblocks * (w == 2 ? 560.0 : w == 1 ? 400.0 : 370.0), finish = 1500.0 * (double)(1 << w);
        const double cost = rounds * (feed > finish ? feed : finish) + (feed > finish ? finish : feed);
        if (w == 0 || cost < least) { best = w; least = cost; }
    }
    return best;
}

// Tiles of an s x s square in tiles of 64 << w columns.
int64_t tiles_of_square(int64_t s, int w) { return square_tiles((int)((s + 255) / 256), (int)((s + (64 << w) - 1) / (64 << w)), 4 >> w); }

// Pieces of the inner dimension of X X^T, where a square of few tiles has a long one: as many as let one matrix's tiles, 128 columns wide,
// fill 74 pairs, at most 8, with 12 blocks of 64 or more each, and four or none (a piece costs the writing and reading of its sums).
// By the matrix alone: the pieces are part of the order of summation.  256 x 8000, eight pieces: 152 us against 223 in one;
// 1000 x 4096, three: 228 against 227; 8 of 200 x 1500, two: 193 against 184.
int splits_of(int64_t s, int64_t long_side) {
    if (s == 0) return 1;                                 // (no tiles: a workspace is asked for, nothing is launched)
    int64_t most = 74 / tiles_of_square(s, 1);
    const int64_t blocks = (long_side + kBK - 1) / kBK;
    if (most > blocks / 12) most = blocks / 12;
    return (int)(most < 4 ? 1 : most > 8 ? 8 : most);
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
    l.off_count = take(256);
    l.off_shift = take(4 * batch);
    for (int i = 0; i < 2; ++i) l.off_trace[i] = take(4 * batch * l.trace_parts);
    for (int i = 0; i < 2; ++i) {
        l.off_hi[i] = take(2 * batch * m * l.ldx);
        l.off_lo[i] = take(2 * batch * m * l.ldx);
    }
    l.off_gram = take(2 * batch * s * l.lds);
    l.off_poly = take(2 * batch * s * l.lds);
    l.splits = splits_of(s, m < n ? n : m);
    int64_t area = 0;
    l.part_counts = 0;
    if (l.splits > 1) {
        for (int w = 0; w < 3; ++w) area = area > tiles_of_square(s, w) * 256 * (64 << w) ? area : tiles_of_square(s, w) * 256 * (64 << w);
        l.part_counts = tiles_of_square(s, 0) * 2 * kEpilogueWarps * batch;
    }
    l.off_part = take(4 * area * l.splits * batch);
    l.off_part_count = take(4 * l.part_counts);
    l.total = off;
    return l;
}

// Waits last as long as a phase: the largest product has 2 s^2 l operations per matrix, here allowed a rate of 10^14 per second (a tenth of what
// it runs at) on top of the limit of every wait.  (100000^2 bf16 in place takes 140 GB and 2 s per phase.)
unsigned long long newton_schulz_wait_ns(int64_t batch, int64_t m, int64_t n) {
    const double s = (double)(m < n ? m : n), l = (double)(m < n ? n : m);
    return kWaitLimitNs + (unsigned long long)(2.0 * s * s * l * (double)batch / 1e5);
}

cudaError_t launch_newton_schulz(const NewtonSchulzArgs& a, int sm_count, cudaStream_t st, int launches[2]) {
    cudaError_t err = a.type == kF32 ? launch_start<float>(a, st, &launches[0])
                      : a.type == kF16 ? launch_start<__half>(a, st, &launches[0]) : launch_start<__nv_bfloat16>(a, st, &launches[0]);
    if (err != cudaSuccess) return err;
    const NewtonSchulzLayout& l = a.lay;
    static int pairs_dev[2][kMaxDevices] = {};
    const auto kernel = l.splits > 1 ? ns_steps_kernel<true> : ns_steps_kernel<false>;
    int& max_pairs = pairs_dev[l.splits > 1][current_device_slot()];
    if (!max_pairs) {
        int pairs = 0;
        if ((err = resident_pairs(kernel, kGemmThreads, kGemmSmem, sm_count, &pairs)) != cudaSuccess) return err;
        max_pairs = pairs;
    }
    NsParams p = {};
    p.m = (int)a.m; p.n = (int)a.n; p.s = (int)(a.m < a.n ? a.m : a.n);
    p.batch = (int)a.batch; p.steps = a.steps;
    for (int i = 0; i < 3 * a.steps; ++i) p.coeffs[i] = a.coeffs[i];
    for (int i = 0; i < 2; ++i) {
        p.trace[i] = (float*)(a.ws + l.off_trace[i]);
        p.hi[i] = (__half*)(a.ws + l.off_hi[i]);
        p.lo[i] = (__half*)(a.ws + l.off_lo[i]);
        for (int w = 0; w < 2; ++w)
            if (!make_half_map(&p.x[i][w], p.hi[i], a.m, a.n, l.ldx, a.batch, 64 << w) || !make_turned_map(&p.x_turned[i][w], p.hi[i], a.m, l.ldx, a.batch, 1 + w))
                return cudaErrorInvalidValue;
    }
    p.trace_parts = l.trace_parts;
    p.splits = l.splits;
    p.part = (float*)(a.ws + l.off_part);
    p.part_count = (uint32_t*)(a.ws + l.off_part_count);
    p.shift = (float*)(a.ws + l.off_shift);
    p.gram = (__half*)(a.ws + l.off_gram);
    p.poly = (__half*)(a.ws + l.off_poly);
    p.lds = l.lds; p.ldx = l.ldx;
    for (int w = 0; w < 2; ++w)
        if (!make_half_map(&p.gram_map[w], p.gram, p.s, p.s, l.lds, a.batch, 64 << w) || !make_half_map(&p.poly_map[w], p.poly, p.s, p.s, l.lds, a.batch, 64 << w))
            return cudaErrorInvalidValue;
    p.out = (__nv_bfloat16*)a.O; p.ld_out = a.ldo; p.stride_out = a.stride_o;
    p.out_vec = ((uintptr_t)a.O & 15) == 0 && a.ldo % 8 == 0 && a.stride_o % 8 == 0;
    p.phase_count = (uint32_t*)(a.ws + l.off_count);
    p.dev_status = a.dev_status;
    p.wait_ns = newton_schulz_wait_ns(a.batch, a.m, a.n);
    auto tiles_of = [](int64_t x, int64_t width) { return (x + width - 1) / width; };
    const int64_t rt = tiles_of(p.s, 256), mt = tiles_of(a.m, 256);
    if (tiles_of(p.s, 64) * (rt + 1) > INT32_MAX / 8 / a.batch || mt * tiles_of(a.n, 64) > INT32_MAX / 8 / a.batch) return cudaErrorInvalidValue;
    int64_t square[3], update[3];
    for (int w = 0; w < 3; ++w) {
        square[w] = tiles_of_square(p.s, w) * l.splits * a.batch;
        update[w] = mt * tiles_of(a.n, 64 << w) * a.batch;
    }
    const int64_t long_side = a.m < a.n ? a.n : a.m;
    const int ws = best_width(square, tiles_of((p.s + long_side / l.splits) / 2, kBK), max_pairs), wu = best_width(update, tiles_of(p.s, kBK), max_pairs);
    p.square_width = 64 << ws;
    p.update_width = 64 << wu;
    const int64_t most = square[ws] > update[wu] ? square[ws] : update[wu];
    const int pairs = (int)(most < max_pairs ? most : max_pairs);
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(2 * pairs);
    c.blockDim = dim3(kGemmThreads);
    c.dynamicSmemBytes = kGemmSmem;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    c.attrs = at;
    c.numAttrs = 1;
    err = cudaLaunchKernelEx(&c, kernel, p);
    if (err == cudaSuccess) ++launches[1];
    return err;
}

}  // namespace gemm2m
