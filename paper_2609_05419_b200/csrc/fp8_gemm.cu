// Product of two 8-bit floating-point matrices with block scales,
//   D[i, j] = C[i, j] + sum_b SA[i / block, b] SB[j / block, b] sum_{p in block b} A[i, p] B[j, p],
// blocks of 128 along k.  Every block's sum is accumulated in 32 bits, scaled, and added to a 32-bit total; D is rounded once.
//
// A block of 128 entries is one 128-byte swizzle row, so one pipeline stage, so four MMAs (K = 32).  Since the scales differ from
// block to block, the tensor core's accumulator holds one block's sums only: it is written afresh every four MMAs, into two TMEM buffers in
// turn (four of a narrow tile), and eight epilogue warps per CTA read each back, multiply by the scales and add to totals in registers (128
// per thread) while the next is being filled.  256 x 256 tiles per CTA pair: the four MMAs of a block take 512 cycles, the
// 128 x 256 multiply-adds of a CTA's half 256 issue slots of the FP32 pipes.  What bounds it is neither: a block takes about 1000
// cycles, the way from the commit through the epilogue warps (wait, scales, four TMEM loads, 128 multiply-adds, two warps per scheduler) back
// to the released buffer, during which each buffer is out of the tensor core's hands.  8192^3 to bf16: 504 us in a short run (2.18 PFLOP/s), 585 in
// a steady stream of calls at the board's power limit; 4096 x 4096 x 8192 with a scale per column: 177 and 203 us.  8192 x 4096 x 4096: tensor
// pipe 49 % active.  Measured and not kept, against 519 us then: packed pairs (f32x2) in place of scalar multiply-adds, whose register pairs
// the compiler feeds with moves (620 us); sixteen epilogue warps of 64 columns (590); the wide tile in two parts of 128 columns with two
// buffers each (577: the first operand is read twice).
#include "layer_ops.cuh"
#include "pair_pipeline.cuh"

#include <cmath>
#include <type_traits>

namespace gemm2m {

namespace {

constexpr int kBM = 128;                 // rows of A per CTA
constexpr int kEpilogueWarps = 8;
// Warps 0 and 1 copy operands and issue MMAs, 2 and 3 fetch scales, 4 .. 11 are the epilogue.  The totals need more registers than an equal
// share (168): the first four warps give up what they do not use.  128 x 40 + 256 x 232 <= 384 x 168.
constexpr int kFirstEpilogueWarp = 4;
constexpr int kThreads = 32 * (kFirstEpilogueWarp + kEpilogueWarps);
constexpr int kLaunchRegs = 168, kPipeRegs = 40, kEpilogueRegs = 232;
static_assert(128 * kPipeRegs + 32 * kEpilogueWarps * kEpilogueRegs <= kThreads * kLaunchRegs, "register shares exceed what the block is launched with");

// Ring of scale slots, one per block; a slot is written kAhead blocks ahead.  A block's scales are there when its tfull barrier completes
// (the two scale warps arrive on it next to the commit).  They turn to block g after tfull of block g - NB (NB accumulators): the MMAs of
// that block were issued after every epilogue warp had released block g - 2 NB, so all of them are through with g - 2 NB - 1 and
// earlier ones: kSlots >= kAhead + 2 NB + 1.
constexpr int kSlots = 16, kAhead = 3, kScaleWarps = 2;

template <int BN, bool COLS>
struct Cfg {
    static constexpr int kHalfRows = BN / 2;                          // rows of B per CTA
    static constexpr int kStageBytes = (kBM + kHalfRows) * kGemmBK;
    static constexpr int kStages = BN == 256 ? 5 : 6;
    static constexpr int kCols = BN / 2;                              // columns per epilogue warp: totals per thread
    static constexpr int kBuffers = 512 / BN;
    static_assert(kSlots >= kAhead + 2 * kBuffers + 1, "scale ring");
    static constexpr uint32_t kTmemCols = 512;
    static constexpr int kSlotFloats = kBM + (COLS ? BN : 2);         // scales of one block: 128 rows, and the columns or their halves
    static constexpr int kSlotBytes = (kSlotFloats * 4 + 15) / 16 * 16;
    static constexpr size_t kScaleBytes = (size_t)kSlots * kSlotBytes;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 + kScaleBytes + PairPipe<kStages, kBuffers>::kBytes + 16 + kEpilogueWarps * 4096;
};

struct Fp8GemmParams {
    int m, n, kblocks, tiles_r, tiles_c, band;
    const float *SA, *SB;
    int64_t ldsa, ldsb;
    int shift_a, shift_b;                // row r has the scale r >> shift (0 or 7)
    uint32_t idesc;
    const void* C; int64_t ldc;
    void* D; int64_t ldd;
    int vec;                             // rows of C and D allow stores of four entries
    int* dev_status;
    unsigned long long wait_ns;
};

// Instruction descriptor of kind::f8f6f4: 32-bit accumulator, both operands K-major, M x N tile; 0 = e4m3, 1 = e5m2.
uint32_t make_idesc_f8(int fmt_a, int fmt_b, int M, int N) {
    return (1u << 4) | ((uint32_t)(fmt_a == kE5M2) << 7) | ((uint32_t)(fmt_b == kE5M2) << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void umma_f8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Tiles in bands of `band` row tiles, column by column inside a band, so that the tiles in flight share operands through L2.
__device__ __forceinline__ void tile_at(const Fp8GemmParams& p, int tile, int* tr, int* tc) {
    const int per_band = p.band * p.tiles_c;
    const int band = tile / per_band, in_band = tile - band * per_band;
    const int rows_here = min(p.band, p.tiles_r - band * p.band);
    *tc = in_band / rows_here;
    *tr = band * p.band + (in_band - *tc * rows_here);
}

template <typename T> __device__ __forceinline__ float from_type(T v);
template <> __device__ __forceinline__ float from_type<float>(float v) { return v; }
template <> __device__ __forceinline__ float from_type<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float from_type<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T to_type(float v);
template <> __device__ __forceinline__ float to_type<float>(float v) { return v; }
template <> __device__ __forceinline__ __half to_type<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 to_type<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// NC columns of 32 rows, one row per lane, to rows [row0, row0 + 32) and columns [col0, col0 + NC) of D (plus C), of which those
// below m and n exist.  Through `turn`, 4 KB of shared memory per warp, 32 columns at a time: a lane writes its row's 128 bytes,
// 16-byte pieces XORed with the row, and then eight lanes store one row's 32 columns side by side (whole 32-byte
// sectors; a lane storing along its own row would leave half-written sectors of 32 rows per instruction).
template <typename T, int NC, bool ADD>
__device__ __forceinline__ void store_rows(const float (&v)[NC], uint32_t turn, const T* C, int64_t ldc, T* D, int64_t ldd, int row0, int col0, int m, int n, bool vec) {
    const int lane = threadIdx.x & 31, piece = lane & 7;
    struct alignas(4 * sizeof(T)) Four { T t[4]; };
#pragma unroll
    for (int c = 0; c < NC; c += 32) {
        const int col = col0 + c + piece * 4, first = lane >> 3;
        const int rows = col < n ? min(32, m - row0) : 0;
        const bool whole = vec && col + 4 <= n;
        // ADD: what is added is asked for at once (row by row, each load would wait for the store before it: 265 against 228 us for
        // 4096 x 4096 x 8192 added to a 32-bit C).  Without it the loop is kept short: it is fetched anew for every tile.
        Four in[8];
        if (ADD && whole)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (first + 4 * i < rows) in[i] = *reinterpret_cast<const Four*>(C + (int64_t)(row0 + first + 4 * i) * ldc + col);
        __syncwarp();                                     // the previous columns have been read
#pragma unroll
        for (int q = 0; q < 8; ++q)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (uint32_t)(lane * 128 + ((q ^ (lane & 7)) << 4))), "f"(v[c + 4 * q]),
                         "f"(v[c + 4 * q + 1]), "f"(v[c + 4 * q + 2]), "f"(v[c + 4 * q + 3]) : "memory");
        __syncwarp();
#pragma unroll(ADD ? 8 : 2)
        for (int i = 0; i < 8; ++i) {
            const int r = first + 4 * i;
            if (r >= rows) continue;
            float x[4];
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3])
                         : "r"(turn + (uint32_t)(r * 128 + ((piece ^ (r & 7)) << 4))) : "memory");
            T* d = D + (int64_t)(row0 + r) * ldd + col;
            if (whole) {
                Four f;
#pragma unroll
                for (int j = 0; j < 4; ++j) f.t[j] = to_type<T>(ADD ? x[j] + from_type<T>(in[i].t[j]) : x[j]);
                *reinterpret_cast<Four*>(d) = f;
            } else {
                const T* s = C + (int64_t)(row0 + r) * ldc + col;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < n) d[j] = to_type<T>(ADD ? x[j] + from_type<T>(s[j]) : x[j]);
            }
        }
    }
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ float lds(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// A block sum v becomes (v s) t with its two scales, in that order: s t may overflow, or lose its bits as a subnormal number, where the scaled
// sum does neither.  |v| lies between 2^-32 and 2^39 (2^-18 and 2^25 for e4m3), so v s is a normal number for s from 2^-94 to 2^89.
// With one s t per thread and block (no scale per column) the product s t serves if it lies between these bounds, which saves 128 multiplications;
// one branch for the whole block (8192^3: 565 us, against 585 with a branch in front of each 32 columns).
constexpr float kLeastScale = 0x1p-96f, kLargestScale = 0x1p88f;

// T: type of C and D.  ADD: C is added.  COLS: B has a scale per row (of B; column of D) and block, otherwise one per 128 rows.
template <typename T, int BN, bool COLS, bool ADD>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
fp8_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Fp8GemmParams p) {
    using cfg = Cfg<BN, COLS>;
    constexpr int STAGES = cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles_base = (raw + 1023u) & ~1023u;
    unsigned char* behind = smem_raw + (tiles_base - raw) + (size_t)STAGES * cfg::kStageBytes;
    const uint32_t scale_ring = smem_u32(behind);
    constexpr int NB = cfg::kBuffers;
    PairPipe<STAGES, NB> pipe;
    pipe.open(behind + cfg::kScaleBytes, kEpilogueWarps, 1 + kScaleWarps, cfg::kTmemCols, p.dev_status, p.wait_ns);
    wait_for_prior_kernels();

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    const int total_tiles = p.tiles_r * p.tiles_c;

    if (warp < kFirstEpilogueWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPipeRegs));
        if (warp == 0) {                                  // copies, both CTAs
            const uint32_t leader_full = map_to_cta(pipe.full, 0);
            RingPos<STAGES> at;
            uint32_t fills = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
                int tr, tc;
                tile_at(p, tile, &tr, &tc);
                const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM, col0 = tc * BN + (int)pipe.rank * cfg::kHalfRows;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!(ok = pipe.wait_warp(pipe.empty + 8 * at.stage, at.phase ^ 1u, kDevTimeoutProducer))) break;
                    const uint32_t dst = tiles_base + at.stage * cfg::kStageBytes;
                    if (elect_one()) {
                        pipe.announce(at.stage, cfg::kStageBytes);
                        tma_load_2d_pair(dst, &map_a, leader_full + 8 * at.stage, kb * kGemmBK, row0);
                        tma_load_2d_pair(dst + kBM * kGemmBK, &map_b, leader_full + 8 * at.stage, kb * kGemmBK, col0);
                    }
                    __syncwarp();
                    ++fills;
                    at.next();
                }
            }
            if (lane == 0) *pipe.fills_issued = fills;
            if (!ok && lane == 0) pipe.tell_peer();
        } else if (warp == 1 && pipe.rank == 0) {         // MMAs, leader
            RingPos<STAGES> at;
            uint32_t it = 0;                              // block counter over all tiles: buffer it % NB, its use number it / NB
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs)
                for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
                    const uint32_t buf = it % NB;
                    if (!(ok = pipe.wait_warp(pipe.tempty + 8 * buf, ((it / NB) & 1u) ^ 1u, kDevTimeoutMma) &&
                               pipe.wait_warp(pipe.full + 8 * at.stage, at.phase, kDevTimeoutMma))) break;
                    tcgen05_fence_after();
                    const uint32_t a_addr = tiles_base + at.stage * cfg::kStageBytes;
                    const uint64_t adesc = make_smem_desc(a_addr), bdesc = make_smem_desc(a_addr + kBM * kGemmBK);
                    if (elect_one()) {
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4)
                            umma_f8_pair(pipe.tmem + buf * BN, adesc + (uint64_t)(k4 * 2), bdesc + (uint64_t)(k4 * 2), p.idesc, (uint32_t)(k4 != 0));
                        umma_commit_pair(pipe.tfull + 8 * buf, 3);
                        umma_commit_pair(pipe.empty + 8 * at.stage, 3);
                    }
                    __syncwarp();
                    at.next();
                }
            if (!ok && lane == 0) pipe.tell_peer();
        } else if (warp >= 2) {                           // scales, both CTAs: asynchronous 4-byte copies, one group per block
            const int t = threadIdx.x - 64;
            int tile = pair, kb = 0, row0 = 0, col0 = 0;  // next block to fetch
            uint32_t fetched = 0;
            auto fetch = [&]() {
                if (tile < total_tiles) {
                    if (kb == 0) {
                        int tr, tc;
                        tile_at(p, tile, &tr, &tc);
                        row0 = tr * (2 * kBM) + (int)pipe.rank * kBM;
                        col0 = tc * BN;
                    }
                    const uint32_t slot = scale_ring + (fetched & (kSlots - 1)) * cfg::kSlotBytes;
                    const float* sa = p.SA + (int64_t)kb * p.ldsa;
                    const float* sb = p.SB + (int64_t)kb * p.ldsb;
#pragma unroll
                    for (int i = 0; i < kBM; i += 64) cp_async4(slot + (i + t) * 4, sa + (min(row0 + i + t, p.m - 1) >> p.shift_a));
                    if (COLS) {
#pragma unroll
                        for (int i = 0; i < BN; i += 64) cp_async4(slot + (kBM + i + t) * 4, sb + min(col0 + i + t, p.n - 1));
                    } else if (t < 2) {
                        cp_async4(slot + (kBM + t) * 4, sb + (min(col0 + t * cfg::kCols, p.n - 1) >> p.shift_b));
                    }
                    ++fetched;
                    if (++kb == p.kblocks) { kb = 0; tile += npairs; }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            for (int i = 0; i < kAhead; ++i) fetch();
            const uint32_t blocks = pair < total_tiles ? (uint32_t)((total_tiles - pair + npairs - 1) / npairs) * (uint32_t)p.kblocks : 0u;
            bool ok = true;
            for (uint32_t g = 0; g < blocks; ++g) {
                const uint32_t bar = pipe.tfull + 8 * (g % NB);
                if (g >= NB && !(ok = __all_sync(0xffffffffu, pipe.wait(bar, ((g / NB) & 1u) ^ 1u, kDevTimeoutProducer)))) break;
                fetch();
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (!ok && lane == 0) pipe.tell_peer();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegs));
        // Epilogue: warp w reads lanes 32 (w & 3) .. of TMEM (rows), columns of half (w - 4) / 4.
        const int half = (warp - kFirstEpilogueWarp) >> 2, quarter = warp & 3;
        constexpr int NC = cfg::kCols;
        const uint32_t row_slot = scale_ring + (uint32_t)(quarter * 32 + lane) * 4;
        const uint32_t col_slot = scale_ring + (uint32_t)(kBM + (COLS ? half * NC : half)) * 4;
        const uint32_t taddr = pipe.tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * NC);
        const uint32_t turn = smem_u32(behind) + (uint32_t)(cfg::kScaleBytes + PairPipe<STAGES, NB>::kBytes + 15) / 16 * 16 + (uint32_t)(warp - kFirstEpilogueWarp) * 4096;
        const uint32_t leader_tempty = map_to_cta(pipe.tempty, 0);
        uint32_t it = 0;
        bool ok = true;
        for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
            int tr, tc;
            tile_at(p, tile, &tr, &tc);
            const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM + quarter * 32;
            const int col0 = tc * BN + half * NC;
            float acc[NC];
#pragma unroll
            for (int i = 0; i < NC; ++i) acc[i] = 0.f;
            for (int kb = p.kblocks; kb > 0; --kb, ++it) {
                const uint32_t buf = it % NB;
                // (a wait that gives up is acted on at the end of the tile: every later one then returns at once)
                ok &= pipe.wait(pipe.tfull + 8 * buf, (it / NB) & 1u, kDevTimeoutEpilogue);
                tcgen05_fence_after();
                const uint32_t slot = (it & (kSlots - 1)) * cfg::kSlotBytes, col_scale = col_slot + slot;
                const uint32_t at = taddr + buf * BN;
                uint32_t v[2][32];                        // one piece is on its way while the other is added
                tmem_ld32(at, v[0]);
                const float row_scale = lds(row_slot + slot);
                // One block's sums into the totals; FIRST: times `first`, then `scale`.
                auto add_block = [&](auto FIRST, float first, float scale) {
                    const uint64_t f2 = pack2(first, first);
#pragma unroll
                    for (int c = 0; c < NC; c += 32) {
                        const uint32_t(&w)[32] = v[(c / 32) & 1];
                        tmem_ld_wait();
                        if (c + 32 < NC) tmem_ld32(at + c + 32, v[(c / 32 + 1) & 1]);
                        else pipe.release_at(leader_tempty + 8 * buf);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float s[4] = {scale, scale, scale, scale}, x[4];
                            if (COLS)
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]) : "r"(col_scale + (c + i) * 4));
                            if constexpr (decltype(FIRST)::value) {
                                mul_pair(w[i], w[i + 1], f2, &x[0], &x[1]);
                                mul_pair(w[i + 2], w[i + 3], f2, &x[2], &x[3]);
                            } else {
#pragma unroll
                                for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[i + j]);
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) fma1(acc[c + i + j], x[j], s[j]);
                        }
                    }
                };
                if constexpr (COLS) {
                    add_block(std::true_type(), row_scale, 0.f);
                } else {
                    const float col = lds(col_scale), both = row_scale * col;
                    const bool fits = fabsf(both) >= kLeastScale && fabsf(both) <= kLargestScale;
                    // (what a lane multiplies by goes by its row alone: a row's result does not depend on its neighbours' scales)
                    if (__all_sync(0xffffffffu, fits)) add_block(std::false_type(), 1.f, both);
                    else add_block(std::true_type(), fits ? 1.f : row_scale, fits ? both : col);
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (ok && row0 < p.m && col0 < p.n) {
                store_rows<T, NC, ADD>(acc, turn, (const T*)p.C, p.ldc, (T*)p.D, p.ldd, row0, col0, p.m, p.n, p.vec != 0);
            }
        }
        if (!ok && lane == 0) pipe.tell_peer();
    }
    pipe.close(cfg::kTmemCols);
}

// rows x k bytes with leading dimension ld; box = 128 bytes of k x box_rows; what lies outside reads as zero.
bool make_byte_map(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kGemmBK, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int BN, bool COLS, bool ADD>
cudaError_t launch_pair(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    static int pairs_dev[kMaxDevices] = {};
    int& max_pairs = pairs_dev[current_device_slot()];
    if (!max_pairs) {
        int pairs = 0;
        cudaError_t err = resident_pairs(fp8_gemm_pair_kernel<T, BN, COLS, ADD>, kThreads, Cfg<BN, COLS>::kSmem, sm_count, &pairs);
        if (err != cudaSuccess) return err;
        max_pairs = pairs;
    }
    CUtensorMap map_a, map_b;
    if (!make_byte_map(&map_a, a.A.Q, a.m, a.k, a.A.ld, kBM) || !make_byte_map(&map_b, a.B.Q, a.n, a.k, a.B.ld, Cfg<BN, COLS>::kHalfRows)) return cudaErrorInvalidValue;
    Fp8GemmParams p = {};
    p.m = (int)a.m; p.n = (int)a.n;
    p.kblocks = (int)((a.k + kScaleBlock - 1) / kScaleBlock);
    const int64_t tr = (a.m + 2 * kBM - 1) / (2 * kBM), tc = (a.n + BN - 1) / BN;
    if (tr * tc > INT32_MAX) return cudaErrorInvalidValue;
    p.tiles_r = (int)tr; p.tiles_c = (int)tc;
    p.band = p.tiles_r < 8 ? p.tiles_r : 8;
    p.SA = a.A.S; p.SB = a.B.S; p.ldsa = a.A.lds; p.ldsb = a.B.lds;
    p.shift_a = a.A.block == 1 ? 0 : 7; p.shift_b = a.B.block == 1 ? 0 : 7;
    p.idesc = make_idesc_f8(a.A.fmt, a.B.fmt, 2 * kBM, BN);
    p.C = a.C; p.ldc = a.ldc; p.D = a.D; p.ldd = a.ldd; 
    const uintptr_t es = sizeof(T), at = (uintptr_t)a.D | (uintptr_t)a.C, ld = (uintptr_t)a.ldd | (a.C ? (uintptr_t)a.ldc : 0);
    p.vec = at % (4 * es) == 0 && ld % 4 == 0;
    p.dev_status = a.dev_status;
    p.wait_ns = kWaitLimitNs;
    const int pairs = (int)(tr * tc < max_pairs ? tr * tc : max_pairs);
    cudaError_t err = launch_chained(fp8_gemm_pair_kernel<T, BN, COLS, ADD>, dim3(2 * pairs), dim3(kThreads), Cfg<BN, COLS>::kSmem, st, map_a, map_b, p);
    if (err == cudaSuccess) ++*launches;
    return err;
}

// ---- thin products -------------------------------------------------------------------------------------------------
// Few rows on one side (a token, a decoding batch), or too few 256 x 256 tiles to fill the GPU: one CTA per tile of 128 rows of
// the lane operand (the weights, for tokens) x N rows of the column operand, N = 16, 32, 64 or 128, and the blocks of k split over a cluster
// of S CTAs, whose totals are added through distributed shared memory in the order of the ranks.  The lane operand is
// what such a product has to read; all stages of the ring are requested at once, so that every SM has 130 to 190 KB on its way.
// 1 x 4096 x 4096 (16.8 MB of weights, split in four): 6 to 7 us on the device, of which set-up 0.7, first bytes 0.5 (from L2; 2 from HBM), eight
// blocks 2.6, the join 1.6; 48 x 16384 x 4096 (67 MB): 18.2 us from HBM, 3.7 TB/s.

constexpr int kThinBuffers = 4;                  // accumulators of N columns
constexpr int kThinSlots = 16, kThinAhead = 6;   // scales turn to block g after tfull of g - 4, so every warp is through with g - 9; slot of g + 6 - 16

template <int N>
struct ThinCfg {
    // Epilogue warps, four per part of the columns: eight from 64 columns on (48 x 16384 x 4096 on the same operands: 16.6 us, with four 19.3).
    static constexpr int kWarps = N >= 64 ? 8 : 4;
    static constexpr int kCols = N / (kWarps / 4);
    static constexpr int kThreads = 128 + 32 * kWarps;     // copies, MMAs, two scale warps, epilogue
    static constexpr int kStageBytes = (kBM + N) * kGemmBK;
    static constexpr int kStages = N == 128 ? 6 : 8;
    static constexpr int kSlotBytes = (kBM + N) * 4;
    static constexpr size_t kBarBytes = 8 * (2 * kStages + 2 * kThinBuffers + 1) + 16;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 + (size_t)kThinSlots * kSlotBytes + kBarBytes;
    static constexpr uint32_t kTmemCols = N * kThinBuffers < 32 ? 32 : N * kThinBuffers;
    static_assert((size_t)kStages * kStageBytes >= (size_t)N * kBM * 4, "the totals of a split product pass through the stages");
};

struct ThinParams {
    int lanes, cols, kblocks, lane_tiles;        // rows of the lane and of the column operand, blocks of k, tiles of the lane operand
    const float *SL, *SC;
    int64_t ldsl, ldsc;
    int shift_l, shift_c;
    uint32_t idesc;
    const void* C; int64_t c_lane, c_col;        // element strides of C and D along the two operands' rows
    void* D; int64_t d_lane, d_col;
    int* dev_status;
    unsigned long long wait_ns;
};

__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

template <typename T, int N>
__global__ void __launch_bounds__(ThinCfg<N>::kThreads, 1)
fp8_gemm_thin_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_c, const __grid_constant__ ThinParams p) {
    using cfg = ThinCfg<N>;
    constexpr int STAGES = cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles_base = (raw + 1023u) & ~1023u;
    unsigned char* behind = smem_raw + (tiles_base - raw) + (size_t)STAGES * cfg::kStageBytes;
    const uint32_t scale_ring = smem_u32(behind);
    uint64_t* bars = reinterpret_cast<uint64_t*>(behind + kThinSlots * cfg::kSlotBytes);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, tfull = empty + 8 * STAGES, tempty = tfull + 8 * kThinBuffers;
    const uint32_t drain = tempty + 8 * kThinBuffers;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 2 * kThinBuffers + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile uint32_t* fills_issued = reinterpret_cast<volatile uint32_t*>(tmem_slot + 2);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = (int)cluster_size(), rank = (int)cluster_ctarank();
    const int tile = blockIdx.x / S;
    const int l0 = tile % p.lane_tiles * kBM, c0 = tile / p.lane_tiles * N;
    const int kb0 = (int)((int64_t)p.kblocks * rank / S), blocks = (int)((int64_t)p.kblocks * (rank + 1) / S) - kb0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (int a = 0; a < kThinBuffers; ++a) { mbar_init(tfull + 8 * a, 1 + kScaleWarps); mbar_init(tempty + 8 * a, cfg::kWarps); }
        mbar_init(drain, 1);
        *abort_flag = 0;
        *fills_issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(cfg::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;
    wait_for_prior_kernels();
    auto wait = [&](uint32_t bar, uint32_t parity, int code) { return mbar_wait(bar, parity, abort_flag, p.dev_status, code, p.wait_ns); };

    constexpr int NC = cfg::kCols;
    float acc[NC];
    if (warp == 0) {
        RingPos<STAGES> at;
        int kb = 0;
        for (; kb < blocks; ++kb) {
            if (!__all_sync(0xffffffffu, wait(empty + 8 * at.stage, at.phase ^ 1u, kDevTimeoutProducer))) break;
            const uint32_t dst = tiles_base + at.stage * cfg::kStageBytes, bar = full + 8 * at.stage;
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, cfg::kStageBytes);
                tma_load_2d(dst, &map_l, bar, (kb0 + kb) * kGemmBK, l0);
                tma_load_2d(dst + kBM * kGemmBK, &map_c, bar, (kb0 + kb) * kGemmBK, c0);
            }
            __syncwarp();
            at.next();
        }
        if (lane == 0) *fills_issued = (uint32_t)kb;
    } else if (warp == 1) {
        RingPos<STAGES> at;
        for (int kb = 0; kb < blocks; ++kb) {
            const uint32_t buf = kb % kThinBuffers, use = kb / kThinBuffers;
            if (!__all_sync(0xffffffffu, wait(tempty + 8 * buf, (use & 1u) ^ 1u, kDevTimeoutMma) && wait(full + 8 * at.stage, at.phase, kDevTimeoutMma))) break;
            tcgen05_fence_after();
            const uint32_t a_addr = tiles_base + at.stage * cfg::kStageBytes;
            const uint64_t adesc = make_smem_desc(a_addr), bdesc = make_smem_desc(a_addr + kBM * kGemmBK);
            if (elect_one()) {
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4)
                    umma_f8(tmem + buf * N, adesc + (uint64_t)(k4 * 2), bdesc + (uint64_t)(k4 * 2), p.idesc, (uint32_t)(k4 != 0));
                umma_commit(tfull + 8 * buf);
                umma_commit(empty + 8 * at.stage);
            }
            __syncwarp();
            at.next();
        }
    } else if (warp < 4) {                       // scales: asynchronous 4-byte copies, one group per block
        const int t = threadIdx.x - 64;
        int fetched = 0;
        auto fetch = [&]() {
            if (fetched < blocks) {
                const uint32_t slot = scale_ring + (uint32_t)(fetched % kThinSlots) * cfg::kSlotBytes;
                const float* sl = p.SL + (int64_t)(kb0 + fetched) * p.ldsl;
                const float* sc = p.SC + (int64_t)(kb0 + fetched) * p.ldsc;
#pragma unroll
                for (int i = 0; i < kBM; i += 64) cp_async4(slot + (i + t) * 4, sl + (min(l0 + i + t, p.lanes - 1) >> p.shift_l));
#pragma unroll
                for (int i = 0; i < N; i += 64)
                    if (i + t < N) cp_async4(slot + (kBM + i + t) * 4, sc + (min(c0 + i + t, p.cols - 1) >> p.shift_c));
                ++fetched;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < kThinAhead; ++i) fetch();
        for (int g = 0; g < blocks; ++g) {
            const uint32_t bar = tfull + 8 * (g % kThinBuffers);
            if (g >= kThinBuffers && !__all_sync(0xffffffffu, wait(bar, ((g / kThinBuffers) & 1u) ^ 1u, kDevTimeoutProducer))) break;
            fetch();
            asm volatile("cp.async.wait_group %0;" ::"n"(kThinAhead) : "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {                                     // epilogue: lane = row of the lane operand
        const int quarter = warp & 3, from = ((warp >> 2) - 1) * NC;      // this warp's rows, and its columns of the tile
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)from;
#pragma unroll
        for (int j = 0; j < NC; ++j) acc[j] = 0.f;
        bool ok = true;
        for (int kb = 0; kb < blocks; ++kb) {
            const uint32_t buf = kb % kThinBuffers, slot = scale_ring + (uint32_t)(kb % kThinSlots) * cfg::kSlotBytes;
            ok &= wait(tfull + 8 * buf, (kb / kThinBuffers) & 1u, kDevTimeoutEpilogue);
            tcgen05_fence_after();
            const float scale = lds(slot + (quarter * 32 + lane) * 4);
            const uint64_t s2 = pack2(scale, scale);
            constexpr int P = NC < 32 ? NC : 32;
#pragma unroll
            for (int c = 0; c < NC; c += P) {
                uint32_t v[P];
                if constexpr (P == 32) tmem_ld32(taddr + buf * N + c, v);
                else tmem_ld16(taddr + buf * N + c, v);
                tmem_ld_wait();
                if (c + P == NC) {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty + 8 * buf);
                }
#pragma unroll
                for (int i = 0; i < P; i += 4) {         // the lane operand's scale first, then the other's (see kLeastScale)
                    float s[4], x[4];
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]) : "r"(slot + (kBM + from + c + i) * 4));
                    mul_pair(v[i], v[i + 1], s2, &x[0], &x[1]);
                    mul_pair(v[i + 2], v[i + 3], s2, &x[2], &x[3]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) fma1(acc[c + i + j], x[j], s[j]);
                }
            }
        }
        if (S > 1) {                             // totals to shared memory, [column][lane]; the stages are free: all MMAs have completed
            float* totals = reinterpret_cast<float*>(smem_raw + (tiles_base - raw));
            if (ok)
#pragma unroll
                for (int j = 0; j < NC; ++j) totals[(from + j) * kBM + quarter * 32 + lane] = acc[j];
        } else if (ok) {
            const int l = l0 + quarter * 32 + lane;
            if (l < p.lanes) {
                const T* cp = (const T*)p.C + (int64_t)l * p.c_lane;
                T* dp = (T*)p.D + (int64_t)l * p.d_lane;
#pragma unroll
                for (int j = 0; j < NC; ++j) {
                    const int col = c0 + from + j;
                    if (col < p.cols) dp[(int64_t)col * p.d_col] = to_type<T>(acc[j] + (p.C ? from_type<T>(cp[(int64_t)col * p.c_col]) : 0.f));
                }
            }
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {                           // nothing may be in flight when shared memory and TMEM go away; both waits are bounded
        if (warp == 1) {
            if (elect_one()) umma_commit(drain);         // by the lane that issued the MMAs
            mbar_wait_quiet(drain, 0, kDrainLimitNs);
        }
        if (warp == 0 && lane == 0) {
            const uint32_t fills = *fills_issued;
            for (uint32_t s = 0; s < (uint32_t)STAGES && s < fills; ++s) {
                const uint32_t last = s + STAGES * ((fills - 1 - s) / STAGES);
                mbar_wait_quiet(full + 8 * s, (last / STAGES) & 1u, kDrainLimitNs);
            }
        }
        __syncthreads();
    }
    if (S > 1) {
        cluster_sync_all();                      // every rank's totals are there
        if (warp >= 4) {                         // this rank's share of the columns, added in the order of the ranks
            const int row = ((int)threadIdx.x - 128) & 127, l = l0 + row;
            // (S, a power of two up to 8, divides 16: sixteen remote loads in flight are 16 / S whole columns)
            const int from = N / S * rank;
#pragma unroll 1
            for (int t0 = ((warp >> 2) - 1) * 16; t0 < N; t0 += 4 * cfg::kWarps) {      // 16 loads at a time, in turn between the parts
                float v[16], s = 0.f;
                const int j0 = from + t0 / S;
                if (c0 + j0 >= p.cols) break;
#pragma unroll
                for (int u = 0; u < 16; ++u)
                    v[u] = __uint_as_float(ld_cluster_u32(map_to_cta(tiles_base + (uint32_t)((j0 + u / S) * kBM + row) * 4, (uint32_t)(u & (S - 1)))));
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    s += v[u];
                    if (((u + 1) & (S - 1)) != 0) continue;
                    const int j = c0 + j0 + u / S;
                    if (l < p.lanes && j < p.cols) {
                        const int64_t dj = (int64_t)l * p.d_lane + (int64_t)j * p.d_col, cj = (int64_t)l * p.c_lane + (int64_t)j * p.c_col;
                        ((T*)p.D)[dj] = to_type<T>(s + (p.C ? from_type<T>(((const T*)p.C)[cj]) : 0.f));
                    }
                    s = 0.f;
                }
            }
        }
        cluster_sync_all();                      // nobody leaves while its totals are being read
    }
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cfg::kTmemCols) : "memory");
    }
}

// Time of a product in microseconds by each kind of tile, from measurements (B200, 1.7 to 1.9 GHz): `round` tiles run at once, each takes
// so much per block of k and for its output, and a launch takes the rest.  (256 x 256 tiles per pair: 1024 x 4096 x 4096, one round of 32 blocks, 27 us,
// 2048^3 18 us; 256 x 128: 512 x 4096 x 4096 21 us, 1001 x 1999 x 1100, nine blocks, 14 us; CTAs of their own, 128 x 128 with k split in
// four: 128 x 4096 x 4096 13.7 us, 1024 x 1024 x 8192 split in two 23.4 us; each a call by itself.  In a stream of calls: 23, 15, 18, 12, 13, 24.)
double pair_cost(const Fp8GemmArgs& a, int width, int sm_count) {
    const double tiles = (double)((a.m + 255) / 256) * (double)((a.n + width - 1) / width), rounds = std::ceil(tiles / (sm_count / 2));
    const double blocks = (double)((a.k + kScaleBlock - 1) / kScaleBlock), cols = a.B.block == 1;
    if (width == 256) return 9.0 + rounds * (blocks * (0.53 + 0.17 * cols) + 2.0);
    return 9.0 + rounds * (blocks * ((rounds > 1 ? 0.40 : 0.30) + 0.17 * cols) + 1.5);
}

// CTAs of clusters of 1, 2, 4 and 8 (index: logarithm) that are resident at once: larger clusters leave SMs of a GPC without a place.
// One CTA per SM for every column count, so that one kernel speaks for all.
struct ThinCapacity { int ctas[4]; };
cudaError_t thin_capacity(int sm_count, ThinCapacity* out) {
    static ThinCapacity known[kMaxDevices] = {};
    ThinCapacity& k = known[current_device_slot()];
    if (!k.ctas[0]) {
        using cfg = ThinCfg<128>;
        cudaError_t err = cudaFuncSetAttribute(fp8_gemm_thin_kernel<float, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg::kSmem);
        if (err != cudaSuccess) return err;
        ThinCapacity c = {{sm_count, 0, 0, 0}};
        for (int i = 1; i < 4; ++i) {
            cudaLaunchConfig_t qc = {};
            qc.gridDim = dim3((unsigned)(sm_count >> i << i));
            qc.blockDim = dim3(cfg::kThreads);
            qc.dynamicSmemBytes = cfg::kSmem;
            cudaLaunchAttribute qa[1];
            qa[0].id = cudaLaunchAttributeClusterDimension;
            qa[0].val.clusterDim.x = 1u << i;
            qa[0].val.clusterDim.y = 1;
            qa[0].val.clusterDim.z = 1;
            qc.attrs = qa;
            qc.numAttrs = 1;
            int clusters = 0;
            if ((err = cudaOccupancyMaxActiveClusters(&clusters, fp8_gemm_thin_kernel<float, 128>, &qc)) != cudaSuccess) return err;
            c.ctas[i] = clusters << i;
        }
        k = c;
    }
    *out = k;
    return cudaSuccess;
}

// How often the blocks of k are split: the least number of rounds of CTAs, each weighed by its length; at least two blocks each.
int thin_split(int64_t tiles, int64_t kblocks, const ThinCapacity& room, double* cost_out) {
    int best = 1;
    double best_cost = 1e30;
    for (int i = 0; i < 4; ++i) {
        const int S = 1 << i;
        if (S > 1 && (kblocks < 2 * S || room.ctas[i] == 0)) break;
        const int64_t rounds = (tiles * S + room.ctas[i] - 1) / room.ctas[i];
        const double cost = (double)rounds * ((double)((kblocks + S - 1) / S) + 6.0);      // a round's fixed part is about six blocks
        if (cost < best_cost * 0.999) { best = S; best_cost = cost; }
    }
    if (cost_out) *cost_out = best_cost;
    return best;
}

template <typename T, int N>
cudaError_t launch_thin(const Fp8GemmArgs& a, bool swapped, const ThinCapacity& room, cudaStream_t st, int* launches) {
    using cfg = ThinCfg<N>;
    static bool ready_dev[kMaxDevices] = {};
    bool& ready = ready_dev[current_device_slot()];
    if (!ready) {
        cudaError_t err = cudaFuncSetAttribute(fp8_gemm_thin_kernel<T, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg::kSmem);
        if (err != cudaSuccess) return err;
        ready = true;
    }
    const Fp8Operand &L = swapped ? a.B : a.A, &R = swapped ? a.A : a.B;
    ThinParams p = {};
    p.lanes = (int)(swapped ? a.n : a.m);
    p.cols = (int)(swapped ? a.m : a.n);
    CUtensorMap map_l, map_c;
    if (!make_byte_map(&map_l, L.Q, p.lanes, a.k, L.ld, kBM) || !make_byte_map(&map_c, R.Q, p.cols, a.k, R.ld, N)) return cudaErrorInvalidValue;
    p.kblocks = (int)((a.k + kScaleBlock - 1) / kScaleBlock);
    p.lane_tiles = (p.lanes + kBM - 1) / kBM;
    p.SL = L.S; p.SC = R.S; p.ldsl = L.lds; p.ldsc = R.lds;
    p.shift_l = L.block == 1 ? 0 : 7; p.shift_c = R.block == 1 ? 0 : 7;
    p.idesc = make_idesc_f8(L.fmt, R.fmt, kBM, N);
    p.C = a.C; p.c_lane = swapped ? 1 : a.ldc; p.c_col = swapped ? a.ldc : 1;
    p.D = a.D; p.d_lane = swapped ? 1 : a.ldd; p.d_col = swapped ? a.ldd : 1;
    p.dev_status = a.dev_status;
    p.wait_ns = kWaitLimitNs;
    const int64_t tiles = (int64_t)p.lane_tiles * ((p.cols + N - 1) / N);
    const int S = thin_split(tiles, p.kblocks, room, nullptr);
    if (tiles * S > INT32_MAX) return cudaErrorInvalidValue;
    cudaError_t err = launch_chained_cluster(fp8_gemm_thin_kernel<T, N>, dim3((unsigned)(tiles * S)), dim3(cfg::kThreads), cfg::kSmem, S, st, map_l, map_c, p);
    if (err == cudaSuccess) ++*launches;
    return err;
}

template <typename T, int BN>
cudaError_t launch_pair_scales(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    if (a.C) return a.B.block == 1 ? launch_pair<T, BN, true, true>(a, sm_count, st, launches) : launch_pair<T, BN, false, true>(a, sm_count, st, launches);
    return a.B.block == 1 ? launch_pair<T, BN, true, false>(a, sm_count, st, launches) : launch_pair<T, BN, false, false>(a, sm_count, st, launches);
}

template <typename T>
cudaError_t launch_typed(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    const bool swapped = !(a.n <= 64 && a.m > a.n);        // lanes run along the rows of B, so that stores run along rows of D, unless B has few
    const int64_t cols = swapped ? a.m : a.n, lanes = swapped ? a.n : a.m;
    ThinCapacity room;
    if (cudaError_t err = thin_capacity(sm_count, &room)) return err;
    if (cols > 64) {                                       // (up to 64 columns a narrower tile reads the lane operand once, which is all there is to do)
        double thin;
        thin_split((lanes + kBM - 1) / kBM * ((cols + 127) / 128), (a.k + kScaleBlock - 1) / kScaleBlock, room, &thin);
        thin = 8.0 + 0.40 * thin;
        const double wide = pair_cost(a, 256, sm_count), narrow = pair_cost(a, 128, sm_count);
        if (wide <= narrow && wide <= thin) return launch_pair_scales<T, 256>(a, sm_count, st, launches);
        if (narrow <= thin) return launch_pair_scales<T, 128>(a, sm_count, st, launches);
    }
    if (cols <= 16) return launch_thin<T, 16>(a, swapped, room, st, launches);
    if (cols <= 32) return launch_thin<T, 32>(a, swapped, room, st, launches);
    if (cols <= 64) return launch_thin<T, 64>(a, swapped, room, st, launches);
    return launch_thin<T, 128>(a, swapped, room, st, launches);
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_typed<float>(a, sm_count, st, launches);
    if (a.type == kF16) return launch_typed<__half>(a, sm_count, st, launches);
    return launch_typed<__nv_bfloat16>(a, sm_count, st, launches);
}

}  // namespace gemm2m
