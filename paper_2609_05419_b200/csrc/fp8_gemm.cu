// Product of two 8-bit floating-point matrices with block scales,
//   D[i, j] = C[i, j] + sum_b SA[i / block, b] SB[j / block, b] sum_{p in block b} A[i, p] B[j, p],
// blocks of 128 along k.  Every block's sum is accumulated in 32 bits, scaled, and added to a 32-bit total; D is rounded once.
//
// A block of 128 entries is one 128-byte swizzle row, so one pipeline stage, so four MMAs (K = 32).  Since the scales differ from
// block to block, the tensor core's accumulator holds one block's sums only: it is written afresh every four MMAs, into two TMEM buffers in
// turn, and eight epilogue warps per CTA read each back, multiply by the scales and add to totals in registers (128 per
// thread) while the other buffer is being filled.  256 x 256 tiles per CTA pair: the four MMAs of a block take 512 cycles, the
// 128 x 256 multiply-adds of a CTA's half 256 cycles of the FP32 pipes (512 with a scale per column), as packed pairs.
#include "layer_ops.cuh"
#include "pair_pipeline.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

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

// Ring of scale slots, one per block; a slot is written 3 blocks ahead.  A block's scales are there when its tfull barrier completes (the
// two scale warps arrive on it next to the commit).  They turn to block g after tfull of block g - 2: the MMAs of g - 2 were issued
// after every epilogue warp had released block g - 4, so all of them are through with block g - 5, whose slot is that of g + 3.
constexpr int kSlots = 8, kAhead = 3, kScaleWarps = 2;

template <int BN, bool COLS>
struct Cfg {
    static constexpr int kHalfRows = BN / 2;                          // rows of B per CTA
    static constexpr int kStageBytes = (kBM + kHalfRows) * kGemmBK;
    static constexpr int kStages = BN == 256 ? 6 : 8;
    static constexpr int kCols = BN / 2;                              // columns per epilogue warp: totals per thread
    static constexpr uint32_t kTmemCols = 2 * BN;
    static constexpr int kSlotFloats = kBM + (COLS ? BN : 2);         // scales of one block: 128 rows, and the columns or their two halves
    static constexpr int kSlotBytes = (kSlotFloats * 4 + 15) / 16 * 16;
    static constexpr size_t kScaleBytes = (size_t)kSlots * kSlotBytes;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 + kScaleBytes + PairPipe<kStages>::kBytes;
};

struct Fp8GemmParams {
    int m, n, kblocks, tiles_r, tiles_c, band;
    const float *SA, *SB;
    int64_t ldsa, ldsb;
    int shift_a, shift_b;                // row r has the scale r >> shift (0 or 7)
    uint32_t idesc;
    const void* C; int64_t ldc;
    void* D; int64_t ldd;
    int type;
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

// NT totals of one row, columns [col, col + NT) of which those below n exist, to D (plus C).  Whole 16-byte pieces where the
// row's address allows it.
template <typename T, int NT>
__device__ __forceinline__ void store_row(const float* v, const T* crow, T* drow, int col, int n) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool vec = ((reinterpret_cast<uintptr_t>(drow + col) | (crow ? reinterpret_cast<uintptr_t>(crow + col) : 0)) & 15) == 0;
#pragma unroll
    for (int i = 0; i < NT; i += V) {
        if (vec && col + i + V <= n) {
            T out[V], in[V];
            if (crow) *reinterpret_cast<uint4*>(in) = *reinterpret_cast<const uint4*>(crow + col + i);
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = to_type<T>(v[i + j] + (crow ? from_type<T>(in[j]) : 0.f));
            *reinterpret_cast<uint4*>(drow + col + i) = *reinterpret_cast<const uint4*>(out);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (col + i + j < n) drow[col + i + j] = to_type<T>(v[i + j] + (crow ? from_type<T>(crow[col + i + j]) : 0.f));
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

// COLS: B has a scale per row (of B; column of D) and block, otherwise one per 128 rows.
template <int BN, bool COLS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
fp8_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Fp8GemmParams p) {
    using cfg = Cfg<BN, COLS>;
    constexpr int STAGES = cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles_base = (raw + 1023u) & ~1023u;
    unsigned char* behind = smem_raw + (tiles_base - raw) + (size_t)STAGES * cfg::kStageBytes;
    const uint32_t scale_ring = smem_u32(behind);
    PairPipe<STAGES> pipe;
    pipe.open(behind + cfg::kScaleBytes, kEpilogueWarps, 1 + kScaleWarps, cfg::kTmemCols, p.dev_status, p.wait_ns);
    wait_for_prior_kernels();

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    const int total_tiles = p.tiles_r * p.tiles_c;

    if (warp < kFirstEpilogueWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPipeRegs));
        if (warp == 0 && lane == 0) {                     // copies, both CTAs
            const uint32_t leader_full = map_to_cta(pipe.full, 0);
            RingPos<STAGES> at;
            uint32_t fills = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
                int tr, tc;
                tile_at(p, tile, &tr, &tc);
                const int row0 = tr * (2 * kBM) + (int)pipe.rank * kBM, col0 = tc * BN + (int)pipe.rank * cfg::kHalfRows;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!(ok = pipe.wait(pipe.empty + 8 * at.stage, at.phase ^ 1u, kDevTimeoutProducer))) break;
                    const uint32_t dst = tiles_base + at.stage * cfg::kStageBytes;
                    if (pipe.rank == 0) mbar_arrive_expect_tx(pipe.full + 8 * at.stage, 2 * cfg::kStageBytes);
                    tma_load_2d_pair(dst, &map_a, leader_full + 8 * at.stage, kb * kGemmBK, row0);
                    tma_load_2d_pair(dst + kBM * kGemmBK, &map_b, leader_full + 8 * at.stage, kb * kGemmBK, col0);
                    ++fills;
                    at.next();
                }
            }
            *pipe.fills_issued = fills;
            if (!ok) pipe.tell_peer();
        } else if (warp == 1 && lane == 0 && pipe.rank == 0) {      // MMAs, leader
            RingPos<STAGES> at;
            uint32_t it = 0;                              // block counter over all tiles: buffer it & 1, its use number it >> 1
            bool ok = true;
            for (int tile = pair; ok && tile < total_tiles; tile += npairs)
                for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
                    const uint32_t buf = it & 1u;
                    if (!(ok = pipe.wait(pipe.tempty + 8 * buf, ((it >> 1) & 1u) ^ 1u, kDevTimeoutMma) &&
                               pipe.wait(pipe.full + 8 * at.stage, at.phase, kDevTimeoutMma))) break;
                    tcgen05_fence_after();
                    const uint32_t a_addr = tiles_base + at.stage * cfg::kStageBytes;
                    const uint64_t adesc = make_smem_desc(a_addr), bdesc = make_smem_desc(a_addr + kBM * kGemmBK);
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4)
                        umma_f8_pair(pipe.tmem + buf * BN, adesc + (uint64_t)(k4 * 2), bdesc + (uint64_t)(k4 * 2), p.idesc, (uint32_t)(k4 != 0));
                    umma_commit_pair(pipe.empty + 8 * at.stage, 3);
                    umma_commit_pair(pipe.tfull + 8 * buf, 3);
                    at.next();
                }
            if (!ok) pipe.tell_peer();
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
                const uint32_t bar = pipe.tfull + 8 * (g & 1u);
                if (g >= 2 && !(ok = __all_sync(0xffffffffu, pipe.wait(bar, ((g >> 1) & 1u) ^ 1u, kDevTimeoutProducer)))) break;
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
        const uint32_t leader_tempty = map_to_cta(pipe.tempty, 0);
        uint32_t it = 0;
        bool ok = true;
        for (int tile = pair; ok && tile < total_tiles; tile += npairs) {
            int tr, tc;
            tile_at(p, tile, &tr, &tc);
            const int row = tr * (2 * kBM) + (int)pipe.rank * kBM + quarter * 32 + lane;
            const int col0 = tc * BN + half * NC;
            uint64_t acc[NC / 2];
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) acc[i] = 0;
            for (int kb = p.kblocks; kb > 0; --kb, ++it) {
                const uint32_t buf = it & 1u;
                // (a wait that gives up is acted on at the end of the tile: every later one then returns at once)
                ok &= pipe.wait(pipe.tfull + 8 * buf, (it >> 1) & 1u, kDevTimeoutEpilogue);
                tcgen05_fence_after();
                const uint32_t slot = (it & (kSlots - 1)) * cfg::kSlotBytes, col_scale = col_slot + slot;
                float scale = lds(row_slot + slot);
                if (!COLS) scale *= lds(col_scale);
                const uint64_t s2 = pack2(scale, scale);
                const uint32_t at = taddr + buf * BN;
                uint32_t v[2][32];                        // one piece is on its way while the other is added
                tmem_ld32(at, v[0]);
#pragma unroll
                for (int c = 0; c < NC; c += 32) {
                    const uint32_t(&w)[32] = v[(c / 32) & 1];
                    tmem_ld_wait();
                    if (c + 32 < NC) tmem_ld32(at + c + 32, v[(c / 32 + 1) & 1]);
                    else pipe.release_at(leader_tempty + 8 * buf);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        uint64_t x = s2, y = s2;
                        if (COLS) {
                            uint64_t f, g;
                            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f), "=l"(g) : "r"(col_scale + (c + i) * 4));
                            x = mul2(s2, f);
                            y = mul2(s2, g);
                        }
                        fma2(acc[(c + i) / 2], pack2(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), x);
                        fma2(acc[(c + i) / 2 + 1], pack2(__uint_as_float(w[i + 2]), __uint_as_float(w[i + 3])), y);
                    }
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (ok && row < p.m && col0 < p.n) {
                float t[NC];
#pragma unroll
                for (int i = 0; i < NC / 2; ++i) unpack2(acc[i], &t[2 * i], &t[2 * i + 1]);
                const int64_t dr = (int64_t)row * p.ldd, cr = (int64_t)row * p.ldc;
                if (p.type == kF32) store_row<float, NC>(t, p.C ? (const float*)p.C + cr : nullptr, (float*)p.D + dr, col0, p.n);
                else if (p.type == kF16) store_row<__half, NC>(t, p.C ? (const __half*)p.C + cr : nullptr, (__half*)p.D + dr, col0, p.n);
                else store_row<__nv_bfloat16, NC>(t, p.C ? (const __nv_bfloat16*)p.C + cr : nullptr, (__nv_bfloat16*)p.D + dr, col0, p.n);
            }
        }
        if (!ok && lane == 0) pipe.tell_peer();
    }
    pipe.close(cfg::kTmemCols, cfg::kStageBytes);
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

template <int BN, bool COLS>
cudaError_t launch_pair(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    static int pairs_dev[kMaxDevices] = {};
    int& max_pairs = pairs_dev[current_device_slot()];
    if (!max_pairs) {
        int pairs = 0;
        cudaError_t err = resident_pairs(fp8_gemm_pair_kernel<BN, COLS>, kThreads, Cfg<BN, COLS>::kSmem, sm_count, &pairs);
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
    p.C = a.C; p.ldc = a.ldc; p.D = a.D; p.ldd = a.ldd; p.type = a.type;
    p.dev_status = a.dev_status;
    p.wait_ns = kWaitLimitNs;
    const int pairs = (int)(tr * tc < max_pairs ? tr * tc : max_pairs);
    cudaError_t err = launch_chained(fp8_gemm_pair_kernel<BN, COLS>, dim3(2 * pairs), dim3(kThreads), Cfg<BN, COLS>::kSmem, st, map_a, map_b, p);
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    return a.B.block == 1 ? launch_pair<256, true>(a, sm_count, st, launches) : launch_pair<256, false>(a, sm_count, st, launches);
}

}  // namespace gemm2m
