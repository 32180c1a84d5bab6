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
    static constexpr int kStages = 5;
    static constexpr int kCols = BN / 2;                              // columns per epilogue warp: totals per thread
    static constexpr uint32_t kTmemCols = 2 * BN;
    static constexpr int kSlotFloats = kBM + (COLS ? BN : 2);         // scales of one block: 128 rows, and the columns or their two halves
    static constexpr int kSlotBytes = (kSlotFloats * 4 + 15) / 16 * 16;
    static constexpr size_t kScaleBytes = (size_t)kSlots * kSlotBytes;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 + kScaleBytes + PairPipe<kStages>::kBytes + 16 + kEpilogueWarps * 4096;
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
template <typename T, int NC>
__device__ __forceinline__ void store_rows(const float (&v)[NC], uint32_t turn, const T* C, int64_t ldc, T* D, int64_t ldd, int row0, int col0, int m, int n, bool vec) {
    const int lane = threadIdx.x & 31, piece = lane & 7;
    struct alignas(4 * sizeof(T)) Four { T t[4]; };
#pragma unroll
    for (int c = 0; c < NC; c += 32) {
        __syncwarp();                                     // the previous columns have been read
#pragma unroll
        for (int q = 0; q < 8; ++q)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (uint32_t)(lane * 128 + ((q ^ (lane & 7)) << 4))), "f"(v[c + 4 * q]),
                         "f"(v[c + 4 * q + 1]), "f"(v[c + 4 * q + 2]), "f"(v[c + 4 * q + 3]) : "memory");
        __syncwarp();
        const int col = col0 + c + piece * 4;
        const int rows = col < n ? min(32, m - row0) : 0;
#pragma unroll 2
        for (int r = lane >> 3; r < rows; r += 4) {       // (kept short: this code is fetched anew for every tile)
            float x[4];
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3])
                         : "r"(turn + (uint32_t)(r * 128 + ((piece ^ (r & 7)) << 4))) : "memory");
            T* d = D + (int64_t)(row0 + r) * ldd + col;
            const T* s = C ? C + (int64_t)(row0 + r) * ldc + col : nullptr;
            if (vec && col + 4 <= n) {
                Four f;
                if (s) {
                    f = *reinterpret_cast<const Four*>(s);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] += from_type<T>(f.t[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) f.t[j] = to_type<T>(x[j]);
                *reinterpret_cast<Four*>(d) = f;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < n) d[j] = to_type<T>(x[j] + (s ? from_type<T>(s[j]) : 0.f));
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

// T: type of C and D.  COLS: B has a scale per row (of B; column of D) and block, otherwise one per 128 rows.
template <typename T, int BN, bool COLS>
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
        const uint32_t turn = smem_u32(behind) + (uint32_t)(cfg::kScaleBytes + PairPipe<STAGES>::kBytes + 15) / 16 * 16 + (uint32_t)(warp - kFirstEpilogueWarp) * 4096;
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
                        float s[4] = {scale, scale, scale, scale};
                        if (COLS) {
                            uint64_t f, g;
                            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f), "=l"(g) : "r"(col_scale + (c + i) * 4));
                            unpack2(mul2(s2, f), &s[0], &s[1]);
                            unpack2(mul2(s2, g), &s[2], &s[3]);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) fma1(acc[c + i + j], __uint_as_float(w[i + j]), s[j]);
                    }
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            if (ok && row0 < p.m && col0 < p.n) {
                store_rows<T, NC>(acc, turn, (const T*)p.C, p.ldc, (T*)p.D, p.ldd, row0, col0, p.m, p.n, p.vec != 0);
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

template <typename T, int BN, bool COLS>
cudaError_t launch_pair(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    static int pairs_dev[kMaxDevices] = {};
    int& max_pairs = pairs_dev[current_device_slot()];
    if (!max_pairs) {
        int pairs = 0;
        cudaError_t err = resident_pairs(fp8_gemm_pair_kernel<T, BN, COLS>, kThreads, Cfg<BN, COLS>::kSmem, sm_count, &pairs);
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
    cudaError_t err = launch_chained(fp8_gemm_pair_kernel<T, BN, COLS>, dim3(2 * pairs), dim3(kThreads), Cfg<BN, COLS>::kSmem, st, map_a, map_b, p);
    if (err == cudaSuccess) ++*launches;
    return err;
}

template <typename T>
cudaError_t launch_typed(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    return a.B.block == 1 ? launch_pair<T, 256, true>(a, sm_count, st, launches) : launch_pair<T, 256, false>(a, sm_count, st, launches);
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, int sm_count, cudaStream_t st, int* launches) {
    if (a.type == kF32) return launch_typed<float>(a, sm_count, st, launches);
    if (a.type == kF16) return launch_typed<__half>(a, sm_count, st, launches);
    return launch_typed<__nv_bfloat16>(a, sm_count, st, launches);
}

}  // namespace gemm2m
