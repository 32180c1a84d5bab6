// Low-rank updates of many adapters, many tokens: tiles of 128 tokens of one adapter on the tensor cores (tcgen05, one CTA per tile).
//
// L = X A_a^T: a block takes a tile and a piece of k, in steps of 64 entries (one 128-byte swizzle row): four MMAs of 128 x rank x 16 per step.  The tile's rows of X lie
// anywhere, so they come by asynchronous 16-byte copies (8- and 4-byte ones where rows start there), three or four steps ahead.
// D = C + L B_a^T: a block takes a tile and pieces of 128 columns.  L, as hi + lo, stays in shared memory; the MMAs of one piece run while the one before is
// read back, added to what was fetched of C a piece earlier, and stored.  The read-back hands a lane pairs of columns 8 apart; the rows of B
// lie in shared memory in such an order that these are eight neighbouring columns of D.
#include "adapters.cuh"
#include "gemm_ptx.cuh"

namespace gemm2m {

namespace {

constexpr int kThreads = 256;
constexpr int kRowBytes = 128;                           // 64 entries of the inner dimension
constexpr int kOperandBytes = kManyTile * kRowBytes;

__device__ __forceinline__ bool elect_lane() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor of kind::f16: operands of one 16-bit type, K-major, 32-bit accumulator, 128 x N tile.
uint32_t make_idesc(int type, int N) {
    const uint32_t t = type == kBF16 ? 1u : 0u;
    return (1u << 4) | (t << 7) | (t << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kManyTile >> 4) << 24);
}

// Eight 16-bit entries of a row, from entry `at` on, into 16 bytes of shared memory; those at or beyond `end` become zero.  align: bytes that rows are aligned to.
__device__ __forceinline__ void copy8(uint32_t dst, const uint16_t* row, int64_t at, int64_t end, int align) {
    const int valid = (int)max((int64_t)0, min((int64_t)8, end - at));
    if (align >= 16) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(valid ? row + at : row), "r"(valid * 2) : "memory");
    } else if (align == 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int v = min(4, max(0, valid - 4 * i));
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst + 8 * i), "l"(v ? row + at + 4 * i : row), "r"(v * 2) : "memory");
        }
    } else if (align == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = min(2, max(0, valid - 2 * i));
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * i), "l"(v ? row + at + 2 * i : row), "r"(v * 2) : "memory");
        }
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = (2 * i < valid ? (uint32_t)row[at + 2 * i] : 0u) | (2 * i + 1 < valid ? (uint32_t)row[at + 2 * i + 1] << 16 : 0u);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 16 rows of 32 columns of an accumulator: lane (g, q) of a warp receives columns 8j + 2q, 8j + 2q + 1 of row g in v[4j], v[4j + 1] and of row g + 8 in v[4j + 2], v[4j + 3].
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}

// 16-byte piece `piece` of row `row` of an operand (8 pieces a row, 128-byte swizzle).
__device__ __forceinline__ uint32_t swizzled(uint32_t base, int row, int piece) { return base + (uint32_t)(row * kRowBytes + ((piece ^ (row & 7)) << 4)); }

// Barriers and TMEM of a block; give-up: the flag is set, everybody leaves, and nothing is in flight when TMEM goes.
template <int BARS>
struct Frame {
    uint32_t bars, tmem;
    volatile int* abort_flag;
    int* dev_status;
    // `mem`: 8 (BARS + 1) + 8 bytes of shared memory, 8-byte aligned
    __device__ __forceinline__ void open(uint64_t* mem, uint32_t cols, int* status) {
        bars = smem_u32(mem);
        uint32_t* slot = reinterpret_cast<uint32_t*>(mem + BARS + 1);
        abort_flag = reinterpret_cast<volatile int*>(slot + 1);
        dev_status = status;
        if (threadIdx.x == 0) {
            for (int i = 0; i <= BARS; ++i) mbar_init(bars + 8 * i, 1);
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            fence_async_proxy();
        }
        if (threadIdx.x >> 5 == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tcgen05_fence_before();
        __syncthreads();
        tcgen05_fence_after();
        tmem = *slot;
    }
    __device__ __forceinline__ bool wait(int bar, uint32_t parity, int code) const { return mbar_wait(bars + 8 * bar, parity, abort_flag, dev_status, code, kWaitLimitNs); }
    // The same for a converged warp, which stays so.
    __device__ __forceinline__ bool wait_warp(int bar, uint32_t parity, int code) const { return __all_sync(0xffffffffu, wait(bar, parity, code)); }
    // All threads, when they have left their loops.
    __device__ __forceinline__ void close(uint32_t cols) const {
        asm volatile("cp.async.wait_all;" ::: "memory");
        tcgen05_fence_before();
        __syncthreads();
        if (*abort_flag) {
            if (threadIdx.x >> 5 == 0) {                 // the lane that issued the MMAs commits them once more
                if (elect_lane()) umma_commit(bars + 8 * BARS);
                __syncwarp();
                mbar_wait_quiet(bars + 8 * BARS, 0, kDrainLimitNs);
            }
            __syncthreads();
        }
        if (threadIdx.x >> 5 == 1) {
            tcgen05_fence_after();
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
        }
    }
};

// RP: padded rank, S: stages.
template <int RP, int S>
__global__ void __launch_bounds__(kThreads, 2) adapter_down_many_kernel(const AdapterArgs a, const AdapterLayout l, int64_t per, int align, uint32_t idesc, int* dev_status) {
    constexpr int kStageBytes = kOperandBytes + RP * kRowBytes, kTmemCols = RP < 32 ? 32 : RP;
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint64_t bars[S + 2];
    wait_for_prior_kernels();
    if ((int)blockIdx.x >= *(const int32_t*)(a.ws + l.off_count)) return;
    const AdapterTile tile = ((const AdapterTile*)(a.ws + l.off_tiles))[blockIdx.x];
    const int32_t* tokens = (const int32_t*)(a.ws + l.off_perm) + tile.start;
    const int rank = rank_of(a, tile.key);
    if (rank == 0) return;
    Frame<S> frame;
    frame.open(bars, kTmemCols, dev_status);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // this thread copies piece `piece` of rows row0, row0 + 32, ...
    const int piece = threadIdx.x & 7, row0 = threadIdx.x >> 3;
    const uint16_t* x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (const uint16_t*)a.X + (row0 + 32 * j < tile.count ? tokens[row0 + 32 * j] : 0) * a.ldx;
    const uint16_t* A = (const uint16_t*)a.A + tile.key * a.stride_a + row0 * a.lda;
    const int64_t total = (a.k + 63) / 64, first = blockIdx.y * per;
    const int steps = (int)(min(total, first + per) - first);
    auto load = [&](int step) {
        const uint32_t stage = base + (uint32_t)(step % S) * kStageBytes;
        const int64_t at = (first + step) * 64 + piece * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (row0 + 32 * j < tile.count) copy8(swizzled(stage, row0 + 32 * j, piece), x[j], at, a.k, align);
#pragma unroll
        for (int j = 0; j < (RP + 31) / 32; ++j)
            if (row0 + 32 * j < rank) copy8(swizzled(stage + kOperandBytes, row0 + 32 * j, piece), A + 32 * j * a.lda, at, a.k, align);
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
        if (i < steps) load(i);
        copies_commit();
    }
    for (int i = 0; i < steps; ++i) {
        copies_wait<S - 2>();
        fence_async_proxy();
        // the stage that is filled next was read by the MMAs of the step before
        if (warp == 0 && i > 0) frame.wait_warp((i - 1) % S, (uint32_t)((i - 1) / S) & 1u, kDevTimeoutProducer);
        __syncthreads();
        if (*frame.abort_flag) break;
        if (warp == 0) {
            tcgen05_fence_after();
            const uint32_t stage = base + (uint32_t)(i % S) * kStageBytes;
            const uint64_t adesc = make_smem_desc(stage), bdesc = make_smem_desc(stage + kOperandBytes);
            if (elect_lane()) {
#pragma unroll
                for (int s = 0; s < 4; ++s) umma_f16(frame.tmem, adesc + (uint64_t)(s * 2), bdesc + (uint64_t)(s * 2), idesc, (uint32_t)((i | s) != 0));
                umma_commit(frame.bars + 8 * (i % S));
            }
            __syncwarp();
        }
        if (i + S - 1 < steps) load(i + S - 1);
        copies_commit();
    }
    // (not the abort flag: a wait that is given up fails at once here too)
    if (frame.wait_warp((steps - 1) % S, (uint32_t)((steps - 1) / S) & 1u, kDevTimeoutEpilogue)) {
        tcgen05_fence_after();
        const int row = (warp & 3) * 32 + lane;
        float* low = (float*)(a.ws + l.off_low) + (blockIdx.y * a.tokens + (row < tile.count ? tokens[row] : 0)) * RP;
        for (int c = (warp >> 2) * 16; c < RP; c += 32) {
            uint32_t v[16];
            tmem_ld16(frame.tmem + ((uint32_t)((warp & 3) * 32) << 16) + c, v);
            tmem_ld_wait();
            if (row < tile.count)
#pragma unroll
                for (int j = 0; j < 16; j += 4) *reinterpret_cast<uint4*>(low + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
    }
    frame.close(kTmemCols);
}

// T: type of B (and of L's two parts), DT: of C and D; KB blocks of 64 along the rank.
template <typename T, typename DT, int KB>
__global__ void __launch_bounds__(kThreads, KB == 1 ? 2 : 1) adapter_up_many_kernel(const AdapterArgs a, const AdapterLayout l, int splits, int align, int vec_d, uint32_t idesc,
                                                                                  int* dev_status) {
    constexpr int kTmemCols = 256, E = 16 / (int)sizeof(DT), kAccesses = 8 / E;      // eight columns of a row per lane, E in one access
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint64_t bars[4];
    __shared__ float backs[kManyTile];
    wait_for_prior_kernels();
    if ((int)blockIdx.x >= *(const int32_t*)(a.ws + l.off_count)) return;
    const AdapterTile tile = ((const AdapterTile*)(a.ws + l.off_tiles))[blockIdx.x];
    const int32_t* tokens = (const int32_t*)(a.ws + l.off_perm) + tile.start;
    const int rank = rank_of(a, tile.key);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const DT* C = (const DT*)a.C;
    DT* D = (DT*)a.D;
    // pieces of 128 columns, dealt out in turn: the blocks of a tile of tokens read and write neighbouring columns at about the same time
    const int64_t all = (a.n + kManyTile - 1) / kManyTile, tiles = (all - blockIdx.y + gridDim.y - 1) / gridDim.y;
    auto column0 = [&](int64_t t) { return (t * gridDim.y + blockIdx.y) * kManyTile; };
    if (rank == 0) {                                     // D = C, or zero
        if (a.C == a.D) return;
        for (int64_t t = 0; t < tiles; ++t)
            for (int i = threadIdx.x; i < tile.count * (kManyTile / E); i += kThreads) {
                const int64_t row = tokens[i / (kManyTile / E)], c = column0(t) + i % (kManyTile / E) * E;
                if (vec_d && c + E <= a.n) {
                    *reinterpret_cast<uint4*>(D + row * a.ldd + c) = C ? *reinterpret_cast<const uint4*>(C + row * a.ldc + c) : make_uint4(0, 0, 0, 0);
                } else {
                    for (int64_t j = c; j < min(a.n, c + E); ++j) D[row * a.ldd + j] = C ? C[row * a.ldc + j] : DT(0.f);
                }
            }
        return;
    }
    Frame<2> frame;
    frame.open(bars, kTmemCols, dev_status);
    const uint32_t low_hi = (smem_u32(smem_raw) + 1023u) & ~1023u, low_lo = low_hi + KB * kOperandBytes, b_base = low_lo + KB * kOperandBytes;

    const uint16_t* B = (const uint16_t*)a.B + tile.key * a.stride_b;
    const int ksteps = (rank + 15) / 16, pieces = 2 * ksteps;         // 16-byte pieces of a row of B that the MMAs read
    auto load_b = [&](int64_t t) {
        const uint32_t dst = b_base + (uint32_t)(t & 1) * (KB * kOperandBytes);
        for (int i = threadIdx.x; i < kManyTile * 8 * KB; i += kThreads) {
            const int piece = i % (8 * KB), c = i / (8 * KB);
            const int64_t col = column0(t) + c;
            const int row = (c & 96) | (c & 6) << 2 | (c & 24) >> 2 | (c & 1);      // columns 8q + 2j + e of every 32 are rows 8j + 2q + e
            if (piece < pieces && col < a.n) copy8(swizzled(dst + (piece >> 3) * kOperandBytes, row, piece & 7), B + col * a.ldb, piece * 8, rank, align);
        }
    };
    load_b(0);
    copies_commit();
    {
        // L: a warp adds the pieces of 16 rows up, all their loads of a piece in flight together, times s_a, and brings each row's largest entry near 1
        constexpr int kRows = kManyTile / (kThreads / 32);
        const float scale = a.scales ? a.scales[tile.key] : 1.f;
        const int token = lane < kRows && warp * kRows + lane < tile.count ? tokens[warp * kRows + lane] : 0;
        const float* low = (const float*)(a.ws + l.off_low) + lane * 2;
        const float* p[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) p[i] = low + (int64_t)__shfl_sync(0xffffffffu, token, i) * l.padded;
        float2 v[KB][kRows];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) v[b][i] = make_float2(0.f, 0.f);
            if (b * 64 + lane * 2 < rank)
                for (int s = 0; s < splits; ++s) {
                    float2 w[kRows];
#pragma unroll
                    for (int i = 0; i < kRows; ++i) w[i] = *reinterpret_cast<const float2*>(p[i] + s * a.tokens * l.padded + b * 64);
#pragma unroll
                    for (int i = 0; i < kRows; ++i) v[b][i].x += w[i].x, v[b][i].y += w[i].y;
                }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = warp * kRows + i;
            float top = 0.f;
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const int c = b * 64 + lane * 2;
                v[b][i] = make_float2(c < rank ? v[b][i].x * scale : 0.f, c + 1 < rank ? v[b][i].y * scale : 0.f);
                top = fmaxf(top, fmaxf(fabsf(v[b][i].x), fabsf(v[b][i].y)));
            }
            float down, back;
            row_power(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))), &down, &back);
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                T hi[2], lo[2];
                split2<T>(v[b][i].x * down, &hi[0], &lo[0]);
                split2<T>(v[b][i].y * down, &hi[1], &lo[1]);
                const uint32_t at = swizzled((uint32_t)(b * kOperandBytes), r, lane >> 2) + (lane & 3) * 4;
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(low_hi + at), "r"(*reinterpret_cast<const uint32_t*>(hi)) : "memory");
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(low_lo + at), "r"(*reinterpret_cast<const uint32_t*>(lo)) : "memory");
            }
            if (lane == 0) backs[r] = back;
        }
    }

    // Read-back: this warp's 32 rows (two halves of 16) and 64 of a piece's 128 columns, 32 at a time.
    const int quarter = warp & 3, half = warp >> 2, g = lane >> 2, q = lane & 3;
    int64_t place_c[4], place_d[4];                      // rows g, g + 8 of either half
    float back[4];
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = quarter * 32 + i * 8 + g;
        there[i] = row < tile.count;
        const int64_t t = there[i] ? tokens[row] : 0;
        place_c[i] = t * a.ldc;
        place_d[i] = t * a.ldd;
    }
    uint4 in[2][4][kAccesses];                           // what is to be added, a piece ahead
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < kAccesses; ++k) in[p][i][k] = make_uint4(0, 0, 0, 0);
    auto column = [&](int64_t t, int p) { return column0(t) + half * 64 + p * 32 + q * 8; };
    auto fetch = [&](int64_t t, int p) {
        if (!C) return;
        const int64_t col = column(t, p);
        if (vec_d && col + 8 <= a.n) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there[i])
#pragma unroll
                    for (int k = 0; k < kAccesses; ++k) in[p][i][k] = reinterpret_cast<const uint4*>(C + place_c[i] + col)[k];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there[i]) {
                    DT* to = reinterpret_cast<DT*>(in[p][i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (col + j < a.n) to[j] = C[place_c[i] + col + j];
                }
        }
    };
    fetch(0, 0);
    fetch(0, 1);
    for (int64_t t = 0; t <= tiles; ++t) {
        copies_wait<0>();
        fence_async_proxy();
        tcgen05_fence_before();
        __syncthreads();                                 // B of this piece and L are there; the accumulator of the piece before the last has been read
        if (*frame.abort_flag) break;
        if (t < tiles && warp == 0) {
            tcgen05_fence_after();
            const uint32_t b = b_base + (uint32_t)(t & 1) * (KB * kOperandBytes), d = frame.tmem + (uint32_t)(t & 1) * kManyTile;
            if (elect_lane()) {
                for (int s = 0; s < ksteps; ++s) {
                    const uint32_t block = (uint32_t)(s >> 2) * kOperandBytes;
                    const uint64_t in_row = (uint64_t)((s & 3) * 2);
                    const uint64_t bdesc = make_smem_desc(b + block) + in_row;
                    umma_f16(d, make_smem_desc(low_hi + block) + in_row, bdesc, idesc, (uint32_t)(s != 0));
                    umma_f16(d, make_smem_desc(low_lo + block) + in_row, bdesc, idesc, 1u);
                }
                umma_commit(frame.bars + 8 * (uint32_t)(t & 1));
            }
            __syncwarp();
        }
        // (a wait that is given up, seconds after this barrier, is acted on by all threads behind the next one)
        const bool ok = t == 0 || frame.wait_warp((int)((t - 1) & 1), (uint32_t)((t - 1) >> 1) & 1u, kDevTimeoutEpilogue);
        // (every thread has seen the MMAs that read this buffer of B complete)
        if (ok && t + 1 < tiles) load_b(t + 1);
        copies_commit();
        if (t == 0 || !ok) continue;
        tcgen05_fence_after();
        if (t == 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) back[i] = backs[quarter * 32 + i * 8 + g];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint32_t v[2][16];
            const uint32_t at = frame.tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((t - 1) & 1) * kManyTile + half * 64 + p * 32;
            tmem_ld_16x32(at, v[0]);
            tmem_ld_16x32(at + (16u << 16), v[1]);
            tmem_ld_wait();
            const int64_t col = column(t - 1, p);
            const bool whole = vec_d && col + 8 <= a.n;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const DT* add = reinterpret_cast<const DT*>(in[p][i]);
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf(__uint_as_float(v[i >> 1][(j >> 1) * 4 + (i & 1) * 2 + (j & 1)]), back[i], to_float<DT>(add[j]));      // (the product is exact)
                if (there[i]) store8_as<DT>(D + place_d[i] + col, x, whole, a.n - col);
            }
            if (t < tiles) fetch(t, p);
        }
    }
    frame.close(kTmemCols);
}

template <typename K>
cudaError_t set_smem(K kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); }

// The largest of 16, 8, 4, 2 bytes that all rows of a 16-bit operand are aligned to.
int alignment(const void* p, int64_t ld, int64_t stride) {
    const uintptr_t all = (uintptr_t)p | (uintptr_t)(ld * 2) | (uintptr_t)(stride * 2);
    return all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : 2;
}

template <int RP, int S>
cudaError_t launch_down(const AdapterArgs& a, const AdapterLayout& l, int splits, int64_t per, int align, int* status, cudaStream_t st) {
    constexpr size_t smem = (size_t)S * (kOperandBytes + RP * kRowBytes) + 1024;
    cudaError_t err = set_smem(adapter_down_many_kernel<RP, S>, smem);
    if (err != cudaSuccess) return err;
    return launch_chained(adapter_down_many_kernel<RP, S>, dim3((unsigned)l.max_tiles, (unsigned)splits), dim3(kThreads), smem, st, a, l, per, align, make_idesc(a.type, RP), status);
}

template <typename T, typename DT, int KB>
cudaError_t launch_up(const AdapterArgs& a, const AdapterLayout& l, int splits, int* status, cudaStream_t st) {
    constexpr size_t smem = (size_t)4 * KB * kOperandBytes + 1024;
    cudaError_t err = set_smem(adapter_up_many_kernel<T, DT, KB>, smem);
    if (err != cudaSuccess) return err;
    const int vec_d = ((uintptr_t)a.D | (uintptr_t)(a.ldd * sizeof(DT))) % 16 == 0 && (!a.C || ((uintptr_t)a.C | (uintptr_t)(a.ldc * sizeof(DT))) % 16 == 0);
    // one round of blocks; those of a tile of tokens share its pieces of 128 columns evenly
    const int64_t pieces = (a.n + kManyTile - 1) / kManyTile, slots = (KB == 1 ? 2 : 1) * kSms / l.max_tiles, most = slots > 1 ? slots : 1;
    const int64_t per = (pieces + most - 1) / most, blocks = (pieces + per - 1) / per;
    return launch_chained(adapter_up_many_kernel<T, DT, KB>, dim3((unsigned)l.max_tiles, (unsigned)blocks), dim3(kThreads), smem, st, a, l, splits,
                          alignment(a.B, a.ldb, a.stride_b), vec_d, make_idesc(a.type, kManyTile), status);
}

template <typename T, int KB>
cudaError_t launch_up_typed(const AdapterArgs& a, const AdapterLayout& l, int splits, int* status, cudaStream_t st) {
    if (a.d_type == kF32) return launch_up<T, float, KB>(a, l, splits, status, st);
    if (a.d_type == kF16) return launch_up<T, __half, KB>(a, l, splits, status, st);
    return launch_up<T, __nv_bfloat16, KB>(a, l, splits, status, st);
}

}  // namespace

cudaError_t launch_adapter_many(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st, int launches[2]) {
    int* status = a.dev_status;
    const int64_t steps = (a.k + 63) / 64;
    int64_t per = (steps + l.splits - 1) / l.splits;
    if (per < 4) per = 4;                                // fewer do not fill the stages
    const int splits = (int)((steps + per - 1) / per);
    const int x_align = alignment(a.X, a.ldx, 0), a_align = alignment(a.A, a.lda, a.stride_a), align = x_align < a_align ? x_align : a_align;
    cudaError_t err = l.padded == 16   ? launch_down<16, 5>(a, l, splits, per, align, status, st)
                      : l.padded == 32 ? launch_down<32, 5>(a, l, splits, per, align, status, st)
                      : l.padded == 64 ? launch_down<64, 4>(a, l, splits, per, align, status, st)
                                       : launch_down<128, 3>(a, l, splits, per, align, status, st);
    if (err != cudaSuccess) return err;
    ++launches[0];
    if (a.type == kF16) err = l.padded <= 64 ? launch_up_typed<__half, 1>(a, l, splits, status, st) : launch_up_typed<__half, 2>(a, l, splits, status, st);
    else err = l.padded <= 64 ? launch_up_typed<__nv_bfloat16, 1>(a, l, splits, status, st) : launch_up_typed<__nv_bfloat16, 2>(a, l, splits, status, st);
    if (err == cudaSuccess) ++launches[1];
    return err;
}

}  // namespace gemm2m
