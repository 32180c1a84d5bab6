// Low-rank updates of many adapters, many tokens: tiles of 128 tokens of one adapter on the tensor cores (tcgen05, one CTA per tile).
//
// L = X A_a^T: a cluster takes a tile, each of its blocks a piece of k, in steps of 64 entries (one 128-byte swizzle row): four MMAs of 128 x rank x 16 per step.  The tile's
// rows of X lie anywhere, so they come by asynchronous 16-byte copies (8- and 4-byte ones where rows start there), three or four steps ahead.  The blocks then add their
// pieces up through one another's shared memory, each for a part of the rows, in the order of k.
// D = C + L B_a^T: all tiles' pieces of 128 columns are cut into even runs, one per block, which goes through the (at most few) tiles of its run.  L, as two or three 16-bit numbers, stays in shared memory; the MMAs of one piece run while the one before is
// read back, added to what was fetched of C a piece earlier, and stored.  The read-back hands a lane pairs of columns 8 apart; the rows of B
// lie in shared memory in such an order that these are eight neighbouring columns of D.
// Both are bound by memory and the hand-overs between copies, MMAs and read-back (8192 tokens, 8192 to 8192 columns, 8 adapters of rank 64, bf16: 31 us, X at 4.4 TB/s, and
// 58 us, C and D at 4.6 TB/s).
#include "adapters.cuh"
#include "gemm_ptx.cuh"

#include <type_traits>

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

__device__ __forceinline__ float2 ld_cluster_f32x2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// T: type of X, A and of L's two parts; RP: padded rank, S: stages; ALIGN: bytes that rows are aligned to, 16 or 0: to be seen at run time.
template <typename T, int RP, int S, int ALIGN>
__global__ void __launch_bounds__(kThreads, 2) adapter_down_many_kernel(const AdapterArgs a, const AdapterLayout l, int splits, int64_t per, int run_align, uint32_t idesc) {
    constexpr int kStageBytes = kOperandBytes + RP * kRowBytes, kTmemCols = 256, kAccs = kTmemCols / RP, kPitch = RP * 4 + 16;
    static_assert(kManyTile * kPitch <= S * kStageBytes, "a piece of L takes the place of the stages");
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint64_t bars[S + 2];
    const int align = ALIGN ? ALIGN : run_align;
    const int part = blockIdx.x % (unsigned)splits;          // (also the block's rank in its cluster)
    wait_for_prior_kernels();
    const AdapterTile tile = ((const AdapterTile*)(a.ws + l.off_tiles))[blockIdx.x / (unsigned)splits];
    if (tile.rank == 0) return;                              // no such tile, or nothing to multiply: the same in all of the cluster
    const int32_t* tokens = (const int32_t*)(a.ws + l.off_perm) + tile.start;
    Frame<S> frame;
    frame.open(bars, kTmemCols, a.dev_status);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // this thread copies piece `piece` of rows row0, row0 + 32, ...
    const int piece = threadIdx.x & 7, row0 = threadIdx.x >> 3;
    const uint16_t* x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (const uint16_t*)a.X + (row0 + 32 * j < tile.count ? tokens[row0 + 32 * j] : 0) * a.ldx;
    const uint16_t* A = (const uint16_t*)a.A + tile.key * a.stride_a + row0 * a.lda;
    const int64_t total = (a.k + 63) / 64, first = part * per;
    const int steps = (int)(min(total, first + per) - first);
    auto load = [&](int step, int slot) {
        const uint32_t stage = base + (uint32_t)slot * kStageBytes;
        const int64_t at = (first + step) * 64 + piece * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (row0 + 32 * j < tile.count) copy8(swizzled(stage, row0 + 32 * j, piece), x[j], at, a.k, align);
#pragma unroll
        for (int j = 0; j < (RP + 31) / 32; ++j)
            if (row0 + 32 * j < tile.rank) copy8(swizzled(stage + kOperandBytes, row0 + 32 * j, piece), A + 32 * j * a.lda, at, a.k, align);
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
        if (i < steps) load(i, i);
        copies_commit();
    }
    // The tensor cores cut what they add to an accumulator, by up to 2^-23 of it and always towards zero, so the run of steps is shared by as many accumulators as there is room for, from 512
    // entries of k each on, which are added up with rounding (8192 tokens, k = 8192: error of L 4.8e-7, in one accumulator 2.1e-6; where all products are positive
    // 8.9e-7 and 5.6e-6; 0.4 of 100 us).
    const int per_acc = max(8, (steps + kAccs - 1) / kAccs);
    int acc = 0, in_acc = 0;                                 // this step's accumulator, and how many steps that has
    int slot = 0, last_slot = S - 1;                         // of this step, and of the one before, which is filled next
    uint32_t phase = 0, last_phase = 1;
    for (int i = 0; i < steps; ++i) {
        copies_wait<S - 2>();
        fence_async_proxy();
        // the stage that is filled next was read by the MMAs of the step before
        if (warp == 0 && i > 0) frame.wait_warp(last_slot, last_phase, kDevTimeoutProducer);
        __syncthreads();
        if (*frame.abort_flag) break;
        if (warp == 0) {
            tcgen05_fence_after();
            const uint32_t stage = base + (uint32_t)slot * kStageBytes;
            const uint64_t adesc = make_smem_desc(stage), bdesc = make_smem_desc(stage + kOperandBytes);
            if (elect_lane()) {
#pragma unroll
                for (int s = 0; s < 4; ++s) umma_f16(frame.tmem + acc * RP, adesc + (uint64_t)(s * 2), bdesc + (uint64_t)(s * 2), idesc, (uint32_t)((in_acc | s) != 0));
                umma_commit(frame.bars + 8 * (uint32_t)slot);
            }
            __syncwarp();
        }
        if (i + S - 1 < steps) load(i + S - 1, last_slot);
        copies_commit();
        last_slot = slot;
        last_phase = phase;
        if (++slot == S) slot = 0, phase ^= 1u;
        if (++in_acc == per_acc) in_acc = 0, ++acc;
    }
    const int accs = acc + (in_acc > 0);
    // (not the abort flag: a wait that is given up fails at once here too)
    if (frame.wait_warp(last_slot, last_phase, kDevTimeoutEpilogue)) {
        tcgen05_fence_after();
        // this block's piece of L takes the place of the stages
        const uint32_t row = base + (uint32_t)((warp & 3) * 32 + lane) * kPitch;
        for (int c = (warp >> 2) * 16; c < RP; c += 32) {
            float v[16];
            for (int k = 0; k < accs; ++k) {
                uint32_t part[16];
                tmem_ld16(frame.tmem + ((uint32_t)((warp & 3) * 32) << 16) + k * RP + c, part);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = k ? v[j] + __uint_as_float(part[j]) : __uint_as_float(part[j]);
            }
#pragma unroll
            for (int j = 0; j < 16; j += 4)
                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(row + (c + j) * 4), "f"(v[j]), "f"(v[j + 1]), "f"(v[j + 2]), "f"(v[j + 3]) : "memory");
        }
    }
    frame.close(kTmemCols);
    cluster_sync_all();
    // a warp per row: the pieces added up, times s_a, the largest entry brought well inside the range, as three 16-bit numbers
    const float scale = a.scales ? a.scales[tile.key] : 1.f;
    T* low = (T*)(a.ws + l.off_low) + (int64_t)tile.start * (kParts * RP);
    float* backs = (float*)(a.ws + l.off_back) + tile.start;
    for (int r = part * (kThreads / 32) + warp; r < tile.count; r += splits * (kThreads / 32)) {
        constexpr int kPairs = (RP + 63) / 64;
        float2 v[kPairs];
        float top = 0.f;
#pragma unroll
        for (int b = 0; b < kPairs; ++b) {
            const int c = b * 64 + lane * 2;
            float2 w[8];
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (p < splits && c < RP) w[p] = ld_cluster_f32x2(map_to_cta(base + (uint32_t)r * kPitch + c * 4, (uint32_t)p));
            v[b] = make_float2(0.f, 0.f);
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (p < splits && c < RP) v[b].x += w[p].x, v[b].y += w[p].y;
            v[b] = make_float2(c < tile.rank ? v[b].x * scale : 0.f, c + 1 < tile.rank ? v[b].y * scale : 0.f);
            top = fmaxf(top, fmaxf(fabsf(v[b].x), fabsf(v[b].y)));
        }
        float down, back;
        row_power<T>(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))), &down, &back);
#pragma unroll
        for (int b = 0; b < kPairs; ++b) {
            const int c = b * 64 + lane * 2;
            T x[kParts], y[kParts];
            split<kParts>(v[b].x * down, x);
            split<kParts>(v[b].y * down, y);
            if (c < RP)
#pragma unroll
                for (int i = 0; i < kParts; ++i) {
                    const T pair[2] = {x[i], y[i]};
                    *reinterpret_cast<uint32_t*>(low + (r * kParts + i) * RP + c) = *reinterpret_cast<const uint32_t*>(pair);
                }
        }
        if (lane == 0) backs[r] = back;
    }
    cluster_sync_all();                                      // nobody's piece goes away while another block reads it
}

// DT: type of C and D; KB: blocks of 64 along the rank.  (The operands' 16-bit type is the instruction descriptor's matter.)  VEC: rows of C and D are whole 16-byte pieces;
// otherwise a warp turns each 16 rows x 32 columns in shared memory and reads and writes row by row, a lane per column (a lane's own eight columns, entry by
// entry, would be as many sectors per instruction as there are lanes: 1001 tokens, 1999 columns: 38 us in all, 29 so).
constexpr int up_blocks(int KB) { return KB == 1 ? 2 : 1; }       // on an SM
// Parts of L that the product takes: a 16-bit D's rounding hides the third.
template <typename DT> __host__ __device__ constexpr int parts_of() { return sizeof(DT) == 4 ? kParts : 2; }
constexpr int kTurnRows = 16, kTurnPitch = 36, kTurnBytes = kTurnRows * kTurnPitch * 4;      // of a warp: half of its rows at a time
template <typename DT, int KB, int ALIGN, bool VEC>
__global__ void __launch_bounds__(kThreads, up_blocks(KB)) adapter_up_many_kernel(const AdapterArgs a, const AdapterLayout l, int run_align, uint32_t idesc) {
    constexpr int PARTS = parts_of<DT>();
    constexpr int kTmemCols = 256, E = 16 / (int)sizeof(DT), kAccesses = 8 / E;      // eight columns of a row per lane, E in one access
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint64_t bars[4];
    const int align = ALIGN ? ALIGN : run_align;
    wait_for_prior_kernels();
    const int64_t pieces = (a.n + kManyTile - 1) / kManyTile, all = *(const int32_t*)(a.ws + l.off_count) * pieces;
    int64_t at = all * blockIdx.x / gridDim.x;
    const int64_t end = all * (blockIdx.x + 1) / gridDim.x;
    if (at == end) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const DT* C = (const DT*)a.C;
    DT* D = (DT*)a.D;
    Frame<2> frame;
    frame.open(bars, kTmemCols, a.dev_status);
    const uint32_t low_base = (smem_u32(smem_raw) + 1023u) & ~1023u, b_base = low_base + PARTS * KB * kOperandBytes;
    // this thread copies piece `piece` (and `piece` + 8) of rows, or columns, c0, c0 + 32, ... of 128; columns 8q + 2j + e of every 32 are rows 8j + 2q + e of B's tile
    const int piece = threadIdx.x & 7, c0 = threadIdx.x >> 3;
    const uint32_t b_dst = swizzled(b_base, (c0 & 6) << 2 | (c0 & 24) >> 2 | (c0 & 1), piece);
    const int quarter = warp & 3, half = warp >> 2, g = lane >> 2, q = lane & 3;
    float* turn = reinterpret_cast<float*>(smem_raw + (low_base - smem_u32(smem_raw)) + (PARTS + 2) * KB * kOperandBytes + warp * kTurnBytes);      // (not VEC)

    uint32_t it = 0;                                     // pieces so far: buffer it % 2, its use number it / 2
    bool ok = true;
    while (ok && at < end) {
        const AdapterTile tile = ((const AdapterTile*)(a.ws + l.off_tiles))[at / pieces];
        const int32_t* tokens = (const int32_t*)(a.ws + l.off_perm) + tile.start;
        const int64_t piece0 = at % pieces;
        const int here = (int)min(pieces - piece0, end - at);
        at += here;
        auto column0 = [&](int t) { return (piece0 + t) * kManyTile; };
        if (tile.rank == 0) {                            // D = C, or zero
            if (a.C == a.D) continue;
            // eight pieces of a row, or entries, in flight per thread (1001 tokens, a sixth without adapter, 1999 columns: 25.4 us in all, 28.9
            // with one at a time)
            using Unit = std::conditional_t<VEC, uint4, DT>;
            constexpr int kPer = VEC ? kManyTile / E : kManyTile, kBatch = 8;
            for (int t = 0; t < here; ++t) {
                const int64_t col = column0(t) + threadIdx.x % kPer * (VEC ? E : 1), from = min(col, a.n - (VEC ? E : 1));
                for (int r0 = threadIdx.x / kPer; r0 < tile.count; r0 += kBatch * (kThreads / kPer)) {
                    int64_t row[kBatch];
                    Unit v[kBatch];
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) row[u] = tokens[min(r0 + u * (kThreads / kPer), tile.count - 1)];
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) v[u] = C ? *reinterpret_cast<const Unit*>(C + row[u] * a.ldc + from) : Unit();
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        if (r0 + u * (kThreads / kPer) < tile.count && col < a.n) *reinterpret_cast<Unit*>(D + row[u] * a.ldd + col) = v[u];
                }
            }
            continue;
        }
        const int ksteps = (tile.rank + 15) / 16, width = 2 * ksteps;         // 16-byte pieces of a row that the MMAs read
        const uint16_t* b_row = (const uint16_t*)a.B + tile.key * a.stride_b + c0 * a.ldb;
        auto load_b = [&](int t) {
            const uint32_t dst = b_dst + ((it + t) & 1) * (KB * kOperandBytes);
            const int64_t col = column0(t);
            const uint16_t* row = b_row + col * a.ldb;
#pragma unroll
            for (int k = 0; k < kManyTile / 32; ++k, row += 32 * a.ldb) {
                if (col + c0 + 32 * k >= a.n) break;
#pragma unroll
                for (int b = 0; b < KB; ++b)
                    if (b * 8 + piece < width) copy8(dst + b * kOperandBytes + k * 32 * kRowBytes, row, (b * 8 + piece) * 8, tile.rank, align);
            }
        };
        // (the MMAs that read the last tile's L and B have been waited for by every thread, and all of them have passed its last barrier since)
        load_b(0);
        {
            const uint16_t* low = (const uint16_t*)(a.ws + l.off_low) + (int64_t)tile.start * (kParts * l.padded);
#pragma unroll
            for (int k = 0; k < kManyTile / 32; ++k) {
                const int r = c0 + 32 * k;
                if (r < tile.count)
#pragma unroll
                    for (int b = 0; b < KB; ++b)
                        if (b * 8 + piece < width) {
                            const uint32_t dst = swizzled(low_base + b * kOperandBytes, r, piece);
#pragma unroll
                            for (int i = 0; i < PARTS; ++i) copy8(dst + i * KB * kOperandBytes, low + (r * kParts + i) * l.padded, (b * 8 + piece) * 8, l.padded, 16);
                        }
            }
        }
        copies_commit();

        // Read-back: this warp's 32 rows (rows g, g + 8 of two halves of 16) and 64 of a piece's 128 columns, 32 at a time.
        float back[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = quarter * 32 + i * 8 + g;
            back[i] = row < tile.count ? ((const float*)(a.ws + l.off_back))[tile.start + row] : 0.f;
        }
        // VEC: rows 8i + g, eight columns; otherwise row `lane`, for all lanes
        int64_t place_c[VEC ? 4 : 1], place_d[VEC ? 4 : 1];
        bool there[VEC ? 4 : 1];
#pragma unroll
        for (int i = 0; i < (VEC ? 4 : 1); ++i) {
            const int row = quarter * 32 + (VEC ? i * 8 + g : lane);
            there[i] = row < tile.count;
            const int64_t t = there[i] ? tokens[row] : 0;
            place_c[i] = t * a.ldc;
            place_d[i] = t * a.ldd;
        }
        const int rows_here = min(32, tile.count - quarter * 32);
        auto column = [&](int t, int p) { return column0(t) + half * 64 + p * 32 + (VEC ? q * 8 : lane); };
        // What is to be added, a piece ahead.  (No branch that goes by the lane: what lies beyond the row's end, or the tile's, reads something that exists.)
        uint4 in[2][VEC ? 4 : 1][kAccesses];
        DT in_rows[VEC ? 1 : 32];                            // (one piece of 32 columns)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int i = 0; i < (VEC ? 4 : 1); ++i)
#pragma unroll
                for (int k = 0; k < kAccesses; ++k) in[p][i][k] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < (VEC ? 1 : 32); ++i) in_rows[i] = from_float<DT>(0.f);
        auto fetch = [&](int t, int p) {
            if (!C) return;
            const int64_t col = column(t, p);
            if constexpr (VEC) {
                const int64_t at = col < a.n ? col : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < kAccesses; ++k) in[p][i][k] = reinterpret_cast<const uint4*>(C + place_c[i] + at)[k * E < a.n - at ? k : 0];
            } else {
                const DT* C_col = C + min(col, a.n - 1);
#pragma unroll
                for (int r = 0; r < 32; ++r) in_rows[r] = C_col[__shfl_sync(0xffffffffu, place_c[0], r)];
            }
        };
        fetch(0, 0);
        if (VEC) fetch(0, 1);
        for (int t = 0; t <= here; ++t) {
            copies_wait<0>();
            fence_async_proxy();
            tcgen05_fence_before();
            __syncthreads();                             // B of this piece and L are there; the accumulator of the piece before the last has been read
            if (*frame.abort_flag) { ok = false; break; }
            const uint32_t buf = (it + t) & 1;
            if (t < here && warp == 0) {
                tcgen05_fence_after();
                const uint32_t b = b_base + buf * (KB * kOperandBytes), d = frame.tmem + buf * kManyTile;
                if (elect_lane()) {
                    // (the last part first: every addition is cut to 32 bits, and those that come before the first part are small)
#pragma unroll
                    for (int i = PARTS - 1; i >= 0; --i)
                        for (int s = 0; s < ksteps; ++s) {
                            const uint32_t block = (uint32_t)(s >> 2) * kOperandBytes;
                            const uint64_t in_row = (uint64_t)((s & 3) * 2);
                            umma_f16(d, make_smem_desc(low_base + i * KB * kOperandBytes + block) + in_row, make_smem_desc(b + block) + in_row, idesc,
                                     (uint32_t)(s != 0 || i != PARTS - 1));
                        }
                    umma_commit(frame.bars + 8 * buf);
                }
                __syncwarp();
            }
            // (a wait that is given up, seconds after this barrier, is acted on by all threads behind the next one)
            const bool done = t == 0 || frame.wait_warp((int)(buf ^ 1), ((it + t - 1) >> 1) & 1u, kDevTimeoutEpilogue);
            // (every thread has seen the MMAs that read this buffer of B complete)
            if (done && t + 1 < here) load_b(t + 1);
            copies_commit();
            if (t == 0 || !done) continue;
            tcgen05_fence_after();
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                uint32_t v[2][16];
                const uint32_t from = frame.tmem + ((uint32_t)(quarter * 32) << 16) + (buf ^ 1) * kManyTile + half * 64 + p * 32;
                tmem_ld_16x32(from, v[0]);
                tmem_ld_16x32(from + (16u << 16), v[1]);
                tmem_ld_wait();
                const int64_t col = column(t - 1, p);
                if constexpr (VEC) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        Raw8<DT> raw;
#pragma unroll
                        for (int k = 0; k < kAccesses; ++k) raw.w[k] = in[p][i][k];
                        float add[8], x[8];
                        to_floats8<DT>(raw, add);
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] = fmaf(__uint_as_float(v[i >> 1][(j >> 1) * 4 + (i & 1) * 2 + (j & 1)]), back[i], add[j]);      // (the product is exact)
                        // (rows of E entries and multiples: a lane's eight columns are there as a whole, or their first half, or not at all)
                        if (there[i] && col + 8 <= a.n) store8_as<DT>(D + place_d[i] + col, x, true, 8);
                        else if (there[i]) store8_as<DT>(D + place_d[i] + col, x, false, a.n - col);
                    }
                } else {
                    DT* D_col = D + col;
                    const int rows_stored = col < a.n ? rows_here : 0;
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += kTurnRows) {
                        __syncwarp();                        // the rows and columns before have been read
#pragma unroll
                        for (int i = r0 / 8; i < (r0 + kTurnRows) / 8; ++i) {
                            float x[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v[i >> 1][(j >> 1) * 4 + (i & 1) * 2 + (j & 1)]) * back[i];
                            float4* to = reinterpret_cast<float4*>(turn + (i * 8 + g - r0) * kTurnPitch + q * 8);
                            to[0] = make_float4(x[0], x[1], x[2], x[3]);
                            to[1] = make_float4(x[4], x[5], x[6], x[7]);
                        }
                        __syncwarp();
#pragma unroll
                        for (int r = r0; r < r0 + kTurnRows; ++r) {
                            const DT out = from_float<DT>(to_float<DT>(in_rows[r]) + turn[(r - r0) * kTurnPitch + lane]);
                            DT* place = D_col + __shfl_sync(0xffffffffu, place_d[0], r);
                            if (r < rows_stored) *place = out;
                        }
                    }
                }
                if (VEC ? t < here : t < here || p == 0) fetch(VEC || p == 1 ? t : t - 1, VEC ? p : p ^ 1);
            }
        }
        it += here;
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

template <typename T, int RP, int S, int ALIGN>
cudaError_t launch_down_as(const AdapterArgs& a, const AdapterLayout& l, int splits, int64_t per, int align, cudaStream_t st) {
    constexpr size_t smem = (size_t)S * (kOperandBytes + RP * kRowBytes) + 1024;
    cudaError_t err = set_smem(adapter_down_many_kernel<T, RP, S, ALIGN>, smem);
    if (err != cudaSuccess) return err;
    return launch_chained_cluster(adapter_down_many_kernel<T, RP, S, ALIGN>, dim3((unsigned)(l.max_tiles * splits)), dim3(kThreads), smem, splits, st, a, l, splits, per, align,
                                  make_idesc(a.type, RP));
}

template <typename T>
cudaError_t launch_down(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st) {
    const int64_t steps = (a.k + 63) / 64;
    int64_t per = (steps + l.splits - 1) / l.splits;
    if (per < 4) per = 4;                                // fewer do not fill the stages
    const int splits = (int)((steps + per - 1) / per);
    const int x_align = alignment(a.X, a.ldx, 0), a_align = alignment(a.A, a.lda, a.stride_a), align = x_align < a_align ? x_align : a_align;
    auto with = [&](auto rp, auto s) {
        constexpr int RP = decltype(rp)::value, S = decltype(s)::value;
        return align == 16 ? launch_down_as<T, RP, S, 16>(a, l, splits, per, align, st) : launch_down_as<T, RP, S, 0>(a, l, splits, per, align, st);
    };
    using std::integral_constant;
    if (l.padded == 16) return with(integral_constant<int, 16>(), integral_constant<int, 5>());
    if (l.padded == 32) return with(integral_constant<int, 32>(), integral_constant<int, 5>());
    if (l.padded == 64) return with(integral_constant<int, 64>(), integral_constant<int, 4>());
    return with(integral_constant<int, 128>(), integral_constant<int, 3>());
}

template <typename DT, int KB, int ALIGN, bool VEC>
cudaError_t launch_up_as(const AdapterArgs& a, const AdapterLayout& l, int align, cudaStream_t st) {
    constexpr size_t smem = (size_t)(parts_of<DT>() + 2) * KB * kOperandBytes + (VEC ? 0 : kThreads / 32 * kTurnBytes) + 1024;
    static_assert(up_blocks(KB) * (smem + 1024) <= 228 * 1024, "the blocks that the grid counts on fit an SM");
    cudaError_t err = set_smem(adapter_up_many_kernel<DT, KB, ALIGN, VEC>, smem);
    if (err != cudaSuccess) return err;
    // as many blocks as the GPU holds, or one for every piece that there can be
    const int64_t pieces = l.max_tiles * ((a.n + kManyTile - 1) / kManyTile), slots = up_blocks(KB) * kSms;
    return launch_chained(adapter_up_many_kernel<DT, KB, ALIGN, VEC>, dim3((unsigned)(pieces < slots ? pieces : slots)), dim3(kThreads), smem, st, a, l, align,
                          make_idesc(a.type, kManyTile));
}

template <typename DT, int KB>
cudaError_t launch_up_shape(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st) {
    const int align = alignment(a.B, a.ldb, a.stride_b);
    const bool vec = ((uintptr_t)a.D | (uintptr_t)(a.ldd * sizeof(DT)) | (uintptr_t)(a.n * sizeof(DT))) % 16 == 0 && (!a.C || ((uintptr_t)a.C | (uintptr_t)(a.ldc * sizeof(DT))) % 16 == 0);
    if (!vec) return launch_up_as<DT, KB, 0, false>(a, l, align, st);
    return align == 16 ? launch_up_as<DT, KB, 16, true>(a, l, align, st) : launch_up_as<DT, KB, 0, true>(a, l, align, st);
}

template <typename DT>
cudaError_t launch_up(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st) {
    return l.padded <= 64 ? launch_up_shape<DT, 1>(a, l, st) : launch_up_shape<DT, 2>(a, l, st);
}

}  // namespace

cudaError_t launch_adapter_many(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st, int launches[2]) {
    cudaError_t err = a.type == kF16 ? launch_down<__half>(a, l, st) : launch_down<__nv_bfloat16>(a, l, st);
    if (err != cudaSuccess) return err;
    ++launches[0];
    err = a.d_type == kF32 ? launch_up<float>(a, l, st) : a.d_type == kF16 ? launch_up<__half>(a, l, st) : launch_up<__nv_bfloat16>(a, l, st);
    if (err == cudaSuccess) ++launches[1];
    return err;
}

}  // namespace gemm2m
