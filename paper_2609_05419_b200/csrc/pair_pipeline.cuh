// Frame of the layer operators' tensor-core kernels on CTA pairs (tcgen05.mma.cta_group::2): barriers and TMEM, the ring of
// operand stages, and the way out when a bounded wait gives up.  A kernel fills in what a stage's copies are, which
// instructions consume it, and what happens to an accumulator.
//
// Two CTAs of a cluster share one output tile of 2 x 128 rows; each loads its 128 rows of one operand and its half of the
// other's rows, the leader issues the MMAs for both, and each CTA's TMEM ends up with its 128 rows of the accumulator.
// Barriers: the leader's full[s] collects the bytes of both CTAs' copies; commits arrive on both CTAs' empty[s] and tfull[a];
// the epilogue warps of both CTAs arrive on the leader's tempty[a].
#pragma once
#include "gemm_ptx.cuh"

namespace gemm2m {

// Arrival that publishes nothing but itself: what it orders are TMEM loads, complete before it (tcgen05.wait::ld), and MMAs issued after
// the waiting side has seen it.  (With release semantics at cluster scope every arrival waits for the warp's outstanding memory
// operations: the scales fetched ahead, the stores of the last tile.  8192^3 product with block scales: 1094 against 544 us, together
// with TMEM loads that overlap the arithmetic.)
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// One lane of a converged warp, the same every time.  The loops that issue copies and MMAs run converged and pick their lane around
// the instructions only: a loop that one lane runs alone costs 350 cycles per stage of two copies (the compiler guards every
// instruction that takes uniform operands), a converged one 190.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

// STAGES of operands, BUFFERS of accumulators.
template <int STAGES, int BUFFERS = 2>
struct PairPipe {
    uint32_t full, empty, tfull, tempty, drain;      // shared-memory addresses of the barriers
    uint32_t* tmem_slot;
    volatile int* abort_flag;
    volatile uint32_t* fills_issued;                 // by this CTA's producer, and the bytes that it loaded in the last fill of each stage
    volatile uint32_t* fill_bytes;
    uint32_t rank, peer_abort, tmem;
    int* dev_status;
    unsigned long long wait_ns;

    static constexpr size_t kBytes = 8 * (2 * STAGES + 2 * BUFFERS + 1) + 16 + 4 * STAGES;

    // All threads.  `mem`: kBytes of shared memory, 8-byte aligned; warp 1 allocates the TMEM columns.  tfull_arrivals: the commit
    // and whatever else of this CTA an accumulator waits for before its epilogue.
    __device__ __forceinline__ void open(unsigned char* mem, int epilogue_warps, int tfull_arrivals, uint32_t tmem_cols, int* status, unsigned long long limit) {
        uint64_t* bars = reinterpret_cast<uint64_t*>(mem);
        full = smem_u32(bars);
        empty = full + 8 * STAGES;
        tfull = empty + 8 * STAGES;
        tempty = tfull + 8 * BUFFERS;
        drain = tempty + 8 * BUFFERS;
        tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 2 * BUFFERS + 1);
        abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
        fills_issued = reinterpret_cast<volatile uint32_t*>(tmem_slot + 2);
        fill_bytes = reinterpret_cast<volatile uint32_t*>(tmem_slot + 3);
        rank = cluster_ctarank();
        dev_status = status;
        wait_ns = limit;
        if (threadIdx.x == 0) {
            for (int s = 0; s < STAGES; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
            for (int a = 0; a < BUFFERS; ++a) { mbar_init(tfull + 8 * a, tfull_arrivals); mbar_init(tempty + 8 * a, 2 * epilogue_warps); }
            mbar_init(drain, 1);
            *abort_flag = 0;
            *fills_issued = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (threadIdx.x >> 5 == 1) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
        tcgen05_fence_before();
        __syncthreads();
        cluster_sync_all();                              // the peer's barriers exist before anything signals them
        tcgen05_fence_after();
        tmem = *tmem_slot;
        peer_abort = map_to_cta(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u);
    }
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, int code) const { return mbar_wait(bar, parity, abort_flag, dev_status, code, wait_ns); }
    // The same for a converged warp, which stays so.
    __device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, int code) const { return __all_sync(0xffffffffu, wait(bar, parity, code)); }
    // A role that gave up tells the peer; its own CTA's flag is set by the wait (or was seen there).
    __device__ __forceinline__ void tell_peer() const { st_cluster_u32(peer_abort, 1u); }
    // Producer: `bytes` are about to be copied into this CTA's stage; the leader announces both CTAs' (they load alike).
    __device__ __forceinline__ void announce(uint32_t stage, uint32_t bytes) const {
        fill_bytes[stage] = bytes;
        if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, 2 * bytes);
    }
    // Epilogue, one warp: the accumulator buffer may be overwritten (`leader_tempty`: that buffer's barrier in the leader).
    __device__ __forceinline__ void release_at(uint32_t leader_tempty) const {
        tcgen05_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive_relaxed(leader_tempty);
    }
    // All threads, after every role has left its loop.  Neither CTA's shared memory, barriers or TMEM may go away while the peer
    // still uses them.  On the way out of a give-up, nothing may be in flight either: MMAs already issued are committed to a
    // barrier of their own and waited for.  Copies still on their way credit the leader's full[stage]; the two producers are at
    // most STAGES fills apart, so each barrier is short of, or ahead by, at most one fill: the leader takes the missing peer bytes off,
    // or announces those it had not got to, and waits for the last fill of every stage.  These waits are bounded too.
    __device__ __forceinline__ void close(uint32_t tmem_cols) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        tcgen05_fence_before();
        __syncthreads();
        cluster_sync_all();
        if (*abort_flag) {                               // both CTAs agree: a flag is set in both before this point
            if (warp == 1 && rank == 0) {
                if (elect_one()) umma_commit_pair(drain, 1);      // by the lane that issued the MMAs
                mbar_wait_quiet(drain, 0, kDrainLimitNs);
            }
            if (warp == 0 && lane == 0 && rank == 0) {
                const uint32_t mine = *fills_issued, peers = ld_cluster_u32(map_to_cta(smem_u32(const_cast<uint32_t*>(fills_issued)), 1u));
                for (uint32_t f = min(mine, peers); f < max(mine, peers); ++f) {
                    const uint32_t bar = full + 8 * (f % STAGES);
                    if (peers < mine) mbar_complete_tx(bar, fill_bytes[f % STAGES]);
                    else mbar_arrive_expect_tx(bar, ld_cluster_u32(map_to_cta(smem_u32(const_cast<uint32_t*>(fill_bytes + f % STAGES)), 1u)));
                }
                const uint32_t fills = max(mine, peers);
                for (uint32_t s = 0; s < (uint32_t)STAGES && s < fills; ++s) {
                    const uint32_t last = s + STAGES * ((fills - 1 - s) / STAGES);
                    mbar_wait_quiet(full + 8 * s, (last / STAGES) & 1u, kDrainLimitNs);
                }
            }
            __syncthreads();
            cluster_sync_all();
        }
        if (warp == 1) {
            tcgen05_fence_after();
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
        }
    }
};

// Position in the ring of stages.
template <int STAGES>
struct RingPos {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next() { if (++stage == STAGES) { stage = 0; phase ^= 1u; } }
};

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster_addr, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar_cluster_addr), "r"(x), "r"(y)
        : "memory");
}

// Packed pairs of 32-bit numbers.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
// (volatile: stays behind the wait for the TMEM load that fills its operand)
__device__ __forceinline__ void fma1(float& acc, float x, float y) { asm volatile("fma.rn.f32 %0, %1, %2, %0;" : "+f"(acc) : "f"(x), "f"(y)); }
// (a, b) times (y, y), as bit patterns in.
__device__ __forceinline__ void mul_pair(uint32_t a, uint32_t b, uint64_t y, float* x0, float* x1) {
    asm volatile("{\n\t.reg .b64 t;\n\tmov.b64 t, {%2, %3};\n\tmul.rn.f32x2 t, t, %4;\n\tmov.b64 {%0, %1}, t;\n\t}" : "=f"(*x0), "=f"(*x1) : "r"(a), "r"(b), "l"(y));
}

// Most CTA pairs that are resident at once.
template <typename K>
inline cudaError_t resident_pairs(K kernel, int threads, size_t smem, int sm_count, int* pairs) {
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t qc = {};
    qc.gridDim = dim3((unsigned)(sm_count & ~1), 1, 1);
    qc.blockDim = dim3(threads, 1, 1);
    qc.dynamicSmemBytes = smem;
    cudaLaunchAttribute qa[1];
    qa[0].id = cudaLaunchAttributeClusterDimension;
    qa[0].val.clusterDim.x = 2;
    qa[0].val.clusterDim.y = 1;
    qa[0].val.clusterDim.z = 1;
    qc.attrs = qa;
    qc.numAttrs = 1;
    int clusters = 0;
    err = cudaOccupancyMaxActiveClusters(&clusters, kernel, &qc);
    if (err != cudaSuccess) return err;
    *pairs = clusters > 0 && clusters < sm_count / 2 ? clusters : sm_count / 2;
    return cudaSuccess;
}

}  // namespace gemm2m
