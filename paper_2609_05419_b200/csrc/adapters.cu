// Low-rank updates of many adapters beside a shared projection: D[t] = C[t] + s_a (X[t] A_a^T) B_a^T with the adapter a = index[t] of each token.
//
// Tokens of one adapter are gathered into tiles.  A first kernel forms L = X A_a^T (tile x rank) with the inner dimension cut over warps and blocks, a second
// adds the pieces up in a fixed order, multiplies by s_a, and adds L B_a^T to C.  A token's numbers depend on its own row and adapter and on
// the sizes of the call alone, not on the tokens that share its tile nor on their order.
//
// Up to 256 tokens (here) the tiles are of 16 tokens and every block finds its own from the indexes.  Both products are bound by the adapters' bytes and by the way of a block
// to its first ones, so they run as warp-level m16n8k16 MMAs whose operands go from global memory straight to registers: the order of the inner dimension is free, so a lane
// takes eight neighbouring entries of a row in one load and hands them to two MMAs, and the same lane's entries of the other operand meet them there.  The order of the columns
// of D is free too: four MMAs take columns such that a lane ends with eight neighbouring ones.  (48 tokens, 24 adapters of rank 16, 4096 to 16384 columns: 13.9 us in a graph,
// 13 MB; rank 128: 44 us, 2.9 TB/s.)  Above, one block sorts the tokens first (6 us for 8192), for tiles of 128 (adapters_many.cu).
//
// L is held in 32 bits, and goes into the second product as the sum of 16-bit numbers, after a power of two per token that keeps its largest entry well inside the range, so that
// no size of L overflows or underflows 16 bits: three for a 32-bit D, which hold all of L's bits (40 tokens, rank 16: error 1.1e-7, with two of bf16 2.5e-6; 48 tokens to
// 16384 columns 13.2 us, with two 12.8; of rank 64 22.5 and 19.5), two for a 16-bit D, whose own rounding hides what is left (2^-17 of L for bf16, 2^-22 for fp16).
#include "adapters.cuh"

#include <type_traits>

namespace gemm2m {

namespace {

constexpr int kFewWarps = 4;

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

AdapterLayout layout_of(int64_t tokens, int rank, int adapters) {
    AdapterLayout l;
    const bool few = tokens <= kFewTokens;
    const int64_t keys = adapters + 1, tile = few ? kFewTile : kManyTile;
    l.max_tiles = tokens / tile + (tokens < keys ? tokens : keys);
    // few tokens: blocks for two rounds; many: the two that an SM holds, in clusters of up to 8
    const int64_t want = l.max_tiles == 0 ? 1 : few ? (2 * kSms + l.max_tiles - 1) / l.max_tiles : 2 * kSms / l.max_tiles, most = few ? 32 : 8;
    l.splits = (int)(want > most ? most : want < 1 ? 1 : want);
    l.padded = rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128;
    l.off_perm = 0;
    l.off_tiles = up(4 * tokens, 256);
    l.off_count = l.off_tiles + up((int64_t)sizeof(AdapterTile) * l.max_tiles, 256);
    l.off_back = l.off_count + 256;
    l.off_low = l.off_back + up(4 * tokens, 256);
    l.total = l.off_low + up(2 * kParts * tokens * l.padded, 256);      // L as three 16-bit numbers
    if (few) {                                                 // nothing but the pieces of L in 32 bits
        l.off_low = 0;
        // up to splits x tokens rows of them: fewer than 32 x tokens, and than 2 kSms x 16 + tokens, since there are more than tokens / 16 tiles.  The bound, unlike what is used,
        // never falls as a size grows.
        const int64_t rows = 32 * tokens < 2 * kSms * kFewTile + tokens ? 32 * tokens : 2 * kSms * kFewTile + tokens;
        l.total = up(4 * rows * l.padded, 256);
    }
    return l;
}

__device__ __forceinline__ int key_of(const AdapterArgs& a, int64_t t) {
    const int i = a.index[t];
    return i >= 0 && i < a.adapters ? i : a.adapters;
}

// Sorts the tokens by adapter (any order among the tokens of one: nothing depends on it) and cuts them into tiles; one block.
__global__ void __launch_bounds__(1024) adapter_tiles_kernel(const AdapterArgs a, const AdapterLayout l) {
    extern __shared__ int32_t counts[];                  // [keys], then where each key's next token goes
    __shared__ int2 warps[32];
    const int keys = a.adapters + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t* perm = (int32_t*)(a.ws + l.off_perm);
    AdapterTile* tiles = (AdapterTile*)(a.ws + l.off_tiles);
    for (int i = threadIdx.x; i < keys; i += 1024) counts[i] = 0;
    __syncthreads();
    wait_for_prior_kernels();
    const int64_t rounds = (a.tokens + 1023) / 1024;
    auto take = [&](bool there, int key) {               // place of this lane's token among those of its key taken so far
        const unsigned same = __match_any_sync(0xffffffffu, key);
        const int leader = __ffs(same) - 1;
        int base = 0;
        if (lane == leader && there) base = atomicAdd(&counts[key], __popc(same));
        return __shfl_sync(0xffffffffu, base, leader) + __popc(same & ((1u << lane) - 1));
    };
    // eight rounds' indexes in flight together
    auto each = [&](auto&& f) {
        for (int64_t r0 = 0; r0 < rounds; r0 += 8) {
            int key[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t t = (r0 + i) * 1024 + threadIdx.x;
                key[i] = t < a.tokens ? key_of(a, t) : -1;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + i < rounds) f((r0 + i) * 1024 + threadIdx.x, key[i]);
        }
    };
    each([&](int64_t t, int key) { take(t < a.tokens, key); });
    __syncthreads();
    // exclusive sums over the keys of tokens and of tiles: a run of keys per thread, then over the lanes, then over the warps
    const int per = (keys + 1023) / 1024, k0 = min(keys, (int)threadIdx.x * per), k1 = min(keys, k0 + per);
    int2 mine = make_int2(0, 0);
    for (int k = k0; k < k1; ++k) mine.x += counts[k], mine.y += (counts[k] + kManyTile - 1) / kManyTile;
    auto scan = [&](int2 v) {
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, v.x, d), y = __shfl_up_sync(0xffffffffu, v.y, d);
            if (lane >= d) v.x += x, v.y += y;
        }
        return v;
    };
    const int2 sum = scan(mine);
    if (lane == 31) warps[warp] = sum;
    __syncthreads();
    const int2 over = scan(warps[lane]);
    int2 before = make_int2(sum.x - mine.x, sum.y - mine.y);
    const int bx = __shfl_sync(0xffffffffu, over.x, max(warp - 1, 0)), by = __shfl_sync(0xffffffffu, over.y, max(warp - 1, 0));
    const int total = __shfl_sync(0xffffffffu, over.y, 31);
    if (warp > 0) before.x += bx, before.y += by;
    for (int64_t i = total + threadIdx.x; i < l.max_tiles; i += 1024) tiles[i] = {a.adapters, 0, 0, 0};
    for (int k = k0; k < k1; ++k) {
        const int count = counts[k], rank = count ? rank_of(a, k) : 0;
        counts[k] = before.x;
        // the last key's tiles, of tokens without adapter, have nothing to do in place
        if (k == a.adapters) *(int32_t*)(a.ws + l.off_count) = a.C == a.D ? before.y : total;
        for (int i = 0; i < count; i += kManyTile) tiles[before.y++] = {k, before.x + i, min(kManyTile, count - i), rank};
        before.x += count;
    }
    __syncthreads();
    each([&](int64_t t, int key) {
        const int place = take(t < a.tokens, key);
        if (t < a.tokens) perm[place] = (int32_t)t;
    });
}

// Tile blockIdx.x: its key and tokens (-1 beyond its last), worked out by every block from the indexes.  Returns the number of tokens, 0 where there is
// no such tile.
__device__ __forceinline__ int find_tile(const AdapterArgs& a, int32_t* tokens, int* key) {
    constexpr int kThreads = kFewWarps * 32, kPer = kFewTokens / kThreads;
    __shared__ __align__(16) int32_t keys[kFewTokens];
    __shared__ int32_t places[kFewTokens];
    __shared__ uint32_t firsts[kFewTokens / 32];
    const int count = (int)a.tokens;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int t = i * kThreads + threadIdx.x;
        keys[t] = t < count ? key_of(a, t) : -1;
    }
    if (threadIdx.x < kFewTile) tokens[threadIdx.x] = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int t = i * kThreads + threadIdx.x;
        int place = 0;
        if (t < count) {
            const int key = keys[t];
#pragma unroll 4
            for (int u = 0; u < t >> 2; ++u) {
                const int4 four = reinterpret_cast<const int4*>(keys)[u];
                place += (four.x == key) + (four.y == key) + (four.z == key) + (four.w == key);
            }
            for (int u = t & ~3; u < t; ++u) place += keys[u] == key;
        }
        places[t] = place;
        const unsigned first = __ballot_sync(0xffffffffu, t < count && place % kFewTile == 0);
        if ((threadIdx.x & 31) == 0) firsts[t >> 5] = first;
    }
    __syncthreads();
    // tile blockIdx.x starts at the token that is the blockIdx.x-th first one of a tile
    int left = blockIdx.x, at = -1;
#pragma unroll
    for (int w = 0; w < kFewTokens / 32; ++w) {
        const int here = __popc(firsts[w]);
        if (at < 0 && left < here) at = w * 32 + __fns(firsts[w], 0, left + 1);
        left -= here;
    }
    if (at < 0) return 0;
    int members = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int t = i * kThreads + threadIdx.x;
        const bool in = t < count && keys[t] == keys[at] && places[t] / kFewTile == places[at] / kFewTile;
        if (in) tokens[places[t] % kFewTile] = t;
        members += __syncthreads_count(in);
    }
    *key = keys[at];
    return members;
}

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (sizeof(T) == 2 && !__is_same(T, __half))
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// W neighbouring entries of a row (4 or 8, in the first words of the result) from entry `at` on; those at or beyond `end` are zero.  No branches, so that loads stay in
// flight together: what is not wanted reads something that exists.  VEC: whole aligned groups that lie in the row's `stored` entries.
template <typename T, int W, bool VEC, typename I>
__device__ __forceinline__ uint4 entries(const T* row, I at, I end, I stored) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (VEC) {
        const T* p = row + (at + W <= stored ? at : 0);
        if (W == 4) {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            w[0] = v.x, w[1] = v.y;
        } else {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
        uint16_t t[W];
#pragma unroll
        for (int i = 0; i < W; ++i) t[i] = p[min(at + (I)i, stored - 1)];
#pragma unroll
        for (int i = 0; i < W; i += 2) w[i >> 1] = (uint32_t)t[i] | (uint32_t)t[i + 1] << 16;
    }
    const I left = end - at;
    const int valid = left < 0 ? 0 : left > W ? W : (int)left;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = valid >= 2 * i + 2 ? w[i] : valid == 2 * i + 1 ? w[i] & 0xffffu : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Pieces of L: block (tile, piece of k), the warps beside each other along k.
template <typename T, int RT>
__global__ void __launch_bounds__(kFewWarps * 32) adapter_down_kernel(const AdapterArgs a, const AdapterLayout l, int splits, int vec) {
    constexpr int kPadded = 16 * RT;
    extern __shared__ __align__(16) float pieces[];      // [warp][token][kPadded]
    __shared__ int32_t tokens[kFewTile];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    wait_for_prior_kernels();
    let_next_kernel_start();                             // (whatever came before has ended here: the second kernel may read all but L)
    int key;
    const int count = find_tile(a, tokens, &key);
    if (count == 0) return;
    const int rank = rank_of(a, key);
    if (rank == 0) return;
    const T* A = (const T*)a.A + key * a.stride_a;
    const T* X0 = (const T*)a.X + max(tokens[g], 0) * a.ldx;
    const T* X1 = (const T*)a.X + max(tokens[g + 8], 0) * a.ldx;
    float acc[2 * RT][4];
#pragma unroll
    for (int j = 0; j < 2 * RT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[j][c] = 0.f;
    // steps of 32 along k, dealt out to the pieces in runs and to the warps in turn
    const int64_t steps = (a.k + 31) / 32, per = (steps + splits - 1) / splits;
    const int64_t first = blockIdx.y * per, last = min(steps, first + per);
    // (What rows beyond the tile's tokens and columns beyond the rank sum up is not looked at: they read what exists.)
    auto multiply = [&](auto whole) {
        constexpr bool VEC = decltype(whole)::value;
        auto step = [&](int64_t s, auto inside) {            // inside: all 32 entries are in the rows
            constexpr bool IN = decltype(inside)::value;
            const int64_t at = s * 32 + q * 8;
            auto load = [&](const T* row) { return IN ? __ldg(reinterpret_cast<const uint4*>(row + at)) : entries<T, 8, VEC>(row, at, a.k, a.k); };
            uint4 w[2 * RT];
            const uint4 x0 = load(X0), x1 = load(X1);
#pragma unroll
            for (int j = 0; j < 2 * RT; ++j) w[j] = load(A + min(j * 8 + g, rank - 1) * a.lda);
#pragma unroll
            for (int j = 0; j < 2 * RT; ++j) {
                mma<T>(acc[j], x0.x, x1.x, x0.y, x1.y, w[j].x, w[j].y);
                mma<T>(acc[j], x0.z, x1.z, x0.w, x1.w, w[j].z, w[j].w);
            }
        };
        int64_t s = first + warp;
        if (VEC)
#pragma unroll 2
            for (; s < last && s * 32 + 32 <= a.k; s += kFewWarps) step(s, std::true_type());
        for (; s < last; s += kFewWarps) step(s, std::false_type());
    };
    if (vec) multiply(std::true_type());
    else multiply(std::false_type());
    float* mine = pieces + warp * kFewTile * kPadded;
#pragma unroll
    for (int j = 0; j < 2 * RT; ++j) {
        *reinterpret_cast<float2*>(mine + g * kPadded + j * 8 + 2 * q) = make_float2(acc[j][0], acc[j][1]);
        *reinterpret_cast<float2*>(mine + (g + 8) * kPadded + j * 8 + 2 * q) = make_float2(acc[j][2], acc[j][3]);
    }
    __syncthreads();
    float* low = (float*)(a.ws + l.off_low) + blockIdx.y * a.tokens * kPadded;
    for (int i = threadIdx.x; i < count * (kPadded / 4); i += kFewWarps * 32) {
        const int row = i / (kPadded / 4), c = i % (kPadded / 4) * 4;
        float4 sum = *reinterpret_cast<const float4*>(pieces + row * kPadded + c);
#pragma unroll
        for (int p = 1; p < kFewWarps; ++p) {
            const float4 v = *reinterpret_cast<const float4*>(pieces + (p * kFewTile + row) * kPadded + c);
            sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
        }
        *reinterpret_cast<float4*>(low + tokens[row] * (int64_t)kPadded + c) = sum;
    }
}

// Eight entries of a row of C as they are in memory, `bytes` each: loads only, and no branch that goes by the lane (vec: whole aligned groups; else entry by entry, those
// beyond the row's end reading its last), so that they can be asked for ahead.  As numbers later, by floats_of.
__device__ __forceinline__ void raw8_of(const char* row, int64_t col, int64_t n, int bytes, bool vec, uint4 (&r)[2]) {
    const int64_t at = vec ? (col < n ? col : 0) : col;
    if (bytes == 4) {
        if (vec) {
            r[0] = reinterpret_cast<const uint4*>(row + at * 4)[0];
            r[1] = reinterpret_cast<const uint4*>(row + at * 4)[1];
        } else {
            uint32_t t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = reinterpret_cast<const uint32_t*>(row)[min(at + j, n - 1)];
            r[0] = make_uint4(t[0], t[1], t[2], t[3]);
            r[1] = make_uint4(t[4], t[5], t[6], t[7]);
        }
    } else if (vec) {
        r[0] = *reinterpret_cast<const uint4*>(row + at * 2);
    } else {
        uint32_t t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = reinterpret_cast<const uint16_t*>(row)[min(at + j, n - 1)];
        r[0] = make_uint4(t[0] | t[1] << 16, t[2] | t[3] << 16, t[4] | t[5] << 16, t[6] | t[7] << 16);
    }
}
__device__ __forceinline__ void floats_of(const uint4 (&r)[2], int type, float (&v)[8]) {
    if (type == kF32) to_floats8<float>({r[0], r[1]}, v);
    else if (type == kF16) to_floats8<__half>({r[0]}, v);
    else to_floats8<__nv_bfloat16>({r[0]}, v);
}
// Eight entries as raw8_of read them back to memory, the first `valid` of them.
__device__ __forceinline__ void store8_raw(char* p, int bytes, int64_t valid, bool vec, const uint4 (&r)[2]) {
    if (vec && valid >= 8) {
        reinterpret_cast<uint4*>(p)[0] = r[0];
        if (bytes == 4) reinterpret_cast<uint4*>(p)[1] = r[1];
        return;
    }
    const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid) {
            if (bytes == 4) reinterpret_cast<uint32_t*>(p)[j] = w[j];
            else reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
}
__device__ __forceinline__ void store8_of(void* p, int type, int64_t at, int64_t valid, bool vec, const float (&v)[8]) {
    const bool whole = vec && valid >= 8;
    if (type == kF32) store8_as<float>((float*)p + at, v, whole, valid);
    else if (type == kF16) store8_as<__half>((__half*)p + at, v, whole, valid);
    else store8_as<__nv_bfloat16>((__nv_bfloat16*)p + at, v, whole, valid);
}

// Blocks of the second kernel on an SM, by its registers.
__host__ __device__ constexpr int up_blocks(int RT) { return RT == 1 ? 4 : RT == 8 ? 2 : 3; }

// D = C + L B^T: block (tile, run of columns), the warps beside each other along the columns, 32 at a time.
template <typename T, int RT, int PARTS>
__global__ void __launch_bounds__(kFewWarps * 32, up_blocks(RT)) adapter_up_kernel(const AdapterArgs a, const AdapterLayout l, int splits, int64_t run, int vec_b, int vec_d) {
    constexpr int kPadded = 16 * RT, kRow = kPadded + 4;
    extern __shared__ __align__(16) float rows[];        // [kFewTile][kRow]: L times s_a
    __shared__ int32_t tokens[kFewTile];
    __shared__ float backs[kFewTile];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    int key;
    const int count = find_tile(a, tokens, &key);
    const int rank = count > 0 ? rank_of(a, key) : 0;
    if (count == 0 || (rank == 0 && a.C == a.D)) {
        wait_for_prior_kernels();                            // (a kernel that ends lets the next one go on: no block may leave before the first kernel has ended)
        return;
    }
    // What the first 32 columns need is asked for while the first kernel is at work (1 token, rank 16: 6.0 us in all, 8.4 without that), that of the next ones before these are
    // worked on.
    const T* B = (const T*)a.B + (rank > 0 ? key : 0) * a.stride_b;
    const int64_t first = blockIdx.y * run, last = min(a.n, first + run);
    constexpr int kWords = RT == 1 ? 1 : RT / 2;         // loads of a row of B per lane
    constexpr int kStride = kFewWarps * 32;
    uint4 b_ahead[4][kWords];
    auto fetch_b = [&](int64_t n0) {
        if (rank == 0) return;
        auto fetch = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t col = n0 + 8 * (g >> 1) + 2 * j + (g & 1);
                const T* b = B + min(col, a.n - 1) * a.ldb;
#pragma unroll
                for (int s = 0; s < kWords; ++s) b_ahead[j][s] = entries<T, RT == 1 ? 4 : 8, decltype(whole)::value>(b, RT == 1 ? q * 4 : s * 32 + q * 8, rank, (int)a.rank);
            }
        };
        if (vec_b && rank == kPadded) {                      // (nothing to leave out)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const T* b = B + min(n0 + 8 * (g >> 1) + 2 * j + (g & 1), a.n - 1) * a.ldb;
                if constexpr (RT == 1) {
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(b + q * 4));
                    b_ahead[j][0] = make_uint4(v.x, v.y, 0, 0);
                } else {
#pragma unroll
                    for (int s = 0; s < kWords; ++s) b_ahead[j][s] = __ldg(reinterpret_cast<const uint4*>(b + s * 32 + q * 8));
                }
            }
        } else if (vec_b) fetch(std::true_type());
        else fetch(std::false_type());
    };
    int64_t row[2];
    bool there[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        there[i] = i * 8 + g < count;
        row[i] = there[i] ? tokens[i * 8 + g] : 0;
    }
    const int es = a.d_type == kF32 ? 4 : 2;
    uint4 c_ahead[2][2] = {};
    auto fetch_c = [&](int64_t n0) {
        if (a.C)
#pragma unroll
            for (int i = 0; i < 2; ++i) raw8_of((const char*)a.C + row[i] * a.ldc * es, n0 + 8 * q, a.n, es, vec_d && a.n % 8 == 0, c_ahead[i]);
    };
    fetch_b(first + warp * 32);
    fetch_c(first + warp * 32);
    wait_for_prior_kernels();
    if (rank > 0) {
        // a warp per row: the pieces added up, times s_a, and the power of two of its largest entry
        const float scale = a.scales ? a.scales[key] : 1.f;
        const float* sums = (const float*)(a.ws + l.off_low);
        for (int r = warp; r < kFewTile; r += kFewWarps) {
            float v[(kPadded + 31) / 32], top = 0.f;
#pragma unroll
            for (int i = 0; i < (kPadded + 31) / 32; ++i) {
                const int c = i * 32 + lane;
                v[i] = 0.f;
                if (c < rank && r < count) {
                    const float* piece = sums + tokens[r] * (int64_t)kPadded + c;
#pragma unroll 8
                    for (int p = 0; p < splits; ++p) v[i] += piece[p * a.tokens * kPadded];
                    v[i] *= scale;
                }
                top = fmaxf(top, fabsf(v[i]));
            }
            const uint32_t all = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
            float down, back;
            row_power<T>(__uint_as_float(all), &down, &back);
#pragma unroll
            for (int i = 0; i < (kPadded + 31) / 32; ++i)
                if (i * 32 + lane < kPadded) rows[r * kRow + i * 32 + lane] = v[i] * down;
            if (lane == 0) backs[r] = back;
        }
        __syncthreads();
    }
    // operand A of the MMAs: lane (g, q) holds entries 4q, 4q+1 | 4q+2, 4q+3 of every 16 (RT = 1) or 8q .. 8q+7 of every 32
    constexpr int kStep = RT == 1 ? 4 : 8;
    uint32_t low[PARTS][RT][4];
    if (rank > 0) {
#pragma unroll
        for (int s = 0; s < RT; ++s)
#pragma unroll
            for (int h = 0; h < 4; ++h) {                    // (row g + 8 (h & 1), pair h >> 1)
                const float* p = rows + (g + 8 * (h & 1)) * kRow + (RT == 1 ? 0 : (s >> 1) * 32) + q * kStep + (RT == 1 ? 0 : (s & 1) * 4) + (h >> 1) * 2;
                T x[PARTS], y[PARTS];
                split<PARTS>(p[0], x);
                split<PARTS>(p[1], y);
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    const T pair[2] = {x[i], y[i]};
                    low[i][s][h] = *reinterpret_cast<const uint32_t*>(pair);
                }
            }
    }
    float back[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) back[i] = rank > 0 ? backs[i * 8 + g] : 0.f;
    if (rank == 0) {                                         // D = C, bit for bit, or zero (a branch for this in the loop below costs all other tiles 3 %)
        constexpr int kSteps = 2;
        for (int64_t n0 = first + warp * 32; n0 < last; n0 += kSteps * kStride) {
            uint4 c[kSteps][2][2] = {};
            if (a.C)
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) raw8_of((const char*)a.C + row[i] * a.ldc * es, n0 + s * kStride + 8 * q, a.n, es, vec_d && a.n % 8 == 0, c[s][i]);
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int64_t col = n0 + s * kStride + 8 * q;
                    if (there[i] && n0 + s * kStride < last && col < a.n) store8_raw((char*)a.D + (row[i] * a.ldd + col) * es, es, a.n - col, vec_d, c[s][i]);
                }
        }
        return;
    }
    for (int64_t n0 = first + warp * 32; n0 < last; n0 += kStride) {
        float acc[4][4], v[2][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[j][c] = 0.f;
        if (rank > 0) {
            // (the last part first: every addition is cut to 32 bits, and those that come before the first part are small)
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int s = 0; s < kWords; ++s) {
                        const uint4 w = b_ahead[j][s];
                        mma<T>(acc[j], low[i][2 * s][0], low[i][2 * s][1], low[i][2 * s][2], low[i][2 * s][3], w.x, w.y);
                        if constexpr (RT > 1) mma<T>(acc[j], low[i][2 * s + 1][0], low[i][2 * s + 1][1], low[i][2 * s + 1][2], low[i][2 * s + 1][3], w.z, w.w);
                    }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            floats_of(c_ahead[i], a.d_type, v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = fmaf(acc[j >> 1][2 * i + (j & 1)], back[i], v[i][j]);      // (the product is exact)
        }
        if (n0 + kStride < last) {
            fetch_b(n0 + kStride);
            fetch_c(n0 + kStride);
        }
        const int64_t col = n0 + 8 * q;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (there[i] && col < a.n) store8_of(a.D, a.d_type, row[i] * a.ldd + col, a.n - col, vec_d, v[i]);
    }
}

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
    return bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
}

template <typename T, int RT>
cudaError_t launch_few(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st, int launches[2]) {
    auto even = [](const void* p, int64_t ld, int64_t stride, int64_t bytes) { return ((uintptr_t)p | (uintptr_t)(ld * 2) | (uintptr_t)(stride * 2)) % bytes == 0; };
    const int64_t steps = (a.k + 31) / 32, most = (steps + 2 * kFewWarps - 1) / (2 * kFewWarps);      // at least two steps for every warp
    const int splits = (int)(l.splits < most ? l.splits : most);
    const int vec = even(a.X, a.ldx, 0, 16) && even(a.A, a.lda, a.stride_a, 16) && a.k % 8 == 0;
    cudaError_t err = launch_chained(adapter_down_kernel<T, RT>, dim3((unsigned)l.max_tiles, (unsigned)splits), dim3(kFewWarps * 32), 4 * (size_t)kFewWarps * kFewTile * 16 * RT, st, a, l,
                                     splits, vec);
    if (err != cudaSuccess) return err;
    ++launches[0];
    const size_t es = a.d_type == kF32 ? 4 : 2;
    const int vec_b = even(a.B, a.ldb, a.stride_b, RT == 1 ? 8 : 16) && a.rank % (RT == 1 ? 4 : 8) == 0;
    const int vec_d = ((uintptr_t)a.D | (uintptr_t)(a.ldd * es)) % 16 == 0 && (!a.C || ((uintptr_t)a.C | (uintptr_t)(a.ldc * es)) % 16 == 0);
    // runs of columns: as many as the SMs take at once, since a block's way to its first columns is long (48 tokens to 16384 columns: 13.9 us; with half as many blocks 17, and
    // loads two steps ahead in these gain nothing), and at least two steps of 32 columns for every warp
    const int64_t groups = (a.n + 32 * kFewWarps - 1) / (32 * kFewWarps), runs = (up_blocks(RT) * kSms + l.max_tiles - 1) / l.max_tiles;
    int64_t per = (groups + runs - 1) / runs;
    if (per < 2) per = 2;
    const int64_t run = per * 32 * kFewWarps;
    const dim3 grid((unsigned)l.max_tiles, (unsigned)((a.n + run - 1) / run)), block(kFewWarps * 32);
    const size_t smem = 4 * (size_t)kFewTile * (16 * RT + 4);
    err = a.d_type == kF32 ? launch_chained(adapter_up_kernel<T, RT, 3>, grid, block, smem, st, a, l, splits, run, vec_b, vec_d)
                           : launch_chained(adapter_up_kernel<T, RT, 2>, grid, block, smem, st, a, l, splits, run, vec_b, vec_d);
    if (err == cudaSuccess) ++launches[1];
    return err;
}

template <typename T>
cudaError_t launch_typed(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st, int launches[2]) {
    if (l.padded == 16) return launch_few<T, 1>(a, l, st, launches);
    if (l.padded == 32) return launch_few<T, 2>(a, l, st, launches);
    if (l.padded == 64) return launch_few<T, 4>(a, l, st, launches);
    return launch_few<T, 8>(a, l, st, launches);
}

}  // namespace

// What the call needs, and any with fewer tokens, adapters or ranks.
int64_t adapter_bytes(int64_t tokens, int rank, int adapters) {
    const int64_t mine = layout_of(tokens, rank, adapters).total, few = tokens > kFewTokens ? layout_of(kFewTokens, rank, adapters).total : 0;
    return mine > few ? mine : few;
}

cudaError_t launch_adapter_add(const AdapterArgs& a, cudaStream_t st, int launches[2]) {
    const AdapterLayout l = layout_of(a.tokens, a.rank, a.adapters);
    if (a.tokens <= kFewTokens) return a.type == kF16 ? launch_typed<__half>(a, l, st, launches) : launch_typed<__nv_bfloat16>(a, l, st, launches);
    const size_t smem = 4 * (size_t)(a.adapters + 1);
    cudaError_t err = allow_smem(adapter_tiles_kernel, smem);
    if (err != cudaSuccess) return err;
    err = launch_chained(adapter_tiles_kernel, dim3(1), dim3(1024), smem, st, a, l);
    if (err != cudaSuccess) return err;
    ++launches[0];
    return launch_adapter_many(a, l, st, launches);
}

}  // namespace gemm2m
