// What the two forms of the low-rank updates share: few tokens (adapters.cu) and many (adapters_many.cu).
#pragma once
#include "layer_ops.cuh"

namespace gemm2m {

constexpr int kFewTokens = 256;           // up to here the first form, whose blocks find their tile themselves; beyond, a kernel sorts the tokens first
constexpr int kFewTile = 16, kManyTile = 128;
constexpr int kParts = 3;                 // 16-bit numbers that hold a 32-bit one

struct AdapterTile { int32_t key, start, count, rank; };     // key = adapter, or `adapters`: tokens without one; start: in the sorted list; rank in use
struct AdapterLayout {
    int64_t off_perm, off_tiles, off_count, off_back, off_low, total;      // bytes: sorted tokens, tiles, how many have something to do, powers of two of the rows of L, L
    int splits, padded;                   // pieces of k at the most, and entries of a token in L
    int64_t max_tiles;
};
cudaError_t launch_adapter_many(const AdapterArgs& a, const AdapterLayout& l, cudaStream_t st, int launches[2]);

#ifdef __CUDACC__
// The rank in use of adapter `key`.
__device__ __forceinline__ int rank_of(const AdapterArgs& a, int key) {
    if (key >= a.adapters) return 0;
    return a.ranks ? min(max(a.ranks[key], 0), a.rank) : a.rank;
}

template <typename T> __device__ __forceinline__ float largest() { return 3.3895314e38f; }
template <> __device__ __forceinline__ float largest<__half>() { return 65504.f; }

// v as the sum of 16-bit numbers, each what the ones before left: three hold all bits of a 32-bit number (8 each for bf16, 11 for fp16), two 2^-17 of it (bf16) or 2^-22 (fp16).  What is
// not finite stays in the first; what is too large (beside something that is not finite) saturates.
template <int PARTS, typename T>
__device__ __forceinline__ void split(float v, T (&part)[PARTS]) {
    const bool finite = (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
    if (finite) v = fminf(fmaxf(v, -largest<T>()), largest<T>());
    part[0] = from_float<T>(v);
#pragma unroll
    for (int p = 1; p < PARTS; ++p) {
        v = finite ? v - to_float<T>(part[p - 1]) : 0.f;
        part[p] = from_float<T>(v);
    }
}

// 2^-s for a row whose largest magnitude is in [2^e, 2^(e+1)), and 2^s; 1 where that is not finite.  fp16: s = e - 14, near the top of its range, so that entries far below the largest keep
// their bits too.  bf16, whose range is that of 32 bits: s = 0 from 2^-60 to 2^60, so that the products with B leave the range only where the results do (with the largest entry brought
// to 1, a B of 1e38 would overflow beside an L of 1e-20); beyond, s brings the largest entry back to that range.
template <typename T>
__device__ __forceinline__ void row_power(float top, float* down, float* back) {
    const int field = (int)(__float_as_uint(top) >> 23), e = field - 127;
    const int s = field == 255 ? 0 : __is_same(T, __half) ? max(e - 14, -126) : e - min(max(e, -60), 60);
    *down = __uint_as_float((uint32_t)(127 - s) << 23);
    *back = __uint_as_float((uint32_t)(127 + s) << 23);
}
#endif

}  // namespace gemm2m
