// What the kernels of the root-mean-square norm share (rms_norm.cu, rms_norm_turned.cu, rms_norm_backward.cu).
//
// A row is held in the registers of a few warps, 8 consecutive entries in each of NV places per thread, so every operand is read once; 16 neighbouring
// threads hold a block of 128.  Sums over a row go by 256 columns: over the lanes of a warp, then, in the order of the columns, over the row's segments; so a
// row's numbers are the same whatever the number of rows, and of warps that share a row, may be.
//
// Rows that do not start on 16-byte boundaries are read and written entry by entry, neighbouring lanes taking neighbouring entries, and change hands inside the warp
// through 1 KB of shared memory (a lane reading its own 8 entries one by one touches as many sectors per instruction as there are lanes).
#pragma once
#include "fp8_pack.cuh"

#include <type_traits>

namespace gemm2m {

constexpr int kSegment = 256;             // columns that a warp holds in one place

// A warp's 256 entries: lane l holds entries 32 j + l on one side, 8 l + j on the other.
__device__ __forceinline__ void to_groups(float (&v)[8], float* turn) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) turn[32 * j + lane] = v[j];
    __syncwarp();
    const float4 a = reinterpret_cast<const float4*>(turn)[2 * lane], b = reinterpret_cast<const float4*>(turn)[2 * lane + 1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void to_lanes(float (&v)[8], float* turn) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
    reinterpret_cast<float4*>(turn)[2 * lane] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(turn)[2 * lane + 1] = make_float4(v[4], v[5], v[6], v[7]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = turn[32 * j + lane];
}

// A thread's 8 entries of one place as they come from memory: its own 8 (VEC), or entries 32 j + lane of the warp's 256.  No load sits in a branch (it would be
// waited for at the branch's end, before the next one is asked for: 59 against 45 us for 8192 x 4096 entries): what lies beyond the end of the row reads something that exists.
template <typename T, bool VEC> struct Place;
// VEC: rows are whole 16-byte pieces.  A lane's entries may be whole, half (the second half is then zero) or not there (they are then of no account; see there()).
template <typename T> struct Place<T, true> {
    Raw8<T> raw;
    // `first`: the warp's first column here
    __device__ __forceinline__ void load(const T* row, int first, int cols) {
        constexpr int kPer = 16 / (int)sizeof(T);
        const int col = first + (threadIdx.x & 31) * 8;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const bool in = col + i * kPer < cols;
            const uint4 v = __ldcs(reinterpret_cast<const uint4*>(row + (in ? col + i * kPer : 0)));
            raw.w[i] = i == 0 || in ? v : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void get(float (&v)[8], float*) const { to_floats8<T>(raw, v); }
};
template <typename T> struct Place<T, false> {
    T raw[8];
    __device__ __forceinline__ void load(const T* row, int first, int cols) {
        const int col = first + (threadIdx.x & 31);
#pragma unroll
        for (int j = 0; j < 8; ++j) raw[j] = row[min(col + 32 * j, cols - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + 32 * j >= cols) raw[j] = from_float<T>(0.f);
    }
    __device__ __forceinline__ void get(float (&v)[8], float* turn) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = to_float<T>(raw[j]);
        to_groups(v, turn);
    }
};
// `write`: whether this row is there.
template <typename T, bool VEC>
__device__ __forceinline__ void store_place(T* row, int first, int cols, bool write, const float (&v)[8], float* turn) {
    if (VEC) {
        const int col = first + (threadIdx.x & 31) * 8;
        Raw8<T> r;
        if constexpr (sizeof(T) == 2) {
            r.w[0] = make_uint4(pack_as<T>(v[0], v[1]), pack_as<T>(v[2], v[3]), pack_as<T>(v[4], v[5]), pack_as<T>(v[6], v[7]));
        } else {
            r.w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            r.w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            if (write && col + i * (16 / (int)sizeof(T)) < cols) *reinterpret_cast<uint4*>(row + col + i * (16 / (int)sizeof(T))) = r.w[i];
    } else {
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = v[j];
        to_lanes(t, turn);
        const int col = first + (threadIdx.x & 31);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (write && col + 32 * j < cols) row[col + 32 * j] = from_float<T>(t[j]);
    }
}
// This thread's weights for its NV places (entries beyond the row's end: something).
template <int NV, typename F>
__device__ __forceinline__ void load_weights(const void* W, int type, bool vec, int cols, F&& first, float (&w)[NV][8]) {
    const int lane = threadIdx.x & 31;
    auto as = [&](auto kind) {
        using T = decltype(kind);
        Raw8<T> raw[NV];
        if (vec) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
                    const int col = first(i) + lane * 8 + k * (16 / (int)sizeof(T));
                    raw[i].w[k] = __ldg(reinterpret_cast<const uint4*>((const T*)W + (col < cols ? col : 0)));
                }
        } else {
            T t[NV][8];
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) t[i][j] = ((const T*)W)[min(first(i) + lane * 8 + j, cols - 1)];
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k) raw[i].w[k] = reinterpret_cast<const uint4*>(t[i])[k];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) to_floats8<T>(raw[i], w[i]);
    };
    if (!W)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j] = 1.f;
    else if (type == kF32) as(float());
    else if (type == kF16) as(__half());
    else as(__nv_bfloat16());
}

// Over the lanes of a warp, NV numbers per lane at once: every exchange halves the numbers that a lane keeps, until it keeps one.  Returns
// that of place (lane >> 3) (four places), (lane >> 4) (two) or 0 (one), over all 32 lanes.
template <int NV, typename F>
__device__ __forceinline__ float over_warp(float (&v)[NV], F&& f) {
    int keep = NV;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        if (keep > 1) {
            keep >>= 1;
            const bool upper = (threadIdx.x & d) != 0;
#pragma unroll
            for (int i = 0; i < keep; ++i) {
                const float mine = upper ? v[i + keep] : v[i], theirs = upper ? v[i] : v[i + keep];
                v[i] = f(mine, __shfl_xor_sync(0xffffffffu, theirs, d));
            }
        } else {
            v[0] = f(v[0], __shfl_xor_sync(0xffffffffu, v[0], d));
        }
    }
    return v[0];
}

// Sums over the segments of each thread's sums of its places: a lane has that of one of them.  `segments`: one number per 256 columns of this row, in shared memory, to be read behind a barrier.
template <int NV>
__device__ __forceinline__ float segment_sums(float (&places)[NV], float* segments, int warp_in_row, int warps, int count) {
    const int lane = threadIdx.x & 31;
    const float mine = over_warp<NV>(places, [](float x, float y) { return x + y; });
    constexpr int kShift = NV == 4 ? 3 : NV == 2 ? 4 : 5;
    const int segment = (lane >> kShift) * warps + warp_in_row;
    if ((lane & ((1 << kShift) - 1)) == 0 && segment < count) segments[segment] = mine;
    return mine;
}
// Sum over a row, in the order of the columns; every thread of the block takes part.
template <int NV>
__device__ __forceinline__ float row_sum(float (&places)[NV], float* segments, int warp_in_row, int warps, int count) {
    segment_sums<NV>(places, segments, warp_in_row, warps, count);
    __syncthreads();
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < count; ++i) sum += segments[i];
    return sum;
}
// A number as the sum of two of 32 bits, the second what the first's rounding left.
struct Two { float hi, lo; };
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = a + b, part = s - a;
    return {s, (a - (s - part)) + (b - part)};
}
// The segments' sums added up as such pairs over the lanes of a warp, in every lane: of the roundings on the way to a sum of squares those of the last few additions would be left
// over, the ones before average out (8192 x 4096 bf16: error of rstd 3.0e-8, its own rounding 2.6e-8; 4.5e-8 with these additions in 32 bits.  In 32 bits 8192 x 512 takes 8.0 us, so
// 8.6, rows of 1024 columns and more as much; added up in 64 bits 8192 x 4096 takes 6.7 us more).
__device__ __forceinline__ Two over_segments(const float* segments, int count) {
    const int over = count <= 4 ? 1 : 2 << (31 - __clz((count - 1) >> 2));      // lanes that share the work, a power of two; up to four numbers each
    const int first = threadIdx.x & (over - 1);
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = first + k * over < count ? segments[first + k * over] : 0.f;
    Two sum = two_sum(x[0], x[1]);
#pragma unroll
    for (int k = 2; k < 4; ++k) {
        const Two t = two_sum(sum.hi, x[k]);
        sum = {t.hi, sum.lo + t.lo};
    }
    for (int d = over >> 1; d; d >>= 1) {
        const Two other = {__shfl_xor_sync(0xffffffffu, sum.hi, d), __shfl_xor_sync(0xffffffffu, sum.lo, d)}, t = two_sum(sum.hi, other.hi);
        sum = {t.hi, t.lo + (sum.lo + other.lo)};
    }
    return sum;
}
// 1 / sqrt(sum / cols + eps), off by little more than half a step (inv_cols: 1 / cols as a pair): the root of the leading number, brought nearer by a Newton step whose residual takes in
// what the pairs hold.
__device__ __forceinline__ float inverse_root(Two sum, Two inv_cols, float eps) {
    const float mean = __fmul_rn(sum.hi, inv_cols.hi);
    const Two m = two_sum(mean, eps);
    const float rest = m.lo + fmaf(sum.lo, inv_cols.hi, fmaf(sum.hi, inv_cols.lo, fmaf(sum.hi, inv_cols.hi, -mean)));
    const float r = rsqrtf(m.hi), t = __fmul_rn(m.hi, r);
    const float residual = fmaf(-rest * r, r, fmaf(-fmaf(m.hi, r, -t), r, fmaf(-t, r, 1.f)));
    return r > 0.f && r < INFINITY ? fmaf(0.5f * r, residual, r) : r;        // (m = 0, infinite or NaN: nothing to improve)
}

// The largest magnitude of three; NaN if there is one among them.
__device__ __forceinline__ float top3(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float top8(const float (&v)[8]) { return top3(top3(top3(v[0], v[1], v[2]), v[3], v[4]), top3(v[5], v[6], v[7]), 0.f); }

template <int FMT>
__device__ __forceinline__ uint2 to_fp8(const float (&y)[8], float inv) {
    return make_uint2(pack4<FMT>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), pack4<FMT>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
}

// Where a warp stands: `warps` warps to a row, several rows to a block; columns [begin, cols) of it.
struct Position {
    int lane, warp, row_in, warp_in_row, warps, begin, cols, segments;
    __device__ __forceinline__ Position(int warps_, int64_t cols_, int begin_ = 0)
        : lane(threadIdx.x & 31), warp(threadIdx.x >> 5), row_in(warp / warps_), warp_in_row(warp - row_in * warps_), warps(warps_), begin(begin_), cols((int)cols_),
          segments((cols - begin + kSegment - 1) / kSegment) {}
    __device__ __forceinline__ int first(int i) const { return begin + (i * warps + warp_in_row) * kSegment; }       // first column of the warp's i-th place
    // whether any of this thread's entries of its i-th place are in the row (their sums and maxima count)
    __device__ __forceinline__ bool there(int i) const { return first(i) + lane * 8 < cols; }
    __device__ __forceinline__ int rows() const { return (int)(blockDim.x / (32u * warps)); }
};

// ---- host side ----
template <typename T>
bool aligned8(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * sizeof(T)) % 16 == 0; }

// Warps that share a row with `places` segments of 256 columns each.
inline int row_warps(int64_t cols, int places) { return (int)((cols + kSegment * places - 1) / (kSegment * places)); }
// Threads of a block: rows side by side up to 256 threads.
inline int block_threads(int warps) { return warps >= 8 ? warps * 32 : 8 / warps * warps * 32; }

cudaError_t launch_rms_norm_turned(const RmsNormArgs& a, bool vec, int w_vec, cudaStream_t st);      // Qt, St from H (or X + R) and rstd

}  // namespace gemm2m
