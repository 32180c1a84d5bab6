// What every kernel that writes 8-bit floating point with block scales needs: scale of a block, conversion, stores of a row's end.
#pragma once
#include "layer_ops.cuh"

#include <cuda_fp8.h>

namespace gemm2m {

template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    constexpr __nv_fp8_interpretation_t kind = FMT == kE4M3 ? __NV_E4M3 : __NV_E5M2;
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, kind);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, kind);
    return lo | (hi << 16);
}

// Scale and inverse scale of a block from the bit pattern of its largest magnitude.
template <int FMT>
__device__ __forceinline__ void scales(uint32_t top, float* s, float* inv) {
    constexpr float kMax = FMT == kE4M3 ? 448.f : 57344.f;
    const float u = fmaxf(__uint_as_float(top), kLeastMax);
    const bool finite = top < 0x7f800000u;
    *s = finite ? __fdiv_rn(u, kMax) : __uint_as_float(0x7fffffffu);
    *inv = finite ? __fdiv_rn(kMax, u) : 0.f;
}

__device__ __forceinline__ void store8(uint8_t* p, uint2 v, int64_t valid) {
    if (valid >= 8) {
        *reinterpret_cast<uint2*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
    }
}

}  // namespace gemm2m
