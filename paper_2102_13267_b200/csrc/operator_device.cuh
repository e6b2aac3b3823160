// Device helpers of the transformer operators.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "operators.h"
#include "pdl.cuh"

namespace ltop {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Over a block of whole warps; `part` has room for 32 values.  Every thread gets the result, the same for all.
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float *part) {
    v = MAX ? warp_max_nan(v) : warp_sum(v);
    const int warps = (int)blockDim.x >> 5;
    if (warps == 1) return v;
    __syncthreads();  // `part` may still be read from the reduction before
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = part[0];
    for (int w = 1; w < warps; ++w) r = MAX ? max_nan(r, part[w]) : r + part[w];
    return r;
}

// The angle of `position` turns at a frequency given as a 64-bit fraction of a turn: the product modulo 2^64 is the
// fraction of a turn that is left, exactly, however far the position; its upper 32 bits (rounded) are the angle to
// 2^-33 of a turn.  Returns scale (cos, sin).
__device__ __forceinline__ float2 turn(int position, uint2 frequency, float scale, bool inverse) {
    const uint64_t f = ((uint64_t)frequency.y << 32) | frequency.x;
    const uint64_t a = (uint64_t)(int64_t)position * f;
    const int32_t top = (int32_t)((a + 0x80000000ull) >> 32);
    float s, c;
    sincospif((float)top * 4.656612873077393e-10f, &s, &c);  // (2^-31: half turns)
    if (inverse) s = -s;
    return make_float2(scale * c, scale * s);
}

}  // namespace ltop
