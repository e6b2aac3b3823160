// Device helpers of the transformer operators.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "operators.h"
#include "pdl.cuh"

namespace ltop {

// launch_pdl for a grid of two dimensions and dynamic shared memory
template <class... KArgs, class... Args>
cudaError_t launch_pdl_shared(void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t bytes, cudaStream_t stream, Args &&...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = LT_PDL;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// Lets a kernel have `bytes` of dynamic shared memory on the current device; asked once per kernel and device (`ready`).
template <class K>
__host__ cudaError_t allow_shared(K kernel, size_t bytes, std::atomic<uint64_t> &ready) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (bit && (ready.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Sets a status word, which lies in host memory: a store, since nobody writes anything else there while kernels run.
__device__ __forceinline__ void report(unsigned int *status) { *(volatile unsigned int *)status = 1u; }

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

// max(|a|, |b|, |c|), keeping a NaN
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Maximum over a warp of values that are not negative (a NaN is larger than all of them, as bits are).
__device__ __forceinline__ float warp_max_nan(float v) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu)); }

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

// Asynchronous copies of 16 bytes into shared memory
__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {  // 16 zero bytes where there is nothing
    const int bytes = there ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void copy_piece(uint32_t dst, const void *src) {  // of 8 or 16 bytes
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }


// 16 bytes of T as binary32 and back
template <class T>
struct Chunk {
    static constexpr int N = 16 / (int)sizeof(T);
};

__device__ __forceinline__ void unpack(const uint4 &v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint2 &v, float (&f)[4]) {
    const uint32_t w[2] = {v.x, v.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
// f += the values of a chunk
__device__ __forceinline__ void add_chunk(const uint4 &v, float (&f)[4]) {
    f[0] += __uint_as_float(v.x);
    f[1] += __uint_as_float(v.y);
    f[2] += __uint_as_float(v.z);
    f[3] += __uint_as_float(v.w);
}
__device__ __forceinline__ void add_chunk(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; add.f32.bf16 %0, l, %0; add.f32.bf16 %1, h, %1;}" : "+f"(f[2 * i]), "+f"(f[2 * i + 1]) : "r"(w[i]));
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// N values as the piece of memory V that holds them
template <class V, int N>
__device__ __forceinline__ V packed(const float (&f)[N]) {
    if constexpr (sizeof(V) == 8) return make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    else return pack(f);
}

// Division of 32-bit numbers by one known on the host (as fastdiv_make does for the row kernels).
struct Divisor {
    uint32_t by, mul, sh1, sh2;
    __host__ static Divisor make(uint32_t d) {
        Divisor r;
        r.by = d;
        uint32_t l = 0;
        while (l < 32 && (1ull << l) < d) ++l;
        r.mul = (uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1);
        r.sh1 = l < 1 ? l : 1;
        r.sh2 = l < 1 ? 0 : l - 1;
        return r;
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const {
        const uint32_t t = __umulhi(mul, n);
        return (t + ((n - t) >> sh1)) >> sh2;
    }
};

// The angle of `position` turns at a frequency given as a 64-bit fraction of a turn: the product modulo 2^64 is the
// fraction of a turn that is left, exactly, however far the position.  Whole quarters are taken off as integers; what
// remains, at most an eighth of a turn either way, keeps 24 bits as binary32: the angle is good to 2^-28 of a turn (converted
// with its quarters it would be to 2^-26, and the cosine off by 1.2e-7 instead of 6e-8).  Returns scale (cos, sin).
__device__ __forceinline__ float2 turn(int position, uint2 frequency, float scale, bool inverse) {
    const uint64_t f = ((uint64_t)frequency.y << 32) | frequency.x;
    const uint64_t a = (uint64_t)(int64_t)position * f;
    const uint32_t top = (uint32_t)((a + 0x80000000ull) >> 32) + 0x20000000u;  // (bits 30 and 31: how many quarters)
    float s, c;
    sincospif((float)((int32_t)(top & 0x3fffffffu) - 0x20000000) * 4.656612873077393e-10f, &s, &c);  // (2^-31: half turns)
    // (c + i s) i^quarters
    const bool odd = top & 0x40000000u;
    const float x = __uint_as_float(__float_as_uint(odd ? s : c) ^ ((top + 0x40000000u) & 0x80000000u));
    const float y = __uint_as_float(__float_as_uint(odd ? c : s) ^ (top & 0x80000000u));
    return make_float2(scale * x, inverse ? -scale * y : scale * y);
}

}  // namespace ltop
