// Device helpers of kernels that multiply matrices on the fifth-generation tensor cores: barriers with a bounded wait, tiled
// asynchronous copies, and the instructions that issue products and read their accumulators.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "operator_device.cuh"

namespace ltop {

// ------------------------------------------------------------------------------------------- barriers in shared memory

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// The address of `at` in the shared memory of block `rank` of the cluster.
__device__ __forceinline__ uint32_t shared_of(uint32_t at, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
__device__ __forceinline__ void barrier_arrive_at(uint32_t cluster_bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory"); }
// (asks only; the form that waits for a while holds a warp up that has something to do: 1300 cycles a step where stages come in late)
__device__ __forceinline__ bool barrier_done(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{.reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p;}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// A warp's number, and one of its lanes, in a form that the compiler knows to be the same for the whole warp: what depends on
// them alone stays in uniform registers, which tensor and copy instructions take their operands from.
__device__ __forceinline__ uint32_t warp_number() { return __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0); }
__device__ __forceinline__ bool one_lane() {
    uint32_t r;
    asm volatile("{.reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p;}" : "=r"(r));
    return r != 0;
}

// Waits of a block that end: when one runs out of time the others give up, too.  A whole warp waits.
struct Waits {
    volatile uint32_t *gave_up;  // shared
    unsigned int *status;
    uint64_t limit_ns;

    // (the clock is slow to read: it is looked at after some tries only, which the compiler takes for one instruction)
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
        uint64_t t0 = 0;
        for (;;) {
            uint32_t done;
            asm volatile(
                "{.reg .pred p, q; .reg .u32 n; mov.u32 n, 0;\n"
                "TRY_%=: mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
                "@p bra DONE_%=;\n"
                "add.u32 n, n, 1; setp.lt.u32 q, n, 64;\n"
                "@q bra TRY_%=;\n"
                "DONE_%=: selp.u32 %0, 1, 0, p;}"
                : "=r"(done)
                : "r"(bar), "r"(parity)
                : "memory");
            if (__all_sync(0xffffffffu, done)) return true;
            const bool over = *gave_up != 0;
            if (__any_sync(0xffffffffu, over)) return false;
            const uint64_t t = now_ns();
            if (!t0) t0 = t;
            if (__any_sync(0xffffffffu, t - t0 >= limit_ns)) {
                *gave_up = 1;
                report(status);
                return false;
            }
        }
    }
};

// ------------------------------------------------------------------------------------------- tiled copies

// Brings the tile at column x, row y into shared memory at `dst`; its bytes count on the barrier `bar`, which for a pair of blocks is
// the first one's.
template <int BLOCKS>
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y) {
    if constexpr (BLOCKS == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y)
                     : "memory");
}

// ------------------------------------------------------------------------------------------- tensor cores

template <int BLOCKS>
__device__ __forceinline__ void tensor_alloc(uint32_t to, uint32_t columns) {  // one warp; the address goes to shared memory at `to`
    if constexpr (BLOCKS == 1) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    else asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    if constexpr (BLOCKS == 1) asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    else asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
template <int BLOCKS>
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {
    if constexpr (BLOCKS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// An operand in shared memory in rows of 128 bytes, swizzled over 1024: K along the rows (`turned` false: the next eight rows lie
// 1024 bytes on), or K across them (the next eight of K lie 1024 bytes on, the next 64 values of the other side `group` bytes).
__device__ __forceinline__ uint32_t operand_low(uint32_t at, bool turned, uint32_t group) { return (at & 0x3ffff) >> 4 | (turned ? group >> 4 : 1) << 16; }
constexpr uint32_t OPERAND_HIGH = 1024 >> 4 | 1u << 14 | 2u << 29;
// bf16 by bf16 into binary32, M x N
__host__ __device__ constexpr uint32_t product_kind(bool a_turned, bool b_turned, uint32_t m, uint32_t n) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a_turned << 15 | (uint32_t)b_turned << 16 | (n >> 3) << 17 | (m >> 4) << 24;
}
// The operands' lower halves vary, the upper ones do not.
template <int BLOCKS>
__device__ __forceinline__ void multiply_tiles(uint32_t to, uint32_t a_low, uint32_t b_low, uint32_t a_high, uint32_t b_high, uint32_t kind, bool add) {
    const uint32_t more = add;
    if constexpr (BLOCKS == 1)
        asm volatile(
            "{.reg .pred p; .reg .b64 a, b; setp.ne.u32 p, %6, 0; mov.b64 a, {%1, %2}; mov.b64 b, {%3, %4}; tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;}" ::"r"(to), "r"(a_low), "r"(a_high),
            "r"(b_low), "r"(b_high), "r"(kind), "r"(more)
            : "memory");
    else
        asm volatile(
            "{.reg .pred p; .reg .b64 a, b; setp.ne.u32 p, %6, 0; mov.b64 a, {%1, %2}; mov.b64 b, {%3, %4}; tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p;}" ::"r"(to), "r"(a_low), "r"(a_high),
            "r"(b_low), "r"(b_high), "r"(kind), "r"(more)
            : "memory");
}
// The barrier at `bar` (of both blocks of a pair) is arrived at when the products issued so far are done.
template <int BLOCKS>
__device__ __forceinline__ void tensor_commit(uint32_t bar) {
    if constexpr (BLOCKS == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("{.reg .b16 m; mov.b16 m, 3; tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;}" ::"r"(bar) : "memory");
}
// 32 columns of the warp's 32 rows, a row per lane
__device__ __forceinline__ void tensor_read(uint32_t at, float (&f)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, "
        "%31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
          "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]);
}

// 16 columns
__device__ __forceinline__ void tensor_read(uint32_t at, float (&f)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(r[i]);
}

}  // namespace ltop
