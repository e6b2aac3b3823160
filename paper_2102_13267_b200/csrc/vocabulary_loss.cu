// The cross entropy of hidden states against a table of rows, and its gradient, without keeping the scores.
//
// z = scale x table^T [tokens, vocabulary]; lse_n = log sum_v exp z_nv; loss_n = lse_n - z[n, target_n].
// P = exp(z - lse_n) - [v = target_n], 0 for tokens without a target; dx = scale dloss_n P table; dtable = P^T (scale dloss_n x).
//
// Three matrix products, one kernel (lt_product) that differs in how its operands lie and in what it does with a tile of the
// result.  Scores never reach memory: the loss keeps of each tile the rows' maxima and sums of exponentials, which
// lt_loss_join adds up in the tiles' order.  The gradient makes P for a piece of the vocabulary at a time, in bf16, and
// multiplies it from both sides.
//
// Few tokens are scored, and their gradients made, by plain loads and products in binary32 (lt_loss_few, lt_loss_some, lt_loss_few_grad).
//
// Types.  bf16 operands are multiplied as they are, with binary32 sums; P is rounded to bf16 (2^-8 of each value at most, as much as storing
// the gradients costs; P is near -1 at most targets and rounded little there, which it would not be with dloss in it).  So is x dloss_n where dloss
// differs from token to token: it is divided by the largest |dloss| and dtable multiplied by it, and stays x where they are all alike.
// Gradients are 2.0e-3 off as a whole for that (257 x 512 against 5003 rows), the table's 2.6e-3 where every dloss is another; storing exact
// ones costs 1.65e-3.
// f32 operands, and P then, are taken as three bf16 parts each (24 bits, exactly, of values above 2^-110; below, the last part is
// subnormal), and of the nine products of parts the six largest are added: what is left out is below 2^-23 of each product.
#include <algorithm>

#include "tensor_device.cuh"

using namespace ltop;

namespace {

constexpr uint32_t ROWS = 128;      // of the left operand, per block
constexpr uint32_t WIDTH = 256;     // columns of a tile
constexpr uint32_t LEAST_WIDTH = 128;
constexpr uint32_t DEPTH = 64;      // of K at a time: rows of 128 bytes
constexpr int TAKERS = 8;           // warps that take the results: two for the 32 rows of tensor memory that a warp can read, half of the columns each
constexpr uint32_t SIDE = WIDTH / 2;
constexpr int THREADS = 128 + 32 * TAKERS;  // before them a warp that copies, one that multiplies, two that do nothing
constexpr uint32_t STAGE_A = ROWS * DEPTH * 2;

template <int BLOCKS>
struct Ring {
    static constexpr uint32_t STAGE_B = WIDTH / BLOCKS * DEPTH * 2;
    static constexpr uint32_t STAGE = STAGE_A + STAGE_B;
    static constexpr int STAGES = BLOCKS == 1 ? 4 : 6, MOST = BLOCKS == 1 ? 8 : STAGES;  // MOST: of narrower tiles
    static constexpr uint32_t BYTES = STAGES * STAGE + TAKERS * 32 * 128 + 1024;  // (to begin on a multiple of 1024)
};

enum { TO_LOSS, TO_P, TO_SUM, TO_F32, TO_BF16, TO_SCORES };  // TO_SUM, TO_SCORES: binary32, each split its own

struct ProductArgs {
    uint32_t m, n;              // of the result
    uint32_t tiles_m, tiles_n, splits;
    uint32_t width;             // columns of a tile, a multiple of 16 x BLOCKS up to WIDTH
    uint32_t blocks_k;          // steps of K of one product
    uint32_t stages, stage_bytes;  // single blocks
    uint32_t part_a, part_b;    // columns from a part to the next
    // TO_LOSS, TO_P
    const int *targets;
    float scale, scale2;        // scale2: times log2(e), as exponentials are powers of two
    float2 *tops;               // [halves of tiles of the vocabulary][tops_pitch tokens]: maximum and sum, base two
    uint32_t tops_pitch;
    float *target_score;        // [tokens], base two
    uint32_t first, first_tile, vocabulary;  // of the table's row that column 0 of the result is: its number, and that of its tile's first half
    const float *lse;
    __nv_bfloat16 *p;
    uint64_t p_pitch;
    uint32_t p_part, p_rows;    // p_rows: those that are written, zeros behind the tokens
    const uint8_t *odd_a, *odd_b;  // f32: which rows of the operands are not finite (1: infinities, 2: no numbers)
    const float *plain_a, *plain_b;
    uint64_t plain_pitch_a, plain_pitch_b;
    uint32_t plain_cols;
    // TO_SUM, TO_F32, TO_BF16
    const float *factors, *unit;  // of each row, or of all
    const float *before;        // [m][n] to be added, or null
    void *out;                  // [m][n]; TO_SUM: [splits][m][n]
    int wide;                   // columns of `out` come in fours (4) or eights (8), aligned as such
    unsigned int *bad_target, *timeout;
    uint64_t limit_ns;
};

// (a, b) parts of the products of three by three that are kept, smallest first
__device__ __forceinline__ uint32_t part_of_a(uint32_t i) { return (0x001120u >> (4 * i)) & 15; }
__device__ __forceinline__ uint32_t part_of_b(uint32_t i) { return (0x010102u >> (4 * i)) & 15; }

struct Tile {
    uint32_t m, n, split;
};
// Tiles side by side in time share operands in the L2 cache: BAND rows of tiles at a time (8192 x 4096 against 32000 rows: 1.52 ms with 16,
// 1.56 with 9 or 12).
constexpr uint32_t BAND = 16;
__device__ __forceinline__ Tile tile_of(const ProductArgs &a, uint32_t t) {
    Tile r;
    const uint32_t per = a.tiles_m * a.tiles_n;
    r.split = t / per;
    t -= r.split * per;
    const uint32_t band = t / (BAND * a.tiles_n), height = min(BAND, a.tiles_m - BAND * band);
    t -= band * BAND * a.tiles_n;
    r.n = t / height;
    r.m = BAND * band + t - r.n * height;
    return r;
}

// The products of K steps [k0, k1) of a tile
template <int PARTS>
__device__ __forceinline__ void steps_of(const ProductArgs &a, uint32_t split, uint32_t *k0, uint32_t *k1) {
    const uint32_t all = a.blocks_k * (PARTS == 1 ? 1 : 6);
    *k0 = (uint32_t)((uint64_t)all * split / a.splits);
    *k1 = (uint32_t)((uint64_t)all * (split + 1) / a.splits);
}

// What a warp does with its part of a tile: 32 rows of the result, a row per lane, 32 columns at a time.
//
// Rows of the result lie far apart in memory, and 32 of them at once would be 32 requests for 16 bytes each (5.5 us a tile of sums): values
// go through shared memory first, from where eight lanes have a row.
constexpr uint32_t ROOM = 32 * 128;  // of a warp

__device__ __forceinline__ void put_rows(unsigned char *room, const float (&f)[32]) {
    const uint32_t lane = threadIdx.x & 31;
    __syncwarp();  // what was there has been read
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) *reinterpret_cast<float4 *>(room + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
    __syncwarp();
}
// Row 4 i + lane / 8, columns 4 (lane % 8) on
__device__ __forceinline__ float4 get_row(const unsigned char *room, uint32_t i) {
    const uint32_t lane = threadIdx.x & 31, r = 4 * i + (lane >> 3);
    return *reinterpret_cast<const float4 *>(room + r * 128 + (((lane ^ r) & 7) << 4));
}

// The same for bf16: 64 columns, half of them at a time; row 4 i + lane / 8, columns 8 (lane % 8) on
__device__ __forceinline__ void put_half_rows(unsigned char *room, const float (&f)[32], uint32_t half) {
    const uint32_t lane = threadIdx.x & 31;
    if (half == 0) __syncwarp();  // what was there has been read
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        *reinterpret_cast<uint4 *>(room + lane * 128 + (((4 * half + i) ^ (lane & 7)) << 4)) =
            make_uint4(pack_bf16(f[8 * i], f[8 * i + 1]), pack_bf16(f[8 * i + 2], f[8 * i + 3]), pack_bf16(f[8 * i + 4], f[8 * i + 5]), pack_bf16(f[8 * i + 6], f[8 * i + 7]));
    if (half == 1) __syncwarp();
}
__device__ __forceinline__ uint4 get_eight(const unsigned char *room, uint32_t i) {
    const uint32_t lane = threadIdx.x & 31, r = 4 * i + (lane >> 3);
    return *reinterpret_cast<const uint4 *>(room + r * 128 + (((lane ^ r) & 7) << 4));
}
// 64 columns of 32 rows to memory, rows `pitch` apart; `end`: behind the last column that is there, `rows`: how many rows are
__device__ __forceinline__ void store_eights(const unsigned char *room, __nv_bfloat16 *to, uint64_t pitch, uint32_t col, uint32_t end, uint32_t rows) {
    const uint32_t lane = threadIdx.x & 31, r0 = lane >> 3, c = 8 * (lane & 7);
    to += r0 * pitch + col + c;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint4 v = get_eight(room, i);
        if (r0 + 4 * i < rows && col + c < end) *reinterpret_cast<uint4 *>(to + 4 * i * pitch) = v;
    }
}

template <int TO, int PARTS>
struct Epilogue;

template <int PARTS>
struct Epilogue<TO_LOSS, PARTS> {
    const ProductArgs &a;
    uint32_t row;
    bool in;
    int target;
    __device__ __forceinline__ Epilogue(const ProductArgs &a_, const Tile &, uint32_t row_, unsigned char *) : a(a_), row(row_ + (threadIdx.x & 31)), in(row < a_.m) {
        target = in ? a.targets[row] : -1;
        if (target >= 0 && (uint32_t)target >= a.vocabulary) report(a.bad_target);
    }
    // half a row of a tile: columns col .. end
    __device__ __forceinline__ void take_half(float (&f)[SIDE / 32][32], uint32_t col, uint32_t end, const Tile &t, uint32_t side) {
        constexpr int C = SIDE / 32;
        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sums[4] = {};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) f[c][i] *= a.scale2;
        if (col + SIDE > end) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (col + 32 * c + i >= end) f[c][i] = -INFINITY;
        }
        const uint32_t at = (uint32_t)target - a.first - col;
        if (in && target >= 0 && at < SIDE && col + at < end) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (at == (uint32_t)(32 * c + i)) a.target_score[row] = f[c][i];
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(tops[i / 2 % 4]) : "f"(f[c][i]), "f"(f[c][i + 1]));
        const float top = max_nan(max_nan(tops[0], tops[1]), max_nan(tops[2], tops[3])), base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float e;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(f[c][i] - base));
                sums[i % 4] += e;
            }
        if (in) a.tops[(uint64_t)(a.first_tile + 2 * t.n + side) * a.tops_pitch + row] = make_float2(top, (sums[0] + sums[1]) + (sums[2] + sums[3]));
    }
};

template <int PARTS>
struct Epilogue<TO_P, PARTS> {
    const ProductArgs &a;
    unsigned char *room;
    uint32_t row0, row;
    int target;
    float lse2;
    __device__ __forceinline__ Epilogue(const ProductArgs &a_, const Tile &, uint32_t row_, unsigned char *room_) : a(a_), room(room_), row0(row_), row(row_ + (threadIdx.x & 31)) {
        target = row < a.m ? a.targets[row] : -1;
        if ((uint32_t)target >= a.vocabulary) target = -1;
        lse2 = target >= 0 ? a.lse[row] * 1.44269504f : 0.f;
    }
    __device__ __forceinline__ void take(float (&f)[32], uint32_t col) {
        if (col >= a.p_part) return;
        const uint32_t at = (uint32_t)target - a.first - col;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float e;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(f[i], a.scale2, -lse2)));
            if (at == (uint32_t)i) e -= 1.f;
            f[i] = target >= 0 && col + i < a.n ? e : 0.f;
        }
        if constexpr (PARTS == 1) {  // (columns come in 64s)
            const uint32_t half = col >> 5 & 1;
            put_half_rows(room, f, half);
            if (half && row0 < a.p_rows) store_eights(room, a.p + (uint64_t)row0 * a.p_pitch, a.p_pitch, col - 32, a.p_part, a.p_rows - row0);
            return;
        }
        put_rows(room, f);
        const uint32_t lane = threadIdx.x & 31, r0 = row0 + (lane >> 3);
        __nv_bfloat16 *to = a.p + (uint64_t)r0 * a.p_pitch + col + 4 * (lane & 7);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i, to += 4 * a.p_pitch) {
            float4 v = get_row(room, i);
            if (r0 + 4 * i >= a.p_rows) break;
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                const uint2 w = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                *reinterpret_cast<uint2 *>(to + part * a.p_part) = w;
                v.x -= __uint_as_float(w.x << 16);
                v.y -= __uint_as_float(w.x & 0xffff0000u);
                v.z -= __uint_as_float(w.y << 16);
                v.w -= __uint_as_float(w.y & 0xffff0000u);
            }
        }
    }
};

template <int TO, int PARTS>
struct Epilogue {
    const ProductArgs &a;
    unsigned char *room;
    uint32_t row0;
    uint64_t first;  // of the split's result
    float factor;
    __device__ __forceinline__ Epilogue(const ProductArgs &a_, const Tile &t, uint32_t row_, unsigned char *room_)
        : a(a_), room(room_), row0(row_), first(TO == TO_SUM || TO == TO_SCORES ? (uint64_t)t.split * a_.m * a_.n : 0), factor(1.f) {
        const uint32_t row = row0 + (threadIdx.x & 31);
        if (TO != TO_SCORES) factor = !a.factors ? *a.unit : row < a.m ? a.factors[row] : 0.f;
    }
    __device__ __forceinline__ void take(float (&f)[32], uint32_t col) {
#pragma unroll
        for (int i = 0; i < 32 && TO != TO_SCORES; ++i) f[i] = factor == 0.f ? 0.f : f[i] * factor;  // (rows of tokens without a target: zeros, whatever the table holds)
        if (TO == TO_BF16 && a.wide == 8 && !a.before) {
            const uint32_t half = col >> 5 & 1;
            if (col - 32 * half >= a.n || row0 >= a.m) return;
            put_half_rows(room, f, half);
            if (half) store_eights(room, (__nv_bfloat16 *)a.out + (uint64_t)row0 * a.n, a.n, col - 32, a.n, a.m - row0);
            return;
        }
        if (col >= a.n || row0 >= a.m) return;
        put_rows(room, f);
        const uint32_t lane = threadIdx.x & 31, r0 = row0 + (lane >> 3), c = col + 4 * (lane & 7);
        uint64_t at = first + (uint64_t)r0 * a.n + c;
        if (a.wide) {  // (columns come in fours)
            if (c >= a.n) return;
            float4 b[8];
            if (a.before) {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (r0 + 4 * i < a.m) b[i] = *reinterpret_cast<const float4 *>(a.before + at + (uint64_t)(4 * i) * a.n);
            }
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i, at += 4ull * a.n) {
                if (r0 + 4 * i >= a.m) break;
                float4 v = get_row(room, i);
                if (a.before) v.x += b[i].x, v.y += b[i].y, v.z += b[i].z, v.w += b[i].w;
                if (TO == TO_BF16) *reinterpret_cast<uint2 *>((__nv_bfloat16 *)a.out + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                else *reinterpret_cast<float4 *>((float *)a.out + at) = v;
            }
            return;
        }
#pragma unroll 1
        for (uint32_t i = 0; i < 8; ++i, at += 4ull * a.n) {
            if (r0 + 4 * i >= a.m) break;
            const float4 v = get_row(room, i);
            const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                if (c + k >= a.n) break;
                const float y = x[k] + (a.before ? a.before[at + k] : 0.f);
                if (TO == TO_BF16) ((__nv_bfloat16 *)a.out)[at + k] = __float2bfloat16_rn(y);
                else ((float *)a.out)[at + k] = y;
            }
        }
    }
};

// The parts of an infinite f32 value are infinity and zeros, whose products with the parts of another value are no numbers where the
// value's product is infinite.  Scores of rows that hold infinities are therefore made one by one.
__device__ __noinline__ float score_of(const ProductArgs &a, uint32_t row, uint32_t col) {
    const float *x = a.plain_a + row * a.plain_pitch_a, *w = a.plain_b + col * a.plain_pitch_b;
    float s = 0.f;
    for (uint32_t k = 0; k < a.plain_cols; ++k) s += x[k] * w[k];
    return s;
}
// Which rows of the table, under half a tile's columns, and which tokens are not finite
struct Odd {
    int row, column;            // of the lane's token; of the lane's four columns of half a tile, a byte each
    bool any;
};
__device__ __forceinline__ Odd odd_ones(const ProductArgs &a, uint32_t row, uint32_t col) {
    const uint32_t lane = threadIdx.x & 31;
    Odd o{row < a.m ? a.odd_a[row] : 0, 0, false};
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
        if (col + 4 * lane + k < a.n) o.column |= a.odd_b[col + 4 * lane + k] << (8 * k);
    o.any = __any_sync(0xffffffffu, (o.row | o.column) != 0);
    return o;
}
// columns 32 c .. of the half
__device__ __forceinline__ void mend_scores(const ProductArgs &a, const Odd &o, float (&f)[32], uint32_t row, uint32_t col, uint32_t c) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const int other = __shfl_sync(0xffffffffu, o.column, 8 * c + i / 4) >> (8 * (i % 4)) & 255;
        if (row >= a.m) continue;
        if (o.row == 2 || other == 2) f[i] = NAN;
        else if ((o.row == 1 || other == 1) && col + i < a.n) f[i] = score_of(a, row, col + i);
    }
}

// result = A B^T over a list of tiles of ROWS x BLOCKS by WIDTH; BLOCKS: blocks that share a tile, a cluster.  A_TURNED, B_TURNED: the operand
// lies in memory with K down the rows.
//
// One warp copies operands ahead into a ring of stages, one multiplies them into an accumulator in tensor memory, eight take
// finished tiles from there while the next one is made in the other half.  All waits are bounded.
//
// Bound by the tensor cores: the scores of 8192 x 4096 bf16 against 32000 rows take 1.52 ms with everything around them, 1.41 PFLOP/s (a long
// run of products alone sustains 1.36 on the same machines, which lower their clocks to hold their power).  A pair of blocks has 256 x 256,
// so that each brings only half of the columns' operand: with 128 x 256 to a block shared memory is the bound.  Counters of one
// launch (8192 x 2048): tensor cores busy 94 % of the time in scores, 89 in P, 80 in dx (4 rounds of 74 tiles where 3.46 would do), 90 in dtable.
//
// The tensor cores cut what they add off at a unit of the sum's 2^-23, each product of 16 by itself, instead of rounding: 256 additions,
// 4096 of K, left scores 7e-6 too small, and since the sum grows meanwhile 64 times as many of one sign left them 7e-3 too small.  Where
// results are binary32, exact_steps steps of K at a time are summed in tensor memory (0: all of them) and those sums added up in
// registers, by the warps that take them.  Of the six products of parts the first five are 2^-8 of the last one or less, and so is what
// is cut off them: ONE_GO steps of them are summed in one go.
// Gradients in bf16, whose storing costs up to 2^-8, are summed in one go up to ONE_GO steps (8192 products, each cut by 2^-23 at most), and P, which
// an error of the score multiplies, up to ONE_GO_P; longer ones are FAR: 64 steps at a time.  Taking sums out in between costs tiles of a
// short K much (loss and gradients of 257 x 512 against 5003 rows: 45 us, 54 if all products did it), which is why they do not.
constexpr uint32_t ONE_GO = 128, ONE_GO_P = 64;
__host__ __device__ constexpr uint32_t exact_steps(int blocks, int to, int parts, bool far) { return parts == 3 ? 8 : to != TO_LOSS && to != TO_SCORES ? (far ? 64 : 0) : blocks == 1 ? 4 : 16; }
template <int PARTS, uint32_t STEPS>
__device__ __forceinline__ uint32_t chunk_end(const ProductArgs &a, uint32_t step, uint32_t k1) {
    if constexpr (STEPS == 0) return k1;
    if constexpr (PARTS == 3)
        if (step < 5 * a.blocks_k) return min(step + ONE_GO, min(k1, 5 * a.blocks_k));
    return min(k1, step + STEPS);
}

template <int BLOCKS, bool A_TURNED, bool B_TURNED, int TO, int PARTS, bool FAR>
__global__ void __launch_bounds__(THREADS, 1) lt_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const ProductArgs a) {
    using R = Ring<BLOCKS>;
    constexpr uint32_t STEPS = exact_steps(BLOCKS, TO, PARTS, FAR);
    constexpr uint32_t WIDTH_B = WIDTH / BLOCKS;  // of B's rows, per block (at most)
    const uint32_t stages = BLOCKS == 1 ? a.stages : R::STAGES, stage_bytes = BLOCKS == 1 ? a.stage_bytes : R::STAGE;
    extern __shared__ unsigned char product_mem[];
    __shared__ __align__(8) uint64_t barriers[2 * R::MOST + 4];
    __shared__ uint32_t tensor_at, gave_up;
    const uint32_t warp = warp_number(), lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (BLOCKS == 2) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const uint32_t ring = (shared_address(product_mem) + 1023) & ~1023u;
    const uint32_t bar = shared_address(barriers);
    auto full = [&](uint32_t s) { return bar + 8 * s; };
    auto empty = [&](uint32_t s) { return bar + 8 * (R::MOST + s); };
    auto ready = [&](uint32_t b) { return bar + 8 * (2 * R::MOST + b); };
    auto taken = [&](uint32_t b) { return bar + 8 * (2 * R::MOST + 2 + b); };
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t s = 0; s < stages; ++s) {
            barrier_init(full(s), 1);
            barrier_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(ready(b), 1);
            barrier_init(taken(b), TAKERS * BLOCKS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 1) tensor_alloc<BLOCKS>(shared_address(&tensor_at), 512);
    tensor_fence_before();
    __syncthreads();
    if constexpr (BLOCKS == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    tensor_fence_after();
    const uint32_t tensor = tensor_at;
    const Waits waits{&gave_up, a.timeout, a.limit_ns};
    const uint32_t tiles = a.tiles_m * a.tiles_n * a.splits, workers = gridDim.x / BLOCKS, worker = blockIdx.x / BLOCKS;
    pdl_wait();

    if (warp == 0) {
        const uint32_t bytes = BLOCKS * (STAGE_A + (B_TURNED ? R::STAGE_B : a.width / BLOCKS * DEPTH * 2));
        uint32_t stage = 0, phase = 0;
        bool ended = false;
        for (uint32_t i = worker; i < tiles && !ended; i += workers) {
            const Tile t = tile_of(a, i);
            uint32_t k0, k1;
            steps_of<PARTS>(a, t.split, &k0, &k1);
            const int row_a = (int)((t.m * BLOCKS + rank) * ROWS), row_b = (int)(t.n * a.width + rank * (a.width / BLOCKS));
            uint32_t product = k0 / a.blocks_k, k = k0 - product * a.blocks_k;
            for (uint32_t step = k0; step < k1; ++step) {
                if (!waits.wait(empty(stage), phase ^ 1)) {
                    ended = true;
                    break;
                }
                const int at_a = PARTS == 1 ? 0 : (int)(part_of_a(product) * a.part_a), at_b = PARTS == 1 ? 0 : (int)(part_of_b(product) * a.part_b);
                const uint32_t to_a = ring + stage * stage_bytes, to_b = to_a + STAGE_A;
                uint32_t on = full(stage);
                if constexpr (BLOCKS == 2) on = shared_of(on, 0);
                if (one_lane()) {
                    if (rank == 0) barrier_expect(full(stage), bytes);
                    if (A_TURNED) {
#pragma unroll
                        for (uint32_t c = 0; c < ROWS / 64; ++c) copy_tile<BLOCKS>(to_a + c * 64 * DEPTH * 2, &map_a, on, at_a + row_a + 64 * (int)c, (int)(k * DEPTH));
                    } else {
                        copy_tile<BLOCKS>(to_a, &map_a, on, at_a + (int)(k * DEPTH), row_a);
                    }
                    if (B_TURNED) {
#pragma unroll
                        for (uint32_t c = 0; c < WIDTH_B / 64; ++c) copy_tile<BLOCKS>(to_b + c * 64 * DEPTH * 2, &map_b, on, at_b + row_b + 64 * (int)c, (int)(k * DEPTH));
                    } else {
                        copy_tile<BLOCKS>(to_b, &map_b, on, at_b + (int)(k * DEPTH), row_b);
                    }
                }
                __syncwarp();
                if (++stage == stages) stage = 0, phase ^= 1;
                if (++k == a.blocks_k) k = 0, ++product;
            }
        }
        // the last commits arrive here, too, before the block may end
        for (uint32_t s = 0; s < stages && !ended; ++s) {
            if (!waits.wait(empty(stage), phase ^ 1)) break;
            if (++stage == stages) stage = 0, phase ^= 1;
        }
        pdl_release();
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t kind = product_kind(A_TURNED, B_TURNED, ROWS * BLOCKS, a.width);
            const uint32_t low_a = operand_low(ring, A_TURNED, 64 * DEPTH * 2), low_b = operand_low(ring + STAGE_A, B_TURNED, 64 * DEPTH * 2);
            // Few products can be on their way at once: whether the next stage is full is asked before this one's are issued, or
            // the tensor cores would wait for the answer.
            uint32_t stage = 0, phase = 0, turn = 0;
            bool ended = false, there = false;
            for (uint32_t i = worker; i < tiles && !ended; i += workers) {
                const Tile t = tile_of(a, i);
                uint32_t k0, k1;
                steps_of<PARTS>(a, t.split, &k0, &k1);
                uint32_t step = k0;
                do {
                    const uint32_t half = turn & 1, to = tensor + half * WIDTH, from = step, end = chunk_end<PARTS, STEPS>(a, step, k1);
                    if (!waits.wait(taken(half), ((turn >> 1) & 1) ^ 1)) {
                        ended = true;
                        break;
                    }
                    tensor_fence_after();
                    for (; step < end; ++step) {
                        if (!there && !waits.wait(full(stage), phase)) {
                            ended = true;
                            break;
                        }
                        tensor_fence_after();
                        const uint32_t next = stage + 1 == stages ? 0 : stage + 1, next_phase = next ? phase : phase ^ 1;
                        there = __all_sync(0xffffffffu, barrier_done(full(next), next_phase));
                        const uint32_t da = low_a + stage * (stage_bytes >> 4), db = low_b + stage * (stage_bytes >> 4);
                        if (one_lane()) {
#pragma unroll
                            for (uint32_t k = 0; k < DEPTH / 16; ++k)
                                multiply_tiles<BLOCKS>(to, da + k * ((A_TURNED ? 16 * 128 : 32) >> 4), db + k * ((B_TURNED ? 16 * 128 : 32) >> 4), OPERAND_HIGH, OPERAND_HIGH, kind, step > from || k > 0);
                            tensor_commit<BLOCKS>(empty(stage));
                        }
                        __syncwarp();
                        stage = next;
                        phase = next_phase;
                    }
                    if (ended) break;
                    if (one_lane()) tensor_commit<BLOCKS>(ready(half));
                    __syncwarp();
                    ++turn;
                } while (step < k1);
            }
        }
    } else if (warp >= 4) {
        const uint32_t part = warp & 3, side = (warp - 4) >> 2, from = side * SIDE;
        unsigned char *const room = product_mem + (ring - shared_address(product_mem)) + R::STAGES * R::STAGE + (warp - 4) * ROOM;
        uint32_t turn = 0;
        bool ended = false;
        for (uint32_t i = worker; i < tiles; i += workers) {
            const Tile t = tile_of(a, i);
            uint32_t k0, k1;
            steps_of<PARTS>(a, t.split, &k0, &k1);
            Epilogue<TO, PARTS> to(a, t, (t.m * BLOCKS + rank) * ROWS + part * 32, room);
            const uint32_t col = t.n * a.width + from, end = min(a.n, (t.n + 1) * a.width);
            auto begin = [&]() {
                if (!waits.wait(ready(turn & 1), (turn >> 1) & 1)) return false;
                tensor_fence_after();
                return true;
            };
            auto place = [&](uint32_t c) { return tensor + ((part * 32) << 16) + (turn & 1) * WIDTH + from + c; };
            auto leave = [&]() {
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (BLOCKS == 2) barrier_arrive_at(shared_of(taken(turn & 1), 0));
                    else barrier_arrive_at(taken(turn & 1));
                }
                ++turn;
            };
            Odd odd{};
            if constexpr (PARTS == 3 && (TO == TO_LOSS || TO == TO_P)) odd = odd_ones(a, to.row, col);
            auto take = [&](float (&f)[32], uint32_t c) {
                if constexpr (TO == TO_P) {
                    if constexpr (PARTS == 3)
                        if (odd.any) mend_scores(a, odd, f, to.row, c, (c - col) / 32);
                } else if (k0 == k1) {  // a split without a step of K
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = 0.f;
                }
                if constexpr (TO != TO_LOSS) to.take(f, c);
                __syncwarp();
            };
            if constexpr (STEPS > 0) {
                float sum[SIDE / 32][32];
#pragma unroll
                for (uint32_t c = 0; c < SIDE; ++c) sum[c / 32][c % 32] = 0.f;
                uint32_t step = k0;
                do {
                    if (!begin()) {
                        ended = true;
                        break;
                    }
#pragma unroll
                    for (uint32_t c = 0; c < SIDE / 16; ++c) {
                        float f[16];
                        tensor_read(place(c * 16), f);
#pragma unroll
                        for (int k = 0; k < 16; ++k) sum[c / 2][c % 2 * 16 + k] += f[k];
                    }
                    leave();
                    step = chunk_end<PARTS, STEPS>(a, step, k1);
                } while (step < k1);
                if (ended) break;
                if constexpr (TO == TO_LOSS) {
                    if constexpr (PARTS == 3)
                        if (odd.any) {
#pragma unroll
                            for (uint32_t c = 0; c < SIDE / 32; ++c) mend_scores(a, odd, sum[c], to.row, col + c * 32, c);
                        }
                    to.take_half(sum, col, end, t, side);
                } else {
#pragma unroll
                    for (uint32_t c = 0; c < SIDE / 32; ++c)
                        if (from + c * 32 < a.width) {
                            asm volatile("" ::: "memory");  // (one after the other: there are no registers for more at once)
                            take(sum[c], col + c * 32);
                        }
                }
            } else {
                if (!begin()) break;
#pragma unroll 1
                for (uint32_t c = 0; c < SIDE && from + c < a.width; c += 32) {
                    float f[32];
                    tensor_read(place(c), f);
                    take(f, col + c);
                }
                leave();
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (gave_up) {  // copies and products that are still on their way end in far less than this
        const uint64_t t0 = now_ns();
        while (now_ns() - t0 < 1000000) __nanosleep(1000);
    }
    __syncwarp();
    if constexpr (BLOCKS == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (warp == 1) {
        tensor_fence_after();
        tensor_free<BLOCKS>(tensor, 512);
    }
}

// ------------------------------------------------------------------------------------------- around the products

// Two maxima and sums (of powers of two) as one
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
    const float m = max_nan(a.x, b.x);
    if (m == -INFINITY) return make_float2(m, 0.f);
    return make_float2(m, (a.x == -INFINITY ? 0.f : a.y * exp2f(a.x - m)) + (b.x == -INFINITY ? 0.f : b.y * exp2f(b.x - m)));
}

// lse and loss of every token from what the tiles left, always in the same order: 32 / ACROSS lanes and the block's eight warps
// have tiles of ACROSS tokens each (few tokens: one across, so that all lanes have work).
template <uint32_t ACROSS>
__global__ void __launch_bounds__(256) lt_loss_join(const float2 *tops, const float *target_score, const int *targets, float *loss, float *lse, uint32_t tokens, uint32_t pitch, uint32_t tiles, uint32_t vocabulary) {
    constexpr uint32_t SHARES = 256 / ACROSS;
    pdl_release();
    pdl_wait();
    const uint32_t n = blockIdx.x * ACROSS + threadIdx.x % ACROSS, share = threadIdx.x / ACROSS;
    __shared__ float2 sums[8][32];
    float2 s = make_float2(-INFINITY, 0.f);
    if (n < tokens) {
        uint32_t t = share;
        for (; t + 3 * SHARES < tiles; t += 4 * SHARES) {
            float2 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = tops[(uint64_t)(t + k * SHARES) * pitch + n];
            s = joined(s, joined(joined(v[0], v[1]), joined(v[2], v[3])));
        }
        for (; t < tiles; t += SHARES) s = joined(s, tops[(uint64_t)t * pitch + n]);
    }
#pragma unroll
    for (int d = 16; d >= (int)ACROSS; d >>= 1) s = joined(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, d), __shfl_xor_sync(0xffffffffu, s.y, d)));
    sums[threadIdx.x >> 5][threadIdx.x & 31] = s;
    __syncthreads();
    if (threadIdx.x >= ACROSS || n >= tokens) return;
    for (int k = 1; k < 8; ++k) s = joined(s, sums[k][threadIdx.x]);
    const float l = fabsf(s.x) == INFINITY ? 0.f : log2f(s.y);
    if (lse) lse[n] = (s.x + l) * 0.693147181f;
    // (the difference of the scores first: a target with nearly all the weight keeps its small loss)
    if (loss) loss[n] = (uint32_t)targets[n] < vocabulary ? ((s.x - target_score[n]) + l) * 0.693147181f : 0.f;
}

cudaError_t launch_join(const ProductArgs &a, uint32_t tiles, float *loss, float *lse, cudaStream_t stream) {
    const float2 *tops = a.tops;
    const float *score = a.target_score;
    if (a.m <= 64) return launch_pdl(lt_loss_join<1>, a.m, 256, (size_t)0, stream, tops, score, a.targets, loss, lse, a.m, a.tops_pitch, tiles, a.vocabulary);
    return launch_pdl(lt_loss_join<8>, (a.m + 7) / 8, 256, (size_t)0, stream, tops, score, a.targets, loss, lse, a.m, a.tops_pitch, tiles, a.vocabulary);
}

// Few scores: one tile after the other would leave most of the GPU idle for the length of K, so that several workers have a tile, for a
// part of K each, and leave sums of scores (see cut_of_scores).  A block adds up those of a token, and makes its loss and
// lse, or its row of P, of them.
template <bool GRAD, int PARTS>
__global__ void __launch_bounds__(256) lt_loss_finish(const ProductArgs a, const float *scores, uint32_t splits, float *loss, float *lse) {
    __shared__ float2 sums[8];
    __shared__ float at_target;
    pdl_release();
    pdl_wait();
    const uint32_t row = blockIdx.x;
    const bool there = row < a.m;
    int target = there ? a.targets[row] : -1;
    if (!GRAD && target >= 0 && (uint32_t)target >= a.vocabulary && threadIdx.x == 0) report(a.bad_target);
    if ((uint32_t)target >= a.vocabulary) target = -1;
    auto score = [&](uint32_t c) {
        float z = 0.f;
        const float *from = scores + (uint64_t)row * a.n + c;
#pragma unroll 8
        for (uint32_t k = 0; k < splits; ++k) z += from[(uint64_t)k * a.m * a.n];
        if constexpr (PARTS == 3) {
            const int odd = a.odd_a[row], other = a.odd_b[c];
            if (odd | other) z = odd == 2 || other == 2 ? NAN : score_of(a, row, c);
        }
        return z * a.scale2;
    };
    if constexpr (GRAD) {
        const float lse2 = target >= 0 ? a.lse[row] * 1.44269504f : 0.f;
        __nv_bfloat16 *to = a.p + (uint64_t)row * a.p_pitch;
        for (uint32_t c = threadIdx.x; c < a.p_part; c += 256) {
            float v = 0.f;
            if (target >= 0 && c < a.n) v = exp2f(score(c) - lse2) - (a.first + c == (uint32_t)target ? 1.f : 0.f);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                const __nv_bfloat16 h = __float2bfloat16_rn(v);
                to[part * a.p_part + c] = h;
                v -= __bfloat162float(h);
            }
        }
    } else {
        float2 s = make_float2(-INFINITY, 0.f);
        for (uint32_t c = threadIdx.x; c < a.n; c += 256) {
            const float z = score(c);
            if ((int)c == target) at_target = z;
            s = joined(s, make_float2(z, 1.f));
        }
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) s = joined(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, d), __shfl_xor_sync(0xffffffffu, s.y, d)));
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
        __syncthreads();
        if (threadIdx.x) return;
        for (int k = 1; k < 8; ++k) s = joined(s, sums[k]);
        const float l = fabsf(s.x) == INFINITY ? 0.f : log2f(s.y);
        if (lse) lse[row] = (s.x + l) * 0.693147181f;
        if (loss) loss[row] = target >= 0 ? ((s.x - at_target) + l) * 0.693147181f : 0.f;
    }
}

// ------------------------------------------------------------------------------------------- few tokens

// One or two tokens: the table is read once, at the memory's rate, by warps that have FEW_ROWS of its rows at a time, 16 bytes of each per lane;
// products and sums in binary32.  (A tile of the tensor cores would be nearly all padding, and f32 rows would have to be taken apart first.)
constexpr int FEW_ROWS = 2, FEW_THREADS = 256, SOME_THREADS = 512;

struct FewArgs {
    const void *x, *table;
    const int *targets;
    float2 *tops;               // [blocks][tokens]
    float *target_score;
    uint64_t x_pitch, table_pitch;
    uint32_t tokens, vocabulary, cols;
    float scale2;
    unsigned int *bad_target;
};

// N values of T that lie side by side: 16 bytes, or one
template <class T, int N>
struct Loaded {
    uint4 v;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (N == 1) v.x = __float_as_uint(to_float(*p));
        else v = __ldcs(reinterpret_cast<const uint4 *>(p));
    }
    __device__ __forceinline__ void load_shared(const T *p) {
        if constexpr (N == 1) v.x = __float_as_uint(to_float(*p));
        else v = *reinterpret_cast<const uint4 *>(p);
    }
    __device__ __forceinline__ void values(float (&f)[N]) const {
        if constexpr (N == 1) f[0] = __uint_as_float(v.x);
        else unpack(v, f);
    }
};

template <class T, int N, int TOKENS>
__global__ void __launch_bounds__(FEW_THREADS, 3) lt_loss_few(const FewArgs a) {
    constexpr int WARPS = FEW_THREADS / 32, AHEAD = 4;
    extern __shared__ uint4 few_mem[];  // x: [tokens][columns], as it lies in memory (N > 1), in pieces of 16 bytes
    T *const xs = reinterpret_cast<T *>(few_mem);
    __shared__ float2 sums[WARPS][TOKENS];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = (a.cols + 7) & ~7u;
    pdl_release();
    pdl_wait();
    for (int t = 0; t < TOKENS; ++t)
        for (uint32_t c = threadIdx.x; c < a.cols; c += FEW_THREADS) xs[t * pitch + c] = ((const T *)a.x)[t * a.x_pitch + c];
    int target[TOKENS];
    float2 s[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        target[t] = a.targets[t];
        if (blockIdx.x == 0 && threadIdx.x == 0 && target[t] >= 0 && (uint32_t)target[t] >= a.vocabulary) report(a.bad_target);
        s[t] = make_float2(-INFINITY, 0.f);
    }
    __syncthreads();
    const uint32_t v0 = (uint32_t)((uint64_t)a.vocabulary * blockIdx.x / gridDim.x), v1 = (uint32_t)((uint64_t)a.vocabulary * (blockIdx.x + 1) / gridDim.x);
    for (uint32_t v = v0 + warp * FEW_ROWS; v < v1; v += WARPS * FEW_ROWS) {
        float dot[FEW_ROWS][TOKENS] = {};
        const T *row[FEW_ROWS];
#pragma unroll
        for (int r = 0; r < FEW_ROWS; ++r) row[r] = (const T *)a.table + (uint64_t)min(v + r, v1 - 1) * a.table_pitch;
        if constexpr (N == 1) {
            for (uint32_t c = lane; c < a.cols; c += 32) {
#pragma unroll
                for (int r = 0; r < FEW_ROWS; ++r) {
                    const float w = to_float(row[r][c]);
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) dot[r][t] += w * to_float(xs[t * pitch + c]);
                }
            }
        } else {
            for (uint32_t c0 = lane * N; c0 < a.cols; c0 += 32 * N * AHEAD) {
                uint4 w[AHEAD][FEW_ROWS];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int r = 0; r < FEW_ROWS; ++r) {
                        const uint32_t c = c0 + k * 32 * N;
                        if (c < a.cols) w[k][r] = __ldcs(reinterpret_cast<const uint4 *>(row[r] + c));
                    }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const uint32_t c = c0 + k * 32 * N;
                    if (c >= a.cols) break;
                    float f[FEW_ROWS][N];
#pragma unroll
                    for (int r = 0; r < FEW_ROWS; ++r) unpack(w[k][r], f[r]);
#pragma unroll
                    for (int t = 0; t < TOKENS; ++t) {
                        float x[N];
                        unpack(*reinterpret_cast<const uint4 *>(xs + t * pitch + c), x);
#pragma unroll
                        for (int r = 0; r < FEW_ROWS; ++r)
#pragma unroll
                            for (int i = 0; i < N; ++i) dot[r][t] += f[r][i] * x[i];
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < FEW_ROWS; ++r)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                const float z = warp_sum(dot[r][t]) * a.scale2;
                if (v + r >= v1) continue;
                s[t] = joined(s[t], make_float2(z, 1.f));
                if ((int)(v + r) == target[t] && lane == 0) a.target_score[t] = z;
            }
    }
    if (lane == 0) {
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sums[warp][t] = s[t];
    }
    __syncthreads();
    if (threadIdx.x < TOKENS) {
        float2 r = sums[0][threadIdx.x];
        for (int w = 1; w < WARPS; ++w) r = joined(r, sums[w][threadIdx.x]);
        a.tops[(uint64_t)blockIdx.x * TOKENS + threadIdx.x] = r;
    }
}

// The same for TOKENS tokens at a time, ROWS of the table's rows to a warp, so that what is read from shared memory serves several rows.
// The warp's ROWS x TOKENS sums over its lanes are made by halving: each lane sends half of its values and keeps the sums of the other half,
// and is left with one or two, of one row.
template <class T, int N, int TOKENS>
__global__ void __launch_bounds__(SOME_THREADS, 1) lt_loss_some(const FewArgs a) {
    constexpr int ROWS_AT_ONCE = TOKENS < 8 ? 32 / TOKENS : 4, VALUES = ROWS_AT_ONCE * TOKENS, EACH = VALUES / 32, WARPS = SOME_THREADS / 32, AHEAD = 8 / ROWS_AT_ONCE;
    extern __shared__ uint4 few_mem[];  // x: [TOKENS][columns], as it lies in memory
    T *const xs = reinterpret_cast<T *>(few_mem);
    __shared__ float2 sums[WARPS][TOKENS];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = (a.cols + 7) & ~7u, first = blockIdx.y * TOKENS, tokens = min((uint32_t)TOKENS, a.tokens - first);
    pdl_release();
    pdl_wait();
    for (uint32_t t = 0; t < TOKENS; ++t)
        for (uint32_t c = threadIdx.x; c < pitch; c += SOME_THREADS) xs[t * pitch + c] = t < tokens && c < a.cols ? ((const T *)a.x)[(first + t) * a.x_pitch + c] : from_float<T>(0.f);
    // the lane's values: of row `mine` of those at once, tokens from `token` on
    const uint32_t value = lane * EACH, mine = value / TOKENS, token = value % TOKENS;
    int target[EACH];
    float2 s[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        target[e] = token + e < tokens ? a.targets[first + token + e] : -1;
        if (blockIdx.x == 0 && warp == 0 && mine == 0 && target[e] >= 0 && (uint32_t)target[e] >= a.vocabulary) report(a.bad_target);
        s[e] = make_float2(-INFINITY, 0.f);
    }
    __syncthreads();
    const uint32_t v0 = (uint32_t)((uint64_t)a.vocabulary * blockIdx.x / gridDim.x), v1 = (uint32_t)((uint64_t)a.vocabulary * (blockIdx.x + 1) / gridDim.x);
    for (uint32_t v = v0 + warp * ROWS_AT_ONCE; v < v1; v += WARPS * ROWS_AT_ONCE) {
        float dot[VALUES] = {};
        const T *row[ROWS_AT_ONCE];
#pragma unroll
        for (int r = 0; r < ROWS_AT_ONCE; ++r) row[r] = (const T *)a.table + (uint64_t)min(v + r, v1 - 1) * a.table_pitch;
        for (uint32_t c0 = lane * N; c0 < a.cols; c0 += 32 * N * AHEAD) {
            Loaded<T, N> w[AHEAD][ROWS_AT_ONCE];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int r = 0; r < ROWS_AT_ONCE; ++r)
                    if (c0 + k * 32 * N < a.cols) w[k][r].load(row[r] + c0 + k * 32 * N);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const uint32_t c = c0 + k * 32 * N;
                if (c >= a.cols) break;
                float f[ROWS_AT_ONCE][N];
#pragma unroll
                for (int r = 0; r < ROWS_AT_ONCE; ++r) w[k][r].values(f[r]);
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) {
                    float x[N];
                    Loaded<T, N> l;
                    l.load_shared(xs + t * pitch + c);
                    l.values(x);
#pragma unroll
                    for (int r = 0; r < ROWS_AT_ONCE; ++r)
#pragma unroll
                        for (int i = 0; i < N; ++i) dot[r * TOKENS + t] += f[r][i] * x[i];
                }
            }
        }
#pragma unroll
        for (int d = 16, n = VALUES / 2; d >= 1; d >>= 1, n >>= 1) {
            const bool upper = lane & d;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float keep = upper ? dot[i + n] : dot[i], send = upper ? dot[i] : dot[i + n];
                dot[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
            }
        }
        if (v + mine < v1) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const float z = dot[e] * a.scale2;
                s[e] = joined(s[e], make_float2(z, 1.f));
                if ((int)(v + mine) == target[e]) a.target_score[first + token + e] = z;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
#pragma unroll
        for (int d = TOKENS / EACH; d < 32; d <<= 1) s[e] = joined(s[e], make_float2(__shfl_xor_sync(0xffffffffu, s[e].x, d), __shfl_xor_sync(0xffffffffu, s[e].y, d)));
    if (mine == 0) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) sums[warp][token + e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x < tokens) {
        float2 r = sums[0][threadIdx.x];
        for (int w = 1; w < WARPS; ++w) r = joined(r, sums[w][threadIdx.x]);
        a.tops[(uint64_t)blockIdx.x * a.tokens + first + threadIdx.x] = r;
    }
}

// The gradients of few tokens, TOKENS at a time (through tiles of 128 tokens most of the work would be padding; figures at FewGrad):
// a block has whole rows of the table, eight columns to a thread, and with them in registers makes the scores (its threads' sums
// joined by the warps and then through shared memory), the rows of dtable, and its share of dx, which lt_loss_few_join adds up.
// The table is read once and dtable written once; the rows to come are on their way meanwhile.  One token of 4096 bf16 against
// 32000 rows: 98 us, 4.7 TB/s, a barrier per four rows; eight of 2048 f32 174, half of them issue slots.
constexpr uint32_t FEW_GRAD_THREADS = 512, FEW_GRAD_COLS = 8;

struct FewGradArgs {
    const void *x, *table;
    const int *targets;
    const float *lse, *dloss;
    void *dtable;               // or null
    float *dx;                  // [blocks][tokens][cols], or null
    uint64_t x_pitch, table_pitch;
    uint32_t tokens, vocabulary, cols;
    float scale, scale2;
    int add;                    // to what dtable holds of the tokens before
    unsigned int *bad_target;
};

// sum += q f, two values an instruction
template <int N>
__device__ __forceinline__ void add_scaled(float (&sum)[N], float q, const float (&f)[N]) {
    if constexpr (N == 1) {
        sum[0] += q * f[0];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            asm("{.reg .b64 s, f, q; mov.b64 s, {%0, %1}; mov.b64 f, {%2, %3}; mov.b64 q, {%4, %4}; fma.rn.f32x2 s, q, f, s; mov.b64 {%0, %1}, s;}"
                : "+f"(sum[i]), "+f"(sum[i + 1])
                : "f"(f[i]), "f"(f[i + 1]), "f"(q));
    }
}

template <class T, int N, int TOKENS>
__global__ void __launch_bounds__(FEW_GRAD_THREADS, 1) lt_loss_few_grad(const FewGradArgs a) {
    constexpr int ROWS_AT_ONCE = sizeof(T) == 2 ? 4 : 2, PIECES = FEW_GRAD_COLS / N, VALUES = ROWS_AT_ONCE * TOKENS, LANES = 32 / VALUES, WARPS = FEW_GRAD_THREADS / 32;
    static_assert(VALUES <= 32, "a lane for each score at least");
    extern __shared__ uint4 few_mem[];  // x: [TOKENS][columns], zeros for tokens that do not count
    T *const xs = reinterpret_cast<T *>(few_mem);
    __shared__ float part[2][WARPS][VALUES];
    __shared__ __align__(16) float weights[WARPS][VALUES];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, pitch = (a.cols + 7) & ~7u;
    // the lane's score of those at once: of row `mine`, token `token`
    const uint32_t value = lane / LANES, mine = value / TOKENS, token = value % TOKENS;
    pdl_release();
    pdl_wait();
    for (uint32_t t = 0; t < TOKENS; ++t) {
        const bool counts = t < a.tokens && (uint32_t)a.targets[t] < a.vocabulary;
        for (uint32_t c = threadIdx.x; c < pitch; c += blockDim.x) xs[t * pitch + c] = counts && c < a.cols ? ((const T *)a.x)[t * a.x_pitch + c] : from_float<T>(0.f);
    }
    int target = token < a.tokens ? a.targets[token] : -1;
    if (blockIdx.x == 0 && warp == 0 && target >= 0 && (uint32_t)target >= a.vocabulary) report(a.bad_target);
    if ((uint32_t)target >= a.vocabulary) target = -1;
    const float lse2 = target >= 0 ? a.lse[token] * 1.44269504f : 0.f, factor = target >= 0 ? a.dloss[token] * a.scale : 0.f;
    __syncthreads();
    const uint32_t v0 = (uint32_t)((uint64_t)a.vocabulary * blockIdx.x / gridDim.x), v1 = (uint32_t)((uint64_t)a.vocabulary * (blockIdx.x + 1) / gridDim.x);
    auto col = [&](int k) { return (k * blockDim.x + threadIdx.x) * N; };
    Loaded<T, N> w[PIECES][ROWS_AT_ONCE], next[PIECES][ROWS_AT_ONCE];
    auto load = [&](Loaded<T, N> (&to)[PIECES][ROWS_AT_ONCE], uint32_t v) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int r = 0; r < ROWS_AT_ONCE; ++r) {
                to[k][r].v = make_uint4(0, 0, 0, 0);
                if (v + r < v1 && col(k) < a.cols) to[k][r].load((const T *)a.table + (uint64_t)(v + r) * a.table_pitch + col(k));
            }
    };
    float dx[TOKENS][PIECES][N] = {};
    load(w, v0);
    uint32_t turn = 0;
    for (uint32_t v = v0; v < v1; v += ROWS_AT_ONCE, turn ^= 1) {
        load(next, v + ROWS_AT_ONCE);
        float dot[VALUES] = {};
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (col(k) >= a.cols) break;
            float f[ROWS_AT_ONCE][N];
#pragma unroll
            for (int r = 0; r < ROWS_AT_ONCE; ++r) w[k][r].values(f[r]);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                float x[N];
                Loaded<T, N> l;
                l.load_shared(xs + t * pitch + col(k));
                l.values(x);
#pragma unroll
                for (int r = 0; r < ROWS_AT_ONCE; ++r)
#pragma unroll
                    for (int i = 0; i < N; ++i) dot[r * TOKENS + t] += f[r][i] * x[i];
            }
        }
        __syncwarp();
        // as lt_loss_some does it, and the last values between all lanes that have them
#pragma unroll
        for (int d = 16, n = VALUES / 2; d >= 1; d >>= 1, n >>= 1) {
            if (n > 0) {
                const bool upper = lane & d;
#pragma unroll
                for (int i = 0; i < n; ++i) {
                    const float keep = upper ? dot[i + n] : dot[i], send = upper ? dot[i] : dot[i + n];
                    dot[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
                }
            } else {
                dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], d);
            }
        }
        if (lane % LANES == 0) part[turn][warp][value] = dot[0];
        __syncthreads();
        float z = 0.f;
#pragma unroll 4
        for (uint32_t k = 0; k < warps; ++k) z += part[turn][k][value];
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(z, a.scale2, -lse2)));
        if (v + mine == (uint32_t)target) e -= 1.f;
        if (lane % LANES == 0) weights[warp][value] = target >= 0 ? e * factor : 0.f;
        __syncwarp();
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (col(k) >= a.cols) break;
            float f[ROWS_AT_ONCE][N], out[ROWS_AT_ONCE][N] = {};
#pragma unroll
            for (int r = 0; r < ROWS_AT_ONCE; ++r) w[k][r].values(f[r]);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                float x[N];
                Loaded<T, N> l;
                l.load_shared(xs + t * pitch + col(k));
                l.values(x);
#pragma unroll
                for (int r = 0; r < ROWS_AT_ONCE; ++r) {
                    const float q = weights[warp][r * TOKENS + t];
                    if (v + r >= v1) continue;  // (its scores are not any row's)
                    add_scaled(out[r], q, x);
                    add_scaled(dx[t][k], q, f[r]);
                }
            }
            if (!a.dtable) continue;
#pragma unroll
            for (int r = 0; r < ROWS_AT_ONCE; ++r) {
                if (v + r >= v1) continue;
                T *to = (T *)a.dtable + (uint64_t)(v + r) * a.cols + col(k);
                if (a.add) {
                    Loaded<T, N> before;
                    float b[N];
                    before.load(to);
                    before.values(b);
#pragma unroll
                    for (int i = 0; i < N; ++i) out[r][i] += b[i];
                }
                if constexpr (N == 1) *to = from_float<T>(out[r][0]);
                else *reinterpret_cast<uint4 *>(to) = pack(out[r]);
            }
        }
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int r = 0; r < ROWS_AT_ONCE; ++r) w[k][r] = next[k][r];
    }
    if (!a.dx) return;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        if (t >= a.tokens) break;
        float *to = a.dx + ((uint64_t)blockIdx.x * a.tokens + t) * a.cols;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (col(k) >= a.cols) break;
#pragma unroll
            for (int i = 0; i < N; ++i) to[col(k) + i] = dx[t][k][i];
        }
    }
}

// dx of few tokens: the blocks' shares, eight warps having an eighth of them each
template <class T>
__global__ void __launch_bounds__(256) lt_loss_few_join(const float *shares, T *dx, const int *targets, const float *dloss, float scale, uint32_t tokens, uint32_t cols, uint32_t blocks, uint32_t vocabulary) {
    __shared__ float sums[8][32];
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, count = tokens * cols, at = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (at < count) {
        const uint32_t k1 = (uint32_t)((uint64_t)blocks * (warp + 1) / 8);
#pragma unroll 16
        for (uint32_t k = (uint32_t)((uint64_t)blocks * warp / 8); k < k1; ++k) s += shares[(uint64_t)k * count + at];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || at >= count) return;
    for (int k = 1; k < 8; ++k) s += sums[k][lane];
    const uint32_t t = at / cols;
    dx[at] = from_float<T>((uint32_t)targets[t] < vocabulary && dloss[t] * scale != 0.f ? s : 0.f);
}

struct PackArgs {
    const void *from;
    uint64_t pitch;
    __nv_bfloat16 *to;          // [rows][parts][padded]; or null
    uint8_t *odd;               // three parts: 1 for rows with infinities, 2 for rows with what is no number
    uint32_t rows, present, cols, padded;  // present: rows that there are; zeros behind them
    // x for the gradient of the table: `scaled`, rows without a target zeros, the others times dloss / unit; rows' factors scale dloss
    __nv_bfloat16 *scaled;
    const int *targets;
    const float *dloss;
    float *factors, *unit;      // *unit: times scale
    float scale;
    uint32_t vocabulary;
    unsigned int *bad_target;
    const float *largest;       // [LARGEST_BLOCKS], or null
};

// The largest finite |dloss| of the tokens that have a target; 1 if there is none but zeros.  Relative to it no row of x becomes larger
// than it is, and what becomes too small for binary32 is below 2^-126 of what the largest one adds.  By a whole block: of all tokens, or
// of what lt_loss_largest has left of each of its blocks.
__device__ __forceinline__ float largest_dloss(const float *dloss, const int *targets, uint32_t vocabulary, uint32_t first, uint32_t tokens, uint32_t step) {
    __shared__ float part[32];
    float most = 0.f;
#pragma unroll 8
    for (uint32_t n = first; n < tokens; n += step) {
        const float d = fabsf(dloss[n]);
        if ((!targets || (uint32_t)targets[n] < vocabulary) && d < INFINITY) most = fmaxf(most, d);
    }
    return block_reduce<true>(most, part);
}
constexpr uint32_t LARGEST_BLOCKS = 256, LARGEST_ALONE = 4096;  // up to so many tokens every block that needs it looks for it itself
__global__ void __launch_bounds__(256) lt_loss_largest(const float *dloss, const int *targets, float *largest, uint32_t tokens, uint32_t vocabulary) {
    pdl_release();
    pdl_wait();
    const float most = largest_dloss(dloss, targets, vocabulary, blockIdx.x * 256 + threadIdx.x, tokens, gridDim.x * 256);
    if (threadIdx.x == 0) largest[blockIdx.x] = most;
}

// Eight values in bf16 parts; returns what is not finite among them (1: infinities, 2: no numbers).
template <int PARTS>
__device__ __forceinline__ int pack_eight(float (&f)[8], uint4 *to, uint32_t apart) {
    int odd = 0;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __nv_bfloat16 h = __float2bfloat16_rn(f[i]);
            if constexpr (PARTS == 3) {
                if (part == 0) {
                    if (!(fabsf(f[i]) <= 3.38953139e38f)) {  // (the largest bf16)
                        odd |= isinf(f[i]) ? 1 : isnan(f[i]) ? 2 : 0;
                        if (!isinf(f[i])) h = __float2bfloat16_rz(f[i]);  // (the nearest might be infinite)
                    }
                }
                f[i] = isfinite(f[i]) ? f[i] - __bfloat162float(h) : 0.f;
            }
            const uint32_t bits = __bfloat16_as_ushort(h);
            w[i / 2] = i & 1 ? w[i / 2] | bits << 16 : bits;
        }
        to[part * apart] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return odd;
}

// A matrix as the products take it: bf16, in three parts if it is f32, rows padded with zeros to whole steps of K.  A thread has eight
// columns at a time, ACROSS threads (a warp, or the block where rows are long) a row.
template <class T, bool WIDE, uint32_t ACROSS>
__global__ void __launch_bounds__(256) lt_loss_pack(const PackArgs a) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr uint32_t BESIDE = 256 / ACROSS;
    pdl_release();
    pdl_wait();
    const uint32_t eights = a.padded / 8, lane = threadIdx.x % ACROSS;
    float unit = 1.f;
    if (a.scaled) {
        unit = a.largest ? largest_dloss(a.largest, nullptr, 0, threadIdx.x, LARGEST_BLOCKS, 256) : largest_dloss(a.dloss, a.targets, a.vocabulary, threadIdx.x, a.present, 256);
        if (unit == 0.f) unit = 1.f;
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.unit = unit * a.scale;
    }
    for (uint32_t r = blockIdx.x * BESIDE + threadIdx.x / ACROSS; r < a.rows; r += gridDim.x * BESIDE) {
        const bool there = r < a.present;
        float factor = 0.f;
        bool counts = true;
        if (a.scaled && there) {
            const int target = a.targets[r];
            counts = (uint32_t)target < a.vocabulary;
            const float d = counts ? a.dloss[r] : 0.f;
            factor = d / unit;
            if (lane == 0) {
                if (!counts && target >= 0) report(a.bad_target);
                a.factors[r] = d * a.scale;
            }
        }
        const T *from = (const T *)a.from + r * a.pitch;
        uint4 *to = reinterpret_cast<uint4 *>(a.to + (uint64_t)r * PARTS * a.padded), *scaled = reinterpret_cast<uint4 *>(a.scaled + (uint64_t)r * PARTS * a.padded);
        int odd = 0;
#pragma unroll 2
        for (uint32_t c = lane; c < eights; c += ACROSS) {
            float f[8];
            if (WIDE && there && 8 * c + 8 <= a.cols) {
                if constexpr (PARTS == 1) {
                    const uint4 v = reinterpret_cast<const uint4 *>(from)[c];
                    unpack(v, f);
                } else {
                    float g[4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        unpack(reinterpret_cast<const uint4 *>(from)[2 * c + h], g);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[4 * h + i] = g[i];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = there && 8 * c + i < a.cols ? to_float(from[8 * c + i]) : 0.f;
            }
            if (a.scaled) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = factor == 0.f ? 0.f : f[i] * factor;
                pack_eight<PARTS>(x, scaled + c, eights);
            }
            if (a.to) odd |= pack_eight<PARTS>(f, to + c, eights);
        }
        if (PARTS == 3 && a.to) {
            int infinite, no_number;
            if constexpr (ACROSS == 32) {
                __syncwarp();
                no_number = __any_sync(0xffffffffu, odd & 2), infinite = __any_sync(0xffffffffu, odd & 1);
            } else {
                no_number = __syncthreads_or(odd & 2), infinite = __syncthreads_or(odd & 1);
            }
            if (lane == 0) a.odd[r] = !counts ? 0 : no_number ? 2 : infinite ? 1 : 0;  // (what does not count is not looked at)
        }
    }
}

// out = the sum of `splits` results of `count` values, in order; N (4 or 1) values of a thread at a time
template <class R, int N>
__global__ void __launch_bounds__(256) lt_loss_sum(const float *sums, R *out, uint64_t count, uint32_t splits) {
    pdl_release();
    pdl_wait();
    for (uint64_t i = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * N; i < count; i += (uint64_t)gridDim.x * 256 * N) {
        float s[N] = {};
#pragma unroll 8
        for (uint32_t k = 0; k < splits; ++k) {
            if constexpr (N == 4) {
                const float4 v = *reinterpret_cast<const float4 *>(sums + k * count + i);
                s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
            } else {
                s[0] += sums[k * count + i];
            }
        }
        if constexpr (N == 4) {
            if constexpr (sizeof(R) == 4) *reinterpret_cast<float4 *>(out + i) = make_float4(s[0], s[1], s[2], s[3]);
            else *reinterpret_cast<uint2 *>(out + i) = make_uint2(pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3]));
        } else {
            out[i] = from_float<R>(s[0]);
        }
    }
}

// ------------------------------------------------------------------------------------------- host

inline bool is_aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// How many columns of a result can be stored at once: 8, 4 or 0 (one)
inline int width_of(const void *out, uint64_t cols, size_t size) { return size == 2 && cols % 8 == 0 && is_aligned(out, 16) ? 8 : cols % 4 == 0 && is_aligned(out, 4 * size) ? 4 : 0; }
inline uint64_t up_to(uint64_t n, uint64_t of) { return (n + of - 1) / of * of; }
inline uint32_t count_of(uint64_t n, uint64_t of) { return (uint32_t)((n + of - 1) / of); }

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t encoder(EncodeTiled *out) {
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled f = known.load(std::memory_order_relaxed);
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return e;
        if (found != cudaDriverEntryPointSuccess || !p) return cudaErrorNotSupported;
        f = (EncodeTiled)p;
        known.store(f, std::memory_order_relaxed);
    }
    *out = f;
    return cudaSuccess;
}

// bf16 rows in memory as an operand: `cols` a multiple of 8 with the pitch, or padded; tiles of 64 columns by `high` rows.
struct Operand {
    const void *p;
    uint64_t pitch, rows, cols;
    uint32_t part;              // columns from a part to the next
    bool turned;
};

cudaError_t map_of(const Operand &o, uint32_t high, CUtensorMap *map) {
    EncodeTiled encode;
    const cudaError_t e = encoder(&encode);
    if (e != cudaSuccess) return e;
    const cuuint64_t dims[2] = {o.cols, o.rows}, strides[1] = {o.pitch * 2};
    const cuuint32_t box[2] = {64, o.turned ? 64u : high}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(o.p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

template <int BLOCKS, bool A_TURNED, bool B_TURNED, int TO, int PARTS, bool FAR>
cudaError_t launch_product_of(const Operand &x, const Operand &y, const ProductArgs &a, int sm_count, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    auto kernel = lt_product<BLOCKS, A_TURNED, B_TURNED, TO, PARTS, FAR>;
    cudaError_t e = allow_shared(kernel, Ring<BLOCKS>::BYTES, ready);
    CUtensorMap map_a, map_b;
    if (e == cudaSuccess) e = map_of(x, ROWS, &map_a);
    if (e == cudaSuccess) e = map_of(y, a.width / BLOCKS, &map_b);
    if (e != cudaSuccess) return e;
    const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n * a.splits;
    if (tiles >= 1ull << 31) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(std::min<uint64_t>(tiles, (uint64_t)sm_count / BLOCKS) * BLOCKS));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Ring<BLOCKS>::BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = LT_PDL;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {BLOCKS, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = BLOCKS == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, a);
}

// How a product of m x n over k steps is cut: a pair of blocks per tile of 256 rows, single blocks where 128 rows are enough.
struct Cut {
    int blocks;
    uint32_t tiles_m, tiles_n, splits = 1, width = WIDTH;
    // `widths`: tiles may have fewer columns than WIDTH, by multiples of as many (0: no)
    Cut(uint64_t m, uint64_t n, int sm_count, uint32_t widths) {
        blocks = m <= ROWS ? 1 : 2;
        tiles_m = count_of(m, (uint64_t)ROWS * blocks);
        tiles_n = count_of(n, WIDTH);
        // What a round of tiles takes: a pair of blocks brings 256 rows and its columns for each step, and is bound by that below WIDTH
        // columns; a single one, which has few rows, by the columns.  Narrower tiles pay where the last round would be nearly empty:
        // one token against 32000 rows of 4096, 143 tiles of 224 columns 49 us, 125 of 256 56.
        auto cost = [&](uint32_t w) { return (uint64_t)count_of((uint64_t)tiles_m * count_of(n, w), (uint64_t)sm_count / blocks) * (w + (blocks == 1 ? 32 : 256)); };
        for (uint32_t w = WIDTH; widths && w >= (blocks == 1 ? LEAST_WIDTH / 2 : LEAST_WIDTH); w -= widths)
            if (cost(w) < cost(width)) width = w;
        tiles_n = count_of(n, width);
    }
    // few tiles: several workers to a tile, with four steps of K each at least
    Cut &split(uint64_t steps, int sm_count) {
        const uint64_t tiles = (uint64_t)tiles_m * tiles_n, workers = (uint64_t)sm_count / blocks;
        if (2 * tiles <= workers) splits = (uint32_t)std::max<uint64_t>(1, std::min(workers / tiles, steps / 4));
        return *this;
    }
};

template <bool A_TURNED, bool B_TURNED, int TO, int PARTS>
cudaError_t launch_product(const Operand &x, const Operand &y, ProductArgs a, const Cut &cut, int sm_count, cudaStream_t stream) {
    a.tiles_m = cut.tiles_m;
    a.tiles_n = cut.tiles_n;
    a.splits = cut.splits;
    a.width = cut.width;
    a.part_a = x.part;
    a.part_b = y.part;
    // (narrow tiles have more stages, which cover the way to memory by their number: loss and gradients of 128 x 2048 f32 against 32000 rows,
    // tiles of 64 columns, 990 us with eight, 1076 with four, 1104 with 128 columns)
    a.stage_bytes = STAGE_A + (B_TURNED ? WIDTH : cut.width) * DEPTH * 2;
    a.stages = std::min<uint32_t>(Ring<1>::MOST, Ring<1>::STAGES * Ring<1>::STAGE / a.stage_bytes);
    // Beside the limit, a wait may last as long as the work of a tile: its steps (0.4 us each), and scores that are made one by one.
    a.limit_ns += (uint64_t)a.blocks_k * (PARTS == 1 ? 1 : 6) * 4000 + (uint64_t)a.plain_cols * SIDE * 200;
    if constexpr (PARTS == 1 && (TO == TO_P || TO == TO_SUM || TO == TO_BF16))
        if (count_of(a.blocks_k, cut.splits) > (TO == TO_P ? ONE_GO_P : ONE_GO))
            return cut.blocks == 1 ? launch_product_of<1, A_TURNED, B_TURNED, TO, PARTS, true>(x, y, a, sm_count, stream) : launch_product_of<2, A_TURNED, B_TURNED, TO, PARTS, true>(x, y, a, sm_count, stream);
    return cut.blocks == 1 ? launch_product_of<1, A_TURNED, B_TURNED, TO, PARTS, false>(x, y, a, sm_count, stream) : launch_product_of<2, A_TURNED, B_TURNED, TO, PARTS, false>(x, y, a, sm_count, stream);
}

// A packed operand has at least so many rows (zeros): of a tile that holds fewer, copies are slower (5 tokens against 32000 rows of 4096: 73
// us, 16 of them 51).
constexpr uint64_t LEAST_ROWS = 16;

// How the scores of m tokens and n rows are cut: a worker to a tile and no scores in memory, or, where workers would be few and K is long,
// several (splits > 1).  300 x 4096 bf16 against 1000 rows, 64 steps: 20.4 us whole, 21.4 split; 174 x 3944 f32 against 252, 372 steps: 82 and
// 29; loss and gradients of 100 x 1024 f32 against 1000, 96 steps: 113 and 78.
inline Cut cut_of_scores(uint64_t m, uint64_t n, uint64_t cols, int dtype, int sm_count, uint32_t widths) {
    const uint64_t steps = count_of(cols, DEPTH) * (dtype == LT_F32 ? 6 : 1);
    const Cut whole = Cut(m, n, sm_count, 0).split(steps, sm_count);
    return whole.splits > 1 && steps >= 96 ? whole : Cut(m, n, sm_count, widths);
}
inline size_t score_bytes(const Cut &cut, uint64_t m, uint64_t n) { return cut.splits > 1 ? (size_t)up_to(cut.splits * m * n * 4, 256) : 0; }

template <class T>
constexpr uint32_t parts_of() { return sizeof(T) == 4 ? 3 : 1; }

// The gradient's part of PackArgs
struct Scaled {
    void *to = nullptr;
    const int *targets = nullptr;
    const float *dloss = nullptr;
    float *factors = nullptr, *unit = nullptr;
    float scale = 1.f;
    uint32_t vocabulary = 0;
    unsigned int *bad_target = nullptr;
    const float *largest = nullptr;
};
template <class T>
cudaError_t launch_pack(const void *from, uint64_t pitch, uint64_t rows, uint64_t cols, void *to, void *odd, const Scaled &scaled, int sm_count, cudaStream_t stream) {
    const PackArgs p{from,          pitch,           (__nv_bfloat16 *)to, (uint8_t *)odd, (uint32_t)std::max<uint64_t>(rows, LEAST_ROWS), (uint32_t)rows, (uint32_t)cols, (uint32_t)up_to(cols, DEPTH),
                     (__nv_bfloat16 *)scaled.to, scaled.targets,  scaled.dloss,        scaled.factors, scaled.unit, scaled.scale, scaled.vocabulary, scaled.bad_target, scaled.largest};
    const bool wide = is_aligned(from, 16) && pitch * sizeof(T) % 16 == 0, long_rows = p.padded > 8192 || (p.padded >= 512 && rows < 8 * (uint64_t)sm_count);
    const unsigned grid = std::min(count_of(p.rows, long_rows ? 1 : 8), (unsigned)sm_count * 8);
    if (long_rows) return wide ? launch_pdl(lt_loss_pack<T, true, 256>, grid, 256, (size_t)0, stream, p) : launch_pdl(lt_loss_pack<T, false, 256>, grid, 256, (size_t)0, stream, p);
    return wide ? launch_pdl(lt_loss_pack<T, true, 32>, grid, 256, (size_t)0, stream, p) : launch_pdl(lt_loss_pack<T, false, 32>, grid, 256, (size_t)0, stream, p);
}
template <class T>
Operand packed_operand(const void *p, uint64_t rows, uint64_t cols, bool turned) {
    const uint64_t padded = up_to(cols, DEPTH);
    return Operand{p, padded * parts_of<T>(), std::max<uint64_t>(rows, LEAST_ROWS), padded * parts_of<T>(), (uint32_t)padded, turned};
}
inline size_t packed_row(int dtype, uint64_t cols) { return (size_t)up_to(up_to(cols, DEPTH) * 2 * (dtype == LT_F32 ? 3 : 1), 256); }
inline size_t packed_bytes(int dtype, uint64_t rows, uint64_t cols) { return (size_t)up_to(std::max<uint64_t>(rows, LEAST_ROWS) * up_to(cols, DEPTH) * 2 * (dtype == LT_F32 ? 3 : 1), 256); }
// May the matrix be an operand where it lies?
inline bool lies_well(int dtype, const void *p, uint64_t pitch) { return dtype == LT_BF16 && is_aligned(p, 16) && pitch % 8 == 0; }

// Pieces of the vocabulary (or of the tokens): P of one, and what a packed piece of the table takes.  Larger pieces of P are fewer sums of
// dx to bring back (loss and gradients of 8192 x 2048 against 32000 rows: 3.62 ms with 256 MB, 3.90 with 160, 4.08 with 96);
// packed f32 rows are read from the L2 cache if there is not much more of them than fits.
constexpr uint64_t P_BYTES = 256 << 20, PACK_BYTES = 96 << 20, SPARE_BYTES = 8 << 20;

// Rows at a time (a multiple of a tile's columns, pieces of about one size), if a row takes `bytes` and a piece `most`.
uint64_t piece_of(uint64_t rows, uint64_t bytes, uint64_t most) {
    most = std::max<uint64_t>(WIDTH, most / bytes / WIDTH * WIDTH);
    const uint64_t pieces = (rows + most - 1) / most;
    return up_to((rows + pieces - 1) / pieces, WIDTH);
}
// Addresses are not known when scratch is planned: bf16 rows whose distance fits lie well unless they begin in an unusual place, for
// which there is some room, too.
inline uint64_t pack_piece(const LtOperator &o, int k, uint64_t rows) {
    return piece_of(rows, packed_row(o.dtype, o.cols), o.dtype == LT_BF16 && o.pitch[k] % 8 == 0 ? SPARE_BYTES : PACK_BYTES);
}

// Tokens that are scored by plain loads, at a time (0: on the tensor cores), and by how many blocks.  bf16: up to two (one token against
// 32000 rows of 4096: 46 us, two 47.5; three 57 so, 54 on the tensor cores).  f32, which takes six products there: up to 64, 16 at a time
// (against 32000 rows of 2048: 5 tokens 54 us, 658 on the tensor cores; 16 88, 382; 64 331, 386), or 8 or 4 where rows are so long that no more
// of them fit (from 3329 and 6657 columns on; 16 x 4096 190 us, 885 on the tensor cores; 64 757, 888; 16 x 8192 659, 2930; 64 2671, 2936).
constexpr size_t FEW_BYTES = 72 << 10, SOME_BYTES = 208 << 10;  // of x in shared memory
struct Few {
    uint32_t at_once = 0, blocks = 0;
    Few(const LtOperator &o, int sm_count) {
        const uint64_t row = up_to(o.cols, 8) * (o.dtype == LT_BF16 ? 2 : 4);
        if (o.rows > (o.dtype == LT_BF16 ? 2 : 64)) return;
        at_once = o.rows <= 2 ? (uint32_t)o.rows : o.rows <= 4 ? 4 : o.rows <= 8 ? 8 : 16;
        while (at_once > 4 && at_once * row > SOME_BYTES) at_once /= 2;
        if (at_once * row > (at_once <= 2 ? FEW_BYTES : SOME_BYTES)) at_once = 0;
        const uint32_t rows = at_once <= 2 ? FEW_THREADS / 32 * FEW_ROWS : SOME_THREADS / 32 * 4;
        blocks = (uint32_t)std::min<uint64_t>((at_once <= 2 ? 3 : 1) * (uint64_t)sm_count, count_of(o.vocabulary, rows));
    }
};

// Tokens whose gradients are made by plain loads, at a time (0: on the tensor cores), of rows that a block's threads can hold, 4096 columns.
// bf16: up to two; f32: up to 16, every eight of them once through the table.  Loss and gradients against 32000 rows of 4096 bf16: one token 150 us, two 169, four 263 (by tiles 255 all of them);
// of 2048 f32: 1 token 144, 4 160, 8 216, 16 523, 32 1150 (by tiles 705, 704, 714, 753, 796).
struct FewGrad {
    uint32_t at_once = 0, blocks = 0, threads = 0;
    FewGrad(const LtOperator &o, int sm_count) {
        if (o.rows > (o.dtype == LT_BF16 ? 2 : 16) || o.cols > FEW_GRAD_THREADS * FEW_GRAD_COLS) return;
        at_once = o.rows <= 2 ? (uint32_t)o.rows : o.rows <= 4 ? 4 : 8;
        threads = (uint32_t)up_to(count_of(o.cols, FEW_GRAD_COLS), 32);
        blocks = (uint32_t)std::min<uint64_t>((uint64_t)sm_count * std::min(8u, FEW_GRAD_THREADS / threads), count_of(o.vocabulary, 4));
    }
};

struct LossScratch {
    size_t score, odd_x, odd_table, tops, scores, x, table, bytes;
    uint64_t piece, x_piece;    // rows that are packed at a time
    LossScratch(const LtOperator &o, int sm_count) {
        piece = pack_piece(o, 1, o.vocabulary);
        x_piece = o.dtype == LT_F32 ? o.rows : std::min(o.rows, pack_piece(o, 0, o.rows));
        // halves of tiles that maxima and sums are left of: of the whole vocabulary, or of pieces
        uint64_t halves = 0;
        for (uint64_t m : {o.rows, x_piece, o.rows % x_piece}) {
            if (!m) continue;
            const uint64_t rest = o.vocabulary % piece;
            uint64_t some = 2ull * Cut(m, std::min(piece, o.vocabulary), sm_count, 32).tiles_n * (o.vocabulary / piece);
            if (rest) some += 2ull * Cut(m, rest, sm_count, 32).tiles_n;
            halves = std::max({halves, some, (uint64_t)2 * Cut(m, o.vocabulary, sm_count, 32).tiles_n});
        }
        score = 0;
        odd_x = up_to(o.rows * 4, 256);
        odd_table = odd_x + up_to(o.rows + LEAST_ROWS, 256);
        tops = odd_table + up_to(piece + LEAST_ROWS, 256);
        const Few few(o, sm_count);
        if (few.at_once) {
            bytes = tops + up_to(few.blocks * o.rows * sizeof(float2), 256);
            return;
        }
        scores = tops + up_to(halves * o.rows * sizeof(float2), 256);
        x = scores + score_bytes(cut_of_scores(o.rows, o.vocabulary, o.cols, o.dtype, sm_count, 32), o.rows, o.vocabulary);
        table = x + packed_bytes(o.dtype, x_piece, o.cols);
        bytes = table + packed_bytes(o.dtype, piece, o.cols);
    }
};

struct GradScratch {
    size_t unit, largest, factors, scaled, x, odd_x, odd_table, table, p, sum_x, sum_table, scores, bytes;
    uint64_t piece, packed_piece;  // the latter where the table does not lie well
    uint64_t x_piece;           // rows of x that are packed at a time where it does not lie well
    uint32_t splits_table;
    GradScratch(const LtOperator &o, int sm_count) {
        const FewGrad few(o, sm_count);
        if (few.at_once) {
            bytes = few.blocks * few.at_once * o.cols * 4;
            return;
        }
        const uint64_t parts = o.dtype == LT_F32 ? 3 : 1;
        piece = piece_of(o.vocabulary, o.rows * 2 * parts, P_BYTES);
        packed_piece = std::min(piece, pack_piece(o, 1, o.vocabulary));
        if (o.dtype == LT_F32 || o.pitch[1] % 8) piece = packed_piece;
        const uint64_t steps = count_of(piece, DEPTH) * (parts == 1 ? 1 : 6), steps_t = count_of(o.rows, DEPTH) * (parts == 1 ? 1 : 6);
        const Cut cx = Cut(o.rows, o.cols, sm_count, 0).split(steps, sm_count), ct = Cut(piece, o.cols, sm_count, 0).split(steps_t, sm_count);
        unit = 0;
        largest = 256;
        factors = largest + LARGEST_BLOCKS * 4;
        scaled = factors + up_to(o.rows * 4, 256);
        x_piece = o.dtype == LT_F32 || o.rows < LEAST_ROWS ? o.rows : std::min(o.rows, pack_piece(o, 0, o.rows));
        x = scaled + packed_bytes(o.dtype, o.rows, o.cols);
        odd_x = x + packed_bytes(o.dtype, x_piece, o.cols);
        odd_table = odd_x + up_to(o.rows + LEAST_ROWS, 256);
        table = odd_table + up_to(piece + LEAST_ROWS, 256);
        splits_table = ct.splits;
        p = table + packed_bytes(o.dtype, packed_piece, o.cols);
        sum_x = p + up_to(std::max<uint64_t>(o.rows, LEAST_ROWS) * piece * 2 * parts, 256);
        sum_table = sum_x + (packed_piece < o.vocabulary || cx.splits > 1 ? up_to(cx.splits * o.rows * o.cols * 4, 256) : 0);
        scores = sum_table + (ct.splits > 1 ? up_to(ct.splits * piece * o.cols * 4, 256) : 0);
        bytes = scores + (piece >= o.vocabulary ? score_bytes(cut_of_scores(o.rows, o.vocabulary, o.cols, o.dtype, sm_count, 64), o.rows, o.vocabulary) : 0);
    }
};

void common_args(const LtOperator &o, ProductArgs &a) {
    a.targets = (const int *)o.in[2];
    a.vocabulary = (uint32_t)o.vocabulary;
    a.scale = (float)lt_attr_double(o.attr[1]);
    a.scale2 = (float)(lt_attr_double(o.attr[1]) * 1.4426950408889634);
    a.bad_target = &o.status->loss;
    a.timeout = &o.status->timeout;
    a.limit_ns = o.wait_ns;
}

// f32: the operands of the scores themselves
void plain_args(const LtOperator &o, ProductArgs &a, const void *x, const void *odd_x, const void *odd_table, const void *table) {
    if (o.dtype != LT_F32) return;
    a.odd_a = (const uint8_t *)odd_x;
    a.odd_b = (const uint8_t *)odd_table;
    a.plain_a = (const float *)x;
    a.plain_b = (const float *)table;
    a.plain_pitch_a = o.pitch[0];
    a.plain_pitch_b = o.pitch[1];
    a.plain_cols = (uint32_t)o.cols;
}

template <class T, int N, int TOKENS>
cudaError_t launch_few_of(const FewArgs &a, unsigned blocks, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    const size_t bytes = TOKENS * up_to(a.cols, 8) * sizeof(T);
    if constexpr (TOKENS <= 2) {
        const cudaError_t e = allow_shared(lt_loss_few<T, N, TOKENS>, FEW_BYTES, ready);
        return e != cudaSuccess ? e : launch_pdl(lt_loss_few<T, N, TOKENS>, blocks, FEW_THREADS, bytes, stream, a);
    } else {
        const cudaError_t e = allow_shared(lt_loss_some<T, N, TOKENS>, SOME_BYTES, ready);
        return e != cudaSuccess ? e : launch_pdl_shared(lt_loss_some<T, N, TOKENS>, dim3(blocks, count_of(a.tokens, TOKENS)), SOME_THREADS, bytes, stream, a);
    }
}
template <class T, int N>
cudaError_t launch_few(const FewArgs &a, const Few &few, cudaStream_t stream) {
    if constexpr (sizeof(T) == 4) {
        if (few.at_once == 16) return launch_few_of<T, N, 16>(a, few.blocks, stream);
        if (few.at_once == 8) return launch_few_of<T, N, 8>(a, few.blocks, stream);
        if (few.at_once == 4) return launch_few_of<T, N, 4>(a, few.blocks, stream);
    }
    return few.at_once == 1 ? launch_few_of<T, N, 1>(a, few.blocks, stream) : launch_few_of<T, N, 2>(a, few.blocks, stream);
}

template <class T>
cudaError_t launch_loss(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    const LossScratch at(o, sm_count);
    char *room = (char *)o.scratch;
    const Few few(o, sm_count);
    if (few.at_once) {
        ProductArgs a{};
        common_args(o, a);
        a.m = (uint32_t)o.rows;
        a.target_score = (float *)(room + at.score);
        a.tops = (float2 *)(room + at.tops);
        a.tops_pitch = a.m;
        constexpr int N = 16 / (int)sizeof(T);
        const FewArgs f{o.in[0], o.in[1], a.targets, a.tops, a.target_score, o.pitch[0], o.pitch[1], a.m, a.vocabulary, (uint32_t)o.cols, a.scale2, a.bad_target};
        const bool wide = o.cols % N == 0 && o.pitch[1] % N == 0 && is_aligned(o.in[1], 16);
        const cudaError_t e = wide ? launch_few<T, N>(f, few, stream) : launch_few<T, 1>(f, few, stream);
        *launched = 2;
        return e != cudaSuccess ? e : launch_join(a, few.blocks, (float *)o.out[0], (float *)o.out[1], stream);
    }
    const bool x_well = lies_well(o.dtype, o.in[0], o.pitch[0]), table_well = lies_well(o.dtype, o.in[1], o.pitch[1]);
    cudaError_t e = cudaSuccess;
    *launched = 0;
    const uint64_t piece = table_well ? o.vocabulary : at.piece, x_piece = x_well ? o.rows : at.x_piece;
    for (uint64_t r0 = 0; r0 < o.rows; r0 += x_piece) {
        const uint64_t m = std::min(x_piece, o.rows - r0);
        ProductArgs a{};
        common_args(o, a);
        a.m = (uint32_t)m;
        a.targets += r0;
        a.blocks_k = count_of(o.cols, DEPTH);
        a.target_score = (float *)(room + at.score) + r0;
        a.tops = (float2 *)(room + at.tops) + r0;
        a.tops_pitch = (uint32_t)o.rows;
        const T *tokens = (const T *)o.in[0] + r0 * o.pitch[0];
        Operand x{tokens, o.pitch[0], m, o.cols, 0, false};
        if (!x_well || m < LEAST_ROWS) {
            e = launch_pack<T>(tokens, o.pitch[0], m, o.cols, room + at.x, room + at.odd_x, Scaled{}, sm_count, stream);
            if (e != cudaSuccess) return e;
            x = packed_operand<T>(room + at.x, m, o.cols, false);
            ++*launched;
        }
        for (uint64_t v0 = 0; v0 < o.vocabulary; v0 += piece) {
            const uint64_t n = std::min(piece, o.vocabulary - v0);
            const T *rows = (const T *)o.in[1] + v0 * o.pitch[1];
            Operand table{rows, o.pitch[1], n, o.cols, 0, false};
            if (!table_well) {
                e = launch_pack<T>(rows, o.pitch[1], n, o.cols, room + at.table, room + at.odd_table, Scaled{}, sm_count, stream);
                if (e != cudaSuccess) return e;
                table = packed_operand<T>(room + at.table, n, o.cols, false);
                ++*launched;
            }
            a.n = (uint32_t)n;
            a.first = (uint32_t)v0;
            plain_args(o, a, tokens, room + at.odd_x, room + at.odd_table, rows);
            const Cut cut = n == o.vocabulary && m == o.rows ? cut_of_scores(m, n, o.cols, o.dtype, sm_count, 32) : Cut(m, n, sm_count, 32);
            if (cut.splits > 1) {
                a.out = room + at.scores;
                a.wide = width_of(a.out, n, 4);
                e = launch_product<false, false, TO_SCORES, (int)parts_of<T>()>(x, table, a, cut, sm_count, stream);
                *launched += 2;
                return e != cudaSuccess ? e
                                        : launch_pdl(lt_loss_finish<false, (int)parts_of<T>()>, a.m, 256, (size_t)0, stream, a, (const float *)a.out, cut.splits, (float *)o.out[0], (float *)o.out[1]);
            }
            e = launch_product<false, false, TO_LOSS, (int)parts_of<T>()>(x, table, a, cut, sm_count, stream);
            if (e != cudaSuccess) return e;
            a.first_tile += 2 * cut.tiles_n;
            ++*launched;
        }
        ++*launched;
        e = launch_join(a, a.first_tile, o.out[0] ? (float *)o.out[0] + r0 : nullptr, o.out[1] ? (float *)o.out[1] + r0 : nullptr, stream);
        if (e != cudaSuccess) return e;
    }
    return e;
}

template <class T>
cudaError_t launch_sum(const float *sums, void *out, uint64_t count, uint32_t splits, int sm_count, cudaStream_t stream) {
    const bool wide = count % 4 == 0 && is_aligned(out, 4 * sizeof(T));
    const unsigned grid = (unsigned)std::min<uint64_t>((count / (wide ? 4 : 1) + 255) / 256, (uint64_t)sm_count * 16);
    return wide ? launch_pdl(lt_loss_sum<T, 4>, grid, 256, (size_t)0, stream, sums, (T *)out, count, splits)
                : launch_pdl(lt_loss_sum<T, 1>, grid, 256, (size_t)0, stream, sums, (T *)out, count, splits);
}

template <class T, int N, int TOKENS>
cudaError_t launch_few_grad_of(const FewGradArgs &a, const FewGrad &few, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(lt_loss_few_grad<T, N, TOKENS>, TOKENS * FEW_GRAD_THREADS * FEW_GRAD_COLS * sizeof(T), ready);
    return e != cudaSuccess ? e : launch_pdl_shared(lt_loss_few_grad<T, N, TOKENS>, dim3(few.blocks), few.threads, (size_t)TOKENS * up_to(a.cols, 8) * sizeof(T), stream, a);
}
template <class T, int N>
cudaError_t launch_few_grad_of(const FewGradArgs &a, const FewGrad &few, cudaStream_t stream) {
    if constexpr (sizeof(T) == 4) {
        if (few.at_once == 8) return launch_few_grad_of<T, N, 8>(a, few, stream);
        if (few.at_once == 4) return launch_few_grad_of<T, N, 4>(a, few, stream);
    }
    return few.at_once == 1 ? launch_few_grad_of<T, N, 1>(a, few, stream) : launch_few_grad_of<T, N, 2>(a, few, stream);
}
template <class T>
cudaError_t launch_few_grad(const LtOperator &o, const FewGrad &few, cudaStream_t stream, unsigned *launched) {
    constexpr int N = 16 / (int)sizeof(T);
    const bool wide = o.cols % N == 0 && o.pitch[1] % N == 0 && is_aligned(o.in[1], 16) && is_aligned(o.out[1], 16);
    const float scale = (float)lt_attr_double(o.attr[1]);
    cudaError_t e = cudaSuccess;
    *launched = 0;
    for (uint64_t r0 = 0; r0 < o.rows && e == cudaSuccess; r0 += few.at_once) {
        const uint32_t tokens = (uint32_t)std::min<uint64_t>(few.at_once, o.rows - r0);
        const FewGradArgs a{(const T *)o.in[0] + r0 * o.pitch[0], o.in[1], (const int *)o.in[2] + r0, (const float *)o.in[3] + r0, (const float *)o.in[4] + r0, o.out[1], o.out[0] ? (float *)o.scratch : nullptr,
                            o.pitch[0], o.pitch[1], tokens, (uint32_t)o.vocabulary, (uint32_t)o.cols, scale, (float)(lt_attr_double(o.attr[1]) * 1.4426950408889634), r0 > 0, &o.status->loss};
        e = wide ? launch_few_grad_of<T, N>(a, few, stream) : launch_few_grad_of<T, 1>(a, few, stream);
        ++*launched;
        if (e != cudaSuccess || !o.out[0]) continue;
        e = launch_pdl(lt_loss_few_join<T>, count_of((uint64_t)tokens * o.cols, 32), 256, (size_t)0, stream, (const float *)a.dx, (T *)o.out[0] + r0 * o.cols, a.targets, a.dloss, scale, tokens, a.cols, few.blocks,
                       a.vocabulary);
        ++*launched;
    }
    return e;
}

template <class T>
cudaError_t launch_loss_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    const FewGrad few(o, sm_count);
    if (few.at_once) return launch_few_grad<T>(o, few, stream, launched);
    constexpr int PARTS = parts_of<T>();
    constexpr int TO_T = sizeof(T) == 4 ? TO_F32 : TO_BF16;
    const GradScratch at(o, sm_count);
    char *room = (char *)o.scratch;
    const bool table_well = lies_well(o.dtype, o.in[1], o.pitch[1]);
    const uint64_t parts = parts_of<T>();
    float *factors = (float *)(room + at.factors), *unit = (float *)(room + at.unit);
    // (x is scaled and rows without a target, which may hold anything, left out for the gradient of the table alone)
    const bool x_well = lies_well(o.dtype, o.in[0], o.pitch[0]) && o.rows >= LEAST_ROWS;
    Scaled scaled{room + at.scaled, (const int *)o.in[2], (const float *)o.in[4], factors, unit, (float)lt_attr_double(o.attr[1]), (uint32_t)o.vocabulary, &o.status->loss};
    cudaError_t e = cudaSuccess;
    *launched = 1;
    if (o.rows > LARGEST_ALONE) {
        float *largest = (float *)(room + at.largest);
        scaled.largest = largest;
        e = launch_pdl(lt_loss_largest, LARGEST_BLOCKS, 256, (size_t)0, stream, scaled.dloss, scaled.targets, largest, (uint32_t)o.rows, scaled.vocabulary);
        if (e != cudaSuccess) return e;
        ++*launched;
    }
    // (an x that does not lie well is packed as a whole here, or piece by piece for its scores)
    const uint64_t x_piece = x_well ? o.rows : at.x_piece;
    const bool x_whole = x_piece == o.rows;
    e = launch_pack<T>(o.in[0], o.pitch[0], o.rows, o.cols, x_well || !x_whole ? nullptr : room + at.x, room + at.odd_x, scaled, sm_count, stream);
    const uint64_t piece = table_well ? at.piece : at.packed_piece;
    for (uint64_t v0 = 0; v0 < o.vocabulary && e == cudaSuccess; v0 += piece) {
        const uint64_t n = std::min(piece, o.vocabulary - v0), padded = up_to(n, WIDTH);
        const bool last = v0 + n == o.vocabulary;
        const void *rows = (const T *)o.in[1] + v0 * o.pitch[1];
        Operand table{rows, o.pitch[1], n, o.cols, 0, false};
        if (!table_well) {
            e = launch_pack<T>(rows, o.pitch[1], n, o.cols, room + at.table, room + at.odd_table, Scaled{}, sm_count, stream);
            if (e != cudaSuccess) return e;
            table = packed_operand<T>(room + at.table, n, o.cols, false);
            ++*launched;
        }
        ProductArgs a{};
        common_args(o, a);
        a.m = (uint32_t)o.rows;
        a.n = (uint32_t)n;
        a.blocks_k = count_of(o.cols, DEPTH);
        a.first = (uint32_t)v0;
        a.lse = (const float *)o.in[3];
        a.p = (__nv_bfloat16 *)(room + at.p);
        a.p_pitch = padded * parts;
        a.p_part = (uint32_t)padded;
        a.p_rows = (uint32_t)std::max<uint64_t>(o.rows, LEAST_ROWS);
        plain_args(o, a, o.in[0], room + at.odd_x, room + at.odd_table, rows);
        for (uint64_t r0 = 0; r0 < o.rows; r0 += x_piece) {
            const uint64_t m = std::min(x_piece, o.rows - r0);
            const T *tokens = (const T *)o.in[0] + r0 * o.pitch[0];
            Operand x{tokens, o.pitch[0], m, o.cols, 0, false};
            if (!x_well) {
                if (!x_whole) {
                    e = launch_pack<T>(tokens, o.pitch[0], m, o.cols, room + at.x, room + at.odd_x, Scaled{}, sm_count, stream);
                    if (e != cudaSuccess) return e;
                    ++*launched;
                }
                x = packed_operand<T>(room + at.x, m, o.cols, false);
            }
            ProductArgs s = a;
            s.m = (uint32_t)m;
            s.targets += r0;
            s.lse += r0;
            s.p += r0 * s.p_pitch;
            s.p_rows = x_whole ? a.p_rows : (uint32_t)m;
            const Cut of_scores = n == o.vocabulary && x_whole ? cut_of_scores(m, n, o.cols, o.dtype, sm_count, 64) : Cut(m, n, sm_count, 64);
            if (of_scores.splits > 1) {
                s.out = room + at.scores;
                s.wide = width_of(s.out, n, 4);
                e = launch_product<false, false, TO_SCORES, PARTS>(x, table, s, of_scores, sm_count, stream);
                if (e == cudaSuccess) e = launch_pdl(lt_loss_finish<true, PARTS>, s.p_rows, 256, (size_t)0, stream, s, (const float *)s.out, of_scores.splits, (float *)nullptr, (float *)nullptr);
                ++*launched;
            } else {
                e = launch_product<false, false, TO_P, PARTS>(x, table, s, of_scores, sm_count, stream);
            }
            if (e != cudaSuccess) return e;
            ++*launched;
        }
        Operand p{a.p, padded * parts, a.p_rows, padded * parts, (uint32_t)padded, false};
        if (o.out[0]) {
            ProductArgs d{};
            common_args(o, d);
            d.m = (uint32_t)o.rows;
            d.n = (uint32_t)o.cols;
            d.blocks_k = count_of(n, DEPTH);
            d.factors = factors;
            // (as many splits for every piece, the last and shorter one too)
            const Cut cut = Cut(o.rows, o.cols, sm_count, 0).split(count_of(piece, DEPTH) * (parts == 1 ? 1 : 6), sm_count);
            float *sum = (float *)(room + at.sum_x);
            table.turned = true;
            if (last && cut.splits == 1) {
                d.before = v0 ? sum : nullptr;
                d.out = o.out[0];
                d.wide = width_of(d.out, o.cols, sizeof(T));
                e = launch_product<false, true, TO_T, PARTS>(p, table, d, cut, sm_count, stream);
            } else {
                d.before = v0 ? sum : nullptr;
                d.out = sum;
                d.wide = width_of(d.out, o.cols, 4);
                e = launch_product<false, true, TO_SUM, PARTS>(p, table, d, cut, sm_count, stream);
                if (e == cudaSuccess && last) {
                    e = launch_sum<T>(sum, o.out[0], o.rows * o.cols, cut.splits, sm_count, stream);
                    ++*launched;
                }
            }
            if (e != cudaSuccess) return e;
            ++*launched;
        }
        if (o.out[1]) {
            ProductArgs d{};
            common_args(o, d);
            d.m = (uint32_t)n;
            d.n = (uint32_t)o.cols;
            d.blocks_k = count_of(o.rows, DEPTH);
            d.unit = unit;
            Cut cut = Cut(n, o.cols, sm_count, 0).split(d.blocks_k * (parts == 1 ? 1 : 6), sm_count);
            cut.splits = std::min(cut.splits, at.splits_table);  // (the last piece is shorter: what the scratch memory holds)
            void *out = (T *)o.out[1] + v0 * o.cols;
            p.turned = true;
            const Operand scaled_x = packed_operand<T>(room + at.scaled, o.rows, o.cols, true);
            if (cut.splits == 1) {
                d.out = out;
                d.wide = width_of(out, o.cols, sizeof(T));
                e = launch_product<true, true, TO_T, PARTS>(p, scaled_x, d, cut, sm_count, stream);
            } else {
                d.out = room + at.sum_table;
                d.wide = width_of(d.out, o.cols, 4);
                e = launch_product<true, true, TO_SUM, PARTS>(p, scaled_x, d, cut, sm_count, stream);
                if (e == cudaSuccess) e = launch_sum<T>((const float *)d.out, out, n * o.cols, cut.splits, sm_count, stream);
                ++*launched;
            }
            if (e != cudaSuccess) return e;
            ++*launched;
        }
    }
    return e;
}

// The bounded wait of lt_product on a barrier that nobody arrives at, with no copy or product on its way.  The first warp's
// limit is `limit_ns`, the second's fifty times that: it ends when the first gives up.
__global__ void lt_product_wait_probe(unsigned int *timeout, uint64_t limit_ns) {
    __shared__ __align__(8) uint64_t barriers[2];
    __shared__ uint32_t gave_up;
    const uint32_t arrived = shared_address(&barriers[0]), never = shared_address(&barriers[1]);
    if (threadIdx.x == 0) {
        gave_up = 0;
        barrier_init(arrived, 1);
        barrier_init(never, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        barrier_arrive_at(arrived);
    }
    __syncthreads();
    const Waits waits{&gave_up, timeout, warp_number() ? 50 * limit_ns : limit_ns};
    if (waits.wait(arrived, 0)) waits.wait(never, 0);
}

}  // namespace

cudaError_t lt_launch_product_wait_probe(LtOperatorStatus *status, uint64_t limit_ns, cudaStream_t stream) {
    lt_product_wait_probe<<<1, 64, 0, stream>>>(&status->timeout, limit_ns);
    return cudaGetLastError();
}

size_t lt_vocabulary_loss_scratch(const LtOperator &o, int sm_count) { return LossScratch(o, sm_count).bytes; }
size_t lt_vocabulary_loss_grad_scratch(const LtOperator &o, int sm_count) { return GradScratch(o, sm_count).bytes; }

cudaError_t lt_launch_vocabulary_loss(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    return o.dtype == LT_BF16 ? launch_loss<__nv_bfloat16>(o, sm_count, stream, launched) : launch_loss<float>(o, sm_count, stream, launched);
}

cudaError_t lt_launch_vocabulary_loss_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    return o.dtype == LT_BF16 ? launch_loss_grad<__nv_bfloat16>(o, sm_count, stream, launched) : launch_loss_grad<float>(o, sm_count, stream, launched);
}
