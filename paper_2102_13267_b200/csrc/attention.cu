// Attention of one query token per sequence over a paged key-value cache.
//
// For each sequence and query head: out = sum_i w_i v_i / sum_i w_i with w_i = exp(scale q k_i - m), m the running
// maximum.  A block works on up to 8 (f32, and any type without 16-byte alignment), 16 (bf16 heads of more than 128 values)
// or 32 (bf16) of the query heads that share a key, and reads its keys and values once for them; more of them are several
// head blocks, each of which reads the cache.  Nothing else of size is read or written, so up to there the bound is the
// cache's bytes over the memory's rate.
//
// Work split: the tokens of all sequences are cut into tiles of TILE; the list of (sequence, head block, tile) is divided
// evenly over the thread blocks, whatever the sequences' lengths (which only the device knows).  Every (sequence, head
// block) counts START tiles more than it has, for what beginning one costs.  A block walks its part of the list; a
// (sequence, head block) that lies within one block's part is finished there.  One that is spread over several leaves
// partial results (maximum, sum, unnormalised output) in scratch memory, and the block that arrives last joins them,
// always in the list's order, so results do not depend on the arrival.
//
// The kernels let the next one on the stream begin late, when their own work is done: blocks that wait beside them for
// their end cost more than an early launch gains (one sequence of 1013 tokens, 8 key heads of 128 values: 7.8 us against
// 9.3; four of 7001 to 32768: 61.5 against 62.7).
#include <algorithm>

#include "operator_device.cuh"

using namespace ltop;

namespace {

constexpr int TILE = 64;         // tokens
constexpr int START = 2;         // tiles that beginning a (sequence, head block) counts for
constexpr int THREADS = 128;
constexpr int WARPS = THREADS / 32;
constexpr uint32_t JOIN = 32;    // parts that are joined at once: a lane each
constexpr uint32_t GROUP = 16;   // more are joined in groups of as many, and then the groups
constexpr uint32_t MOST_PARTS = GROUP * JOIN;  // blocks that one (sequence, head block) is spread over

struct AttendArgs {
    const void *q, *cache;
    const int *table, *lengths;
    void *out;
    float *partial;             // [2 x blocks][block_heads][dim + 2]: outputs, then (maximum, sum) of each head; null: every (sequence, head block) has a block of its own
    unsigned int *arrivals;     // [2][LT_ARRIVALS / 2], zero between launches: how many groups (or all parts) of what begins in block i are there; and how many parts of its groups (i, i + 1, ..)
    unsigned int *status;       // set to 1 (by whoever finds it) where an index lies outside what it indexes
    uint64_t q_pitch, page_stride, value_offset, token_stride, head_stride;
    uint32_t batch, heads, kv_heads, group, block_heads, head_blocks, dim, pages, page, table_width;  // block_heads: query heads a block works on at a time
    float scale;                // times log2(e): weights are powers of two
};

__device__ __forceinline__ int length_of(const AttendArgs &a, uint32_t b) {
    const int n = a.lengths[b];
    const int64_t most = (int64_t)a.table_width * a.page;
    return n < 0 ? 0 : (int64_t)n > most ? (int)most : n;
}

__device__ __forceinline__ void check_length(const AttendArgs &a, uint32_t b) {
    if (threadIdx.x == 0 && a.lengths[b] > 0 && (int64_t)a.lengths[b] > (int64_t)a.table_width * a.page) report(a.status);
}

__device__ __forceinline__ uint32_t tiles_in(int n) { return ((uint32_t)n + TILE - 1) / TILE; }

__device__ __forceinline__ uint32_t items_of(int n) { return n ? tiles_in(n) + START : 0; }

// What a block works on: items [idx, end) of the list.
struct Share {
    uint32_t idx, end, size;    // size: of a share
    uint32_t b, base;           // the sequence it is in, and where that begins in the list
    int n;                      // its length
};

// The block's part of the list, from the sequences' lengths.  Every warp finds it for itself, without a barrier: the lanes
// have a run of sequences each, whose sums are added up across lanes; the run that holds the block's first item is divided
// among the lanes again, until it is one sequence.
__device__ __forceinline__ Share my_share(const AttendArgs &a) {
    const uint32_t per = a.kv_heads * a.head_blocks, lane = threadIdx.x & 31;
    Share s{};
    if (!a.partial) {  // a block per (sequence, head block)
        s.b = blockIdx.x / per;
        s.n = length_of(a, s.b);
        const uint32_t t = items_of(s.n);
        s.idx = (blockIdx.x - s.b * per) * t;
        s.end = s.idx + t;
        return s;
    }
    for (uint32_t count = a.batch; ; ) {
        const uint32_t run = (count + 31) / 32, b0 = s.b + lane * run, b1 = s.b + min(count, (lane + 1) * run);
        uint32_t mine = 0, most = 0;
        int n = 0;
#pragma unroll 8
        for (uint32_t b = b0; b < b1; ++b) {
            n = length_of(a, b);
            mine += items_of(n);
            most = max(most, items_of(n));
        }
        mine *= per;
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= (uint32_t)d) upto += o;
        }
        if (s.size == 0) {  // all sequences: an even share, and no (sequence, head block) over more than MOST_PARTS blocks
            const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
            most = __reduce_max_sync(0xffffffffu, most);
            s.size = max(max((total + gridDim.x - 1) / gridDim.x, (most + MOST_PARTS - 2) / (MOST_PARTS - 1)), 1u);
            s.idx = min(blockIdx.x * s.size, total);
            s.end = min(s.idx + s.size, total);
            if (s.idx == s.end) return s;
        }
        const uint32_t base = s.base + upto - mine;
        const uint32_t holder = __ffs(__ballot_sync(0xffffffffu, s.idx >= base && s.idx < base + mine)) - 1;
        s.base = __shfl_sync(0xffffffffu, base, holder);
        s.n = __shfl_sync(0xffffffffu, n, holder);
        s.b += holder * run;
        if (run == 1) return s;
        count = min(run, count - holder * run);
    }
}

// A stretch of tiles of one (sequence, head block).
struct Stretch {
    uint32_t first;             // of the (sequence, head block) in the list
    uint32_t b, kv, h0;         // h0: first query head
    int n, heads;               // tokens of the sequence, query heads
    uint32_t t0, t1, tiles;     // tiles: of the sequence
    uint32_t items;             // of the list
};

// The next stretch of the share, or false when it is done; `done`: items of the one before.
__device__ __forceinline__ bool next_stretch(const AttendArgs &a, Share &s, Stretch &w, uint32_t done) {
    const uint32_t per = a.kv_heads * a.head_blocks;
    for (;;) {
        s.idx += done;
        if (s.idx >= s.end) return false;
        while (s.idx >= s.base + items_of(s.n) * per) {
            s.base += items_of(s.n) * per;
            s.n = length_of(a, ++s.b);
        }
        const uint32_t all = items_of(s.n), hb = (s.idx - s.base) / all;
        w.tiles = all - START;
        w.first = s.base + hb * all;
        const uint32_t v0 = s.idx - w.first, v1 = min(all, v0 + (s.end - s.idx));
        done = w.items = v1 - v0;
        w.t0 = max(v0, (uint32_t)START) - START;
        w.t1 = max(v1, (uint32_t)START) - START;
        if (w.t1 == w.t0) continue;  // only of what beginning counts for
        w.b = s.b;
        w.n = s.n;
        w.kv = a.head_blocks == 1 ? hb : hb / a.head_blocks;
        const uint32_t first = (hb - w.kv * a.head_blocks) * a.block_heads;
        w.h0 = w.kv * a.group + first;
        w.heads = (int)min(a.block_heads, a.group - first);
        return true;
    }
}

__device__ __forceinline__ float quotient(float o, float l) { return l > 0.f ? o / l : l == 0.f ? 0.f : l; }

// Where a block leaves its parts: of the first or the second stretch that it does not finish.
// (an even number of heads each, so that parts of four-value rows start on 16 bytes)
__host__ __device__ constexpr int part_heads(int heads) { return heads + (heads & 1); }
__device__ __forceinline__ uint64_t part_floats(const AttendArgs &a) { return (uint64_t)part_heads((int)a.block_heads) * (a.dim + 2); }
__device__ __forceinline__ float *part_of(const AttendArgs &a, uint32_t block, bool second) { return a.partial + (2 * (uint64_t)block + (second ? 1 : 0)) * part_floats(a); }

// The parts of a stretch's (sequence, head block), in order.
struct Parts {
    const float *head, *rest;   // the first part; where the others are `stride` apart, from the second on
    uint32_t count;
    uint64_t stride;
    __device__ __forceinline__ const float *at(uint32_t i) const { return i ? rest + (i - 1) * stride : head; }
};

// One more of `count` has arrived; true if that was the last.  What the block wrote before is then seen by whoever that is.
__device__ __forceinline__ bool last_arrival(unsigned int *arrived, uint32_t count, uint32_t *flag) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *flag = atomicAdd(arrived, 1u) == count - 1;
        __threadfence();
    }
    __syncthreads();
    const bool last = *flag != 0;
    if (last && threadIdx.x == 0) *arrived = 0;
    return last;
}

// The block has left its part of stretch w.  Joins the parts if it was the last one of the (sequence, head block).  Many
// parts are joined in two steps, groups first, so that several blocks work on them (one sequence of 100000 tokens with one
// key head of 128 values, bf16: 24 us over all blocks, 44 over up to 64 or 256 whose parts are joined at once).
// join(parts, to): into the result, or (`to` not null) into one part.
template <class F>
__device__ __forceinline__ void leave_part(const AttendArgs &a, const Share &s, const Stretch &w, uint32_t *flag, F join) {
    const uint32_t i0 = w.first + START, c0 = i0 / s.size, c1 = (i0 + w.tiles - 1) / s.size;
    Parts p;
    p.count = c1 - c0 + 1;
    p.stride = 2 * part_floats(a);
    p.head = part_of(a, c0, c0 * s.size < w.first);
    p.rest = part_of(a, c0 + 1, false);
    if (p.count > JOIN) {
        const uint32_t g = (blockIdx.x - c0) / GROUP;
        Parts some;
        some.count = min(GROUP, p.count - g * GROUP);
        some.stride = p.stride;
        some.head = p.at(g * GROUP);
        some.rest = p.at(g * GROUP + 1);
        if (!last_arrival(a.arrivals + LT_ARRIVALS / 2 + c0 + g, some.count, flag)) return;
        join(some, const_cast<float *>(some.head));
        p.count = (p.count + GROUP - 1) / GROUP;
        p.rest = p.at(GROUP);
        p.stride *= GROUP;
    }
    if (last_arrival(a.arrivals + c0, p.count, flag)) join(p, nullptr);
}

// The parts' weights 2^(maximum - largest maximum) and, of each head, in `sums` the largest maximum and the weighted sum of
// their sums: a warp per head, a lane per part.
__device__ __forceinline__ void weigh_parts(const AttendArgs &a, const Stretch &w, const Parts &p, float *weights, float2 *sums) {
    const uint32_t lane = threadIdx.x & 31;
    for (int h = threadIdx.x >> 5; h < w.heads; h += WARPS) {
        const float *ml = p.at(lane) + a.block_heads * a.dim + 2 * h;
        const float m = lane < p.count ? __ldcg(ml) : -INFINITY, l = lane < p.count ? __ldcg(ml + 1) : 0.f;
        float top = m;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float f = exp2f(m - (top == -INFINITY ? 0.f : top));
        weights[h * JOIN + lane] = f;
        const float sum = warp_sum(f * l);
        if (lane == 0) sums[h] = make_float2(top, sum);
    }
}

// Joins parts, one value at a time (any head size).  `room`: shared, block_heads x JOIN values.
template <class T>
__device__ __forceinline__ void join_any(const AttendArgs &a, const Stretch &w, const Parts &p, float *to, float *room, float2 *sums) {
    const uint32_t dim = a.dim;
    weigh_parts(a, w, p, room, sums);
    __syncthreads();
    for (uint32_t x = threadIdx.x; x < (uint32_t)w.heads * dim; x += THREADS) {
        const uint32_t h = x / dim, d = x - h * dim;
        float o = 0.f;
#pragma unroll 8
        for (uint32_t i = 0; i < p.count; ++i) o += room[h * JOIN + i] * __ldcg(p.at(i) + h * dim + d);
        if (to) to[x] = o;
        else ((T *)a.out)[((uint64_t)w.b * a.heads + w.h0 + h) * dim + d] = from_float<T>(quotient(o, sums[h].y));
    }
    if (to && threadIdx.x < w.heads) {
        to[a.block_heads * dim + 2 * threadIdx.x] = sums[threadIdx.x].x;
        to[a.block_heads * dim + 2 * threadIdx.x + 1] = sums[threadIdx.x].y;
    }
    __syncthreads();  // `room` is used again
}

template <class T>
__device__ __forceinline__ void store4(T *to, const float4 &v);
template <>
__device__ __forceinline__ void store4<float>(float *to, const float4 &v) { *reinterpret_cast<float4 *>(to) = v; }
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *to, const float4 &v) { *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)); }

// Joins parts, four values at a time: as many parts as fit are brought into shared memory at once, while the weights are
// found (one trip to L2 for both, instead of one for the maxima and one for every few parts after them).
// `mem`: `bytes` of shared memory; a.dim a multiple of 4; HEADS x WIDTH values at most.
template <class T, int HEADS, int WIDTH>
__device__ __forceinline__ void join_staged(const AttendArgs &a, const Stretch &w, const Parts &p, float *to, float *mem, uint32_t bytes) {
    constexpr int MINE = (HEADS * WIDTH / 4 + THREADS - 1) / THREADS;  // groups of four values of a thread
    const uint32_t dim = a.dim, quads = (uint32_t)w.heads * dim / 4;
    float *weights = mem;                                             // [HEADS][JOIN]
    float2 *sums = reinterpret_cast<float2 *>(weights + HEADS * JOIN);
    constexpr int PADDED = (HEADS + 1) / 2 * 2;
    float4 *staged = reinterpret_cast<float4 *>(sums + PADDED);
    const uint32_t room = (bytes - (HEADS * JOIN + 2 * PADDED) * 4) / (quads * 16);
    float4 acc[MINE];
#pragma unroll
    for (int k = 0; k < MINE; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (uint32_t i0 = 0; i0 < p.count; i0 += room) {
        const uint32_t n = min(room, p.count - i0);
        if (i0) __syncthreads();  // the parts before have been read
        for (uint32_t x = threadIdx.x; x < quads; x += THREADS) {
            uint32_t at = shared_address(staged + x), i = 0;
            if (i0 == 0) {
                copy16(at, p.head + 4 * x, true);
                at += quads * 16;
                i = 1;
            }
            const float *from = p.rest + (i0 + i - 1) * p.stride + 4 * x;
#pragma unroll 4
            for (; i < n; ++i) {
                copy16(at, from, true);
                at += quads * 16;
                from += p.stride;
            }
        }
        copy_commit();
        if (i0 == 0) weigh_parts(a, w, p, weights, sums);
        copy_wait<0>();
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t x = threadIdx.x + k * THREADS;
            if (x >= quads) continue;
            const float *f = weights + (4 * x / dim) * JOIN + i0;
            const float4 *from = staged + x;
            float4 v = acc[k];
#pragma unroll 4
            for (uint32_t i = 0; i < n; ++i) {
                const float4 o = *from;
                v.x += f[i] * o.x;
                v.y += f[i] * o.y;
                v.z += f[i] * o.z;
                v.w += f[i] * o.w;
                from += quads;
            }
            acc[k] = v;
        }
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
        const uint32_t x = threadIdx.x + k * THREADS;
        if (x >= quads) continue;
        if (to) {
            reinterpret_cast<float4 *>(to)[x] = acc[k];
            continue;
        }
        const float l = sums[4 * x / dim].y;
        store4((T *)a.out + ((uint64_t)w.b * a.heads + w.h0) * dim + 4 * x, make_float4(quotient(acc[k].x, l), quotient(acc[k].y, l), quotient(acc[k].z, l), quotient(acc[k].w, l)));
    }
    if (to && threadIdx.x < w.heads) *reinterpret_cast<float2 *>(to + a.block_heads * dim + 2 * threadIdx.x) = sums[threadIdx.x];
}

// The zeros of empty sequences, and the check of the lengths.
template <class T>
__device__ __forceinline__ void finish(const AttendArgs &a) {
    if (!a.partial) {  // the block's own sequence
        const uint32_t per = a.kv_heads * a.head_blocks, b = blockIdx.x / per;
        check_length(a, b);
        if (length_of(a, b)) return;
        const uint32_t hb = blockIdx.x - b * per, kv = hb / a.head_blocks, first = (hb - kv * a.head_blocks) * a.block_heads;
        const uint32_t count = min(a.block_heads, a.group - first) * a.dim;
        T *out = (T *)a.out + ((uint64_t)b * a.heads + kv * a.group + first) * a.dim;
        for (uint32_t x = threadIdx.x; x < count; x += THREADS) out[x] = from_float<T>(0.f);
        return;
    }
    for (uint32_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        check_length(a, b);
        if (length_of(a, b)) continue;
        T *out = (T *)a.out + (uint64_t)b * a.heads * a.dim;
        for (uint32_t x = threadIdx.x; x < a.heads * a.dim; x += THREADS) out[x] = from_float<T>(0.f);
    }
}

// First element of token i's key in head `kv`; false where its page is no page of the cache.
__device__ __forceinline__ bool locate(const AttendArgs &a, const int *row, int i, uint32_t kv, uint64_t *at) {
    const uint32_t e = (uint32_t)i / a.page, off = (uint32_t)i - e * a.page;
    const int p = row[e];
    if ((uint32_t)p >= a.pages) {
        report(a.status);
        return false;
    }
    *at = (uint64_t)p * a.page_stride + (uint64_t)off * a.token_stride + (uint64_t)kv * a.head_stride;
    return true;
}

constexpr int ANY_HEADS = 8;    // block_heads of lt_attend_any

// Any alignment, either dtype: a warp per token, a lane has values lane, lane + 32, ..; NE = ceil(dim / 32) of them.
template <class T, int NE>
__global__ void __launch_bounds__(THREADS) lt_attend_any(const AttendArgs a) {
    constexpr int HEADS = ANY_HEADS;
    __shared__ uint32_t flag;
    __shared__ float sm_m[4][HEADS], sm_l[4][HEADS];
    __shared__ float2 sums[HEADS];
    __shared__ float sm_o[4][HEADS][NE * 32];
    static_assert(4 * NE * 32 >= (int)JOIN, "the parts' weights fit where the warps' outputs are");
    pdl_wait();
    const T *q = (const T *)a.q, *cache = (const T *)a.cache;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Share s = my_share(a);
    const uint32_t start = s.idx;
    Stretch w;
    for (uint32_t done = 0; next_stretch(a, s, w, done); done = w.items) {
        const int *row = a.table + (uint64_t)w.b * a.table_width;
        float qr[HEADS][NE], acc[HEADS][NE], m[HEADS], l[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const uint32_t d = lane + 32 * e;
                qr[h][e] = (h < w.heads && d < a.dim) ? to_float(q[(uint64_t)w.b * a.q_pitch + (uint64_t)(w.h0 + h) * a.dim + d]) * a.scale : 0.f;
                acc[h][e] = 0.f;
            }
        }
        const int last = min(w.n, (int)(w.t1 * TILE));
        for (int i = (int)(w.t0 * TILE) + warp; i < last; i += 4) {
            uint64_t at;
            if (!locate(a, row, i, w.kv, &at)) continue;
            float k[NE], v[NE];
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const uint32_t d = lane + 32 * e;
                k[e] = d < a.dim ? to_float(cache[at + d]) : 0.f;
                v[e] = d < a.dim ? to_float(cache[at + a.value_offset + d]) : 0.f;
            }
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                if (h >= w.heads) break;
                float sc = 0.f;
#pragma unroll
                for (int e = 0; e < NE; ++e) sc += qr[h][e] * k[e];
                sc = warp_sum(sc);
                const float mn = fmaxf(m[h], sc), base = mn == -INFINITY ? 0.f : mn;
                const float keep = exp2f(m[h] - base), p = exp2f(sc - base);
                m[h] = mn;
                l[h] = l[h] * keep + p;
#pragma unroll
                for (int e = 0; e < NE; ++e) acc[h][e] = acc[h][e] * keep + p * v[e];
            }
        }
        __syncthreads();  // the warps' shares may still be read from the stretch before
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            if (lane == 0) sm_m[warp][h] = m[h], sm_l[warp][h] = l[h];
#pragma unroll
            for (int e = 0; e < NE; ++e) sm_o[warp][h][lane + 32 * e] = acc[h][e];
        }
        __syncthreads();
        const bool whole = w.t0 == 0 && w.t1 == w.tiles;
        float *slot = whole ? nullptr : part_of(a, blockIdx.x, s.idx != start);
        for (int x = threadIdx.x; x < w.heads * (int)a.dim; x += THREADS) {
            const int h = x / (int)a.dim, d = x - h * (int)a.dim;
            float mm = -INFINITY;
            for (int k = 0; k < 4; ++k) mm = fmaxf(mm, sm_m[k][h]);
            const float base = mm == -INFINITY ? 0.f : mm;
            float ll = 0.f, oo = 0.f;
            for (int k = 0; k < 4; ++k) {
                const float f = exp2f(sm_m[k][h] - base);
                ll += sm_l[k][h] * f;
                oo += sm_o[k][h][d] * f;
            }
            if (whole) {
                ((T *)a.out)[((uint64_t)w.b * a.heads + w.h0 + h) * a.dim + d] = from_float<T>(quotient(oo, ll));
            } else {
                slot[h * a.dim + d] = oo;
                if (d == 0) slot[HEADS * a.dim + 2 * h] = mm, slot[HEADS * a.dim + 2 * h + 1] = ll;
            }
        }
        if (!whole) leave_part(a, s, w, &flag, [&](const Parts &p, float *to) { join_any<T>(a, w, p, to, &sm_o[0][0][0], sums); });
    }
    pdl_release();
    finish<T>(a);
}

// ------------------------------------------------------------------------------------------- on the matrix units

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t turned(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (2 ulp; a weight below 2^-126 of the largest counts nothing)
__device__ __forceinline__ float power2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr int STEP = 16;        // tokens a warp takes at a time: a quarter of a tile

// Sizes of the kernels for heads of up to DP values.  Rows of keys and values in shared memory are padded so that what is
// read at once falls into different banks: eight rows of a matrix (bf16), four tokens by two chunks (f32).
template <class T, int DP, int HEADS>
struct Shape {
    static constexpr int CHUNKS = DP * (int)sizeof(T) / 16;
    static constexpr int PITCH = DP * (int)sizeof(T) + (sizeof(T) == 4 ? 32 : 16);
    static constexpr int STAGE = 2 * STEP * PITCH;
    static constexpr int STAGES = sizeof(T) == 2 ? (DP == 256 ? 3 : 2) : DP == 64 && HEADS <= 4 ? 2 : 1;
    static constexpr int OUTPUTS = HEADS * (DP + 4) * 4;  // of a warp
    static constexpr int BYTES = WARPS * (STAGES * STAGE > OUTPUTS ? STAGES * STAGE : OUTPUTS);
};
// Resident blocks per SM: what the stages and the registers leave room for.  More blocks with fewer stages each carry more
// than the other way round, until the registers run short (us, bf16, 16 sequences of 2000 to 3000 tokens, 16 heads of 64:
// 36.4 with two stages and five blocks, 39.7 with three and four, 38.0 with two and six, 36.6 with one and six; 8 of them,
// 8 heads of 128: 21.3 with two and three, 23.4 with three and two, 21.9 with one and four; 8 heads of 192: 30.7 with two
// and two, 37.2 with three and one; f32, 28 of them, 8 key heads of 64 shared by 16 each: 106 with one and four, 134 with
// two and two; 28 of 300 to 500 tokens, 32 heads of 128: 64 with one and three, 84 with three and one).
__host__ __device__ constexpr int tensor_blocks(int width, int tiles) {
    return width <= 64 ? (tiles == 1 ? 5 : tiles == 2 ? 4 : 2) : width <= 128 ? (tiles == 1 ? 3 : 2) : width <= 192 ? 2 : 1;
}
__host__ __device__ constexpr int single_blocks(int width, int heads) { return width <= 64 ? (heads <= 4 ? 3 : 4) : width <= 128 ? 3 : width <= 192 ? 2 : 1; }

// A warp's copies of one stretch: steps of STEP tokens, every WARPS-th of the stretch's quarter tiles, into its stages.
//
// Page numbers are fetched ahead of the copies they address.  Where a step never crosses a page (WHOLE_STEPS) one number
// serves a step, and the lanes hold those of the next 32 steps; otherwise lane i has the number of token i.
template <class T, int DP, int HEADS, bool WHOLE_STEPS>
struct Stages {
    using S = Shape<T, DP, HEADS>;
    static constexpr int N = 16 / (int)sizeof(T);
    const AttendArgs &a;
    const Stretch &w;
    const int *row;
    unsigned char *mine;
    uint32_t at, *masks;        // shared address of the stages; which tokens of the step in a stage count
    int lane, first, steps, ahead;

    __device__ __forceinline__ Stages(const AttendArgs &a_, const Stretch &w_, unsigned char *mine_, uint32_t *masks_)
        : a(a_), w(w_), row(a_.table + (uint64_t)w_.b * a_.table_width), mine(mine_), at(shared_address(mine_)), masks(masks_), lane(threadIdx.x & 31),
          first((int)(w_.t0 * TILE) + (int)(threadIdx.x >> 5) * STEP), steps((int)(w_.t1 - w_.t0)), ahead(-1) {
        fetch_pages(0);
    }
    __device__ __forceinline__ void fetch_pages(int step) {
        const int i = WHOLE_STEPS ? first + (step + lane) * TILE : first + step * TILE + (lane & 15);
        ahead = i < w.n ? row[(uint32_t)i / a.page] : -2;
    }
    // columns from dim to DP stay zero (the memory is also used to join warps)
    __device__ __forceinline__ void clear_rest() {
        const int chunks = (int)a.dim / N, rest = S::CHUNKS - chunks;
        if (rest == 0) return;
        for (int x = lane; x < S::STAGES * 2 * STEP * rest; x += 32) {
            const int r = x / rest, c = x - r * rest;
            *reinterpret_cast<uint4 *>(mine + r * S::PITCH + (chunks + c) * 16) = make_uint4(0, 0, 0, 0);
        }
    }
    // The copies of a step, committed as one group (an empty one behind the last step).
    __device__ __forceinline__ void issue(int step) {
        const T *cache = (const T *)a.cache;
        const int chunks = (int)a.dim / N;
        if (step < steps) {
            const uint32_t to = at + (uint32_t)(step % S::STAGES) * S::STAGE;
            const int i0 = first + step * TILE, left = w.n - i0;
            uint32_t mask = left >= STEP ? 0xffffu : left <= 0 ? 0u : (1u << left) - 1u;
            if (WHOLE_STEPS) {
                if (step > 0 && (step & 31) == 0) fetch_pages(step);
                const int p = __shfl_sync(0xffffffffu, ahead, step & 31);
                if (mask && (uint32_t)p >= a.pages) {
                    mask = 0;
                    report(a.status);
                }
                const uint32_t off = (uint32_t)i0 % a.page;
                const T *src = cache + (mask ? (uint64_t)p * a.page_stride + (uint64_t)off * a.token_stride + (uint64_t)w.kv * a.head_stride : 0);
#pragma unroll
                for (int x = 0; x < STEP * S::CHUNKS; x += 32) {
                    const int r = (x + lane) / S::CHUNKS, c = (x + lane) % S::CHUNKS;
                    const bool there = (mask >> r) & 1u;
                    const T *from = there ? src + (uint64_t)r * a.token_stride + c * N : cache;
                    if (c < chunks) {
                        copy16(to + r * S::PITCH + c * 16, from, there);
                        copy16(to + (STEP + r) * S::PITCH + c * 16, there ? from + a.value_offset : cache, there);
                    }
                }
            } else {
                const int i = i0 + (lane & 15), p = ahead;
                const bool known = i < w.n && (uint32_t)p < a.pages;
                if (i < w.n && !known) report(a.status);
                mask = __ballot_sync(0xffffffffu, known) & 0xffffu;
                const uint64_t off = known ? (uint64_t)p * a.page_stride + (uint64_t)((uint32_t)i % a.page) * a.token_stride + (uint64_t)w.kv * a.head_stride : 0;
#pragma unroll
                for (int x = 0; x < STEP * S::CHUNKS; x += 32) {
                    const int r = (x + lane) / S::CHUNKS, c = (x + lane) % S::CHUNKS;
                    const uint64_t o = __shfl_sync(0xffffffffu, off, r);
                    const bool there = (mask >> r) & 1u;
                    const T *from = there ? cache + o + c * N : cache;
                    if (c < chunks) {
                        copy16(to + r * S::PITCH + c * 16, from, there);
                        copy16(to + (STEP + r) * S::PITCH + c * 16, there ? from + a.value_offset : cache, there);
                    }
                }
                if (step + 1 < steps) fetch_pages(step + 1);
            }
            if (lane == 0) masks[step % S::STAGES] = mask;
        }
        copy_commit();
    }
};

// Joins the warps' outputs in `sm_o` [WARPS][HEADS][DP + 4], with their maxima and sums, into the result or a part; then,
// if the block's part was the last one, the parts.
template <class T, int HEADS, int DP>
__device__ __forceinline__ void leave_stretch(const AttendArgs &a, const Share &s, const Stretch &w, bool first_stretch, float *sm_o, const float (*sm_m)[HEADS],
                                              const float (*sm_l)[HEADS], uint32_t bytes, uint32_t *flag) {
    const bool whole = w.t0 == 0 && w.t1 == w.tiles;
    float *slot = whole ? nullptr : part_of(a, blockIdx.x, !first_stretch);
    for (int x = threadIdx.x; x < w.heads * (int)(a.dim / 4); x += THREADS) {
        const int h = x / (int)(a.dim / 4), d = 4 * (x - h * (int)(a.dim / 4));
        float mm = -INFINITY;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) mm = fmaxf(mm, sm_m[k][h]);
        const float base = mm == -INFINITY ? 0.f : mm;
        float ll = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            const float f = exp2f(sm_m[k][h] - base);
            const float4 u = *reinterpret_cast<const float4 *>(sm_o + (k * HEADS + h) * (DP + 4) + d);
            ll += sm_l[k][h] * f;
            v.x += u.x * f;
            v.y += u.y * f;
            v.z += u.z * f;
            v.w += u.w * f;
        }
        if (whole) {
            store4((T *)a.out + ((uint64_t)w.b * a.heads + w.h0 + h) * a.dim + d, make_float4(quotient(v.x, ll), quotient(v.y, ll), quotient(v.z, ll), quotient(v.w, ll)));
        } else {
            *reinterpret_cast<float4 *>(slot + h * a.dim + d) = v;
            if (d == 0) *reinterpret_cast<float2 *>(slot + a.block_heads * a.dim + 2 * h) = make_float2(mm, ll);
        }
    }
    static_assert((HEADS * (JOIN + 3) + HEADS * DP) * 4 <= Shape<T, DP, HEADS>::BYTES, "the parts' weights and one part fit");
    if (!whole) leave_part(a, s, w, flag, [&](const Parts &p, float *to) { join_staged<T, HEADS, DP>(a, w, p, to, sm_o, bytes); });
    __syncthreads();  // the next stretch's copies go where the parts were
}

// f32, 16-byte aligned rows, head sizes filled up to DP with zeros; up to NH query heads per block.
//
// Full binary32 products rule the matrix units out (in two tf32 parts each, taking the numbers apart cost more than these
// products: 40 us against 32 on 16 sequences of 16 heads of 64 values), and memory is slow enough for the others.  Two
// lanes share a token's key, every other chunk each; the weights go through shared memory to all lanes, which have the
// output's values between them, two neighbouring ones of every 64.  Warps, stages and joins as in lt_attend_tensor.
// 28 sequences of 300 to 500 tokens, 32 heads of 128: 64 us, 5.7 TB/s.  With 16 query heads per key head the cache is read by
// two head blocks (28 of 1500 to 2000, 8 key heads of 64: 92 us, 2.2 TB/s of the cache's bytes counted once; 106 when each
// head's maximum was followed at once), and every four products of a head wait for 16 bytes of its query out of shared memory,
// with one stage that a warp cannot fill while it computes: a quarter of the products that the units could do.
template <int DP, int NH, bool WHOLE_STEPS>
__global__ void __launch_bounds__(THREADS, single_blocks(DP, NH)) lt_attend_single(const AttendArgs a) {
    using S = Shape<float, DP, NH>;
    constexpr int J = DP / 64;
    extern __shared__ __align__(128) unsigned char stage_mem[];
    __shared__ uint32_t flag;
    __shared__ float sm_m[WARPS][NH], sm_l[WARPS][NH];
    __shared__ uint32_t sm_mask[WARPS][S::STAGES];
    __shared__ __align__(16) float sm_p[WARPS][NH][STEP], sm_q[NH][DP];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, token = lane >> 1, half = lane & 1;
    unsigned char *mine = stage_mem + warp * S::STAGES * S::STAGE;
    pdl_wait();
    Share s = my_share(a);
    const uint32_t start = s.idx;
    Stretch w;
    for (uint32_t done = 0; next_stretch(a, s, w, done); done = w.items) {
        Stages<float, DP, NH, WHOLE_STEPS> stages(a, w, mine, sm_mask[warp]);
        for (int x = threadIdx.x; x < NH * DP; x += THREADS) {  // (the stretch before has ended with a barrier)
            const int h = x / DP, d = x % DP;
            sm_q[h][d] = h < w.heads && d < (int)a.dim ? ((const float *)a.q)[(uint64_t)w.b * a.q_pitch + (uint64_t)(w.h0 + h) * a.dim + d] * a.scale : 0.f;
        }
        stages.clear_rest();
        float o[NH][J][2], m[NH], l[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) o[h][j][0] = o[h][j][1] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < S::STAGES; ++k) stages.issue(k);
        __syncthreads();  // q is there
        for (int step = 0; step < stages.steps; ++step) {
            copy_wait<S::STAGES - 1>();
            __syncwarp();  // the step's copies of all lanes are there
            const uint32_t mask = stages.masks[step % S::STAGES];  // the tokens that count
            if (mask) {
                const unsigned char *stage = mine + (step % S::STAGES) * S::STAGE;
                float c[NH];
#pragma unroll
                for (int h = 0; h < NH; ++h) c[h] = 0.f;
                const float4 *key = reinterpret_cast<const float4 *>(stage + token * S::PITCH) + half;
                const float4 *query = reinterpret_cast<const float4 *>(&sm_q[0][0]) + half;
#pragma unroll 8
                for (int k = 0; k < DP / 8; ++k) {
                    const float4 x = key[2 * k];
#pragma unroll
                    for (int h = 0; h < NH; ++h) {
                        const float4 y = query[h * (DP / 4) + 2 * k];
                        c[h] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, c[h]))));
                    }
                }
                const bool in = (mask >> token) & 1u;
                float top[NH];
                bool larger = false;
#pragma unroll
                for (int h = 0; h < NH; ++h) {
                    const float v = c[h] + __shfl_xor_sync(0xffffffffu, c[h], 1);
                    top[h] = c[h] = in ? v : -INFINITY;
                }
#pragma unroll
                for (int d = 2; d < 32; d <<= 1)
#pragma unroll
                    for (int h = 0; h < NH; ++h) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], d));
#pragma unroll
                for (int h = 0; h < NH; ++h) larger |= top[h] > m[h];
                if (larger) {  // (the same in all lanes)
#pragma unroll
                    for (int h = 0; h < NH; ++h) {
                        const float n = fmaxf(m[h], top[h]), f = power2(m[h] - (n == -INFINITY ? 0.f : n));
                        m[h] = n;
                        l[h] *= f;
#pragma unroll
                        for (int j = 0; j < J; ++j) {
                            o[h][j][0] *= f;
                            o[h][j][1] *= f;
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < NH; ++h) {
                    const float p = power2(c[h] - (m[h] == -INFINITY ? 0.f : m[h]));
                    l[h] += p;  // (twice, once in each of the token's lanes)
                    if (half == 0) sm_p[warp][h][token] = p;
                }
                __syncwarp();
                const float2 *value = reinterpret_cast<const float2 *>(stage + STEP * S::PITCH) + lane;
#pragma unroll
                for (int t0 = 0; t0 < STEP; t0 += 4) {
                    float4 p[NH];
#pragma unroll
                    for (int h = 0; h < NH; ++h) p[h] = *reinterpret_cast<const float4 *>(&sm_p[warp][h][t0]);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int j = 0; j < J; ++j) {
                            const float2 v = value[(t0 + t) * (S::PITCH / 8) + j * 32];
#pragma unroll
                            for (int h = 0; h < NH; ++h) {
                                const float f = t == 0 ? p[h].x : t == 1 ? p[h].y : t == 2 ? p[h].z : p[h].w;
                                o[h][j][0] = fmaf(f, v.x, o[h][j][0]);
                                o[h][j][1] = fmaf(f, v.y, o[h][j][1]);
                            }
                        }
                }
            }
            __syncwarp();  // everybody is done with the stage, and with the weights
            stages.issue(step + S::STAGES);
        }
        copy_wait<0>();
        float *sm_o = reinterpret_cast<float *>(stage_mem);  // [WARPS][NH][DP + 4]
        __syncthreads();  // every warp is done with its stages
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const float sum = warp_sum(l[h]) * 0.5f;
            if (lane == 0) sm_m[warp][h] = m[h], sm_l[warp][h] = sum;
#pragma unroll
            for (int j = 0; j < J; ++j) *reinterpret_cast<float2 *>(sm_o + (warp * NH + h) * (DP + 4) + j * 64 + lane * 2) = make_float2(o[h][j][0], o[h][j][1]);
        }
        __syncthreads();
        leave_stretch<float, NH, DP>(a, s, w, s.idx == start, sm_o, sm_m, sm_l, S::BYTES, &flag);
    }
    pdl_release();
    finish<float>(a);
}

// bf16, 16-byte aligned rows, head sizes filled up to DP with zeros; NT x 8 query heads per block.
//
// The few query heads make the narrow side of the products: scores are K (16 tokens x dims) times q^T (dims x 8 heads),
// the output is V^T (16 dims x 16 tokens) times the weights (16 tokens x 8 heads), so no matrix row is wasted on
// padding of the group to 16.  The weights leave the first product with tokens along the rows and enter the second with
// tokens along the columns of a register's pair: movmatrix turns them, as two bf16 parts (p and what its rounding left), which keeps
// the weights to 2^-17 and costs one more product.  Each warp has steps and a copy pipeline of its own -- no barrier
// in the loop -- and its own running maximum and sum; warps are joined once per stretch.  64 sequences of 17 to 4096
// tokens, 32 heads on 8 key heads of 128: 95 us, 5.7 TB/s; issue slots are 34 % busy, the tensor units 13 %, what is left is
// latency: beginning stretches, joining parts, and SMs that reach memory more slowly than others.
template <int DP, int NT, bool WHOLE_STEPS>
__global__ void __launch_bounds__(THREADS, tensor_blocks(DP, NT)) lt_attend_tensor(const AttendArgs a) {
    constexpr int HEADS = 8 * NT;
    using S = Shape<__nv_bfloat16, DP, HEADS>;
    constexpr int STAGES = S::STAGES, KS = DP / 16;
    extern __shared__ __align__(128) unsigned char stage_mem[];
    __shared__ uint32_t flag;
    __shared__ float sm_m[WARPS][HEADS], sm_l[WARPS][HEADS];
    __shared__ uint32_t sm_mask[WARPS][STAGES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, eighth = lane >> 2;
    unsigned char *mine = stage_mem + warp * STAGES * S::STAGE;
    const __nv_bfloat16 *q = (const __nv_bfloat16 *)a.q;
    pdl_wait();
    Share s = my_share(a);
    const uint32_t start = s.idx;
    Stretch w;
    for (uint32_t done = 0; next_stretch(a, s, w, done); done = w.items) {
        Stages<__nv_bfloat16, DP, HEADS, WHOLE_STEPS> stages(a, w, mine, sm_mask[warp]);
        uint32_t qf[NT][KS][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int h = t * 8 + eighth;
            const __nv_bfloat16 *from = q + (uint64_t)w.b * a.q_pitch + (uint64_t)(w.h0 + h) * a.dim;
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t d = k * 16 + i * 8 + quad * 2;
                    qf[t][k][i] = h < w.heads && d < a.dim ? *reinterpret_cast<const uint32_t *>(from + d) : 0u;
                }
        }
        stages.clear_rest();
        float o[NT][KS][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) o[t][k][0] = o[t][k][1] = o[t][k][2] = o[t][k][3] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) stages.issue(k);
        for (int step = 0; step < stages.steps; ++step) {
            copy_wait<STAGES - 2>();
            __syncwarp();  // the step's copies of all lanes are there, and everybody is done with the stage that the next ones fill
            const uint32_t mask = stages.masks[step % STAGES];  // the tokens that count
            stages.issue(step + STAGES - 1);
            if (mask == 0) continue;
            const uint32_t from = stages.at + (uint32_t)(step % STAGES) * S::STAGE;
            // scores, in two sums, so that a product does not wait for the one before it
            float c[NT][4], c2[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t][0] = c[t][1] = c[t][2] = c[t][3] = c2[t][0] = c2[t][1] = c2[t][2] = c2[t][3] = 0.f;
            const uint32_t ka = from + (lane & 15) * S::PITCH + (lane >> 4) * 16;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t f[4];
                load_matrices(f, ka + k * 32);
#pragma unroll
                for (int t = 0; t < NT; ++t) multiply(k & 1 ? c2[t] : c[t], f, qf[t][k][0], qf[t][k][1]);
            }
            const bool in0 = (mask >> eighth) & 1u, in1 = (mask >> (eighth + 8)) & 1u;
            uint32_t p_hi[NT][2], p_lo[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int j = 0; j < 4; ++j) c[t][j] = (j < 2 ? in0 : in1) ? (c[t][j] + c2[t][j]) * a.scale : -INFINITY;
                float top0 = fmaxf(c[t][0], c[t][2]), top1 = fmaxf(c[t][1], c[t][3]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, d));
                    top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, d));
                }
                if (__any_sync(0xffffffffu, top0 > m[t][0] || top1 > m[t][1])) {
                    const float n0 = fmaxf(m[t][0], top0), n1 = fmaxf(m[t][1], top1);
                    const float f0 = power2(m[t][0] - (n0 == -INFINITY ? 0.f : n0)), f1 = power2(m[t][1] - (n1 == -INFINITY ? 0.f : n1));
                    m[t][0] = n0;
                    m[t][1] = n1;
                    l[t][0] *= f0;
                    l[t][1] *= f1;
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        o[t][k][0] *= f0;
                        o[t][k][1] *= f1;
                        o[t][k][2] *= f0;
                        o[t][k][3] *= f1;
                    }
                }
                const float b0 = m[t][0] == -INFINITY ? 0.f : m[t][0], b1 = m[t][1] == -INFINITY ? 0.f : m[t][1];
                c[t][0] = power2(c[t][0] - b0);
                c[t][1] = power2(c[t][1] - b1);
                c[t][2] = power2(c[t][2] - b0);
                c[t][3] = power2(c[t][3] - b1);
                l[t][0] += c[t][0] + c[t][2];
                l[t][1] += c[t][1] + c[t][3];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = c[t][2 * i], y = c[t][2 * i + 1];
                    const uint32_t hi = pack_bf16(x, y);
                    const uint32_t lo = pack_bf16(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
                    p_hi[t][i] = turned(hi);
                    p_lo[t][i] = turned(lo);
                }
            }
            const uint32_t va = from + STEP * S::PITCH + ((lane & 7) + ((lane >> 4) & 1) * 8) * S::PITCH + ((lane >> 3) & 1) * 16;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t f[4];
                load_matrices_turned(f, va + k * 32);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    multiply(o[t][k], f, p_hi[t][0], p_hi[t][1]);
                    multiply(o[t][k], f, p_lo[t][0], p_lo[t][1]);
                }
            }
        }
        copy_wait<0>();
        float *sm_o = reinterpret_cast<float *>(stage_mem);  // [WARPS][HEADS][DP + 4]
        __syncthreads();  // every warp is done with its stages
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = t * 8 + quad * 2 + j;
                float sum = l[t][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane < 4) sm_m[warp][h] = m[t][j], sm_l[warp][h] = sum;
                float *to = sm_o + (warp * HEADS + h) * (DP + 4) + eighth;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    to[k * 16] = o[t][k][j];
                    to[k * 16 + 8] = o[t][k][2 + j];
                }
            }
        __syncthreads();
        leave_stretch<__nv_bfloat16, HEADS, DP>(a, s, w, s.idx == start, sm_o, sm_m, sm_l, S::BYTES, &flag);
    }
    pdl_release();
    finish<__nv_bfloat16>(a);
}

// A block of its own per (sequence, head block) when no sequence can hold more than a few tiles.
bool split(const LtOperator &o) { return (uint64_t)o.table_width * o.page > 2 * TILE; }

// lt_attend_tensor and lt_attend_single: widths they are built for (0: none), and query heads per block -- as many as share
// a key, while queries and output fit the registers.
int row_width(int dtype, uint32_t dim) {
    const int w = dim <= 64 ? 64 : dim <= 96 && dtype == LT_BF16 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256;
    return dim % (dtype == LT_BF16 ? 8 : 4) == 0 ? w : 0;
}
int row_heads(int dtype, int width, uint32_t group) {
    if (dtype == LT_F32) return group <= 1 ? 1 : group <= 2 ? 2 : group <= 4 ? 4 : 8;
    return group <= 8 ? 8 : group <= 16 || width > 128 ? 16 : 32;
}
int row_blocks(int dtype, int width, int heads) { return dtype == LT_F32 ? single_blocks(width, heads) : tensor_blocks(width, heads / 8); }
constexpr int ANY_BLOCKS = 4;  // resident blocks per SM of lt_attend_any

inline bool is_aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

template <class T>
cudaError_t launch_any(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    if (a.dim <= 64) return launch_pdl(lt_attend_any<T, 2>, grid, THREADS, (size_t)0, stream, a);
    if (a.dim <= 128) return launch_pdl(lt_attend_any<T, 4>, grid, THREADS, (size_t)0, stream, a);
    return launch_pdl(lt_attend_any<T, 8>, grid, THREADS, (size_t)0, stream, a);
}

template <int DP, int NT, bool WHOLE>
cudaError_t launch_tensor(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    constexpr size_t bytes = Shape<__nv_bfloat16, DP, 8 * NT>::BYTES;
    const cudaError_t e = allow_shared(lt_attend_tensor<DP, NT, WHOLE>, bytes, ready);
    if (e != cudaSuccess) return e;
    return launch_pdl(lt_attend_tensor<DP, NT, WHOLE>, grid, THREADS, bytes, stream, a);
}

template <int DP>
cudaError_t launch_tensor_heads(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    const bool whole = a.page % STEP == 0;
    if (a.block_heads == 8) return whole ? launch_tensor<DP, 1, true>(a, grid, stream) : launch_tensor<DP, 1, false>(a, grid, stream);
    if (a.block_heads == 16) return whole ? launch_tensor<DP, 2, true>(a, grid, stream) : launch_tensor<DP, 2, false>(a, grid, stream);
    if constexpr (DP <= 128)
        if (a.block_heads == 32) return whole ? launch_tensor<DP, 4, true>(a, grid, stream) : launch_tensor<DP, 4, false>(a, grid, stream);
    return cudaErrorInvalidValue;
}

template <int DP, int NH, bool WHOLE>
cudaError_t launch_single(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    constexpr size_t bytes = Shape<float, DP, NH>::BYTES;
    const cudaError_t e = allow_shared(lt_attend_single<DP, NH, WHOLE>, bytes, ready);
    if (e != cudaSuccess) return e;
    return launch_pdl(lt_attend_single<DP, NH, WHOLE>, grid, THREADS, bytes, stream, a);
}

template <int DP>
cudaError_t launch_single_heads(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    const bool whole = a.page % STEP == 0;
    switch (a.block_heads) {
    case 1: return whole ? launch_single<DP, 1, true>(a, grid, stream) : launch_single<DP, 1, false>(a, grid, stream);
    case 2: return whole ? launch_single<DP, 2, true>(a, grid, stream) : launch_single<DP, 2, false>(a, grid, stream);
    case 4: return whole ? launch_single<DP, 4, true>(a, grid, stream) : launch_single<DP, 4, false>(a, grid, stream);
    default: return whole ? launch_single<DP, 8, true>(a, grid, stream) : launch_single<DP, 8, false>(a, grid, stream);
    }
}

// blocks of a launch that splits sequences: what the SMs hold, and what the counters suffice for
unsigned split_blocks(int sm_count, int per_sm) {
    const unsigned n = (unsigned)sm_count * (unsigned)per_sm;
    return n < LT_ARRIVALS / 2 ? n : LT_ARRIVALS / 2;
}

}  // namespace

size_t lt_paged_attention_scratch(const LtOperator &o, int sm_count) {
    if (!split(o)) return 0;
    // (whether the addresses are aligned is not known yet: room for either kernel)
    const size_t any = (size_t)split_blocks(sm_count, ANY_BLOCKS) * ANY_HEADS;
    size_t rows = 0;
    if (const int width = row_width(o.dtype, o.dim)) {
        const int heads = row_heads(o.dtype, width, o.heads / o.kv_heads);
        rows = (size_t)split_blocks(sm_count, row_blocks(o.dtype, width, heads)) * part_heads(heads);
    }
    return 2 * (any > rows ? any : rows) * (o.dim + 2) * sizeof(float);
}

cudaError_t lt_launch_paged_attention(const LtOperator &o, int sm_count, cudaStream_t stream) {
    AttendArgs a{};
    a.q = o.in[0];
    a.cache = o.in[1];
    a.table = (const int *)o.in[2];
    a.lengths = (const int *)o.in[3];
    a.out = o.out[0];
    a.partial = split(o) ? (float *)o.scratch : nullptr;
    a.arrivals = (unsigned int *)o.arrivals;
    a.status = &o.status->attention;
    a.q_pitch = o.pitch[0];
    a.value_offset = (uint64_t)o.page * o.kv_heads * o.dim;
    a.page_stride = 2 * a.value_offset;
    a.token_stride = o.attr[0] ? o.dim : (uint64_t)o.kv_heads * o.dim;
    a.head_stride = o.attr[0] ? (uint64_t)o.page * o.dim : o.dim;
    a.batch = (uint32_t)o.rows;
    a.heads = o.heads;
    a.kv_heads = o.kv_heads;
    a.group = o.heads / o.kv_heads;
    a.dim = o.dim;
    a.pages = o.pages;
    a.page = o.page;
    a.table_width = o.table_width;
    a.scale = (float)(lt_attr_double(o.attr[1]) * 1.4426950408889634);
    const int width = row_width(o.dtype, o.dim);
    const bool rows = width && is_aligned(a.cache, 16) && is_aligned(a.q, 4) && (o.dtype == LT_F32 || a.q_pitch % 2 == 0) && is_aligned(a.out, 16);
    a.block_heads = rows ? row_heads(o.dtype, width, a.group) : ANY_HEADS;
    a.head_blocks = (a.group + a.block_heads - 1) / a.block_heads;
    unsigned grid = a.batch * a.kv_heads * a.head_blocks;
    if (a.partial) {  // (no more blocks than the page table has room for items)
        const uint64_t items = (uint64_t)grid * (((uint64_t)a.table_width * a.page + TILE - 1) / TILE + START);
        grid = (unsigned)std::min<uint64_t>(items, split_blocks(sm_count, rows ? row_blocks(o.dtype, width, (int)a.block_heads) : ANY_BLOCKS));
    }
    if (!rows) return o.dtype == LT_BF16 ? launch_any<__nv_bfloat16>(a, grid, stream) : launch_any<float>(a, grid, stream);
    if (o.dtype == LT_F32) {
        switch (width) {
        case 64: return launch_single_heads<64>(a, grid, stream);
        case 128: return launch_single_heads<128>(a, grid, stream);
        case 192: return launch_single_heads<192>(a, grid, stream);
        default: return launch_single_heads<256>(a, grid, stream);
        }
    }
    switch (width) {
    case 64: return launch_tensor_heads<64>(a, grid, stream);
    case 96: return launch_tensor_heads<96>(a, grid, stream);
    case 128: return launch_tensor_heads<128>(a, grid, stream);
    case 192: return launch_tensor_heads<192>(a, grid, stream);
    default: return launch_tensor_heads<256>(a, grid, stream);
    }
}
