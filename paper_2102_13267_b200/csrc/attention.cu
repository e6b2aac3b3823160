// Attention of one query token per sequence over a paged key-value cache.
//
// For each sequence and query head: out = sum_i w_i v_i / sum_i w_i with w_i = exp(scale q k_i - m), m the running
// maximum.  Every key and value is read once for all the query heads that share it; nothing else of size is read or
// written, so the bound is the cache's bytes over the memory's rate.
//
// Work split: the tokens of all sequences are cut into tiles of TILE; the list of (sequence, head block, tile) is divided
// evenly over the thread blocks, whatever the sequences' lengths (which only the device knows).  Every (sequence, head
// block) counts START tiles more than it has, for what beginning one costs (measured below).  A block walks its part of
// the list; a (sequence, head block) that lies within one block's part is finished there.  One that is spread over
// several blocks leaves partial results (maximum, sum, unnormalised output) in scratch memory, and the block that
// arrives last joins them, always in the list's order, so results do not depend on the arrival.
#include "operator_device.cuh"

using namespace ltop;

namespace {

constexpr int TILE = 64;        // tokens
constexpr int START = 2;        // tiles that beginning a (sequence, head block) counts for
constexpr int MOST_PARTS = 64;  // blocks one (sequence, head block) is spread over
constexpr int THREADS = 128;

struct AttendArgs {
    const void *q, *cache;
    const int *table, *lengths;
    void *out;
    float *partial;             // [2 x blocks][block_heads][dim + 2]: outputs, then (maximum, sum) of each head; null: every (sequence, head block) has a block of its own
    unsigned int *arrivals;     // [blocks], zero between launches: how many of the blocks that share what begins in block i have left their part
    unsigned int *status;
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
    if (threadIdx.x == 0 && a.lengths[b] > 0 && (int64_t)a.lengths[b] > (int64_t)a.table_width * a.page) atomicOr(a.status, 1u);
}

__device__ __forceinline__ uint32_t tiles_of(const AttendArgs &a, uint32_t b) { return ((uint32_t)length_of(a, b) + TILE - 1) / TILE; }

// Length of sequence b's part of the list, per head block.
__device__ __forceinline__ uint32_t items_of(const AttendArgs &a, uint32_t b) {
    const uint32_t t = tiles_of(a, b);
    return t ? t + START : 0;
}

// Inclusive sums over the block's threads of a 64-bit value each; *all: over the whole block; *most: the largest `w`.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint32_t w, uint64_t *part, uint64_t *all, uint32_t *most) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += o;
    }
    w = __reduce_max_sync(0xffffffffu, w);
    __syncthreads();  // `part` may still be read from the scan before
    if (lane == 31) part[warp] = v, part[THREADS / 32 + warp] = w;
    __syncthreads();
    uint64_t before = 0, sum = 0;
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
        if (k < warp) before += part[k];
        sum += part[k];
        top = max(top, (uint32_t)part[THREADS / 32 + k]);
    }
    *all = sum;
    *most = top;
    return v + before;
}

// What a block works on: items [idx, end) of the list, the first in sequence b, whose own first item is `base`.
struct Share {
    uint64_t idx, end, base, size;  // size: of a block's share
    uint32_t b;
};

// The block's part of the list, from the sequences' lengths.  `part`, `found`: shared, 32 and 2 values.
__device__ __forceinline__ Share my_share(const AttendArgs &a, uint64_t *part, uint64_t *found) {
    const uint32_t per = a.kv_heads * a.head_blocks;
    Share s{};
    if (!a.partial) {  // a block per (sequence, head block)
        s.b = blockIdx.x / per;
        const uint64_t t = items_of(a, s.b);
        s.idx = (uint64_t)(blockIdx.x - s.b * per) * t;
        s.end = s.idx + t;
        return s;
    }
    uint64_t total = 0, sum;
    uint32_t most, more = 0;
    uint32_t items = threadIdx.x < a.batch ? items_of(a, threadIdx.x) : 0;
    uint64_t mine = (uint64_t)items * per, upto = block_scan(mine, items, part, &sum, &most);
    if (a.batch > THREADS) {
        uint64_t rest = 0;
        uint32_t top = 0;
        for (uint32_t b = threadIdx.x + THREADS; b < a.batch; b += THREADS) {
            const uint32_t n = items_of(a, b);
            rest += (uint64_t)n * per;
            top = max(top, n);
        }
        block_scan(rest, top, part, &total, &more);
    }
    total += sum;
    most = max(most, more);
    // an even share, and no (sequence, head block) over more than MOST_PARTS blocks
    s.size = max((total + gridDim.x - 1) / gridDim.x, (uint64_t)((most + MOST_PARTS - 2) / (MOST_PARTS - 1)));
    s.idx = (uint64_t)blockIdx.x * s.size;
    s.end = min(s.idx + s.size, total);
    if (s.idx >= s.end) {
        s.idx = s.end = 0;
        return s;
    }
    uint64_t before = 0;
    for (uint32_t b0 = 0;;) {
        if (s.idx < before + sum) {
            if (s.idx >= before + upto - mine && s.idx < before + upto) found[0] = b0 + threadIdx.x, found[1] = before + upto - mine;
            break;
        }
        before += sum;
        b0 += THREADS;
        mine = b0 + threadIdx.x < a.batch ? (uint64_t)items_of(a, b0 + threadIdx.x) * per : 0;
        upto = block_scan(mine, 0, part, &sum, &more);
    }
    __syncthreads();
    s.b = (uint32_t)found[0];
    s.base = found[1];
    return s;
}

// A stretch of tiles of one (sequence, head block).
struct Stretch {
    uint64_t first;         // list index of the first item of the (sequence, head block)
    uint32_t b, kv, h0;     // h0: first query head
    int n, heads;           // tokens of the sequence, query heads
    uint32_t t0, t1, tiles;
    uint32_t items;         // of the list
};

// The next stretch of the share, or false when it is done; `done`: items of the one before.
__device__ __forceinline__ bool next_stretch(const AttendArgs &a, Share &s, Stretch &w, uint32_t done) {
    const uint32_t per = a.kv_heads * a.head_blocks;
    for (;;) {
        s.idx += done;
        if (s.idx >= s.end) return false;
        uint32_t all;
        for (;;) {
            w.n = length_of(a, s.b);
            w.tiles = ((uint32_t)w.n + TILE - 1) / TILE;
            all = w.tiles ? w.tiles + START : 0;
            if (s.idx < s.base + (uint64_t)all * per) break;
            s.base += (uint64_t)all * per;
            ++s.b;
        }
        const uint32_t hb = (uint32_t)((s.idx - s.base) / all);
        w.first = s.base + (uint64_t)hb * all;
        const uint32_t v0 = (uint32_t)(s.idx - w.first), v1 = (uint32_t)min((uint64_t)all, v0 + (s.end - s.idx));
        done = w.items = v1 - v0;
        w.t0 = max(v0, (uint32_t)START) - START;
        w.t1 = max(v1, (uint32_t)START) - START;
        if (w.t1 == w.t0) continue;  // only of what beginning counts for
        w.b = s.b;
        w.kv = hb / a.head_blocks;
        const uint32_t first = (hb - w.kv * a.head_blocks) * a.block_heads;
        w.h0 = w.kv * a.group + first;
        w.heads = (int)min(a.block_heads, a.group - first);
        return true;
    }
}

// Where the block leaves its part of a stretch that others share.
__device__ __forceinline__ float *part_of(const AttendArgs &a, uint64_t block, bool second) {
    return a.partial + (2 * block + (second ? 1 : 0)) * a.block_heads * (a.dim + 2);
}

__device__ __forceinline__ float quotient(float o, float l) { return l > 0.f ? o / l : l == 0.f ? 0.f : l; }

// The block has left its part of stretch w: if it is the last of those that share the (sequence, head block), it joins the
// parts.  `room`: shared memory for block_heads x MOST_PARTS values; `sums`: for block_heads values.  V values at a time
// (dim a multiple of V, scratch and output aligned accordingly).
template <class T, int V>
__device__ __forceinline__ void join_if_last(const AttendArgs &a, const Share &s, const Stretch &w, float *room, float *sums, uint64_t *flag) {
    const uint64_t c0 = (w.first + START) / s.size, c1 = (w.first + START + w.tiles - 1) / s.size;
    const uint32_t count = (uint32_t)(c1 - c0) + 1;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *flag = atomicAdd(a.arrivals + c0, 1u) == count - 1;
        __threadfence();
    }
    __syncthreads();
    if (!*flag) return;
    if (threadIdx.x == 0) a.arrivals[c0] = 0;
    const uint32_t dim = a.dim;
    const uint64_t slot = (uint64_t)2 * a.block_heads * (dim + 2);
    const float *head = part_of(a, c0, c0 * s.size < w.first), *rest = part_of(a, c0, false);  // of the first part; of the others, i x slot on
    auto of = [&](uint32_t i) { return i ? rest + i * slot : head; };
    for (uint32_t x = threadIdx.x; x < (uint32_t)w.heads * MOST_PARTS; x += THREADS) {
        const uint32_t h = x / MOST_PARTS, i = x % MOST_PARTS;
        if (i < count) room[x] = __ldcg(of(i) + a.block_heads * dim + 2 * h);
    }
    __syncthreads();
    for (int h = threadIdx.x >> 5; h < w.heads; h += THREADS / 32) {  // a warp per head: maxima to weights
        float top = -INFINITY, sum = 0.f;
        for (uint32_t i = threadIdx.x & 31; i < count; i += 32) top = fmaxf(top, room[h * MOST_PARTS + i]);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (top == -INFINITY) top = 0.f;
        for (uint32_t i = threadIdx.x & 31; i < count; i += 32) {
            const float f = exp2f(room[h * MOST_PARTS + i] - top);
            room[h * MOST_PARTS + i] = f;
            sum += f * __ldcg(of(i) + a.block_heads * dim + 2 * h + 1);
        }
        sum = warp_sum(sum);
        if ((threadIdx.x & 31) == 0) sums[h] = sum;
    }
    __syncthreads();
    for (uint32_t x = threadIdx.x; x < (uint32_t)w.heads * (dim / V); x += THREADS) {
        const uint32_t h = x / (dim / V), d = (x - h * (dim / V)) * V;
        float o[V] = {};
#pragma unroll 8
        for (uint32_t i = 0; i < count; ++i) {
            const float *p = of(i) + h * dim + d;
            const float f = room[h * MOST_PARTS + i];
            if constexpr (V == 4) {
                const float4 v = __ldcg(reinterpret_cast<const float4 *>(p));
                o[0] += f * v.x;
                o[1] += f * v.y;
                o[2] += f * v.z;
                o[3] += f * v.w;
            } else {
                o[0] += f * __ldcg(p);
            }
        }
        T *out = (T *)a.out + ((uint64_t)w.b * a.heads + w.h0 + h) * dim + d;
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = from_float<T>(quotient(o[k], sums[h]));
    }
    __syncthreads();  // `room` is used again
}

// The zeros of empty sequences, and the check of the lengths.
template <class T>
__device__ __forceinline__ void finish(const AttendArgs &a) {
    if (!a.partial) {  // the block's own sequence
        const uint32_t per = a.kv_heads * a.head_blocks, b = blockIdx.x / per;
        check_length(a, b);
        if (tiles_of(a, b)) return;
        const uint32_t hb = blockIdx.x - b * per, kv = hb / a.head_blocks, first = (hb - kv * a.head_blocks) * a.block_heads;
        const uint32_t count = min(a.block_heads, a.group - first) * a.dim;
        T *out = (T *)a.out + ((uint64_t)b * a.heads + kv * a.group + first) * a.dim;
        for (uint32_t x = threadIdx.x; x < count; x += THREADS) out[x] = from_float<T>(0.f);
        return;
    }
    for (uint32_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        check_length(a, b);
        if (tiles_of(a, b)) continue;
        T *out = (T *)a.out + (uint64_t)b * a.heads * a.dim;
        for (uint32_t x = threadIdx.x; x < a.heads * a.dim; x += THREADS) out[x] = from_float<T>(0.f);
    }
}

// First element of token i's key in head `kv`; false where its page is no page of the cache.
__device__ __forceinline__ bool locate(const AttendArgs &a, const int *row, int i, uint32_t kv, uint64_t *at) {
    const uint32_t e = (uint32_t)i / a.page, off = (uint32_t)i - e * a.page;
    const int p = row[e];
    if ((uint32_t)p >= a.pages) {
        atomicOr(a.status, 1u);
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
    __shared__ uint64_t part[32], found[2];
    __shared__ float sm_m[4][HEADS], sm_l[4][HEADS];
    __shared__ float sm_o[4][HEADS][NE * 32];
    float *sm_room = &sm_o[0][0][0];
    static_assert(4 * NE * 32 >= MOST_PARTS, "the parts' weights fit");
    pdl_release();
    pdl_wait();
    const T *q = (const T *)a.q, *cache = (const T *)a.cache;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Share s = my_share(a, part, found);
    const uint64_t start = s.idx;
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
        if (!whole) join_if_last<T, 1>(a, s, w, sm_room, &sm_l[0][0], found);
    }
    finish<T>(a);
}

// ------------------------------------------------------------------------------------------- bf16 on the matrix units

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
__device__ __forceinline__ float power2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr int STEP = 16;        // tokens a warp takes at a time: a quarter of a tile
constexpr int STAGES = 3;

// Resident blocks per SM: what the stages leave room for, fewer where 16 or 32 heads of 64 values take the registers.
constexpr int tensor_blocks(int width, int tiles) { return width <= 64 ? (tiles == 1 ? 4 : tiles == 2 ? 3 : 2) : width <= 128 ? 2 : 1; }

// Shared memory of a block: per warp STAGES steps of keys and values, rows padded by 16 bytes so that eight rows of a
// matrix fall into different banks.
template <int DP>
constexpr size_t tensor_bytes() { return (size_t)(THREADS / 32) * STAGES * 2 * STEP * (DP * 2 + 16); }

// bf16, 16-byte aligned, head sizes that are multiples of 8, filled up to DP with zeros; NT x 8 query heads per block.
//
// The few query heads make the narrow side of the products: scores are K (16 tokens x dims) times q^T (dims x 8 heads),
// the output is V^T (16 dims x 16 tokens) times the weights (16 tokens x 8 heads), so no matrix row is wasted on
// padding of the group to 16.  The weights leave the first product with tokens along the rows and enter the second with
// tokens along the columns of a register's pair: movmatrix turns them, as two bf16 parts (p and what its rounding left), which keeps
// the weights to 2^-17 and costs one more product.  Each warp has steps and a copy pipeline of its own -- no barrier
// in the loop -- and its own running maximum and sum; warps are joined once per stretch.
template <int DP, int NT, bool WHOLE_STEPS>
__global__ void __launch_bounds__(THREADS, tensor_blocks(DP, NT)) lt_attend_tensor(const AttendArgs a) {
    constexpr int HEADS = 8 * NT, PITCH = DP * 2 + 16, KS = DP / 16, CHUNKS = DP / 8;
    constexpr uint32_t STAGE_BYTES = 2 * STEP * PITCH;
    extern __shared__ __align__(128) unsigned char stage_mem[];
    __shared__ uint64_t part[32], found[2];
    __shared__ float sm_m[4][HEADS], sm_l[4][HEADS];
    __shared__ uint32_t sm_mask[4][STAGES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t chunks = a.dim / 8;
    unsigned char *mine = stage_mem + warp * STAGES * STAGE_BYTES;
    const uint32_t stages = shared_address(mine);
    const __nv_bfloat16 *q = (const __nv_bfloat16 *)a.q, *cache = (const __nv_bfloat16 *)a.cache;
    pdl_release();
    pdl_wait();
    Share s = my_share(a, part, found);
    const uint64_t start = s.idx;
    Stretch w;
    for (uint32_t done = 0; next_stretch(a, s, w, done); done = w.items) {
        // columns from dim to DP stay zero (the memory is also used to join warps)
        if (chunks < CHUNKS)
            for (int x = lane; x < STAGES * 2 * STEP * (CHUNKS - (int)chunks); x += 32) {
                const int r = x / (CHUNKS - (int)chunks), c = x - r * (CHUNKS - (int)chunks);
                *reinterpret_cast<uint4 *>(mine + r * PITCH + (chunks + c) * 16) = make_uint4(0, 0, 0, 0);
            }
        uint32_t qf[NT][KS][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int h = t * 8 + (lane >> 2);
                    const uint32_t d = k * 16 + i * 8 + (lane & 3) * 2;
                    qf[t][k][i] = (h < w.heads && d < a.dim) ? *reinterpret_cast<const uint32_t *>(q + (uint64_t)w.b * a.q_pitch + (uint64_t)(w.h0 + h) * a.dim + d) : 0u;
                }
        float o[NT][KS][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) o[t][k][0] = o[t][k][1] = o[t][k][2] = o[t][k][3] = 0.f;
        }
        const int *row = a.table + (uint64_t)w.b * a.table_width;
        const int first = (int)(w.t0 * TILE) + warp * STEP;  // first token of this warp's first step
        const int steps = (int)(w.t1 - w.t0);

        // Page numbers are fetched ahead of the copies they address.  Where a step never crosses a page (WHOLE_STEPS) one
        // number serves a step, and the lanes hold those of the next 32 steps; otherwise lane i has the number of token i.
        int ahead = -1;
        auto fetch_pages = [&](int step) {
            const int i = WHOLE_STEPS ? first + (step + lane) * TILE : first + step * TILE + (lane & 15);
            ahead = i < w.n ? row[(uint32_t)i / a.page] : -2;
        };
        auto issue = [&](int step) {
            if (step < steps) {
                const uint32_t to = stages + (uint32_t)(step % STAGES) * STAGE_BYTES;
                const int i0 = first + step * TILE, left = w.n - i0;
                uint32_t mask = left >= STEP ? 0xffffu : left <= 0 ? 0u : (1u << left) - 1u;
                if (WHOLE_STEPS) {
                    if (step > 0 && (step & 31) == 0) fetch_pages(step);
                    const int p = __shfl_sync(0xffffffffu, ahead, step & 31);
                    if (mask && (uint32_t)p >= a.pages) {
                        mask = 0;
                        atomicOr(a.status, 1u);
                    }
                    const uint32_t off = (uint32_t)i0 % a.page;
                    const __nv_bfloat16 *src = cache + (mask ? (uint64_t)p * a.page_stride + (uint64_t)off * a.token_stride + (uint64_t)w.kv * a.head_stride : 0);
#pragma unroll
                    for (int x = 0; x < STEP * CHUNKS; x += 32) {
                        const int r = (x + lane) / CHUNKS, c = (x + lane) % CHUNKS;
                        const bool there = (mask >> r) & 1u;
                        const __nv_bfloat16 *at = there ? src + (uint64_t)r * a.token_stride + c * 8 : cache;
                        if (c < (int)chunks) {
                            copy16(to + r * PITCH + c * 16, at, there);
                            copy16(to + (STEP + r) * PITCH + c * 16, there ? at + a.value_offset : cache, there);
                        }
                    }
                } else {
                    const int i = i0 + (lane & 15), p = ahead;
                    const bool known = i < w.n && (uint32_t)p < a.pages;
                    if (i < w.n && !known) atomicOr(a.status, 1u);
                    mask = __ballot_sync(0xffffffffu, known) & 0xffffu;
                    const uint64_t off = known ? (uint64_t)p * a.page_stride + (uint64_t)((uint32_t)i % a.page) * a.token_stride + (uint64_t)w.kv * a.head_stride : 0;
#pragma unroll
                    for (int x = 0; x < STEP * CHUNKS; x += 32) {
                        const int r = (x + lane) / CHUNKS, c = (x + lane) % CHUNKS;
                        const uint64_t from = __shfl_sync(0xffffffffu, off, r);
                        const bool there = (mask >> r) & 1u;
                        const __nv_bfloat16 *at = there ? cache + from + c * 8 : cache;
                        if (c < (int)chunks) {
                            copy16(to + r * PITCH + c * 16, at, there);
                            copy16(to + (STEP + r) * PITCH + c * 16, there ? at + a.value_offset : cache, there);
                        }
                    }
                    if (step + 1 < steps) fetch_pages(step + 1);
                }
                if (lane == 0) sm_mask[warp][step % STAGES] = mask;
            }
            copy_commit();
        };
        if (steps > 0) fetch_pages(0);
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) issue(k);
        for (int step = 0; step < steps; ++step) {
            copy_wait<STAGES - 2>();
            __syncwarp();  // the step's copies of all lanes are there, and everybody is done with the stage that the next ones fill
            const uint32_t mask = sm_mask[warp][step % STAGES];  // the tokens that count
            issue(step + STAGES - 1);
            if (mask == 0) continue;
            const uint32_t from = stages + (uint32_t)(step % STAGES) * STAGE_BYTES;
            float c[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t][0] = c[t][1] = c[t][2] = c[t][3] = 0.f;
            const uint32_t ka = from + (lane & 15) * PITCH + (lane >> 4) * 16;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t f[4];
                load_matrices(f, ka + k * 32);
#pragma unroll
                for (int t = 0; t < NT; ++t) multiply(c[t], f, qf[t][k][0], qf[t][k][1]);
            }
            const bool in0 = (mask >> (lane >> 2)) & 1u, in1 = (mask >> ((lane >> 2) + 8)) & 1u;
            uint32_t p_hi[NT][2], p_lo[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int j = 0; j < 4; ++j) c[t][j] = (j < 2 ? in0 : in1) ? c[t][j] * a.scale : -INFINITY;
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
            const uint32_t va = from + STEP * PITCH + ((lane & 7) + ((lane >> 4) & 1) * 8) * PITCH + ((lane >> 3) & 1) * 16;
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
        // join the warps
        copy_wait<0>();
        float *sm_o = reinterpret_cast<float *>(stage_mem);  // [4][HEADS][DP + 4]
        __syncthreads();  // every warp is done with its stages
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = t * 8 + (lane & 3) * 2 + j;
                float sum = l[t][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane < 4) sm_m[warp][h] = m[t][j], sm_l[warp][h] = sum;
                float *to = sm_o + (warp * HEADS + h) * (DP + 4) + (lane >> 2);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    to[k * 16] = o[t][k][j];
                    to[k * 16 + 8] = o[t][k][2 + j];
                }
            }
        __syncthreads();
        const bool whole = w.t0 == 0 && w.t1 == w.tiles;
        float *slot = whole ? nullptr : part_of(a, blockIdx.x, s.idx != start);
        for (int x = threadIdx.x; x < w.heads * (int)(a.dim / 2); x += THREADS) {
            const int h = x / (int)(a.dim / 2), d = 2 * (x - h * (int)(a.dim / 2));
            float mm = -INFINITY;
#pragma unroll
            for (int k = 0; k < 4; ++k) mm = fmaxf(mm, sm_m[k][h]);
            const float base = mm == -INFINITY ? 0.f : mm;
            float ll = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = power2(sm_m[k][h] - base);
                const float2 v = *reinterpret_cast<const float2 *>(sm_o + (k * HEADS + h) * (DP + 4) + d);
                ll += sm_l[k][h] * f;
                o0 += v.x * f;
                o1 += v.y * f;
            }
            if (whole) {
                *reinterpret_cast<uint32_t *>((__nv_bfloat16 *)a.out + ((uint64_t)w.b * a.heads + w.h0 + h) * a.dim + d) = pack_bf16(quotient(o0, ll), quotient(o1, ll));
            } else {
                *reinterpret_cast<float2 *>(slot + h * a.dim + d) = make_float2(o0, o1);
                if (d == 0) *reinterpret_cast<float2 *>(slot + HEADS * a.dim + 2 * h) = make_float2(mm, ll);
            }
        }
        if (!whole) join_if_last<__nv_bfloat16, 4>(a, s, w, sm_o, &sm_l[0][0], found);
        __syncthreads();  // the next stretch's copies go where the parts were
    }
    finish<__nv_bfloat16>(a);
}

// A block of its own per (sequence, head block) when no sequence can hold more than a few tiles.
bool split(const LtOperator &o) { return (uint64_t)o.table_width * o.page > 2 * TILE; }

// Query heads per block of lt_attend_tensor: as many heads as share a key, while queries and
// output fit the registers (32 heads of 128 values, 16 of 256).
int tensor_width(uint32_t dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256; }
int tensor_tiles(uint32_t dim, uint32_t group) { return group <= 8 ? 1 : group <= 16 || dim > 128 ? 2 : 4; }
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
    const cudaError_t e = allow_shared(lt_attend_tensor<DP, NT, WHOLE>, tensor_bytes<DP>(), ready);
    if (e != cudaSuccess) return e;
    return launch_pdl(lt_attend_tensor<DP, NT, WHOLE>, grid, THREADS, tensor_bytes<DP>(), stream, a);
}

template <int DP>
cudaError_t launch_tensor_heads(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    const bool whole = a.page % STEP == 0;
    if (a.block_heads == 8) return whole ? launch_tensor<DP, 1, true>(a, grid, stream) : launch_tensor<DP, 1, false>(a, grid, stream);
    if (a.block_heads == 16) return whole ? launch_tensor<DP, 2, true>(a, grid, stream) : launch_tensor<DP, 2, false>(a, grid, stream);
    if constexpr (DP <= 128) return whole ? launch_tensor<DP, 4, true>(a, grid, stream) : launch_tensor<DP, 4, false>(a, grid, stream);
    return cudaErrorInvalidValue;
}

}  // namespace

size_t lt_paged_attention_scratch(const LtOperator &o, int sm_count) {
    if (!split(o)) return 0;
    const size_t any = (size_t)ANY_BLOCKS * ANY_HEADS, tiles = (size_t)tensor_tiles(o.dim, o.heads / o.kv_heads),
                 tensor = (size_t)tensor_blocks(tensor_width(o.dim), (int)tiles) * 8 * tiles;
    return 2 * (size_t)sm_count * (any > tensor ? any : tensor) * (o.dim + 2) * sizeof(float);
}

cudaError_t lt_launch_paged_attention(const LtOperator &o, unsigned int *status, int sm_count, cudaStream_t stream) {
    AttendArgs a{};
    a.q = o.in[0];
    a.cache = o.in[1];
    a.table = (const int *)o.in[2];
    a.lengths = (const int *)o.in[3];
    a.out = o.out[0];
    a.partial = split(o) ? (float *)o.scratch : nullptr;
    a.arrivals = (unsigned int *)o.arrivals;
    a.status = status;
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
    const bool tensor = o.dtype == LT_BF16 && o.dim % 8 == 0 && is_aligned(a.cache, 16) && is_aligned(a.q, 4) && a.q_pitch % 2 == 0 && is_aligned(a.out, 4);
    a.block_heads = tensor ? 8 * tensor_tiles(o.dim, a.group) : ANY_HEADS;
    a.head_blocks = (a.group + a.block_heads - 1) / a.block_heads;
    const unsigned per = a.kv_heads * a.head_blocks;
    const unsigned grid = a.partial ? (unsigned)sm_count * (tensor ? tensor_blocks(tensor_width(o.dim), (int)a.block_heads / 8) : ANY_BLOCKS) : a.batch * per;
    cudaError_t e;
    if (!tensor) {
        e = o.dtype == LT_BF16 ? launch_any<__nv_bfloat16>(a, grid, stream) : launch_any<float>(a, grid, stream);
    } else {
        switch (tensor_width(o.dim)) {
        case 64: e = launch_tensor_heads<64>(a, grid, stream); break;
        case 96: e = launch_tensor_heads<96>(a, grid, stream); break;
        case 128: e = launch_tensor_heads<128>(a, grid, stream); break;
        case 192: e = launch_tensor_heads<192>(a, grid, stream); break;
        default: e = launch_tensor_heads<256>(a, grid, stream); break;
        }
    }
    return e;
}
