// Attention of one query token per sequence over a paged key-value cache.
//
// For each sequence and query head: out = sum_i w_i v_i / sum_i w_i with w_i = exp(scale q k_i - m), m the running
// maximum.  Every key and value is read once for all the query heads that share it; nothing else of size is read or
// written, so the bound is the cache's bytes over the memory's rate.
//
// Work split: the tokens of all sequences are cut into tiles of TILE; the list of (sequence, head block, tile) is divided
// evenly over the thread blocks, whatever the sequences' lengths (which only the device knows).  A block walks its part
// of the list; a (sequence, head block) that lies within one block's part is finished there, one that is spread over
// several leaves partial results (m, sum, unnormalised out), which a second kernel joins in the list's order.
#include "operator_device.cuh"

using namespace ltop;

namespace {

constexpr int TILE = 64;        // tokens
constexpr int HEADS = 8;        // query heads a block works on at a time
constexpr int THREADS = 128;

struct AttendArgs {
    const void *q, *cache;
    const int *table, *lengths;
    void *out;
    float *partial;             // [2 x blocks][HEADS][dim + 2]; null: every (sequence, head block) has a block of its own
    unsigned int *status;
    uint64_t q_pitch, page_stride, value_offset, token_stride, head_stride;
    uint32_t batch, heads, kv_heads, group, head_blocks, dim, pages, page, table_width;
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

// Sum over the block of a 64-bit value per thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, uint64_t *part) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    uint64_t r = 0;
    for (unsigned w = 0; w < blockDim.x >> 5; ++w) r += part[w];
    return r;
}

// Tiles of the sequences before `upto`, and of all.
__device__ void count_tiles(const AttendArgs &a, uint32_t upto, uint64_t *part, uint64_t *before, uint64_t *all) {
    uint64_t s = 0, t = 0;
    for (uint32_t b = threadIdx.x; b < a.batch; b += blockDim.x) {
        const uint64_t n = tiles_of(a, b);
        t += n;
        if (b < upto) s += n;
    }
    *before = block_sum(s, part);
    *all = block_sum(t, part);
}

// A block's share of the list, in tiles.
__device__ __forceinline__ uint64_t share_of(uint64_t items, unsigned blocks) {
    const uint64_t s = (items + blocks - 1) / blocks;
    return s < 1 ? 1 : s;
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

// Any alignment, either dtype: a warp per token, a lane has values lane, lane + 32, ..; NE = ceil(dim / 32) of them.
template <class T, int NE>
__global__ void __launch_bounds__(THREADS) lt_attend_any(const AttendArgs a) {
    __shared__ uint64_t part[32];
    __shared__ float sm_m[4][HEADS], sm_l[4][HEADS];
    __shared__ float sm_o[4][HEADS][NE * 32];
    __shared__ uint32_t sh_b;
    __shared__ uint64_t sh_first;
    pdl_release();
    pdl_wait();
    const T *q = (const T *)a.q, *cache = (const T *)a.cache;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t blocks_per = a.kv_heads * a.head_blocks;

    uint64_t idx, end;
    uint32_t b = 0;
    uint64_t base = 0;  // list index of the first tile of sequence b
    if (a.partial) {
        uint64_t none, all;
        count_tiles(a, 0, part, &none, &all);
        const uint64_t items = all * blocks_per, share = share_of(items, gridDim.x);
        idx = (uint64_t)blockIdx.x * share;
        end = min(idx + share, items);
        if (idx >= end) return;
        // the sequence that holds item idx
        for (uint32_t b0 = 0;; b0 += THREADS) {
            const uint32_t mine = b0 + threadIdx.x;
            const uint64_t n = mine < a.batch ? (uint64_t)tiles_of(a, mine) * blocks_per : 0;
            const uint64_t sum = block_sum(n, part);
            if (idx < base + sum) {
                if (threadIdx.x == 0) {
                    uint64_t s = base;
                    uint32_t k = b0;
                    for (;; ++k) {
                        const uint64_t nk = (uint64_t)tiles_of(a, k) * blocks_per;
                        if (idx < s + nk) break;
                        s += nk;
                    }
                    sh_b = k;
                    sh_first = s;
                }
                __syncthreads();
                b = sh_b;
                base = sh_first;
                break;
            }
            base += sum;
        }
    } else {
        b = blockIdx.x / blocks_per;
        idx = (uint64_t)(blockIdx.x - b * blocks_per) * tiles_of(a, b);
        end = idx + tiles_of(a, b);
    }
    const uint64_t start = idx;

    while (idx < end) {
        const int n = length_of(a, b);
        const uint32_t tiles = ((uint32_t)n + TILE - 1) / TILE;
        if (tiles == 0 || idx >= base + (uint64_t)tiles * blocks_per) {
            base += (uint64_t)tiles * blocks_per;
            ++b;
            continue;
        }
        const uint32_t hb = (uint32_t)((idx - base) / tiles), t0 = (uint32_t)((idx - base) - (uint64_t)hb * tiles);
        const uint32_t t1 = (uint32_t)min((uint64_t)tiles, t0 + (end - idx));
        const uint32_t kv = hb / a.head_blocks, h0 = kv * a.group + (hb - kv * a.head_blocks) * HEADS;
        const int nh = min(HEADS, (int)(a.group - (hb - kv * a.head_blocks) * HEADS));
        const int *row = a.table + (uint64_t)b * a.table_width;

        float qr[HEADS][NE], acc[HEADS][NE], m[HEADS], l[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const uint32_t d = lane + 32 * e;
                qr[h][e] = (h < nh && d < a.dim) ? to_float(q[(uint64_t)b * a.q_pitch + (uint64_t)(h0 + h) * a.dim + d]) * a.scale : 0.f;
                acc[h][e] = 0.f;
            }
        }
        const int last = min(n, (int)(t1 * TILE));
        for (int i = (int)(t0 * TILE) + warp; i < last; i += 4) {
            uint64_t at;
            if (!locate(a, row, i, kv, &at)) continue;
            float k[NE], v[NE];
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const uint32_t d = lane + 32 * e;
                k[e] = d < a.dim ? to_float(cache[at + d]) : 0.f;
                v[e] = d < a.dim ? to_float(cache[at + a.value_offset + d]) : 0.f;
            }
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                if (h >= nh) break;
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < NE; ++e) s += qr[h][e] * k[e];
                s = warp_sum(s);
                const float mn = fmaxf(m[h], s);
                const float keep = m[h] == -INFINITY ? 0.f : exp2f(m[h] - mn), w = s == -INFINITY ? 0.f : exp2f(s - mn);
                m[h] = mn;
                l[h] = l[h] * keep + w;
#pragma unroll
                for (int e = 0; e < NE; ++e) acc[h][e] = acc[h][e] * keep + w * v[e];
            }
        }
        __syncthreads();  // the warps' shares may still be read from the segment before
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            if (lane == 0) sm_m[warp][h] = m[h], sm_l[warp][h] = l[h];
#pragma unroll
            for (int e = 0; e < NE; ++e) sm_o[warp][h][lane + 32 * e] = acc[h][e];
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == tiles;
        float *slot = a.partial ? a.partial + ((uint64_t)2 * blockIdx.x + (idx == start ? 0 : 1)) * HEADS * (a.dim + 2) : nullptr;
        for (int x = threadIdx.x; x < nh * (int)a.dim; x += THREADS) {
            const int h = x / (int)a.dim, d = x - h * (int)a.dim;
            float mm = -INFINITY;
            for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm_m[w][h]);
            float ll = 0.f, oo = 0.f;
            for (int w = 0; w < 4; ++w) {
                const float f = sm_m[w][h] == -INFINITY ? 0.f : exp2f(sm_m[w][h] - mm);
                ll += sm_l[w][h] * f;
                oo += sm_o[w][h][d] * f;
            }
            if (whole) {
                ((T *)a.out)[((uint64_t)b * a.heads + h0 + h) * a.dim + d] = from_float<T>(ll > 0.f ? oo / ll : ll == 0.f ? 0.f : ll);
            } else {
                slot[h * (a.dim + 2) + d] = oo;
                if (d == 0) slot[h * (a.dim + 2) + a.dim] = mm, slot[h * (a.dim + 2) + a.dim + 1] = ll;
            }
        }
        idx += t1 - t0;
    }
    if (!a.partial && start == end) {  // an empty sequence
        const uint32_t hb = blockIdx.x - b * blocks_per, kv = hb / a.head_blocks, first = (hb - kv * a.head_blocks) * HEADS;
        const int nh = min(HEADS, (int)(a.group - first));
        for (int x = threadIdx.x; x < nh * (int)a.dim; x += THREADS) ((T *)a.out)[((uint64_t)b * a.heads + kv * a.group + first) * a.dim + x] = from_float<T>(0.f);
    }
    if (!a.partial) check_length(a, b);
}

// Joins what several blocks left for one (sequence, head block), in the order of its tiles; writes the zeros of empty sequences.
template <class T>
__global__ void __launch_bounds__(THREADS) lt_attend_join(const AttendArgs a, const unsigned blocks) {
    __shared__ uint64_t part[32];
    pdl_release();
    pdl_wait();
    const uint32_t hb = blockIdx.x, b = blockIdx.y, blocks_per = a.kv_heads * a.head_blocks;
    check_length(a, b);
    uint64_t before, all;
    count_tiles(a, b, part, &before, &all);
    const uint32_t tiles = tiles_of(a, b), kv = hb / a.head_blocks, first = (hb - kv * a.head_blocks) * HEADS;
    const int nh = min(HEADS, (int)(a.group - first));
    T *out = (T *)a.out + ((uint64_t)b * a.heads + kv * a.group + first) * a.dim;
    if (tiles == 0) {
        for (int x = threadIdx.x; x < nh * (int)a.dim; x += THREADS) out[x] = from_float<T>(0.f);
        return;
    }
    const uint64_t share = share_of(all * blocks_per, blocks), s = before * blocks_per + (uint64_t)hb * tiles, e = s + tiles;
    const uint64_t c0 = s / share, c1 = (e - 1) / share;
    if (c0 == c1) return;  // finished by its block
    for (int x = threadIdx.x; x < nh * (int)a.dim; x += THREADS) {
        const int h = x / (int)a.dim, d = x - h * (int)a.dim;
        float mm = -INFINITY, ll = 0.f, oo = 0.f;
        for (uint64_t c = c0; c <= c1; ++c) {
            const float *slot = a.partial + (2 * c + (c == c0 && s != c * share ? 1 : 0)) * HEADS * (a.dim + 2) + h * (a.dim + 2);
            const float m = slot[a.dim], mn = fmaxf(mm, m);
            const float f0 = mm == -INFINITY ? 0.f : exp2f(mm - mn), f1 = m == -INFINITY ? 0.f : exp2f(m - mn);
            ll = ll * f0 + slot[a.dim + 1] * f1;
            oo = oo * f0 + slot[d] * f1;
            mm = mn;
        }
        out[x] = from_float<T>(ll > 0.f ? oo / ll : ll == 0.f ? 0.f : ll);
    }
}

// A block of its own per (sequence, head block) when no sequence can hold more than a few tiles.
bool split(const LtOperator &o) { return (uint64_t)o.table_width * o.page > 2 * TILE; }

unsigned attend_blocks(const LtOperator &o, int sm_count) {
    (void)o;
    return (unsigned)sm_count * 4;
}

template <class T, int NE>
cudaError_t launch_any(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    return launch_pdl(lt_attend_any<T, NE>, grid, THREADS, (size_t)0, stream, a);
}

template <class T>
cudaError_t launch_attend(const AttendArgs &a, unsigned grid, cudaStream_t stream) {
    if (a.dim <= 64) return launch_any<T, 2>(a, grid, stream);
    if (a.dim <= 128) return launch_any<T, 4>(a, grid, stream);
    return launch_any<T, 8>(a, grid, stream);
}

}  // namespace

size_t lt_paged_attention_scratch(const LtOperator &o, int sm_count) {
    return split(o) ? (size_t)2 * attend_blocks(o, sm_count) * HEADS * (o.dim + 2) * sizeof(float) : 0;
}

cudaError_t lt_launch_paged_attention(const LtOperator &o, unsigned int *status, int sm_count, cudaStream_t stream, unsigned *launched) {
    AttendArgs a{};
    a.q = o.in[0];
    a.cache = o.in[1];
    a.table = (const int *)o.in[2];
    a.lengths = (const int *)o.in[3];
    a.out = o.out[0];
    a.partial = split(o) ? (float *)o.scratch : nullptr;
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
    a.head_blocks = (a.group + HEADS - 1) / HEADS;
    a.dim = o.dim;
    a.pages = o.pages;
    a.page = o.page;
    a.table_width = o.table_width;
    a.scale = (float)(lt_attr_double(o.attr[1]) * 1.4426950408889634);
    const unsigned per = a.kv_heads * a.head_blocks, grid = a.partial ? attend_blocks(o, sm_count) : a.batch * per;
    *launched = 1;
    cudaError_t e = o.dtype == LT_BF16 ? launch_attend<__nv_bfloat16>(a, grid, stream) : launch_attend<float>(a, grid, stream);
    if (e != cudaSuccess || !a.partial) return e;
    *launched = 2;
    const dim3 g2(per, a.batch);
    return o.dtype == LT_BF16 ? launch_pdl_grid(lt_attend_join<__nv_bfloat16>, g2, THREADS, stream, a, grid)
                              : launch_pdl_grid(lt_attend_join<float>, g2, THREADS, stream, a, grid);
}
