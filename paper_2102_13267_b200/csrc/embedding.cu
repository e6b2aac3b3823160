// Looking tokens up in a table [vocabulary, columns], and the gradient of that.
//
// Both move every value once and are bound by memory.  The gradient of row v is the sum of the rows of dy whose token is v.
// Tokens are sorted first (lt_token_sort), so that a row's sum is made by the threads that write the row, in the order
// of the tokens: no atomics on values, and the same result every time.  A token that makes up much of a text would keep one
// block busy with its row while the others have finished, so rows of more than WINDOW tokens are summed in pieces,
// which end at multiples of WINDOW of the sorted order, and the pieces are joined in order (lt_embedding_join).
#include <algorithm>

#include "operator_device.cuh"

using namespace ltop;

namespace {

constexpr int THREADS = 256;

// N values of T that a thread has at once: 16 bytes of them, or one where alignment or sizes forbid more
template <class T, int N>
__device__ __forceinline__ void load_values(const T *from, float (&f)[N]) {
    if constexpr (N == 1) {
        f[0] = to_float(*from);
    } else if constexpr (N * sizeof(T) == 16) {
        unpack(*reinterpret_cast<const uint4 *>(from), f);
    } else {  // eight f32
        const float4 a = reinterpret_cast<const float4 *>(from)[0], b = reinterpret_cast<const float4 *>(from)[1];
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
}
template <class T, int N>
__device__ __forceinline__ void store_values(T *to, const float (&f)[N]) {
    if constexpr (N == 1) {
        *to = from_float<T>(f[0]);
    } else if constexpr (N * sizeof(T) == 16) {
        *reinterpret_cast<uint4 *>(to) = pack(f);
    } else {
        reinterpret_cast<float4 *>(to)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4 *>(to)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
}

// How the threads of a block are laid over rows of `chunks` pieces: `across` threads (a power of two) to a slice of a row.
struct Layout {
    uint32_t across, beside, slices;  // beside: rows side by side
    Divisor by_slices;
};
Layout layout_of(uint64_t chunks) {
    Layout l;
    l.across = 32;
    while (l.across < THREADS && l.across < chunks) l.across *= 2;
    l.beside = THREADS / l.across;
    l.slices = (uint32_t)((chunks + l.across - 1) / l.across);
    l.by_slices = Divisor::make(l.slices);
    return l;
}
__device__ __forceinline__ uint32_t row_of(const Layout &l, uint64_t unit) { return unit >> 32 ? (uint32_t)(unit / l.slices) : l.by_slices.quotient((uint32_t)unit); }

// ------------------------------------------------------------------------------------------- lookup

struct LookupArgs {
    const void *table;
    const int *ids;
    void *out;
    unsigned int *status;
    uint64_t pitch;
    uint32_t tokens, vocabulary, cols;
    float scale;
    Layout l;
};

constexpr int LOOKUP_FLIGHT = 4;  // rows a thread has on their way

template <class T, int N>
__global__ void __launch_bounds__(THREADS) lt_embedding(const LookupArgs a) {
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & (a.l.across - 1), row = threadIdx.x / a.l.across;
    const uint64_t units = (uint64_t)a.tokens * a.l.slices, step = (uint64_t)gridDim.x * a.l.beside;
    for (uint64_t u0 = (uint64_t)blockIdx.x * a.l.beside + row; u0 < units; u0 += step * LOOKUP_FLIGHT) {
        float f[LOOKUP_FLIGHT][N];
        uint32_t token[LOOKUP_FLIGHT], col[LOOKUP_FLIGHT];
        int id[LOOKUP_FLIGHT];
#pragma unroll
        for (int k = 0; k < LOOKUP_FLIGHT; ++k) {
            const uint64_t u = u0 + k * step;
            token[k] = row_of(a.l, u);
            col[k] = ((uint32_t)(u - (uint64_t)token[k] * a.l.slices) * a.l.across + lane) * N;
            if (u >= units) col[k] = a.cols;
            id[k] = u < units ? a.ids[token[k]] : -1;
        }
#pragma unroll
        for (int k = 0; k < LOOKUP_FLIGHT; ++k) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[k][i] = 0.f;
            if (col[k] >= a.cols || id[k] < 0) continue;
            if ((uint32_t)id[k] >= a.vocabulary) {
                report(a.status);
                continue;
            }
            load_values((const T *)a.table + (uint64_t)id[k] * a.pitch + col[k], f[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) f[k][i] *= a.scale;
        }
#pragma unroll
        for (int k = 0; k < LOOKUP_FLIGHT; ++k)
            if (col[k] < a.cols) store_values((T *)a.out + (uint64_t)token[k] * a.cols + col[k], f[k]);
    }
}

template <class T, int N>
cudaError_t launch_lookup(LookupArgs &a, int sm_count, cudaStream_t stream) {
    a.l = layout_of((a.cols + N - 1) / N);
    const uint64_t blocks = ((uint64_t)a.tokens * a.l.slices + a.l.beside - 1) / a.l.beside, most = (uint64_t)sm_count * 8;
    return launch_pdl(lt_embedding<T, N>, (unsigned)std::min(blocks, most), THREADS, (size_t)0, stream, a);
}

inline bool is_aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// ------------------------------------------------------------------------------------------- sorting tokens

constexpr int SORT_THREADS = 1024;
constexpr uint32_t SORT_STEP = 4 * SORT_THREADS;  // tokens a block looks at at once
constexpr uint32_t SORT_LIST = 2 * SORT_STEP;
constexpr uint32_t SORT_COUNTS = 16384;           // rows of a class, at most
constexpr uint32_t SORT_CLASSES = 128;            // at least

struct Segment {
    uint32_t start, count;  // a row's tokens in the sorted order
};

struct SortArgs {
    const int *ids;
    Segment *segments;      // [classes][rows of a class]
    uint32_t *order;        // tokens, row by row
    uint32_t *total;        // how many tokens name a row
    unsigned int *status;
    uint32_t tokens, vocabulary, shift, per_class;  // classes: 2^shift
};

__device__ __forceinline__ void four_ids(const SortArgs &a, uint32_t i, int (&id)[4]) {
    if (i + 4 <= a.tokens && ((uintptr_t)a.ids & 15) == 0) {
        const int4 v = *reinterpret_cast<const int4 *>(a.ids + i);
        id[0] = v.x, id[1] = v.y, id[2] = v.z, id[3] = v.w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = i + k < a.tokens ? a.ids[i + k] : -1;
    }
}

// Exclusive sum over the block; `parts`: room for 32 values; *all: the sum of all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *parts, uint32_t *all) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= (uint32_t)d) upto += o;
    }
    __syncthreads();  // `parts` may still be read from the sum before
    if (lane == 31) parts[warp] = upto;
    __syncthreads();
    uint32_t w = parts[lane], before = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= (uint32_t)d) before += o;
    }
    *all = __shfl_sync(0xffffffffu, before, 31);
    before -= w;
    return upto - v + __shfl_sync(0xffffffffu, before, warp);
}

// Sorts tokens by row, those of a row in their own order, in one launch whose blocks do not wait for one another: a block has
// a class of rows (v modulo the number of classes, which deals frequent tokens out evenly where vocabularies are sorted by
// frequency), reads all tokens, counts those of its rows and those of the classes before, and places its own.  Reading the tokens
// once per class costs little beside rows of hundreds of values: 4 bytes each, out of the L2 cache.
__global__ void __launch_bounds__(SORT_THREADS) lt_token_sort(const SortArgs a) {
    extern __shared__ uint32_t counts[];  // [rows of a class]; then uint2 [SORT_LIST]
    __shared__ uint32_t parts[32];
    uint2 *list = reinterpret_cast<uint2 *>(counts + ((a.per_class + 1) & ~1u));
    const uint32_t mine = blockIdx.x, mask = (1u << a.shift) - 1;
    pdl_release();
    pdl_wait();
    for (uint32_t l = threadIdx.x; l < a.per_class; l += SORT_THREADS) counts[l] = 0;
    __syncthreads();
    uint32_t below = 0;
#pragma unroll 4
    for (uint32_t i = 4 * threadIdx.x; i < a.tokens; i += SORT_STEP) {
        int id[4];
        four_ids(a, i, id);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (id[k] < 0) continue;
            if ((uint32_t)id[k] >= a.vocabulary) {
                if (mine == 0) report(a.status);
                continue;
            }
            const uint32_t c = (uint32_t)id[k] & mask;
            below += c < mine;
            if (c == mine) atomicAdd(&counts[(uint32_t)id[k] >> a.shift], 1u);
        }
    }
    uint32_t base, own;
    block_scan(below, parts, &base);
    // counts become the places of the rows' first tokens
    const uint32_t run = (a.per_class + SORT_THREADS - 1) / SORT_THREADS, l0 = min(threadIdx.x * run, a.per_class), l1 = min(l0 + run, a.per_class);
    uint32_t sum = 0;
    for (uint32_t l = l0; l < l1; ++l) sum += counts[l];
    uint32_t at = base + block_scan(sum, parts, &own);
    for (uint32_t l = l0; l < l1; ++l) {
        const uint32_t n = counts[l];
        a.segments[(uint64_t)mine * a.per_class + l] = Segment{at, n};
        counts[l] = at;
        at += n;
    }
    if (mine == mask && threadIdx.x == 0) *a.total = base + own;
    if (!own) return;
    // The block's tokens, in order, into a list; whenever that may be full, one warp places them, 32 at a time.
    uint32_t held = 0;
    auto place = [&]() {
        __syncthreads();
        if (threadIdx.x < 32) {
            for (uint32_t j = 0; j < held; j += 32) {
                const bool there = j + threadIdx.x < held;
                const uint2 e = there ? list[j + threadIdx.x] : make_uint2(0xffffffffu, 0);
                const uint32_t same = __match_any_sync(0xffffffffu, e.x);
                const uint32_t first = there ? counts[e.x] : 0;
                __syncwarp();
                if (there && (int)threadIdx.x == __ffs(same) - 1) counts[e.x] = first + __popc(same);
                __syncwarp();
                if (there) a.order[first + __popc(same & ((1u << threadIdx.x) - 1))] = e.y;
            }
        }
        __syncthreads();
        held = 0;
    };
    for (uint32_t i0 = 0; i0 < a.tokens; i0 += SORT_STEP) {
        const uint32_t i = i0 + 4 * threadIdx.x;
        int id[4];
        four_ids(a, i, id);
        uint32_t n = 0, all;
#pragma unroll
        for (int k = 0; k < 4; ++k) n += (uint32_t)id[k] < a.vocabulary && ((uint32_t)id[k] & mask) == mine;
        uint32_t to = held + block_scan(n, parts, &all);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if ((uint32_t)id[k] < a.vocabulary && ((uint32_t)id[k] & mask) == mine) list[to++] = make_uint2((uint32_t)id[k] >> a.shift, i + k);
        held += all;
        if (held + SORT_STEP > SORT_LIST) place();
    }
    if (held) place();
}

// ------------------------------------------------------------------------------------------- sums

constexpr uint32_t WINDOW = 64;  // tokens of a row that are summed at once
constexpr int SUM_FLIGHT = 8;    // rows of dy a thread has on their way

struct SumArgs {
    const void *dy, *base;
    void *out;
    const int *ids;
    const Segment *segments;
    const uint32_t *order, *total;
    float *partial;         // [2 x windows][cols]: what a window holds of the row it begins in, and of one that begins in it
    uint64_t dy_pitch, partial_pitch;
    uint32_t vocabulary, cols, shift, per_class, windows;
    int in_place;           // rows without a token are as they should be
    float scale;
    Layout l;
};

__device__ __forceinline__ Segment segment_of(const SumArgs &a, uint32_t row) {
    return a.segments[(uint64_t)(row & ((1u << a.shift) - 1)) * a.per_class + (row >> a.shift)];
}

// The sum of the rows order[p0 .. p1) from column `col` on, in order.
template <class T, int N>
__device__ __forceinline__ void sum_rows(const SumArgs &a, uint32_t col, uint32_t p0, uint32_t p1, float (&sum)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
    const T *dy = (const T *)a.dy + col;
    for (uint32_t p = p0; p < p1; p += SUM_FLIGHT) {
        float f[SUM_FLIGHT][N];
#pragma unroll
        for (int k = 0; k < SUM_FLIGHT; ++k)
            if (p + k < p1) load_values(dy + (uint64_t)a.order[p + k] * a.dy_pitch, f[k]);
#pragma unroll
        for (int k = 0; k < SUM_FLIGHT; ++k)
            if (p + k < p1) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += f[k][i];
            }
    }
}

// out = base + scale sum
template <class R, int N>
__device__ __forceinline__ void finish_row(const SumArgs &a, uint32_t row, uint32_t col, float (&sum)[N]) {
    const uint64_t at = (uint64_t)row * a.cols + col;
    float b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) b[i] = 0.f;
    if (a.base) load_values((const R *)a.base + at, b);
#pragma unroll
    for (int i = 0; i < N; ++i) b[i] += a.scale * sum[i];
    store_values((R *)a.out + at, b);
}

// Pieces of the rows of many tokens, then all other rows.
template <class T, class R, int N>
__global__ void __launch_bounds__(THREADS) lt_embedding_sum(const SumArgs a) {
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & (a.l.across - 1), beside = threadIdx.x / a.l.across;
    const uint64_t pieces = (uint64_t)a.windows * a.l.slices, units = pieces + (uint64_t)a.vocabulary * a.l.slices;
    const uint32_t total = *a.total;
    for (uint64_t u = (uint64_t)blockIdx.x * a.l.beside + beside; u < units; u += (uint64_t)gridDim.x * a.l.beside) {
        const uint64_t r = u < pieces ? u : u - pieces;
        const uint32_t row = row_of(a.l, r);
        const uint32_t col = ((uint32_t)(r - (uint64_t)row * a.l.slices) * a.l.across + lane) * N;
        if (col >= a.cols) continue;
        float sum[N];
        if (u < pieces) {
            const uint32_t p0 = row * WINDOW, p1 = min(p0 + WINDOW, total);
            if (p0 >= total) continue;
            const Segment s = segment_of(a, (uint32_t)a.ids[a.order[p0]]);
            if (s.count > WINDOW) {
                sum_rows<T>(a, col, p0, min(p1, s.start + s.count), sum);
                store_values(a.partial + 2 * (uint64_t)row * a.partial_pitch + col, sum);
            }
            const Segment e = segment_of(a, (uint32_t)a.ids[a.order[p1 - 1]]);
            if (e.count > WINDOW && e.start > p0) {
                sum_rows<T>(a, col, e.start, p1, sum);
                store_values(a.partial + (2 * (uint64_t)row + 1) * a.partial_pitch + col, sum);
            }
            continue;
        }
        const Segment s = segment_of(a, row);
        if (s.count > WINDOW || (s.count == 0 && a.in_place)) continue;
        sum_rows<T>(a, col, s.start, s.start + s.count, sum);
        finish_row<R>(a, row, col, sum);
    }
}

// Joins the pieces of rows of more than WINDOW tokens.  Such a row's piece in the window it begins in ends with the window, so
// at most one begins there.  A block has N x 32 columns and looks at all windows; its eight warps have a run of a row's
// windows each, and their sums are added up in order.
template <class R, int N>
__global__ void __launch_bounds__(THREADS) lt_embedding_join(const SumArgs a) {
    constexpr int WARPS = THREADS / 32;
    __shared__ float sums[WARPS][32 * N];
    __shared__ uint32_t rows[THREADS], n_rows;
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = (blockIdx.x * 32 + lane) * N;
    const uint32_t total = *a.total, windows = (total + WINDOW - 1) / WINDOW;
    for (uint32_t w0 = blockIdx.y * THREADS; w0 < windows; w0 += gridDim.y * THREADS) {
        __syncthreads();
        if (threadIdx.x == 0) n_rows = 0;
        __syncthreads();
        const uint32_t w = w0 + threadIdx.x;
        if (w < windows) {
            const uint32_t row = (uint32_t)a.ids[a.order[min((w + 1) * WINDOW, total) - 1]];
            const Segment s = segment_of(a, row);
            if (s.count > WINDOW && s.start >= w * WINDOW) rows[atomicAdd(&n_rows, 1u)] = row;  // (in any order: every row is a sum of its own)
        }
        __syncthreads();
        for (uint32_t k = 0; k < n_rows; ++k) {
            const uint32_t row = rows[k];
            const Segment s = segment_of(a, row);
            const uint32_t first = s.start / WINDOW, count = (s.start + s.count - 1) / WINDOW - first + 1, run = (count + WARPS - 1) / WARPS;
            float sum[N];
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = 0.f;
            if (col < a.cols) {
                const uint32_t i1 = min((warp + 1) * run, count);
#pragma unroll 8
                for (uint32_t i = warp * run; i < i1; ++i) {
                    float f[N];
                    load_values(a.partial + (2 * (uint64_t)(first + i) + (i == 0 && s.start % WINDOW ? 1 : 0)) * a.partial_pitch + col, f);
#pragma unroll
                    for (int x = 0; x < N; ++x) sum[x] += f[x];
                }
            }
            __syncthreads();  // `sums` may still be read from the row before
#pragma unroll
            for (int i = 0; i < N; ++i) sums[warp][lane * N + i] = sum[i];
            __syncthreads();
            if (warp == 0 && col < a.cols) {
#pragma unroll
                for (int w2 = 1; w2 < WARPS; ++w2)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += sums[w2][lane * N + i];
                finish_row<R>(a, row, col, sum);
            }
        }
    }
}

uint32_t sort_shift(uint64_t vocabulary) {
    uint32_t shift = 7;
    static_assert(SORT_CLASSES == 1u << 7, "");
    while (((vocabulary + (1ull << shift) - 1) >> shift) > SORT_COUNTS) ++shift;
    return shift;
}

// Where the scratch memory of embedding_grad holds what.
struct SumScratch {
    size_t segments, order, partial, bytes;
    uint64_t partial_pitch;
    explicit SumScratch(const LtOperator &o) {
        const uint32_t shift = sort_shift(o.vocabulary);
        const uint64_t rows = ((o.vocabulary + (1ull << shift) - 1) >> shift) << shift, windows = (o.rows + WINDOW - 1) / WINDOW;
        auto up = [](uint64_t b) { return (size_t)((b + 255) & ~255ull); };
        partial_pitch = (o.cols + 7) & ~7ull;
        segments = 256;  // (the total is at the beginning)
        order = segments + up(rows * sizeof(Segment));
        partial = order + up(o.rows * 4);
        bytes = partial + up(o.rows > WINDOW ? 2 * windows * partial_pitch * 4 : 0);
    }
};

template <class T, class R, int N>
cudaError_t launch_sums(SumArgs &a, uint64_t tokens, int sm_count, cudaStream_t stream, unsigned *launched) {
    a.l = layout_of((a.cols + N - 1) / N);
    const uint64_t units = ((uint64_t)a.windows + a.vocabulary) * a.l.slices, blocks = (units + a.l.beside - 1) / a.l.beside;
    const unsigned grid = (unsigned)std::min<uint64_t>(blocks, (uint64_t)sm_count * 8);
    cudaError_t e = launch_pdl(lt_embedding_sum<T, R, N>, grid, THREADS, (size_t)0, stream, a);
    if (e != cudaSuccess || tokens <= WINDOW) return e;
    ++*launched;
    // as many blocks for a slice as there may be rows to join, within reason
    const uint32_t across = (a.cols + 32 * N - 1) / (32 * N);
    const unsigned deep = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((a.windows + THREADS - 1) / THREADS, 2 * (uint64_t)sm_count / across));
    return launch_pdl_shared(lt_embedding_join<R, N>, dim3(across, deep), THREADS, (size_t)0, stream, a);
}

}  // namespace

cudaError_t lt_launch_embedding(const LtOperator &o, int sm_count, cudaStream_t stream) {
    LookupArgs a{};
    a.table = o.in[0];
    a.ids = (const int *)o.in[1];
    a.out = o.out[0];
    a.status = &o.status->embedding;
    a.pitch = o.pitch[0];
    a.tokens = (uint32_t)o.rows;
    a.vocabulary = (uint32_t)o.vocabulary;
    a.cols = (uint32_t)o.cols;
    a.scale = (float)lt_attr_double(o.attr[0]);
    const unsigned n = o.dtype == LT_BF16 ? 8 : 4;
    const bool wide = a.cols % n == 0 && a.pitch % n == 0 && is_aligned(a.table, 16) && is_aligned(a.out, 16);
    if (o.dtype == LT_BF16) return wide ? launch_lookup<__nv_bfloat16, 8>(a, sm_count, stream) : launch_lookup<__nv_bfloat16, 1>(a, sm_count, stream);
    return wide ? launch_lookup<float, 4>(a, sm_count, stream) : launch_lookup<float, 1>(a, sm_count, stream);
}

size_t lt_embedding_grad_scratch(const LtOperator &o) { return SumScratch(o).bytes; }

cudaError_t lt_launch_embedding_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    const SumScratch at(o);
    char *room = (char *)o.scratch;
    SortArgs s{};
    s.ids = (const int *)o.in[1];
    s.segments = (Segment *)(room + at.segments);
    s.order = (uint32_t *)(room + at.order);
    s.total = (uint32_t *)room;
    s.status = &o.status->embedding;
    s.tokens = (uint32_t)o.rows;
    s.vocabulary = (uint32_t)o.vocabulary;
    s.shift = sort_shift(o.vocabulary);
    s.per_class = (uint32_t)((o.vocabulary + (1ull << s.shift) - 1) >> s.shift);
    static std::atomic<uint64_t> ready{0};
    cudaError_t e = allow_shared(lt_token_sort, ((size_t)SORT_COUNTS + 2 * SORT_LIST) * 4, ready);
    if (e != cudaSuccess) return e;
    e = launch_pdl(lt_token_sort, 1u << s.shift, SORT_THREADS, ((size_t)((s.per_class + 1) & ~1u) + 2 * SORT_LIST) * 4, stream, s);
    if (e != cudaSuccess) return e;
    *launched = 2;
    SumArgs a{};
    a.dy = o.in[0];
    a.base = o.attr[1] ? o.in[2] : nullptr;
    a.out = o.out[0];
    a.ids = s.ids;
    a.segments = s.segments;
    a.order = s.order;
    a.total = s.total;
    a.partial = (float *)(room + at.partial);
    a.dy_pitch = o.pitch[0];
    a.partial_pitch = at.partial_pitch;
    a.vocabulary = s.vocabulary;
    a.cols = (uint32_t)o.cols;
    a.shift = s.shift;
    a.per_class = s.per_class;
    a.windows = (uint32_t)((o.rows > WINDOW ? o.rows + WINDOW - 1 : 0) / WINDOW);
    a.in_place = a.base == a.out;
    a.scale = (float)lt_attr_double(o.attr[2]);
    const unsigned n = o.dtype == LT_BF16 ? 8 : 4;
    const bool wide = a.cols % n == 0 && a.dy_pitch % n == 0 && is_aligned(a.dy, 16) && is_aligned(a.base, 16) && is_aligned(a.out, 16);
    if (o.dtype == LT_F32) return wide ? launch_sums<float, float, 4>(a, o.rows, sm_count, stream, launched) : launch_sums<float, float, 1>(a, o.rows, sm_count, stream, launched);
    if (o.gamma_dtype == LT_F32)
        return wide ? launch_sums<__nv_bfloat16, float, 8>(a, o.rows, sm_count, stream, launched) : launch_sums<__nv_bfloat16, float, 1>(a, o.rows, sm_count, stream, launched);
    return wide ? launch_sums<__nv_bfloat16, __nv_bfloat16, 8>(a, o.rows, sm_count, stream, launched)
                : launch_sums<__nv_bfloat16, __nv_bfloat16, 1>(a, o.rows, sm_count, stream, launched);
}
