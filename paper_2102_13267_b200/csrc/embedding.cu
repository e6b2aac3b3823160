// Looking tokens up in a table [vocabulary, columns], and the gradient of that.
//
// Both move every value once and are bound by memory.  The gradient of row v is the sum of the rows of dy whose token is v.
// Tokens are sorted first (lt_token_sort); the sorted order is cut into windows of tokens, whatever rows they belong to, so
// that a token that makes up much of a text is no more work for anyone than others are (lt_embedding_sum).  A row whose tokens
// lie in one window is finished there, what a window holds of others is left as a partial sum, and those are joined in order
// (lt_embedding_join): no atomics on values, and the same result every time.
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

// The same as they lie in memory: what is on its way takes no more registers than bytes.
template <class T, int N>
struct Piece {
    static constexpr int WORDS = N * sizeof(T) / 16;
    uint4 v[WORDS > 0 ? WORDS : 1];
    __device__ __forceinline__ void load(const T *from) {
        if constexpr (N == 1) {
            const float f = to_float(*from);
            v[0].x = __float_as_uint(f);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) v[i] = reinterpret_cast<const uint4 *>(from)[i];
        }
    }
    __device__ __forceinline__ void add_to(float (&f)[N]) const {
        if constexpr (N == 1) {
            f[0] += __uint_as_float(v[0].x);
        } else {
            constexpr int PER = 16 / sizeof(T);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                float g[PER];
                unpack(v[i], g);
#pragma unroll
                for (int k = 0; k < PER; ++k) f[i * PER + k] += g[k];
            }
        }
    }
};

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

// Bound by memory: 32768 tokens of 32000 x 4096 bf16 take 80 us, 6.6 TB/s of named rows and results (rows named twice come from the L2 cache).  A step of
// few tokens takes what recording and launching do, 4 us.
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
constexpr int SORT_VECTORS = 8;                   // of four tokens, that a thread has at once
constexpr uint32_t SORT_STEP = 4 * SORT_VECTORS * SORT_THREADS;
constexpr uint32_t SORT_LIST = 8192;
constexpr uint32_t SORT_COUNTS = 2048;            // rows of a class, at most
constexpr uint32_t SORT_PLACERS = 16;             // warps that place a long list
constexpr uint32_t SORT_CLASSES = 128;            // at least

struct SortArgs {
    const int *ids;
    uint32_t *counts;       // of a row's tokens: [classes][rows of a class]
    uint4 *order;           // row by row: a token, its row, where the row's tokens start, and how many they are
    uint32_t *total;        // how many tokens name a row
    unsigned int *status;
    uint32_t tokens, vocabulary, shift, per_class;  // classes: 2^shift
};

// Looks at the thread's tokens of the step that begins at `step`, four at a time, neighbours' beside them: a bit for each that
// belongs to class `mine`; *below: how many belong to classes before.
__device__ __forceinline__ uint32_t look(const SortArgs &a, uint32_t step, uint32_t mine, uint32_t *below) {
    const bool wide = ((uintptr_t)a.ids & 15) == 0;
    const uint32_t mask = (1u << a.shift) - 1;
    int id[SORT_VECTORS][4];
#pragma unroll
    for (int v = 0; v < SORT_VECTORS; ++v) {
        const uint32_t i = step + 4 * (v * SORT_THREADS + threadIdx.x);
#pragma unroll
        for (int k = 0; k < 4; ++k) id[v][k] = -1;
        if (step + v * 4 * SORT_THREADS >= a.tokens) continue;  // (the same for all)
        if (wide && i + 4 <= a.tokens) {
            const int4 x = *reinterpret_cast<const int4 *>(a.ids + i);
            id[v][0] = x.x, id[v][1] = x.y, id[v][2] = x.z, id[v][3] = x.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < a.tokens) id[v][k] = a.ids[i + k];
        }
    }
    uint32_t bits = 0;
#pragma unroll
    for (int v = 0; v < SORT_VECTORS; ++v) {
        if (step + v * 4 * SORT_THREADS >= a.tokens) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t c = (uint32_t)id[v][k] < a.vocabulary ? (uint32_t)id[v][k] & mask : 0xffffffffu;
            *below += c < mine;
            bits |= (uint32_t)(c == mine) << (4 * v + k);
            if (mine == 0 && c > mask && id[v][k] >= 0) report(a.status);
        }
    }
    return bits;
}
// The token of bit x
__device__ __forceinline__ uint32_t token_of(uint32_t step, uint32_t x) { return step + 4 * ((x >> 2) * SORT_THREADS + threadIdx.x) + (x & 3); }

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
// once per class costs little beside rows of hundreds of values: 4 bytes and a few instructions each (16384 tokens 12 us, 301 7 us, most of
// it the way from one dependent read and barrier to the next).
__global__ void __launch_bounds__(SORT_THREADS) lt_token_sort(const SortArgs a) {
    extern __shared__ uint32_t places[];  // [rows of a class]: where the row's next token goes; [one more]: where its first is; [PLACERS][rows]; uint2 [LIST]
    __shared__ uint32_t parts[32], vector_parts[SORT_VECTORS][32];
    const uint32_t room = (a.per_class + 4) & ~3u;
    uint32_t *starts = places + room;
    uint16_t *shares = reinterpret_cast<uint16_t *>(starts + room);
    uint2 *list = reinterpret_cast<uint2 *>(shares + SORT_PLACERS * room);
    const uint32_t mine = blockIdx.x, mask = (1u << a.shift) - 1;
    pdl_release();
    for (uint32_t l = threadIdx.x; l < a.per_class; l += SORT_THREADS) places[l] = 0;
    __syncthreads();
    pdl_wait();
    uint32_t below = 0, bits = 0;
    for (uint32_t step = 0; step < a.tokens; step += SORT_STEP) {
        bits = look(a, step, mine, &below);
        for (uint32_t m = bits; m; m &= m - 1) atomicAdd(&places[(uint32_t)a.ids[token_of(step, __ffs(m) - 1)] >> a.shift], 1u);
    }
    uint32_t base, own;
    block_scan(below, parts, &base);
    // counts become the places of the rows' first tokens
    const uint32_t run = (a.per_class + SORT_THREADS - 1) / SORT_THREADS, l0 = min(threadIdx.x * run, a.per_class), l1 = min(l0 + run, a.per_class);
    uint32_t sum = 0;
    for (uint32_t l = l0; l < l1; ++l) sum += places[l];
    uint32_t at = base + block_scan(sum, parts, &own);
    for (uint32_t l = l0; l < l1; ++l) {
        const uint32_t n = places[l];
        a.counts[(uint64_t)mine * a.per_class + l] = n;
        places[l] = starts[l] = at;
        at += n;
    }
    if (threadIdx.x == 0) starts[a.per_class] = base + own;
    if (mine == mask && threadIdx.x == 0) *a.total = base + own;
    if (!own) return;
    // The block's tokens go into a list, in order, as many as it holds at a time, and from there to their places, 32 at once.
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, before_me = (1u << lane) - 1;
    auto put = [&](const uint2 &e, uint32_t to) { a.order[to] = make_uint4(e.y, (e.x << a.shift) + mine, starts[e.x], starts[e.x + 1] - starts[e.x]); };
    auto fetch = [&](uint32_t x, uint32_t end) { return x < end ? list[x] : make_uint2(0xffffffffu, 0); };
    // a short list: one warp; who has the same row is found for several times 32 ahead of the places, which follow one another
    auto place_short = [&](uint32_t held) {
        constexpr int AHEAD = 4;
        for (uint32_t j = 0; j < held; j += 32 * AHEAD) {
            uint2 e[AHEAD];
            uint32_t same[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) e[k] = fetch(j + 32 * k + lane, held);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) same[k] = __match_any_sync(0xffffffffu, e[k].x);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const bool there = e[k].x != 0xffffffffu;
                const uint32_t first = there ? places[e[k].x] : 0;
                __syncwarp();
                if (there && (int)lane == __ffs(same[k]) - 1) places[e[k].x] = first + __popc(same[k]);
                __syncwarp();
                if (there) put(e[k], first + __popc(same[k] & before_me));
            }
        }
    };
    // a long one: warps have a run of it each, count their shares of the rows, and place them behind those of the warps before
    auto place_long = [&](uint32_t held) {
        const uint32_t run = (held + 32 * SORT_PLACERS - 1) / (32 * SORT_PLACERS) * 32, j0 = min(warp * run, held), j1 = warp < SORT_PLACERS ? min(j0 + run, held) : j0;
        uint16_t *share = shares + warp * room;
        for (uint32_t x = threadIdx.x; x < SORT_PLACERS * room; x += SORT_THREADS) shares[x] = 0;
        __syncthreads();
        for (uint32_t j = j0; j < j1; j += 32) {
            const uint2 e = fetch(j + lane, j1);
            const uint32_t same = __match_any_sync(0xffffffffu, e.x);
            if (e.x != 0xffffffffu && (int)lane == __ffs(same) - 1) share[e.x] += (uint16_t)__popc(same);
            __syncwarp();
        }
        __syncthreads();
        for (uint32_t l = threadIdx.x; l < a.per_class; l += SORT_THREADS) {
            uint32_t sum = 0;
            for (uint32_t w = 0; w < SORT_PLACERS; ++w) {
                const uint32_t n = shares[w * room + l];
                shares[w * room + l] = (uint16_t)sum;
                sum += n;
            }
        }
        __syncthreads();
        for (uint32_t j = j0; j < j1; j += 32) {
            const uint2 e = fetch(j + lane, j1);
            const uint32_t same = __match_any_sync(0xffffffffu, e.x);
            const bool there = e.x != 0xffffffffu;
            const uint32_t first = there ? share[e.x] : 0;
            __syncwarp();
            if (there && (int)lane == __ffs(same) - 1) share[e.x] = (uint16_t)(first + __popc(same));
            __syncwarp();
            if (there) put(e, places[e.x] + first + __popc(same & before_me));
        }
        __syncthreads();
        for (uint32_t l = threadIdx.x; l < a.per_class; l += SORT_THREADS) places[l] += shares[(SORT_PLACERS - 1) * room + l];
    };
    for (uint32_t step = 0; step < a.tokens; step += SORT_STEP) {
        if (a.tokens > SORT_STEP) bits = look(a, step, mine, &below);
        // how many of the block's tokens lie before each vector of the thread's: within the warp (a byte for each vector), then by warps
        uint32_t mine_of[2] = {0, 0};
#pragma unroll
        for (int v = 0; v < SORT_VECTORS; ++v) mine_of[v / 4] |= (uint32_t)__popc(bits >> (4 * v) & 15) << (v % 4 * 8);
        uint32_t upto[2] = {mine_of[0], mine_of[1]};
        static_assert(SORT_VECTORS == 8 && 32 * 4 < 256, "bytes of two words");
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o0 = __shfl_up_sync(0xffffffffu, upto[0], d), o1 = __shfl_up_sync(0xffffffffu, upto[1], d);
            if (lane >= (uint32_t)d) upto[0] += o0, upto[1] += o1;
        }
        if (lane == 31) {
#pragma unroll
            for (int v = 0; v < SORT_VECTORS; ++v) vector_parts[v][warp] = upto[v / 4] >> (v % 4 * 8) & 255;
        }
        __syncthreads();
        uint32_t all;
        const uint32_t part = threadIdx.x < 32 * SORT_VECTORS ? vector_parts[warp][lane] : 0, ahead = block_scan(part, parts, &all);
        if (threadIdx.x < 32 * SORT_VECTORS) vector_parts[warp][lane] = ahead;
        __syncthreads();
        for (uint32_t r = 0; r < all; r += SORT_LIST) {
            for (uint32_t m = bits; m; m &= m - 1) {
                const uint32_t x = __ffs(m) - 1, v = x >> 2, i = token_of(step, x);
                const uint32_t to = vector_parts[v][warp] + ((v < 4 ? upto[0] - mine_of[0] : upto[1] - mine_of[1]) >> (v % 4 * 8) & 255) + __popc(bits & (15u << (4 * v)) & ((1u << x) - 1)) - r;
                if (to < SORT_LIST) list[to] = make_uint2((uint32_t)a.ids[i] >> a.shift, i);
            }
            __syncthreads();
            const uint32_t held = min(all - r, SORT_LIST);
            if (held > 512) place_long(held);
            else if (warp == 0) place_short(held);
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------------------------------- sums

constexpr uint32_t MOST_WINDOW = 64;  // tokens of the sorted order that are summed at once, at most
constexpr uint32_t EMPTY_ROWS = 16;

struct SumArgs {
    const void *dy, *base;
    void *out;
    const uint32_t *counts, *total;
    const uint4 *order;
    float *partial;         // [2 x windows][cols]: what a window holds of the row it begins in, and of the one it ends in
    uint64_t dy_pitch, partial_pitch;
    uint32_t vocabulary, cols, shift, per_class, window, windows, window_blocks;  // window: tokens, a power of two from 8 on
    float scale;
    Layout l;
};

// The first blocks: a window's rows of dy, FLIGHT of them (and of the base's rows that end there) on their way at a time,
// whichever rows of the table they belong to.
// The other blocks, if rows without a token have to be written: EMPTY_ROWS rows of a class each.
// Bound by memory: 16384 x 4096 bf16 into 32000 rows 56 us, 340 MB at 6.1 TB/s; with sort and join 74 us (a unit of work per row of the table:
// 385, since one token may be a fifth of a text; windows of 64 without rows of the base ahead: 88).
template <class T, class R, int N, bool BASE>
__global__ void __launch_bounds__(THREADS, BASE && sizeof(R) > sizeof(T) ? 3 : 4) lt_embedding_sum(const SumArgs a) {
    constexpr int FLIGHT = BASE ? 4 : 8;
    __shared__ uint32_t tokens[THREADS / 32][MOST_WINDOW], rows[THREADS / 32][MOST_WINDOW];  // rows: with the highest bit where a row ends
    __shared__ bool begins[THREADS / 32];  // does a row begin with the window?
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & (a.l.across - 1), beside = threadIdx.x / a.l.across;
    if (blockIdx.x >= a.window_blocks) {
        const uint64_t u = (uint64_t)(blockIdx.x - a.window_blocks) * a.l.beside + beside;
        const uint32_t batch = row_of(a.l, u), batches = (a.per_class + EMPTY_ROWS - 1) / EMPTY_ROWS;
        const uint32_t col = ((uint32_t)(u - (uint64_t)batch * a.l.slices) * a.l.across + lane) * N, c = batch / batches, l0 = (batch - c * batches) * EMPTY_ROWS;
        if (c >> a.shift) return;
        const uint32_t l = l0 + (threadIdx.x & 31);
        uint32_t empty = __ballot_sync(0xffffffffu, (threadIdx.x & 31) < EMPTY_ROWS && l < a.per_class && (l << a.shift) + c < a.vocabulary && a.counts[(uint64_t)c * a.per_class + l] == 0);
        if (col >= a.cols) return;
#pragma unroll 4
        for (uint32_t k = 0; k < EMPTY_ROWS; ++k) {
            if (!(empty >> k & 1)) continue;
            const uint64_t at = (uint64_t)(((l0 + k) << a.shift) + c) * a.cols + col;
            float f[N] = {};
            if (BASE) load_values((const R *)a.base + at, f);
            store_values((R *)a.out + at, f);
        }
        return;
    }
    const uint32_t total = *a.total;
    const uint64_t u = (uint64_t)blockIdx.x * a.l.beside + beside;
    const uint32_t w = row_of(a.l, u), p0 = w * a.window, n = w < a.windows && p0 < total ? min(a.window, total - p0) : 0;
    const uint32_t col = ((uint32_t)(u - (uint64_t)w * a.l.slices) * a.l.across + lane) * N;
    for (uint32_t p = lane; p < n; p += a.l.across) {
        const uint4 e = a.order[p0 + p];
        tokens[beside][p] = e.x;
        rows[beside][p] = e.y | (e.z + e.w == p0 + p + 1 ? 0x80000000u : 0);
        if (p == 0) begins[beside] = e.z == p0;
    }
    __syncthreads();
    if (!n || col >= a.cols) return;
    const T *dy = (const T *)a.dy + col;
    const uint32_t *token = tokens[beside], *row = rows[beside];
    bool begun = begins[beside];
    float sum[N] = {};
    for (uint32_t p = 0; p < n; p += FLIGHT) {
        Piece<T, N> f[FLIGHT];
        Piece<R, N> base[BASE ? FLIGHT : 1];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (p + k >= n) break;
            f[k].load(dy + (uint64_t)token[p + k] * a.dy_pitch);
            if (BASE && row[p + k] >> 31) base[BASE ? k : 0].load((const R *)a.base + (uint64_t)(row[p + k] & 0x7fffffffu) * a.cols + col);
        }
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (p + k >= n) break;
            f[k].add_to(sum);
            if (!(row[p + k] >> 31)) continue;
            if (begun) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] *= a.scale;
                if (BASE) base[BASE ? k : 0].add_to(sum);
                store_values((R *)a.out + (uint64_t)(row[p + k] & 0x7fffffffu) * a.cols + col, sum);
            } else {
                store_values(a.partial + 2 * (uint64_t)w * a.partial_pitch + col, sum);
            }
            begun = true;
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = 0.f;
        }
    }
    if (!(row[n - 1] >> 31)) store_values(a.partial + (2 * (uint64_t)w + (begun ? 1 : 0)) * a.partial_pitch + col, sum);
}

// Joins the partial sums of rows that end in another window than they begin in: at most one begins in a window.  A warp has a
// window and 32 pieces of the columns; where a row has many windows, the block's warps take a run of them each and their sums
// are added up in order.  (The 16384 tokens above: 9 us.)
constexpr uint32_t JOIN_ALONE = 8;  // windows of a row
template <class R, int N>
__global__ void __launch_bounds__(THREADS, 4) lt_embedding_join(const SumArgs a) {
    constexpr uint32_t WARPS = THREADS / 32;
    __shared__ float sums[WARPS][32 * N];
    __shared__ uint32_t many[WARPS], many_rows[WARPS];
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slices = (a.cols + 32 * N - 1) / (32 * N), w0 = blockIdx.x / slices * WARPS, w = w0 + warp,
                   col = (blockIdx.x % slices * 32 + lane) * N;
    const uint32_t total = *a.total;
    auto add = [&](uint32_t first, uint32_t i0, uint32_t i1, float (&sum)[N]) {  // windows first + i0 .. first + i1; the first holds the row's beginning
        constexpr int FLIGHT = N == 8 ? 4 : 8;
        for (uint32_t i = i0; i < i1; i += FLIGHT) {
            Piece<float, N> f[FLIGHT];
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
                if (i + k < i1) f[k].load(a.partial + (2 * (uint64_t)(first + i + k) + (i + k == 0 ? 1 : 0)) * a.partial_pitch + col);
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
                if (i + k < i1) f[k].add_to(sum);
        }
    };
    // out = base + scale sum, the base being on its way while the sum is made
    Piece<R, N> base;
    auto ask = [&](uint32_t row) {
        if (a.base) base.load((const R *)a.base + (uint64_t)row * a.cols + col);
    };
    auto finish = [&](uint32_t row, float (&sum)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] *= a.scale;
        if (a.base) base.add_to(sum);
        store_values((R *)a.out + (uint64_t)row * a.cols + col, sum);
    };
    uint32_t count = 0, row = 0xffffffffu;
    const uint32_t begin = w * a.window, end = begin + a.window;
    if (w < a.windows && end < total) {
        const uint4 e = a.order[end - 1];
        row = e.y;
        if (e.z >= begin && e.z + e.w > end) count = (e.z + e.w - 1) / a.window - w + 1;
    }
    if (lane == 0) {
        many[warp] = count > JOIN_ALONE ? count : 0;
        many_rows[warp] = row;
    }
    if (count && count <= JOIN_ALONE && col < a.cols) {
        float sum[N] = {};
        ask(row);
        add(w, 0, count, sum);
        finish(row, sum);
    }
    __syncthreads();
    for (uint32_t k = 0; k < WARPS; ++k) {
        if (!many[k]) continue;
        const uint32_t run = (many[k] + WARPS - 1) / WARPS;
        float sum[N] = {};
        if (warp == 0 && col < a.cols) ask(many_rows[k]);
        if (col < a.cols) add(w0 + k, warp * run, min((warp + 1) * run, many[k]), sum);
        __syncthreads();  // `sums` may still be read from the row before
#pragma unroll
        for (int i = 0; i < N; ++i) sums[warp][lane * N + i] = sum[i];
        __syncthreads();
        if (warp == 0 && col < a.cols) {
#pragma unroll
            for (uint32_t o = 1; o < WARPS; ++o)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += sums[o][lane * N + i];
            finish(many_rows[k], sum);
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
    size_t counts, order, partial, bytes;
    uint64_t partial_pitch;
    uint32_t window;
    SumScratch(const LtOperator &o, int sm_count) {
        // Few tokens: smaller windows, so that there are some for every SM (301 x 200 f32: 12 us with 8 tokens, 18 with 64); many:
        // larger ones, which leave fewer partial sums.
        window = MOST_WINDOW;
        while (window > 8 && o.rows * o.cols * (o.dtype == LT_BF16 ? 2 : 4) / window < (uint64_t)sm_count * 4 * THREADS * 16) window /= 2;
        const uint32_t shift = sort_shift(o.vocabulary);
        const uint64_t rows = ((o.vocabulary + (1ull << shift) - 1) >> shift) << shift, windows = (o.rows + window - 1) / window;
        auto up = [](uint64_t b) { return (size_t)((b + 255) & ~255ull); };
        partial_pitch = (o.cols + 7) & ~7ull;
        counts = 256;  // (the total is at the beginning)
        order = counts + up(rows * 4);
        partial = order + up(o.rows * 16);
        bytes = partial + up(windows > 1 ? 2 * windows * partial_pitch * 4 : 0);
    }
};

template <class T, class R, int N>
cudaError_t launch_sums(SumArgs &a, int sm_count, cudaStream_t stream, unsigned *launched) {
    a.l = layout_of((a.cols + N - 1) / N);
    auto blocks = [&](uint64_t units) { return (units * a.l.slices + a.l.beside - 1) / a.l.beside; };
    const uint64_t windows = blocks(a.windows), batches = a.base && a.base == a.out ? 0 : blocks((uint64_t)((a.per_class + EMPTY_ROWS - 1) / EMPTY_ROWS) << a.shift);
    if (windows + batches >= (1ull << 31)) return cudaErrorInvalidValue;
    a.window_blocks = (uint32_t)windows;
    const cudaError_t e = a.base ? launch_pdl(lt_embedding_sum<T, R, N, true>, (unsigned)(windows + batches), THREADS, (size_t)0, stream, a)
                                 : launch_pdl(lt_embedding_sum<T, R, N, false>, (unsigned)(windows + batches), THREADS, (size_t)0, stream, a);
    if (e != cudaSuccess || a.windows <= 1) return e;
    ++*launched;
    const uint64_t join = (uint64_t)((a.cols + 32 * N - 1) / (32 * N)) * ((a.windows + THREADS / 32 - 1) / (THREADS / 32));
    return launch_pdl(lt_embedding_join<R, N>, (unsigned)join, THREADS, (size_t)0, stream, a);
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

size_t lt_embedding_grad_scratch(const LtOperator &o, int sm_count) { return SumScratch(o, sm_count).bytes; }

cudaError_t lt_launch_embedding_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    const SumScratch at(o, sm_count);
    char *room = (char *)o.scratch;
    SortArgs s{};
    s.ids = (const int *)o.in[1];
    s.counts = (uint32_t *)(room + at.counts);
    s.order = (uint4 *)(room + at.order);
    s.total = (uint32_t *)room;
    s.status = &o.status->embedding;
    s.tokens = (uint32_t)o.rows;
    s.vocabulary = (uint32_t)o.vocabulary;
    s.shift = sort_shift(o.vocabulary);
    s.per_class = (uint32_t)((o.vocabulary + (1ull << s.shift) - 1) >> s.shift);
    static std::atomic<uint64_t> ready{0};
    auto shared = [](uint32_t rows) {
        const size_t room = (rows + 4) & ~3u;
        return room * (4 + 4 + 2 * SORT_PLACERS) + SORT_LIST * 8;
    };
    cudaError_t e = allow_shared(lt_token_sort, shared(SORT_COUNTS), ready);
    if (e != cudaSuccess) return e;
    e = launch_pdl(lt_token_sort, 1u << s.shift, SORT_THREADS, shared(s.per_class), stream, s);
    if (e != cudaSuccess) return e;
    *launched = 2;
    SumArgs a{};
    a.dy = o.in[0];
    a.base = o.attr[1] ? o.in[2] : nullptr;
    a.out = o.out[0];
    a.counts = s.counts;
    a.order = s.order;
    a.total = s.total;
    a.partial = (float *)(room + at.partial);
    a.dy_pitch = o.pitch[0];
    a.partial_pitch = at.partial_pitch;
    a.vocabulary = s.vocabulary;
    a.cols = (uint32_t)o.cols;
    a.shift = s.shift;
    a.per_class = s.per_class;
    a.window = at.window;
    a.windows = (uint32_t)((o.rows + at.window - 1) / at.window);
    a.scale = (float)lt_attr_double(o.attr[2]);
    const unsigned n = o.dtype == LT_BF16 ? 8 : 4;
    const bool wide = a.cols % n == 0 && a.dy_pitch % n == 0 && is_aligned(a.dy, 16) && is_aligned(a.base, 16) && is_aligned(a.out, 16);
    if (o.dtype == LT_F32) return wide ? launch_sums<float, float, 4>(a, sm_count, stream, launched) : launch_sums<float, float, 1>(a, sm_count, stream, launched);
    if (o.gamma_dtype == LT_F32)
        return wide ? launch_sums<__nv_bfloat16, float, 8>(a, sm_count, stream, launched) : launch_sums<__nv_bfloat16, float, 1>(a, sm_count, stream, launched);
    return wide ? launch_sums<__nv_bfloat16, __nv_bfloat16, 8>(a, sm_count, stream, launched)
                : launch_sums<__nv_bfloat16, __nv_bfloat16, 1>(a, sm_count, stream, launched);
}
