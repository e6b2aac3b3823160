// The cross entropy of hidden states against a table of rows, and its gradient, without keeping the scores.
//
// z = scale x table^T [tokens, vocabulary]; lse_n = log sum_v exp z_nv; loss_n = lse_n - z[n, target_n].
// P = scale dloss_n (exp(z - lse_n) - [v = target_n]); dx = P table; dtable = P^T x.
//
// Scores are made a tile at a time.  The loss keeps of each tile the rows' maxima and sums of exponentials, which are joined in the
// tiles' order; the gradient makes P for a piece of the vocabulary at a time and multiplies it from both sides.
#include <algorithm>

#include "operator_device.cuh"

using namespace ltop;

namespace {

constexpr int TILE = 64, DEPTH = 16, THREADS = 256;

// A matrix in memory: element (i, k) at p + i * row + k * col.
struct Matrix {
    const void *p;
    uint64_t row, col;
};

struct ProductArgs {
    Matrix a, b;                // [m, depth], [n, depth]
    uint32_t m, n, depth;
    const int *targets;
    const float *lse, *dloss;
    float2 *tops;               // [tiles of n][m]
    float *target_score;        // [m]
    float *p;                   // [m][n]
    float *sum;                 // [m][n] so far, or null
    void *out;
    uint32_t first, vocabulary; // first: row of the table that column 0 of the product is
    float scale;
    unsigned int *status;
    int more;                   // more pieces follow: the sum goes back to `sum`
};

enum { TO_LOSS, TO_P, TO_RESULT };

template <class TA, class TB, class R, int TO>
__global__ void __launch_bounds__(THREADS) lt_product(const ProductArgs a) {
    __shared__ float sa[DEPTH][TILE + 1], sb[DEPTH][TILE + 1];
    pdl_release();
    pdl_wait();
    const uint32_t i0 = blockIdx.y * TILE, j0 = blockIdx.x * TILE, ti = threadIdx.x / 16, tj = threadIdx.x % 16;
    float c[4][4] = {};
    for (uint32_t k0 = 0; k0 < a.depth; k0 += DEPTH) {
        for (uint32_t x = threadIdx.x; x < TILE * DEPTH; x += THREADS) {
            const uint32_t i = x / DEPTH, k = x % DEPTH;
            const bool in = k0 + k < a.depth;
            sa[k][i] = in && i0 + i < a.m ? to_float(((const TA *)a.a.p)[(i0 + i) * a.a.row + (k0 + k) * a.a.col]) : 0.f;
            sb[k][i] = in && j0 + i < a.n ? to_float(((const TB *)a.b.p)[(j0 + i) * a.b.row + (k0 + k) * a.b.col]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < DEPTH; ++k)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) c[u][v] += sa[k][ti * 4 + u] * sb[k][tj * 4 + v];
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint32_t i = i0 + ti * 4 + u;
        const int target = TO != TO_RESULT && i < a.m ? a.targets[i] : -1;
        if (TO == TO_LOSS) {
            if (target >= 0 && (uint32_t)target >= a.vocabulary && threadIdx.x % 16 == 0) report(a.status);
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (j0 + tj * 4 + v < a.n) top = max_nan(top, c[u][v] * a.scale);
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (j0 + tj * 4 + v < a.n) {
                    sum += expf(c[u][v] * a.scale - (top == -INFINITY ? 0.f : top));
                    if (i < a.m && (int)(j0 + tj * 4 + v) == target) a.target_score[i] = c[u][v] * a.scale;
                }
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (tj == 0 && i < a.m) a.tops[(uint64_t)blockIdx.x * a.m + i] = make_float2(top, sum);
            continue;
        }
        if (i >= a.m) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint32_t j = j0 + tj * 4 + v;
            if (j >= a.n) continue;
            const uint64_t at = (uint64_t)i * a.n + j;
            if (TO == TO_P) {
                const bool counts = target >= 0 && (uint32_t)target < a.vocabulary;
                a.p[at] = counts ? (expf(c[u][v] * a.scale - a.lse[i]) - ((int)(a.first + j) == target ? 1.f : 0.f)) * a.dloss[i] * a.scale : 0.f;
            } else {
                const float s = c[u][v] + (a.sum && a.first ? a.sum[at] : 0.f);
                if (a.more) a.sum[at] = s;
                else ((R *)a.out)[at] = from_float<R>(s);
            }
        }
    }
}

__global__ void __launch_bounds__(256) lt_loss_join(const float2 *tops, const float *target_score, const int *targets, float *loss, float *lse, uint32_t tokens, uint32_t tiles, uint32_t vocabulary) {
    pdl_release();
    pdl_wait();
    const uint32_t n = blockIdx.x * 256 + threadIdx.x;
    if (n >= tokens) return;
    float top = -INFINITY, sum = 0.f;
    for (uint32_t t = 0; t < tiles; ++t) top = max_nan(top, tops[(uint64_t)t * tokens + n].x);
    for (uint32_t t = 0; t < tiles; ++t) {
        const float2 v = tops[(uint64_t)t * tokens + n];
        if (v.x != -INFINITY) sum += v.y * expf(v.x - top);
    }
    const float l = fabsf(top) == INFINITY ? top : top + logf(sum);
    if (lse) lse[n] = l;
    if (loss) loss[n] = targets[n] >= 0 && (uint32_t)targets[n] < vocabulary ? l - target_score[n] : 0.f;
}

// x without the rows that have no target
template <class T>
__global__ void __launch_bounds__(256) lt_loss_rows(const T *x, uint64_t pitch, const int *targets, T *to, uint32_t tokens, uint32_t cols, uint32_t vocabulary, unsigned int *status) {
    pdl_release();
    pdl_wait();
    for (uint32_t n = blockIdx.x; n < tokens; n += gridDim.x) {
        const bool counts = (uint32_t)targets[n] < vocabulary;
        if (targets[n] >= 0 && !counts && threadIdx.x == 0) report(status);
        for (uint32_t c = threadIdx.x; c < cols; c += 256) to[(uint64_t)n * cols + c] = counts ? x[n * pitch + c] : from_float<T>(0.f);
    }
}

uint32_t tiles_of(uint64_t n) { return (uint32_t)((n + TILE - 1) / TILE); }

constexpr uint64_t PIECE_BYTES = 64 << 20;

struct GradScratch {
    size_t rows, p, sum, bytes;
    uint64_t piece;
    explicit GradScratch(const LtOperator &o) {
        auto up = [](uint64_t b) { return (size_t)((b + 255) & ~255ull); };
        const uint64_t es = o.dtype == LT_BF16 ? 2 : 4;
        piece = std::max<uint64_t>(TILE, PIECE_BYTES / (4 * o.rows) / TILE * TILE);
        piece = std::min(piece, o.vocabulary);
        rows = 0;
        p = up(o.rows * o.cols * es);
        sum = p + up(o.rows * piece * 4);
        bytes = sum + up(o.rows * o.cols * 4);
    }
};

template <class T>
cudaError_t launch_loss(const LtOperator &o, cudaStream_t stream) {
    ProductArgs a{};
    a.a = Matrix{o.in[0], o.pitch[0], 1};
    a.b = Matrix{o.in[1], o.pitch[1], 1};
    a.m = (uint32_t)o.rows;
    a.n = a.vocabulary = (uint32_t)o.vocabulary;
    a.depth = (uint32_t)o.cols;
    a.targets = (const int *)o.in[2];
    a.target_score = (float *)o.scratch;
    a.tops = (float2 *)((char *)o.scratch + ((o.rows * 4 + 255) & ~255ull));
    a.status = &o.status->loss;
    a.scale = (float)lt_attr_double(o.attr[1]);
    const uint32_t tiles = tiles_of(a.n);
    const cudaError_t e = launch_pdl_grid(lt_product<T, T, T, TO_LOSS>, dim3(tiles, tiles_of(a.m)), THREADS, stream, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(lt_loss_join, (a.m + 255) / 256, 256, (size_t)0, stream, (const float2 *)a.tops, (const float *)a.target_score, a.targets, (float *)o.out[0], (float *)o.out[1], a.m, tiles,
                      a.vocabulary);
}

template <class T>
cudaError_t launch_loss_grad(const LtOperator &o, cudaStream_t stream, unsigned *launched) {
    const GradScratch at(o);
    char *room = (char *)o.scratch;
    const uint32_t tokens = (uint32_t)o.rows, cols = (uint32_t)o.cols, vocabulary = (uint32_t)o.vocabulary;
    const int *targets = (const int *)o.in[2];
    T *rows = (T *)(room + at.rows);
    cudaError_t e = launch_pdl(lt_loss_rows<T>, std::min(tokens, 4096u), 256, (size_t)0, stream, (const T *)o.in[0], o.pitch[0], targets, rows, tokens, cols, vocabulary, &o.status->loss);
    *launched = 1;
    for (uint32_t v0 = 0; v0 < vocabulary && e == cudaSuccess; v0 += (uint32_t)at.piece) {
        const uint32_t n = std::min((uint32_t)at.piece, vocabulary - v0);
        const T *table = (const T *)o.in[1] + v0 * o.pitch[1];
        ProductArgs a{};
        a.a = Matrix{rows, cols, 1};
        a.b = Matrix{table, o.pitch[1], 1};
        a.m = tokens;
        a.n = n;
        a.depth = cols;
        a.targets = targets;
        a.lse = (const float *)o.in[3];
        a.dloss = (const float *)o.in[4];
        a.p = (float *)(room + at.p);
        a.first = v0;
        a.vocabulary = vocabulary;
        a.scale = (float)lt_attr_double(o.attr[1]);
        e = launch_pdl_grid(lt_product<T, T, T, TO_P>, dim3(tiles_of(n), tiles_of(tokens)), THREADS, stream, a);
        ++*launched;
        if (o.out[0] && e == cudaSuccess) {
            ProductArgs d{};
            d.a = Matrix{a.p, n, 1};
            d.b = Matrix{table, 1, o.pitch[1]};
            d.m = tokens;
            d.n = cols;
            d.depth = n;
            d.sum = (float *)(room + at.sum);
            d.first = v0;
            d.out = o.out[0];
            d.more = v0 + n < vocabulary;
            e = launch_pdl_grid(lt_product<float, T, T, TO_RESULT>, dim3(tiles_of(cols), tiles_of(tokens)), THREADS, stream, d);
            ++*launched;
        }
        if (o.out[1] && e == cudaSuccess) {
            ProductArgs d{};
            d.a = Matrix{a.p, 1, n};
            d.b = Matrix{rows, 1, cols};
            d.m = n;
            d.n = cols;
            d.depth = tokens;
            d.out = (T *)o.out[1] + (uint64_t)v0 * cols;
            e = launch_pdl_grid(lt_product<float, T, T, TO_RESULT>, dim3(tiles_of(cols), tiles_of(n)), THREADS, stream, d);
            ++*launched;
        }
    }
    return e;
}

}  // namespace

size_t lt_vocabulary_loss_scratch(const LtOperator &o, int) { return ((o.rows * 4 + 255) & ~255ull) + (size_t)tiles_of(o.vocabulary) * o.rows * sizeof(float2); }
size_t lt_vocabulary_loss_grad_scratch(const LtOperator &o, int) { return GradScratch(o).bytes; }

cudaError_t lt_launch_vocabulary_loss(const LtOperator &o, int, cudaStream_t stream, unsigned *launched) {
    *launched = 2;
    return o.dtype == LT_BF16 ? launch_loss<__nv_bfloat16>(o, stream) : launch_loss<float>(o, stream);
}

cudaError_t lt_launch_vocabulary_loss_grad(const LtOperator &o, int, cudaStream_t stream, unsigned *launched) {
    return o.dtype == LT_BF16 ? launch_loss_grad<__nv_bfloat16>(o, stream, launched) : launch_loss_grad<float>(o, stream, launched);
}
