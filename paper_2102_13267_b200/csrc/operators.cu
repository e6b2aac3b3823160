// Kernels of the transformer operators that move every value once: rotary positions, appending to a paged key-value
// cache, the root-mean-square norm (with the residual's addition and an 8-bit output) and its gradient.  The attention
// that reads the cache is in attention.cu, what follows tokens into a table in embedding.cu and vocabulary_loss.cu.
#include <cuda_fp8.h>

#include <algorithm>
#include <cstring>
#include <deque>
#include <mutex>
#include <type_traits>

#include "operator_device.cuh"

using namespace ltop;

static __device__ unsigned int lt_operator_arrivals[LT_ARRIVALS];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;
void *g_arrivals[kMaxDevices];

// Status words of contexts, in host memory that every device writes to and that lasts as long as the process: a graph may
// still report to the word of a context that is gone.  So a word that is given back waits until all others have been used.
// The first one is shared by contexts that find no free one.
constexpr size_t kStatusWords = 4096;
LtOperatorStatus *g_status;
std::deque<LtOperatorStatus *> g_status_free;

// Address of a device variable on the current device, looked up once per device.
template <class S>
cudaError_t address_of(const S &symbol, void **known, void **out) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 0 || device >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> hold(g_lock);
    if (!known[device]) {
        void *p = nullptr;
        e = cudaGetSymbolAddress(&p, symbol);
        if (e != cudaSuccess) return e;
        known[device] = p;
    }
    *out = known[device];
    return cudaSuccess;
}

inline bool is_aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// ------------------------------------------------------------------------------------------- rotary, cache_append

struct TurnArgs {
    const void *x, *v;          // v: cache_append only
    void *out;                  // rotary: the result; cache_append: the cache
    const int *positions, *slots;
    const uint2 *frequencies;
    unsigned int *status;
    uint64_t tokens, x_pitch, v_pitch;
    uint64_t page_stride, value_offset, token_stride, head_stride;  // of the cache, in elements
    uint32_t heads, dim, pairs, page;
    uint64_t n_slots;
    float scale;
    int interleaved, inverse;
};

// Where token t goes: the element index of its first head's first value (rotary: dense), or false when it goes nowhere.
template <bool APPEND>
__device__ __forceinline__ bool destination(const TurnArgs &a, uint64_t t, uint64_t *at) {
    if (!APPEND) {
        *at = t * a.heads * a.dim;
        return true;
    }
    const int slot = a.slots[t];
    if (slot < 0) return false;
    if ((uint64_t)slot >= a.n_slots) {
        report(a.status);
        return false;
    }
    const uint32_t p = (uint32_t)slot / a.page, off = (uint32_t)slot - p * a.page;
    *at = (uint64_t)p * a.page_stride + (uint64_t)off * a.token_stride;
    return true;
}

// Any shape and alignment: a thread has one pair (or one value that passes through) of a token, and walks the heads.
template <class T, bool APPEND>
__global__ void __launch_bounds__(256) lt_turn_any(const TurnArgs a) {
    pdl_release();
    pdl_wait();
    const T *x = (const T *)a.x, *v = (const T *)a.v;
    T *out = (T *)a.out;
    const uint32_t per = a.dim - a.pairs;  // pairs and single values of a head
    const uint64_t total = a.tokens * per;
    const uint64_t hs = APPEND ? a.head_stride : a.dim;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
        const uint64_t t = i / per;
        const uint32_t e = (uint32_t)(i - t * per);
        uint64_t at;
        if (!destination<APPEND>(a, t, &at)) continue;
        uint32_t i0 = e + a.pairs, i1 = i0;  // a value that passes through
        float2 cs = make_float2(1.f, 0.f);
        if (e < a.pairs) {
            cs = turn(a.positions[t], a.frequencies[e], a.scale, a.inverse != 0);
            i0 = a.interleaved ? 2 * e : e;
            i1 = a.interleaved ? 2 * e + 1 : e + a.pairs;
        }
        for (uint32_t h = 0; h < a.heads; ++h) {
            const T *src = x + t * a.x_pitch + (uint64_t)h * a.dim;
            T *dst = out + at + (uint64_t)h * hs;
            const T p = src[i0], q = src[i1];
            if (i0 != i1) {
                const float fp = to_float(p), fq = to_float(q);
                dst[i0] = from_float<T>(fp * cs.x - fq * cs.y);
                dst[i1] = from_float<T>(fp * cs.y + fq * cs.x);
            } else {
                dst[i0] = p;
            }
            if (APPEND) {
                const T *vs = v + t * a.v_pitch + (uint64_t)h * a.dim;
                dst[a.value_offset + i0] = vs[i0];
                if (i0 != i1) dst[a.value_offset + i1] = vs[i1];
            }
        }
    }
}

// (tokens in flight per thread and stages ahead, on rotary 8192 x 32 x 128 and append 8192 x 8 x 128, bf16, both with the
// next kernel let in at once: 4 and 1:
// 25.7 and 14.4 us; 2 and 2: 25.6 and 15.5; 2 and 3: 26.3 and 16.6; 1 and 4: 25.4 and 18.5; 4 and 2: 27.7 and 16.3)
constexpr int TURN_THREADS = 256, TURN_FLIGHT = 4, TURN_STAGES = 1;
constexpr uint32_t TURN_ANGLES = 2048;  // of a batch, at most: 16 KB, twice
__host__ __device__ constexpr size_t turn_ring(int bytes) { return (size_t)TURN_STAGES * TURN_FLIGHT * 2 * TURN_THREADS * bytes; }

struct TurnShape {
    uint32_t batch;             // tokens a block works on at once
    uint32_t side;              // of those, tokens side by side
    uint32_t units, span;       // units of a token, and how many of them a block has (blockIdx.y: which)
    uint32_t turned, passed;    // units of a head that turn and that pass through
    Divisor span_by, turned_by, passed_by, value_by, pairs;
};

// BYTES (16, or 8 where 16 do not fit the pairs) at a time.  A unit is what a thread reads and writes of a token: two chunks whose values form pairs, one chunk
// of neighbouring pairs (interleaved), one that passes through, or one of the values (cache_append).  A thread keeps its
// unit and walks over tokens, so what it addresses is found once.  The bound is memory; the angles would not be free if
// every head computed them (a sine and a cosine are some fifty instructions), so a block computes those of a batch of
// tokens once, into shared memory, one batch ahead.  The chunks of the next batches are on their way meanwhile: each
// thread copies its own ahead and reads them back, as in lt_norm_rows.  Rotary 8192 x 32 x 128 bf16: 24.3 us, 5.5 TB/s;
// append 8192 x 8 x 128 bf16: 14.5 us, 4.6 TB/s.
// With 8 bytes, rotary 8192 x 32 x 80 bf16, 40 turned in halves of 20: 19.5 us, against 43 with lt_turn_any.
template <class T, bool APPEND, bool INTER, int BYTES>
__global__ void __launch_bounds__(TURN_THREADS, 4) lt_turn_chunks(const TurnArgs a, const TurnShape sh) {
    constexpr int N = BYTES / (int)sizeof(T);
    using V = typename std::conditional<BYTES == 16, uint4, uint2>::type;
    extern __shared__ uint4 turn_room[];
    V *const turn_mem = reinterpret_cast<V *>(turn_room);  // the ring [STAGES][FLIGHT][2][threads], then twice cosines and sines [batch][pairs]
    __shared__ uint64_t sm_at[2][TURN_THREADS];  // where a token goes (all ones: nowhere)
    float *const angles = reinterpret_cast<float *>(turn_room + turn_ring(BYTES) / 16);
    const uint32_t half = sh.batch * a.pairs;
    // the block's tokens
    const uint64_t t0 = a.tokens * blockIdx.x / gridDim.x, t1 = a.tokens * (blockIdx.x + 1) / gridDim.x;
    const uint32_t tokens = (uint32_t)(t1 - t0);
    // the thread's unit: first those that turn, head by head, then those that pass, then the values
    const uint32_t beside = sh.span_by.quotient(threadIdx.x), unit = blockIdx.y * sh.span + threadIdx.x - beside * sh.span;
    const bool busy = beside < sh.side && unit < sh.units;
    uint32_t r = unit, head, chunk, from;
    bool turns = false, value = false;
    if (r < a.heads * sh.turned) {
        turns = true;
        head = sh.turned_by.quotient(r);
        chunk = r - head * sh.turned;
        from = chunk * N;
    } else if ((r -= a.heads * sh.turned) < a.heads * sh.passed) {
        head = sh.passed_by.quotient(r);
        chunk = r - head * sh.passed;
        from = 2 * a.pairs + chunk * N;
    } else {
        value = APPEND;
        r -= a.heads * sh.passed;
        head = sh.value_by.quotient(r);
        chunk = r - head * (a.dim / N);
        from = chunk * N;
    }
    const bool two = !INTER && turns;
    const uint64_t pitch = value ? a.v_pitch : a.x_pitch;
    const T *src = (const T *)(value ? a.v : a.x) + (t0 + beside) * pitch + (uint64_t)head * a.dim + from;
    T *const dst = (T *)a.out + (uint64_t)head * (APPEND ? a.head_stride : (uint64_t)a.dim) + (value ? a.value_offset : 0) + from;
    const uint64_t step = sh.side * pitch;
    const uint32_t mine = shared_address(turn_mem + threadIdx.x);
    uint32_t fetched = beside;  // next token to fetch
    // (where there is much to do the next kernel begins when the blocks end: rotary 8192 x 32 x 128 bf16 24.4 us against 25.8)
    if (tokens <= sh.batch) pdl_release();
    pdl_wait();
    auto issue = [&](uint32_t stage) {
#pragma unroll
        for (int k = 0; k < TURN_FLIGHT; ++k) {
            if (busy && fetched < tokens) {
                copy_piece<BYTES>(mine + ((stage * TURN_FLIGHT + k) * 2) * TURN_THREADS * BYTES, src);
                if (two) copy_piece<BYTES>(mine + ((stage * TURN_FLIGHT + k) * 2 + 1) * TURN_THREADS * BYTES, src + a.pairs);
            }
            fetched += sh.side;
            src += step;
        }
        copy_commit();
    };
    auto prepare = [&](uint32_t first, uint32_t which) {  // angles and destinations of the tokens from `first` on
        const uint32_t n = min(sh.batch, tokens - first);
        float *cosines = angles + which * 2 * half, *sines = cosines + half;
        for (uint32_t i = threadIdx.x; i < n * a.pairs; i += TURN_THREADS) {
            const uint32_t t = sh.pairs.quotient(i);
            const float2 cs = turn(a.positions[t0 + first + t], a.frequencies[i - t * a.pairs], a.scale, a.inverse != 0);
            cosines[i] = cs.x;
            sines[i] = cs.y;
        }
        if (threadIdx.x < n) {
            uint64_t at;
            sm_at[which][threadIdx.x] = destination<APPEND>(a, t0 + first + threadIdx.x, &at) ? at : ~0ull;
        }
    };
#pragma unroll
    for (int s = 0; s < TURN_STAGES; ++s) issue(s);
    if (tokens) prepare(0, 0);
    uint32_t stage = 0, which = 0;
    for (uint32_t first = 0; first < tokens; first += sh.batch, which ^= 1, stage = stage + 1 >= TURN_STAGES ? 0 : stage + 1) {
        __syncthreads();  // this batch's angles are there, and nobody reads the ones before it any more
        copy_wait<TURN_STAGES - 1>();
        const float *cosines = angles + which * 2 * half, *sines = cosines + half;
#pragma unroll
        for (int k = 0; k < TURN_FLIGHT; ++k) {
            const uint32_t token = beside + k * sh.side;
            if (!busy || first + token >= tokens) break;
            const uint64_t at = sm_at[which][token];
            if (APPEND && at == ~0ull) continue;
            const V lo = turn_mem[((stage * TURN_FLIGHT + k) * 2) * TURN_THREADS + threadIdx.x];
            if (!turns) {
                *reinterpret_cast<V *>(dst + at) = lo;
                continue;
            }
            float p[N], q[N];
            unpack(lo, p);
            if constexpr (INTER) {
                const float *c = cosines + token * a.pairs + chunk * (N / 2), *s = sines + token * a.pairs + chunk * (N / 2);
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    q[2 * i] = p[2 * i] * c[i] - p[2 * i + 1] * s[i];
                    q[2 * i + 1] = p[2 * i] * s[i] + p[2 * i + 1] * c[i];
                }
                *reinterpret_cast<V *>(dst + at) = packed<V>(q);
            } else {
                const float4 *c = reinterpret_cast<const float4 *>(cosines + token * a.pairs + chunk * N), *s = reinterpret_cast<const float4 *>(sines + token * a.pairs + chunk * N);
                unpack(turn_mem[((stage * TURN_FLIGHT + k) * 2 + 1) * TURN_THREADS + threadIdx.x], q);
#pragma unroll
                for (int i = 0; i < N / 4; ++i) {
                    const float4 cc = c[i], ss = s[i];
                    const float co[4] = {cc.x, cc.y, cc.z, cc.w}, si[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float fp = p[4 * i + j], fq = q[4 * i + j];
                        p[4 * i + j] = fp * co[j] - fq * si[j];
                        q[4 * i + j] = fp * si[j] + fq * co[j];
                    }
                }
                *reinterpret_cast<V *>(dst + at) = packed<V>(p);
                *reinterpret_cast<V *>(dst + at + a.pairs) = packed<V>(q);
            }
        }
        issue(stage);
        if (first + sh.batch < tokens) prepare(first + sh.batch, which ^ 1);
    }
}

template <class T, bool APPEND, bool INTER, int BYTES>
cudaError_t launch_turn_chunks(const TurnArgs &a, const TurnShape &sh, uint32_t across, int sm_count, cudaStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    constexpr size_t most = turn_ring(BYTES) + 2 * TURN_ANGLES * 8;
    const cudaError_t e = allow_shared(lt_turn_chunks<T, APPEND, INTER, BYTES>, most, ready);
    if (e != cudaSuccess) return e;
    // as many blocks as the SMs hold (by threads, by shared memory), each going on to further tokens
    const size_t mem = turn_ring(BYTES) + (size_t)2 * sh.batch * a.pairs * 8;
    const uint64_t per_sm = std::min<uint64_t>(4, 220 * 1024 / (mem + 5 * 1024)), wave = std::max<uint64_t>(1, (uint64_t)sm_count * per_sm / across);
    const uint64_t batches = (a.tokens + sh.batch - 1) / sh.batch;
    const dim3 grid((unsigned)std::min(batches, wave), across);
    return launch_pdl_shared(lt_turn_chunks<T, APPEND, INTER, BYTES>, grid, TURN_THREADS, mem, stream, a, sh);
}

// lt_turn_chunks, if pieces of BYTES fit the shape and the addresses.
template <class T, bool APPEND, int BYTES>
bool launch_turn_pieces(const TurnArgs &a, int sm_count, cudaStream_t stream, cudaError_t *e) {
    constexpr uint32_t N = BYTES / sizeof(T);
    const bool fits = a.dim % N == 0 && (a.interleaved ? 2 * a.pairs : a.pairs) % N == 0 && a.x_pitch % N == 0 && is_aligned(a.x, BYTES) && is_aligned(a.out, BYTES) &&
                      (!APPEND || (a.v_pitch % N == 0 && is_aligned(a.v, BYTES)));
    const uint64_t units = (uint64_t)(a.dim / N - (a.interleaved ? 0 : a.pairs / N) + (APPEND ? a.dim / N : 0)) * a.heads;
    if (!fits || TURN_FLIGHT * a.pairs > TURN_ANGLES || units >= (1u << 20) || a.tokens >= (1ull << 31)) return false;
    TurnShape sh;
    sh.turned = (a.interleaved ? 2 * a.pairs : a.pairs) / N;
    sh.passed = (a.dim - 2 * a.pairs) / N;
    sh.units = (uint32_t)units;
    // a token's units over as few blocks as hold them, evenly; several tokens side by side where they leave room
    const uint32_t across = (sh.units + TURN_THREADS - 1) / TURN_THREADS;
    sh.span = (sh.units + across - 1) / across;
    sh.side = TURN_THREADS / sh.span;
    if (a.pairs) sh.side = std::min(sh.side, TURN_ANGLES / (TURN_FLIGHT * a.pairs));
    sh.side = std::min<uint32_t>(sh.side, TURN_THREADS / TURN_FLIGHT);
    sh.batch = sh.side * TURN_FLIGHT;
    sh.span_by = Divisor::make(sh.span);
    sh.turned_by = Divisor::make(sh.turned ? sh.turned : 1);
    sh.passed_by = Divisor::make(sh.passed ? sh.passed : 1);
    sh.value_by = Divisor::make(a.dim / N);
    sh.pairs = Divisor::make(a.pairs ? a.pairs : 1);
    *e = a.interleaved ? launch_turn_chunks<T, APPEND, true, BYTES>(a, sh, across, sm_count, stream) : launch_turn_chunks<T, APPEND, false, BYTES>(a, sh, across, sm_count, stream);
    return true;
}

template <class T, bool APPEND>
cudaError_t launch_turn(const TurnArgs &a, int sm_count, cudaStream_t stream) {
    cudaError_t e = cudaSuccess;
    if (launch_turn_pieces<T, APPEND, 16>(a, sm_count, stream, &e)) return e;
    if constexpr (sizeof(T) == 2)
        if (launch_turn_pieces<T, APPEND, 8>(a, sm_count, stream, &e)) return e;
    const uint64_t total = a.tokens * (a.dim - a.pairs);
    const uint64_t blocks = (total + 255) / 256, most = (uint64_t)sm_count * 32;
    return launch_pdl(lt_turn_any<T, APPEND>, (unsigned)(blocks < most ? blocks : most), 256, (size_t)0, stream, a);
}

// ------------------------------------------------------------------------------------------- norms

struct NormArgs {
    const void *x, *r, *gamma;  // r: residual, or null
    void *y, *sum;
    uint8_t *codes;
    float *scales;
    uint64_t rows, cols, x_pitch, r_pitch;
    uint32_t group, groups;     // columns of a group (0: the row)
    uint32_t group_shift;       // lt_norm_rows: log2 of the chunks of a group
    float eps;
    float down, up;             // 2^-k <= 1 / cols and 2^k / cols: a mean of squares is summed as h (h 2^-k), which fits where the mean does
    int gamma_f32;
};

template <class T>
__device__ __forceinline__ float gamma_at(const void *gamma, int f32, uint64_t c) {
    return f32 ? ((const float *)gamma)[c] : to_float(((const T *)gamma)[c]);
}

// 448 / top, the factor from values to e4m3 codes, by the reciprocal unit (1 ulp: far below half a step of a code; 0 for a
// group of zeros).  A NaN stays.  So small a group that the quotient might overflow is raised by a power of two first, the
// values and their maximum alike.
constexpr float SMALL = 0x1p-100f, RAISE = 0x1p100f;
__device__ __forceinline__ float raise_of(float top) { return top < SMALL ? RAISE : 1.f; }
__device__ __forceinline__ float code_factor(float top) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(top));
    return top == 0.f ? 0.f : r * 448.f;
}
__device__ __forceinline__ float scale_of(float top) { return top * (1.f / 448.f); }

// Any shape and alignment: a block per row, which is read once for its mean square, once more for each output.  Taken by rows
// of more than 1024 values that cannot be read in pieces of 16 bytes, of more than 16384 f32 or 32768 bf16 values, and, beyond
// 1024 values, by groups of 256 in f32 (which 32 lanes of four values do not hold).  1000 x 20480 f32 with a residual: 165 us,
// where 1000 x 16384 takes 47; 4096 x 4096 f32 to eight bits in groups of 256: 94 us, where groups of 128 take 39.
template <class T>
__global__ void __launch_bounds__(256) lt_norm_any(const NormArgs a) {
    __shared__ float part[32];
    pdl_release();
    pdl_wait();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.x_pitch;
        const T *r = a.r ? (const T *)a.r + row * a.r_pitch : nullptr;
        auto h_at = [&](uint64_t c) { return to_float(x[c]) + (r ? to_float(r[c]) : 0.f); };
        float ss = 0.f;
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float h = h_at(c);
            ss += h * (h * a.down);
        }
        const float inv = rsqrtf(block_reduce<false>(ss, part) * a.up + a.eps);
        if (a.codes || a.scales) {
            if (!a.group) {
                float top = 0.f;
                for (uint64_t c = threadIdx.x; c < a.cols; c += 256) top = max_nan(top, fabsf(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c)));
                top = block_reduce<true>(top, part);
                if (a.scales && threadIdx.x == 0) a.scales[row] = scale_of(top);
                const float up = raise_of(top), f = code_factor(top * up);
                if (a.codes)
                    for (uint64_t c = threadIdx.x; c < a.cols; c += 256)
                        a.codes[row * a.cols + c] = __nv_cvt_float_to_fp8(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c) * up * f, __NV_SATFINITE, __NV_E4M3);
            } else {
                for (uint32_t g = threadIdx.x >> 5; g < a.groups; g += 8) {  // a warp per group
                    const uint64_t c0 = (uint64_t)g * a.group, c1 = min(c0 + a.group, a.cols);
                    float top = 0.f;
                    for (uint64_t c = c0 + (threadIdx.x & 31); c < c1; c += 32) top = max_nan(top, fabsf(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c)));
                    top = warp_max_nan(top);
                    if (a.scales && (threadIdx.x & 31) == 0) a.scales[row * a.groups + g] = scale_of(top);
                    const float up = raise_of(top), f = code_factor(top * up);
                    if (a.codes)
                        for (uint64_t c = c0 + (threadIdx.x & 31); c < c1; c += 32)
                            a.codes[row * a.cols + c] = __nv_cvt_float_to_fp8(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c) * up * f, __NV_SATFINITE, __NV_E4M3);
                }
                __syncthreads();  // (y or the sum may overwrite x or the residual)
            }
        }
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float h = h_at(c);
            if (a.y) ((T *)a.y)[row * a.cols + c] = from_float<T>(h * inv * gamma_at<T>(a.gamma, a.gamma_f32, c));
            if (a.sum) ((T *)a.sum)[row * a.cols + c] = from_float<T>(h);
        }
    }
}

// Rows of up to NARROW_COLS values at any alignment, where 16 bytes at a time are not to be had: RT threads per row (32, 64
// or 128, the fewest that hold the row with eight values of each in registers -- values t, t + RT, ..), so that every value
// is still read once.  The largest values of 32 columns each go through shared memory to whoever needs them.  Bound by its
// instructions, one or two dozen per value; against lt_norm_any and lt_norm_grad_any, which read a row up to three times:
// 8000 x 999 bf16 to eight bits 50 us against 55, the gradient of 8000 x 999 bf16 42 against 118, of 30000 x 131 f32 23
// against 48.  (Groups of 256 in f32 come here too: 8192 x 1024 to eight bits 40 us, where groups of 128 take 22.)
constexpr int NARROW_COLS = 1024, NARROW_VALUES = 8, NARROW_BLOCKS = 4;  // blocks that share an SM
constexpr int narrow_threads(uint64_t cols) { return cols <= 32 * NARROW_VALUES ? 32 : cols <= 64 * NARROW_VALUES ? 64 : 128; }

unsigned narrow_blocks(uint64_t rows, uint64_t cols, int sm_count) {
    const uint64_t at_once = 256 / narrow_threads(cols);
    return (unsigned)std::min<uint64_t>((rows + at_once - 1) / at_once, (uint64_t)sm_count * NARROW_BLOCKS);
}

// Both sums over the RT threads of a row group inside a block (`group`: which).  `part`: room for 2 x 32 values, used in
// turn, as in row_reduce below.
template <int RT>
__device__ __forceinline__ float2 group_sum(float x, float y, float2 *part, int group, int &turn) {
    x = warp_sum(x);
    y = warp_sum(y);
    if constexpr (RT == 32) return make_float2(x, y);
    constexpr int W = RT / 32;
    float2 *mine = part + (turn & 1) * 32 + group * W;
    ++turn;
    if ((threadIdx.x & 31) == 0) mine[(threadIdx.x % RT) >> 5] = make_float2(x, y);
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(RT) : "memory");
    float2 s = mine[threadIdx.x & (W - 1)];
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, d);
        s.y += __shfl_xor_sync(0xffffffffu, s.y, d);
    }
    return s;
}

// `n` values of a row from `row` on, RT apart; zeros after them.  All are read before the first is used.
template <class T, int RT>
__device__ __forceinline__ void load_narrow(float *v, const T *row, int n) {
    T raw[NARROW_VALUES];
#pragma unroll
    for (int k = 0; k < NARROW_VALUES; ++k) {
        raw[k] = from_float<T>(0.f);
        if (k < n) raw[k] = row[RT * k];
    }
#pragma unroll
    for (int k = 0; k < NARROW_VALUES; ++k) v[k] = to_float(raw[k]);
}

template <class T, int RT>
__global__ void __launch_bounds__(256, NARROW_BLOCKS) lt_norm_narrow(const NormArgs a) {
    constexpr int E = NARROW_VALUES, GROUPS = 256 / RT, W = RT / 32;
    __shared__ float2 part[64];
    __shared__ float tops[GROUPS][E * W];  // of 32 columns each
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x % RT, group = threadIdx.x / RT, cols = (uint32_t)a.cols;
    const uint32_t steps = a.group ? a.group / 32 : E * W;  // of 32 columns, in a group of the output
    const int n = lane < cols ? (int)((cols - lane + RT - 1) / RT) : 0;  // values of a row that are this thread's
    int turn = 0;
    float g[E];
#pragma unroll
    for (int k = 0; k < E; ++k) g[k] = k < n ? gamma_at<T>(a.gamma, a.gamma_f32, lane + RT * k) : 0.f;
    for (uint64_t row = (uint64_t)blockIdx.x * GROUPS + group; row < a.rows; row += (uint64_t)gridDim.x * GROUPS) {
        float h[E], ss = 0.f;
        load_narrow<T, RT>(h, (const T *)a.x + row * a.x_pitch + lane, n);
        if (a.r) {
            float r[E];
            load_narrow<T, RT>(r, (const T *)a.r + row * a.r_pitch + lane, n);
#pragma unroll
            for (int k = 0; k < E; ++k) h[k] += r[k];
        }
#pragma unroll
        for (int k = 0; k < E; ++k) ss += h[k] * (h[k] * a.down);
        const float inv = rsqrtf(group_sum<RT>(ss, 0.f, part, (int)group, turn).x * a.up + a.eps);
        const uint64_t at = row * cols + lane;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (a.sum && k < n) ((T *)a.sum)[at + RT * k] = from_float<T>(h[k]);
            h[k] = h[k] * inv * g[k];
            if (k >= n) h[k] = 0.f;  // (not infinity times nothing)
            if (a.y && k < n) ((T *)a.y)[at + RT * k] = from_float<T>(h[k]);
        }
        if (!a.codes && !a.scales) continue;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float t = 0.f;
            if (RT * k + (lane & ~31u) < cols) t = warp_max_nan(fabsf(h[k]));  // (the same in all lanes)
            if ((lane & 31) == 0) tops[group][k * W + (lane >> 5)] = t;
        }
        if constexpr (RT == 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(RT) : "memory");
        float t = 0.f;
        uint32_t known = 0;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (RT * k + (lane & ~31u) >= cols) break;
            const uint32_t mine = k * W + (lane >> 5), first = mine & ~(steps - 1);
            if (k == 0 || first != known) {  // (the same in all lanes)
                t = 0.f;
                for (uint32_t i = 0; i < steps; ++i) t = max_nan(t, tops[group][first + i]);
                known = first;
            }
            if (a.scales && (lane & 31) == 0 && mine == first) a.scales[row * a.groups + (a.group ? mine * 32 / a.group : 0)] = scale_of(t);
            if (a.codes && k < n) a.codes[at + RT * k] = __nv_cvt_float_to_fp8(h[k] * raise_of(t) * code_factor(t * raise_of(t)), __NV_SATFINITE, __NV_E4M3);
        }
        if constexpr (RT == 32) __syncwarp();  // (128 threads: the next row's sums have a barrier before `tops` is written again)
    }
}

// N values of gamma from column c on, which is a multiple of N
template <class T>
__device__ __forceinline__ void gamma_chunk(const void *gamma, int f32, uint32_t c, float (&g)[Chunk<T>::N]) {
    constexpr int N = Chunk<T>::N;
    if (f32 || sizeof(T) == 4) {
        const float4 *p = reinterpret_cast<const float4 *>((const float *)gamma + c);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 v = p[i];
            g[4 * i] = v.x;
            g[4 * i + 1] = v.y;
            g[4 * i + 2] = v.z;
            g[4 * i + 3] = v.w;
        }
    } else {
        unpack(*reinterpret_cast<const uint4 *>((const T *)gamma + c), g);
    }
}

// Sum or maximum over the RT threads of a row: a warp, or a block of its own.  `part`: room for 2 x 32 values, used in turn
// (`turn` counts the reductions), so that one barrier per reduction is enough: whoever writes a half for the second time
// has passed the barrier behind everybody's reading of it.
template <int RT, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *part, int &turn) {
    v = MAX ? warp_max_nan(v) : warp_sum(v);
    if constexpr (RT == 32) return v;
    constexpr int W = RT / 32;
    float *mine = part + (turn & 1) * 32;
    ++turn;
    if ((threadIdx.x & 31) == 0) mine[threadIdx.x >> 5] = v;
    __syncthreads();
    v = mine[threadIdx.x & (W - 1)];
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, v, d);
        v = MAX ? max_nan(v, o) : v + o;
    }
    return v;
}

__host__ __device__ constexpr int norm_block(int rt) { return rt == 32 ? 128 : rt; }
// Rows on their way while one is worked on: some 130 to 190 KB per SM at the occupancy the registers allow.
__host__ __device__ constexpr int norm_stages(int rt, int ch) { return ch == 1 ? 3 : norm_block(rt) * ch <= 2048 ? 3 : 1; }
__host__ __device__ constexpr size_t norm_bytes(int rt, int ch) { return (size_t)norm_stages(rt, ch) * 2 * ch * norm_block(rt) * 16; }

// 16 bytes at a time, a row in the registers of its RT threads (CH chunks each): every value is read once and every
// result written once, so the bound is memory.  Threads keep their columns of gamma from row to row.  The rows to come
// travel through shared memory ahead of their turn: a thread copies and reads back only its own chunks, so the ring
// needs no barrier; registers alone kept too little on its way (8192 x 4096 bf16: 88 us with four chunks per thread and
// the next row in registers, 52 us with one chunk per thread).  The same size with a residual, to eight bits: 42.5 us, 5.5
// TB/s.
template <class T, int RT, int CH, bool EIGHT>
__global__ void __launch_bounds__(norm_block(RT), norm_block(RT) == 1024 ? 1 : (CH == 1 ? 1536 : CH == 2 ? 1024 : 512) / norm_block(RT)) lt_norm_rows(const NormArgs a) {
    constexpr int N = Chunk<T>::N, BLOCK = norm_block(RT), STAGES = norm_stages(RT, CH);
    extern __shared__ uint4 ring[];  // [STAGES][x, residual][CH][BLOCK]
    __shared__ float part[64];
    int turn = 0;
    const uint32_t lane = RT == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const uint32_t chunks = (uint32_t)a.cols / N;
    const uint64_t step = RT == 32 ? (uint64_t)gridDim.x * 4 : gridDim.x;
    uint64_t row = RT == 32 ? (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    pdl_release();
    pdl_wait();
    // where the thread's first chunk of the next row to fetch lies, and in the ring
    const T *next_x = (const T *)a.x + row * a.x_pitch + lane * N, *next_r = (const T *)a.r + (a.r ? row * a.r_pitch + lane * N : 0);
    const uint64_t x_step = step * a.x_pitch, r_step = step * a.r_pitch;
    const uint32_t mine = shared_address(ring + threadIdx.x);
    constexpr uint32_t STAGE_BYTES = 2 * CH * BLOCK * 16;
    uint64_t fetched = row;
    auto issue = [&](uint32_t stage) {
        if (fetched < a.rows) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (lane + k * RT >= chunks) continue;
                copy16(mine + stage + k * BLOCK * 16, next_x + k * RT * N, true);
                if (a.r) copy16(mine + stage + (CH + k) * BLOCK * 16, next_r + k * RT * N, true);
            }
        }
        copy_commit();
        fetched += step;
        next_x += x_step;
        next_r += r_step;
    };
#pragma unroll
    for (int s = 0; s < STAGES; ++s) issue(s * STAGE_BYTES);
    float g[CH][N];
#pragma unroll
    for (int k = 0; k < CH; ++k)
        if (lane + k * RT < chunks) gamma_chunk<T>(a.gamma, a.gamma_f32, (lane + k * RT) * N, g[k]);
    for (uint32_t stage = 0; row < a.rows; row += step, stage = stage + STAGE_BYTES == STAGES * STAGE_BYTES ? 0 : stage + STAGE_BYTES) {
        copy_wait<STAGES - 1>();
        const uint4 *slot = ring + threadIdx.x + stage / 16;
        float h[CH][N], ss = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (lane + k * RT >= chunks) continue;
            unpack(slot[k * BLOCK], h[k]);
            if (a.r) add_chunk(slot[(CH + k) * BLOCK], h[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) ss += h[k][i] * h[k][i];
        }
        issue(stage);  // (results go over the operands of their own row only)
        float mean = row_reduce<RT, false>(ss, part, turn) * a.down;
        if (mean > 3.402823466e38f) {  // the sum of the squares does not fit, their mean may
            ss = 0.f;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (lane + k * RT < chunks) {
#pragma unroll
                    for (int i = 0; i < N; ++i) ss += h[k][i] * (h[k][i] * a.down);
                }
            mean = row_reduce<RT, false>(ss, part, turn);
        }
        const float inv = rsqrtf(mean * a.up + a.eps);
        const uint64_t at = row * a.cols;
        if (a.sum) {
            T *to = (T *)a.sum + at;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (lane + k * RT < chunks) *reinterpret_cast<uint4 *>(to + (lane + k * RT) * N) = pack(h[k]);
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (lane + k * RT >= chunks) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) h[k][i] = h[k][i] * inv * g[k][i];
        }
        if (!EIGHT || a.y) {
            T *to = (T *)a.y + at;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (a.y && lane + k * RT < chunks) *reinterpret_cast<uint4 *>(to + (lane + k * RT) * N) = pack(h[k]);
        }
        if constexpr (EIGHT) {
            float top[CH], row_top = 0.f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                top[k] = 0.f;
                if (lane + k * RT >= chunks) continue;
#pragma unroll
                for (int i = 0; i < N; i += 2) top[k] = max_abs(top[k], h[k][i], h[k][i + 1]);
                row_top = max_nan(row_top, top[k]);
            }
            if (!a.group) {
                row_top = row_reduce<RT, true>(row_top, part, turn);
                if (a.scales && lane == 0) a.scales[row] = scale_of(row_top);
            }
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const uint32_t c = lane + k * RT;
                float t = row_top;
                if (a.group) {  // a power of two of lanes share a scale
                    t = top[k];
#pragma unroll
                    for (int d = 0; d < 5; ++d)
                        if (d < (int)a.group_shift) t = max_nan(t, __shfl_xor_sync(0xffffffffu, t, 1 << d));
                    if (a.scales && c < chunks && (c & ((1u << a.group_shift) - 1)) == 0) a.scales[row * a.groups + (c >> a.group_shift)] = scale_of(t);
                }
                if (!a.codes || c >= chunks) continue;
                if (t < SMALL) {
                    t *= RAISE;
#pragma unroll
                    for (int i = 0; i < N; ++i) h[k][i] *= RAISE;
                }
                const float f = code_factor(t);
                uint32_t w[N / 4];
#pragma unroll
                for (int i = 0; i < N / 4; ++i) {
                    const uint32_t p0 = __nv_cvt_float2_to_fp8x2(make_float2(h[k][4 * i] * f, h[k][4 * i + 1] * f), __NV_SATFINITE, __NV_E4M3);
                    const uint32_t p1 = __nv_cvt_float2_to_fp8x2(make_float2(h[k][4 * i + 2] * f, h[k][4 * i + 3] * f), __NV_SATFINITE, __NV_E4M3);
                    w[i] = p0 | (p1 << 16);
                }
                uint8_t *to = a.codes + at + c * N;
                if constexpr (N == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t *>(to) = w[0];
            }
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *gamma, *dh;
    void *dx;
    float *partial;             // [blocks, cols], or null
    uint64_t rows, cols, dy_pitch, h_pitch, dh_pitch;
    float eps, down, up;
    int gamma_f32;
};

// The gradient's kernels sum gamma dy h first and scale it afterwards, as the norm is not known before.  Where that sum does not
// fit (or is no number), they sum gamma dy u over the row a second time.
__device__ __forceinline__ bool finite_sum(float v) { return fabsf(v) <= 3.402823466e38f; }

// (not inlined: the loops of lt_norm_grad_any take 4 to 20 % longer beside it)
template <class T>
__device__ __noinline__ float dot_again(const NormGradArgs &a, const T *dy, const T *h, float inv) {
    float dot = 0.f;
    for (uint64_t c = threadIdx.x; c < a.cols; c += 256) dot += to_float(dy[c]) * gamma_at<T>(a.gamma, a.gamma_f32, c) * (to_float(h[c]) * inv * a.down);
    return dot;
}

// u = h / rms.  dx = dh + (gamma dy - u mean(gamma dy u)) / rms; a block adds up dy u over its rows in its own row of
// `partial`.  Taken by rows of more than 1024 values that cannot be read in pieces of 16 bytes, and of more than 8192 f32 or
// 16384 bf16 values: 1000 x 12288 f32 190 us, where 1000 x 8192 takes 28; 3000 x 4095 bf16 175 us, where 4096 takes 24.
template <class T>
__global__ void __launch_bounds__(256) lt_norm_grad_any(const NormGradArgs a) {
    __shared__ float part[32];
    pdl_release();
    pdl_wait();
    float *mine = a.partial ? a.partial + (uint64_t)blockIdx.x * a.cols : nullptr;
    if (mine)
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) mine[c] = 0.f;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = (const T *)a.dy + row * a.dy_pitch, *h = (const T *)a.h + row * a.h_pitch;
        const T *dh = a.dh ? (const T *)a.dh + row * a.dh_pitch : nullptr;
        float ss = 0.f, dot = 0.f;
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float hv = to_float(h[c]);
            ss += hv * (hv * a.down);
            dot += to_float(dy[c]) * gamma_at<T>(a.gamma, a.gamma_f32, c) * (hv * a.down);
        }
        ss = block_reduce<false>(ss, part);
        dot = block_reduce<false>(dot, part);
        const float inv = rsqrtf(ss * a.up + a.eps);
        float m = dot * inv * a.up;
        if (!finite_sum(dot)) m = block_reduce<false>(dot_again<T>(a, dy, h, inv), part) * a.up;
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float d = to_float(dy[c]), u = to_float(h[c]) * inv;
            const float g = (d * gamma_at<T>(a.gamma, a.gamma_f32, c) - u * m) * inv + (dh ? to_float(dh[c]) : 0.f);
            if (a.dx) ((T *)a.dx)[row * a.cols + c] = from_float<T>(g);
            if (mine) mine[c] += d * u;
        }
    }
}

// The gradient for rows as in lt_norm_narrow; a thread keeps its columns' sums for gamma.
template <class T, int RT>
__global__ void __launch_bounds__(256, NARROW_BLOCKS) lt_norm_grad_narrow(const NormGradArgs a) {
    constexpr int E = NARROW_VALUES, GROUPS = 256 / RT;
    __shared__ float2 part[64];
    __shared__ float sums[GROUPS][RT * E];
    pdl_release();
    pdl_wait();
    const uint32_t lane = threadIdx.x % RT, group = threadIdx.x / RT, cols = (uint32_t)a.cols;
    const int n = lane < cols ? (int)((cols - lane + RT - 1) / RT) : 0;  // values of a row that are this thread's
    int turn = 0;
    float g[E], sum[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
        g[k] = k < n ? gamma_at<T>(a.gamma, a.gamma_f32, lane + RT * k) : 0.f;
        sum[k] = 0.f;
    }
    for (uint64_t row = (uint64_t)blockIdx.x * GROUPS + group; row < a.rows; row += (uint64_t)gridDim.x * GROUPS) {
        float d[E], u[E], e[E] = {}, ss = 0.f, dot = 0.f;
        if (a.dh) load_narrow<T, RT>(e, (const T *)a.dh + row * a.dh_pitch + lane, n);
        load_narrow<T, RT>(d, (const T *)a.dy + row * a.dy_pitch + lane, n);
        load_narrow<T, RT>(u, (const T *)a.h + row * a.h_pitch + lane, n);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            ss += u[k] * (u[k] * a.down);
            dot += d[k] * g[k] * (u[k] * a.down);
        }
        const float2 s = group_sum<RT>(ss, dot, part, (int)group, turn);
        const uint64_t at = row * cols + lane;
        const float inv = rsqrtf(s.x * a.up + a.eps);
        float m = s.y * inv * a.up;
        if (!finite_sum(s.y)) {
            dot = 0.f;
#pragma unroll
            for (int k = 0; k < E; ++k) dot += d[k] * g[k] * (u[k] * inv * a.down);
            m = group_sum<RT>(dot, 0.f, part, (int)group, turn).x * a.up;
        }
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float v = u[k] * inv;
            sum[k] += d[k] * v;
            if (a.dx && k < n) ((T *)a.dx)[at + RT * k] = from_float<T>((d[k] * g[k] - v * m) * inv + e[k]);
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int k = 0; k < E; ++k) sums[group][lane + RT * k] = sum[k];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < cols; c += 256) {
        float t = sums[0][c];
#pragma unroll
        for (int w = 1; w < GROUPS; ++w) t += sums[w][c];
        a.partial[(uint64_t)blockIdx.x * cols + c] = t;
    }
}

__host__ __device__ constexpr int grad_block(int rt) { return rt > 256 ? rt : 256; }
// Rows on their way: as many as fit (at most 2048 chunks a row: 825 x 8192 f32 19.4 us with two of them, 23.9 with one).
__host__ __device__ constexpr int grad_stages(int rt, int ch) { return grad_block(rt) * ch <= 512 ? 4 : 2; }
__host__ __device__ constexpr size_t grad_bytes(int rt, int ch) { return (size_t)grad_stages(rt, ch) * 3 * ch * grad_block(rt) * 16; }
constexpr int GRAD_CHUNKS = 4;  // of a thread, at most

// 16 bytes at a time, RT threads per row; a block has several rows at once and goes on to others, the sums for gamma
// staying in registers.  Bound by memory like lt_norm_rows, and like there the rows to come travel through shared
// memory, from which a row is read twice: for its sums, and for its results.  16384 x 1024 bf16 with the sum's own
// gradient: 24 us, 5.6 TB/s, and 5 more for lt_norm_grad_join.
template <class T, int RT, int CH>
__global__ void __launch_bounds__(grad_block(RT), RT > 256 ? 1 : 2) lt_norm_grad_rows(const NormGradArgs a) {
    constexpr int N = Chunk<T>::N, BLOCK = grad_block(RT), GROUPS = BLOCK / RT, STAGES = grad_stages(RT, CH);
    __shared__ float2 part[64];
    int turn = 0;
    extern __shared__ uint4 ring[];  // [STAGES][dy, h, dh][CH][BLOCK]; at the end [GROUPS - 1][cols]: the groups' sums for gamma
    float4 *grad_mem = reinterpret_cast<float4 *>(ring);
    const int group = threadIdx.x / RT;
    const uint32_t lane = threadIdx.x % RT, chunks = (uint32_t)a.cols / N;
    const uint64_t step = (uint64_t)gridDim.x * GROUPS;
    if (a.rows <= step) pdl_release();  // (otherwise the next kernel begins when the blocks end: 16384 x 1024 bf16 29.0 us against 29.8)
    pdl_wait();
    auto place = [&](int stage, int which, int k) { return ring + ((stage * 3 + which) * CH + k) * BLOCK + threadIdx.x; };
    auto issue = [&](uint64_t at, int stage) {
        if (at < a.rows) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const uint64_t c = (uint64_t)(lane + k * RT) * N;
                if (lane + k * RT >= chunks) continue;
                copy16(shared_address(place(stage, 0, k)), (const T *)a.dy + at * a.dy_pitch + c, true);
                copy16(shared_address(place(stage, 1, k)), (const T *)a.h + at * a.h_pitch + c, true);
                if (a.dh) copy16(shared_address(place(stage, 2, k)), (const T *)a.dh + at * a.dh_pitch + c, true);
            }
        }
        copy_commit();
    };
    uint64_t row = (uint64_t)blockIdx.x * GROUPS + group;
#pragma unroll
    for (int s = 0; s < STAGES; ++s) issue(row + s * step, s);
    float g[CH][N], sum[CH][N];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[k][i] = sum[k][i] = 0.f;
        if (lane + k * RT < chunks) gamma_chunk<T>(a.gamma, a.gamma_f32, (lane + k * RT) * N, g[k]);
    }
    for (int stage = 0; row < a.rows; row += step, stage = stage + 1 == STAGES ? 0 : stage + 1) {
        float ss = 0.f, dot = 0.f;
        copy_wait<STAGES - 1>();
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (lane + k * RT >= chunks) continue;
            float d[N], u[N];
            unpack(*place(stage, 0, k), d);
            unpack(*place(stage, 1, k), u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ss += u[i] * u[i];
                dot += d[i] * g[k][i] * u[i];
            }
        }
        float2 s = group_sum<RT>(ss, dot, part, group, turn);
        s.x *= a.down;
        if (s.x > 3.402823466e38f) {  // the sum of the squares does not fit, their mean may
            ss = 0.f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (lane + k * RT >= chunks) continue;
                float u[N];
                unpack(*place(stage, 1, k), u);
#pragma unroll
                for (int i = 0; i < N; ++i) ss += u[i] * (u[i] * a.down);
            }
            s.x = group_sum<RT>(ss, 0.f, part, group, turn).x;
        }
        const float inv = rsqrtf(s.x * a.up + a.eps);
        float m = s.y * a.down * inv * a.up;
        if (!finite_sum(s.y)) {
            dot = 0.f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (lane + k * RT >= chunks) continue;
                float d[N], u[N];
                unpack(*place(stage, 0, k), d);
                unpack(*place(stage, 1, k), u);
#pragma unroll
                for (int i = 0; i < N; ++i) dot += d[i] * g[k][i] * (u[i] * inv * a.down);
            }
            m = group_sum<RT>(dot, 0.f, part, group, turn).x * a.up;
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (lane + k * RT >= chunks) continue;
            float d[N], u[N], e[N];
            unpack(*place(stage, 0, k), d);
            unpack(*place(stage, 1, k), u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float n = u[i] * inv;
                sum[k][i] += d[i] * n;
                e[i] = (d[i] * g[k][i] - n * m) * inv;
            }
            if (a.dh) add_chunk(*place(stage, 2, k), e);
            if (a.dx) *reinterpret_cast<uint4 *>((T *)a.dx + row * a.cols + (uint64_t)(lane + k * RT) * N) = pack(e);
        }
        issue(row + STAGES * step, stage);
    }
    if (!a.partial) return;
    if (GROUPS > 1) {
        copy_wait<0>();
        __syncthreads();  // the other groups' rows are done
        if (group > 0) {
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (lane + k * RT < chunks) {
#pragma unroll
                    for (int i = 0; i < N / 4; ++i)
                        grad_mem[((uint64_t)(group - 1) * a.cols + (uint64_t)(lane + k * RT) * N) / 4 + i] = make_float4(sum[k][4 * i], sum[k][4 * i + 1], sum[k][4 * i + 2], sum[k][4 * i + 3]);
                }
        }
        __syncthreads();
        if (group > 0) return;
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const uint32_t c = lane + k * RT;
        if (c >= chunks) continue;
        for (int o = 1; o < GROUPS; ++o)
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float4 v = grad_mem[((uint64_t)(o - 1) * a.cols + (uint64_t)c * N) / 4 + i];
                sum[k][4 * i] += v.x;
                sum[k][4 * i + 1] += v.y;
                sum[k][4 * i + 2] += v.z;
                sum[k][4 * i + 3] += v.w;
            }
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            *reinterpret_cast<float4 *>(a.partial + (uint64_t)blockIdx.x * a.cols + (uint64_t)c * N + 4 * i) = make_float4(sum[k][4 * i], sum[k][4 * i + 1], sum[k][4 * i + 2], sum[k][4 * i + 3]);
    }
}

// The blocks' sums, in binary64, always in the same order: a warp's lanes have neighbouring columns, its 32 warps every
// 32nd block each.
template <class G>
__global__ void __launch_bounds__(1024) lt_norm_grad_join(const float *partial, G *out, uint64_t cols, unsigned blocks) {
    __shared__ double sums[32][33];
    pdl_release();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (uint64_t c0 = (uint64_t)blockIdx.x * 32; c0 < cols; c0 += (uint64_t)gridDim.x * 32) {
        double s = 0.0;
        if (c0 + lane < cols) {
#pragma unroll 10
            for (unsigned b = warp; b < blocks; b += 32) s += (double)partial[(uint64_t)b * cols + c0 + lane];
        }
        __syncthreads();
        sums[warp][lane] = s;
        __syncthreads();
        s = sums[lane][warp];  // (a warp per column from here on)
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        if (lane == 0 && c0 + warp < cols) out[c0 + warp] = from_float<G>((float)s);
    }
}

// 2^-k with 2^k >= cols, and 2^k / cols
void mean_factors(uint64_t cols, float *down, float *up) {
    int k = 0;
    while ((1ull << k) < cols) ++k;
    *down = (float)(1.0 / (double)(1ull << k));
    *up = (float)((double)(1ull << k) / (double)cols);
}

// Threads per row: enough that a thread has at most `most` chunks.  0: the row does not fit.
int row_threads(uint64_t chunks, int most) {
    for (int rt : {32, 128, 256, 512, 1024})
        if (chunks <= (uint64_t)rt * most) return rt;
    return 0;
}

template <class T, int RT, int CH, bool EIGHT>
cudaError_t launch_norm_rows(const NormArgs &a, int sm_count, cudaStream_t stream) {
    const uint64_t blocks = RT == 32 ? (a.rows + 3) / 4 : a.rows;
    // as many blocks as an SM holds, each going on to further rows
    static std::atomic<uint64_t> ready{0};
    static std::atomic<int> resident{0};
    cudaError_t e = allow_shared(lt_norm_rows<T, RT, CH, EIGHT>, norm_bytes(RT, CH), ready);
    if (e != cudaSuccess) return e;
    if (!resident.load(std::memory_order_relaxed)) {
        int n = 0;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, lt_norm_rows<T, RT, CH, EIGHT>, norm_block(RT), norm_bytes(RT, CH));
        if (e != cudaSuccess) return e;
        resident.store(n < 1 ? 1 : n, std::memory_order_relaxed);
    }
    const uint64_t most = (uint64_t)sm_count * resident.load(std::memory_order_relaxed);
    return launch_pdl(lt_norm_rows<T, RT, CH, EIGHT>, (unsigned)(blocks < most ? blocks : most), norm_block(RT), norm_bytes(RT, CH), stream, a);
}

template <class T, int CH, bool EIGHT>
cudaError_t launch_norm_threads(const NormArgs &a, int rt, int sm_count, cudaStream_t stream) {
    switch (rt) {
    case 32: return launch_norm_rows<T, 32, CH, EIGHT>(a, sm_count, stream);
    case 128: return launch_norm_rows<T, 128, CH, EIGHT>(a, sm_count, stream);
    case 256: return launch_norm_rows<T, 256, CH, EIGHT>(a, sm_count, stream);
    case 512: return launch_norm_rows<T, 512, CH, EIGHT>(a, sm_count, stream);
    default: return launch_norm_rows<T, 1024, CH, EIGHT>(a, sm_count, stream);
    }
}

template <class T, bool EIGHT>
cudaError_t launch_norm_chunks(const NormArgs &a, uint64_t chunks, int sm_count, cudaStream_t stream) {
    // few rows: one chunk per thread, the most threads a row can use; many: four, which halves what a row costs besides its
    // values (8192 x 4096 bf16 in 8 bits: 42 us against 45 with one chunk per thread and 49 with two)
    const int rt = row_threads(chunks, a.rows <= 2 * (uint64_t)sm_count && chunks <= 1024 ? 1 : 4);
    const int ch = chunks <= (uint64_t)rt ? 1 : chunks <= 2 * (uint64_t)rt ? 2 : 4;
    if (ch == 1) return launch_norm_threads<T, 1, EIGHT>(a, rt, sm_count, stream);
    if (ch == 2) return launch_norm_threads<T, 2, EIGHT>(a, rt, sm_count, stream);
    return launch_norm_threads<T, 4, EIGHT>(a, rt, sm_count, stream);
}

template <class T>
cudaError_t launch_norm(NormArgs a, int sm_count, cudaStream_t stream) {
    constexpr uint64_t N = Chunk<T>::N;
    while (a.group && (N << a.group_shift) < a.group) ++a.group_shift;
    const uint64_t chunks = a.cols / N;
    const bool fits = a.cols % N == 0 && a.x_pitch % N == 0 && (!a.r || (a.r_pitch % N == 0 && is_aligned(a.r, 16))) && is_aligned(a.x, 16) && is_aligned(a.gamma, 16) &&
                      is_aligned(a.y, 16) && is_aligned(a.sum, 16) && is_aligned(a.codes, 8) && a.group <= 32 * N;
    if (fits && chunks <= 4096) return a.codes || a.scales ? launch_norm_chunks<T, true>(a, chunks, sm_count, stream) : launch_norm_chunks<T, false>(a, chunks, sm_count, stream);
    const uint64_t blocks = (uint64_t)sm_count * 8;
    if (a.cols <= NARROW_COLS) {
        const int threads = narrow_threads(a.cols);
        const unsigned grid = narrow_blocks(a.rows, a.cols, sm_count);
        if (threads == 32) return launch_pdl(lt_norm_narrow<T, 32>, grid, 256, (size_t)0, stream, a);
        if (threads == 64) return launch_pdl(lt_norm_narrow<T, 64>, grid, 256, (size_t)0, stream, a);
        return launch_pdl(lt_norm_narrow<T, 128>, grid, 256, (size_t)0, stream, a);
    }
    return launch_pdl(lt_norm_any<T>, (unsigned)(a.rows < blocks ? a.rows : blocks), 256, (size_t)0, stream, a);
}

// Blocks of the gradient's first kernel, and the threads per row of lt_norm_grad_rows (0: lt_norm_grad_any).  What the
// scratch holds is planned before the addresses are known: the most either takes.
unsigned norm_grad_any_blocks(uint64_t rows, int sm_count) { return (unsigned)std::min<uint64_t>(rows, (uint64_t)sm_count * 2); }
unsigned norm_grad_row_blocks(uint64_t rows, int rt, int sm_count) {
    const uint64_t groups = grad_block(rt) / rt, n = (rows + groups - 1) / groups;
    return (unsigned)std::min<uint64_t>(n, (uint64_t)sm_count * (rt > 256 ? 1 : 2));
}

template <class T, int RT, int CH>
cudaError_t launch_norm_grad_rows(const NormGradArgs &a, unsigned grid, cudaStream_t stream) {
    constexpr int BLOCK = grad_block(RT), GROUPS = BLOCK / RT;
    static_assert((GROUPS - 1) * RT * CH * Chunk<T>::N * 4 <= (int)grad_bytes(RT, CH), "the groups' sums fit");
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_shared(lt_norm_grad_rows<T, RT, CH>, grad_bytes(RT, CH), ready);
    if (e != cudaSuccess) return e;
    return launch_pdl(lt_norm_grad_rows<T, RT, CH>, grid, BLOCK, grad_bytes(RT, CH), stream, a);
}

template <class T, int CH>
cudaError_t launch_norm_grad_threads(const NormGradArgs &a, int rt, unsigned grid, cudaStream_t stream) {
    switch (rt) {
    case 32: return launch_norm_grad_rows<T, 32, CH>(a, grid, stream);
    case 128: return launch_norm_grad_rows<T, 128, CH>(a, grid, stream);
    case 256: return launch_norm_grad_rows<T, 256, CH>(a, grid, stream);
    default: return launch_norm_grad_rows<T, 512, CH>(a, grid, stream);
    }
}

template <class T>
cudaError_t launch_norm_grad(const NormGradArgs &a, int sm_count, cudaStream_t stream, unsigned *grid) {
    constexpr uint64_t N = Chunk<T>::N;
    const bool fits = a.cols % N == 0 && a.dy_pitch % N == 0 && a.h_pitch % N == 0 && (!a.dh || (a.dh_pitch % N == 0 && is_aligned(a.dh, 16))) && is_aligned(a.dy, 16) &&
                      is_aligned(a.h, 16) && is_aligned(a.gamma, 16) && is_aligned(a.dx, 16);
    const uint64_t chunks = a.cols / N;
    if (!fits || chunks > 512 * GRAD_CHUNKS) {
        *grid = norm_grad_any_blocks(a.rows, sm_count);
        if (a.cols <= NARROW_COLS) {
            const int threads = narrow_threads(a.cols);
            *grid = narrow_blocks(a.rows, a.cols, sm_count);
            if (threads == 32) return launch_pdl(lt_norm_grad_narrow<T, 32>, *grid, 256, (size_t)0, stream, a);
            if (threads == 64) return launch_pdl(lt_norm_grad_narrow<T, 64>, *grid, 256, (size_t)0, stream, a);
            return launch_pdl(lt_norm_grad_narrow<T, 128>, *grid, 256, (size_t)0, stream, a);
        }
        return launch_pdl(lt_norm_grad_any<T>, *grid, 256, (size_t)0, stream, a);
    }
    const int rt = row_threads(chunks, a.rows <= 2 * (uint64_t)sm_count && chunks <= 512 ? 1 : GRAD_CHUNKS);
    *grid = norm_grad_row_blocks(a.rows, rt, sm_count);
    if (chunks <= (uint64_t)rt) return launch_norm_grad_threads<T, 1>(a, rt, *grid, stream);
    if (chunks <= 2 * (uint64_t)rt) return launch_norm_grad_threads<T, 2>(a, rt, *grid, stream);
    return launch_norm_grad_threads<T, 4>(a, rt, *grid, stream);
}

}  // namespace

cudaError_t lt_launch_rotary(const LtOperator &o, int sm_count, cudaStream_t stream) {
    TurnArgs a{};
    a.x = o.in[0];
    a.positions = (const int *)o.in[1];
    a.frequencies = (const uint2 *)o.in[2];
    a.out = o.out[0];
    a.tokens = o.rows;
    a.x_pitch = o.pitch[0];
    a.heads = o.heads;
    a.dim = o.dim;
    a.pairs = o.pairs;
    a.interleaved = (int)o.attr[0];
    a.inverse = (int)o.attr[1];
    a.scale = (float)lt_attr_double(o.attr[2]);
    return o.dtype == LT_BF16 ? launch_turn<__nv_bfloat16, false>(a, sm_count, stream) : launch_turn<float, false>(a, sm_count, stream);
}

cudaError_t lt_launch_cache_append(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    const size_t es = o.dtype == LT_BF16 ? 2 : 4;
    *launched = 1;
    if (o.out[0] != o.in[0]) {
        const cudaError_t e = cudaMemcpyAsync(o.out[0], o.in[0], (size_t)o.pages * 2 * o.page * o.kv_heads * o.dim * es, cudaMemcpyDeviceToDevice, stream);
        if (e != cudaSuccess) return e;
    }
    TurnArgs a{};
    a.x = o.in[1];
    a.v = o.in[2];
    a.slots = (const int *)o.in[3];
    a.positions = (const int *)o.in[4];
    a.frequencies = (const uint2 *)o.in[5];
    a.status = &o.status->append;
    a.out = o.out[0];
    a.tokens = o.rows;
    a.x_pitch = o.pitch[1];
    a.v_pitch = o.pitch[2];
    a.heads = o.kv_heads;
    a.dim = o.dim;
    a.pairs = o.pairs;
    a.page = o.page;
    a.n_slots = (uint64_t)o.pages * o.page;
    a.value_offset = (uint64_t)o.page * o.kv_heads * o.dim;
    a.page_stride = 2 * a.value_offset;
    a.token_stride = o.attr[0] ? o.dim : (uint64_t)o.kv_heads * o.dim;
    a.head_stride = o.attr[0] ? (uint64_t)o.page * o.dim : o.dim;
    a.interleaved = (int)o.attr[1];
    a.scale = (float)lt_attr_double(o.attr[2]);
    return o.dtype == LT_BF16 ? launch_turn<__nv_bfloat16, true>(a, sm_count, stream) : launch_turn<float, true>(a, sm_count, stream);
}

cudaError_t lt_launch_rms_norm(const LtOperator &o, int sm_count, cudaStream_t stream) {
    const bool residual = o.attr[1] != 0;
    NormArgs a{};
    a.x = o.in[0];
    a.r = residual ? o.in[1] : nullptr;
    a.gamma = o.in[residual ? 2 : 1];
    a.y = o.out[0];
    a.sum = o.out[1];
    a.codes = (uint8_t *)o.out[2];
    a.scales = (float *)o.out[3];
    a.rows = o.rows;
    a.cols = o.cols;
    a.x_pitch = o.pitch[0];
    a.r_pitch = o.pitch[1];
    a.group = (uint32_t)o.attr[2];
    a.groups = (uint32_t)lt_row_groups(o.cols, o.attr[2]);
    a.eps = (float)lt_attr_double(o.attr[3]);
    mean_factors(o.cols, &a.down, &a.up);
    a.gamma_f32 = o.gamma_dtype == LT_F32;
    return o.dtype == LT_BF16 ? launch_norm<__nv_bfloat16>(a, sm_count, stream) : launch_norm<float>(a, sm_count, stream);
}

size_t lt_rms_norm_grad_scratch(const LtOperator &o, int sm_count) {
    const size_t blocks = o.cols <= NARROW_COLS ? std::max(norm_grad_any_blocks(o.rows, sm_count), narrow_blocks(o.rows, o.cols, sm_count)) : norm_grad_any_blocks(o.rows, sm_count);
    return (o.wanted & 2u) ? blocks * o.cols * sizeof(float) : 0;
}

cudaError_t lt_launch_rms_norm_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    NormGradArgs a{};
    a.dy = o.in[0];
    a.h = o.in[1];
    a.gamma = o.in[2];
    a.dh = o.attr[1] ? o.in[3] : nullptr;
    a.dx = o.out[0];
    a.partial = o.out[1] ? (float *)o.scratch : nullptr;
    a.rows = o.rows;
    a.cols = o.cols;
    a.dy_pitch = o.pitch[0];
    a.h_pitch = o.pitch[1];
    a.dh_pitch = o.pitch[3];
    a.eps = (float)lt_attr_double(o.attr[2]);
    mean_factors(o.cols, &a.down, &a.up);
    a.gamma_f32 = o.gamma_dtype == LT_F32;
    unsigned grid = 0;
    *launched = 1;
    const cudaError_t e = o.dtype == LT_BF16 ? launch_norm_grad<__nv_bfloat16>(a, sm_count, stream, &grid) : launch_norm_grad<float>(a, sm_count, stream, &grid);
    if (e != cudaSuccess || !o.out[1]) return e;
    *launched = 2;
    const uint64_t blocks = (o.cols + 31) / 32;
    const unsigned g2 = (unsigned)(blocks < 4096 ? blocks : 4096);
    return o.gamma_dtype == LT_F32 ? launch_pdl(lt_norm_grad_join<float>, g2, 1024, (size_t)0, stream, (const float *)a.partial, (float *)o.out[1], o.cols, grid)
                                   : launch_pdl(lt_norm_grad_join<__nv_bfloat16>, g2, 1024, (size_t)0, stream, (const float *)a.partial, (__nv_bfloat16 *)o.out[1], o.cols, grid);
}

size_t lt_operator_scratch_bytes(const LtOperator &o, int sm_count) {
    if (o.op == LT_OP_PAGED_ATTENTION) return lt_paged_attention_scratch(o, sm_count);
    if (o.op == LT_OP_RMS_NORM_GRAD) return lt_rms_norm_grad_scratch(o, sm_count);
    if (o.op == LT_OP_EMBEDDING_GRAD) return lt_embedding_grad_scratch(o, sm_count);
    if (o.op == LT_OP_VOCABULARY_LOSS) return lt_vocabulary_loss_scratch(o, sm_count);
    if (o.op == LT_OP_VOCABULARY_LOSS_GRAD) return lt_vocabulary_loss_grad_scratch(o, sm_count);
    return 0;
}

cudaError_t lt_launch_operator(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    *launched = 1;
    switch (o.op) {
    case LT_OP_ROTARY: return lt_launch_rotary(o, sm_count, stream);
    case LT_OP_CACHE_APPEND: return lt_launch_cache_append(o, sm_count, stream, launched);
    case LT_OP_PAGED_ATTENTION: return lt_launch_paged_attention(o, sm_count, stream);
    case LT_OP_RMS_NORM: return lt_launch_rms_norm(o, sm_count, stream);
    case LT_OP_RMS_NORM_GRAD: return lt_launch_rms_norm_grad(o, sm_count, stream, launched);
    case LT_OP_EMBEDDING: return lt_launch_embedding(o, sm_count, stream);
    case LT_OP_EMBEDDING_GRAD: return lt_launch_embedding_grad(o, sm_count, stream, launched);
    case LT_OP_VOCABULARY_LOSS: return lt_launch_vocabulary_loss(o, sm_count, stream, launched);
    case LT_OP_VOCABULARY_LOSS_GRAD: return lt_launch_vocabulary_loss_grad(o, sm_count, stream, launched);
    default: return cudaErrorInvalidValue;
    }
}

cudaError_t lt_static_arrivals(void **out) { return address_of(lt_operator_arrivals, g_arrivals, out); }

cudaError_t lt_operator_status_claim(LtOperatorStatus **out) {
    std::lock_guard<std::mutex> hold(g_lock);
    if (!g_status) {
        void *p = nullptr;
        cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // (the first context may be made while a stream is captured)
        cudaThreadExchangeStreamCaptureMode(&mode);
        const cudaError_t e = cudaHostAlloc(&p, kStatusWords * sizeof(LtOperatorStatus), cudaHostAllocPortable | cudaHostAllocMapped);
        cudaThreadExchangeStreamCaptureMode(&mode);
        if (e != cudaSuccess) return e;
        memset(p, 0, kStatusWords * sizeof(LtOperatorStatus));
        g_status = (LtOperatorStatus *)p;
        for (size_t i = 1; i < kStatusWords; ++i) g_status_free.push_back(g_status + i);
    }
    *out = g_status;
    if (g_status_free.empty()) return cudaSuccess;
    *out = g_status_free.front();
    g_status_free.pop_front();
    lt_operator_status_take(*out);
    return cudaSuccess;
}

void lt_operator_status_return(LtOperatorStatus *status) {
    std::lock_guard<std::mutex> hold(g_lock);
    if (status && status != g_status) g_status_free.push_back(status);
}

LtOperatorStatus lt_operator_status_take(LtOperatorStatus *status) {
    LtOperatorStatus s;
    s.attention = __atomic_exchange_n(&status->attention, 0u, __ATOMIC_ACQ_REL);
    s.append = __atomic_exchange_n(&status->append, 0u, __ATOMIC_ACQ_REL);
    s.embedding = __atomic_exchange_n(&status->embedding, 0u, __ATOMIC_ACQ_REL);
    s.loss = __atomic_exchange_n(&status->loss, 0u, __ATOMIC_ACQ_REL);
    s.timeout = lt_operator_timeout_take(status);
    return s;
}

unsigned lt_operator_timeout_take(LtOperatorStatus *status) { return __atomic_exchange_n(&status->timeout, 0u, __ATOMIC_ACQ_REL); }
