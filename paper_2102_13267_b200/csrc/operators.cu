// Kernels of the transformer operators that move every value once: rotary positions, appending to a paged key-value
// cache, the root-mean-square norm (with the residual's addition and an 8-bit output) and its gradient.  The attention
// that reads the cache is in attention.cu.
#include <cuda_fp8.h>

#include <mutex>

#include "operator_device.cuh"

using namespace ltop;

static __device__ unsigned int lt_operator_status = 0;
static __device__ unsigned int lt_operator_arrivals[LT_ARRIVALS];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_lock;
void *g_status[kMaxDevices], *g_arrivals[kMaxDevices];

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
        atomicOr(a.status, 2u);
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

template <class T, bool APPEND>
cudaError_t launch_turn(const TurnArgs &a, int sm_count, cudaStream_t stream) {
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
    float eps;
    float down, up;             // 2^-k <= 1 / cols and 2^k / cols: a mean of squares is summed as h (h 2^-k), which fits where the mean does
    int gamma_f32;
};

template <class T>
__device__ __forceinline__ float gamma_at(const void *gamma, int f32, uint64_t c) {
    return f32 ? ((const float *)gamma)[c] : to_float(((const T *)gamma)[c]);
}

// 448 / top, the factor from values to e4m3 codes (0 for a group of zeros; a group so small that the quotient would
// overflow takes the largest number instead)
__device__ __forceinline__ float code_factor(float top) {
    if (top == 0.f) return 0.f;
    return fminf(__fdiv_rn(448.f, top), 3.402823466e38f) + (top != top ? top : 0.f);
}

// Any shape and alignment: a block per row, which is read once for its mean square, once more for each output.
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
                if (a.scales && threadIdx.x == 0) a.scales[row] = __fdiv_rn(top, 448.f);
                const float f = code_factor(top);
                if (a.codes)
                    for (uint64_t c = threadIdx.x; c < a.cols; c += 256)
                        a.codes[row * a.cols + c] = __nv_cvt_float_to_fp8(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c) * f, __NV_SATFINITE, __NV_E4M3);
            } else {
                for (uint32_t g = threadIdx.x >> 5; g < a.groups; g += 8) {  // a warp per group
                    const uint64_t c0 = (uint64_t)g * a.group, c1 = min(c0 + a.group, a.cols);
                    float top = 0.f;
                    for (uint64_t c = c0 + (threadIdx.x & 31); c < c1; c += 32) top = max_nan(top, fabsf(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c)));
                    top = warp_max_nan(top);
                    if (a.scales && (threadIdx.x & 31) == 0) a.scales[row * a.groups + g] = __fdiv_rn(top, 448.f);
                    const float f = code_factor(top);
                    if (a.codes)
                        for (uint64_t c = c0 + (threadIdx.x & 31); c < c1; c += 32)
                            a.codes[row * a.cols + c] = __nv_cvt_float_to_fp8(h_at(c) * inv * gamma_at<T>(a.gamma, a.gamma_f32, c) * f, __NV_SATFINITE, __NV_E4M3);
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

struct NormGradArgs {
    const void *dy, *h, *gamma, *dh;
    void *dx;
    float *partial;             // [blocks, cols], or null
    uint64_t rows, cols, dy_pitch, h_pitch, dh_pitch;
    float eps, down, up;
    int gamma_f32;
};

// u = h / rms.  dx = dh + (gamma dy - u mean(gamma dy u)) / rms; a block adds up dy u over its rows in its own row of
// `partial`.
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
        const float inv = rsqrtf(ss * a.up + a.eps), m = dot * inv * a.up;
        for (uint64_t c = threadIdx.x; c < a.cols; c += 256) {
            const float d = to_float(dy[c]), u = to_float(h[c]) * inv;
            const float g = (d * gamma_at<T>(a.gamma, a.gamma_f32, c) - u * m) * inv + (dh ? to_float(dh[c]) : 0.f);
            if (a.dx) ((T *)a.dx)[row * a.cols + c] = from_float<T>(g);
            if (mine) mine[c] += d * u;
        }
    }
}

// The blocks' sums, in their order, in binary64.
template <class G>
__global__ void __launch_bounds__(256) lt_norm_grad_join(const float *partial, G *out, uint64_t cols, unsigned blocks) {
    pdl_release();
    pdl_wait();
    for (uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (uint64_t)gridDim.x * 256) {
        double s = 0.0;
        for (unsigned b = 0; b < blocks; ++b) s += (double)partial[(uint64_t)b * cols + c];
        out[c] = from_float<G>((float)s);
    }
}

// 2^-k with 2^k >= cols, and 2^k / cols
void mean_factors(uint64_t cols, float *down, float *up) {
    int k = 0;
    while ((1ull << k) < cols) ++k;
    *down = (float)(1.0 / (double)(1ull << k));
    *up = (float)((double)(1ull << k) / (double)cols);
}

unsigned norm_grad_blocks(const LtOperator &o, int sm_count) {
    const uint64_t most = (uint64_t)sm_count * 4;
    return (unsigned)(o.rows < most ? o.rows : most);
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

cudaError_t lt_launch_cache_append(const LtOperator &o, unsigned int *status, int sm_count, cudaStream_t stream, unsigned *launched) {
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
    a.status = status;
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
    const uint64_t most = (uint64_t)sm_count * 8;
    const unsigned grid = (unsigned)(o.rows < most ? o.rows : most);
    return o.dtype == LT_BF16 ? launch_pdl(lt_norm_any<__nv_bfloat16>, grid, 256, (size_t)0, stream, a) : launch_pdl(lt_norm_any<float>, grid, 256, (size_t)0, stream, a);
}

size_t lt_rms_norm_grad_scratch(const LtOperator &o, int sm_count) {
    return (o.wanted & 2u) ? (size_t)norm_grad_blocks(o, sm_count) * o.cols * sizeof(float) : 0;
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
    const unsigned grid = norm_grad_blocks(o, sm_count);
    *launched = 1;
    cudaError_t e = o.dtype == LT_BF16 ? launch_pdl(lt_norm_grad_any<__nv_bfloat16>, grid, 256, (size_t)0, stream, a)
                                       : launch_pdl(lt_norm_grad_any<float>, grid, 256, (size_t)0, stream, a);
    if (e != cudaSuccess || !o.out[1]) return e;
    *launched = 2;
    const uint64_t blocks = (o.cols + 255) / 256;
    const unsigned g2 = (unsigned)(blocks < 4096 ? blocks : 4096);
    return o.gamma_dtype == LT_F32 ? launch_pdl(lt_norm_grad_join<float>, g2, 256, (size_t)0, stream, (const float *)a.partial, (float *)o.out[1], o.cols, grid)
                                   : launch_pdl(lt_norm_grad_join<__nv_bfloat16>, g2, 256, (size_t)0, stream, (const float *)a.partial, (__nv_bfloat16 *)o.out[1], o.cols, grid);
}

size_t lt_operator_scratch_bytes(const LtOperator &o, int sm_count) {
    if (o.op == LT_OP_PAGED_ATTENTION) return lt_paged_attention_scratch(o, sm_count);
    if (o.op == LT_OP_RMS_NORM_GRAD) return lt_rms_norm_grad_scratch(o, sm_count);
    return 0;
}

cudaError_t lt_launch_operator(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched) {
    *launched = 1;
    void *word = nullptr;
    if (o.op == LT_OP_CACHE_APPEND || o.op == LT_OP_PAGED_ATTENTION) {
        const cudaError_t e = address_of(lt_operator_status, g_status, &word);
        if (e != cudaSuccess) return e;
    }
    unsigned int *status = (unsigned int *)word;
    switch (o.op) {
    case LT_OP_ROTARY: return lt_launch_rotary(o, sm_count, stream);
    case LT_OP_CACHE_APPEND: return lt_launch_cache_append(o, status, sm_count, stream, launched);
    case LT_OP_PAGED_ATTENTION: return lt_launch_paged_attention(o, status, sm_count, stream);
    case LT_OP_RMS_NORM: return lt_launch_rms_norm(o, sm_count, stream);
    case LT_OP_RMS_NORM_GRAD: return lt_launch_rms_norm_grad(o, sm_count, stream, launched);
    default: return cudaErrorInvalidValue;
    }
}

cudaError_t lt_static_arrivals(void **out) { return address_of(lt_operator_arrivals, g_arrivals, out); }

cudaError_t lt_operator_status_read(unsigned int *out) {
    cudaError_t e = cudaMemcpyFromSymbol(out, lt_operator_status, sizeof(*out));
    if (e == cudaSuccess && *out) {
        const unsigned int zero = 0;
        e = cudaMemcpyToSymbol(lt_operator_status, &zero, sizeof(zero));
    }
    return e;
}
