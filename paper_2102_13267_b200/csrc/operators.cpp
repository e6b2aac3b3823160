// The transformer operators on the host side: checks of their operands, shapes of their results, what the planner and the
// executor ask about them.  The kernels are in operators.cu (rotary, cache_append, norms) and attention.cu.
#include <cmath>
#include <cstring>
#include <string>

#include "engine.h"

namespace lt {

namespace {

bool is_float(int dt) { return dt == LT_F32 || dt == LT_BF16; }

bool same_shape(const Node &a, const Node &b) {
    if (a.rank != b.rank) return false;
    for (int i = 0; i < a.rank; ++i)
        if (a.dims[i] != b.dims[i]) return false;
    return true;
}

bool flag(int64_t v) { return v == 0 || v == 1; }

}  // namespace

// Shape and dtype of the result `opcode` gives on these operands, or why it gives none.
lt_status operator_infer(lt_ctx *c, int opcode, const Node *const *ops, int n_in, const int64_t *attrs, int n_attrs, int64_t *od, int *orank,
                         int *odtype) {
    const std::string name = op_name(opcode);
    auto bad = [&](lt_status s, const std::string &why) { return fail(c, s, name + ": " + why); };
    static const int want_attrs[] = {3, 3, 2, 4, 3};
    if (n_attrs != want_attrs[opcode - LT_OP_ROTARY]) return bad(LT_ERR_INVALID_ARG, "wrong number of attributes");
    for (int i = 0; i < n_in; ++i)
        if (ops[i]->op == N_SCALAR) return bad(LT_ERR_INVALID_ARG, "operands are tensors, not constants");
    auto finite = [](int64_t bits) { return std::isfinite(lt_attr_double(bits)); };
    auto result = [&](const Node &like, int dtype) {
        *orank = like.rank;
        for (int i = 0; i < like.rank; ++i) od[i] = like.dims[i];
        *odtype = dtype;
    };
    // frequencies as cache_append and rotary take them, for heads of `dim` values
    auto check_positions = [&](const Node &pos, const Node &freq, int64_t tokens, int64_t dim) -> lt_status {
        if (pos.dtype != LT_I32 || pos.rank != 1) return bad(LT_ERR_DTYPE, "positions are an i32 vector");
        if (pos.dims[0] != tokens) return bad(LT_ERR_SHAPE, "one position per token is needed");
        if (freq.dtype != LT_U32 || freq.rank != 2 || freq.dims[1] != 2) return bad(LT_ERR_DTYPE, "frequencies are a u32 tensor [pairs, 2]");
        if (2 * freq.dims[0] > dim) return bad(LT_ERR_SHAPE, "more pairs than a head has");
        return LT_OK;
    };

    if (opcode == LT_OP_ROTARY) {
        if (n_in != 3 && n_in != 4) return bad(LT_ERR_INVALID_ARG, "takes x, positions, frequencies and optionally the result's buffer");
        if (!flag(attrs[0]) || !flag(attrs[1]) || !finite(attrs[2])) return bad(LT_ERR_INVALID_ARG, "attrs are {interleaved, inverse, scale}");
        const Node &x = *ops[0];
        if (!is_float(x.dtype)) return bad(LT_ERR_DTYPE, "x is f32 or bf16");
        if (x.rank < 2) return bad(LT_ERR_SHAPE, "x is [tokens, .., head size]");
        const lt_status s = check_positions(*ops[1], *ops[2], x.dims[0], x.dims[x.rank - 1]);
        if (s) return s;
        if (x.dims[x.rank - 1] >= (1 << 20) || x.dims[0] >= (1ll << 31) || shape_numel(x.dims, x.rank) / x.dims[0] >= (1ll << 31))
            return bad(LT_ERR_UNSUPPORTED, "more tokens or values per token than the kernel counts");
        result(x, x.dtype);
    } else if (opcode == LT_OP_CACHE_APPEND) {
        if (n_in != 4 && n_in != 6) return bad(LT_ERR_INVALID_ARG, "takes cache, k, v, slots and optionally positions, frequencies");
        if (!flag(attrs[0]) || !flag(attrs[1]) || !finite(attrs[2])) return bad(LT_ERR_INVALID_ARG, "attrs are {head_major, interleaved, scale}");
        const Node &ca = *ops[0], &k = *ops[1], &v = *ops[2], &sl = *ops[3];
        if (!is_float(ca.dtype) || k.dtype != ca.dtype || v.dtype != ca.dtype) return bad(LT_ERR_DTYPE, "cache, k and v are all f32 or all bf16");
        if (ca.rank != 5 || ca.dims[1] != 2) return bad(LT_ERR_SHAPE, "the cache is [pages, 2, page, heads, head size], or [pages, 2, heads, page, head size] with head_major");
        const int64_t heads = attrs[0] ? ca.dims[2] : ca.dims[3], page = attrs[0] ? ca.dims[3] : ca.dims[2];
        if (k.rank != 3 || !same_shape(k, v) || k.dims[1] != heads || k.dims[2] != ca.dims[4]) return bad(LT_ERR_SHAPE, "k and v are [tokens, heads, head size] of the cache");
        if (sl.dtype != LT_I32 || sl.rank != 1) return bad(LT_ERR_DTYPE, "slots are an i32 vector");
        if (sl.dims[0] != k.dims[0]) return bad(LT_ERR_SHAPE, "one slot per token is needed");
        if (ca.dims[0] > 0x7fffffffll / page) return bad(LT_ERR_UNSUPPORTED, "the cache has more slots than an i32 numbers");
        if (ca.dims[4] >= (1 << 20) || heads * ca.dims[4] >= (1ll << 31)) return bad(LT_ERR_UNSUPPORTED, "more values per token than the kernel counts");
        if (n_in == 6) {
            const lt_status s = check_positions(*ops[4], *ops[5], k.dims[0], ca.dims[4]);
            if (s) return s;
        }
        result(ca, ca.dtype);
    } else if (opcode == LT_OP_PAGED_ATTENTION) {
        if (n_in != 4 && n_in != 5) return bad(LT_ERR_INVALID_ARG, "takes q, cache, page table, lengths and optionally the result's buffer");
        if (!flag(attrs[0]) || !finite(attrs[1])) return bad(LT_ERR_INVALID_ARG, "attrs are {head_major, scale}");
        const Node &q = *ops[0], &ca = *ops[1], &tb = *ops[2], &ln = *ops[3];
        if (!is_float(q.dtype) || ca.dtype != q.dtype) return bad(LT_ERR_DTYPE, "q and the cache are both f32 or both bf16");
        if (q.rank != 3) return bad(LT_ERR_SHAPE, "q is [sequences, heads, head size]");
        if (ca.rank != 5 || ca.dims[1] != 2) return bad(LT_ERR_SHAPE, "the cache is [pages, 2, page, heads, head size], or [pages, 2, heads, page, head size] with head_major");
        const int64_t kv = attrs[0] ? ca.dims[2] : ca.dims[3], page = attrs[0] ? ca.dims[3] : ca.dims[2];
        if (q.dims[2] != ca.dims[4] || q.dims[1] % kv) return bad(LT_ERR_SHAPE, "q's heads are a multiple of the cache's, with the same head size");
        if (q.dims[2] > 256) return bad(LT_ERR_UNSUPPORTED, "heads of more than 256 values");
        if (tb.dtype != LT_I32 || ln.dtype != LT_I32) return bad(LT_ERR_DTYPE, "page table and lengths are i32");
        if (tb.rank != 2 || tb.dims[0] != q.dims[0] || ln.rank != 1 || ln.dims[0] != q.dims[0])
            return bad(LT_ERR_SHAPE, "the page table is [sequences, most pages of one], lengths [sequences]");
        if (ca.dims[0] > 0x7fffffffll || tb.dims[1] > (1ll << 30) / page) return bad(LT_ERR_UNSUPPORTED, "more than 2^30 tokens per sequence");  // (so that a step beyond the last token has a number too)
        if (q.dims[0] > 65535 || q.dims[0] * q.dims[1] >= (1ll << 31)) return bad(LT_ERR_UNSUPPORTED, "more than 65535 sequences, or more heads than the kernel counts");
        // (tiles of 64 tokens, two more for each beginning: the kernel numbers them in 31 bits)
        if ((double)q.dims[0] * (double)q.dims[1] * ((double)(tb.dims[1] * page) / 64.0 + 3.0) >= 2147483648.0)
            return bad(LT_ERR_UNSUPPORTED, "sequences x heads x the most tokens a sequence can hold are more than the kernel counts");
        result(q, q.dtype);
    } else if (opcode == LT_OP_RMS_NORM) {
        if (!flag(attrs[1])) return bad(LT_ERR_INVALID_ARG, "attrs are {result, residual, group, eps}");
        const int core = 2 + (int)attrs[1];
        if (n_in != core && n_in != core + 1) return bad(LT_ERR_INVALID_ARG, "takes x, the residual if there is one, gamma and optionally the result's buffer");
        if (attrs[0] < 0 || attrs[0] > 3) return bad(LT_ERR_INVALID_ARG, "result is 0 (normalised), 1 (sum), 2 (8-bit codes) or 3 (scales)");
        if (attrs[0] == 1 && !attrs[1]) return bad(LT_ERR_INVALID_ARG, "without a residual there is no sum");
        if (attrs[2] != 0 && attrs[2] != 32 && attrs[2] != 64 && attrs[2] != 128 && attrs[2] != 256)
            return bad(LT_ERR_INVALID_ARG, "group is 0 (the row), 32, 64, 128 or 256 columns");
        const double eps = lt_attr_double(attrs[3]);
        if (!std::isfinite(eps) || eps < 0) return bad(LT_ERR_INVALID_ARG, "eps is not negative");
        const Node &x = *ops[0], &gamma = *ops[core - 1];
        if (!is_float(x.dtype) || (gamma.dtype != LT_F32 && gamma.dtype != x.dtype)) return bad(LT_ERR_DTYPE, "x is f32 or bf16, gamma f32 or like x");
        if (x.rank < 1) return bad(LT_ERR_SHAPE, "x has at least one dimension");
        if (attrs[1] && (ops[1]->dtype != x.dtype || !same_shape(*ops[1], x))) return bad(LT_ERR_SHAPE, "the residual has x's shape and dtype");
        const int64_t cols = x.dims[x.rank - 1];
        if (gamma.rank != 1 || gamma.dims[0] != cols) return bad(LT_ERR_SHAPE, "gamma is a vector of the row's length");
        if (cols >= (1ll << 30) || shape_numel(x.dims, x.rank) / cols >= (1ll << 31)) return bad(LT_ERR_UNSUPPORTED, "more rows or columns than the kernel counts");
        result(x, attrs[0] == 2 ? LT_U8 : attrs[0] == 3 ? LT_F32 : x.dtype);
        if (attrs[0] == 3) od[*orank - 1] = (int64_t)lt_row_groups((uint64_t)cols, attrs[2]);
    } else {  // LT_OP_RMS_NORM_GRAD
        if (!flag(attrs[1])) return bad(LT_ERR_INVALID_ARG, "attrs are {result, residual gradient, eps}");
        const int core = 3 + (int)attrs[1];
        if (n_in != core && n_in != core + 1)
            return bad(LT_ERR_INVALID_ARG, "takes dy, what was normalised, gamma, the sum's own gradient if there is one and optionally the result's buffer");
        if (!flag(attrs[0])) return bad(LT_ERR_INVALID_ARG, "result is 0 (gradient of the input) or 1 (of gamma)");
        const double eps = lt_attr_double(attrs[2]);
        if (!std::isfinite(eps) || eps < 0) return bad(LT_ERR_INVALID_ARG, "eps is not negative");
        const Node &dy = *ops[0], &h = *ops[1], &gamma = *ops[2];
        if (!is_float(h.dtype) || dy.dtype != h.dtype || (gamma.dtype != LT_F32 && gamma.dtype != h.dtype))
            return bad(LT_ERR_DTYPE, "dy and h are both f32 or both bf16, gamma f32 or like them");
        if (h.rank < 1 || !same_shape(dy, h)) return bad(LT_ERR_SHAPE, "dy and h have one shape");
        if (attrs[1] && (ops[3]->dtype != h.dtype || !same_shape(*ops[3], h))) return bad(LT_ERR_SHAPE, "the sum's gradient has h's shape and dtype");
        const int64_t cols = h.dims[h.rank - 1];
        if (gamma.rank != 1 || gamma.dims[0] != cols) return bad(LT_ERR_SHAPE, "gamma is a vector of the row's length");
        if (cols >= (1ll << 30) || shape_numel(h.dims, h.rank) / cols >= (1ll << 31)) return bad(LT_ERR_UNSUPPORTED, "more rows or columns than the kernel counts");
        if (attrs[0]) result(gamma, gamma.dtype);
        else result(h, h.dtype);
    }
    const int core = operator_inputs(opcode, n_in, attrs);
    if (n_in > core) {
        const Node &b = *ops[core];
        bool same = b.dtype == *odtype && b.rank == *orank;
        for (int i = 0; same && i < *orank; ++i) same = b.dims[i] == od[i];
        if (!same) return bad(LT_ERR_SHAPE, "the buffer for the result has another shape or dtype");
    }
    return LT_OK;
}

int operator_core_inputs(const CNode &n) {
    const int64_t attrs[4] = {n.attr0, n.attr1, n.attr2, n.attr3};
    return operator_inputs(n.op, n.n_in, attrs);
}

// which of its operator's results a node is
int operator_result(const CNode &n) { return n.op == LT_OP_RMS_NORM || n.op == LT_OP_RMS_NORM_GRAD ? (int)n.attr0 : 0; }

// Two nodes that are results (the same or different ones) of one operator on the same operands.
bool operator_same_launch(const CNode &a, const CNode &b) {
    if (a.op != b.op || a.attr1 != b.attr1 || a.attr2 != b.attr2 || a.attr3 != b.attr3) return false;
    const bool selects = a.op == LT_OP_RMS_NORM || a.op == LT_OP_RMS_NORM_GRAD;
    if (!selects && a.attr0 != b.attr0) return false;
    const int core = operator_core_inputs(a);
    if (core != operator_core_inputs(b)) return false;
    for (int k = 0; k < core; ++k)
        if (a.in[k] != b.in[k]) return false;
    return true;
}

// Rows (tokens, sequences) of operand k, when the kernel takes a distance between them: such an operand may be a slice
// that is read in place.  0: the operand has to be dense.
uint64_t operator_operand_rows(const CNode &n, int k, const CNode &operand) {
    bool row_operand = false, last_dim = false;
    const int core = operator_core_inputs(n);
    switch (n.op) {
    case LT_OP_ROTARY: case LT_OP_PAGED_ATTENTION: row_operand = k == 0; break;
    case LT_OP_CACHE_APPEND: row_operand = k == 1 || k == 2; break;
    case LT_OP_RMS_NORM: row_operand = k < core - 1; last_dim = true; break;
    default: row_operand = k < core && k != 2; last_dim = true; break;
    }
    if (!row_operand) return 0;
    uint64_t rows = 1;
    for (int d = 0; d < (last_dim ? operand.rank - 1 : 1); ++d) rows *= (uint64_t)operand.dims[d];
    return rows;
}

// May the result be written over operand k?  Yes where a thread reads its elements of that operand before it writes the
// same ones, and nobody else reads them.
bool operator_in_place(const CNode &n, int k) {
    const int core = operator_core_inputs(n);
    switch (n.op) {
    case LT_OP_ROTARY: case LT_OP_CACHE_APPEND: return k == 0;
    case LT_OP_RMS_NORM: return (n.attr0 == 0 || n.attr0 == 1) && k < core - 1;
    case LT_OP_RMS_NORM_GRAD: return n.attr0 == 0 && k < core && k != 2;
    default: return false;
    }
}

// Sizes of the launch of which `n` is a result; which results are wanted is added by the planner's later results.
void operator_fill(const Canonical &cg, const CNode &n, LtOperator &o) {
    memset(&o, 0, sizeof(o));
    o.op = n.op;
    o.n_in = operator_core_inputs(n);
    o.attr[0] = n.attr0;
    o.attr[1] = n.attr1;
    o.attr[2] = n.attr2;
    o.attr[3] = n.attr3;
    const CNode &x = cg.nodes[n.in[0]];
    o.dtype = x.dtype;
    auto inner = [&](const CNode &t, int from) {
        uint64_t v = 1;
        for (int d = from; d < t.rank; ++d) v *= (uint64_t)t.dims[d];
        return v;
    };
    if (n.op == LT_OP_ROTARY) {
        o.rows = (uint64_t)x.dims[0];
        o.dim = (uint32_t)x.dims[x.rank - 1];
        o.heads = (uint32_t)(inner(x, 1) / o.dim);
        o.pairs = (uint32_t)cg.nodes[n.in[2]].dims[0];
        o.pitch[0] = inner(x, 1);
    } else if (n.op == LT_OP_CACHE_APPEND) {
        const CNode &k = cg.nodes[n.in[1]];
        o.rows = (uint64_t)k.dims[0];
        o.kv_heads = (uint32_t)k.dims[1];
        o.dim = (uint32_t)k.dims[2];
        o.pages = (uint32_t)x.dims[0];
        o.page = (uint32_t)(n.attr0 ? x.dims[3] : x.dims[2]);
        o.pairs = o.n_in == 6 ? (uint32_t)cg.nodes[n.in[5]].dims[0] : 0;
        o.pitch[1] = o.pitch[2] = inner(k, 1);
    } else if (n.op == LT_OP_PAGED_ATTENTION) {
        const CNode &ca = cg.nodes[n.in[1]];
        o.rows = (uint64_t)x.dims[0];
        o.heads = (uint32_t)x.dims[1];
        o.dim = (uint32_t)x.dims[2];
        o.pages = (uint32_t)ca.dims[0];
        o.kv_heads = (uint32_t)(n.attr0 ? ca.dims[2] : ca.dims[3]);
        o.page = (uint32_t)(n.attr0 ? ca.dims[3] : ca.dims[2]);
        o.table_width = (uint32_t)cg.nodes[n.in[2]].dims[1];
        o.pitch[0] = inner(x, 1);
    } else {
        const int gamma = n.op == LT_OP_RMS_NORM ? o.n_in - 1 : 2;
        o.cols = (uint64_t)x.dims[x.rank - 1];
        o.rows = inner(x, 0) / o.cols;
        o.gamma_dtype = cg.nodes[n.in[gamma]].dtype;
        for (int k = 0; k < o.n_in; ++k) o.pitch[k] = o.cols;
    }
}

// bytes a launch is planned to move (a cache: as much of it as the page table can name)
uint64_t operator_bytes(const LtOperator &o) {
    const uint64_t es = dtype_size(o.dtype);
    switch (o.op) {
    case LT_OP_ROTARY: return 2 * o.rows * o.heads * o.dim * es + 4 * o.rows + 8ull * o.pairs;
    case LT_OP_CACHE_APPEND: return 4 * o.rows * o.kv_heads * o.dim * es + 8 * o.rows;
    case LT_OP_PAGED_ATTENTION: {
        const uint64_t named = o.rows * o.table_width < o.pages ? o.rows * o.table_width : o.pages;
        return 2 * o.rows * o.heads * o.dim * es + named * o.page * o.kv_heads * o.dim * 2 * es + 4 * o.rows * o.table_width;
    }
    case LT_OP_RMS_NORM: {
        uint64_t b = (uint64_t)(o.n_in - 1) * o.rows * o.cols * es;
        if (o.wanted & 1u) b += o.rows * o.cols * es;
        if (o.wanted & 2u) b += o.rows * o.cols * es;
        if (o.wanted & 4u) b += o.rows * o.cols;
        if (o.wanted & 8u) b += 4 * o.rows * lt_row_groups(o.cols, o.attr[2]);
        return b + o.cols * dtype_size(o.gamma_dtype);
    }
    default: return (uint64_t)(o.n_in - 1 + (o.wanted & 1u)) * o.rows * o.cols * es + 2 * o.cols * dtype_size(o.gamma_dtype);
    }
}

}  // namespace lt
