// The transformer operators: what a launch needs to know, shared by the host runtime and the kernels.
#pragma once
#include <cuda_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lazytensor.h"

#define LT_OPERATOR_INPUTS 6
#define LT_OPERATOR_RESULTS 4

// Where a context's operators leave word that an index in device memory lay outside what it indexes.
struct LtOperatorStatus {
    unsigned int attention, append, embedding, loss;
    unsigned int timeout;                  // a wait inside a kernel ran out of time
};

// One launch of an operator.  Everything but the addresses is known when the graph is planned.
struct LtOperator {
    int op;
    int dtype;                             // of the data: x, the cache, ..
    int gamma_dtype;                       // norms; embedding_grad: of the result and the base
    int n_in;                              // operands that are read
    int64_t attr[4];                       // as passed to lt_op
    const void *in[LT_OPERATOR_INPUTS];
    uint64_t pitch[LT_OPERATOR_INPUTS];    // row operands: elements from one row (token) to the next
    void *out[LT_OPERATOR_RESULTS];        // per result; null where the graph does not ask for it
    unsigned wanted;                       // bit k: result k is asked for
    void *scratch;
    LtOperatorStatus *status;              // operators that follow indices in device memory
    uint64_t wait_ns;                      // how long a wait inside a kernel may last
    void *arrivals;                        // paged_attention: LT_ARRIVALS counters that are zero between launches
    // sizes (those that the operator has)
    uint64_t rows;                         // tokens, sequences or rows
    uint32_t heads, kv_heads, dim, pairs;  // pairs: rotated pairs of a head
    uint32_t pages, page, table_width;
    uint64_t cols;
    uint64_t vocabulary;                   // rows of a table that tokens name
};

static inline double lt_attr_double(int64_t bits) {
    double d;
    __builtin_memcpy(&d, &bits, 8);
    return d;
}

// Groups of a quantised row: `group` columns each (0: the whole row), the last one possibly shorter.
static inline uint64_t lt_row_groups(uint64_t cols, int64_t group) { return group > 0 ? (cols + (uint64_t)group - 1) / (uint64_t)group : 1; }

// How many of an operation's `n_in` operands the operator reads; one more is the buffer meant for its result.
static inline int operator_inputs(int op, int n_in, const int64_t *attrs) {
    switch (op) {
    case LT_OP_ROTARY: return 3;
    case LT_OP_CACHE_APPEND: return n_in;
    case LT_OP_PAGED_ATTENTION: return 4;
    case LT_OP_RMS_NORM: return 2 + (attrs[1] ? 1 : 0);
    case LT_OP_EMBEDDING: return 2;
    case LT_OP_EMBEDDING_GRAD: return 2 + (attrs[1] ? 1 : 0);
    case LT_OP_VOCABULARY_LOSS: return 3;
    case LT_OP_VOCABULARY_LOSS_GRAD: return 5;
    default: return 3 + (attrs[1] ? 1 : 0);  // LT_OP_RMS_NORM_GRAD
    }
}

size_t lt_operator_scratch_bytes(const LtOperator &o, int sm_count);
// Counters of blocks that have left their part of a result that several share.  A context has its own for its flushes, a
// graph that captures one has its own in the graph's memory; flushes that may not allocate share one array per device, like
// the static scratch.
#define LT_ARRIVALS 2048
cudaError_t lt_static_arrivals(void **out);
// Enqueues the operator on `stream`; *launched receives the number of kernels.
cudaError_t lt_launch_operator(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
// A status for a context, which gives it back when it is destroyed.
cudaError_t lt_operator_status_claim(LtOperatorStatus **out);
void lt_operator_status_return(LtOperatorStatus *status);
// What was left there since the last call (by kernels that have completed), and is from now on not.
LtOperatorStatus lt_operator_status_take(LtOperatorStatus *status);
// The same for a wait that ran out alone; words about indices stay.
unsigned lt_operator_timeout_take(LtOperatorStatus *status);

// the operators' own launchers
cudaError_t lt_launch_rotary(const LtOperator &o, int sm_count, cudaStream_t stream);
cudaError_t lt_launch_cache_append(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
cudaError_t lt_launch_paged_attention(const LtOperator &o, int sm_count, cudaStream_t stream);
size_t lt_paged_attention_scratch(const LtOperator &o, int sm_count);
cudaError_t lt_launch_rms_norm(const LtOperator &o, int sm_count, cudaStream_t stream);
cudaError_t lt_launch_rms_norm_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
size_t lt_rms_norm_grad_scratch(const LtOperator &o, int sm_count);
cudaError_t lt_launch_embedding(const LtOperator &o, int sm_count, cudaStream_t stream);
cudaError_t lt_launch_embedding_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
size_t lt_embedding_grad_scratch(const LtOperator &o, int sm_count);
cudaError_t lt_launch_vocabulary_loss(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
size_t lt_vocabulary_loss_scratch(const LtOperator &o, int sm_count);
cudaError_t lt_launch_vocabulary_loss_grad(const LtOperator &o, int sm_count, cudaStream_t stream, unsigned *launched);
size_t lt_vocabulary_loss_grad_scratch(const LtOperator &o, int sm_count);
// A kernel whose bounded wait, that of the matrix products, runs out after `limit_ns`.
cudaError_t lt_launch_product_wait_probe(LtOperatorStatus *status, uint64_t limit_ns, cudaStream_t stream);
