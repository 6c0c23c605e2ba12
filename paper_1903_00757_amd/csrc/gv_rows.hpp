// Internal interface between the checks of the operators on rows (gv_rows_api.cpp) and their kernels (gv_rows.hip, gv_scores.hip,
// gv_lookup.hip, gv_dense.hip, gv_select.hip).  Not part of the C boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace gv {

// Items i = 0, 1, ... of rows of `each` items, taken by threads in turn: a thread goes on by the grid's threads, which are
// rows_on rows and items_on items (divided on the host).
struct Walk {
    uint64_t all, stride, rows_on;
    uint32_t each, items_on;
};
inline Walk walk_of(uint64_t rows, uint32_t each, uint64_t threads) {
    return {rows * each, threads, threads / each, each, (uint32_t)(threads % each)};
}

struct DropArgs {
    uint32_t threshold;  // a value is kept when its 16-bit number is not below; 0: all are kept
    float factor;        // of the values that are kept
    uint64_t seed, first_row;
};

struct NormArgs {
    const void *x, *residual;  // residual may be null
    const float *gain;
    void *sum, *out;           // sum may be null
    float *out_scale, *rstd;   // rstd may be null
    uint64_t rows, x_stride, residual_stride, sum_stride, out_stride;
    uint32_t cols;
    int type, out_type;
    float eps;
    DropArgs drop;
};

struct NormGradArgs {
    const void *grad_out, *sum, *grad_sum;  // grad_sum may be null
    const float *gain, *rstd;
    void *grad_x, *grad_residual;           // both may be null
    float *grad_gain;                       // may be null
    float *partial;                         // norm_grad_parts x cols, where grad_gain is wanted
    uint64_t rows, grad_out_stride, sum_stride, grad_sum_stride, grad_x_stride, grad_residual_stride;
    uint32_t cols;
    int type;
    DropArgs drop;
};

struct DropRowsArgs {
    const void *x;
    void *out;
    uint64_t rows, x_stride, out_stride;
    uint32_t cols;
    int type;
    DropArgs drop;
};

struct QuantizeArgs {
    const void *x;
    uint8_t *codes;
    uint16_t *scales;
    uint64_t rows, x_stride;
    uint32_t cols, group;
    int type;
};

struct ScoreArgs {
    const uint8_t *codes;
    const uint16_t *scales;
    const void *x;
    const float *x_scale;
    float *out;
    uint64_t rows, queries, x_stride, out_stride;
    uint32_t cols, group;
    int type;
};

struct Index {
    const void *at;
    uint64_t stride;
    int type;  // GV_I32 or GV_I64
};

struct LookupArgs {
    Index index;
    const void *table;
    void *out;
    uint64_t count, table_stride, out_stride;
    uint32_t rows, cols;  // of the table
    int type, out_type;
    float scale;
};

struct LookupGradArgs {
    Index index;
    const void *grad;
    void *out;
    uint64_t count, grad_stride, out_stride;
    uint32_t rows, cols;  // of the result
    int type, out_type;
    float scale;
    bool add;
    // of the workspace, and how the batch is cut
    uint2 *sorted;  // rows and the places that name them
    uint32_t *digit_counts, *digit_totals;
    uint8_t *flags;
    float *partial;
    uint32_t lanes, chunk, chunks;
};

// rows x outs sums over cols products of x and weight, and what becomes of them
struct DenseArgs {
    const void *x, *weight, *bias, *residual;  // bias and residual may be null
    void *pre, *out;                           // pre may be null
    uint64_t x_stride, weight_stride, residual_stride, pre_stride, out_stride;
    uint32_t rows, cols, outs;
    int type, act;
    float *partial;    // where cols are cut
    uint32_t split_k;  // and how many are taken together
};

struct DenseGradArgs {
    const void *grad, *x, *weight, *pre;         // pre may be null, without an activation
    void *grad_x, *grad_weight, *grad_bias;      // may be null
    uint64_t rows, grad_stride, x_stride, weight_stride, pre_stride, grad_x_stride, grad_weight_stride;
    uint32_t cols, outs;
    int type, act;
    void *gz;             // of the workspace
    float *bias_partial;  // likewise
    uint32_t chunk;       // rows of each of its parts
};

struct SelectArgs {
    const void *scores;
    const float *totals;   // may be null
    const uint8_t *done;   // may be null
    int64_t *parent, *row;
    float *total;
    uint64_t queries, rows, stride;
    uint32_t beams, best, end;
    int type;
    bool log_softmax;
    // of the workspace, and how scores are cut
    void *summaries, *candidates;
    uint32_t parts, part_rows, slots;
};

// Launches a kernel.  hipLaunchKernel says itself what became of it: the thread's last error may be of a call before, and is its
// caller's to ask for; that of a launch is returned here and left to nobody else.
template <class... Parameters, class... Arguments>
hipError_t launch(void (*kernel)(Parameters...), uint32_t blocks, uint32_t threads, uint32_t shared_bytes, hipStream_t stream,
                  const Arguments &...arguments) {
    static_assert((std::is_same_v<Parameters, Arguments> && ...), "a kernel is given its own parameters");
    void *at[] = {const_cast<Arguments *>(&arguments)...};
    const hipError_t e = hipLaunchKernel((const void *)kernel, dim3(blocks), dim3(threads), at, shared_bytes, stream);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
}

// how many partial sums of the gain's gradient the backward pass leaves; one goes to its place at once
uint32_t norm_grad_parts(uint64_t rows, uint32_t cols);

hipError_t launch_norm(const NormArgs &a, hipStream_t stream);
hipError_t launch_norm_grad(const NormGradArgs &a, hipStream_t stream);
hipError_t launch_drop(const DropRowsArgs &a, hipStream_t stream);
hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream);
hipError_t launch_score(const ScoreArgs &a, hipStream_t stream);
hipError_t launch_lookup(const LookupArgs &a, hipStream_t stream);
uint64_t lookup_grad_workspace(uint64_t count, uint64_t rows, uint32_t cols, bool add);
uint64_t dense_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type);
hipError_t launch_dense(const DenseArgs &a, void *workspace, hipStream_t stream);
uint64_t dense_grad_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type, int act, bool want_x, bool want_weight, bool want_bias);
hipError_t launch_dense_grad(const DenseGradArgs &a, void *workspace, hipStream_t stream);
uint64_t select_workspace(uint64_t queries, uint64_t rows, uint32_t beams, uint32_t best);
hipError_t launch_select(const SelectArgs &a, void *workspace, hipStream_t stream);
hipError_t launch_lookup_grad(const LookupGradArgs &a, void *workspace, hipStream_t stream);

}  // namespace gv
