// Internal interface between the checks of the operators on rows (gv_rows_api.cpp) and their kernels
// (gv_rows.hip, gv_scores.hip).  Not part of the C boundary.
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

}  // namespace gv
