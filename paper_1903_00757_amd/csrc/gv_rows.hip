// gfx950 kernels of rows in device memory: dropout, and the root-mean-square norm of a sum with its gradients.
#include "gv_device.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

// each operation rounds by itself: the 8-bit codes of a row are the same bits wherever they are computed
#pragma clang fp contract(off)

namespace gv {
namespace {

constexpr int kThreads = 256;

template <class T>
__device__ __forceinline__ float value(const T *at) {
    return (float)*at;
}

// the factor on value (row, col): 0 where it is dropped
__device__ __forceinline__ bool kept(const DropArgs &d, uint64_t row, uint32_t col) {
    const uint64_t r = d.first_row + row;
    const uint4 w = philox4x32_10((uint32_t)r, (uint32_t)(r >> 32), col / 8, 5u, (uint32_t)d.seed, (uint32_t)(d.seed >> 32));
    const uint32_t word = col % 8 < 2 ? w.x : col % 8 < 4 ? w.y : col % 8 < 6 ? w.z : w.w;
    return (col % 2 ? word >> 16 : word & 0xFFFFu) >= d.threshold;
}

__device__ __forceinline__ float dropped(const DropArgs &d, uint64_t row, uint32_t col, float x) {
    return d.threshold == 0 ? x : kept(d, row, col) ? x * d.factor : 0.0f;
}

template <class F>
__device__ __forceinline__ float over_block(float x, float *scratch, F &&join) {
    scratch[threadIdx.x] = x;
    __syncthreads();
    for (int step = kThreads / 2; step > 0; step /= 2) {
        if ((int)threadIdx.x < step) scratch[threadIdx.x] = join(scratch[threadIdx.x], scratch[threadIdx.x + step]);
        __syncthreads();
    }
    const float all = scratch[0];
    __syncthreads();
    return all;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_drop(DropRowsArgs a) {
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x)
        for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads)
            ((T *)a.out)[row * a.out_stride + c] = (T)dropped(a.drop, row, c, (float)((const T *)a.x)[row * a.x_stride + c]);
}

// One workgroup to a row at a time; the row waits in LDS.
template <class T, bool kBytes>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
    __shared__ float h[GV_MAX_ROW_COLS];
    __shared__ float scratch[kThreads];
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float squares = 0.0f, largest = 0.0f, strange = 0.0f;
        for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) {
            float v = dropped(a.drop, row, c, (float)((const T *)a.x)[row * a.x_stride + c]);
            if (a.residual) v = (float)((const T *)a.residual)[row * a.residual_stride + c] + v;
            h[c] = v;
            squares += v * v;
            const float w = fabsf(v * a.gain[c]);
            if (w < __builtin_inff()) largest = fmaxf(largest, w); else strange = 1.0f;
        }
        squares = over_block(squares, scratch, [](float p, float q) { return p + q; });
        const float rstd = 1.0f / sqrtf(squares / (float)a.cols + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        float step = 0.0f, up = 0.0f;
        if (kBytes) {
            largest = over_block(largest, scratch, [](float p, float q) { return fmaxf(p, q); });
            strange = over_block(strange, scratch, [](float p, float q) { return fmaxf(p, q); });
            if (strange == 0.0f && largest >= 0x1p-100f) {
                step = largest * (float)(1.0 / 127.0);
                up = 1.0f / step;
            }
            if (threadIdx.x == 0) a.out_scale[row] = strange != 0.0f ? __builtin_nanf("") : up == 0.0f ? 0.0f : step * rstd;
        }
        for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) {
            if (a.sum) ((T *)a.sum)[row * a.sum_stride + c] = (T)h[c];
            if (kBytes)
                ((int8_t *)a.out)[row * a.out_stride + c] = up == 0.0f ? 0 : (int8_t)(int)rintf(h[c] * a.gain[c] * up);
            else
                ((T *)a.out)[row * a.out_stride + c] = (T)(h[c] * rstd * a.gain[c]);
        }
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_grad(NormGradArgs a) {
    __shared__ float scratch[kThreads];
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        float inner = 0.0f;
        for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float n = (float)((const T *)a.sum)[row * a.sum_stride + c] * rstd;
            inner += (float)((const T *)a.grad_out)[row * a.grad_out_stride + c] * a.gain[c] * n;
        }
        inner = over_block(inner, scratch, [](float p, float q) { return p + q; }) / (float)a.cols;
        for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float n = (float)((const T *)a.sum)[row * a.sum_stride + c] * rstd;
            const float u = (float)((const T *)a.grad_out)[row * a.grad_out_stride + c] * a.gain[c];
            float dh = rstd * (u - n * inner);
            if (a.grad_sum) dh += (float)((const T *)a.grad_sum)[row * a.grad_sum_stride + c];
            if (a.grad_residual) ((T *)a.grad_residual)[row * a.grad_residual_stride + c] = (T)dh;
            if (a.grad_x) ((T *)a.grad_x)[row * a.grad_x_stride + c] = (T)dropped(a.drop, row, c, dh);
        }
    }
}

// Part p of the gain's gradient: its share of the rows, one thread to a column.
template <class T>
__global__ __launch_bounds__(kThreads) void k_gain_parts(NormGradArgs a, uint32_t parts) {
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.cols) return;
    const uint64_t each = (a.rows + parts - 1) / parts, lo = blockIdx.y * each;
    const uint64_t hi = lo + each < a.rows ? lo + each : a.rows;
    float sum = 0.0f;
    for (uint64_t row = lo; row < hi; ++row)
        sum += (float)((const T *)a.grad_out)[row * a.grad_out_stride + c] * ((float)((const T *)a.sum)[row * a.sum_stride + c] * a.rstd[row]);
    a.partial[(uint64_t)blockIdx.y * a.cols + c] = sum;
}

__global__ __launch_bounds__(kThreads) void k_gain_join(const float *partial, float *grad_gain, uint32_t parts, uint32_t cols) {
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float sum = 0.0f;
    for (uint32_t p = 0; p < parts; ++p) sum += partial[(uint64_t)p * cols + c];
    grad_gain[c] = sum;
}

uint32_t blocks_for(uint64_t rows) { return (uint32_t)(rows < (1u << 16) ? rows : 1u << 16); }

template <class Run>
hipError_t by_type(int type, Run &&run) {
    if (type == GV_F32) run((float *)nullptr);
    else if (type == GV_BF16) run((__bf16 *)nullptr);
    else run((_Float16 *)nullptr);
    return hipGetLastError();
}

}  // namespace

uint32_t norm_grad_parts(uint64_t rows, uint32_t) { return (uint32_t)(rows < 1024 ? rows : 1024); }

hipError_t launch_drop(const DropRowsArgs &a, hipStream_t stream) {
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        k_drop<T><<<blocks_for(a.rows), kThreads, 0, stream>>>(a);
    });
}

hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (a.out_type == GV_I8) k_norm<T, true><<<blocks_for(a.rows), kThreads, 0, stream>>>(a);
        else k_norm<T, false><<<blocks_for(a.rows), kThreads, 0, stream>>>(a);
    });
}

hipError_t launch_norm_grad(const NormGradArgs &a, hipStream_t stream) {
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const uint32_t parts = norm_grad_parts(a.rows, a.cols), across = (a.cols + kThreads - 1) / kThreads;
        if (a.grad_gain) {  // first: grad_x may take the place of grad_out
            if (parts) k_gain_parts<T><<<dim3(across, parts), kThreads, 0, stream>>>(a, parts);
            k_gain_join<<<across, kThreads, 0, stream>>>(a.partial, a.grad_gain, parts, a.cols);
        }
        if (a.rows && (a.grad_x || a.grad_residual)) k_norm_grad<T><<<blocks_for(a.rows), kThreads, 0, stream>>>(a);
    });
}

}  // namespace gv
