// gfx950 kernels of tables of rows in 4 bits: making one, and the scores of queries against all of its rows.
#include "gv_device.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#pragma clang fp contract(off)

namespace gv {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float scale_of(uint16_t bits) { return __uint_as_float((uint32_t)bits << 16); }

// One thread to a group.
template <class T>
__global__ __launch_bounds__(kThreads) void k_quantize(QuantizeArgs a) {
    const uint32_t groups = (a.cols + a.group - 1) / a.group;
    const uint64_t pitch = 16ull * ((a.cols + 31) / 32), all = a.rows * groups;
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (uint64_t)gridDim.x * kThreads) {
        const uint64_t row = i / groups;
        const uint32_t g = (uint32_t)(i % groups), first = g * a.group;
        const uint32_t last = first + a.group < a.cols ? first + a.group : a.cols;
        const T *x = (const T *)a.x + row * a.x_stride;
        float largest = 0.0f;
        bool strange = false;
        for (uint32_t c = first; c < last; ++c) {
            const float w = fabsf((float)x[c]);
            if (w < __builtin_inff()) largest = fmaxf(largest, w); else strange = true;
        }
        const __bf16 scale = strange ? (__bf16)__builtin_nanf("") : (__bf16)(largest < 0x1p-100f ? 0.0f : largest * (float)(1.0 / 7.0));
        const float up = strange || largest < 0x1p-100f ? 0.0f : 1.0f / (float)scale;
        a.scales[i] = __builtin_bit_cast(uint16_t, scale);
        const uint32_t end = first + a.group < 2 * (uint32_t)pitch ? first + a.group : 2 * (uint32_t)pitch;
        for (uint32_t c = first; c < end; c += 2) {
            uint32_t byte = 0;
            for (uint32_t k = 0; k < 2; ++k) {
                const float w = up == 0.0f || c + k >= last ? 0.0f : (float)x[c + k] * up;
                byte |= ((uint32_t)(int)rintf(fminf(fmaxf(w, -7.0f), 7.0f)) & 15u) << (4 * k);
            }
            a.codes[row * pitch + c / 2] = (uint8_t)byte;
        }
    }
}

// Queries one after the other: the workgroup makes whole numbers of the query, then a thread takes a row of the table.
template <class T>
__global__ __launch_bounds__(kThreads) void k_score(ScoreArgs a) {
    __shared__ int whole[GV_MAX_ROW_COLS];
    __shared__ uint32_t top;
    const uint32_t groups = (a.cols + a.group - 1) / a.group;
    const uint64_t pitch = 16ull * ((a.cols + 31) / 32);
    for (uint64_t b = blockIdx.y; b < a.queries; b += gridDim.y) {
        const T *x = (const T *)a.x + b * a.x_stride;
        float unit = 1.0f;
        if (threadIdx.x == 0) top = 0;
        __syncthreads();
        if (sizeof(T) > 1) {
            for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) atomicMax(&top, __float_as_uint((float)x[c]) & 0x7FFFFFFFu);
            __syncthreads();
            // the largest |x| is below 2^(exponent - 126); the units are normal floats
            const int exponent = top >> 23 > 31 ? (int)(top >> 23) : 31;
            unit = exponent == 255 ? __builtin_nanf("") : ldexpf(1.0f, exponent - 126 - 30);
            for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads)
                whole[c] = exponent == 255 ? 0 : (int)rintf(ldexpf((float)x[c], 30 + 126 - exponent));
        } else {
            for (uint32_t c = threadIdx.x; c < a.cols; c += kThreads) whole[c] = (int)(float)x[c];
            unit = a.x_scale[b];
        }
        __syncthreads();
        for (uint64_t row = (uint64_t)blockIdx.x * kThreads + threadIdx.x; row < a.rows; row += (uint64_t)gridDim.x * kThreads) {
            float score = 0.0f;
            for (uint32_t g = 0; g < groups; ++g) {
                const uint32_t first = g * a.group, last = first + a.group < a.cols ? first + a.group : a.cols;
                int64_t sum = 0;
                for (uint32_t c = first; c < last; ++c) {
                    const int code = (int)((uint32_t)a.codes[row * pitch + c / 2] << (c % 2 ? 24 : 28)) >> 28;
                    sum += (int64_t)code * whole[c];
                }
                score += scale_of(a.scales[row * groups + g]) * (float)sum;
            }
            a.out[b * a.out_stride + row] = score * unit;
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream) {
    const uint64_t all = a.rows * ((a.cols + a.group - 1) / a.group), blocks = (all + kThreads - 1) / kThreads;
    const uint32_t grid = (uint32_t)(blocks < (1u << 16) ? blocks : 1u << 16);
    if (a.type == GV_F32) k_quantize<float><<<grid, kThreads, 0, stream>>>(a);
    else if (a.type == GV_BF16) k_quantize<__bf16><<<grid, kThreads, 0, stream>>>(a);
    else k_quantize<_Float16><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_score(const ScoreArgs &a, hipStream_t stream) {
    const uint64_t blocks = (a.rows + kThreads - 1) / kThreads;
    const dim3 grid((uint32_t)(blocks < 4096 ? blocks : 4096), (uint32_t)(a.queries < 64 ? a.queries : 64));
    if (a.type == GV_F32) k_score<float><<<grid, kThreads, 0, stream>>>(a);
    else if (a.type == GV_BF16) k_score<__bf16><<<grid, kThreads, 0, stream>>>(a);
    else if (a.type == GV_F16) k_score<_Float16><<<grid, kThreads, 0, stream>>>(a);
    else k_score<int8_t><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace gv
