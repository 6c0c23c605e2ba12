// Device functions of the kernels on rows (gv_rows.hip, gv_scores.hip, gv_lookup.hip, gv_dense.hip, gv_select.hip): pieces of eight
// columns, and what the lanes of a row share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gv {
namespace {

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_word(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xF, 0xF, false);
}

// Joins the values of kLanes lanes (a power of two, aligned); all of them get the result.
template <int kLanes, class Join>
__device__ __forceinline__ uint32_t join_lanes(uint32_t x, Join &&join) {
    if constexpr (kLanes >= 2) x = join(x, dpp_word<0xB1>(x));    // quad_perm [1,0,3,2]
    if constexpr (kLanes >= 4) x = join(x, dpp_word<0x4E>(x));    // quad_perm [2,3,0,1]
    if constexpr (kLanes >= 8) x = join(x, dpp_word<0x141>(x));   // row_half_mirror
    if constexpr (kLanes >= 16) x = join(x, dpp_word<0x140>(x));  // row_mirror
    if constexpr (kLanes >= 32) x = join(x, (uint32_t)__shfl_xor((int)x, 16));
    if constexpr (kLanes >= 64) x = join(x, (uint32_t)__shfl_xor((int)x, 32));
    return x;
}
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x) {
    return __uint_as_float(join_lanes<kLanes>(__float_as_uint(x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
template <int kLanes>
__device__ __forceinline__ uint32_t largest_of_lanes(uint32_t x) {
    return join_lanes<kLanes>(x, larger);
}

// Calls take(row, item) for the items of this thread (see Walk), of a workgroup that is `block` in the walk.
template <class Walk, class Take>
__device__ __forceinline__ void walk_items(const Walk &w, Take &&take, uint32_t block = blockIdx.x) {
    uint64_t i = (uint64_t)block * blockDim.x + threadIdx.x, row;
    uint32_t item;
    if (w.all >> 32 == 0) {
        row = (uint32_t)i / w.each;
        item = (uint32_t)i % w.each;
    } else {
        row = i / w.each;
        item = (uint32_t)(i % w.each);
    }
    for (; i < w.all; i += w.stride) {
        take(row, item);
        row += w.rows_on;
        item += w.items_on;
        if (item >= w.each) item -= w.each, ++row;
    }
}

// Columns k .. k + 7 of a row as they lie there, 0 past its end: one load or two of 16 bytes wherever the row starts, for
// a whole piece.  Several are asked for before the first is used.
template <class T>
struct Piece {
    T at[8];
    __device__ __forceinline__ void load(const T *row, uint32_t k, uint32_t cols) {
        if (k + 8 <= cols) {
            __builtin_memcpy(this, row + k, sizeof *this);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) at[i] = k + i < cols ? row[k + i] : (T)0.0f;
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)at[i];
    }
};
template <class T>
__device__ __forceinline__ void load_piece(const T *row, uint32_t k, uint32_t cols, float (&v)[8]) {
    Piece<T> p;
    p.load(row, k, cols);
    p.values(v);
}

// The same columns of a result: each is rounded once.
template <class T>
__device__ __forceinline__ void store_piece(T *row, uint32_t k, uint32_t cols, const float (&v)[8]) {
    Piece<T> p;
    if constexpr (sizeof(T) == 2) {  // two at a time: the machine rounds pairs
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const t2 pair = __builtin_convertvector((f2{v[i], v[i + 1]}), t2);
            p.at[i] = pair[0], p.at[i + 1] = pair[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p.at[i] = (T)v[i];
    }
    if (k + 8 <= cols) {
        __builtin_memcpy(row + k, &p, sizeof p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols) row[k + i] = p.at[i];
    }
}

}  // namespace
}  // namespace gv
