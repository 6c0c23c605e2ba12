// gfx950 kernels of rows in device memory: dropout, and the root-mean-square norm of a sum with its gradients.
//
// All of them are bound by memory: a value is read once, stays in a register until everything that its row decides is
// known, and is written once.  A lane takes pieces of eight columns: 16 bytes of a 16-bit type, and one block of the generator
// (eight numbers of 16 bits: p is met within 2^-17; numbers of 32 bits would take two blocks, and the generator longer than
// the memory traffic of a 16-bit type).
#include "gv_device.hpp"
#include "gv_row_pieces.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#include <algorithm>
#include <type_traits>

// a product and a sum round by themselves where no fmaf is written: codes are the same bits wherever they are computed
#pragma clang fp contract(off)

namespace gv {
namespace {

// Drops values of piece k / 8 of a row; numbers 2 w and 2 w + 1 are the halves of word w.
__device__ __forceinline__ void drop_piece(const DropArgs &d, uint64_t row, uint32_t piece, float (&v)[8]) {
    const uint64_t r = d.first_row + row;
    const uint4 w = philox4x32_10<true>((uint32_t)r, (uint32_t)(r >> 32), piece, 5u, (uint32_t)d.seed, (uint32_t)(d.seed >> 32));
    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t number = i % 2 ? words[i / 2] >> 16 : words[i / 2] & 0xFFFFu;
        v[i] = number >= d.threshold ? v[i] * d.factor : 0.0f;
    }
}

// ---------------------------------------------------------------------------
// Dropout: one piece a lane and turn.  2^20 rows of 512 in bfloat16: 350 us for 2.15 GB, 6.1 TB/s (a copy reaches 4.9).  The
// vector units are busy for most of that too: 21 products of 32 x 32 bits, at a quarter of the rate, and 60 other
// instructions a piece; with an instruction for each exclusive or and for each rounding it took 385 us.
constexpr int kDropThreads = 256;

template <class T>
__global__ __launch_bounds__(kDropThreads) void k_drop(DropRowsArgs a, Walk walk) {
    walk_items(walk, [&](uint64_t row, uint32_t piece) {
        float v[8];
        load_piece((const T *)a.x + row * a.x_stride, 8 * piece, a.cols, v);
        drop_piece(a.drop, row, piece, v);
        store_piece((T *)a.out + row * a.out_stride, 8 * piece, a.cols, v);
    });
}

// ---------------------------------------------------------------------------
// Rows over lanes: kLanes lanes (up to 64, or a whole workgroup of 256 or 512) hold a row, kPieces pieces each: lane l has
// pieces l, l + kLanes, ...
constexpr int kMostLanes = 512;
constexpr int threads_of(int lanes) { return lanes > 64 ? lanes : 256; }

// Sums over the lanes of a row; all of them get the result.  A whole workgroup's: `turn` says which part of the scratch
// this row takes, 0 and 1 in turn, so that one barrier a row is enough (2: a second sum of the same row).
template <int kLanes>
__device__ __forceinline__ float row_sum(float x, float (*scratch)[kMostLanes / 64], int turn) {
    if constexpr (kLanes <= 64) return sum_lanes<kLanes>(x);
    x = sum_lanes<64>(x);
    if (threadIdx.x % 64 == 0) scratch[turn][threadIdx.x / 64] = x;
    __syncthreads();
    float all = 0.0f;
#pragma unroll
    for (int w = 0; w < kLanes / 64; ++w) all += scratch[turn][w];
    return all;
}
template <int kLanes>
__device__ __forceinline__ uint32_t row_largest(uint32_t x, uint32_t (*scratch)[kMostLanes / 64], int turn) {
    if constexpr (kLanes <= 64) return largest_of_lanes<kLanes>(x);
    x = largest_of_lanes<64>(x);
    if (threadIdx.x % 64 == 0) scratch[turn][threadIdx.x / 64] = x;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kLanes / 64; ++w) all = larger(all, scratch[turn][w]);
    return all;
}

// 1 / sqrt(x), within one unit in the last place; the instruction takes no subnormal x.  0 for 0: the norm of a row without
// values is such a row, with any eps, and its gradients pass nothing on.
__device__ __forceinline__ float inverse_root(float x) {
    const bool small = x < 0x1p-100f;
    const float root = __builtin_amdgcn_rsqf(small ? x * 0x1p64f : x) * (small ? 0x1p32f : 1.0f);
    return x == 0.0f ? 0.0f : root;
}

// The norm.  The sum of squares and the largest |h gain| of a row are joined over its lanes by register exchanges (a
// workgroup's through LDS), so a row is read once.  2^20 rows of 128 in bfloat16 with dropout, sum kept: 185 us for 1.07 GB,
// 5.8 TB/s; 8192 rows of 4096 47 us, 5.8 TB/s; 65 536 rows of 512 into 8 bits 50 us for 235 MB, 4.7 TB/s.
template <class T, int kLanes, int kPieces, bool kBytes>
__global__ __launch_bounds__(threads_of(kLanes)) void k_norm(NormArgs a) {
    constexpr int kRows = threads_of(kLanes) / kLanes;
    __shared__ float sums[3][kMostLanes / 64];
    __shared__ uint32_t tops[2][kMostLanes / 64];
    const uint32_t lane = threadIdx.x % kLanes;
    float gain[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) load_piece(a.gain, 8 * (lane + p * kLanes), a.cols, gain[p]);
    int turn = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.rows; row += (uint64_t)gridDim.x * kRows) {
        float h[kPieces][8], squares = 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) load_piece((const T *)a.x + row * a.x_stride, 8 * (lane + p * kLanes), a.cols, h[p]);
        if (a.drop.threshold != 0) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) drop_piece(a.drop, row, lane + p * kLanes, h[p]);
        }
        if (a.residual) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                float r[8];
                load_piece((const T *)a.residual + row * a.residual_stride, 8 * (lane + p * kLanes), a.cols, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[p][i] = r[i] + h[p][i];
            }
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                squares = fmaf(h[p][i], h[p][i], squares);
                if (kBytes) top = larger(top, __float_as_uint(h[p][i] * gain[p][i]) & 0x7FFFFFFFu);
            }
        squares = row_sum<kLanes>(squares, sums, turn);
        const float power = squares / (float)a.cols + a.eps;
        float rstd = inverse_root(power);
        if (!(power < __builtin_inff()) || power < 0x1p-100f) {
            // Squares that left the range of fp32 are taken again, of values times a power of two: values below 2^56, of which
            // 16384 squares are below 2^126, or values below 2^53 whose least square is normal.  A row's lanes come here together.
            const float scale = power < 0x1p-100f ? 0x1p96f : 0x1p-72f;
            squares = 0.0f;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) squares = fmaf(h[p][i] * scale, h[p][i] * scale, squares);
            squares = row_sum<kLanes>(squares, sums, 2);
            rstd = inverse_root(squares / (float)a.cols + a.eps * scale * scale) * scale;
            if (rstd == __builtin_inff()) rstd = 0.0f;
        }
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
        if (a.sum) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) store_piece((T *)a.sum + row * a.sum_stride, 8 * (lane + p * kLanes), a.cols, h[p]);
        }
        if constexpr (kBytes) {
            const float largest = __uint_as_float(row_largest<kLanes>(top, tops, turn));
            const bool finite = largest < __builtin_inff(), any = finite && largest >= 0x1p-100f;
            const float step = largest * (float)(1.0 / 127.0), up = any ? 1.0f / step : 0.0f;
            if (lane == 0) a.out_scale[row] = !finite ? __builtin_nanf("") : any ? step * rstd : 0.0f;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = any ? rintf(h[p][i] * gain[p][i] * up) : 0.0f;
                store_piece((int8_t *)a.out + row * a.out_stride, 8 * (lane + p * kLanes), a.cols, v);
            }
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = h[p][i] * rstd * gain[p][i];
                store_piece((T *)a.out + row * a.out_stride, 8 * (lane + p * kLanes), a.cols, v);
            }
        }
        turn ^= 1;
    }
}

// ---------------------------------------------------------------------------
// Gradients.  A lane adds up its columns of the gain's gradient over the rows that its workgroup takes; rows side by side in
// a wave are joined by lane exchanges, waves in LDS, workgroups by k_gain_join: an order that rows and
// cols decide.  2^20 rows of 128 in bfloat16 with both gradients: 247 us for 1.34 GB, 5.4 TB/s; 8192 rows of 4096 51 us,
// 5.3 TB/s.  The grid loops here, for the sums: four waves a SIMD is what 125 registers allow.
constexpr int grad_threads_of(int lanes) { return lanes > 64 ? lanes : 512; }
constexpr uint32_t kGradLanes = 1 << 18;  // of the whole launch at most: four waves to each of the chip's 1024 SIMDs

template <class T, int kLanes, int kPieces>
__global__ __launch_bounds__(grad_threads_of(kLanes)) void k_norm_grad(NormGradArgs a) {
    constexpr int kGradThreads = grad_threads_of(kLanes), kRows = kGradThreads / kLanes;
    __shared__ float sums[2][kMostLanes / 64];
    __shared__ float joined[kGradThreads / 64][kLanes <= 64 ? kLanes * kPieces * 8 : 1];
    const uint32_t lane = threadIdx.x % kLanes;
    float gain[kPieces][8], grad_gain[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        if (a.rows > 0) load_piece(a.gain, 8 * (lane + p * kLanes), a.cols, gain[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) grad_gain[p][i] = 0.0f;
    }
    int turn = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / kLanes; row < a.rows; row += (uint64_t)gridDim.x * kRows) {
        const float rstd = a.rstd[row];
        float n[kPieces][8], u[kPieces][8], inner = 0.0f;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            load_piece((const T *)a.sum + row * a.sum_stride, 8 * (lane + p * kLanes), a.cols, n[p]);
            load_piece((const T *)a.grad_out + row * a.grad_out_stride, 8 * (lane + p * kLanes), a.cols, u[p]);
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[p][i] *= rstd;
                grad_gain[p][i] = fmaf(u[p][i], n[p][i], grad_gain[p][i]);
                u[p][i] *= gain[p][i];
                inner = fmaf(u[p][i], n[p][i], inner);
            }
        inner = row_sum<kLanes>(inner, sums, turn) / (float)a.cols;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = rstd * (u[p][i] - n[p][i] * inner);
            if (a.grad_sum) {
                float g[8];
                load_piece((const T *)a.grad_sum + row * a.grad_sum_stride, 8 * (lane + p * kLanes), a.cols, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += g[i];
            }
            if (a.grad_residual) store_piece((T *)a.grad_residual + row * a.grad_residual_stride, 8 * (lane + p * kLanes), a.cols, v);
            if (a.grad_x) {
                if (a.drop.threshold != 0) drop_piece(a.drop, row, lane + p * kLanes, v);
                store_piece((T *)a.grad_x + row * a.grad_x_stride, 8 * (lane + p * kLanes), a.cols, v);
            }
        }
        turn ^= 1;
    }
    if (!a.grad_gain) return;
    float *to = a.partial + (uint64_t)blockIdx.x * a.cols;
    if constexpr (kLanes <= 64) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int side = kLanes; side < 64; side *= 2) grad_gain[p][i] += __shfl_xor(grad_gain[p][i], side);
        if (threadIdx.x % 64 < kLanes) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
                __builtin_memcpy(&joined[threadIdx.x / 64][(lane + p * kLanes) * 8], grad_gain[p], sizeof grad_gain[p]);
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.cols; c += kGradThreads) {
            float all = 0.0f;
#pragma unroll
            for (int w = 0; w < kGradThreads / 64; ++w) all += joined[w][c];
            to[c] = all;
        }
    } else {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) store_piece(to, 8 * (lane + p * kLanes), a.cols, grad_gain[p]);
    }
}

// 32 columns a workgroup, 32 threads to a column.  512 parts of 128 columns: 4.6 us, the latency of two rounds of loads; it is a
// launch of its own because a counter of the workgroups that are done would have to be cleared before every call.
__global__ __launch_bounds__(1024) void k_gain_join(const float *partial, float *grad_gain, uint32_t parts, uint32_t cols) {
    __shared__ float scratch[32][33];
    const uint32_t c = blockIdx.x * 32 + threadIdx.x % 32, first = threadIdx.x / 32;
    float sum = 0.0f;
    for (uint32_t p = first; p < parts && c < cols; p += 32 * 8) {
        float v[8];  // asked for together: the launch is as long as its loads wait for each other
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p + 32 * i < parts ? partial[(uint64_t)(p + 32 * i) * cols + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i];
    }
    scratch[first][threadIdx.x % 32] = sum;
    __syncthreads();
    sum = scratch[threadIdx.x % 32][first];  // column `first`, part threadIdx.x % 32
    sum = sum_lanes<32>(sum);
    if (threadIdx.x % 32 == 0 && blockIdx.x * 32 + first < cols) grad_gain[blockIdx.x * 32 + first] = sum;
}

// ---------------------------------------------------------------------------

// Lanes and pieces of a row of `cols` columns: at least eight lanes (a line of a 16-bit type) where the row has that many
// pieces, and two pieces a lane as far as that goes.  With up to four, a row takes fewer exchanges, but the gradients take 200
// registers instead of 125 and two waves a SIMD do not keep the memory busy (10^5 rows of 1024 in bfloat16, forward and
// backward: 371 us, 291 with two; 2*10^5 of 160: 141 and 116).
struct Shape {
    int lanes, pieces;
};
Shape shape_of(uint32_t cols) {
    const int pieces = (int)((cols + 7) / 8);
    const int lanes = pieces <= 1 ? 1 : pieces <= 2 ? 2 : pieces <= 4 ? 4 : pieces <= 16 ? 8 : pieces <= 32 ? 16 : pieces <= 64 ? 32
                      : pieces <= 128 ? 64 : pieces <= 256 ? 256 : kMostLanes;
    return {lanes, (pieces + lanes - 1) / lanes};
}

template <int kLanes, int kPieces, class Run>
hipError_t with_shape(Run &&run) {
    return run(std::integral_constant<int, kLanes>(), std::integral_constant<int, kPieces>());
}
template <class Run>
hipError_t by_shape(uint32_t cols, Run &&run) {
    const Shape s = shape_of(cols);
    if (s.lanes == 1) return with_shape<1, 1>(run);
    if (s.lanes == 2) return with_shape<2, 1>(run);
    if (s.lanes == 4) return with_shape<4, 1>(run);
    if (s.lanes == 8 && s.pieces == 1) return with_shape<8, 1>(run);
    if (s.lanes == 8) return with_shape<8, 2>(run);
    if (s.lanes == 16) return with_shape<16, 2>(run);
    if (s.lanes == 32) return with_shape<32, 2>(run);
    if (s.lanes == 64) return with_shape<64, 2>(run);
    if (s.lanes == 256) return with_shape<256, 1>(run);
    if (s.pieces == 1) return with_shape<kMostLanes, 1>(run);
    if (s.pieces == 2) return with_shape<kMostLanes, 2>(run);
    if (s.pieces == 3) return with_shape<kMostLanes, 3>(run);
    return with_shape<kMostLanes, 4>(run);
}

template <class Run>
hipError_t by_type(int type, Run &&run) {
    if (type == GV_F32) return run((float *)nullptr);
    if (type == GV_BF16) return run((__bf16 *)nullptr);
    return run((_Float16 *)nullptr);
}

// Workgroups of the gradients, and the rows that one takes in a turn.
struct GradGrid {
    uint64_t each;
    uint32_t blocks;
};
GradGrid grad_grid(uint64_t rows, uint32_t cols) {
    const int lanes = shape_of(cols).lanes, threads = grad_threads_of(lanes);
    const uint64_t each = threads / lanes;
    return {each, (uint32_t)std::min<uint64_t>((rows + each - 1) / each, kGradLanes / threads)};
}

}  // namespace

uint32_t norm_grad_parts(uint64_t rows, uint32_t cols) {
    const GradGrid grid = grad_grid(rows, cols);
    // A few turns of one workgroup mostly take less than a launch that joins several (200 rows of 128 through the norm and back: 21 us
    // among others, 27 with the launch, 37 alone either way; 30 rows of 1000 22 and 27, alone 42 and 38; twice as many turns
    // 31 and 27 at 128 rows of 357).
    return rows <= 4 * grid.each ? 1 : grid.blocks;
}

// Workgroups that come and go pass through memory side by side; a grid that loops drifts apart (dropout of
// 2^20 rows of 512 in bfloat16, there and back: 755 us, 901 with 4096 workgroups; 2^20 rows of 128 through the norm
// and back: 435 and 462 us).  They loop past 2^22 workgroups alone (2^30 or 2^31 threads; a launch takes up to 2^32).
constexpr uint64_t kMostBlocks = 1 << 22;

hipError_t launch_drop(const DropRowsArgs &a, hipStream_t stream) {
    const uint32_t pieces = (a.cols + 7) / 8;  // of a row
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((a.rows * pieces + kDropThreads - 1) / kDropThreads, kMostBlocks);
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return launch(k_drop<T>, blocks, kDropThreads, 0, stream, a, walk_of(a.rows, pieces, (uint64_t)blocks * kDropThreads));
    });
}

hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return by_shape(a.cols, [&](auto lanes, auto pieces) {
            constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(pieces)::value, kThreads = threads_of(kLanes);
            constexpr uint64_t kRows = kThreads / kLanes;
            const uint32_t blocks = (uint32_t)std::min<uint64_t>((a.rows + kRows - 1) / kRows, kMostBlocks);
            if (a.out_type == GV_I8) return launch(k_norm<T, kLanes, kPieces, true>, blocks, kThreads, 0, stream, a);
            return launch(k_norm<T, kLanes, kPieces, false>, blocks, kThreads, 0, stream, a);
        });
    });
}

hipError_t launch_norm_grad(const NormGradArgs &args, hipStream_t stream) {
    return by_type(args.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        NormGradArgs a = args;
        const uint32_t parts = a.grad_gain ? norm_grad_parts(a.rows, a.cols) : grad_grid(a.rows, a.cols).blocks;
        if (parts == 1) a.partial = a.grad_gain;
        const hipError_t e = by_shape(a.cols, [&](auto lanes, auto pieces) {
            constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(pieces)::value;
            return launch(k_norm_grad<T, kLanes, kPieces>, parts, grad_threads_of(kLanes), 0, stream, a);
        });
        if (e != hipSuccess || !a.grad_gain || parts == 1) return e;
        return launch(k_gain_join, (a.cols + 31) / 32, 1024, 0, stream, (const float *)a.partial, a.grad_gain, parts, a.cols);
    });
}

}  // namespace gv
