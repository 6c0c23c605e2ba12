// gfx950 kernels of a layer: out = residual + act(x weight^T + bias), and its gradients.
//
// All products are sums over k of A(m, k) B(n, k) on matrix instructions, with sums in fp32.  An operand lies with the values
// of one row together (k runs along memory: x and weight in the forward pass), or with those of one k together (the gradients'
// operands); the latter are transposed in registers on the way into LDS, so that there the tiles are all alike: rows of 128
// bytes of k, in eight pieces of 16 bytes, piece p of row r at place p ^ (r ^ r / 8) % 8.  Eight rows in a row then have a
// piece in eight different places (what a matrix instruction's lanes read), and so have rows 4 i + j for eight i in a row (what
// is written transposed).
#include "gv_row_pieces.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#pragma clang fp contract(off)

namespace gv {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// The normal distribution's Phi(z) and, on the way, exp(-z^2 / 2).
// For 16-bit types Phi(-|z|) = (a1 t + ... + a5 t^5) exp(-z^2 / 2) / 2 with t = 1 / (1 + 0.3275911 |z| / sqrt 2) (the halves are in the
// numbers below): formula 7.1.26 of Abramowitz and Stegun's Handbook, within 1.5e-7 / 2 of the true value, and 2.9e-7 with the
// roundings of these steps (4 x 10^6 values from -12 to 12); z Phi(z) is off by 3.1e-7 at most, since the factor exp(-z^2 / 2) makes the
// error small where z is large.  erff takes three times the instructions: 65536 x 512 x 2048 in bfloat16 with gelu took 520 us by it.
__device__ __forceinline__ float normal(float z, float &bell, __bf16 *) {
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(x, 0.23164190f, 1.0f));
    bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float poly = fmaf(fmaf(fmaf(fmaf(0.5307027145f, t, -0.7265760135f), t, 0.7107068705f), t, -0.142248368f), t, 0.127414796f);
    const float tail = t * poly * bell;
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float normal(float z, float &bell, _Float16 *) { return normal(z, bell, (__bf16 *)nullptr); }
// For float what that leaves would be seen: 1/2 + z q(z^2) below |z| = 1, beyond it t r(t) exp(-z^2 / 2), t = 1 / (1 + 0.3 |z|), with
// polynomials whose largest relative error is the least (7e-10 and 4.4e-9; they were fitted to erf and to exp(z^2 / 2) Phi(-z)) and an
// exponential of the exact square.  Phi is off by two units of fp32 where z >= 0 and by 12 2^-24 of itself down to where it ends
// at z = -13, so z Phi(z) is as near as its plain form in fp32 where that is near, and stays so where 1 + erf cancels.  8192 x 4096 x 4096
// floats with gelu take 2.09 ms (2.07 by the formula above), 65536 x 512 x 512 325 us (306).
__device__ __forceinline__ float normal(float z, float &bell, float *) {
    constexpr double kScale = -0.72134752044448170;  // of z^2, for a power of 2
    constexpr float kHigh = (float)kScale, kLow = (float)(kScale - (double)kHigh);
    const float x = fminf(fabsf(z), 16.0f), square = x * x, rest = fmaf(x, x, -square);
    const float power = square * kHigh, more = fmaf(rest, kHigh, fmaf(square, kLow, fmaf(square, kHigh, -power)));
    bell = __builtin_amdgcn_exp2f(power);
    bell = fmaf(bell, more * 0.69314718f, bell);
    const float t = __builtin_amdgcn_rcpf(fmaf(x, 0.3f, 1.0f));
    float r = 0.02492264285683632f;
    r = fmaf(r, t, -0.06721436232328415f);
    r = fmaf(r, t, 0.02352323941886425f);
    r = fmaf(r, t, 0.03048762120306492f);
    r = fmaf(r, t, 0.04969059303402901f);
    r = fmaf(r, t, 0.0910872220993042f);
    r = fmaf(r, t, 0.10807470977306366f);
    r = fmaf(r, t, 0.11977948248386383f);
    r = fmaf(r, t, 0.11967810243368149f);
    float q = -7.65420827519847e-06f;
    q = fmaf(q, square, 0.00011348637053743005f);
    q = fmaf(q, square, -0.0011863299878314137f);
    q = fmaf(q, square, 0.009973322972655296f);
    q = fmaf(q, square, -0.06649035960435867f);
    q = fmaf(q, square, 0.3989422917366028f);
    const float tail = r * t * bell;
    return x < 1.0f ? fmaf(z, q, 0.5f) : z < 0.0f ? tail : 1.0f - tail;
}
// act(z), and its slope, for a layer of type T
template <class T>
__device__ __forceinline__ float act_of(int act, float z) {
    if (act == GV_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (act == GV_ACT_GELU) {
        float bell;
        return z * normal(z, bell, (T *)nullptr);
    }
    if (act == GV_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return z;
}
template <class T>
__device__ __forceinline__ float slope_of(int act, float z) {
    if (act == GV_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == GV_ACT_GELU) {
        float bell;
        const float phi = normal(z, bell, (T *)nullptr);
        return fmaf(z * 0.39894228040143268f, bell, phi);
    }
    if (act == GV_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

// sums += 16 x 16 products over the k's of a piece of each lane: lane l has row l % 16 and the pieces of group l / 16.
__device__ __forceinline__ void multiply(uint4 a, uint4 b, f4 &sums, float *) {
    const float *x = (const float *)&a, *y = (const float *)&b;
#pragma unroll
    for (int i = 0; i < 4; ++i) sums = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], sums, 0, 0, 0);
}
__device__ __forceinline__ void multiply(uint4 a, uint4 b, f4 &sums, __bf16 *) {
    sums = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), sums, 0, 0, 0);
}
__device__ __forceinline__ void multiply(uint4 a, uint4 b, f4 &sums, _Float16 *) {
    sums = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), sums, 0, 0, 0);
}

// N values from p, of which those before `left` are there; the others are 0.
template <class T, int N>
struct Values {
    T at[N];
    __device__ __forceinline__ void load(const T *p, uint32_t left) {
        if (left >= (uint32_t)N) {
            __builtin_memcpy(this, p, sizeof *this);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) at[i] = (uint32_t)i < left ? p[i] : (T)0.0f;
        }
    }
    __device__ __forceinline__ void round(const float (&v)[N]) {
        if constexpr (sizeof(T) == 2) {  // two at a time: the machine rounds pairs
            typedef float f2 __attribute__((ext_vector_type(2)));
            typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const t2 pair = __builtin_convertvector((f2{v[i], v[i + 1]}), t2);
                at[i] = pair[0], at[i + 1] = pair[1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) at[i] = (T)v[i];
        }
    }
    __device__ __forceinline__ void store(T *p, uint32_t left) const {
        if (left >= (uint32_t)N) {
            __builtin_memcpy(p, this, sizeof *this);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((uint32_t)i < left) p[i] = at[i];
        }
    }
};
__device__ __forceinline__ uint32_t left_of(uint32_t at, uint32_t all) { return at < all ? all - at : 0; }

// What becomes of the N sums of row m from column n on.
template <class T, int N>
__device__ __forceinline__ void finish(const DenseArgs &a, uint32_t m, uint32_t n, uint32_t split, float (&z)[N]) {
    if (m >= a.rows || n >= a.outs) return;
    const uint32_t left = a.outs - n;
    if (a.partial) {
        Values<float, N> v = __builtin_bit_cast(decltype(v), z);
        v.store(a.partial + ((uint64_t)split * a.rows + m) * a.outs + n, left);
        return;
    }
    if (a.bias) {
        Values<T, N> b;
        b.load((const T *)a.bias + n, left);
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] += (float)b.at[i];
    }
    Values<T, N> to;
    if (a.pre) {
        to.round(z);
        to.store((T *)a.pre + m * a.pre_stride + n, left);
    }
    if (a.act != GV_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = act_of<T>(a.act, z[i]);
    }
    if (a.residual) {
        Values<T, N> r;
        r.load((const T *)a.residual + m * a.residual_stride + n, left);
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] += (float)r.at[i];
    }
    to.round(z);
    to.store((T *)a.out + m * a.out_stride + n, left);
}

// ---------------------------------------------------------------------------
// Tiles of kTile x kTile, 2 kTile threads: eight or four waves side by side.  The next step's values are loaded into registers
// while this step's are multiplied, and go to the other half of LDS.
constexpr int kStep = 128;  // bytes of k

template <class T>
constexpr int kEach = 16 / (int)sizeof(T);  // values of a piece

__device__ __forceinline__ uint32_t place_of(uint32_t row, uint32_t piece) { return row * kStep + (piece ^ ((row ^ row >> 3) & 7)) * 16; }

// A thread's share of an operand's step: four pieces.
template <class T, int kTile, bool kAlong>
struct Share {
    uint4 pieces[4];
    // rows first .. first + kTile - 1 of `rows`, from k on of `count`
    __device__ __forceinline__ void load(const T *p, uint64_t stride, uint32_t first, uint32_t rows, uint32_t k, uint32_t count) {
        constexpr int N = kEach<T>;
        if constexpr (kAlong) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t id = q * 2 * kTile + threadIdx.x, row = first + id / 8, at = k + id % 8 * N;
                Values<T, N> v;
                v.load(p + row * stride + at, row < rows ? left_of(at, count) : 0);
                pieces[q] = __builtin_bit_cast(uint4, v);
            }
        } else {
            const uint32_t row = first + 4 * (threadIdx.x % (kTile / 4)), at = k + threadIdx.x / (kTile / 4) * N;
            const uint32_t left = left_of(row, rows);
            Values<T, 4> v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i].load(p + (at + i) * stride + row, at + i < count ? left : 0);
            Values<T, N> turned;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int i = 0; i < N; ++i) turned.at[i] = v[i].at[j];
                pieces[j] = __builtin_bit_cast(uint4, turned);
            }
        }
    }
    // kAgain: its places are taken anew in every step, which is a few instructions and leaves the sums their registers.  One operand along
    // k and the other turned needs that at tiles of 256 (five were spilled: 8192 x 4095 x 4097 in bfloat16 672 us, 627 without);
    // the others are a few per cent longer by it.
    template <bool kAgain>
    __device__ __forceinline__ void put(char *tile) const {
        uint32_t thread = threadIdx.x;
        if constexpr (kAgain) asm volatile("" : "+v"(thread));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t row, piece;
            if constexpr (kAlong) {
                const uint32_t id = q * 2 * kTile + thread;
                row = id / 8, piece = id % 8;
            } else {
                row = 4 * (thread % (kTile / 4)) + q, piece = thread / (kTile / 4);
            }
            *(uint4 *)(tile + place_of(row, piece)) = pieces[q];
        }
    }
};

template <class T, int kTile, bool kAAlong, bool kBAlong>
__global__ __launch_bounds__(2 * kTile) void k_product(DenseArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    // waves: kTile / 64 x 2 of 64 x kTile / 2 (m x n)
    constexpr int kMs = 4, kNs = kTile / 32;
    constexpr bool kAgain = kAAlong != kBAlong;
    __shared__ __attribute__((aligned(16))) char tiles[2][2][kTile * kStep];
    const uint32_t all = tiles_m * tiles_n, split = blockIdx.x / all;
    uint32_t id = blockIdx.x % all;
    // neighbours share rows in an L2: workgroup b runs on die b % 8, so a die takes tiles in a row, eight rows of tiles high
    if (id < all / 8 * 8) id = id % 8 * (all / 8) + id / 8;
    const uint32_t band = id / (8 * tiles_n), high = std::min(8u, tiles_m - 8 * band), in_band = id - 8 * band * tiles_n;
    const uint32_t m0 = (8 * band + in_band % high) * kTile, n0 = in_band / high * kTile;
    const uint32_t k_first = split * a.split_k, k_last = std::min<uint64_t>(a.cols, (uint64_t)k_first + a.split_k);
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave / 2 * 64, wn = wave % 2 * (kTile / 2);
    constexpr uint32_t kCount = kStep / sizeof(T);
    f4 sums[kMs][kNs];
#pragma unroll
    for (int i = 0; i < kMs; ++i)
#pragma unroll
        for (int j = 0; j < kNs; ++j) sums[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    Share<T, kTile, kAAlong> share_a;
    Share<T, kTile, kBAlong> share_b;
    const T *pa = (const T *)a.x, *pb = (const T *)a.weight;
    if (k_first < k_last) {
        share_a.load(pa, a.x_stride, m0, a.rows, k_first, k_last);
        share_b.load(pb, a.weight_stride, n0, a.outs, k_first, k_last);
        share_a.template put<kAgain>(tiles[0][0]);
        share_b.template put<kAgain>(tiles[0][1]);
    }
    __syncthreads();
    uint32_t half = 0;
    for (uint32_t k = k_first; k < k_last; k += kCount, half ^= 1) {
        const bool more = k + kCount < k_last;
        if (more) {
            share_a.load(pa, a.x_stride, m0, a.rows, k + kCount, k_last);
            share_b.load(pb, a.weight_stride, n0, a.outs, k + kCount, k_last);
        }
        const char *ta = tiles[half][0], *tb = tiles[half][1];
#pragma unroll
        for (uint32_t p = 0; p < 8; p += 4) {
            uint4 ma[kMs], nb[kNs];
#pragma unroll
            for (int i = 0; i < kMs; ++i) ma[i] = *(const uint4 *)(ta + place_of(wm + 16 * i + lane % 16, p + lane / 16));
#pragma unroll
            for (int j = 0; j < kNs; ++j) nb[j] = *(const uint4 *)(tb + place_of(wn + 16 * j + lane % 16, p + lane / 16));
#pragma unroll
            for (int i = 0; i < kMs; ++i)
#pragma unroll
                for (int j = 0; j < kNs; ++j) multiply(nb[j], ma[i], sums[i][j], (T *)nullptr);
        }
        if (more) {
            share_a.template put<kAgain>(tiles[half ^ 1][0]);
            share_b.template put<kAgain>(tiles[half ^ 1][1]);
        }
        __syncthreads();
    }
    // a lane has four columns in a row of one row
    uint32_t thread = threadIdx.x;
    if constexpr (kAgain) asm volatile("" : "+v"(thread));
    const uint32_t m = m0 + thread / 128 * 64 + thread % 16, n = n0 + thread / 64 % 2 * (kTile / 2) + thread % 64 / 16 * 4;
#pragma unroll
    for (int i = 0; i < kMs; ++i)
#pragma unroll
        for (int j = 0; j < kNs; ++j) {
            float z[4] = {sums[i][j][0], sums[i][j][1], sums[i][j][2], sums[i][j][3]};
            finish<T>(a, m + 16 * i, n + 16 * j, split, z);
        }
}

// ---------------------------------------------------------------------------
// Small products, of any type and alignment: tiles of 32 x 64, four waves with 16 x 32 of it each, so that there are many
// workgroups, and values asked for three steps ahead, since a step's products take a quarter of what its loads take (six make
// no difference).  1021 x 357 x 500 in fp32: 10 us, where tiles of 64 x 64 and one step ahead took 25.
constexpr int kSmallM = 32, kSmallN = 64, kSmallThreads = 256, kSmallAhead = 3;

template <class T, int kRows, bool kAlong>
struct SmallShare {
    static constexpr int N = kEach<T>, kPieces = kRows * 8 / kSmallThreads;
    Values<T, N> pieces[kPieces];
    // k's k .. k + 8 N - 1, of which `left` are there (kWhole: all)
    template <bool kWhole>
    __device__ __forceinline__ void load(const T *p, uint64_t stride, uint32_t first, uint32_t rows, uint32_t k, uint32_t left) {
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            const uint32_t id = q * kSmallThreads + threadIdx.x;
            if constexpr (kAlong) {
                const uint32_t row = std::min(first + id / 8, rows - 1), at = id % 8 * N;  // rows past the end are not used
                const T *from = p + row * stride + k + at;
                if constexpr (kWhole) __builtin_memcpy(&pieces[q], from, 16);
                else pieces[q].load(from, left_of(at, left));
            } else {
                const uint32_t row = std::min(first + id % kRows, rows - 1), at = id / kRows * N;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint32_t to = kWhole ? at + i : std::min(at + i, left - 1);
                    const T v = p[(uint64_t)(k + to) * stride + row];
                    pieces[q].at[i] = kWhole || at + i < left ? v : (T)0.0f;
                }
            }
        }
    }
    __device__ __forceinline__ void put(char *tile) const {
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            const uint32_t id = q * kSmallThreads + threadIdx.x, row = kAlong ? id / 8 : id % kRows, piece = kAlong ? id % 8 : id / kRows;
            *(uint4 *)(tile + row * kStep + (piece ^ (row & 7)) * 16) = __builtin_bit_cast(uint4, pieces[q]);
        }
    }
};

template <class T, bool kAAlong, bool kBAlong>
__global__ __launch_bounds__(kSmallThreads) void k_product_small(DenseArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    constexpr uint32_t kCount = kStep / sizeof(T);
    __shared__ __attribute__((aligned(16))) char tiles[2][(kSmallM + kSmallN) * kStep];
    const uint32_t all = tiles_m * tiles_n, split = blockIdx.x / all, id = blockIdx.x % all;
    const uint32_t m0 = id / tiles_n * kSmallM, n0 = id % tiles_n * kSmallN;
    const uint32_t k_first = split * a.split_k, k_last = std::min<uint64_t>(a.cols, (uint64_t)k_first + a.split_k);
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave % 2 * 16, wn = wave / 2 * 32;
    f4 sums[2] = {};
    SmallShare<T, kSmallM, kAAlong> of_a[kSmallAhead];
    SmallShare<T, kSmallN, kBAlong> of_b[kSmallAhead];
    const T *pa = (const T *)a.x, *pb = (const T *)a.weight;
    const auto load = [&](auto stage, uint32_t k) {
        constexpr int kStage = decltype(stage)::value;
        if (k + kCount <= k_last) {
            of_a[kStage].template load<true>(pa, a.x_stride, m0, a.rows, k, kCount);
            of_b[kStage].template load<true>(pb, a.weight_stride, n0, a.outs, k, kCount);
        } else if (k < k_last) {
            of_a[kStage].template load<false>(pa, a.x_stride, m0, a.rows, k, k_last - k);
            of_b[kStage].template load<false>(pb, a.weight_stride, n0, a.outs, k, k_last - k);
        }
    };
    uint32_t half = 0;
    const auto step = [&](auto stage, uint32_t k) {
        constexpr int kStage = decltype(stage)::value;
        char *tile = tiles[half];
        of_a[kStage].put(tile);
        of_b[kStage].put(tile + kSmallM * kStep);
        load(stage, k + kSmallAhead * kCount);
        __syncthreads();  // one a step: the other half is written next, and was read before this
#pragma unroll
        for (uint32_t p = 0; p < 8; p += 4) {
            const uint32_t at = ((p + lane / 16) ^ (lane & 7)) * 16;
            const uint4 ma = *(const uint4 *)(tile + (wm + lane % 16) * kStep + at);
#pragma unroll
            for (int j = 0; j < 2; ++j)
                multiply(*(const uint4 *)(tile + (kSmallM + wn + 16 * j + lane % 16) * kStep + at), ma, sums[j], (T *)nullptr);
        }
        half ^= 1;
    };
    constexpr std::integral_constant<int, 0> kFirst;
    constexpr std::integral_constant<int, 1> kSecond;
    constexpr std::integral_constant<int, 2> kThird;
    load(kFirst, k_first);
    load(kSecond, k_first + kCount);
    load(kThird, k_first + 2 * kCount);
    for (uint32_t k = k_first; k < k_last; k += 3 * kCount) {
        step(kFirst, k);
        if (k + kCount >= k_last) break;
        step(kSecond, k + kCount);
        if (k + 2 * kCount >= k_last) break;
        step(kThird, k + 2 * kCount);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float z[4] = {sums[j][0], sums[j][1], sums[j][2], sums[j][3]};
        finish<T>(a, m0 + wm + lane % 16, n0 + wn + 16 * j + 4 * (lane / 16), split, z);
    }
}

// ---------------------------------------------------------------------------
// The same for 16-bit types whose rows are whole pieces (of 8 values, aligned): a step's 64 k's go from memory straight into
// LDS, where an operand lies as it does in memory, and what lies with the values of a k together is turned by the loads that
// transpose. A wave's values of half a step are read while those of the half before are multiplied; one barrier a step says
// that the next step has arrived and that this one's place is free for the step after that.  8192 x 4096 x 4096 in bfloat16
// with bias, gelu and residual 242 us, 1.14 PFLOP/s (229 where the same operands come again and again): the matrix units are busy for
// half of the compute units' cycles, LDS for a fifth (a wave's 128 x 64 take 24 KB of reads a step for 2^20 products), and the
// epilogue goes on beside nothing.
typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v LdsFour;
typedef __attribute__((address_space(3))) void LdsAny;

constexpr uint32_t kWide = 64;                 // k's of a step
constexpr uint64_t kWideStride = 1ull << 21;   // a tile's rows lie within 2^31 bytes

// kSpread: row 4 g + r of tile j of the matrix instruction is row 32 (j / 2) + 8 g + 4 (j % 2) + r of 64 rows, and tiles 4 to 7
// are of the next 64.  For B that leaves the lanes of group g with 8 columns of the result in a row, twice, and four of them
// write 64 bytes in a row with each store; operands that are turned are read at fewer different addresses.
template <int kTile, bool kAlong, bool kSpread>
struct Operand {
    static constexpr uint32_t kThreads = 2 * kTile, kLoads = kTile * 128 / 16 / kThreads;
    static constexpr uint32_t kLine = kAlong ? 8 : kTile / 8;  // pieces
    static constexpr uint32_t kRows = kThreads / kLine;        // that the workgroup loads at once
    const char *at, *end;  // the tile's first value of the next step, and of the matrix behind its last
    uint64_t step, rows;   // bytes to the next step, and to the next rows
    uint32_t stride;       // values
    // A piece's place: along k rows of 128 bytes, piece p of row r at p ^ turn(r); otherwise rows of kTile values of one k,
    // piece p of row k at p ^ turn(k): what lanes read together lies in different banks.
    static __device__ __forceinline__ uint32_t turn(uint32_t row) {
        if constexpr (kAlong) return kSpread ? (row & 3) | (row >> 3 & 1) << 2 : row & 7;
        else return (row & 3) << 2;
    }
    // value k (and first row) of a matrix of `lines` lines of `length` values
    __device__ __forceinline__ void begin(const void *p, uint64_t stride, uint64_t lines, uint64_t length, uint32_t first, uint32_t k) {
        at = (const char *)p + 2 * (kAlong ? first * stride + k : k * stride + first);
        end = (const char *)p + 2 * ((lines - 1) * stride + length);
        step = kAlong ? 2 * kWide : 2 * kWide * stride;
        rows = 2 * kRows * stride;
        this->stride = (uint32_t)stride;
    }
    // What a thread loads of the first rows (and of the others likewise), in bytes from there.
    __device__ __forceinline__ uint32_t from(uint32_t thread) const {
        return 2 * (thread / kLine * stride + (thread % kLine ^ turn(thread / kLine)) * 8);
    }
    // Asks for the next step.  Nothing is read behind the matrix's end; what lies behind its rows and columns is not used.
    __device__ __forceinline__ void fetch(char *tile, uint32_t wave) {
        uint32_t thread = threadIdx.x;
        asm volatile("" : "+v"(thread));  // a few instructions a step, and no register that the sums need
        const uint32_t offset = from(thread);
        const char *p = at;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j, p += rows) {
            const int64_t left = end - p;  // scalar instructions compare words
            const int high = (int)(left >> 32);
            const uint32_t bytes = high < 0 ? 0u : high > 0 ? 0xFFFFFFFFu : (uint32_t)left;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000),
                                                     (LdsAny *)(tile + j * kThreads * 16 + wave), 16, offset, 0, 0, 0);
        }
        at += step;
    }
    // a step of `left` k's, `steps` steps on, and zeros behind them
    __device__ __forceinline__ void fetch_some(char *tile, uint32_t steps, uint32_t left) const {
        const char *p = at + steps * step;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j, p += rows) {
            const uint32_t id = j * kThreads + threadIdx.x;
            const uint32_t k = kAlong ? (id % kLine ^ turn(id / kLine)) * 8 : id / kLine;
            const char *piece = p + from(threadIdx.x);  // whole: 8 k's of a row, or 8 rows of a k
            uint4 v = {};
            if (k < left && piece < end) __builtin_memcpy(&v, piece, 16);
            *(uint4 *)(tile + id * 16) = v;
        }
    }
};

// How a lane reads eight k's (piece 4 half + its group of a step) of tile i of the wave's rows, for the matrix instruction.
template <int kTile, bool kAlong, bool kSpread>
struct Reader {
    uint32_t base;  // in a step, for half 0 and tile 0
    __device__ __forceinline__ void begin(uint32_t row) {
        using Of = Operand<kTile, kAlong, kSpread>;
        const uint32_t lane = threadIdx.x % 64, group = lane / 16, at = lane % 16;
        if constexpr (kAlong) {
            row += kSpread ? at / 4 * 8 + at % 4 : at;
            base = row * 128 + (group ^ Of::turn(row)) * 16;
        } else {
            // lanes point to four rows of one k each, and get four k's of one row
            const uint32_t k = 8 * group + at / 4;
            base = k * (2 * kTile) + ((row / 8 + at % 4) ^ Of::turn(k)) * 16;
        }
    }
    __device__ __forceinline__ uint4 read(const char *tile, int half, int i) const {
        if constexpr (kAlong) {
            // turn() is the same for all tiles' rows
            return *(const uint4 *)(tile + (base ^ 64 * half) + (kSpread ? 512 * (i % 2) + 4096 * (i / 2) : 2048 * i));
        } else {
            static_assert(kSpread, "what is turned is spread");
            const char *at = tile + (base ^ (64 * (i % 4 / 2) + 128 * (i / 4))) + 8 * (i % 2) + half * (32 * 2 * kTile);
            const s4v low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour *)at);
            const s4v high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour *)(at + 8 * kTile));
            const uint2 x = __builtin_bit_cast(uint2, low), y = __builtin_bit_cast(uint2, high);
            return uint4{x.x, x.y, y.x, y.y};
        }
    }
};

template <class T, int kTile, bool kAAlong, bool kBAlong>
__global__ __launch_bounds__(2 * kTile, 2) void k_product_wide(DenseArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    // waves: 2 x kTile / 64, of kTile / 2 x 64
    constexpr int kMs = kTile / 32, kNs = 4;
    constexpr uint32_t kBytes = kTile * 128;
    // of one step and of the next; they are apart so that the compiler sees that what is read is not what is being fetched
    __shared__ __attribute__((aligned(16))) char a0[kBytes], a1[kBytes], b0[kBytes], b1[kBytes];
    const uint32_t all = tiles_m * tiles_n, split = blockIdx.x / all;
    uint32_t id = blockIdx.x % all;
    if (id < all / 8 * 8) id = id % 8 * (all / 8) + id / 8;
    const uint32_t band = id / (8 * tiles_n), high = std::min(8u, tiles_m - 8 * band), in_band = id - 8 * band * tiles_n;
    const uint32_t m0 = (8 * band + in_band % high) * kTile, n0 = in_band / high * kTile;
    const uint32_t k_first = split * a.split_k, k_last = std::min<uint64_t>(a.cols, (uint64_t)k_first + a.split_k);
    const uint32_t wave = threadIdx.x / 64, wm = wave % 2 * (kTile / 2), wn = wave / 2 * 64;
    f4 sums[kMs][kNs];
#pragma unroll
    for (int i = 0; i < kMs; ++i)
#pragma unroll
        for (int j = 0; j < kNs; ++j) sums[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    Operand<kTile, kAAlong, !kAAlong> of_a;
    Operand<kTile, kBAlong, true> of_b;
    of_a.begin(a.x, a.x_stride, kAAlong ? a.rows : a.cols, kAAlong ? a.cols : a.rows, m0, k_first);
    of_b.begin(a.weight, a.weight_stride, kBAlong ? a.outs : a.cols, kBAlong ? a.cols : a.outs, n0, k_first);
    // Steps go in pairs.  What is left of k behind the whole steps goes first, and a step of zeros makes the number even.
    uint32_t whole = (k_last - k_first) / kWide;
    const uint32_t left = (k_last - k_first) % kWide, odd = (whole + (left ? 1 : 0)) % 2;
    const uint32_t wave_at = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 1024;  // in LDS, of what a wave loads
    const auto fetch = [&](char *ta, char *tb) {
        if (whole == 0) return;
        of_a.fetch(ta, wave_at);
        of_b.fetch(tb, wave_at);
        --whole;
    };
    const auto arrived = [] {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    Reader<kTile, kAAlong, !kAAlong> read_a;
    Reader<kTile, kBAlong, true> read_b;
    read_a.begin(wm);
    read_b.begin(wn);
    uint4 ma[kMs], nb[2][kNs];
    // the products of half a step; the values of the next half, of these tiles, replace those that are done with
    const auto products = [&](auto now, const char *ta, const char *tb) {
        constexpr int kHalf = decltype(now)::value, kNext = kHalf ^ 1;
#pragma unroll
        for (int j = 0; j < kNs; ++j) nb[kNext][j] = read_b.read(tb, kNext, j);
#pragma unroll
        for (int i = 0; i < kMs; ++i) {
#pragma unroll
            for (int j = 0; j < kNs; ++j) multiply(nb[kHalf][j], ma[i], sums[i][j], (T *)nullptr);
            ma[i] = read_a.read(ta, kNext, i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr std::integral_constant<int, 0> kFirst;
    constexpr std::integral_constant<int, 1> kSecond;
    const uint32_t pairs = (whole + (left ? 1 : 0) + odd) / 2;
    if (left || odd) {
        of_a.fetch_some(a0, whole, left);
        of_b.fetch_some(b0, whole, left);
    } else {
        fetch(a0, b0);
    }
    if (left && odd) {
        of_a.fetch_some(a1, 0, 0);
        of_b.fetch_some(b1, 0, 0);
        arrived();
    } else {
        arrived();
        fetch(a1, b1);
    }
#pragma unroll
    for (int i = 0; i < kMs; ++i) ma[i] = read_a.read(a0, 0, i);
#pragma unroll
    for (int j = 0; j < kNs; ++j) nb[0][j] = read_b.read(b0, 0, j);
    for (uint32_t pair = 0; pair < pairs; ++pair) {
        products(kFirst, a0, b0);
        arrived();
        fetch(a0, b0);
        products(kSecond, a1, b1);
        products(kFirst, a1, b1);
        arrived();
        fetch(a1, b1);
        products(kSecond, a0, b0);
    }
    // What the results' places are made of is taken again here: kept through the steps, it took registers that they need.
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const uint32_t end_lane = thread % 64, end_wave = __builtin_amdgcn_readfirstlane(thread / 64);
    const uint32_t end_m = m0 + end_wave % 2 * (kTile / 2), end_n = n0 + end_wave / 2 * 64;
    // a lane has twice 8 columns in a row of each of its rows
    const auto row_of = [&](int i) {
        return end_m + (kAAlong ? 16 * i + end_lane % 16 : 64 * (i / 4) + 32 * (i % 4 / 2) + end_lane % 16 / 4 * 8 + 4 * (i % 2) + end_lane % 4);
    };
    const auto column_of = [&](int h) { return end_n + 32 * h + 8 * (end_lane / 16); };
    // A whole tile without a check: bias is read once, and the residual's values are asked for a row ahead (what is written may
    // be they, so the compiler leaves each load behind the stores before it).  A value that is read under a condition of its
    // own is waited for on the way past it, and with it all stores before: 65536 x 512 x 2048 took 290 us instead of 200.
    const auto whole_tile = [&](auto with) {
        constexpr bool kResidual = decltype(with)::value;
        float bias[2][8];
        Values<T, 8> residual[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Values<T, 8> b = {};
            if (a.bias) b.load((const T *)a.bias + column_of(h), 8);
#pragma unroll
            for (int c = 0; c < 8; ++c) bias[h][c] = (float)b.at[c];
        }
        const auto ask = [&](int i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) residual[i % 2][h].load((const T *)a.residual + row_of(i) * a.residual_stride + column_of(h), 8);
        };
        if constexpr (kResidual) ask(0);
#pragma unroll
        for (int i = 0; i < kMs; ++i) {
            if (kResidual && i + 1 < kMs) ask(i + 1);
            float z[2][8];
            Values<T, 8> to[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 8; ++c) z[h][c] = sums[i][2 * h + c / 4][c % 4] + bias[h][c];
            if (a.pre) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    to[h].round(z[h]);
                    to[h].store((T *)a.pre + row_of(i) * a.pre_stride + column_of(h), 8);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (a.act != GV_ACT_NONE) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) z[h][c] = act_of<T>(a.act, z[h][c]);
                }
                if constexpr (kResidual) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) z[h][c] += (float)residual[i % 2][h].at[c];
                }
                to[h].round(z[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) to[h].store((T *)a.out + row_of(i) * a.out_stride + column_of(h), 8);
        }
    };
    if (!a.partial && m0 + kTile <= a.rows && n0 + kTile <= a.outs) {
        if (a.residual) whole_tile(std::true_type());
        else whole_tile(std::false_type());
        return;
    }
#pragma unroll
    for (int i = 0; i < kMs; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float z[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) z[c] = sums[i][2 * h + c / 4][c % 4];
            finish<T>(a, row_of(i), column_of(h), split, z);
        }
}

// The sums of the parts that a product's k was cut into, in their order.
template <class T>
__global__ __launch_bounds__(256) void k_join_product(DenseArgs a, uint32_t splits) {
    const uint32_t each = (a.outs + 3) / 4;
    const uint64_t all = (uint64_t)a.rows * each, step = (uint64_t)gridDim.x * 256;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const uint32_t m = (uint32_t)(i / each), n = (uint32_t)(i % each) * 4;
        f4 sums = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t s = 0; s < splits; ++s) {
            Values<float, 4> v;
            v.load(a.partial + ((uint64_t)s * a.rows + m) * a.outs + n, a.outs - n);
            sums += __builtin_bit_cast(f4, v);
        }
        float z[4] = {sums[0], sums[1], sums[2], sums[3]};
        DenseArgs whole = a;
        whole.partial = nullptr;
        finish<T>(whole, m, n, 0, z);
    }
}

// ---------------------------------------------------------------------------
// Few rows of x: every value of the weight is read once, from memory straight into the matrix instruction's registers.  A
// workgroup takes 16 columns of the result, its waves take lines of k (256 bytes of each row) in turn and are joined through
// LDS.  What is bound by memory is so by what is asked for at once: whole lines are loaded without a check, eight pieces a lane
// ahead.  16 x 4096 x 4096 in bfloat16: 11 us, 3.1 TB/s; with four pieces of 64 bytes each, checked, 16 us.
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64;

template <class T, int kMs>
__global__ __launch_bounds__(kFewThreads) void k_product_few(DenseArgs a) {
    constexpr int N = kEach<T>, kLine = 4, kAhead = kMs == 1 ? 8 : 4;
    constexpr uint32_t kStride = kFewWaves * kLine * 4 * N;  // k's from a wave's line to its next
    __shared__ f4 joined[kFewWaves][kMs][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = blockIdx.x * 16 + lane % 16;
    // rows past the ends are not used
    const T *weight = (const T *)a.weight + std::min(n, a.outs - 1) * a.weight_stride + lane / 16 * N;
    const T *x[kMs];
#pragma unroll
    for (int i = 0; i < kMs; ++i) x[i] = (const T *)a.x + std::min(16 * i + lane % 16, a.rows - 1) * a.x_stride + lane / 16 * N;
    f4 sums[kMs] = {};
    const auto take = [&](auto whole, uint32_t first, auto number) {
        constexpr int kNumber = decltype(number)::value;
        Values<T, N> w[kNumber], v[kNumber][kMs];
#pragma unroll
        for (int u = 0; u < kNumber; ++u) {
            const uint32_t k = first + u / kLine * kStride + u % kLine * 4 * N;
            const uint32_t left = decltype(whole)::value ? N : left_of(k + lane / 16 * N, a.cols);
            w[u].load(weight + k, left);
#pragma unroll
            for (int i = 0; i < kMs; ++i) v[u][i].load(x[i] + k, left);
        }
#pragma unroll
        for (int u = 0; u < kNumber; ++u)
#pragma unroll
            for (int i = 0; i < kMs; ++i) multiply(__builtin_bit_cast(uint4, w[u]), __builtin_bit_cast(uint4, v[u][i]), sums[i], (T *)nullptr);
    };
    uint32_t k = wave * (kLine * 4 * N);
    for (; k + (kAhead / kLine - 1) * kStride + kLine * 4 * N <= a.cols; k += kAhead / kLine * kStride)
        take(std::true_type(), k, std::integral_constant<int, kAhead>());
    for (; k + kLine * 4 * N <= a.cols; k += kStride) take(std::true_type(), k, std::integral_constant<int, kLine>());
    if (k < a.cols) take(std::false_type(), k, std::integral_constant<int, kLine>());
#pragma unroll
    for (int i = 0; i < kMs; ++i) joined[wave][i][lane] = sums[i];
    __syncthreads();
    if (wave >= (uint32_t)kMs) return;
    f4 all = joined[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) all += joined[w][wave][lane];
    float z[4] = {all[0], all[1], all[2], all[3]};
    finish<T>(a, 16 * wave + lane % 16, blockIdx.x * 16 + 4 * (lane / 16), 0, z);
}

// ---------------------------------------------------------------------------
// gz = grad * slope(pre), and the sums over its rows: a lane has eight columns, a wave 512, the waves of a workgroup take rows
// in turn. 65536 x 2048 in bfloat16 with gelu: 190 us for 810 MB, 4.2 TB/s, the vector units busy for half of it; the bias'
// gradient alone 126 us for 537.
constexpr int kSlopeThreads = 256, kSlopeWaves = kSlopeThreads / 64;

// Rows of eight columns and more (kWide) have no broken piece: the last one lies back so far that it is whole, and two lanes
// have the columns that it shares with the one before, and the same of them.  A part has 512 columns, or 504 where the last
// would have fewer than eight.
__host__ __device__ __forceinline__ uint32_t part_of(uint32_t cols) { return cols > 512 && cols % 512 > 0 && cols % 512 < 8 ? 504 : 512; }

template <class T, bool kWide>
__global__ __launch_bounds__(kSlopeThreads) void k_slope(DenseGradArgs a) {
    __shared__ float joined[kSlopeWaves][512];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, width = part_of(a.outs), parts = (a.outs + width - 1) / width;
    const uint32_t part = blockIdx.x % parts, chunk = blockIdx.x / parts;
    const bool used = 8 * lane < width && width * part + 8 * lane < a.outs;
    const uint32_t k = kWide ? std::min(width * part + 8 * lane, a.outs - 8) : width * part + 8 * lane, cols = kWide ? k + 8 : a.outs;
    const uint64_t first = (uint64_t)chunk * a.chunk, last = std::min<uint64_t>(a.rows, first + a.chunk);
    constexpr int kAhead = 2;  // rows of a wave asked for at once (four: the bias' gradient of 65536 x 2048 121 us, of 200000 x 96 88 instead of 81)
    float sums[8] = {};
    if (used) {
        for (uint64_t row = first + wave; row < last; row += kAhead * kSlopeWaves) {
            Piece<T> g[kAhead], z[kAhead];
#pragma unroll
            for (int h = 0; h < kAhead; ++h) {
                const uint64_t at = row + h * kSlopeWaves;
                if (at >= last) continue;
                g[h].load((const T *)a.grad + at * a.grad_stride, k, cols);
                if (a.act != GV_ACT_NONE) z[h].load((const T *)a.pre + at * a.pre_stride, k, cols);
            }
#pragma unroll
            for (int h = 0; h < kAhead; ++h) {
                const uint64_t at = row + h * kSlopeWaves;
                if (at >= last) continue;
                float v[8];
                g[h].values(v);
                if (a.act != GV_ACT_NONE) {
                    float of[8];
                    z[h].values(of);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= slope_of<T>(a.act, of[i]);
                    if (a.gz) store_piece((T *)a.gz + at * a.outs, k, cols, v);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[i] += v[i];
            }
        }
    }
    if (!a.bias_partial) return;
    if (used) __builtin_memcpy(&joined[wave][k - width * part], sums, sizeof sums);
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < width && width * part + c < a.outs; c += kSlopeThreads) {
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < kSlopeWaves; ++w) all += joined[w][c];
        a.bias_partial[(uint64_t)chunk * a.outs + width * part + c] = all;
    }
}

// 32 columns a workgroup, 32 threads to a column.
template <class T>
__global__ __launch_bounds__(1024) void k_join_bias(DenseGradArgs a, uint32_t chunks) {
    __shared__ float scratch[32][33];
    const uint32_t c = blockIdx.x * 32 + threadIdx.x % 32, first = threadIdx.x / 32;
    float sum = 0.0f;
    for (uint32_t p = first; p < chunks && c < a.outs; p += 32) sum += a.bias_partial[(uint64_t)p * a.outs + c];
    scratch[first][threadIdx.x % 32] = sum;
    __syncthreads();
    sum = sum_lanes<32>(scratch[threadIdx.x % 32][first]);
    if (threadIdx.x % 32 == 0 && blockIdx.x * 32 + first < a.outs) ((T *)a.grad_bias)[blockIdx.x * 32 + first] = (T)sum;
}

// ---------------------------------------------------------------------------

template <class Run>
hipError_t by_type(int type, Run &&run) {
    if (type == GV_F32) return run((float *)nullptr);
    if (type == GV_BF16) return run((__bf16 *)nullptr);
    return run((_Float16 *)nullptr);
}

// How a product of rows x outs over `cols` k's is cut: the way that is the shortest by what steps were measured to take.
// Larger tiles ask for fewer values (8192 x 4096 x 4096 in bfloat16: 214 us by tiles of 256, 244 by 128, 607 by the small ones; 65536 x
// 512 x 2048 156, 181 and 364; with bias, gelu and pre 230, 263 and 523), smaller ones are more workgroups (1021 x 357 x 500 floats:
// 65, 26 and 10 us; 1000 x 1000 x 1000 in bfloat16 29, 15, which is taken, and 10), and a long k is cut where there are few (a
// weight's gradient of 65536 x 128 x 512: 49 us in 64 parts of tiles of 128, 92 in 8; 103 and 180 by the small ones).
struct Cut {
    uint32_t tile, tiles_m, tiles_n, splits, split_k;
};

Cut cut_of(uint64_t rows, uint64_t cols, uint64_t outs, int type, bool wide) {
    const uint64_t step = kStep / (type == GV_F32 ? 4 : 2), steps = std::max<uint64_t>(1, (cols + step - 1) / step);
    // tiles, workgroups that run at once, and what a step of theirs takes then, in microseconds
    struct Way {
        uint32_t m, n;
        double at_once, each;
    };
    const bool f32 = type == GV_F32;
    const Way ways[3] = {{256, 256, 256, f32 ? 7.5 : wide ? 2.1 : 5.0},
                         {128, 128, 512, f32 ? 4.0 : wide ? 1.2 : 2.6},
                         {kSmallM, kSmallN, 1024, f32 ? 1.0 : 0.8}};
    Cut best{};
    double least = 1e300;
    for (const Way &w : ways) {
        const uint64_t m = (rows + w.m - 1) / w.m, n = (outs + w.n - 1) / w.n;
        for (uint64_t splits = 1; splits <= 64 && (splits == 1 || steps >= 4 * splits); splits *= 2) {
            const uint64_t each = (steps + splits - 1) / splits, cut = (steps + each - 1) / each;
            const double rounds = (double)(m * n * cut) / w.at_once, alone = 0.3 + 0.7 * std::min(1.0, rounds);
            const double join = cut > 1 ? 4.0 + (double)(cut * rows * outs) * 2e-6 : 0.0;
            const double time = std::ceil(rounds) * ((double)each * w.each * alone + 3.0) + join;
            if (time < least) {
                least = time;
                best = {w.m, (uint32_t)m, (uint32_t)n, (uint32_t)cut, (uint32_t)(each * step)};
            }
        }
    }
    return best;
}
uint64_t partial_of(const Cut &c, uint64_t rows, uint64_t outs) { return c.splits > 1 ? 4ull * c.splits * rows * outs : 0; }

// of any alignment
uint64_t most_partial_of(uint64_t rows, uint64_t cols, uint64_t outs, int type) {
    uint64_t most = 0;
    for (int i = 0; i < 2; ++i) most = std::max(most, partial_of(cut_of(rows, cols, outs, type, i), rows, outs));
    return most;
}

// Whether a layer goes by k_product_few: up to 16 rows, and up to 64 where a workgroup has little of x to read for its 16 columns.  us by
// it and by tiles, of 4096 x 4096 in bfloat16: 16 rows 10 and 12, 24 rows 12.5 and 12.3, 32 rows 13.4 and 12.7, 64 rows 20.5 and 14;
// 2048 x 2048: 32 rows 8.2 and 12.2, 64 rows 11.4 and 12.3; 32 x 4096 x 16384 45 and 28; in fp32 of 4096 x 4096 24 rows 22 and 26, 64 rows 39
// and 32; 64 x 1024 x 4096 12.6 and 14.5, 64 x 2048 x 2048 21 and 16.  Rows that do not begin at whole pieces (`whole`) of 16-bit types 64 x
// 4095 x 4097 118 and 24, of floats 40 and 28 at 32 rows.
bool few_rows(uint64_t rows, uint32_t cols, uint32_t outs, int type, bool whole) {
    if (rows <= 16) return true;
    if (rows > 64 || outs > 4096 || (type != GV_F32 && !whole)) return false;
    return cols <= (rows > 32 ? (type == GV_F32 ? 1024u : 2048u) : whole ? 4096u : 2048u);
}

template <class T, bool kAAlong, bool kBAlong>
hipError_t product(DenseArgs a, void *workspace, hipStream_t stream) {
    if (a.rows == 0 || a.outs == 0) return hipSuccess;
    const auto whole = [](const void *p, uint64_t stride, uint64_t together) {
        return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && together % 8 == 0 && together > 0 && stride < kWideStride;
    };
    const bool wide = sizeof(T) == 2 && whole(a.x, a.x_stride, kAAlong ? a.cols : a.rows) &&
                      whole(a.weight, a.weight_stride, kBAlong ? a.cols : a.outs);
    const Cut c = cut_of(a.rows, a.cols, a.outs, a.type, wide);
    const uint32_t threads = c.tile == 256 ? 512 : 256;  // of all three ways
    static_assert(kSmallThreads == 256, "as many as of a tile of 128");
    const uint64_t blocks = (uint64_t)c.tiles_m * c.tiles_n * c.splits;
    if (kAAlong && blocks * threads > 0xFFFFFFFFull) {  // more than a launch takes: two halves; k is never cut where tiles are so many
        const uint32_t first = a.rows / 2;
        DenseArgs rest = a;
        const auto behind = [&](auto *&p, uint64_t stride) {
            if (p) p = (T *)p + first * stride;
        };
        behind(rest.x, a.x_stride), behind(rest.residual, a.residual_stride), behind(rest.pre, a.pre_stride), behind(rest.out, a.out_stride);
        rest.rows -= first, a.rows = first;
        const hipError_t e = product<T, kAAlong, kBAlong>(a, workspace, stream);
        return e != hipSuccess ? e : product<T, kAAlong, kBAlong>(rest, workspace, stream);
    }
    a.split_k = c.split_k;
    a.partial = c.splits > 1 ? (float *)workspace : nullptr;
    const auto run = [&](auto kernel) { return launch(kernel, (uint32_t)blocks, threads, 0, stream, a, c.tiles_m, c.tiles_n); };
    hipError_t e = hipSuccess;
    if (c.tile == kSmallM) {
        e = run(k_product_small<T, kAAlong, kBAlong>);
    } else if (!wide) {
        e = c.tile == 256 ? run(k_product<T, 256, kAAlong, kBAlong>) : run(k_product<T, 128, kAAlong, kBAlong>);
    } else if constexpr (sizeof(T) == 2) {
        e = c.tile == 256 ? run(k_product_wide<T, 256, kAAlong, kBAlong>) : run(k_product_wide<T, 128, kAAlong, kBAlong>);
    }
    if (e != hipSuccess || c.splits == 1) return e;
    const uint64_t pieces = (uint64_t)a.rows * ((a.outs + 3) / 4);
    return launch(k_join_product<T>, (uint32_t)std::min<uint64_t>((pieces + 255) / 256, 1 << 16), 256, 0, stream, a, c.splits);
}

// The parts of the gradients' workspace, in bytes.
struct GradPlan {
    uint64_t gz, bias, product, bytes;
    uint32_t chunk, chunks;
};
GradPlan grad_plan_of(uint64_t rows, uint32_t cols, uint32_t outs, int type, int act, bool want_x, bool want_weight, bool want_bias) {
    GradPlan p{};
    const uint64_t parts = (outs + 511) / 512, most = std::max<uint64_t>(1, 2048 / parts);
    p.chunk = (uint32_t)std::max<uint64_t>(4 * kSlopeWaves, (rows + most - 1) / most);
    p.chunks = (uint32_t)((rows + p.chunk - 1) / p.chunk);
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 15) & ~15ull;
        return here;
    };
    p.gz = take(act != GV_ACT_NONE && (want_x || want_weight) ? rows * outs * (type == GV_F32 ? 4 : 2) : 0);
    p.bias = take(want_bias ? 4ull * p.chunks * outs : 0);
    p.product = take(std::max(want_x ? most_partial_of(rows, outs, cols, type) : 0,
                              want_weight ? most_partial_of(outs, rows, cols, type) : 0));
    p.bytes = at;
    return p;
}

}  // namespace

uint64_t dense_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type) {
    return few_rows(rows, cols, outs, type, false) ? 0 : most_partial_of(rows, cols, outs, type);
}

hipError_t launch_dense(const DenseArgs &a, void *workspace, hipStream_t stream) {
    return by_type(a.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const auto whole = [](const void *p, uint64_t stride) { return ((uintptr_t)p | stride * sizeof(T)) % 16 == 0; };
        if (!few_rows(a.rows, a.cols, a.outs, a.type, whole(a.x, a.x_stride) && whole(a.weight, a.weight_stride)))
            return product<T, true, true>(a, workspace, stream);
        const uint32_t blocks = (a.outs + 15) / 16;
        if (a.rows <= 16) return launch(k_product_few<T, 1>, blocks, kFewThreads, 0, stream, a);
        if (a.rows <= 32) return launch(k_product_few<T, 2>, blocks, kFewThreads, 0, stream, a);
        return launch(k_product_few<T, 4>, blocks, kFewThreads, 0, stream, a);
    });
}

uint64_t dense_grad_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type, int act, bool want_x, bool want_weight, bool want_bias) {
    return grad_plan_of(rows, cols, outs, type, act, want_x, want_weight, want_bias).bytes;
}

hipError_t launch_dense_grad(const DenseGradArgs &args, void *workspace, hipStream_t stream) {
    return by_type(args.type, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        DenseGradArgs a = args;
        const bool products = a.grad_x || a.grad_weight;
        const GradPlan p = grad_plan_of(a.rows, a.cols, a.outs, a.type, a.act, a.grad_x, a.grad_weight, a.grad_bias);
        a.chunk = p.chunk;
        a.gz = a.act != GV_ACT_NONE && products ? (char *)workspace + p.gz : nullptr;
        a.bias_partial = a.grad_bias ? (float *)((char *)workspace + p.bias) : nullptr;
        void *space = (char *)workspace + p.product;
        hipError_t e = hipSuccess;
        const uint32_t slope_blocks = p.chunks * ((a.outs + part_of(a.outs) - 1) / part_of(a.outs));
        if ((a.gz || a.grad_bias) && a.rows > 0)
            e = launch(a.outs >= 8 ? k_slope<T, true> : k_slope<T, false>, slope_blocks, kSlopeThreads, 0, stream, a);
        if (e == hipSuccess && a.grad_bias) e = launch(k_join_bias<T>, (a.outs + 31) / 32, 1024, 0, stream, a, p.chunks);
        const void *gz = a.gz ? a.gz : a.grad;
        const uint64_t gz_stride = a.gz ? a.outs : a.grad_stride;
        if (e == hipSuccess && a.grad_x) {
            DenseArgs d{};
            d.x = gz, d.weight = a.weight, d.out = a.grad_x, d.x_stride = gz_stride, d.weight_stride = a.weight_stride;
            d.out_stride = a.grad_x_stride, d.rows = (uint32_t)a.rows, d.cols = a.outs, d.outs = a.cols, d.type = a.type;
            e = product<T, true, false>(d, space, stream);
        }
        if (e == hipSuccess && a.grad_weight) {
            DenseArgs d{};
            d.x = gz, d.weight = a.x, d.out = a.grad_weight, d.x_stride = gz_stride, d.weight_stride = a.x_stride;
            d.out_stride = a.grad_weight_stride, d.rows = a.outs, d.cols = (uint32_t)a.rows, d.outs = a.cols, d.type = a.type;
            e = product<T, false, false>(d, space, stream);
        }
        return e;
    });
}

}  // namespace gv
