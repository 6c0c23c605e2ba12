// gfx950 kernels of tables of rows in 4 bits: making one, and the scores of queries against all of its rows.
//
// A score is sum_g scale_g sum_{c in g} code_c x_c.  The inner sums are taken in whole numbers: x is a 32-bit whole number
// times a power of two (of its query), split into four signed digits of 8 bits, and the codes are the high halves of
// bytes (16 code, which costs a mask and a shift for eight of them and no sign extension); products of bytes are what the
// dot-product and matrix instructions of this machine take, exactly.  A query is read and split once by every workgroup
// and then stays, in registers or in LDS, while rows of the table pass by.
#include "gv_row_pieces.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#include <algorithm>
#include <type_traits>

// a product and a sum round by themselves where no fmaf is written: codes are the same bits wherever they are computed
#pragma clang fp contract(off)

namespace gv {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr uint32_t kSlot = 32;  // columns to 16 bytes of codes

typedef int i4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float scale_of(uint16_t bits) { return __uint_as_float((uint32_t)bits << 16); }

__device__ __forceinline__ void load_piece_of(int type, const void *x, uint64_t at, uint32_t k, uint32_t cols, float (&v)[8]) {
    if (type == GV_F32) load_piece((const float *)x + at, k, cols, v);
    else if (type == GV_BF16) load_piece((const __bf16 *)x + at, k, cols, v);
    else load_piece((const _Float16 *)x + at, k, cols, v);
}

// a value that all lanes have, in a scalar register
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

__device__ __forceinline__ float value_of(int type, const void *x, uint64_t at) {
    return type == GV_F32 ? ((const float *)x)[at] : type == GV_BF16 ? (float)((const __bf16 *)x)[at] : (float)((const _Float16 *)x)[at];
}

// Whole numbers of a query whose largest |x| has these bits: x = number * 2^(exponent - 156), |number| <= 2^30.
struct Whole {
    int exponent;
    __device__ __forceinline__ explicit Whole(uint32_t top) : exponent((int)larger(top >> 23, 34u)) {}  // units are normal floats
    // 0 where the query is not finite: its unit is NaN
    __device__ __forceinline__ float factor() const { return exponent == 255 ? 0.0f : __uint_as_float((uint32_t)(283 - exponent) << 23); }
    static __device__ __forceinline__ int number(float x, float factor) { return factor == 0.0f ? 0 : __float2int_rn(x * factor); }
    // of a sum of 16 code * number
    __device__ __forceinline__ float unit() const { return power(exponent); }
    // The same in two steps: times a sum, up to 2^44, the first stays inside fp32.
    static constexpr int kRest = 238;
    __device__ __forceinline__ float first_unit() const { return power(std::min(exponent, kRest)); }
    __device__ __forceinline__ float rest() const { return __uint_as_float((uint32_t)(127 + std::max(exponent, kRest) - kRest) << 23); }
    __device__ __forceinline__ float power(int e) const {
        return exponent == 255 ? __builtin_nanf("") : __uint_as_float((uint32_t)(e - 33) << 23);
    }
};
// The two steps of an 8-bit query, whose sums are of 16 code * x: the power of two in its scale, and the rest of that.
struct Bytes {
    float scale;
    int exponent;  // 2^-100 to 2^100: a sum, up to 2^21, times the first and the rest of a subnormal scale are normal floats
    __device__ __forceinline__ explicit Bytes(uint32_t bits)
        : scale(__uint_as_float(bits)), exponent(std::min(std::max((int)(bits >> 23 & 255u), 27), 227)) {}
    // of a sum; NaN where it is subnormal and may be rounded, so that the scores are made again
    __device__ __forceinline__ float unit() const {
        const float all = scale * 0.0625f;
        return scale != 0.0f && fabsf(all) < 0x1p-126f ? __builtin_nanf("") : all;
    }
    __device__ __forceinline__ float first_unit() const { return __uint_as_float((uint32_t)(exponent - 4) << 23); }
    __device__ __forceinline__ float rest() const { return scale * __uint_as_float((uint32_t)(254 - exponent) << 23); }
};

// The digits of eight columns in the order of the codes' halves: digits[p][0] has digit p of columns 0, 2, 4, 6, [1] of 1, 3, 5, 7.
__device__ __forceinline__ void split(const float (&v)[8], float factor, uint32_t (&digits)[4][2]) {
    uint32_t z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)  // number = sum_p digit_p 256^p with digits -128..127
        z[i] = factor == 0.0f ? 0u : ((uint32_t)Whole::number(v[i], factor) + 0x00808080u) ^ 0x00808080u;
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
        const uint32_t a = z[odd], b = z[2 + odd], c = z[4 + odd], d = z[6 + odd];
        const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u), ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u);
        const uint32_t cd = __builtin_amdgcn_perm(d, c, 0x05010400u), cd2 = __builtin_amdgcn_perm(d, c, 0x07030602u);
        digits[0][odd] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
        digits[1][odd] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
        digits[2][odd] = __builtin_amdgcn_perm(cd2, ab2, 0x05040100u);
        digits[3][odd] = __builtin_amdgcn_perm(cd2, ab2, 0x07060302u);
    }
}
// Eight columns of an 8-bit row, in the same order.
__device__ __forceinline__ void split_bytes(const int8_t *row, uint32_t k, uint32_t cols, uint32_t (&digits)[2]) {
    uint32_t w[2] = {0, 0};
    if (k + 8 <= cols) {
        __builtin_memcpy(w, row + k, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < cols) w[i / 4] |= (uint32_t)(uint8_t)row[k + i] << (8 * (i % 4));
    }
    digits[0] = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u);
    digits[1] = __builtin_amdgcn_perm(w[1], w[0], 0x07050301u);
}

// The codes of a word as bytes of 16 code: the low halves (columns 0, 2, 4, 6), the high halves (1, 3, 5, 7).
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return (w << 4) & 0xF0F0F0F0u; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0xF0F0F0F0u; }

__device__ __forceinline__ long half_of(i4 x, int j) { return (long)(((uint64_t)(uint32_t)x[2 * j + 1] << 32) | (uint32_t)x[2 * j]); }

// sum_p s[p] 256^p; |s[p]| <= 2^21
__device__ __forceinline__ float join_digits(int s0, int s1, int s2, int s3) {
    return fmaf((float)((s3 << 8) + s2), 65536.0f, (float)((s1 << 8) + s0));
}

// With many queries, a row's groups are joined before the query's unit goes onto them: sums that may leave the range of fp32 where
// the score does not (scales beyond 2^75 with small queries, or parts that cancel).  What is joined then is inf or NaN to the
// end, never a wrong number: so the kernels look at what they write, and a score that is not finite is made again here
// by the lane that wrote it, from sums that have their unit and are as large as the score's parts.  The unit on every sum from
// the start took 83 us instead of 77 (16 8-bit queries x 10^6 rows of 512) and 196 instead of 188 (64 bfloat16 queries).
// `bits`: of the largest |x| of the query, or of the scale of an 8-bit one.
template <bool kFloat>
__device__ __forceinline__ void score_again(const ScoreArgs &a, uint64_t row, uint64_t query, uint32_t bits) {
    float *out = a.out + query * a.out_stride + row;
    if (fabsf(*out) < __builtin_inff() || (bits & 0x7FFFFFFFu) >= 0x7F800000u) return;
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot, groups = (a.cols + a.group - 1) / a.group;
    const uint8_t *codes = a.codes + row * slots * 16;
    const uint16_t *scales = a.scales + row * groups;
#pragma nounroll
    for (uint32_t g = 0; g < groups; ++g)
        if ((scales[g] & 0x7FFFu) >= 0x7F80u) return;  // nor is the row
    const std::conditional_t<kFloat, Whole, Bytes> units(bits);
    float score = 0.0f;
#pragma nounroll
    for (uint32_t g = 0; g < groups; ++g) {
        int64_t sum = 0;
#pragma nounroll
        for (uint32_t c = g * a.group; c < std::min((g + 1) * a.group, a.cols); ++c) {
            const uint64_t at = query * a.x_stride + c;
            int number;
            if constexpr (kFloat) number = Whole::number(value_of(a.type, a.x, at), units.factor());
            else number = ((const int8_t *)a.x)[at];
            sum += (int64_t)((int)((uint32_t)codes[c / 2] << (c % 2 ? 24 : 28)) >> 28) * number;
        }
        score = fmaf((float)(16 * sum) * units.first_unit(), scale_of(scales[g]), score);
    }
    *out = score * units.rest();
}

// ---------------------------------------------------------------------------
// Few queries: kLanes lanes to a row of the table, each with 16 bytes of it (32 columns) and the digits of those columns
// in registers; kColumns digit columns (one query of four digits, or 1, 2 or 4 queries in 8 bits).  A wave has kUnroll loads of 64
// consecutive pieces in flight.  Rows longer than 2048 columns (kLong): the digits stay in LDS, a lane goes along the row.
// Bound by memory: a query in floats takes 1.9 vector instructions a code (of eight codes: three to make bytes of them, eight
// dot products, the rest to join sums), counted 6 us of the 16.2 that one query x 10^6 rows of 128 takes (4.7 TB/s); rows of
// 512 65 us (4.5 TB/s), in 8 bits 53 us (5.5).
template <bool kFloat, int kColumns, int kLanes, int kUnroll, bool kLong>
__global__ __launch_bounds__(kThreads) void k_score_few(ScoreArgs a) {
    constexpr int kQueries = kFloat ? 1 : kColumns, kRows = 64 / kLanes;
    extern __shared__ uint4 shared_digits[];  // [digit column][half][slot]
    const int lane = threadIdx.x % 64, h = lane % kLanes, sub = lane / kLanes;
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot, groups = (a.cols + a.group - 1) / a.group;
    const uint32_t shift = a.group == 32 ? 0 : a.group == 64 ? 1 : 2;
    const bool mine = (uint32_t)h < slots;

    // The queries are split once by the workgroup: eight columns a thread, word p % 4 of slot p / 4.
    auto keep = [&](int column, uint32_t p, uint32_t even, uint32_t odd) {
        ((uint2 *)shared_digits)[((column * 2 + p % 4 / 2) * (uint64_t)slots + p / 4) * 2 + p % 2] = make_uint2(even, odd);
    };
    float unit[kQueries], rest[kQueries];
    if constexpr (kFloat) {
        __shared__ uint32_t tops[kWaves];
        uint32_t top = 0;
        float v[8];
        for (uint32_t p = threadIdx.x; p < 4 * slots; p += kThreads) {
            load_piece_of(a.type, a.x, 0, 8 * p, a.cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = larger(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        top = largest_of_lanes<64>(top);
        if (lane == 0) tops[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = larger(top, tops[w]);
        const Whole whole(top);
        unit[0] = uniform(whole.first_unit()), rest[0] = uniform(whole.rest());
        for (uint32_t p = threadIdx.x; p < 4 * slots; p += kThreads) {
            uint32_t d[4][2];
            if constexpr (kLong) load_piece_of(a.type, a.x, 0, 8 * p, a.cols, v);  // otherwise it is the one piece of above
            split(v, whole.factor(), d);
#pragma unroll
            for (int c = 0; c < 4; ++c) keep(c, p, d[c][0], d[c][1]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < kQueries; ++q) {
            const bool there = (uint64_t)q < a.queries;
            const int8_t *x = (const int8_t *)a.x + (there ? q : 0) * a.x_stride;
            const Bytes of(there ? __float_as_uint(a.x_scale[q]) : 0u);
            unit[q] = uniform(of.first_unit()), rest[q] = uniform(of.rest());
            for (uint32_t p = threadIdx.x; p < 4 * slots; p += kThreads) {
                uint32_t d[2];
                split_bytes(x, 8 * p, there ? a.cols : 0, d);
                keep(q, p, d[0], d[1]);
            }
        }
    }
    __syncthreads();
    auto digits_of = [&](uint32_t slot, uint32_t (&d)[kColumns][8]) {
#pragma unroll
        for (int c = 0; c < kColumns; ++c) {
            const uint4 lo = shared_digits[(c * 2) * (uint64_t)slots + slot], hi = shared_digits[(c * 2 + 1) * (uint64_t)slots + slot];
            d[c][0] = lo.x, d[c][1] = lo.y, d[c][2] = lo.z, d[c][3] = lo.w;
            d[c][4] = hi.x, d[c][5] = hi.y, d[c][6] = hi.z, d[c][7] = hi.w;
        }
    };
    uint32_t d[kColumns][8];
    if constexpr (!kLong) digits_of(mine ? h : 0, d);

    const uint64_t tiles = (a.rows + kRows * kUnroll - 1) / (kRows * kUnroll);
    for (uint64_t tile = (uint64_t)blockIdx.x * kWaves + threadIdx.x / 64; tile < tiles; tile += (uint64_t)gridDim.x * kWaves) {
        const uint64_t first = tile * (kRows * kUnroll) + sub;
        float score[kUnroll][kQueries];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int q = 0; q < kQueries; ++q) score[u][q] = 0.0f;
        for (uint32_t slot = h; kLong ? slot < slots : slot == (uint32_t)h; slot += kLanes) {
            uint4 codes[kUnroll];
            float scale[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const uint64_t row = first + u * kRows;
                const bool there = row < a.rows && (kLong || mine);
                codes[u] = there ? ((const uint4 *)a.codes)[row * slots + slot] : make_uint4(0, 0, 0, 0);
                scale[u] = there ? scale_of(a.scales[row * groups + (slot >> shift)]) : 0.0f;
            }
            if constexpr (kLong) digits_of(slot, d);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const uint32_t word[4] = {codes[u].x, codes[u].y, codes[u].z, codes[u].w};
                int sums[kColumns] = {};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int lo = (int)low_codes(word[j]), hi = (int)high_codes(word[j]);
#pragma unroll
                    for (int c = 0; c < kColumns; ++c) {
                        sums[c] = __builtin_amdgcn_sdot4(lo, (int)d[c][2 * j], sums[c], false);
                        sums[c] = __builtin_amdgcn_sdot4(hi, (int)d[c][2 * j + 1], sums[c], false);
                    }
                }
                if constexpr (kFloat) {
                    score[u][0] = fmaf(join_digits(sums[0], sums[1], sums[2], sums[3]) * unit[0], scale[u], score[u][0]);
                } else {
#pragma unroll
                    for (int q = 0; q < kQueries; ++q) score[u][q] = fmaf((float)sums[q] * unit[q], scale[u], score[u][q]);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kQueries; ++q) {
            if (!kFloat && (uint64_t)q >= a.queries) break;
            float *out = a.out + q * a.out_stride;
            if constexpr (kLanes >= kUnroll) {  // lane u of a row's lanes writes row u: neighbours in memory, one store
                float all = 0.0f;
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const float s = sum_lanes<kLanes>(score[u][q]) * rest[q];
                    all = h == u ? s : all;
                }
                const uint64_t row = first + h * kRows;
                if (h < kUnroll && row < a.rows) out[row] = all;
            } else {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const float s = sum_lanes<kLanes>(score[u][q]) * rest[q];
                    const uint64_t row = first + u * kRows;
                    if (h == u % kLanes && row < a.rows) out[row] = s;
                }
            }
        }
    }
}

// A workgroup's work on the kQueries queries of its pass.  A thread keeps to one query and one word of eight columns and goes
// along the slots, four at a time.
template <int kQueries, int kThreads>
struct Queries {
    static constexpr uint32_t kStep = kThreads / (4 * kQueries);  // slots that the workgroup takes at a time
    static_assert(kStep >= 1, "a slot of every query fits a workgroup");
    const ScoreArgs &a;
    const uint64_t first;
    const uint32_t count, word, q, slot;
    __device__ __forceinline__ Queries(const ScoreArgs &args, uint64_t first_query, uint32_t queries, uint32_t thread)
        : a(args), first(first_query), count(queries), word(thread % 4), q(thread / 4 % kQueries), slot(thread / (4 * kQueries)) {}
    __device__ __forceinline__ uint32_t cols() const { return q < count ? a.cols : 0; }
    template <class T>
    __device__ __forceinline__ const T *row() const {
        return (const T *)a.x + (first + (q < count ? q : 0)) * a.x_stride;
    }
    // the bits of the largest |x| of every query
    template <class T>
    __device__ __forceinline__ void tops_of(uint32_t slots, uint32_t *tops) const {
        uint32_t top = 0;
        for (uint32_t s = slot; s < slots; s += 4 * kStep) {
            Piece<T> p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i].load(row<T>(), kSlot * (s + i * kStep) + 8 * word, cols());
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[8];
                p[i].values(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) top = larger(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
            }
        }
        top = largest_of_lanes<4>(top);
        if (word == 0) atomicMax(tops + q, top);
    }
    __device__ __forceinline__ void tops(uint32_t slots, uint32_t *to) const {
        if (threadIdx.x < kQueries) to[threadIdx.x] = 0;
        __syncthreads();
        if (a.type == GV_F32) tops_of<float>(slots, to);
        else if (a.type == GV_BF16) tops_of<__bf16>(slots, to);
        else tops_of<_Float16>(slots, to);
        __syncthreads();
    }
    // the digits of slots begin .. end - 1: uint2 [pair of slots][tile][lane][slot of the pair]
    template <class T>
    __device__ __forceinline__ void split_of(uint32_t begin, uint32_t end, float factor, uint2 *digits) const {
        constexpr uint32_t kTiles = kQueries / 4;
        for (uint32_t s = slot; s < end - begin; s += 4 * kStep) {
            Piece<T> p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i].load(row<T>(), kSlot * (begin + s + i * kStep) + 8 * word, cols());
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = s + i * kStep;
                float v[8];
                uint32_t d[4][2];
                p[i].values(v);
                split(v, factor, d);
                if (at < end - begin) {
                    uint2 *to = digits + 2 * ((at / 2 * kTiles + q / 4) * 64 + 16 * word + 4 * (q % 4)) + at % 2;
#pragma unroll
                    for (int c = 0; c < 4; ++c) to[2 * c] = make_uint2(d[c][0], d[c][1]);
                }
            }
        }
    }
    __device__ __forceinline__ void split_floats(uint32_t begin, uint32_t end, float factor, uint2 *digits) const {
        if (a.type == GV_F32) split_of<float>(begin, end, factor, digits);
        else if (a.type == GV_BF16) split_of<__bf16>(begin, end, factor, digits);
        else split_of<_Float16>(begin, end, factor, digits);
    }
    __device__ __forceinline__ void split_8_bits(uint32_t begin, uint32_t end, uint2 *digits) const {
        constexpr uint32_t kTiles = kQueries / 16;
        for (uint32_t s = slot; s < end - begin; s += 4 * kStep) {
            uint32_t d[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) split_bytes(row<int8_t>(), kSlot * (begin + s + i * kStep) + 8 * word, cols(), d[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = s + i * kStep;
                if (at < end - begin) digits[2 * ((at / 2 * kTiles + q / 16) * 64 + 16 * word + q % 16) + at % 2] = make_uint2(d[i][0], d[i][1]);
            }
        }
    }
};

// Words j of lanes r, r + 16, r + 32, r + 48 transposed: word j of lane r + 16 h becomes word h of lane r + 16 j.
__device__ __forceinline__ void transpose(const uint4 &codes, uint32_t (&word)[4]) {
    const auto p = __builtin_amdgcn_permlane32_swap(codes.x, codes.z, false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(codes.y, codes.w, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
    word[0] = lo[0], word[1] = lo[1], word[2] = hi[0], word[3] = hi[1];
}
// the codes of two words, as the matrix instruction takes them
__device__ __forceinline__ i4 code_bytes(uint32_t u, uint32_t v) {
    return i4{(int)low_codes(u), (int)high_codes(u), (int)low_codes(v), (int)high_codes(v)};
}

// What lane r + 16 h of a pass wrote for a row, see score_again.
template <bool kFloat>
__device__ __forceinline__ void scores_again(const ScoreArgs &a, uint64_t row, uint64_t first_query, uint32_t queries, uint32_t h,
                                             const uint32_t *tops) {
#pragma nounroll
    for (uint32_t q = 0; row < a.rows && q < queries; ++q)
        if ((kFloat ? q : q / 4) % 4 == h)
            score_again<kFloat>(a, row, first_query + q, kFloat ? tops[q] : __float_as_uint(a.x_scale[first_query + q]));
}

constexpr int many_threads(int tiles) { return tiles == 8 ? 512 : 256; }  // 64 KB of digits serve twice the waves

// ---------------------------------------------------------------------------
// Many queries: the matrix instruction multiplies 16 digit columns by 16 rows of the table over 32 columns of theirs.  A
// wave loads 16 rows x 128 columns with 16 bytes a lane (lane r + 16 h: slot h of row r), four such tiles at a time; the
// 4 x 4 words that lanes r, r + 16, r + 32, r + 48 hold are transposed by four lane swaps, so that word j is slot j
// everywhere, as the instruction wants it.  The digits of kTiles x 16 columns lie in LDS in the order of the lanes.  The digit
// columns are the rows of the product: its lane r + 16 h then holds four digits of one query (or four queries in 8 bits) for
// row r alone, whose scale is one value, and the digits join without another lane.
// With few tiles bound by memory: 16 queries in 8 bits x 4*10^6 rows of 128 in 116 us, 288 MB read and 256 written, 4.7 TB/s.
// With many by vector instructions, for unpacking codes and joining sums: 64 bfloat16 queries (16 tiles, two passes) x 10^6
// rows of 512 in 190 us, 2.7 TB/s and 1.4*10^15 operations/s on digits; the SIMDs spend 56 % of their cycles on vector and 31 % on matrix
// instructions, LDS is busy for 33 % of its own.
template <bool kFloat, int kTiles, int kPer, int kRowTiles>
__global__ __launch_bounds__(many_threads(kTiles), 4) void k_score_many(ScoreArgs a, uint32_t segment, uint32_t passes) {
    constexpr int kQueries = kFloat ? 4 : 16;  // of a tile
    constexpr int kOut = kFloat ? 1 : 4;       // queries of a tile that a lane holds
    constexpr int kThreads = many_threads(kTiles), kWaves = kThreads / 64, kBlockRows = kWaves * kRowTiles * 16;
    extern __shared__ uint4 shared_digits[];   // uint2 [pair of slots of the segment][tile][lane][slot of the pair]
    __shared__ uint32_t tops[kQueries * kTiles];
    uint2 *digits = (uint2 *)shared_digits;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, h = lane / 16;
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot, groups = (a.cols + a.group - 1) / a.group;
    // workgroup b runs on die b mod 8: the passes over the same rows are neighbours on one die and share its L2
    const uint32_t turn = blockIdx.x / 8, blocks_across = gridDim.x / passes;
    const uint64_t first_query = (uint64_t)(turn % passes) * (kQueries * kTiles);
    const uint32_t queries = (uint32_t)std::min<uint64_t>(kQueries * kTiles, a.queries - first_query);

    if constexpr (kFloat) Queries<kQueries * kTiles, kThreads>(a, first_query, queries, threadIdx.x).tops(slots, tops);
    float unit[kTiles][kOut];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            if constexpr (kFloat) {
                unit[t][i] = Whole(tops[kQueries * t + h]).unit();
            } else {
                const uint32_t q = kQueries * t + 4 * h + i;
                unit[t][i] = q < queries ? Bytes(__float_as_uint(a.x_scale[first_query + q])).unit() : 0.0f;
            }
        }

    const uint64_t blocks = (a.rows + kBlockRows - 1) / kBlockRows;
    const uint64_t all_scales = a.rows * groups;
    bool staged = false;
    for (uint64_t block = turn / passes * 8 + blockIdx.x % 8; block < blocks; block += blocks_across) {
        const uint64_t first = block * kBlockRows + wave * (kRowTiles * 16) + r;
        float score[kRowTiles][kTiles][kOut];
#pragma unroll
        for (int n = 0; n < kRowTiles; ++n)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int i = 0; i < kOut; ++i) score[n][t][i] = 0.0f;
        for (uint32_t begin = 0; begin < slots; begin += segment) {
            const uint32_t end = std::min(begin + segment, slots);
            if (!staged) {
                __syncthreads();
                uint32_t thread = threadIdx.x;
                asm volatile("" : "+v"(thread));  // nothing of this waits in registers through the loops
                const Queries<kQueries * kTiles, kThreads> stage(a, first_query, queries, thread);
                if constexpr (kFloat) stage.split_floats(begin, end, Whole(tops[stage.q]).factor(), digits);
                else stage.split_8_bits(begin, end, digits);
                __syncthreads();
                staged = segment >= slots;
            }
            for (uint32_t base = begin; base < end; base += 4) {
                uint4 codes[kRowTiles];
                float scale[kRowTiles][4 / kPer];
#pragma unroll
                for (int n = 0; n < kRowTiles; ++n) {
                    const uint64_t row = first + 16 * n;
                    const bool there = row < a.rows;
                    codes[n] = there && base + h < end ? ((const uint4 *)a.codes)[row * slots + base + h] : make_uint4(0, 0, 0, 0);
                    // one load, which may reach into the next row's scales but not past the table's last; those count as 0
                    uint16_t bits[4 / kPer] = {};
                    const uint64_t at = row * groups + base / kPer;
                    if (there && at + 4 / kPer <= all_scales) {
                        __builtin_memcpy(bits, a.scales + at, sizeof bits);
                    } else if (there) {
#pragma unroll
                        for (int g = 0; g < 4 / kPer; ++g)
                            if (at + g < all_scales) bits[g] = a.scales[at + g];
                    }
#pragma unroll
                    for (int g = 0; g < 4 / kPer; ++g) scale[n][g] = base / kPer + g < groups ? scale_of(bits[g]) : 0.0f;
                }
                uint32_t word[kRowTiles][4];
#pragma unroll
                for (int n = 0; n < kRowTiles; ++n) transpose(codes[n], word[n]);
                i4 sums[kRowTiles][kTiles];
                auto add = [&](int g) {  // the sums of group g of these 128 columns
#pragma unroll
                    for (int n = 0; n < kRowTiles; ++n)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            const i4 d = sums[n][t];
                            if constexpr (kFloat) {
                                score[n][t][0] = fmaf(join_digits(d[0], d[1], d[2], d[3]), scale[n][g], score[n][t][0]);
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) score[n][t][i] = fmaf((float)d[i], scale[n][g], score[n][t][i]);
                            }
                        }
                    __builtin_amdgcn_sched_barrier(0);  // the sums of one group at a time: registers for more waves
                };
#pragma unroll
                for (int pair = 0; pair < 2; ++pair) {
                    // past the row's end whatever lies in LDS meets codes of 0
                    i4 x[kTiles], w[kRowTiles];
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        x[t] = __builtin_bit_cast(i4, shared_digits[((base - begin) / 2 + pair) * (kTiles * 64) + t * 64 + lane]);
#pragma unroll
                    for (int n = 0; n < kRowTiles; ++n) w[n] = code_bytes(word[n][2 * pair], word[n][2 * pair + 1]);
                    if constexpr (kPer == 1) {  // a slot at a time: 32 columns
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
#pragma unroll
                            for (int n = 0; n < kRowTiles; ++n)
#pragma unroll
                                for (int t = 0; t < kTiles; ++t)
                                    sums[n][t] = __builtin_amdgcn_mfma_i32_16x16x32_i8(half_of(x[t], j), half_of(w[n], j), i4{0, 0, 0, 0}, 0, 0, 0);
                            add(2 * pair + j);
                        }
                    } else {  // both
#pragma unroll
                        for (int n = 0; n < kRowTiles; ++n)
#pragma unroll
                            for (int t = 0; t < kTiles; ++t)
                                sums[n][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], w[n], kPer == 2 || pair == 0 ? i4{0, 0, 0, 0} : sums[n][t], 0, 0, 0);
                        if (kPer == 2 || pair == 1) add(kPer == 2 ? pair : 0);
                    }
                }
            }
        }
        float wrong = 0.0f;  // inf or NaN once a score is
#pragma unroll
        for (int n = 0; n < kRowTiles; ++n) {
            const uint64_t row = first + 16 * n;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int i = 0; i < kOut; ++i) {
                    const uint32_t q = kFloat ? kQueries * t + h : kQueries * t + 4 * h + i;
                    const float s = score[n][t][i] * unit[t][i];
                    if (row < a.rows && q < queries) a.out[(first_query + q) * a.out_stride + row] = s;
                    wrong = __builtin_elementwise_maximum(wrong, fabsf(s));
                }
        }
        if (!(wrong < __builtin_inff())) {
#pragma nounroll
            for (int n = 0; n < kRowTiles; ++n) scores_again<kFloat>(a, first + 16 * n, first_query, queries, h, tops);
        }
    }
}

// Many queries and rows of up to 64 columns: a load holds 64 / kSlots rows of kSlots slots (lane r + 16 h: slot h mod kSlots
// of row 16 (h / kSlots) + r), so that after the transposition word j is slot j mod kSlots of tile j / kSlots.
// One group: of the row (kPer = kSlots), or of each slot.  20 bfloat16 queries x 10^6 rows of 64 in 26 us, 4.5 TB/s; with loads
// of 16 rows that leave lanes idle 30.
template <bool kFloat, int kTiles, int kPer, int kSlots>
__global__ __launch_bounds__(many_threads(kTiles), 4) void k_score_narrow(ScoreArgs a, uint32_t passes) {
    constexpr int kQueries = kFloat ? 4 : 16, kOut = kFloat ? 1 : 4, kGroups = kSlots / kPer;
    constexpr int kThreads = many_threads(kTiles), kLoadRows = 64 / kSlots, kBlockRows = kThreads / 64 * kLoadRows;
    __shared__ uint4 shared_digits[kTiles * 64];
    __shared__ uint32_t tops[kQueries * kTiles];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, h = lane / 16;
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot;  // kSlots
    const uint32_t turn = blockIdx.x / 8, blocks_across = gridDim.x / passes;
    const uint64_t first_query = (uint64_t)(turn % passes) * (kQueries * kTiles);
    const uint32_t queries = (uint32_t)std::min<uint64_t>(kQueries * kTiles, a.queries - first_query);
    const Queries<kQueries * kTiles, kThreads> stage(a, first_query, queries, threadIdx.x);
    if constexpr (kFloat) {
        stage.tops(slots, tops);
        stage.split_floats(0, slots, Whole(tops[stage.q]).factor(), (uint2 *)shared_digits);
    } else {
        stage.split_8_bits(0, slots, (uint2 *)shared_digits);
    }
    __syncthreads();
    float unit[kTiles][kOut];
    i4 x[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        x[t] = __builtin_bit_cast(i4, shared_digits[t * 64 + lane]);  // of one slot: the second half is not used
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            const uint32_t q = kFloat ? kQueries * t + h : kQueries * t + 4 * h + i;
            if constexpr (kFloat) unit[t][i] = Whole(tops[q]).unit();
            else unit[t][i] = q < queries ? Bytes(__float_as_uint(a.x_scale[first_query + q])).unit() : 0.0f;
        }
    }
    const uint64_t blocks = (a.rows + kBlockRows - 1) / kBlockRows;
    for (uint64_t block = turn / passes * 8 + blockIdx.x % 8; block < blocks; block += blocks_across) {
        const uint64_t first = block * kBlockRows + wave * kLoadRows;
        const uint64_t mine = first + 16 * (h / kSlots) + r;
        const uint4 codes = mine < a.rows ? ((const uint4 *)a.codes)[mine * kSlots + h % kSlots] : make_uint4(0, 0, 0, 0);
        float scale[4 / kSlots][kGroups];
#pragma unroll
        for (int n = 0; n < 4 / kSlots; ++n) {
            const uint64_t row = first + 16 * n + r;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) scale[n][g] = row < a.rows ? scale_of(a.scales[row * kGroups + g]) : 0.0f;
        }
        uint32_t word[4];
        transpose(codes, word);
        float wrong = 0.0f;  // inf or NaN once a score is
#pragma unroll
        for (int n = 0; n < 4 / kSlots; ++n) {
            const uint64_t row = first + 16 * n + r;
            const i4 w = kSlots == 2 ? code_bytes(word[2 * n], word[2 * n + 1]) : code_bytes(word[n], 0);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                float score[kOut] = {};
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    i4 d = {0, 0, 0, 0};
                    if constexpr (kPer == 2) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], w, d, 0, 0, 0);
                    else d = __builtin_amdgcn_mfma_i32_16x16x32_i8(half_of(x[t], g), half_of(w, g), d, 0, 0, 0);
                    if constexpr (kFloat) {
                        score[0] = fmaf(join_digits(d[0], d[1], d[2], d[3]), scale[n][g], score[0]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) score[i] = fmaf((float)d[i], scale[n][g], score[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < kOut; ++i) {
                    const uint32_t q = kFloat ? kQueries * t + h : kQueries * t + 4 * h + i;
                    if (row < a.rows && q < queries) {
                        const float s = score[i] * unit[t][i];
                        a.out[(first_query + q) * a.out_stride + row] = s;
                        wrong = __builtin_elementwise_maximum(wrong, fabsf(s));
                    }
                }
            }
        }
        if (!(wrong < __builtin_inff())) {
#pragma nounroll
            for (int n = 0; n < 4 / kSlots; ++n) scores_again<kFloat>(a, first + 16 * n + r, first_query, queries, h, tops);
        }
    }
}

// ---------------------------------------------------------------------------
// A table from rows: 8 columns a lane, kLanes lanes to a group.  10^6 rows of 128 floats in 112 us, 5.2 TB/s.
template <class T, int kLanes>
__global__ __launch_bounds__(kThreads) void k_quantize(QuantizeArgs a, Walk walk) {
    const uint32_t groups = walk.each / kLanes, slots = (a.cols + kSlot - 1) / kSlot;
    walk_items(walk, [&](uint64_t row, uint32_t piece) {
        float v[8];
        load_piece((const T *)a.x + row * a.x_stride, 8 * piece, a.cols, v);
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = larger(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
        const float largest = __uint_as_float(largest_of_lanes<kLanes>(top));
        const bool finite = largest < __builtin_inff(), any = finite && largest >= 0x1p-100f;
        const __bf16 scale = !finite ? (__bf16)__builtin_nanf("") : any ? (__bf16)(largest * (float)(1.0 / 7.0)) : (__bf16)0.0f;
        const float up = any ? 1.0f / (float)scale : 0.0f;
        uint32_t word = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float w = fminf(fmaxf(v[k] * up, -7.0f), 7.0f);
            word |= (any ? (uint32_t)__float2int_rn(w) & 15u : 0u) << (4 * k);
        }
        if (piece < 4 * slots) ((uint32_t *)a.codes)[row * 4 * slots + piece] = word;
        if (piece % kLanes == 0) a.scales[row * groups + piece / kLanes] = __builtin_bit_cast(uint16_t, scale);
    });
}

// ---------------------------------------------------------------------------

template <bool kFloat, int kColumns, int kLanes, bool kLong>
hipError_t score_few(const ScoreArgs &a, hipStream_t stream) {
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot;
    const uint32_t bytes = kColumns * 32 * slots;
    const uint64_t waves = (a.rows + 64 / kLanes - 1) / (64 / kLanes);  // of one load each
    if (waves <= 4096)  // fewer than four loads for each of four waves on every compute unit: spread them
        return launch(k_score_few<kFloat, kColumns, kLanes, 1, kLong>, (uint32_t)((waves + kWaves - 1) / kWaves), kThreads, bytes, stream, a);
    const uint64_t tiles = (waves + 3) / 4, all = (tiles + kWaves - 1) / kWaves;
    const uint64_t turns = (all + (kLong ? 1024 : 2048) - 1) / (kLong ? 1024 : 2048);  // of every workgroup, as many of each
    return launch(k_score_few<kFloat, kColumns, kLanes, 4, kLong>, (uint32_t)((all + turns - 1) / turns), kThreads, bytes, stream, a);
}

template <bool kFloat, int kColumns>
hipError_t score_few_by_length(const ScoreArgs &a, hipStream_t stream) {
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot;
    if (slots <= 1) return score_few<kFloat, kColumns, 1, false>(a, stream);
    if (slots <= 2) return score_few<kFloat, kColumns, 2, false>(a, stream);
    if (slots <= 4) return score_few<kFloat, kColumns, 4, false>(a, stream);
    if (slots <= 8) return score_few<kFloat, kColumns, 8, false>(a, stream);
    if (slots <= 16) return score_few<kFloat, kColumns, 16, false>(a, stream);
    if (slots <= 32) return score_few<kFloat, kColumns, 32, false>(a, stream);
    if (slots <= 64) return score_few<kFloat, kColumns, 64, false>(a, stream);
    return score_few<kFloat, kColumns, 64, true>(a, stream);
}

template <bool kFloat, int kTiles, int kPer>
hipError_t score_many(const ScoreArgs &a, hipStream_t stream) {
    // Two row tiles a wave write whole lines of a query's scores and read its digits once for both (16 queries x 4*10^6
    // rows of 128: 119 us, 124 with one; 4 queries in floats: 69 and 97; 16 bfloat16 queries x 5*10^5 rows of 1024 in groups
    // of 32: 139 and 173).  Rows of over 256 columns in larger groups, whose sums are joined more seldom, gain more from more
    // waves (4 queries x 10^6 rows of 512 in groups of 128: 73 us and 63), and more tiles of 8-bit queries do not fit the
    // registers twice (64 queries x 10^6 rows of 128: 165 us, 92 with one).
    constexpr int kRowTiles = kTiles == 1 || (kFloat && kTiles < 8) ? 2 : 1, kAll = many_threads(kTiles), kEach = (kFloat ? 4 : 16) * kTiles;
    const uint32_t slots = (a.cols + kSlot - 1) / kSlot;
    const uint32_t segment = std::min((slots + 3) / 4 * 4, 128u / kTiles), bytes = segment * kTiles * 512;
    const uint32_t passes = (uint32_t)((a.queries + kEach - 1) / kEach);
    const uint64_t tiles = (a.rows + 15) / 16;
    // workgroups across the rows, a multiple of the dies; more than are resident gain nothing, each splits its queries first
    auto across = [&](uint32_t row_tiles) {
        const uint64_t each = row_tiles * (kAll / 64), all = (tiles + each - 1) / each;
        const uint64_t most = std::max<uint64_t>(1, (bytes > 32768 || kAll > 256 ? 512 : 1024) / passes);
        return (uint32_t)((std::min(all, most) + 7) / 8 * 8);
    };
    if (tiles <= 4096 || (slots > 8 && kPer > 1))
        return launch(k_score_many<kFloat, kTiles, kPer, 1>, across(1) * passes, kAll, bytes, stream, a, segment, passes);
    return launch(k_score_many<kFloat, kTiles, kPer, kRowTiles>, across(kRowTiles) * passes, kAll, bytes, stream, a, segment, passes);
}

template <bool kFloat, int kTiles, int kPer, int kSlots>
hipError_t score_narrow(const ScoreArgs &a, hipStream_t stream) {
    constexpr int kAll = many_threads(kTiles), kEach = (kFloat ? 4 : 16) * kTiles, kRows = kAll / kSlots;
    const uint32_t passes = (uint32_t)((a.queries + kEach - 1) / kEach);
    const uint64_t across = std::min<uint64_t>((a.rows + kRows - 1) / kRows, std::max<uint64_t>(1, (kAll > 256 ? 512 : 1024) / passes));
    return launch(k_score_narrow<kFloat, kTiles, kPer, kSlots>, (uint32_t)((across + 7) / 8 * 8) * passes, kAll, 0, stream, a, passes);
}

template <bool kFloat, int kTiles>
hipError_t score_many_by_group(const ScoreArgs &a, hipStream_t stream) {
    if (a.cols <= kSlot) return score_narrow<kFloat, kTiles, 1, 1>(a, stream);
    if (a.cols <= 2 * kSlot && a.group == 32) return score_narrow<kFloat, kTiles, 1, 2>(a, stream);
    if (a.cols <= 2 * kSlot) return score_narrow<kFloat, kTiles, 2, 2>(a, stream);
    if (a.group == 32) return score_many<kFloat, kTiles, 1>(a, stream);
    if (a.group == 64) return score_many<kFloat, kTiles, 2>(a, stream);
    return score_many<kFloat, kTiles, 4>(a, stream);
}

template <class T>
hipError_t quantize(const QuantizeArgs &a, hipStream_t stream) {
    const uint32_t pieces = (a.cols + a.group - 1) / a.group * (a.group / 8);  // of a row, with those that fill its last group
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((a.rows * pieces + kThreads - 1) / kThreads, 8192);
    const Walk walk = walk_of(a.rows, pieces, (uint64_t)blocks * kThreads);
    if (a.group == 32) return launch(k_quantize<T, 4>, blocks, kThreads, 0, stream, a, walk);
    if (a.group == 64) return launch(k_quantize<T, 8>, blocks, kThreads, 0, stream, a, walk);
    return launch(k_quantize<T, 16>, blocks, kThreads, 0, stream, a, walk);
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream) {
    if (a.type == GV_F32) return quantize<float>(a, stream);
    if (a.type == GV_BF16) return quantize<__bf16>(a, stream);
    return quantize<_Float16>(a, stream);
}

hipError_t launch_score(const ScoreArgs &a, hipStream_t stream) {
    const uint64_t q = a.queries;
    if (a.type == GV_I8) {
        if (q == 1) return score_few_by_length<false, 1>(a, stream);
        if (q == 2) return score_few_by_length<false, 2>(a, stream);
        if (q <= 4) return score_few_by_length<false, 4>(a, stream);
        if (q <= 16) return score_many_by_group<false, 1>(a, stream);
        if (q <= 32) return score_many_by_group<false, 2>(a, stream);
        return score_many_by_group<false, 4>(a, stream);
    }
    if (q == 1) return score_few_by_length<true, 4>(a, stream);
    if (q <= 4) return score_many_by_group<true, 1>(a, stream);
    if (q <= 8) return score_many_by_group<true, 2>(a, stream);
    if (q <= 16) return score_many_by_group<true, 4>(a, stream);
    return score_many_by_group<true, 8>(a, stream);
}

}  // namespace gv
