// gfx950 kernels of rows by index: the rows of a table that indices name, and the gradient of that, the sums of the rows of a
// batch by index.
//
// Both are bound by memory: a row of the batch is read once and a row of the table written once.  Sums are taken in an order
// that the indices decide, never by atomics: indices are sorted (stably, so equal ones stay in the order of the batch),
// workgroups take equal pieces of the sorted batch and sum up its runs of equal indices; a long run that crosses borders leaves
// a partial sum for each piece, which are joined by a launch of their own.
#include "gv_row_pieces.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#include <algorithm>
#include <type_traits>

namespace gv {
namespace {

// The row that place t of a batch names; `rows` where it names none.
__device__ __forceinline__ uint32_t row_at(const Index &index, uint64_t t, uint32_t rows) {
    if (index.type == GV_I32) {
        const uint32_t i = ((const uint32_t *)index.at)[t * index.stride];
        return i < rows ? i : rows;
    }
    const uint64_t i = ((const uint64_t *)index.at)[t * index.stride];
    return i < rows ? (uint32_t)i : rows;
}

// ---------------------------------------------------------------------------
// Rows by index: one piece of eight columns a lane and turn.  2^20 rows of 128 floats out of 10^6, into bfloat16: 122 us for
// 775 MB, 6.4 TB/s; many loads wait at once because a lane has one piece and workgroups come and go.
constexpr int kLookupThreads = 256;

template <class In, class Out>
__global__ __launch_bounds__(kLookupThreads) void k_lookup(LookupArgs a, Walk walk) {
    walk_items(walk, [&](uint64_t t, uint32_t piece) {
        const uint32_t row = row_at(a.index, t, a.rows);
        float v[8] = {};
        if (row < a.rows) load_piece((const In *)a.table + row * a.table_stride, 8 * piece, a.cols, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = row < a.rows ? v[i] * a.scale : 0.0f;
        store_piece((Out *)a.out + t * a.out_stride, 8 * piece, a.cols, v);
    });
}

// The same without arithmetic: the values are copied as they are, of any type of that size.
template <class Word>
__global__ __launch_bounds__(kLookupThreads) void k_copy_rows(LookupArgs a, Walk walk) {
    walk_items(walk, [&](uint64_t t, uint32_t piece) {
        const uint32_t row = row_at(a.index, t, a.rows), k = 8 * piece;
        Piece<Word> p{};
        if (row < a.rows) p.load((const Word *)a.table + row * a.table_stride, k, a.cols);
        Word *to = (Word *)a.out + t * a.out_stride;
        if (k + 8 <= a.cols) {
            __builtin_memcpy(to + k, &p, sizeof p);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < a.cols) to[k + i] = p.at[i];
        }
    });
}

// ---------------------------------------------------------------------------
// The gradient.  A row takes `lanes` lanes (a power of two up to 64), a piece of eight columns each, and one part of 512 columns
// after the other where it is longer.

// Rows of eight columns and more (kWide) have no broken piece: the last one lies back so far that it is whole, and two lanes of
// a group have the columns that it shares with the one before, and the same sums of them.  A part of a row has 512 columns, or
// 504 where the last would have fewer than eight: pieces of two parts share none.  (A piece that may be broken is loaded in so
// many parts that a step of the sums waits for each of them: 2^20 rows of 128 took 240 us instead of 120.)  They are the same
// wave's, so that with add both have read what was there before either writes.
__host__ __device__ __forceinline__ uint32_t part_of(uint32_t cols) { return cols > 512 && cols % 512 > 0 && cols % 512 < 8 ? 504 : 512; }
template <bool kWide>
__device__ __forceinline__ uint32_t first_of(uint32_t k, uint32_t cols) {
    return kWide ? std::min(k, cols - 8) : k;
}
template <bool kWide>
__device__ __forceinline__ uint32_t cols_of(uint32_t k, uint32_t cols) {
    return kWide ? k + 8 : cols;
}
// A finished sum goes to its row.
template <class Out, bool kWide>
__device__ __forceinline__ void put_sum(const LookupGradArgs &a, uint32_t row, uint32_t k, float (&v)[8]) {
    Out *to = (Out *)a.out + row * a.out_stride;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= a.scale;
    if (a.add) {
        float there[8];
        load_piece(to, k, cols_of<kWide>(k, a.cols), there);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there[i] + v[i];
    }
    store_piece(to, k, cols_of<kWide>(k, a.cols), v);
}

// Sums over the groups of a workgroup, in their order, for group 0: lane l of a group has piece l of them.
constexpr int kGradThreads = 256;
__device__ __forceinline__ void join_groups(float (&v)[8], float (*scratch)[8], uint32_t lanes) {
    __builtin_memcpy(scratch[threadIdx.x], v, sizeof v);
    __syncthreads();
    if (threadIdx.x >= lanes) return;
    for (uint32_t g = threadIdx.x + lanes; g < kGradThreads; g += lanes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += scratch[g][i];
    }
}

// Few places: every workgroup reads all indices, so one launch does it.  The workgroup of a place whose row no place before it
// names adds up all places of that row; others end.  Workgroups behind those write zeros to the rows that are not named.
constexpr uint32_t kFew = 1024, kFillRows = 4096;

template <class In, class Out, bool kWide>
__global__ __launch_bounds__(kGradThreads) void k_grad_few(LookupGradArgs a, uint32_t parts, uint32_t fill_blocks, uint32_t fill_rows) {
    constexpr int kEach = kFew / kGradThreads;
    __shared__ float scratch[kGradThreads][8];
    __shared__ uint16_t same[kFew];
    __shared__ uint32_t counts[kGradThreads / 64], named[kFillRows / 32];
    const uint32_t tid = threadIdx.x, count = (uint32_t)a.count;
    if (blockIdx.x >= count * parts) {
        const uint64_t pieces = (a.cols + 7) / 8;
        for (uint64_t first = (uint64_t)(blockIdx.x - count * parts) * fill_rows; first < a.rows; first += (uint64_t)fill_blocks * fill_rows) {
            const uint32_t some = (uint32_t)std::min<uint64_t>(fill_rows, a.rows - first);
            for (uint32_t w = tid; w < kFillRows / 32; w += kGradThreads) named[w] = 0;
            __syncthreads();
            for (uint32_t t = tid; t < count; t += kGradThreads) {
                const uint64_t row = row_at(a.index, t, a.rows);
                if (row >= first && row < first + some) atomicOr(&named[(row - first) / 32], 1u << ((row - first) % 32));
            }
            __syncthreads();
            for (uint64_t i = tid; i < some * pieces; i += kGradThreads) {
                const uint32_t r = (uint32_t)(i / pieces), piece = (uint32_t)(i % pieces);
                if (named[r / 32] >> (r % 32) & 1) continue;
                const float zeros[8] = {};
                store_piece((Out *)a.out + (first + r) * a.out_stride, 8 * piece, a.cols, zeros);
            }
            __syncthreads();
        }
        return;
    }
    const uint32_t place = blockIdx.x / parts, part = blockIdx.x % parts;
    const uint32_t row = row_at(a.index, place, a.rows);
    if (row >= a.rows) return;  // all threads alike
    bool before = false;
    uint32_t found = 0, mine = 0;  // places kEach * tid + i that name the row, as bits
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t t = kEach * tid + i;
        if (t < count && row_at(a.index, t, a.rows) == row) {
            before |= t < place;
            found |= 1u << i;
            ++mine;
        }
    }
    if (__syncthreads_or(before)) return;
    uint32_t upto = mine;  // over the threads of this wave
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = __shfl_up(upto, d);
        if (tid % 64 >= (uint32_t)d) upto += other;
    }
    if (tid % 64 == 63) counts[tid / 64] = upto;
    __syncthreads();
    uint32_t to = upto - mine, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kGradThreads / 64; ++w) {
        if (w < tid / 64) to += counts[w];
        all += counts[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (found >> i & 1) same[to++] = (uint16_t)(kEach * tid + i);
    __syncthreads();
    const uint32_t lanes = a.lanes, lane = tid % lanes, groups = kGradThreads / lanes;
    const uint32_t width = part_of(a.cols), column = width * part + 8 * lane;
    const bool used = 8 * lane < width && column < a.cols;
    const uint32_t k = first_of<kWide>(column, a.cols);
    float sum[8] = {};
    if (used) {
        for (uint32_t j = tid / lanes; j < all; j += 4 * groups) {
            Piece<In> p[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
                if (j + u * groups < all) p[u].load((const In *)a.grad + same[j + u * groups] * a.grad_stride, k, cols_of<kWide>(k, a.cols));
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                if (j + u * groups >= all) continue;
                float v[8];
                p[u].values(v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[i];
            }
        }
    }
    join_groups(sum, scratch, lanes);
    if (tid < lanes && used) put_sum<Out, kWide>(a, row, k, sum);
}

// --- the order of the places by row: pairs of a row (`rows` for places without one, at the end) and a place, sorted.

// Some thousand places: the place of each is how many go before it.  A workgroup of 16 waves takes 64 places, each wave a
// sixteenth of those that they are compared with.  (Places added to 10^6 rows of 128 by ranks and by
// digits, which are six launches but few comparisons, us: 2048 17 and 32, 4096 24 and 34, 8192 39 and 36, 16384 68 and 38.)
constexpr int kRankThreads = 1024;
constexpr uint32_t kRanked = 1 << 13;

__device__ __forceinline__ void clear_flags(uint8_t *flags, uint64_t rows) {
    if (!flags) return;
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; 4 * i < rows; i += (uint64_t)gridDim.x * blockDim.x)
        ((uint32_t *)flags)[i] = 0;  // whole words: the workspace has room for them
}

__global__ __launch_bounds__(kRankThreads) void k_rank(LookupGradArgs a) {
    __shared__ uint32_t ranks[kRankThreads / 64][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, t = blockIdx.x * 64 + lane, count = (uint32_t)a.count;
    const uint32_t mine = t < count ? row_at(a.index, t, a.rows) : 0;
    const uint32_t each = ((count + 15) / 16 + 63) & ~63u, first = wave * each, last = std::min(count, first + each);
    uint32_t rank = 0;
    for (uint32_t s = first; s < last; s += 64) {
        const uint32_t theirs = s + lane < last ? row_at(a.index, s + lane, a.rows) : 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < 64; ++i) {
            const uint32_t other = __builtin_amdgcn_readlane(theirs, i);
            rank += other < mine || (other == mine && s + i < t) ? 1 : 0;
        }
    }
    ranks[wave][lane] = rank;
    __syncthreads();
    if (wave > 0 || t >= count) return;
#pragma unroll
    for (int w = 1; w < kRankThreads / 64; ++w) rank += ranks[w][lane];
    a.sorted[rank] = uint2{mine, t};
}

// Sets the flag of every row that is named.
__global__ __launch_bounds__(256) void k_flag(LookupGradArgs a) {
    for (uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x; t < a.count; t += (uint64_t)gridDim.x * 256) {
        const uint32_t row = row_at(a.index, t, a.rows);
        if (row < a.rows) a.flags[row] = 1;
    }
}
__global__ __launch_bounds__(256) void k_clear_flags(uint8_t *flags, uint64_t rows) { clear_flags(flags, rows); }

// More: digits of up to 11 bits, the lowest first; places with equal digits keep their order.  Three launches a digit: how
// often each workgroup's places have each digit, where those begin, and the places moved there (2^20 places: 10, 6 and 21 us,
// each bound by the latency of a few dependent steps; pieces of 2048 places, 4096 and 8192 took 65, 73 and 100 us for two
// digits).
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64, kSortSteps = 4;
constexpr uint32_t kSortTile = kSortThreads * kSortSteps, kMostDigits = 1u << 11;

struct Digit {
    const uint2 *from;  // null: as the batch has them
    uint2 *to;
    uint32_t shift, bits, tiles;
    uint8_t *set_flags;  // of the last digit, or null
};

__global__ __launch_bounds__(kSortThreads) void k_count_digits(LookupGradArgs a, Digit d) {
    __shared__ uint32_t counts[kMostDigits];
    const uint32_t digits = 1u << d.bits;
    for (uint32_t i = threadIdx.x; i < digits; i += kSortThreads) counts[i] = 0;
    if (!d.from) clear_flags(a.flags, a.rows);
    __syncthreads();
    const uint64_t first = (uint64_t)blockIdx.x * kSortTile;
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const uint64_t t = first + s * kSortThreads + threadIdx.x;
        if (t >= a.count) continue;
        const uint32_t key = d.from ? d.from[t].x : row_at(a.index, t, a.rows);
        atomicAdd(&counts[key >> d.shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < digits; i += kSortThreads) a.digit_counts[(uint64_t)i * d.tiles + blockIdx.x] = counts[i];
}

// A wave to a digit: its counts become the sums of those before, its total goes behind them all.
__global__ __launch_bounds__(256) void k_sum_digits(LookupGradArgs a, Digit d) {
    const uint32_t digit = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (digit >= 1u << d.bits) return;
    uint32_t *counts = a.digit_counts + (uint64_t)digit * d.tiles, before = 0;
    for (uint32_t i = lane; i - lane < d.tiles; i += 64) {
        const uint32_t mine = i < d.tiles ? counts[i] : 0;
        uint32_t upto = mine;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const uint32_t other = __shfl_up(upto, s);
            if (lane >= (uint32_t)s) upto += other;
        }
        if (i < d.tiles) counts[i] = before + upto - mine;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (lane == 0) a.digit_totals[digit] = before;
}

__global__ __launch_bounds__(kSortThreads) void k_place_digits(LookupGradArgs a, Digit d) {
    __shared__ uint32_t base[kMostDigits], sums[kSortWaves];
    __shared__ uint16_t counts[kSortWaves][kMostDigits];
    const uint32_t digits = 1u << d.bits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (uint32_t i = lane; i < digits; i += 64) counts[wave][i] = 0;
    // where each digit's places begin: four digits a thread
    uint32_t total[kMostDigits / kSortThreads], upto = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMostDigits / kSortThreads; ++i) {
        const uint32_t digit = threadIdx.x * (kMostDigits / kSortThreads) + i;
        total[i] = digit < digits ? a.digit_totals[digit] : 0;
        upto += total[i];
    }
    const uint32_t mine = upto;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const uint32_t other = __shfl_up(upto, s);
        if (lane >= (uint32_t)s) upto += other;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    upto -= mine;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) upto += w < wave ? sums[w] : 0;
#pragma unroll
    for (uint32_t i = 0; i < kMostDigits / kSortThreads; ++i) {
        const uint32_t digit = threadIdx.x * (kMostDigits / kSortThreads) + i;
        if (digit < digits) base[digit] = upto + a.digit_counts[(uint64_t)digit * d.tiles + blockIdx.x];
        upto += total[i];
    }
    // a wave takes 256 places in a row, and counts those with the same digit before each
    uint2 pair[kSortSteps];
    uint32_t rank[kSortSteps];
    const uint64_t first = (uint64_t)blockIdx.x * kSortTile + wave * (64 * kSortSteps) + lane;
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const uint64_t t = first + 64 * s;
        pair[s] = t >= a.count ? uint2{0, 0} : d.from ? d.from[t] : uint2{row_at(a.index, t, a.rows), (uint32_t)t};
    }
    volatile uint16_t *mine_of = counts[wave];
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const bool there = first + 64 * s < a.count;
        const uint32_t digit = pair[s].x >> d.shift & (digits - 1);
        uint64_t same = __ballot(there);
        for (uint32_t b = 0; b < d.bits; ++b) {
            const bool one = digit >> b & 1;
            const uint64_t set = __ballot(one);
            same &= one ? set : ~set;
        }
        const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
        if (there) {
            const uint32_t before = mine_of[digit];
            rank[s] = before + below;
            if (below == 0) mine_of[digit] = (uint16_t)(before + __popcll(same));
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < digits; i += kSortThreads) {  // over the waves
        uint32_t before = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t some = counts[w][i];
            counts[w][i] = (uint16_t)before;
            before += some;
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const uint64_t t = first + 64 * s;
        if (t >= a.count) continue;
        const uint32_t digit = pair[s].x >> d.shift & (digits - 1);
        const uint32_t to = base[digit] + counts[wave][digit] + rank[s];
        d.to[to] = pair[s];
        if (d.set_flags && pair[s].x < a.rows) d.set_flags[pair[s].x] = 1;
    }
}

// --- the sums over the sorted places

// A workgroup takes `chunk` sorted places, whose runs of equal rows its groups of lanes take in turn; long ones are taken by
// all groups together. A run that begins there and ends within chunk / 4 places behind them is finished, and the workgroup of
// the next chunk leaves it out.  A longer one leaves partial[2 c + 1] where it begins, and partial[2 c] where it began before
// (whether it ends there or not).  So the many short runs are summed and written once, and only the few long ones pass through
// memory.  Workgroups behind those write zeros to the rows that are not named.  2^20 bfloat16 rows of 128 into 10^6 of floats:
// 190 to 200 us for 801 MB, 4.0 TB/s, of 285 for the whole call; a run's rows are asked for four at a time, and what else waits
// at once is other groups'.
constexpr uint32_t kMostChunk = 1024, kLong = 32;

__device__ __forceinline__ uint32_t key_at(const LookupGradArgs &a, uint64_t p) { return p < a.count ? a.sorted[p].x : 0xFFFFFFFFu; }
// whether the run of `key` that goes on behind `border`, the first border that it passes, ends soon
__device__ __forceinline__ bool ends_soon(const LookupGradArgs &a, uint64_t border, uint32_t key) { return key_at(a, border + a.chunk / 4) != key; }

template <class In, class Out, bool kWide>
__global__ __launch_bounds__(kGradThreads) void k_sum_runs(LookupGradArgs a, Walk fill, uint32_t sum_blocks) {
    constexpr uint32_t kEach = kMostChunk / kGradThreads;
    __shared__ uint2 pairs[kMostChunk + kMostChunk / 4 + 1];
    __shared__ uint16_t begins[kMostChunk + 1], longs[kMostChunk / kLong + 2];
    __shared__ uint32_t counts[kGradThreads / 64], found_longs;
    __shared__ float scratch[kGradThreads][8];
    if (blockIdx.x >= sum_blocks) {
        walk_items(fill, [&](uint64_t row, uint32_t piece) {
            if (a.flags[row]) return;
            const float zeros[8] = {};
            store_piece((Out *)a.out + row * a.out_stride, 8 * piece, a.cols, zeros);
        }, blockIdx.x - sum_blocks);
        return;
    }
    const uint32_t tid = threadIdx.x, c = blockIdx.x % a.chunks, part = blockIdx.x / a.chunks;
    const uint64_t first = (uint64_t)c * a.chunk;
    const uint32_t size = (uint32_t)std::min<uint64_t>(a.chunk, a.count - first), reach = size + a.chunk / 4;
    for (uint32_t i = tid; i <= reach; i += kGradThreads) pairs[i] = first + i < a.count ? a.sorted[first + i] : uint2{0xFFFFFFFFu, 0};
    const uint32_t before = first ? a.sorted[first - 1].x : 0xFFFFFFFFu, far = first > a.chunk ? a.sorted[first - a.chunk - 1].x : 0xFFFFFFFFu;
    if (tid == 0) found_longs = 0;
    __syncthreads();
    // where runs begin, and the first place
    uint32_t mine = 0, number = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t at = tid * kEach + i;
        if (at < size && (at == 0 || pairs[at].x != pairs[at - 1].x)) mine |= 1u << i, ++number;
    }
    uint32_t upto = number;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = __shfl_up(upto, d);
        if (tid % 64 >= (uint32_t)d) upto += other;
    }
    if (tid % 64 == 63) counts[tid / 64] = upto;
    __syncthreads();
    uint32_t to = upto - number, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kGradThreads / 64; ++w) {
        if (w < tid / 64) to += counts[w];
        all += counts[w];
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
        if (mine >> i & 1) begins[to++] = (uint16_t)(tid * kEach + i);
    __syncthreads();
    const bool headless = pairs[0].x == before;  // the first run began before, and ended soon behind its first border:
    const bool left_out = headless && far != before && pairs[a.chunk / 4].x != before;
    const uint32_t lanes = a.lanes, lane = tid % lanes, groups = kGradThreads / lanes;
    const uint32_t width = part_of(a.cols), column = width * part + 8 * lane;
    const bool used = 8 * lane < width && column < a.cols;
    const uint32_t k = first_of<kWide>(column, a.cols);
    // run j from place p on, behind `end`; whether it is finished here
    const auto run_of = [&](uint32_t j, uint32_t &p, uint32_t &end, bool &goes_on) {
        p = begins[j];
        goes_on = false;
        if (j + 1 < all) {
            end = begins[j + 1];
            return;
        }
        end = size;
        const uint32_t key = pairs[p].x;
        if (pairs[end].x != key) return;
        goes_on = (j == 0 && headless) || pairs[reach].x == key;
        while (!goes_on && pairs[end].x == key) ++end;
    };
    const auto add_up = [&](uint32_t p, uint32_t end, uint32_t step, float (&sum)[8]) {
        for (; p < end; p += 4 * step) {
            Piece<In> rows[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
                if (p + u * step < end) rows[u].load((const In *)a.grad + pairs[p + u * step].y * a.grad_stride, k, cols_of<kWide>(k, a.cols));
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                if (p + u * step >= end) continue;
                float v[8];
                rows[u].values(v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[i];
            }
        }
    };
    const auto finish = [&](uint32_t j, uint32_t key, bool goes_on, float (&sum)[8]) {
        const bool head = j == 0 && headless;
        if (!head && !goes_on) put_sum<Out, kWide>(a, key, k, sum);
        else store_piece(a.partial + (2ull * c + (head ? 0 : 1)) * a.cols, k, cols_of<kWide>(k, a.cols), sum);
    };
    for (uint32_t j = tid / lanes; j < all; j += groups) {
        uint32_t p, end;
        bool goes_on;
        run_of(j, p, end, goes_on);
        const uint32_t key = pairs[p].x;
        if (key >= a.rows || (j == 0 && left_out)) continue;
        if (end - p > kLong) {
            if (lane == 0) longs[atomicAdd(&found_longs, 1u)] = (uint16_t)j;
            continue;
        }
        if (!used) continue;
        float sum[8] = {};
        add_up(p, end, 1, sum);
        finish(j, key, goes_on, sum);
    }
    __syncthreads();
    for (uint32_t l = 0; l < found_longs; ++l) {
        uint32_t p, end;
        bool goes_on;
        run_of(longs[l], p, end, goes_on);
        float sum[8] = {};
        if (used) add_up(p + tid / lanes, end, groups, sum);
        join_groups(sum, scratch, lanes);
        if (tid < lanes && used) finish(longs[l], pairs[p].x, goes_on, sum);
        __syncthreads();
    }
}

// Joins the partial sums of the long runs that begin among the places of kJoinChunks chunks: a thread looks at each chunk, and
// the workgroup goes through what was found.
constexpr uint32_t kJoinChunks = 16;

template <class Out, bool kWide>
__global__ __launch_bounds__(kGradThreads) void k_join_runs(LookupGradArgs a) {
    __shared__ float scratch[kGradThreads][8];
    __shared__ uint64_t found;
    const uint32_t blocks = (a.chunks + kJoinChunks - 1) / kJoinChunks, base = blockIdx.x % blocks * kJoinChunks;
    const uint32_t lanes = a.lanes, lane = threadIdx.x % lanes, groups = kGradThreads / lanes;
    const uint32_t width = part_of(a.cols), column = width * (blockIdx.x / blocks) + 8 * lane;
    const bool used = 8 * lane < width && column < a.cols;
    const uint32_t k = first_of<kWide>(column, a.cols);
    if (threadIdx.x < 64) {
        const uint64_t first = (uint64_t)(base + threadIdx.x) * a.chunk, last = first + a.chunk;
        bool mine = false;
        if (threadIdx.x < kJoinChunks && base + threadIdx.x < a.chunks && last < a.count) {
            const uint32_t key = key_at(a, last - 1);
            const bool began = key_at(a, first) != key || first == 0 || key_at(a, first - 1) != key;
            mine = key < a.rows && key_at(a, last) == key && began && !ends_soon(a, last, key);
        }
        const uint64_t all = __ballot(mine);
        if (threadIdx.x == 0) found = all;
    }
    __syncthreads();
    for (uint64_t left = found; left; left &= left - 1) {
        const uint32_t c = base + __builtin_ctzll(left);
        const uint64_t last = (uint64_t)(c + 1) * a.chunk;
        const uint32_t key = key_at(a, last);
        uint32_t more = 0;  // chunks behind c that begin inside the run
        for (;;) {
            const uint32_t some = __syncthreads_count(key_at(a, last + (uint64_t)(more + threadIdx.x) * a.chunk) == key);
            more += some;
            if (some < kGradThreads) break;
        }
        float sum[8] = {};
        if (used) {
            for (uint32_t j = threadIdx.x / lanes; j <= more; j += 4 * groups) {  // 0: its own
                float v[4][8];
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) {
                    const uint32_t at = j + u * groups;
                    if (at <= more) load_piece(a.partial + (2ull * (c + at) + (at == 0 ? 1 : 0)) * a.cols, k, cols_of<kWide>(k, a.cols), v[u]);
                }
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u)
                    if (j + u * groups <= more)
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[i] += v[u][i];
            }
        }
        join_groups(sum, scratch, lanes);
        if (threadIdx.x < lanes && used) put_sum<Out, kWide>(a, key, k, sum);
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------

template <class Run>
hipError_t by_type(int type, Run &&run) {
    if (type == GV_F32) return run((float *)nullptr);
    if (type == GV_BF16) return run((__bf16 *)nullptr);
    return run((_Float16 *)nullptr);
}
template <class Run>
hipError_t by_types(int in, int out, Run &&run) {
    return by_type(in, [&](auto *i) { return by_type(out, [&](auto *o) { return run(i, o); }); });
}

constexpr uint64_t kMostBlocks = 1 << 22;

uint32_t lanes_of(uint32_t cols) {
    uint32_t lanes = 1;
    while (lanes < 64 && 8 * lanes < cols) lanes *= 2;
    return lanes;
}

// How a batch is cut, and where its parts of the workspace lie (in words of four bytes).
struct Plan {
    uint32_t lanes, parts, chunk, chunks, bits, passes, tiles;
    uint64_t sorted[2], counts, totals, flags, partial, words;
};

Plan plan_of(uint64_t count, uint64_t rows, uint32_t cols, bool add) {
    Plan p{};
    p.lanes = lanes_of(cols);
    p.parts = (cols + part_of(cols) - 1) / part_of(cols);
    // a thousand workgroups, of at least 32 places and of at most 256, unless the partial sums of long rows took over 32 MB
    p.chunk = 32;
    while (p.chunk < 256 && p.chunk * 1024ull < count) p.chunk *= 2;
    while (p.chunk < kMostChunk && count / p.chunk * cols > (1 << 22)) p.chunk *= 2;
    p.chunks = (uint32_t)((count + p.chunk - 1) / p.chunk);
    while (rows >> p.bits) ++p.bits;  // `rows` itself is a key
    p.passes = (p.bits + 10) / 11;
    p.tiles = (uint32_t)((count + kSortTile - 1) / kSortTile);
    uint64_t at = 0;
    const auto take = [&](uint64_t words) {
        const uint64_t here = at;
        at += (words + 3) & ~3ull;
        return here;
    };
    const int pairs = count <= kRanked ? 1 : 2;
    for (int i = 0; i < pairs; ++i) p.sorted[i] = take(2 * count);
    if (count > kRanked) {
        p.counts = take((uint64_t)kMostDigits * p.tiles);
        p.totals = take(kMostDigits);
    }
    p.flags = take(add ? 0 : (rows + 3) / 4);
    p.partial = take(2ull * p.chunks * cols);
    p.words = at;
    return p;
}

}  // namespace

uint64_t lookup_grad_workspace(uint64_t count, uint64_t rows, uint32_t cols, bool add) {
    return count <= kFew ? 0 : 4 * plan_of(count, rows, cols, add).words;
}

hipError_t launch_lookup(const LookupArgs &a, hipStream_t stream) {
    const uint32_t pieces = (a.cols + 7) / 8;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((a.count * pieces + kLookupThreads - 1) / kLookupThreads, kMostBlocks);
    const Walk walk = walk_of(a.count, pieces, (uint64_t)blocks * kLookupThreads);
    const auto copy = [&](auto word) { return launch(k_copy_rows<decltype(word)>, blocks, kLookupThreads, 0, stream, a, walk); };
    if (a.type == a.out_type && a.scale == 1.0f) {
        if (a.type == GV_I8) return copy(uint8_t());
        if (a.type == GV_BF16 || a.type == GV_F16) return copy(uint16_t());
        if (a.type == GV_I64) return copy(uint64_t());
        return copy(uint32_t());
    }
    return by_types(a.type, a.out_type, [&](auto *i, auto *o) {
        return launch(k_lookup<std::remove_pointer_t<decltype(i)>, std::remove_pointer_t<decltype(o)>>, blocks, kLookupThreads, 0, stream, a, walk);
    });
}

hipError_t launch_lookup_grad(const LookupGradArgs &args, void *workspace, hipStream_t stream) {
    LookupGradArgs a = args;
    const uint32_t pieces = (a.cols + 7) / 8;
    if (a.count <= kFew) {
        a.lanes = lanes_of(a.cols);
        const uint32_t parts = (a.cols + part_of(a.cols) - 1) / part_of(a.cols);
        // rows that a workgroup writes zeros to: 16 KB of them at least, and a thousand workgroups where that is enough
        const uint64_t each = std::max<uint64_t>(std::max<uint64_t>(1, 512 / pieces), (a.rows + 1023) / 1024);
        const uint32_t fill_rows = (uint32_t)std::min<uint64_t>(each, kFillRows);
        const uint32_t fill = a.add ? 0 : (uint32_t)std::min<uint64_t>((a.rows + fill_rows - 1) / fill_rows, 1 << 16);
        if (a.count == 0 && fill == 0) return hipSuccess;
        return by_types(a.type, a.out_type, [&](auto *i, auto *o) {
            using In = std::remove_pointer_t<decltype(i)>;
            using Out = std::remove_pointer_t<decltype(o)>;
            return launch(a.cols >= 8 ? k_grad_few<In, Out, true> : k_grad_few<In, Out, false>, (uint32_t)a.count * parts + fill, kGradThreads, 0,
                          stream, a, parts, fill, fill_rows);
        });
    }
    const Plan p = plan_of(a.count, a.rows, a.cols, a.add);
    uint32_t *words = (uint32_t *)workspace;
    a.lanes = p.lanes, a.chunk = p.chunk, a.chunks = p.chunks;
    a.digit_counts = words + p.counts, a.digit_totals = words + p.totals;
    a.flags = a.add ? nullptr : (uint8_t *)(words + p.flags);
    a.partial = (float *)(words + p.partial);
    hipError_t e = hipSuccess;
    const auto then = [&](hipError_t next) {
        if (e == hipSuccess) e = next;
        return e == hipSuccess;
    };
    a.sorted = (uint2 *)(words + p.sorted[0]);
    if (a.count <= kRanked) {
        if (a.flags) {
            const uint32_t blocks = (uint32_t)std::min<uint64_t>((a.rows / 4 + 256) / 256, 4096);
            if (!then(launch(k_clear_flags, blocks, 256, 0, stream, a.flags, (uint64_t)a.rows))) return e;
            if (!then(launch(k_flag, (uint32_t)((a.count + 255) / 256), 256, 0, stream, a))) return e;
        }
        if (!then(launch(k_rank, (uint32_t)((a.count + 63) / 64), kRankThreads, 0, stream, a))) return e;
    } else {
        Digit d{};
        d.tiles = p.tiles;
        for (uint32_t pass = 0, done = 0; pass < p.passes; ++pass) {
            d.shift = done;
            d.bits = (p.bits - done + p.passes - pass - 1) / (p.passes - pass);
            done += d.bits;
            d.to = (uint2 *)(words + p.sorted[pass % 2]);
            d.set_flags = pass + 1 == p.passes ? a.flags : nullptr;
            if (!then(launch(k_count_digits, p.tiles, kSortThreads, 0, stream, a, d))) return e;
            if (!then(launch(k_sum_digits, ((1u << d.bits) + 3) / 4, 256, 0, stream, a, d))) return e;
            if (!then(launch(k_place_digits, p.tiles, kSortThreads, 0, stream, a, d))) return e;
            d.from = d.to;
        }
        a.sorted = d.to;
    }
    const uint32_t sum_blocks = p.chunks * p.parts;
    const uint32_t fill = a.add ? 0 : (uint32_t)std::min<uint64_t>(((uint64_t)a.rows * pieces + kGradThreads - 1) / kGradThreads, 1 << 16);
    const Walk walk = fill ? walk_of(a.rows, pieces, (uint64_t)fill * kGradThreads) : Walk{};
    return by_types(a.type, a.out_type, [&](auto *i, auto *o) {
        using In = std::remove_pointer_t<decltype(i)>;
        using Out = std::remove_pointer_t<decltype(o)>;
        const auto sums = a.cols >= 8 ? k_sum_runs<In, Out, true> : k_sum_runs<In, Out, false>;
        const auto join = a.cols >= 8 ? k_join_runs<Out, true> : k_join_runs<Out, false>;
        const uint32_t join_blocks = (p.chunks + kJoinChunks - 1) / kJoinChunks * p.parts;
        if (!then(launch(sums, sum_blocks + fill, kGradThreads, 0, stream, a, walk, sum_blocks))) return e;
        if (p.chunks > 1) then(launch(join, join_blocks, kGradThreads, 0, stream, a));
        return e;
    });
}

}  // namespace gv
