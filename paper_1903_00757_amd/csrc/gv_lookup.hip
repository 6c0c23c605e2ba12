// gfx950 kernels of rows by index: the rows of a table that indices name, and the gradient of that, the sums of the rows of a
// batch by index.
//
// Both are bound by memory: a row of the batch is read once and a row of the table written once.  Sums are taken in an
// order that the indices decide, never by atomics: indices are sorted (stably, so equal ones stay in the order of the batch), and
// groups of lanes go along equal pieces of the sorted batch; a run of equal indices that crosses such borders leaves a partial sum for
// each piece, which are joined by a launch of their own.
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
// Rows by index: one piece of eight columns a lane and turn.
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

// A finished sum goes to its row.
template <class Out>
__device__ __forceinline__ void put_sum(const LookupGradArgs &a, uint32_t row, uint32_t k, float (&v)[8]) {
    Out *to = (Out *)a.out + row * a.out_stride;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= a.scale;
    if (a.add) {
        float there[8];
        load_piece(to, k, a.cols, there);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there[i] + v[i];
    }
    store_piece(to, k, a.cols, v);
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

template <class In, class Out>
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
    const uint32_t lanes = a.lanes, lane = tid % lanes, groups = kGradThreads / lanes, k = 512 * part + 8 * lane;
    float sum[8] = {};
    if (k < a.cols) {
        for (uint32_t j = tid / lanes; j < all; j += 4 * groups) {
            Piece<In> p[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
                if (j + u * groups < all) p[u].load((const In *)a.grad + same[j + u * groups] * a.grad_stride, k, a.cols);
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
    if (tid < lanes && k < a.cols) put_sum<Out>(a, row, k, sum);
}

// --- the order of the places by row.  keys: the rows, sorted (`rows` for places without one, at the end); order: the places.

// Some thousand places: the place of each is how many go before it.  A workgroup of 16 waves takes 64 places, each wave a
// sixteenth of those that they are compared with.
constexpr int kRankThreads = 1024;
constexpr uint32_t kRanked = 1 << 14;

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
    a.keys[rank] = mine;
    a.order[rank] = t;
}

// Sets the flag of every row that is named.
__global__ __launch_bounds__(256) void k_flag(LookupGradArgs a) {
    for (uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x; t < a.count; t += (uint64_t)gridDim.x * 256) {
        const uint32_t row = row_at(a.index, t, a.rows);
        if (row < a.rows) a.flags[row] = 1;
    }
}
__global__ __launch_bounds__(256) void k_clear_flags(uint8_t *flags, uint64_t rows) { clear_flags(flags, rows); }

// More: digits of up to 11 bits, the lowest first; places with equal digits keep their order.  Three launches a digit: how often
// each workgroup's places have each digit, where those begin, and the places moved there.
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64, kSortSteps = 16;
constexpr uint32_t kSortTile = kSortThreads * kSortSteps, kMostDigits = 1u << 11;

struct Digit {
    const uint32_t *keys, *order;  // null: as the batch has them
    uint32_t *to_keys, *to_order;
    uint32_t shift, bits, tiles;
    uint8_t *set_flags;            // of the last digit, or null
};

__global__ __launch_bounds__(kSortThreads) void k_count_digits(LookupGradArgs a, Digit d) {
    __shared__ uint32_t counts[kMostDigits];
    const uint32_t digits = 1u << d.bits;
    for (uint32_t i = threadIdx.x; i < digits; i += kSortThreads) counts[i] = 0;
    if (!d.keys) clear_flags(a.flags, a.rows);
    __syncthreads();
    const uint64_t first = (uint64_t)blockIdx.x * kSortTile;
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const uint64_t t = first + s * kSortThreads + threadIdx.x;
        if (t >= a.count) continue;
        const uint32_t key = d.keys ? d.keys[t] : row_at(a.index, t, a.rows);
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
    // a wave takes 1024 places in a row, and counts those with the same digit before each
    uint32_t key[kSortSteps], rank[kSortSteps];
    const uint64_t first = (uint64_t)blockIdx.x * kSortTile + wave * (64 * kSortSteps) + lane;
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const uint64_t t = first + 64 * s;
        key[s] = t < a.count ? d.keys ? d.keys[t] : row_at(a.index, t, a.rows) : 0;
    }
    volatile uint16_t *mine_of = counts[wave];
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const bool there = first + 64 * s < a.count;
        const uint32_t digit = key[s] >> d.shift & (digits - 1);
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
        const uint32_t digit = key[s] >> d.shift & (digits - 1);
        const uint32_t to = base[digit] + counts[wave][digit] + rank[s];
        d.to_keys[to] = key[s];
        d.to_order[to] = d.order ? d.order[t] : (uint32_t)t;
        if (d.set_flags && key[s] < a.rows) d.set_flags[key[s]] = 1;
    }
}

// --- the sums over the sorted places

// A group of lanes goes along `chunk` sorted places.  A run of equal rows that lies within them is finished; one that goes on
// behind them leaves partial[2 c + 1] where it begins here, and partial[2 c] where it began before (whether it ends here or not).
// Workgroups behind those write zeros to the rows that are not named.
template <class In, class Out>
__global__ __launch_bounds__(kGradThreads) void k_sum_runs(LookupGradArgs a, uint32_t sum_blocks) {
    if (blockIdx.x >= sum_blocks) {
        const uint64_t pieces = (a.cols + 7) / 8;
        const uint64_t step = (uint64_t)(gridDim.x - sum_blocks) * kGradThreads;
        for (uint64_t i = (uint64_t)(blockIdx.x - sum_blocks) * kGradThreads + threadIdx.x; i < a.rows * pieces; i += step) {
            const uint64_t row = i / pieces;
            if (a.flags[row]) continue;
            const float zeros[8] = {};
            store_piece((Out *)a.out + row * a.out_stride, 8 * (uint32_t)(i % pieces), a.cols, zeros);
        }
        return;
    }
    constexpr int kAhead = 4;
    const uint32_t group = (blockIdx.x * kGradThreads + threadIdx.x) / a.lanes, lane = threadIdx.x % a.lanes;
    const uint32_t c = group % a.chunks, k = 512 * (group / a.chunks) + 8 * lane;
    if (k >= a.cols) return;
    const uint64_t first = (uint64_t)c * a.chunk, last = std::min<uint64_t>(a.count, first + a.chunk);
    if (first >= last) return;
    uint32_t key = a.keys[first];
    bool inside = first == 0 || a.keys[first - 1] != key;  // the run began here
    float sum[8] = {};
    for (uint64_t p = first; p < last; p += kAhead) {
        Piece<In> rows[kAhead];
        uint32_t next[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u >= last) continue;
            rows[u].load((const In *)a.grad + a.order[p + u] * a.grad_stride, k, a.cols);
            next[u] = p + u + 1 < a.count ? a.keys[p + u + 1] : 0xFFFFFFFFu;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u >= last) continue;
            float v[8];
            rows[u].values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
            if (next[u] != key || p + u + 1 == last) {
                if (key < a.rows) {
                    if (inside && next[u] != key) put_sum<Out>(a, key, k, sum);
                    else store_piece(a.partial + (2ull * c + (inside ? 1 : 0)) * a.cols, k, a.cols, sum);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
                key = next[u];
                inside = true;
            }
        }
    }
}

// Joins the partial sums of a run that begins among the places of c and goes on behind them.
template <class Out>
__global__ __launch_bounds__(kGradThreads) void k_join_runs(LookupGradArgs a) {
    __shared__ float scratch[kGradThreads][8];
    const uint32_t c = blockIdx.x % a.chunks;
    const uint64_t first = (uint64_t)c * a.chunk, last = first + a.chunk;
    if (last >= a.count) return;
    const uint32_t key = a.keys[last - 1];
    if (key >= a.rows || a.keys[last] != key) return;
    if (a.keys[first] == key && first > 0 && a.keys[first - 1] == key) return;
    uint32_t more = 0;  // chunks behind c that begin inside the run
    for (;;) {
        const uint64_t at = last + (uint64_t)(more + threadIdx.x) * a.chunk;
        const uint32_t some = __syncthreads_count(at < a.count && a.keys[at] == key);
        more += some;
        if (some < kGradThreads) break;
    }
    const uint32_t lanes = a.lanes, lane = threadIdx.x % lanes, groups = kGradThreads / lanes, k = 512 * (blockIdx.x / a.chunks) + 8 * lane;
    float sum[8] = {};
    if (k < a.cols) {
        for (uint32_t j = threadIdx.x / lanes; j <= more; j += 4 * groups) {  // 0: its own
            float v[4][8];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                const uint32_t at = j + u * groups;
                if (at <= more) load_piece(a.partial + (2ull * (c + at) + (at == 0 ? 1 : 0)) * a.cols, k, a.cols, v[u]);
            }
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
                if (j + u * groups <= more)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += v[u][i];
        }
    }
    join_groups(sum, scratch, lanes);
    if (threadIdx.x < lanes && k < a.cols) put_sum<Out>(a, key, k, sum);
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
    uint64_t keys[2], order[2], counts, totals, flags, partial, words;
};
constexpr uint64_t kSumLanes = 1 << 18;

Plan plan_of(uint64_t count, uint64_t rows, uint32_t cols, bool add) {
    Plan p{};
    p.lanes = lanes_of(cols);
    p.parts = (cols + 511) / 512;
    const uint64_t most = std::max<uint64_t>(1, kSumLanes / ((uint64_t)p.lanes * p.parts));
    p.chunk = (uint32_t)std::max<uint64_t>(8, (count + most - 1) / most);
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
    for (int i = 0; i < pairs; ++i) p.keys[i] = take(count), p.order[i] = take(count);
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
        const uint32_t parts = (a.cols + 511) / 512;
        // rows that a workgroup writes zeros to: 16 KB of them at least, and a thousand workgroups where that is enough
        const uint64_t each = std::max<uint64_t>(std::max<uint64_t>(1, 512 / pieces), (a.rows + 1023) / 1024);
        const uint32_t fill_rows = (uint32_t)std::min<uint64_t>(each, kFillRows);
        const uint32_t fill = a.add ? 0 : (uint32_t)std::min<uint64_t>((a.rows + fill_rows - 1) / fill_rows, 1 << 16);
        if (a.count == 0 && fill == 0) return hipSuccess;
        return by_types(a.type, a.out_type, [&](auto *i, auto *o) {
            return launch(k_grad_few<std::remove_pointer_t<decltype(i)>, std::remove_pointer_t<decltype(o)>>, (uint32_t)a.count * parts + fill,
                          kGradThreads, 0, stream, a, parts, fill, fill_rows);
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
    a.keys = words + p.keys[0], a.order = words + p.order[0];
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
            d.to_keys = words + p.keys[pass % 2], d.to_order = words + p.order[pass % 2];
            d.set_flags = pass + 1 == p.passes ? a.flags : nullptr;
            if (!then(launch(k_count_digits, p.tiles, kSortThreads, 0, stream, a, d))) return e;
            if (!then(launch(k_sum_digits, ((1u << d.bits) + 3) / 4, 256, 0, stream, a, d))) return e;
            if (!then(launch(k_place_digits, p.tiles, kSortThreads, 0, stream, a, d))) return e;
            d.keys = d.to_keys, d.order = d.to_order;
        }
        a.keys = d.to_keys, a.order = d.to_order;
    }
    const uint32_t sum_blocks = (uint32_t)(((uint64_t)p.chunks * p.parts * p.lanes + kGradThreads - 1) / kGradThreads);
    const uint32_t fill = a.add ? 0 : (uint32_t)std::min<uint64_t>((a.rows * pieces + kGradThreads - 1) / kGradThreads, 4096);
    return by_types(a.type, a.out_type, [&](auto *i, auto *o) {
        using In = std::remove_pointer_t<decltype(i)>;
        using Out = std::remove_pointer_t<decltype(o)>;
        if (!then(launch(k_sum_runs<In, Out>, sum_blocks + fill, kGradThreads, 0, stream, a, sum_blocks))) return e;
        if (p.chunks > 1) then(launch(k_join_runs<Out>, p.chunks * p.parts, kGradThreads, 0, stream, a));
        return e;
    });
}

}  // namespace gv
