// gfx950 kernels of the selection of the best rows over the scores of beams.
//
// A score s of beam b counts total[b] + (s - M) - log sum exp(s' - M), M the largest of the beam (or total[b] + s).  Within a
// beam that is the order of the scores, so one pass over them is enough: every workgroup reads a part of a beam, keeps what may
// be among its best in LDS and adds up the exponentials; a workgroup of each group joins the sums, and ranks what is left of
// the beams by what it counts.
//
// What may be among the best is told by a bound, a value that at least `best` scores seen so far reach.  The largest score of each
// thread is one of them, and in a wave the k-th largest of its lanes' takes 32 steps of a ballot: with every wave's
// ceil(best / waves)-th, the least of those is reached by `best` scores.  For scores in no special order some 1.3 `best` reach it.
// Scores that do are few, and what few there are is kept; where they are more than there is room for, as with equal scores, the
// bound is made exact by a search over the bits of (score, row), and `best` are left.
#include "gv_row_pieces.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

#include <algorithm>
#include <type_traits>

#pragma clang fp contract(off)

namespace gv {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64, kEach = 32, kPieces = kEach / 8;
constexpr uint32_t kTile = kThreads * kEach, kSlots = 2048;  // scores of a turn; candidates that LDS has room for
constexpr uint32_t kFewToRank = 256;  // each compared with all others; more are narrowed first
constexpr float kLowest = -3.402823466e38f;
static_assert(GV_MAX_BEST <= kSlots / 2, "room for the best and as many");

struct Candidate {
    float score;
    uint32_t row;
};
// What a workgroup leaves of its part.
struct Part {
    double sum;      // of exp(score - top)
    float top;       // -inf: there is no score
    float bound;     // at least `best` scores of the part reach it; -inf where that is not known
    uint32_t count;  // of its candidates
    uint32_t unused;
};

__device__ __forceinline__ float infinity() { return __builtin_inff(); }

// Numbers in the order of the floats (no NaN; -0 comes as 0).
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t bits = __float_as_uint(x + 0.0f);
    return bits ^ (bits >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order ^ (order >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
// What a score has to reach to be of interest still, when those that equal x are not: above infinity NaN, which nothing reaches and
// which then stays.  (std::max would leave it out.)
__device__ __forceinline__ float raised_above(float least, float x) {
    const float next = value_of(ordered(x) + 1);
    return next <= least ? least : next;
}

// exp(d), d <= 700, within 2^-34 of it, and 1 of 0: 2^n times 2^f, |f| <= 1/2, by a polynomial whose first number is 1 and whose
// others make the largest error the least.  What is below exp(-700) counts as that, which no sum that has a term of 1 notices.
// Fifteen instructions in fp64.  __expf takes four in fp32, but is off by up to (|d| + 1) 2^-23 of a term, and the sum of equal
// scores by as much of it: beams whose totals lie closer came in the wrong order (the call for 16 x 8 beams of 10^6 took 116 us by it, 147
// to 151 by this).
__device__ __forceinline__ double exp_of(double d) {
    constexpr double kLog2E = 1.4426950408889634, kWhole = 0x1.8p52;  // added, it leaves a whole number in the low word
    d = fmax(d, -700.0);
    const double t = fma(d, kLog2E, kWhole), f = fma(d, kLog2E, kWhole - t);
    double p = 1.519615612132076e-05;
    p = fma(p, f, 0.00015466756367126918);
    p = fma(p, f, 0.0013333935057608427);
    p = fma(p, f, 0.009618038131876797);
    p = fma(p, f, 0.05550410365988536);
    p = fma(p, f, 0.2402265106656269);
    p = fma(p, f, 0.693147180704533);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}

// The k-th largest of the kOf numbers of each of the 64 lanes (1 <= k <= 64 kOf).
template <int kOf>
__device__ __forceinline__ uint32_t kth_of_lanes(const uint32_t (&x)[kOf], uint32_t k) {
    uint32_t found = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t to = found | 1u << bit;
        uint32_t reach = 0;
#pragma unroll
        for (int i = 0; i < kOf; ++i) reach += (uint32_t)__popcll(__ballot(x[i] >= to));
        if (reach >= k) found = to;
    }
    return found;
}

// A bound that `best` of a workgroup's numbers reach: by every wave's ceil(best / waves)-th, or by the best-th of one wave.  A
// few are looked for among the threads' largest, many among all kOf numbers of each.
template <int kWavesOf, int kOf>
__device__ __forceinline__ uint32_t bound_of_threads(const uint32_t (&x)[kOf], uint32_t best, uint32_t (*scratch)[kWavesOf]) {
    const uint32_t wave = threadIdx.x / 64, each = (best + kWavesOf - 1) / kWavesOf;
    uint32_t spread = 0, alone = 0;
    if (best <= 64) {
        uint32_t largest[1] = {x[0]};
#pragma unroll
        for (int i = 1; i < kOf; ++i) largest[0] = larger(largest[0], x[i]);
        spread = kth_of_lanes(largest, each);
        alone = kth_of_lanes(largest, best);
    } else if (each <= 64 * kOf) {
        spread = kth_of_lanes(x, each);
    }
    if (threadIdx.x % 64 == 0) scratch[0][wave] = spread, scratch[1][wave] = alone;
    __syncthreads();
    uint32_t least = 0xFFFFFFFFu, most = 0;
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) {
        least = std::min(least, scratch[0][w]);
        most = std::max(most, scratch[1][w]);
    }
    __syncthreads();
    return std::max(least, most);
}

template <int kOf>
__device__ __forceinline__ double block_sum(double x, double *scratch) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = x;
    __syncthreads();
    double all = 0;
#pragma unroll
    for (int w = 0; w < kOf; ++w) all += scratch[w];
    __syncthreads();
    return all;
}
template <int kOf>
__device__ __forceinline__ uint32_t block_largest(uint32_t x, uint32_t *scratch) {
    x = largest_of_lanes<64>(x);
    if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = x;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kOf; ++w) all = larger(all, scratch[w]);
    __syncthreads();
    return all;
}


__device__ __forceinline__ uint64_t key_of(float score, uint32_t row) { return (uint64_t)ordered(score) << 32 | (0xFFFFFFFFu - row); }

// This thread's scores of a turn from row `first` on; what is not there, and NaN, as -inf.
template <class T>
__device__ __forceinline__ void load_turn(const T *scores, uint32_t first, uint32_t end, float (&v)[kEach]) {
    const uint32_t row = first + 8 * threadIdx.x;  // and so on in every quarter of the turn
    Piece<T> p[kPieces];
    if (first + kTile <= end) {
#pragma unroll
        for (int h = 0; h < kPieces; ++h) __builtin_memcpy(&p[h], scores + row + h * (kTile / kPieces), sizeof p[h]);
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = fmaxf((float)p[i / 8].at[i % 8], -infinity());
    } else {
#pragma unroll
        for (int h = 0; h < kPieces; ++h) p[h].load(scores, row + h * (kTile / kPieces), end);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            v[i] = row + (i / 8) * (kTile / kPieces) + i % 8 < end ? fmaxf((float)p[i / 8].at[i % 8], -infinity()) : -infinity();
    }
}

template <int kWavesOf>
struct SearchShared {
    uint64_t some, differ[kWavesOf];
    uint32_t reach[2][kWavesOf];
};
// How many of a workgroup's conditions hold.
template <int kWavesOf, int kOf>
__device__ __forceinline__ uint32_t block_count(const bool (&x)[kOf], uint32_t (&scratch)[kWavesOf]) {
    uint32_t own = 0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) own += (uint32_t)__popcll(__ballot(x[i]));
    if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = own;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) all += scratch[w];
    return all;
}
// A number that exactly the k largest of a workgroup's reach, unless several equal the k-th: then that.  0 is none; there are k
// others.
template <int kWavesOf, int kOf>
__device__ __forceinline__ uint64_t block_kth(const uint64_t (&x)[kOf], uint32_t k, SearchShared<kWavesOf> &s) {
    uint64_t one = 0, differ = 0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) one = x[i] ? x[i] : one;
    if (one) s.some = one;  // whichever of them: bits that all share need no look
    __syncthreads();
    one = s.some;
#pragma unroll
    for (int i = 0; i < kOf; ++i) differ |= x[i] ? x[i] ^ one : 0;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) differ |= __shfl_xor(differ, d);
    if (threadIdx.x % 64 == 0) s.differ[threadIdx.x / 64] = differ;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) differ |= s.differ[w];
    const int bits = differ ? 64 - __builtin_clzll(differ) : 0;
    uint64_t found = bits == 64 ? 0 : one >> bits << bits;
#pragma unroll 1
    for (int bit = bits - 1; bit >= 0; --bit) {
        const uint64_t to = found | 1ull << bit;
        bool reach[kOf];
#pragma unroll
        for (int i = 0; i < kOf; ++i) reach[i] = x[i] >= to;
        const uint32_t all = block_count(reach, s.reach[bit % 2]);
        if (all >= k) found = to;
        if (all == k) break;
    }
    __syncthreads();
    return found;
}

struct Shared {
    Candidate kept[kSlots];
    uint32_t count, waves[2][kWaves];
    double sums[kWaves];
    SearchShared<kWaves> search;
};

// Leaves the `best` first of the n kept (at least as many); returns a score that they reach.
__device__ __forceinline__ float narrow(Shared &s, uint32_t n, uint32_t best) {
    constexpr int kOwn = kSlots / kThreads;
    uint64_t own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const uint32_t at = threadIdx.x + i * kThreads;
        own[i] = at < n ? key_of(s.kept[at].score, s.kept[at].row) : 0;
    }
    const uint64_t found = block_kth(own, best, s.search);
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
        if (own[i] >= found && own[i]) s.kept[atomicAdd(&s.count, 1u)] = {value_of((uint32_t)(own[i] >> 32)), 0xFFFFFFFFu - (uint32_t)own[i]};
    __syncthreads();
    return value_of((uint32_t)(found >> 32));
}

// A turn with more candidates than there is room for: `kept` of the turns before, and the turn's scores that reach `least`, two
// of each thread at a time, narrowed whenever the next may not fit.  Returns how many are kept; `bound` is raised to what
// `best` of them reach.
template <class T>
__device__ __forceinline__ uint32_t take_slowly(Shared &s, uint32_t kept, uint32_t best, const T *scores, uint32_t first, uint32_t end, float least,
                                                float &bound) {
    if (threadIdx.x == 0) s.count = kept;
    __syncthreads();
#pragma unroll 1
    for (int i = kEach - 2; i >= 0; i -= 2) {  // the last first: scores that rise are done with soonest
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const uint32_t row = first + 8 * threadIdx.x + i / 8 * (kTile / kPieces) + i % 8 + o;
            const float x = row < end ? (float)scores[row] : -infinity();
            if (x >= least) s.kept[atomicAdd(&s.count, 1u)] = {x, row};
        }
        __syncthreads();
        kept = s.count;
        __syncthreads();
        if (kept + 2 * kThreads > kSlots) {
            bound = std::max(bound, narrow(s, kept, best));
            least = std::max(least, bound);
            kept = best;
        }
    }
    return kept;
}
static_assert(GV_MAX_BEST + 2 * kThreads <= kSlots, "narrowed, the next fit");

__device__ __forceinline__ bool offers(const SelectArgs &a, uint64_t beam, float &total) {
    total = a.totals ? a.totals[beam] : 0.0f;
    return fabsf(total) < infinity();
}

// What a score counts beyond its beam's total: at most 0, as what is counted from may lie below the largest score and the sum is rounded.
__device__ __forceinline__ double log_of(float score, float top, double log_sum) {
    return fmin((score == top ? 0.0 : (double)score - (double)top) - log_sum, 0.0);
}

__device__ __forceinline__ void put_none(const SelectArgs &a, uint64_t group, uint32_t rank) {
    const uint64_t at = group * a.best + rank;
    a.parent[at] = -1;
    a.row[at] = -1;
    a.total[at] = -infinity();
}
// What a rank goes to; what counts -inf (finite scores beside infinity) goes behind all others, and is nothing.
__device__ __forceinline__ void put(const SelectArgs &a, uint64_t group, uint32_t rank, uint64_t parent, uint32_t row, double total) {
    if (total == -infinity()) return put_none(a, group, rank);
    const uint64_t at = group * a.best + rank;
    a.parent[at] = (int64_t)parent;
    a.row[at] = row;
    a.total[at] = (float)total;
}

// One part of one beam.  kAlone: groups of one beam in one part are finished here.  64 x 10^6 floats, best 1: 43 us, 6 TB/s;
// best 100: 60, for the search of the bound and the candidates of the first turns; 128 x 10^6 with softmax 139 us, for the
// exponentials in fp64.
template <class T, bool kLog, bool kAlone>
__global__ __launch_bounds__(kThreads, 4) void k_select_parts(SelectArgs a) {
    __shared__ Shared s;
    const uint64_t beam = blockIdx.x / a.parts;
    const uint32_t part = blockIdx.x % a.parts, tid = threadIdx.x;
    const uint64_t begin = (uint64_t)part * a.part_rows;
    const uint32_t end = (uint32_t)std::min<uint64_t>(a.rows, begin + a.part_rows);
    float base;
    const bool some = offers(a, beam, base), ended = some && a.done && a.done[beam];
    Part *to = (Part *)a.summaries + beam * a.parts + part;
    if (!some || ended) {
        if constexpr (kAlone) {
            for (uint32_t r = tid; r < a.best; r += kThreads) {
                if (ended && r == 0) put(a, beam, 0, beam, a.end, base);
                else put_none(a, beam, r);
            }
        } else if (tid == 0) {
            *to = Part{0.0, -infinity(), -infinity(), 0, 0};
        }
        return;
    }
    if (tid == 0) s.count = 0;
    __syncthreads();
    const T *scores = (const T *)a.scores + beam * a.stride;
    float bound = -infinity(), least = kLowest, top = -infinity();
    float largest[kPieces];  // so far, of each piece's places
#pragma unroll
    for (int h = 0; h < kPieces; ++h) largest[h] = -infinity();
    double sum = 0.0;
    uint32_t kept = 0, turn = 0;
    for (uint64_t first = begin; first < end; first += kTile, ++turn) {
        const uint32_t row = (uint32_t)first + 8 * tid;  // and so on in every quarter of the turn
        float v[kEach];
        load_turn(scores, (uint32_t)first, end, v);
        float most = -infinity();
#pragma unroll
        for (int h = 0; h < kPieces; ++h) {
            float some = v[8 * h];
#pragma unroll
            for (int i = 1; i < 8; ++i) some = fmaxf(some, v[8 * h + i]);
            largest[h] = fmaxf(largest[h], some);
            most = fmaxf(most, some);
        }
        if constexpr (kLog) {
            // exponentials of differences from a score of this thread that is not far below its largest
            if (most > top + 20.0f || top == -infinity()) {
                if (most > top) {
                    sum = top == -infinity() || most == infinity() ? 0.0 : sum * exp_of((double)top - (double)most);
                    top = most;
                }
            }
            double terms[2] = {};
            if (top < infinity()) {
                const double from = top == -infinity() ? 0.0 : (double)top;
#pragma unroll
                for (int i = 0; i < kEach; ++i) terms[i % 2] += exp_of((double)v[i] - from);
            } else {  // scores of infinity share everything
#pragma unroll
                for (int i = 0; i < kEach; ++i) terms[i % 2] += v[i] == infinity() ? 1.0 : 0.0;
            }
            sum += terms[0] + terms[1];
        }
        if ((turn & (turn + 1)) == 0 || first + kTile >= end) {  // turns 0, 1, 3, 7, ..., and the last
            uint32_t order[kPieces];
#pragma unroll
            for (int h = 0; h < kPieces; ++h) order[h] = ordered(largest[h]);
            const uint32_t found = bound_of_threads<kWaves>(order, a.best, s.waves);
            if (found > ordered(-infinity()) && value_of(found) > bound) {
                // scores that are kept may lie below it; of those in later turns, equal ones come behind
                bound = value_of(found);
                least = std::max(least, bound);
            }
        }
        bool full = false;
        if (most >= least) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (!(v[i] >= least)) continue;
                const uint32_t at = atomicAdd(&s.count, 1u);
                if (at < kSlots) s.kept[at] = {v[i], row + (i / 8) * (kTile / kPieces) + i % 8};
                else full = true;
            }
        }
        if (__syncthreads_or(full)) {
            if (kept >= a.best) {  // scores that equal the last of those come behind
                bound = std::max(bound, narrow(s, kept, a.best));
                least = raised_above(least, bound);
                kept = a.best;
            }
            kept = take_slowly(s, kept, a.best, scores, (uint32_t)first, end, least, bound);
        } else {
            kept = s.count;
        }
        if (kept >= a.best && bound > -infinity()) least = raised_above(least, bound);
        __syncthreads();
    }
    double log_sum = 0.0;
    float all_top = 0.0f;
    if constexpr (kLog) {
        const uint32_t found = block_largest<kWaves>(ordered(top), s.waves[0]);
        all_top = value_of(found);
        const double mine = top == -infinity() || (all_top == infinity() && top < all_top) ? 0.0
                            : top == all_top ? sum : sum * exp((double)top - (double)all_top);
        log_sum = block_sum<kWaves>(mine, s.sums);
    }
    const uint32_t most_kept = kAlone ? std::max(a.best, kFewToRank) : a.slots;
    if (kept > most_kept) {
        bound = narrow(s, kept, a.best);
        kept = a.best;
    }
    if constexpr (kAlone) {
        log_sum = log(log_sum);
        for (uint32_t i = tid; i < kept; i += kThreads) {
            const uint64_t key = key_of(s.kept[i].score, s.kept[i].row);
            uint32_t rank = 0;
            for (uint32_t j = 0; j < kept; ++j) rank += key_of(s.kept[j].score, s.kept[j].row) > key;
            if (rank >= a.best) continue;
            const float score = s.kept[i].score;
            const double total = (double)base + (kLog ? log_of(score, all_top, log_sum) : (double)score);
            put(a, beam, rank, beam, s.kept[i].row, total);
        }
        for (uint32_t r = kept + tid; r < a.best; r += kThreads) put_none(a, beam, r);
    } else {
        Candidate *out = (Candidate *)a.candidates + (beam * a.parts + part) * a.slots;
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        for (uint32_t i = tid; i < kept; i += kThreads) {
            const Candidate c = s.kept[i];
            if (c.score >= bound) out[atomicAdd(&s.count, 1u)] = c;  // some were kept before the bound rose
        }
        __syncthreads();
        if (tid == 0) *to = Part{log_sum, all_top, bound, s.count, 0};
    }
}

// --- the beams of a group joined: one workgroup for each, as long as its few dependent loads and searches take (11 to 24 us)
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64;
constexpr uint32_t kJoinSlots = 2 * kJoinThreads, kMostLists = 2048, kMostBeams = GV_MAX_BEAMS;
static_assert(GV_MAX_BEST + kJoinThreads <= kJoinSlots, "room for the best and a turn");

struct JoinShared {
    double total[kJoinSlots];
    float score[kJoinSlots];
    uint32_t row[kJoinSlots], beam[kJoinSlots];
    uint32_t ends[kMostLists];  // of the lists, counted together
    double log_sum[kMostBeams];
    float top[kMostBeams], base[kMostBeams];
    uint32_t count, waves[2][kJoinWaves];
    SearchShared<kJoinWaves> search;
};

__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t bits = (uint64_t)__double_as_longlong(x + 0.0);
    return bits ^ (bits >> 63 ? ~0ull : 1ull << 63);
}

// Leaves the `best` first of n candidates (n > best): by total; of those that equal the last one by beam and score; of those by
// row.
__device__ __forceinline__ void narrow(JoinShared &s, uint32_t n, uint32_t best) {
    double total[2];
    float score[2];
    uint32_t row[2], beam[2];
    uint64_t key[2];
    bool stays[2], above[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t i = threadIdx.x + h * kJoinThreads;
        key[h] = 0;
        if (i < n) total[h] = s.total[i], score[h] = s.score[i], row[h] = s.row[i], beam[h] = s.beam[i], key[h] = ordered(total[h]);
        stays[h] = false;
    }
    uint32_t need = best;
#pragma unroll
    for (int round = 0; round < 3; ++round) {
        const uint64_t found = block_kth(key, need, s.search);
#pragma unroll
        for (int h = 0; h < 2; ++h) above[h] = key[h] > found;
        const uint32_t more = block_count(above, s.search.reach[0]);
        bool reach[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) reach[h] = key[h] >= found && key[h];
        const uint32_t all = block_count(reach, s.search.reach[1]);
        __syncthreads();
        // all that reach it, where those are as many as are asked for; else those above, and the others by what comes next
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            stays[h] |= all == need ? reach[h] : above[h];
            const bool open = all > need && key[h] == found;
            key[h] = !open ? 0 : round == 0 ? (uint64_t)(0xFFFFFFFFu - beam[h]) << 32 | ordered(score[h]) : 0xFFFFFFFFu - row[h];
        }
        if (all == need) break;
        need -= more;
    }
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (!stays[h]) continue;
        const uint32_t to = atomicAdd(&s.count, 1u);
        s.total[to] = total[h], s.score[to] = score[h], s.row[to] = row[h], s.beam[to] = beam[h];
    }
    __syncthreads();
}


// How many of n candidates go before candidate i: by total, beam, score and row.
__device__ __forceinline__ uint32_t rank_of(const JoinShared &s, uint32_t i, uint32_t n) {
    const double total = s.total[i];
    uint32_t rank = 0, equal = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < n; ++j) {
        const double other = s.total[j];
        rank += other > total;
        equal += other == total;
    }
    if (equal > 1) {
        const uint32_t beam = s.beam[i], row = s.row[i];
        const float score = s.score[i];
        for (uint32_t j = 0; j < n; ++j) {
            if (s.total[j] != total || j == i) continue;
            rank += s.beam[j] != beam ? s.beam[j] < beam : s.score[j] != score ? s.score[j] > score : s.row[j] < row;
        }
    }
    return rank;
}

template <bool kLog>
__global__ __launch_bounds__(kJoinThreads) void k_select_join(SelectArgs a) {
    __shared__ JoinShared s;
    const uint32_t tid = threadIdx.x, lane = tid % 64, wave = tid / 64, lists = a.beams * a.parts;
    const uint64_t group = blockIdx.x, first_beam = group * a.beams;
    const Part *parts = (const Part *)a.summaries + first_beam * a.parts;
    const Candidate *candidates = (const Candidate *)a.candidates + first_beam * a.parts * a.slots;
    if (tid == 0) s.count = 0;
    // what the scores of each beam count from
    for (uint32_t beam = wave; beam < a.beams; beam += kJoinWaves) {
        float base;
        const bool some = offers(a, first_beam + beam, base);
        if (lane == 0) s.base[beam] = some ? base : -infinity();
        if constexpr (kLog) {
            uint32_t top = 0;
            for (uint32_t p = lane; p < a.parts; p += 64) top = larger(top, ordered(parts[beam * a.parts + p].top));
            top = largest_of_lanes<64>(top);
            const float all = value_of(top);
            double sum = 0.0;
            if (top > ordered(-infinity()))
                for (uint32_t p = lane; p < a.parts; p += 64) {
                    const Part part = parts[beam * a.parts + p];
                    if (part.top == all) sum += part.sum;
                    else if (all < infinity() && part.top > -infinity()) sum += part.sum * exp((double)part.top - (double)all);
                }
#pragma unroll
            for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
            if (lane == 0) s.top[beam] = all, s.log_sum[beam] = log(sum);
        }
    }
    // where each list ends
    uint32_t mine[kMostLists / kJoinThreads], upto = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMostLists / kJoinThreads; ++i) {
        const uint32_t list = tid * (kMostLists / kJoinThreads) + i;
        mine[i] = list < lists ? parts[list].count : 0;
        upto += mine[i];
    }
    const uint32_t own = upto;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = __shfl_up(upto, d);
        if (lane >= (uint32_t)d) upto += other;
    }
    if (lane == 63) s.waves[0][wave] = upto;
    __syncthreads();
    uint32_t all = 0, at = upto - own;
#pragma unroll
    for (uint32_t w = 0; w < kJoinWaves; ++w) {
        at += w < wave ? s.waves[0][w] : 0;
        all += s.waves[0][w];
    }
#pragma unroll
    for (uint32_t i = 0; i < kMostLists / kJoinThreads; ++i) {
        at += mine[i];
        s.ends[tid * (kMostLists / kJoinThreads) + i] = at;
    }
    __syncthreads();
    const auto total_of = [&](uint32_t beam, float score) {
        const double base = (double)s.base[beam];
        return base + (kLog ? log_of(score, s.top[beam], s.log_sum[beam]) : (double)score);
    };
    const auto take = [&](uint32_t i, uint32_t &beam, Candidate &c) {
        uint32_t lo = 0, hi = lists - 1;  // the first list that ends behind i
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (s.ends[mid] > i) hi = mid;
            else lo = mid + 1;
        }
        beam = lo / a.parts;
        c = candidates[(uint64_t)lo * a.slots + (i - (lo ? s.ends[lo - 1] : 0))];
        return total_of(beam, c.score);
    };
    // Candidates are read once, as far as registers hold them: four a thread, asked for together.
    constexpr uint32_t kHeld = 4;
    double held_total[kHeld];
    Candidate held[kHeld];
    uint32_t held_beam[kHeld];
    double largest = -infinity();
#pragma unroll
    for (uint32_t h = 0; h < kHeld; ++h) {
        held_total[h] = -infinity();
        if (tid + h * kJoinThreads < all) held_total[h] = take(tid + h * kJoinThreads, held_beam[h], held[h]);
    }
    // a bound of the totals, as in a part
    double bound = -infinity();
    if (all > 2 * a.best) {
        for (uint32_t i = tid + kHeld * kJoinThreads; i < all; i += kJoinThreads) {
            uint32_t beam;
            Candidate c;
            largest = fmax(largest, take(i, beam, c));
        }
        const uint32_t order[kHeld] = {ordered((float)fmax(largest, held_total[0])), ordered((float)held_total[1]), ordered((float)held_total[2]),
                                       ordered((float)held_total[3])};
        const uint32_t found = bound_of_threads<kJoinWaves>(order, a.best, s.waves);
        // the float nearest to a total may lie above it: the one below does not
        if (found > ordered(kLowest)) bound = (double)value_of(found - 1);
    }
    const auto keep = [&](double total, uint32_t beam, float score, uint32_t row) {
        const uint32_t to = atomicAdd(&s.count, 1u);
        if (to >= kJoinSlots) return true;
        s.total[to] = total, s.beam[to] = beam, s.score[to] = score, s.row[to] = row;
        return false;
    };
    bool full = false;
    for (uint32_t beam = tid; a.done && beam < a.beams; beam += kJoinThreads)
        if (a.done[first_beam + beam] && s.base[beam] > -infinity() && (double)s.base[beam] >= bound)
            full |= keep((double)s.base[beam], beam, infinity(), a.end);
#pragma unroll
    for (uint32_t h = 0; h < kHeld; ++h)
        if (tid + h * kJoinThreads < all && held_total[h] >= bound) full |= keep(held_total[h], held_beam[h], held[h].score, held[h].row);
    for (uint32_t i = tid + kHeld * kJoinThreads; i < all; i += kJoinThreads) {
        uint32_t beam;
        Candidate c;
        const double total = take(i, beam, c);
        if (total >= bound) full |= keep(total, beam, c.score, c.row);
    }
    uint32_t n;
    if (__syncthreads_or(full)) {
        // more than there is room for: a turn at a time, and the best are left whenever the next may not fit
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        n = 0;
        const uint32_t ended = a.done ? a.beams : 0;
        for (uint32_t from = 0; from < ended + all; from += kJoinThreads) {
            if (n + kJoinThreads > kJoinSlots) {
                if (n > a.best) narrow(s, n, a.best);
                if (n >= a.best) {
                    double least = infinity();
                    for (uint32_t i = lane; i < a.best; i += 64) least = fmin(least, s.total[i]);
#pragma unroll
                    for (int d = 32; d > 0; d /= 2) least = fmin(least, __shfl_xor(least, d));
                    bound = fmax(bound, least);
                }
            }
            const uint32_t i = from + tid;
            if (i < ended) {
                if (a.done[first_beam + i] && s.base[i] > -infinity() && (double)s.base[i] >= bound)
                    (void)keep((double)s.base[i], i, infinity(), a.end);
            } else if (i < ended + all) {
                uint32_t beam;
                Candidate c;
                const double total = take(i - ended, beam, c);
                if (total >= bound) (void)keep(total, beam, c.score, c.row);
            }
            __syncthreads();
            n = s.count;
            __syncthreads();
        }
    } else {
        n = s.count;
    }
    if (n > std::max(a.best, kFewToRank)) {
        narrow(s, n, a.best);
        n = a.best;
    }
    for (uint32_t i = tid; i < n; i += kJoinThreads) {
        const uint32_t rank = rank_of(s, i, n);
        if (rank < a.best) put(a, group, rank, first_beam + s.beam[i], s.row[i], s.total[i]);
    }
    for (uint32_t r = n + tid; r < a.best; r += kJoinThreads) put_none(a, group, r);
}

// How scores are cut: parts of whole turns, so many that a thousand workgroups are at work, but no more than leave the join
// with candidates that its registers hold (some 1.3 `best` a part; one query, 4 x 10^6 scores, best 100: 245 parts took 99 us),
// as far as the chip is filled once.
struct Cut {
    uint32_t parts, part_rows, slots;
    bool alone;
};
Cut cut_of(uint64_t queries, uint64_t rows, uint32_t beams, uint32_t best) {
    constexpr uint64_t kWanted = 1024;
    const uint64_t tiles = std::max<uint64_t>(1, (rows + kTile - 1) / kTile);
    uint64_t parts = std::min<uint64_t>(tiles, std::max<uint64_t>(1, kWanted / queries));
    const uint64_t held = 3 * kJoinThreads / ((uint64_t)best * beams), filled = std::min<uint64_t>(32, kWanted / 2 / queries);
    parts = std::min<uint64_t>(parts, std::max<uint64_t>({1, held, filled}));
    parts = std::min<uint64_t>(parts, kMostLists / beams);
    const uint64_t each = (tiles + parts - 1) / parts;
    parts = (tiles + each - 1) / each;
    return {(uint32_t)parts, (uint32_t)(each * kTile), std::min<uint32_t>(kSlots, 512 + 4 * best), beams == 1 && parts == 1};
}

uint64_t summaries_of(uint64_t queries, const Cut &c) { return (queries * c.parts * sizeof(Part) + 15) & ~15ull; }

}  // namespace

uint64_t select_workspace(uint64_t queries, uint64_t rows, uint32_t beams, uint32_t best) {
    if (queries == 0) return 0;
    const Cut c = cut_of(queries, rows, beams, best);
    return c.alone ? 0 : summaries_of(queries, c) + queries * c.parts * c.slots * sizeof(Candidate);
}

hipError_t launch_select(const SelectArgs &args, void *workspace, hipStream_t stream) {
    SelectArgs a = args;
    const Cut c = cut_of(a.queries, a.rows, a.beams, a.best);
    a.parts = c.parts, a.part_rows = c.part_rows, a.slots = c.slots;
    a.summaries = workspace;
    a.candidates = (char *)workspace + summaries_of(a.queries, c);
    const uint32_t blocks = (uint32_t)(a.queries * c.parts);
    const auto first = [&](auto type) {
        using T = decltype(type);
        if (c.alone) {
            return a.log_softmax ? launch(k_select_parts<T, true, true>, blocks, kThreads, 0, stream, a)
                                 : launch(k_select_parts<T, false, true>, blocks, kThreads, 0, stream, a);
        }
        return a.log_softmax ? launch(k_select_parts<T, true, false>, blocks, kThreads, 0, stream, a)
                             : launch(k_select_parts<T, false, false>, blocks, kThreads, 0, stream, a);
    };
    const hipError_t e = a.type == GV_F32 ? first(float()) : a.type == GV_BF16 ? first(__bf16()) : first(_Float16());
    if (e != hipSuccess || c.alone) return e;
    const uint32_t groups = (uint32_t)(a.queries / a.beams);
    return a.log_softmax ? launch(k_select_join<true>, groups, kJoinThreads, 0, stream, a)
                         : launch(k_select_join<false>, groups, kJoinThreads, 0, stream, a);
}

}  // namespace gv
