// Log probabilities of given columns, entropy and alternatives of rows of scores, from one read of the scores.
#pragma once

#include "regot_rows.hpp"

namespace regot {

struct RowArgs {
    int64_t n;
    uint32_t m;
    const void *S;
    int64_t ldS;
    const float *bias;
    float inv_eta, log2_scale;  // 1 / eta, log2(e) / eta
    const int32_t *target;
    int targets, k;
    float *logprob, *entropy, *stats;
    int32_t *top_idx;
    float *top_logprob;
    // a row is cut into slices of kSlice columns, `block` of them a block; a workgroup takes part_blocks blocks of a row.
    // What the parts of rows found is in the workspace.
    int block, block_log2, blocks, scan_log2, parts, part_blocks;  // (block: a power of two; 1 << scan_log2 is not below blocks)
    uint32_t part_columns;
    float *part_sums;       // [n][parts][3]
    float *part_max;        // [n][blocks][kThreads]
    // gradient
    const float *stats_in, *entropy_in, *g_logprob, *g_entropy;
    void *dS;
    int64_t ldD;
    // distillation
    const float *t_score, *row_weight;
    float *loss;
};

constexpr int kGroup = 16;                    // scores a lane works on at a time
constexpr uint32_t kSlice = kThreads * kGroup;  // columns of a row that a workgroup works on at a time
constexpr int kWholeBlocks = 16;              // blocks of a row that one workgroup reads
constexpr int kPartBlocks = 32;               // of one that several do, at most
constexpr int kList = 512;                    // blocks, and columns, that may hold the best k

// A column and its score as one number: larger for what comes first among a row's alternatives.  0 is none.
__device__ __forceinline__ uint64_t alternative(float x, uint32_t column) { return (uint64_t)ordered(x + 0.f) << 32 | (uint32_t)~column; }
__device__ __forceinline__ float score_of(uint64_t a) { return from_ordered((uint32_t)(a >> 32)); }
__device__ __forceinline__ uint32_t column_of(uint64_t a) { return ~(uint32_t)a; }
constexpr uint64_t kForbidden = (uint64_t)0x007fffffu << 32 | 0xffffffffu;  // (-inf, column 0)

// The k-th largest of COUNT scores a lane over the wave, its low 16 bits cut off: k of them are not below it; -inf if there
// are fewer than k above that.
template <int COUNT>
__device__ __forceinline__ float kth_largest_bound(const float (&x)[COUNT], int k)
{
    uint32_t p[COUNT], t = 0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) p[i] = ordered(x[i]) >> 16;
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t c = t | 1u << bit;
        int have = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) have += __builtin_popcountll(__ballot(p[i] >= c));
        if (have >= k) t = c;
    }
    return t > 0x007fu ? from_ordered(t << 16) : -kInf;
}

// The same for few: the k-th largest of one score a lane (k <= 64), by counting for each lane those above its own.  About 800
// cycles, where the 16 rounds above, one after the other, are about 3700 for four scores a lane.
constexpr int kFew = 32;
__device__ __forceinline__ float kth_largest_few(float x, int k)
{
    int above = 0;
#pragma unroll
    for (int l = 0; l < kLanes; ++l) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)) > x;
    return -wave_all<OpMaxF>(above < k ? -x : -kInf);
}

// Ranks `count` different alternatives by comparing each with all: place(rank, alternative) for those among the first k.
// The list has kRankPad entries of room behind them.
constexpr int kRankPad = 8;
template <typename F>
__device__ __forceinline__ void rank_all(const uint64_t *list, int count, int thread, int threads, int k, F place)
{
    for (int i = thread; i < count; i += threads) {
        const uint64_t mine = list[i];
        int rank = 0;
        for (int o = 0; o < count; o += kRankPad) {
            uint64_t v[kRankPad];
#pragma unroll
            for (int q = 0; q < kRankPad; ++q) v[q] = list[o + q];
#pragma unroll
            for (int q = 0; q < kRankPad; ++q) rank += v[q] > mine && o + q < count;
        }
        if (rank < k) place(rank, mine);
    }
}

// What is written of a row once its sums are known.
struct RowOut {
    const RowArgs &A;
    int64_t row;
    bool none, bad;
    float max, log_sum;
    __device__ __forceinline__ RowOut(const RowArgs &A_, int64_t row_, const Softmax &soft, bool first) : A(A_), row(row_), none(soft.none()), bad(soft.bad())
    {
        max = bad ? kNan : soft.max;
        log_sum = bad ? kNan : soft.log_sum();
        if (first) {
            if (A.stats) {
                A.stats[2 * row] = max;
                A.stats[2 * row + 1] = log_sum;
            }
            if (A.entropy) A.entropy[row] = bad ? kNan : soft.entropy();
        }
    }
    __device__ __forceinline__ float logprob(float x) const { return none ? -kInf : (x - max) * A.inv_eta - log_sum; }
    __device__ __forceinline__ void top(int rank, uint64_t a) const
    {
        A.top_idx[row * A.k + rank] = (int32_t)column_of(a);
        A.top_logprob[row * A.k + rank] = logprob(score_of(a));
    }
    __device__ __forceinline__ void no_top(int rank) const
    {
        A.top_idx[row * A.k + rank] = -1;
        A.top_logprob[row * A.k + rank] = bad ? kNan : -kInf;
    }
};

// The scores of one row.
template <int TYPE, bool BIAS>
struct RowScores {
    using T = Score<TYPE>;
    using Chunk = typename T::Chunk;
    static constexpr int kGroupVecs = kGroup / T::kVec;
    const typename T::Raw *S;
    const float *bias;
    uint32_t m;
    __device__ __forceinline__ RowScores(const RowArgs &A, int64_t row) : S(static_cast<const typename T::Raw *>(A.S) + row * A.ldS), bias(A.bias), m(A.m) {}
    __device__ __forceinline__ float operator()(uint32_t j) const
    {
        const float v = T::get(S[j]);
        return BIAS ? v + bias[j] : v;
    }
    template <bool ONCE>
    __device__ __forceinline__ Chunk ask(uint32_t j) const { return Span<TYPE>(j, m).template load<ONCE>(S); }
    __device__ __forceinline__ void unpack(Chunk chunk, uint32_t j, float *x) const
    {
        const Span<TYPE> span(j, m);
        T::unpack(chunk, x);
        if constexpr (BIAS) span.add_bias(x, bias);
        span.mask(x);
    }
    // the same with the bias that was asked for beside the chunk (b: nothing without a bias)
    __device__ __forceinline__ void ask_bias(uint32_t j, float *b) const
    {
        if constexpr (BIAS) Span<TYPE>(j, m).load_bias(b, bias);
    }
    __device__ __forceinline__ void unpack(Chunk chunk, const float *b, uint32_t j, float *x) const
    {
        T::unpack(chunk, x);
        if constexpr (BIAS) {
#pragma unroll
            for (int e = 0; e < T::kVec; ++e) x[e] += b[e];
        }
        Span<TYPE>(j, m).mask(x);
    }
    __device__ __forceinline__ void read(uint32_t j, float *x) const { unpack(ask<false>(j), j, x); }
};

// The given columns' log probabilities.  The first one of each thread is asked for before the row is read.
template <int TYPE, bool BIAS>
struct Given {
    int column = -1;
    float x = 0.f;
    __device__ __forceinline__ void ask(const RowArgs &A, int64_t row, const RowScores<TYPE, BIAS> &scores, int t)
    {
        if (t >= A.targets) return;
        column = A.target[row * A.targets + t];
        if ((uint32_t)column < A.m) x = scores((uint32_t)column);
    }
    __device__ __forceinline__ void tell(const RowArgs &A, const RowOut &out, const RowScores<TYPE, BIAS> &scores, int thread, int threads)
    {
        for (int t = thread; t < A.targets; t += threads) {
            if (t != thread) ask(A, out.row, scores, t);
            A.logprob[out.row * A.targets + t] = (uint32_t)column < A.m ? out.logprob(x) : 0.f;
        }
    }
};

// The best of a thread's columns (the 16 bytes number thread, thread + threads, ... of the row) that comes behind `last`; 0: none.
template <int TYPE, bool BIAS>
__device__ __forceinline__ uint64_t best_before(const RowScores<TYPE, BIAS> &scores, uint64_t last, int thread, int threads)
{
    using T = Score<TYPE>;
    uint64_t best = 0;
    for (uint32_t j = thread * T::kVec; j < scores.m; j += threads * T::kVec) {
        float x[T::kVec];
        scores.read(j, x);
        const uint32_t first = Span<TYPE>(j, scores.m).first;
#pragma unroll
        for (int e = 0; e < T::kVec; ++e) {
            const uint64_t a = alternative(x[e], first + e);
            if (a < last && a > best && a > kForbidden) best = a;
        }
    }
    return best;
}

// push(a) for each of a thread's columns that does not come behind `bound`.
template <int TYPE, bool BIAS, typename F>
__device__ __forceinline__ void each_from(const RowScores<TYPE, BIAS> &scores, uint64_t bound, int thread, int threads, F push)
{
    using T = Score<TYPE>;
    const float least = score_of(bound);
    for (uint32_t j = thread * T::kVec; j < scores.m; j += threads * T::kVec) {
        float x[T::kVec];
        scores.read(j, x);
        if (!(largest(x) >= least)) continue;
        const uint32_t first = Span<TYPE>(j, scores.m).first;
#pragma unroll
        for (int e = 0; e < T::kVec; ++e) {
            const uint64_t a = alternative(x[e], first + e);
            if (a >= bound && a > kForbidden) push(a);
        }
    }
}

// The k best of a row of at most VECS loads a lane, by a wave: the k-th largest by bisection over the scores in their order, two
// bits a round, each round counting over the row again (from the caches, so that no registers are held for it): 16 bits
// first, the rest if more than HELD columns are still in, then over the columns that have the score that all k are at or above.
// push(is, a) is called by all lanes at once, for at most HELD columns in all, the k best among them.
template <int HELD, int VECS, int TYPE, bool BIAS, typename F>
__device__ __forceinline__ void best_by_bisection(const RowScores<TYPE, BIAS> &scores, int k, uint32_t at, F push)
{
    using T = Score<TYPE>;
    constexpr uint32_t kStep = kLanes * T::kVec;
    constexpr int kAtOnce = VECS < 8 ? 1 : 2;  // loads in flight (4: 169 registers where the rest of the kernel has 155)
    const auto each = [&](auto look) {
#pragma unroll 1
        for (uint32_t begin = 0; begin < scores.m; begin += kAtOnce * kStep) {
            const uint32_t j0 = here(begin + at);
            float x[kAtOnce][T::kVec];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) scores.read(j0 + u * kStep, x[u]);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t first = Span<TYPE>(j0 + u * kStep, scores.m).first;
#pragma unroll
                for (int e = 0; e < T::kVec; ++e) look(ordered(x[u][e] + 0.f), first + e);
            }
        }
    };
    const auto count = [&](auto in) {
        int have = 0;
        each([&](uint32_t o, uint32_t column) { have += __builtin_popcountll(__ballot(in(o, column))); });
        return have;
    };
    // the two bits of v above `shift`: how many of v + 1, 2, 3 << shift hold(.) is true of
    const auto two_bits = [&](uint32_t &v, int shift, auto in, auto hold) {
        int have[3] = {0, 0, 0};
        const uint32_t step = 1u << shift, base = v;
        each([&](uint32_t o, uint32_t column) {
#pragma unroll
            for (int q = 0; q < 3; ++q) have[q] += __builtin_popcountll(__ballot(in(o, column, base + (q + 1) * step)));
        });
        for (int q = 0; q < 3; ++q) v += hold(have[q]) ? step : 0;
    };
    constexpr uint32_t kLeast = 0x00800000u;  // (-inf, which is forbidden, comes just before)
    uint32_t least = 0, last = 0xffffffffu;   // k columns are at or above `least`; of those equal to it, columns up to `last` are taken
    const auto reach = [](uint32_t o, uint32_t, uint32_t middle) { return o >= middle; };
    const auto enough = [&](int have) { return have >= k; };
#pragma unroll 1
    for (int shift = 30; shift >= 0; shift -= 2) {
        if (shift == 14 && count([&](uint32_t o, uint32_t) { return o >= max(least, kLeast); }) <= HELD) break;
        two_bits(least, shift, reach, enough);
    }
    least = max(least, kLeast);
    if (count([&](uint32_t o, uint32_t) { return o >= least; }) > HELD) {
        // the largest number below which fewer equal columns are than are wanted: that column is the last one
        const int wanted = k - count([&](uint32_t o, uint32_t) { return o > least; });
        last = 0;
#pragma unroll 1
        for (int shift = (cbits((int64_t)VECS * kStep) - 1) / 2 * 2; shift >= 0; shift -= 2)
            two_bits(last, shift, [&](uint32_t o, uint32_t column, uint32_t middle) { return o == least && column < middle; },
                     [&](int have) { return have < wanted; });
    }
    each([&](uint32_t o, uint32_t column) { push(o > least || (o == least && column <= last), (uint64_t)o << 32 | (uint32_t)~column); });
}

struct TopShared {
    float lane_max[kThreads];
    uint32_t hot[kThreads], block[kList];
    __align__(16) uint64_t list[kList + kRankPad];
    uint64_t best[kWaves];
    int hots, blocks, count;
};

// The k best columns of a row, by a workgroup that knows the maximum of each thread's columns in each block of the row
// (block_max[b], thread t having the 16 bytes number t, t + kThreads, ... of the row): k columns are at or above the
// k-th largest of the threads' maxima, and little more than k are, in little more than k of the (block, thread) pairs.
// Those are read again.  Where more than fit the lists may be among the best (many equal scores, or open columns that are the columns of
// fewer than k threads), the bound is made of scores and columns, and the list in the place of the maxima, which has room for the columns
// of 16 bytes for each of k threads; where that does not do either, the best are found one by one, each thread offering the best of
// its columns that is behind the last one found.  (A row of one value, 131072 columns, 20 alternatives: 467 us one by one, 71 us with the second
// bound; 9 us where scores differ.)
template <int TYPE, bool BIAS>
__device__ __forceinline__ void best_columns(const RowArgs &A, const RowOut &out, const RowScores<TYPE, BIAS> &scores, float my_max,
                                             float (*block_max)[kThreads], TopShared &L)
{
    using T = Score<TYPE>;
    const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
    constexpr uint32_t kStep = kThreads * T::kVec;
    const int vecs_log2 = A.block_log2 + cbits(kSlice / kStep);  // 16-byte loads of a pair
    L.lane_max[threadIdx.x] = my_max;
    if (threadIdx.x == 0) L.hots = L.blocks = L.count = 0;
    __syncthreads();
    int count = 0;
    if (!out.bad && !out.none) {
        float all[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all[w] = L.lane_max[w * kLanes + lane];
        const float bound = A.k <= kFew ? kth_largest_few(largest(all), A.k) : kth_largest_bound(all, A.k);
        if (my_max >= bound && my_max > -kInf) L.hot[atomicAdd(&L.hots, 1)] = threadIdx.x;
        __syncthreads();
        const int hots = L.hots;
        for (int i = threadIdx.x; i < hots << A.scan_log2; i += kThreads) {
            const uint32_t thread = L.hot[i >> A.scan_log2];
            const int b = i & ((1 << A.scan_log2) - 1);
            if (b >= A.blocks) continue;
            const float top = block_max[b][thread];
            if (top >= bound && top > -kInf) {
                const int at = atomicAdd(&L.blocks, 1);
                if (at < kList) L.block[at] = (uint32_t)b * kThreads + thread;
            }
        }
        __syncthreads();
        const int pairs = L.blocks;
        if (pairs <= kList) {
            for (int i = threadIdx.x; i < pairs << vecs_log2; i += kThreads) {
                const uint32_t pair = L.block[i >> vecs_log2];
                const uint32_t j = (((pair / kThreads) << vecs_log2) + (i & ((1 << vecs_log2) - 1))) * kStep + (pair % kThreads) * T::kVec;
                if (j >= A.m) continue;
                float x[T::kVec];
                scores.read(j, x);
                const uint32_t first = Span<TYPE>(j, A.m).first;
#pragma unroll
                for (int e = 0; e < T::kVec; ++e)
                    if (x[e] >= bound && x[e] > -kInf) {
                        const int at = atomicAdd(&L.count, 1);
                        if (at < kList) L.list[at] = alternative(x[e], first + e);
                    }
            }
        }
        __syncthreads();
        count = L.count;
        if (pairs > kList || count > kList) {
            // once more with a bound that tells equal scores apart: the k-th of the threads' best columns
            uint64_t mine = best_before(scores, ~0ull, threadIdx.x, kThreads);
            __syncthreads();  // (the counts are read)
            L.list[threadIdx.x] = mine;
            if (threadIdx.x == 0) L.best[0] = kForbidden, L.count = 0;
            __syncthreads();
            int better = 0;
#pragma unroll 8
            for (int o = 0; o < kThreads; ++o) better += L.list[o] > mine;
            if (better == A.k - 1 && mine != 0) L.best[0] = mine;
            __syncthreads();
            const uint64_t from = L.best[0];
            constexpr int kWide = kWholeBlocks * kThreads * (int)sizeof(float) / (int)sizeof(uint64_t) - kRankPad;
            static_assert(kWide >= REGOT_ROW_MAX_TOP * 8, "16 bytes of 16-bit scores for each of k threads");
            uint64_t *const list = reinterpret_cast<uint64_t *>(block_max);  // (nothing reads the maxima any more)
            each_from(scores, from, threadIdx.x, kThreads, [&](uint64_t a) {
                const int at = atomicAdd(&L.count, 1);
                if (at < kWide) list[at] = a;
            });
            __syncthreads();
            count = L.count;
            if (count <= kWide) {
                rank_all(list, count, threadIdx.x, kThreads, A.k, [&](int rank, uint64_t a) { out.top(rank, a); });
            } else for (count = 0; count < A.k; ++count) {
                uint64_t best = mine;
#pragma unroll
                for (int d = 1; d < kLanes; d *= 2) {
                    const uint64_t other = __shfl_xor((unsigned long long)best, d);
                    best = other > best ? other : best;
                }
                __syncthreads();
                if (lane == 0) L.best[wave] = best;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kWaves; ++w) best = L.best[w] > best ? L.best[w] : best;
                if (best == 0) break;
                if (threadIdx.x == 0) out.top(count, best);
                if (best == mine) mine = best_before(scores, best, threadIdx.x, kThreads);
            }
        } else {
            rank_all(L.list, count, threadIdx.x, kThreads, A.k, [&](int rank, uint64_t a) { out.top(rank, a); });
        }
    }
    for (int i = count + threadIdx.x; i < A.k; i += kThreads) out.no_top(i);
}

// A row, or a part of one, by a workgroup: one pass with a running maximum in every thread, whose sums are brought together at
// the end, and the threads' maxima in each block for the alternatives.  VECS: 16-byte loads a lane has in flight.
// Bound by memory for long rows: 4096 x 131072 bf16 170 us = 6.3 TB/s, with 20 alternatives 174-182; about 10 vector
// instructions a score, four of them the exponential's, would take 130 us.  For rows of one or two slices by what comes behind the pass:
// 10000 x 5000 bf16 33 us, with 20 alternatives 59.
// (Six workgroups to a compute unit, which is one register less than without the bound: 10000 x 5000 bf16, 20 alternatives 66 us and 59.)
template <int TYPE, bool BIAS, bool TOP, int VECS, bool PARTS>
__global__ __launch_bounds__(kThreads, BIAS ? 5 : 6) void row_logprob_kernel(RowArgs A)
{
    using T = Score<TYPE>;
    using Scores = RowScores<TYPE, BIAS>;
    constexpr uint32_t kStep = kThreads * T::kVec;
    constexpr int kVecsOfGroup = Scores::kGroupVecs, kGroups = VECS / kVecsOfGroup;
    __shared__ __align__(16) float block_max[kWholeBlocks][kThreads];  // (TOP and whole rows)
    __shared__ float team_sums[3 * kWaves];
    __shared__ TopShared shared;
    const uint32_t at = threadIdx.x * T::kVec;

    const int64_t tasks = PARTS ? A.n * A.parts : A.n;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t row = PARTS ? task / A.parts : task;
        const int part = PARTS ? (int)(task - row * A.parts) : 0;
        const Scores scores(A, row);
        const uint32_t part_columns = PARTS ? (uint32_t)A.part_blocks * A.block * kSlice : 0;
        const uint32_t begin = part * part_columns, end = PARTS ? min(A.m, begin + part_columns) : A.m;
        Given<TYPE, BIAS> given;
        if constexpr (!PARTS) given.ask(A, row, scores, threadIdx.x);

        Softmax soft;
        float top_of_block = -kInf;
        int block = part * A.part_blocks, left = A.block;  // slices of the block still to come
        const auto block_done = [&]() {
            if constexpr (PARTS) A.part_max[(row * A.blocks + block) * kThreads + threadIdx.x] = top_of_block;
            else block_max[block][threadIdx.x] = top_of_block;
            top_of_block = -kInf;
            ++block;
            left = A.block;
        };
        for (uint32_t j0 = begin; j0 < end; j0 += VECS * kStep) {
            typename T::Chunk raw[VECS];
            float bias[VECS][T::kVec];
#pragma unroll
            for (int u = 0; u < VECS; ++u)
                if (j0 + u / kVecsOfGroup * kSlice < end) {
                    raw[u] = scores.template ask<true>(j0 + u * kStep + at);
                    scores.ask_bias(j0 + u * kStep + at, bias[u]);
                }
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                if (j0 + g * kSlice < end) {
                    float x[kGroup];
#pragma unroll
                    for (int v = 0; v < kVecsOfGroup; ++v) scores.unpack(raw[g * kVecsOfGroup + v], bias[g * kVecsOfGroup + v], j0 + (g * kVecsOfGroup + v) * kStep + at, x + v * T::kVec);
                    const float top = largest(x);
                    soft.add(x, top, A.log2_scale);
                    if constexpr (TOP) {
                        top_of_block = max_nan(top_of_block, top);
                        if (--left == 0) block_done();
                    }
                }
            }
        }
        if constexpr (TOP)
            if (left < A.block) block_done();
        const float my_max = soft.max;
        soft.over_block<kWaves>(A.log2_scale, team_sums);
        if constexpr (PARTS) {
            if (threadIdx.x == 0) {
                float *const sums = A.part_sums + 3 * task;
                sums[0] = soft.max, sums[1] = soft.sum, sums[2] = soft.weighted;
            }
        } else {
            const RowOut out(A, row, soft, threadIdx.x == 0);
            given.tell(A, out, scores, threadIdx.x, kThreads);
            if constexpr (TOP) best_columns(A, out, scores, my_max, block_max, shared);
        }
        __syncthreads();  // the sums and the lists are read
    }
}

// A row's parts joined: a workgroup a row.  A chain of latencies: 6.2 us at 1 x 131072 bf16 with 20 alternatives (about: the maxima 1.2, the sums
// 1.0, the bound 0.7, the blocks 0.4, the second read 1.3, the ranks 1.0), 2 without.
template <int TYPE, bool BIAS, bool TOP>
__global__ __launch_bounds__(kThreads) void row_logprob_join_kernel(RowArgs A)
{
    __shared__ float team_sums[3 * kWaves];
    __shared__ TopShared shared;
    __shared__ __align__(16) float block_max[kPartBlocks][kThreads];
    for (int64_t row = blockIdx.x; row < A.n; row += gridDim.x) {
        const RowScores<TYPE, BIAS> scores(A, row);
        Given<TYPE, BIAS> given;
        given.ask(A, row, scores, threadIdx.x);
        float my_max = -kInf;
        if constexpr (TOP) {
            const float *const maxima = A.part_max + row * A.blocks * kThreads + threadIdx.x;
            constexpr int kAsked = 32;  // (all of them, but for long rows)
            for (int b0 = 0; b0 < A.blocks; b0 += kAsked) {
                float top[kAsked];
#pragma unroll
                for (int i = 0; i < kAsked; ++i) top[i] = b0 + i < A.blocks ? maxima[(b0 + i) * kThreads] : -kInf;
#pragma unroll
                for (int i = 0; i < kAsked; ++i) block_max[b0 + i][threadIdx.x] = top[i], my_max = max_nan(my_max, top[i]);
            }
        }
        Softmax soft;
        for (int p = threadIdx.x; p < A.parts; p += kThreads) {  // (at most kThreads parts)
            const float *const sums = A.part_sums + 3 * (row * A.parts + p);
            soft.max = sums[0], soft.sum = sums[1], soft.weighted = sums[2];
        }
        soft.over_block<kWaves>(A.log2_scale, team_sums);
        const RowOut out(A, row, soft, threadIdx.x == 0);
        given.tell(A, out, scores, threadIdx.x, kThreads);
        if constexpr (TOP) best_columns(A, out, scores, my_max, block_max, shared);
        __syncthreads();
    }
}

// Narrow rows: a wave a row, which is held in registers as it was read: VECS 16-byte loads a lane.  Bound by instructions: 16384 x 2000
// bf16 17 us = 3.8 TB/s, with 10 alternatives 39; by workgroups of four waves a row 42 and 137.
template <int TYPE, bool BIAS, bool TOP, int VECS>
__global__ __launch_bounds__(kThreads) void row_logprob_narrow_kernel(RowArgs A)
{
    using T = Score<TYPE>;
    using Scores = RowScores<TYPE, BIAS>;
    constexpr uint32_t kStep = kLanes * T::kVec;
    constexpr int kHeld = 256;
    static_assert(T::kVec > 1 || VECS * kLanes <= kHeld, "all columns of a row of single loads");
    __shared__ uint16_t pair[kWaves][VECS * kLanes];
    __shared__ int counts[kWaves];
    __shared__ __align__(16) uint64_t list[kWaves][kHeld + kRankPad];
    const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
    const uint32_t at = lane * T::kVec;
    for (int64_t row = (int64_t)blockIdx.x * kWaves + wave; row < A.n; row += (int64_t)gridDim.x * kWaves) {
        const Scores scores(A, row);
        Given<TYPE, BIAS> given;
        given.ask(A, row, scores, lane);
        typename T::Chunk raw[VECS];
        if (A.m > 0) {
#pragma unroll
            for (int u = 0; u < VECS; ++u) raw[u] = scores.template ask<true>(u * kStep + at);
        }
        Softmax soft;
        float top[VECS];  // the largest of each load
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            top[u] = -kInf;
            if (u * kStep < A.m) {
                float x[T::kVec];
                scores.unpack(raw[u], u * kStep + at, x);
                top[u] = largest(x);
                soft.add(x, top[u], A.log2_scale);
            }
        }
        soft.over_wave(A.log2_scale);
        const RowOut out(A, row, soft, lane == 0);
        given.tell(A, out, scores, lane, kLanes);
        if constexpr (TOP) {
            // as in best_columns, with two maxima a lane for the bound, and (load, lane) for (block, thread)
            int count = 0;
            if (!out.bad && !out.none) {
                const auto push = [&](bool is, uint64_t a) {
                    const uint64_t mask = __ballot(is);
                    const int to = count + lanes_below(mask);
                    if (is && to < kHeld) list[wave][to] = a;
                    count += __builtin_popcountll(mask);
                };
                // Where k is more than three quarters of the maxima that the bound comes from (13 of 16 for 8 loads, whose rounds of
                // counting are longer), so many columns of ordinary scores pass it that counting is faster, or does not
                // even fit the list.  us, 8192 rows bf16, bound / counting: 512 columns k = 49 21 / 22, k = 56 32 / 22; 2000 columns
                // k = 96 77 / 95, k = 104 96 / 95, k = 105 (some lists too short) over 150 / 95; 4096 columns k = 96 83 / 158, k = 104 115 / 158.
                constexpr int kHalves = VECS == 1 ? 1 : 2;
                const int maxima = min((A.m + T::kVec - 1) / T::kVec, (uint32_t)kHalves * kLanes);
                bool found = T::kVec == 1 || 16 * A.k <= (VECS == 8 ? 13 : 12) * maxima;
                if (found) {
                    float half[kHalves];
#pragma unroll
                    for (int u = 0; u < VECS; ++u) half[u % kHalves] = u < kHalves ? top[u] : max_nan(half[u % kHalves], top[u]);
                    const float bound = kth_largest_bound(half, A.k);
                    int pairs = 0;
                    wave_lds();
#pragma unroll
                    for (int u = 0; u < VECS; ++u) {
                        const bool is = top[u] >= bound && top[u] > -kInf;
                        const uint64_t mask = __ballot(is);
                        if (is) pair[wave][pairs + lanes_below(mask)] = u * kLanes + lane;
                        pairs += __builtin_popcountll(mask);
                    }
                    wave_lds();
                    for (int i0 = 0; i0 < pairs; i0 += kLanes) {
                        float x[T::kVec];
                        uint32_t first = 0;
                        if (i0 + lane < pairs) {
                            const uint32_t j = pair[wave][i0 + lane] * T::kVec;
                            scores.read(j, x);
                            first = Span<TYPE>(j, A.m).first;
                        }
#pragma unroll
                        for (int e = 0; e < T::kVec; ++e) push(i0 + lane < pairs && x[e] >= bound && x[e] > -kInf, alternative(x[e], first + e));
                    }
                    wave_lds();
                    found = T::kVec == 1 || count <= kHeld;  // (rows of single loads have no more than kHeld columns)
                    // (of equal scores, the bound by columns too would leave kVec for each of the k)
                    if (T::kVec > 1 && !found && (A.k - 1) * T::kVec < kHeld) {
                        const uint64_t mine = best_before(scores, ~0ull, lane, kLanes);
                        int better = 0;
                        for (int l = 0; l < kLanes; ++l) better += __shfl((unsigned long long)mine, l) > mine;
                        const uint64_t kth = __ballot(better == A.k - 1 && mine != 0);
                        const uint64_t from = kth != 0 ? __shfl((unsigned long long)mine, __builtin_ctzll(kth)) : kForbidden;
                        if (lane == 0) counts[wave] = 0;
                        wave_lds();
                        each_from(scores, from, lane, kLanes, [&](uint64_t a) {
                            const int to = atomicAdd(&counts[wave], 1);
                            if (to < kHeld) list[wave][to] = a;
                        });
                        wave_lds();
                        count = counts[wave];
                        found = count <= kHeld;
                    }
                }
                if constexpr (T::kVec > 1) {
                    if (!found) {
                        count = 0;
                        wave_lds();
                        best_by_bisection<kHeld, VECS>(scores, A.k, at, push);
                        wave_lds();
                    }
                }
                rank_all(list[wave], count, lane, kLanes, A.k, [&](int rank, uint64_t a) { out.top(rank, a); });
            }
            for (int i = count + lane; i < A.k; i += kLanes) out.no_top(i);
        }
    }
}

}  // namespace regot
