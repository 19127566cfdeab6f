// A router's choices in the order of their experts, and the weighted sum of the experts' rows with its gradient (gfx950, wave64).
#pragma once

#include "regot_experts.hpp"

namespace regot {

constexpr int kOrderWaves = 16, kOrderThreads = kOrderWaves * kLanes;

struct OrderArgs {
    const int32_t *idx;
    int64_t count;      // choices
    int experts;        // choice `experts` stands for none
    int key_bits;       // of numbers up to `experts`
    int64_t each;       // choices of a workgroup, a multiple of kOrderThreads
    int groups;         // workgroups
    uint32_t *counts;   // [groups][experts + 1], where there are several
    int64_t *start;
    int32_t *order, *place;
};

__device__ __forceinline__ int choice(const OrderArgs &A, int64_t s)
{
    const int32_t v = A.idx[s];
    return (uint32_t)v < (uint32_t)A.experts ? v : A.experts;
}

// How many choices of each expert (and of none) each wave of the workgroup has: its part of the workgroup's choices, one after the other.
__device__ __forceinline__ void count_choices(const OrderArgs &A, int64_t from, int64_t to, uint32_t *mine)
{
    const int lane = threadIdx.x % kLanes;
#pragma unroll 4
    for (int64_t s = from + lane; s < to; s += kLanes) atomicAdd(&mine[choice(A, s)], 1u);
}

__global__ void __launch_bounds__(kOrderThreads) expert_count_kernel(const OrderArgs A)
{
    __shared__ uint32_t counts[REGOT_ROW_MAX_EXPERTS + 1];
    for (int e = threadIdx.x; e <= A.experts; e += kOrderThreads) counts[e] = 0;
    __syncthreads();
    const int64_t from = blockIdx.x * A.each, to = min(from + A.each, A.count);
    for (int64_t s = from + threadIdx.x; s < to; s += kOrderThreads) atomicAdd(&counts[choice(A, s)], 1u);
    __syncthreads();
    for (int e = threadIdx.x; e <= A.experts; e += kOrderThreads) A.counts[(int64_t)blockIdx.x * (A.experts + 1) + e] = counts[e];
}

// Each workgroup puts its choices where they belong: behind those of the experts before, of the same expert in the workgroups before, and in the waves
// before; within a wave, 64 choices at a time, behind the equal ones in lower lanes (a ballot for each bit of the expert's number).  The counts
// are sums of integers: nothing depends on the order of the additions.  A chain of short steps is what bounds it: 524288 choices of 256 experts 13 us behind the counting's 3,
// 32768 of 60 6.6 behind 2.4.
__global__ void __launch_bounds__(kOrderThreads) expert_order_kernel(const OrderArgs A)
{
    __shared__ uint32_t next[kOrderWaves * (REGOT_ROW_MAX_EXPERTS + 1)];  // [kOrderWaves][experts + 1]: where the next choice of an expert goes
    __shared__ uint32_t totals[kOrderWaves];
    const int E = A.experts + 1, wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    for (int i = threadIdx.x; i < kOrderWaves * E; i += kOrderThreads) next[i] = 0;
    __syncthreads();
    const int64_t from = blockIdx.x * A.each, to = min(from + A.each, A.count);
    const int64_t of_wave = (to - from + kOrderThreads - 1) / kOrderThreads * kLanes;
    const int64_t mine = min(from + wave * of_wave, to), end = min(mine + of_wave, to);
    uint32_t *const my_next = next + wave * E;
    count_choices(A, mine, end, my_next);
    __syncthreads();
    // what all workgroups have of each expert, and those before this one: every thread takes a share of the workgroups
    __shared__ uint32_t of_all[REGOT_ROW_MAX_EXPERTS + 1], of_before[REGOT_ROW_MAX_EXPERTS + 1];
    if (A.groups > 1) {
        for (int e = threadIdx.x; e < E; e += kOrderThreads) of_all[e] = of_before[e] = 0;
        __syncthreads();
        const int shares = max(kOrderThreads / E, 1), share = threadIdx.x / E;
        for (int e = threadIdx.x % E; e < E && share < shares; e += kOrderThreads) {
            uint32_t all = 0, before = 0;
#pragma unroll 8
            for (int b = share; b < A.groups; b += shares) {
                const uint32_t v = A.counts[(int64_t)b * E + e];
                all += v;
                before += b < (int)blockIdx.x ? v : 0;
            }
            atomicAdd(&of_all[e], all);
            atomicAdd(&of_before[e], before);
        }
    } else {
        for (int e = threadIdx.x; e < E; e += kOrderThreads) {
            uint32_t v = 0;
            for (int w = 0; w < kOrderWaves; ++w) v += next[w * E + e];
            of_all[e] = v;
            of_before[e] = 0;
        }
    }
    __syncthreads();
    // thread t: experts 2 t and 2 t + 1 (1025 of them at most, with none), a thread's and then the experts' sums
    const auto of = [&](const uint32_t *counts, int e) { return e < E ? counts[e] : 0; };
    const uint32_t all[2] = {of(of_all, 2 * threadIdx.x), of(of_all, 2 * threadIdx.x + 1)};
    uint32_t sum = all[0] + all[1];
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) {
        const uint32_t v = __shfl_up(sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == kLanes - 1) totals[wave] = sum;
    __syncthreads();
    uint32_t first = sum - all[0] - all[1];
    for (int w = 0; w < wave; ++w) first += totals[w];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int e = 2 * threadIdx.x + j;
        if (e >= E) continue;
        const uint32_t begin = first + (j ? all[0] : 0);
        if (blockIdx.x == 0) A.start[e] = begin;
        uint32_t at = begin + of_before[e];
        for (int w = 0; w < kOrderWaves; ++w) {
            const uint32_t here = next[w * E + e];
            next[w * E + e] = at;
            at += here;
        }
    }
    __syncthreads();
    constexpr int kHeld = 8;  // choices that a lane asks for at a time
    for (int64_t s0 = mine; s0 < end; s0 += kHeld * kLanes) {
        int held[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) held[j] = s0 + j * kLanes + lane < end ? choice(A, s0 + j * kLanes + lane) : 0;
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            if (s0 + j * kLanes >= end) break;
            const int64_t s = s0 + j * kLanes + lane;
            const bool live = s < end;
            const int e = held[j];
            uint64_t same = __ballot(live);
            for (int bit = 0; bit < A.key_bits; ++bit) {
                const bool set = e >> bit & 1;
                const uint64_t b = __ballot(set);
                same &= set ? b : ~b;
            }
            if (live) {
                const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
                const uint32_t r = my_next[e] + rank;
                wave_lds();
                if (rank == 0) my_next[e] = r + __popcll(same);
                A.order[r] = e < A.experts ? (int32_t)s : -1;
                A.place[s] = e < A.experts ? (int32_t)r : -1;
            }
            wave_lds();
        }
    }
}

struct CombineArgs {
    int64_t n, m, rows;
    int k;
    const void *Y;
    int64_t ldY;
    const int32_t *place;
    const float *weight;    // NULL: 1
    const void *g;          // gradient to the sums
    int64_t ldG;
    void *out;              // the sums, or dY
    int64_t ldO;
    float *g_weight;
    uint32_t parts;         // stretches of a row's columns
};

// Columns first .. first + kVec - 1 of a row of m, as a lane has them: whole where they are, otherwise one at a time.  (Rows begin at any multiple of
// their element.)
template <int TYPE>
struct Stretch {
    using T = Score<TYPE>;
    using Raw = typename T::Raw;
    typedef u32x4 Any __attribute__((aligned(alignof(uint16_t))));
    static constexpr int kVec = T::kVec;
    static __device__ __forceinline__ u32x4 load(const Raw *row, int64_t first, int64_t m)
    {
        if (first + kVec <= m) return *reinterpret_cast<const Any *>(row + first);
        Raw part[kVec];
#pragma unroll
        for (int c = 0; c < kVec; ++c) part[c] = first + c < m ? row[first + c] : Raw(0.f);
        return WideChunk::pack(part);
    }
    static __device__ __forceinline__ void store(Raw *row, int64_t first, int64_t m, const float *v)
    {
        Raw part[kVec];
#pragma unroll
        for (int c = 0; c < kVec; ++c) part[c] = T::put(v[c]);
        if (first + kVec <= m) {
            __builtin_nontemporal_store(WideChunk::pack(part), reinterpret_cast<Any *>(row + first));
        } else {
#pragma unroll
            for (int c = 0; c < kVec; ++c)
                if (first + c < m) row[first + c] = part[c];
        }
    }
};

// A wave: 64 x 16 bytes of one token's sum.  The rows are asked for four at a time.  Memory bounds it: 65536 tokens x 8 rows of 2048 bf16 423 us = 5.7 TB/s.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) expert_combine_kernel(const CombineArgs A)
{
    using S = Stretch<TYPE>;
    using Raw = typename S::Raw;
    const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const int64_t waves = A.n * A.parts, step = (int64_t)gridDim.x * kWaves;
    for (int64_t w = (int64_t)blockIdx.x * kWaves + wave; w < waves; w += step) {
        const int64_t i = w / A.parts, c = (w % A.parts * kLanes + lane) * S::kVec;
        if (c >= A.m) continue;
        float sum[S::kVec] = {};
        for (int l0 = 0; l0 < A.k; l0 += 4) {
            u32x4 v[4];
            int32_t p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = l0 + j < A.k ? A.place[i * A.k + l0 + j] : -1;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if ((uint32_t)p[j] < (uint64_t)A.rows) v[j] = S::load(static_cast<const Raw *>(A.Y) + p[j] * A.ldY, c, A.m);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((uint32_t)p[j] >= (uint64_t)A.rows) continue;
                const float weight = A.weight ? A.weight[i * A.k + l0 + j] : 1.f;
                float x[S::kVec];
                S::T::unpack(v[j], x);
#pragma unroll
                for (int e = 0; e < S::kVec; ++e) sum[e] = fmaf(weight, x[e], sum[e]);
            }
        }
        S::store(static_cast<Raw *>(A.out) + i * A.ldO, c, A.m, sum);
    }
}

// A wave: one choice.  dY = weight times the token's gradient, and the weight's gradient, the product of the two rows.  The token's row comes from the caches but for
// once: 65536 tokens x 8 rows of 2048 bf16 845 us = 5.4 TB/s of reads and writes.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) expert_combine_grad_kernel(const CombineArgs A)
{
    using S = Stretch<TYPE>;
    using Raw = typename S::Raw;
    const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const int64_t slots = A.n * A.k, step = (int64_t)gridDim.x * kWaves;
    for (int64_t s = (int64_t)blockIdx.x * kWaves + wave; s < slots; s += step) {
        const int32_t p = A.place[s];
        float dot = 0.f;
        if ((uint32_t)p < (uint64_t)A.rows) {
            const float weight = A.weight ? A.weight[s] : 1.f;
            const Raw *g = static_cast<const Raw *>(A.g) + s / A.k * A.ldG, *y = static_cast<const Raw *>(A.Y) + p * A.ldY;
            Raw *out = static_cast<Raw *>(A.out) + p * A.ldO;
            for (int64_t c = lane * S::kVec; c < A.m; c += kLanes * S::kVec) {
                float gv[S::kVec], yv[S::kVec];
                S::T::unpack(S::load(g, c, A.m), gv);
                if (A.g_weight) {
                    S::T::unpack(S::load(y, c, A.m), yv);
#pragma unroll
                    for (int e = 0; e < S::kVec; ++e) dot = fmaf(gv[e], yv[e], dot);
                }
#pragma unroll
                for (int e = 0; e < S::kVec; ++e) gv[e] *= weight;
                S::store(out, c, A.m, gv);
            }
        }
        if (A.g_weight) {
            dot = wave_all<OpSumF>(dot);
            if (lane == 0) A.g_weight[s] = dot;
        }
    }
}

}  // namespace regot
