// Gradients to rows of scores: of log probabilities and entropy, and of the divergence from sparse targets with its loss.
#pragma once

#include <type_traits>

#include "regot_rows_logprob.hpp"

namespace regot {

// A row by WAVES waves: WAVES = 1, four rows to a workgroup; otherwise a workgroup a row (or a part of one).
template <int WAVES>
struct Team {
    static constexpr int kRows = WAVES == 1 ? kWaves : 1;
    static constexpr int kSize = WAVES * kLanes;              // threads of a row
    static constexpr int kBlock = kRows * kSize;
    static __device__ __forceinline__ int thread() { return WAVES == 1 ? threadIdx.x & (kLanes - 1) : threadIdx.x; }
    static __device__ __forceinline__ int row() { return WAVES == 1 ? threadIdx.x / kLanes : 0; }
    static __device__ __forceinline__ void sync()
    {
        if constexpr (WAVES == 1) wave_lds();
        else __syncthreads();
    }
    // lds: WAVES floats (not looked at for one wave)
    template <typename Op>
    static __device__ __forceinline__ float all(float v, float *lds)
    {
        if constexpr (WAVES == 1) return wave_all<Op>(v);
        else return block_all<Op, WAVES>(v, lds);
    }
};

// Columns that a list of a row names are written a second time, behind a barrier, by the threads that have the entries: each
// with the sum over all entries of its column (columns listed twice are written twice, with the same number).

// dS of log probabilities and entropy.  With t = log2 p, a = (sum g + h H) / eta and b = h ln 2 / eta:  -p (a + b t), and
// g / eta more at the given columns.  The sums are known, so a row is cut into as many parts as there are loads for; each
// reads and writes its columns once.  Bound by memory: 4096 x 131072 bf16 350 us = 6.1 TB/s, 2048 x 40000 57 us = 5.7 TB/s.
template <int TYPE, bool BIAS, int WAVES, int VECS>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void row_logprob_grad_kernel(RowArgs A)
{
    using T = Score<TYPE>;
    using Row = Team<WAVES>;
    constexpr uint32_t kStep = (uint32_t)Row::kSize * T::kVec;
    const int thread = Row::thread(), lane = threadIdx.x & (kLanes - 1);
    const int64_t tasks = A.n * A.parts;
    for (int64_t task = (int64_t)blockIdx.x * Row::kRows + Row::row(); task < tasks; task += (int64_t)gridDim.x * Row::kRows) {
        const int64_t row = task / A.parts;
        const uint32_t begin = (uint32_t)(task - row * A.parts) * A.part_columns, end = min(A.m, begin + A.part_columns);
        const RowScores<TYPE, BIAS> scores(A, row);
        typename T::Raw *const out = static_cast<typename T::Raw *>(A.dS) + row * A.ldD;
        const int32_t *const target = A.target + row * A.targets;
        const float *const weight = A.g_logprob + row * A.targets;
        typename T::Chunk raw[VECS];
        const auto ask = [&](uint32_t j0) {
#pragma unroll
            for (int u = 0; u < VECS; ++u)
                if (j0 + u * kStep < end) raw[u] = scores.template ask<true>(j0 + u * kStep + thread * T::kVec);
        };
        ask(begin);
        const float max = A.stats_in[2 * row], log_sum = A.stats_in[2 * row + 1];
        const bool none = max == -kInf;
        const float h = A.g_entropy ? A.g_entropy[row] : 0.f, entropy = A.g_entropy ? A.entropy_in[row] : 0.f;
        float g = 0.f;
        for (int t = lane; t < A.targets; t += kLanes)
            if ((uint32_t)target[t] < A.m) g += weight[t];
        g = wave_all<OpSumF>(g);
        const float a = A.inv_eta * fmaf(h, entropy, g), b = A.inv_eta * h * kLn2;
        const float from = none ? 0.f : max, less = none ? 0.f : log_sum * kLog2e;
        const auto value = [&](float x) {
            // (far below any p that is not 0; a NaN stays one)
            const float t = max_nan(fmaf(x - from, A.log2_scale, -less), -16384.f);
            return -exp2_fast(t) * fmaf(b, t, a);
        };
        for (uint32_t j0 = begin; j0 < end; j0 += VECS * kStep) {
            if (j0 != begin) ask(j0);
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                if (j0 + u * kStep >= end) continue;
                const Span<TYPE> span(j0 + u * kStep + thread * T::kVec, A.m);
                if (span.own >= end) continue;
                float x[T::kVec];
                scores.unpack(raw[u], span.own, x);
#pragma unroll
                for (int e = 0; e < T::kVec; ++e) x[e] = value(x[e]);
                span.store(out, x);
            }
        }
        if (A.targets == 0 || none) continue;
        __threadfence_block();
        Row::sync();
        for (int t = thread; t < A.targets; t += Row::kSize) {
            const uint32_t j = (uint32_t)target[t];
            if (j < begin || j >= end) continue;
            float mine = 0.f;
            for (int u = 0; u < A.targets; ++u) mine += (uint32_t)target[u] == j ? weight[u] : 0.f;
            out[j] = T::put(fmaf(mine, A.inv_eta, value(scores(j))));
        }
    }
}

// The loss against a sparse target, and dS = w (p - q) / eta.
//
// The sum over a row comes before its first gradient, so a row is read twice (PARTS: here, and by the kernel that left the sums
// of its parts).  Backwards the second time: the last stretch of VECS loads a thread is still in registers, the first KEPT loads of the one before are in
// LDS, and what is before that is likeliest in the caches.  Bound by traffic: 4096 x 131072 bf16 431 us for 2.1 GB that have to move and 0.5 that is
// read again (6.2 TB/s); 513 without KEPT.  Shorter rows by the chain of each row (target, sum, loss, list) and the rows under way.
// Four waves to a SIMD, as the LDS allows, and columns that are computed where they are used: fp32 178 registers otherwise, and 40 of
// them in memory with 16 waves (256 x 131072 fp32 71 us against 63, 999 x 33333 74 against 68).
// LIST: the room for a row's entries (a wave a row: 128 where they fit, 16384 x 400 fp32 24.2 us with 1024 and 21.2 with 128).
template <int TYPE, int WAVES, int VECS, int KEPT, bool PARTS, int LIST = REGOT_ROW_MAX_LIST>
__global__ __launch_bounds__(Team<WAVES>::kBlock, KEPT > 0 ? 4 : 1) void row_distill_kernel(RowArgs A)
{
    using T = Score<TYPE>;
    using Row = Team<WAVES>;
    constexpr uint32_t kStep = (uint32_t)Row::kSize * T::kVec;
    __shared__ float team_lds[3 * WAVES];
    __shared__ typename T::Chunk kept[KEPT > 0 ? KEPT : 1][KEPT > 0 ? Row::kBlock : 1];
    __shared__ uint32_t list_column[Row::kRows][LIST];
    __shared__ float list_q[Row::kRows][LIST];
    const int thread = Row::thread(), lane = threadIdx.x & (kLanes - 1), team = Row::row();
    const int64_t tasks = PARTS ? A.n * A.parts : A.n;
    for (int64_t task = (int64_t)blockIdx.x * Row::kRows + team; task < tasks; task += (int64_t)gridDim.x * Row::kRows) {
        const int64_t row = PARTS ? task / A.parts : task;
        const uint32_t begin = PARTS ? (uint32_t)(task - row * A.parts) * A.part_columns : 0, end = PARTS ? min(A.m, begin + A.part_columns) : A.m;
        const RowScores<TYPE, false> scores(A, row);
        typename T::Raw *const out = A.dS ? static_cast<typename T::Raw *>(A.dS) + row * A.ldD : nullptr;
        const int32_t *const target = A.target + row * A.k;
        const float *const score = A.t_score + row * A.k;

        // the first loads of the row, and of the target's columns, are on their way while the target is looked at
        typename T::Chunk raw[VECS];
        const auto ask = [&](uint32_t j0, auto once) {
#pragma unroll
            for (int u = 0; u < VECS; ++u)
                if (j0 + u * kStep < end) raw[u] = scores.template ask<decltype(once)::value>(j0 + u * kStep + thread * T::kVec);
        };
        using Once = std::integral_constant<bool, PARTS>;
        ask(begin, Once{});
        uint32_t my_column = 0xffffffffu;
        float my_score = 0.f, my_x = 0.f;
        if (thread < A.k) {
            my_column = (uint32_t)target[thread];
            my_score = score[thread];
            if (my_column < A.m) my_x = scores(my_column);
        }
        // every wave has the whole target, so that none waits for another
        float t_max = -kInf;
        for (int l = lane; l < A.k; l += kLanes)
            if ((uint32_t)target[l] < A.m) t_max = max_nan(t_max, score[l]);
        t_max = wave_all<OpMaxF>(t_max);
        const bool padding = t_max == -kInf;
        Softmax soft;
        if (!padding) {
            if constexpr (PARTS) {
                if (thread < A.parts) {  // (no more parts than threads)
                    const float *const sums = A.part_sums + 3 * (row * A.parts + thread);
                    soft.max = sums[0], soft.sum = sums[1];
                }
            } else {
                for (uint32_t j0 = 0; j0 < end; j0 += VECS * kStep) {
                    if (j0 != 0) ask(j0, Once{});
                    if (KEPT > 0 && j0 + VECS * kStep < end && j0 + 2 * VECS * kStep >= end) {
#pragma unroll
                        for (int u = 0; u < KEPT; ++u) kept[u][threadIdx.x] = raw[u];
                    }
                    constexpr int kVecsOfGroup = VECS % 2 == 0 ? 2 : 1;
#pragma unroll
                    for (int g = 0; g < VECS / kVecsOfGroup; ++g) {
                        if (j0 + g * kVecsOfGroup * kStep >= end) continue;
                        float x[kVecsOfGroup * T::kVec];
#pragma unroll
                        for (int v = 0; v < kVecsOfGroup; ++v) {
                            const uint32_t j = here(j0 + (g * kVecsOfGroup + v) * kStep + thread * T::kVec);
                            if (v > 0 && j0 + (g * kVecsOfGroup + v) * kStep >= end) {
#pragma unroll
                                for (int e = 0; e < T::kVec; ++e) x[v * T::kVec + e] = -kInf;
                            } else {
                                scores.unpack(raw[g * kVecsOfGroup + v], j, x + v * T::kVec);
                            }
                        }
                        soft.template add<false>(x, largest(x), A.log2_scale);
                    }
                }
            }
        }
        float q_sum = 0.f;
        for (int l = lane; l < A.k && !padding; l += kLanes)
            if ((uint32_t)target[l] < A.m) q_sum += exp2_fast((score[l] - t_max) * A.log2_scale);
        q_sum = wave_all<OpSumF>(q_sum);
        soft.over_block<WAVES>(A.log2_scale, team_lds);
        const bool bad = !padding && (soft.bad() || q_sum != q_sum), none = padding || soft.none();
        const float max = none ? 0.f : soft.max, log_sum = soft.log_sum(), log_q = logf(q_sum), inv_q = 1.f / q_sum;
        const float weight = (A.row_weight ? A.row_weight[row] : 1.f) * A.inv_eta;
        const float of_p = bad ? kNan : none ? 0.f : weight / soft.sum;
        float loss = 0.f;
        const uint32_t first_column = my_column;
        const float first_x = my_x;
        for (int l = thread; l < A.k; l += Row::kSize) {
            if (l != thread) {
                my_column = (uint32_t)target[l];
                my_score = score[l];
                if (my_column < A.m) my_x = scores(my_column);
            }
            const uint32_t j = my_column;
            const float t = my_score - t_max, q = j < A.m && !padding ? exp2_fast(t * A.log2_scale) * inv_q : 0.f;
            list_column[team][l] = j;
            list_q[team][l] = q;
            // (q times the distance before it is divided by eta: a mask of the type's lowest value stays finite)
            if (q != 0.f) loss += none ? kInf : q * (t * A.inv_eta - log_q + log_sum) + q * A.inv_eta * (max - my_x);
        }
        loss = Row::template all<OpSumF>(loss, team_lds + 2 * WAVES);
        if (thread == 0 && begin == 0) A.loss[row] = bad ? kNan : loss;
        if (out) {
            const auto p_weighted = [&](float x) { return exp2_fast((x - max) * A.log2_scale) * of_p; };
            // backwards: the columns read last are still here, those before them in the caches
            const int stretches = (int)((end - begin + VECS * kStep - 1) / (VECS * kStep));
            for (int i = 0; i < stretches; ++i) {
                const uint32_t j0 = begin + (PARTS ? i : stretches - 1 - i) * VECS * kStep;
                if (KEPT > 0 && i == 1) {
#pragma unroll
                    for (int u = 0; u < VECS; ++u) raw[u] = u < KEPT ? kept[u < KEPT ? u : 0][threadIdx.x] : scores.template ask<true>(j0 + u * kStep + thread * T::kVec);
                } else if (i > 0 && !none) {
                    ask(j0, std::true_type{});
                }
#pragma unroll
                for (int u = 0; u < VECS; ++u) {
                    if (j0 + u * kStep >= end) continue;
                    const Span<TYPE> span(here(j0 + u * kStep + thread * T::kVec), A.m);
                    if (span.own >= end) continue;
                    float x[T::kVec] = {};
                    if (!none) {
                        scores.unpack(raw[u], span.own, x);
#pragma unroll
                        for (int e = 0; e < T::kVec; ++e) x[e] = p_weighted(x[e]);
                    }
                    span.store(out, x);
                }
            }
            if (!none) {
                __threadfence_block();
                Row::sync();
                for (int l = thread; l < A.k; l += Row::kSize) {
                    const uint32_t j = l == thread ? first_column : list_column[team][l];
                    if (j < begin || j >= end) continue;
                    float q = 0.f;
#pragma unroll 8
                    for (int u = 0; u < A.k; ++u) q += list_column[team][u] == j ? list_q[team][u] : 0.f;
                    out[j] = T::put(p_weighted(l == thread ? first_x : scores(j)) - (bad ? kNan : weight) * q);
                }
            }
        }
        Row::sync();  // the list and the sums are read
    }
}

}  // namespace regot
