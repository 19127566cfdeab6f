// Routing of rows to k of their columns, and its gradient.
//
// A row is LANES lanes', which hold VALUES of its scores each; a wave has 64 / LANES rows, a workgroup four waves.  The k best
// come out of a network without branches: each lane sorts what it has to a list of its KEPT best, and lists of
// pairs of lanes are merged until every lane has the row's.  Keys and columns are one number, so that ties need nothing
// of their own.  Bound by instructions: 870 of the vector unit for four rows of 256 (the network of 8 of 16 values about 380, keys and scores
// the rest), 1010 with groups.  65536 rows of 256 fp32 scores 27 us, sigmoid in 8 groups 36 us, where reading them takes 10; a wave a row and k rounds
// of the largest left: choice and gradient 323 us, now 56.
#pragma once

#include "regot_rows.hpp"

namespace regot {

struct RouteArgs {
    int64_t n;
    uint32_t m;
    const void *S;
    int64_t ldS;
    const float *bias;
    int bias_on, score, groups, groups_kept, group_by, k, renormalise;
    uint32_t group_size, group_magic;  // column / group_size = (column * group_magic) >> 32; 0 for groups of one column
    int group_lanes;                   // lanes that look at one group (a power of two)
    float scale;
    int32_t *idx;
    float *weight;
    const int32_t *idx_in;
    const float *g_weight;
    void *dS;
    int64_t ldD;
};

constexpr int kMaxGroups = 64;

// A key and its column as a double, larger for what is chosen first: 48 bits, the key's 32 in the order of numbers above the
// column's complement, below a fixed exponent.  -inf comes below all other keys, and no_choice() below that.
__device__ __forceinline__ double choice(float key, uint32_t column)
{
    const uint32_t o = ordered(key + 0.f);
    return __hiloint2double((int)__builtin_amdgcn_alignbit(0x4000u, o, 16), (int)(o << 16 | (0xffffu - column)));
}
__device__ __forceinline__ double no_choice() { return __hiloint2double(0x40000000, 0); }
__device__ __forceinline__ bool is_choice(double c) { return (uint32_t)__double2hiint(c) > 0x4000007fu; }  // (-inf: 0x4000007f)
__device__ __forceinline__ uint32_t chosen_column(double c) { return 0xffffu - ((uint32_t)__double2loint(c) & 0xffffu); }

// The larger and the smaller of two such numbers.  (Written out because fmax first makes each operand a proper number, which
// they are: a fourth more instructions in the network.)
__device__ __forceinline__ double larger(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double smaller(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// Both in order, the larger first.
__device__ __forceinline__ void in_order(double &a, double &b)
{
    const double hi = larger(a, b), lo = smaller(a, b);
    a = hi;
    b = lo;
}

// A sequence that rises once and falls once (either way around), into descending order.
template <int COUNT>
__device__ __forceinline__ void merge_down(double *a)
{
    if constexpr (COUNT > 1) {
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) in_order(a[i], a[i + COUNT / 2]);
        merge_down<COUNT / 2>(a);
        merge_down<COUNT / 2>(a + COUNT / 2);
    }
}

// Batcher's odd-even merge sort: 19 comparisons for 8 values, where merges of sequences that rise and fall take 24.
// (even_odd: every STEP-th of COUNT values, both halves of which are in descending order)
template <int COUNT, int STEP>
__device__ __forceinline__ void even_odd(double *a)
{
    if constexpr (2 * STEP < COUNT) {
        even_odd<COUNT, 2 * STEP>(a);
        even_odd<COUNT, 2 * STEP>(a + STEP);
#pragma unroll
        for (int i = STEP; i + STEP < COUNT; i += 2 * STEP) in_order(a[i], a[i + STEP]);
    } else {
        in_order(a[0], a[STEP]);
    }
}

template <int COUNT>
__device__ __forceinline__ void sort_down(double *a)
{
    if constexpr (COUNT > 1) {
        sort_down<COUNT / 2>(a);
        sort_down<COUNT / 2>(a + COUNT / 2);
        even_odd<COUNT, 1>(a);
    }
}

// a: the best KEPT of a and b, both in descending order
template <int KEPT, typename F>
__device__ __forceinline__ void merge_lists(double (&a)[KEPT], F b)
{
    double c[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) c[i] = larger(a[i], b(KEPT - 1 - i));
#pragma unroll
    for (int i = 0; i < KEPT; ++i) a[i] = c[i];
    merge_down<KEPT>(a);
}

// over the LANES lanes of a row, in a fixed order, the result in all of them
template <typename Op, int LANES>
__device__ __forceinline__ float row_all(float v)
{
    if constexpr (LANES == kLanes) return wave_all<Op>(v);
    v = Op::apply(v, dpp_f32<kDppXor1>(v));
    v = Op::apply(v, dpp_f32<kDppXor2>(v));
    v = Op::apply(v, dpp_f32<kDppHalfMirror>(v));
    if constexpr (LANES > 8) v = Op::apply(v, dpp_f32<kDppMirror>(v));
    if constexpr (LANES == 32) v = Op::apply(v, __shfl_xor(v, 16));
    return v;
}

// whether `is` holds in any of the LANES lanes of a row, in all of them
template <int LANES>
__device__ __forceinline__ bool row_any(bool is)
{
    const uint64_t lanes = __ballot(is);
    if constexpr (LANES == kLanes) return lanes != 0;
    else return (lanes >> ((threadIdx.x & (kLanes - 1)) / LANES * LANES) & ((1ull << LANES) - 1)) != 0;
}
__device__ __forceinline__ bool is_nan(float v) { return v != v; }

// Where column j of a row is kept in LDS: rows of 16 apart by four more, so that lanes that go through neighbouring groups do not
// meet, and 16 bytes stay together.
__device__ __forceinline__ uint32_t place(uint32_t j) { return j + (j >> 4) * 4; }
constexpr int places(int columns) { return columns + columns / 4; }

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A lane's columns of its row.
template <int TYPE, int LANES, int VALUES>
struct RouteRow {
    using T = Score<TYPE>;
    static constexpr int kChunks = VALUES / T::kVec;
    static constexpr int kColumns = LANES * VALUES;
    uint32_t m;
    int l;
    // the columns of chunk c; of value v
    __device__ __forceinline__ Span<TYPE> span(int c) const { return Span<TYPE>((uint32_t)(c * LANES + l) * T::kVec, m); }
    __device__ __forceinline__ uint32_t column(int v) const { return span(v / T::kVec).first + v % T::kVec; }

    __device__ __forceinline__ void load(const typename T::Raw *S, float (&x)[VALUES]) const
    {
        if (m == 0) {
#pragma unroll
            for (int v = 0; v < VALUES; ++v) x[v] = -kInf;
            return;
        }
        typename T::Chunk raw[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) raw[c] = span(c).template load<false>(S);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) T::unpack(raw[c], x + c * T::kVec);
        if (m < kColumns) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) span(c).mask(x + c * T::kVec);
        }
    }

};

// What makes a row's scores of its logits: e^(x - from) / sum, or 1 / (1 + e^-x).  Which one it is is looked at once for all
// values (a choice for each value made half of the kernel's instructions branches).
struct RouteScore {
    bool sigmoid;
    float from = 0.f, inv = 1.f;
    // from a row's logits; their scores in s
    template <int LANES, int VALUES>
    __device__ __forceinline__ void of_row(const float (&x)[VALUES], float (&s)[VALUES])
    {
        if (sigmoid) {
            (*this)(x, s);
            return;
        }
        const float top = row_all<OpMaxF, LANES>(largest(x));
        from = top == -kInf ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) sum += s[v] = exp2_fast((x[v] - from) * kLog2e);
        sum = row_all<OpSumF, LANES>(sum);
        inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) s[v] *= inv;
    }
    template <int VALUES>
    __device__ __forceinline__ void operator()(const float (&x)[VALUES], float (&s)[VALUES]) const
    {
        if (sigmoid) {
#pragma unroll
            for (int v = 0; v < VALUES; ++v) s[v] = __builtin_amdgcn_rcpf(1.f + exp2_fast(-x[v] * kLog2e));
        } else {
#pragma unroll
            for (int v = 0; v < VALUES; ++v) s[v] = exp2_fast((x[v] - from) * kLog2e) * inv;
        }
    }
};

template <int TYPE, int LANES, int VALUES, int KEPT>
__global__ __launch_bounds__(kThreads) void row_route_kernel(RouteArgs A)
{
    using T = Score<TYPE>;
    using Row = RouteRow<TYPE, LANES, VALUES>;
    constexpr int kRows = kThreads / LANES;
    __shared__ __align__(16) float held[kRows][places(Row::kColumns)];
    __shared__ float value[kRows][kMaxGroups];
    __shared__ uint32_t shut[kRows][kMaxGroups];
    const int at = threadIdx.x / LANES;
    const Row R{A.m, (int)(threadIdx.x % LANES)};
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < A.n; row0 += (int64_t)gridDim.x * kRows) {
        const bool there = row0 + at < A.n;
        const int64_t row = there ? row0 + at : A.n - 1;
        const typename T::Raw *const S = static_cast<const typename T::Raw *>(A.S) + row * A.ldS;
        float x[VALUES], key[VALUES];
        R.load(S, x);
        RouteScore score{A.score == REGOT_SIGMOID};
        float s[VALUES];
        score.template of_row<LANES>(x, s);
        if (A.bias) {
            if (A.bias_on == REGOT_BIAS_SCORE) {
#pragma unroll
                for (int v = 0; v < VALUES; ++v) key[v] = s[v];
            } else {
#pragma unroll
                for (int v = 0; v < VALUES; ++v) key[v] = x[v];
            }
            if (A.m > 0) {
#pragma unroll
                for (int c = 0; c < Row::kChunks; ++c) R.span(c).add_bias(key + c * T::kVec, A.bias);
            }
#pragma unroll
            for (int v = 0; v < VALUES; ++v) key[v] = x[v] == -kInf ? -kInf : key[v];
        } else {
#pragma unroll
            for (int v = 0; v < VALUES; ++v) key[v] = x[v];
        }
        const bool bad = row_any<LANES>(is_nan(largest(key)) || is_nan(score.inv));
        float *const mine = held[at];
        if (A.groups > 1 && A.m > 0) {
            wave_lds();
            // (without a bias, what groups are valued by is the score, but for forbidden columns)
#pragma unroll
            for (int v = 0; v < VALUES; ++v) s[v] = A.bias || key[v] == -kInf ? key[v] : s[v];
#pragma unroll
            for (int c = 0; c < Row::kChunks; ++c) {
                const Span<TYPE> span = R.span(c);
                float *const to = mine + place(span.first);
                if constexpr (T::kVec > 1) {
                    if (span.first == span.own && span.first % 4 == 0) {
#pragma unroll
                        for (int e = 0; e < T::kVec; e += 4) {
                            const f32x4 four = {s[c * T::kVec + e], s[c * T::kVec + e + 1], s[c * T::kVec + e + 2], s[c * T::kVec + e + 3]};
                            *reinterpret_cast<f32x4 *>(to + e) = four;
                        }
                        continue;
                    }
                }
#pragma unroll
                for (int e = 0; e < T::kVec; ++e)
                    if (span.first + e >= span.own) mine[place(span.first + e)] = s[c * T::kVec + e];
            }
            wave_lds();
            // the value of each group, by group_lanes lanes
            const int lanes = A.group_lanes, part = R.l & (lanes - 1);
            const uint32_t each = (A.group_size + lanes - 1) / lanes;
            for (int g = R.l / lanes; g < A.groups; g += LANES / lanes) {
                const uint32_t from = g * A.group_size + part * each, to = min(from + each, (uint32_t)(g + 1) * A.group_size);
                float first = -kInf, second = -kInf;
                if ((A.group_size | each) % 4 == 0) {
                    for (uint32_t j = from; j < to; j += 4) {
                        const f32x4 c = *reinterpret_cast<const f32x4 *>(mine + place(j));
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            second = __builtin_amdgcn_fmed3f(first, second, c[e]);  // (first >= second)
                            first = fmaxf(first, c[e]);
                        }
                    }
                } else {
                    for (uint32_t j = from; j < to; ++j) {
                        const float c = mine[place(j)];
                        second = __builtin_amdgcn_fmed3f(first, second, c);
                        first = fmaxf(first, c);
                    }
                }
                for (int d = 1; d < lanes; d *= 2) {
                    const float first_o = __shfl_xor(first, d), second_o = __shfl_xor(second, d);
                    second = fmaxf(fmaxf(second, second_o), fminf(first, first_o));
                    first = fmaxf(first, first_o);
                }
                // (two keys of the type's lowest value are still a group, which comes before one that has none)
                if (part == 0) value[at][g] = A.group_by == REGOT_GROUP_TOP2 && second > -kInf ? fmaxf(first + second, -__FLT_MAX__) : first;
            }
            wave_lds();
            for (int g = R.l; g < A.groups; g += LANES) {
                const float v = value[at][g];
                int better = 0;
                for (int o = 0; o < A.groups; ++o) better += before(value[at][o], o, v, g);
                shut[at][g] = better >= A.groups_kept;
            }
            wave_lds();
#pragma unroll
            for (int c = 0; c < Row::kChunks; ++c) {  // (a chunk lies in one group)
                const uint32_t first = R.span(c).first;
                if (shut[at][A.group_magic ? __umulhi(first, A.group_magic) : first]) {
#pragma unroll
                    for (int e = 0; e < T::kVec; ++e) key[c * T::kVec + e] = -kInf;
                }
            }
            wave_lds();
        }
        double best[KEPT];
        {
            constexpr int kList = VALUES < KEPT ? VALUES : KEPT;
            double list[VALUES];
#pragma unroll
            for (int v = 0; v < VALUES; ++v) list[v] = choice(key[v], R.column(v));
#pragma unroll
            for (int i = 0; i < VALUES; i += kList) sort_down<kList>(list + i);
#pragma unroll
            for (int i = 0; i < KEPT; ++i) best[i] = i < kList ? list[i] : no_choice();
#pragma unroll
            for (int p = kList; p < VALUES; p += kList) merge_lists<KEPT>(best, [&](int i) { return list[p + i]; });
        }
        merge_lists<KEPT>(best, [&](int i) { return dpp_f64<kDppXor1>(best[i]); });
        merge_lists<KEPT>(best, [&](int i) { return dpp_f64<kDppXor2>(best[i]); });
        merge_lists<KEPT>(best, [&](int i) { return dpp_f64<kDppHalfMirror>(best[i]); });
        if constexpr (LANES > 8) merge_lists<KEPT>(best, [&](int i) { return dpp_f64<kDppMirror>(best[i]); });
        if constexpr (LANES > 16) merge_lists<KEPT>(best, [&](int i) { return __shfl_xor(best[i], 16); });
        if constexpr (LANES == kLanes) merge_lists<KEPT>(best, [&](int i) { return __shfl_xor(best[i], 32); });
        constexpr int kRounds = (KEPT + LANES - 1) / LANES;
        int column[kRounds];
        float w[kRounds], at_chosen[kRounds], sum = 0.f;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            double c = no_choice();
#pragma unroll
            for (int i = r * LANES; i < KEPT && i < (r + 1) * LANES; ++i) c = R.l == i - r * LANES ? best[i] : c;
            const bool is = !bad && r * LANES + R.l < A.k && is_choice(c);
            column[r] = is ? (int)chosen_column(c) : -1;
            at_chosen[r] = is ? T::get(S[column[r]]) : 0.f;
        }
        score(at_chosen, w);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) sum += w[r] = column[r] < 0 ? 0.f : w[r];
        sum = row_all<OpSumF, LANES>(sum);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = r * LANES + R.l;
            if (!there || i >= A.k) continue;
            A.idx[row * A.k + i] = column[r];
            // (divided first: scale / sum is beyond 32 bits for the smallest sums)
            const float part = !A.renormalise ? w[r] : sum > 0.f ? w[r] / sum : 0.f;
            A.weight[row * A.k + i] = bad ? kNan : part * A.scale;
        }
    }
}

// dS at given choices: the row's scores again, the chosen columns' parts through LDS, one read and one write of the row.  Bound by
// memory: 65536 x 256 fp32, 8 choices 22-23 us = 5.8-6.1 TB/s of reads and writes.
// LIST: the room for a row's choices (8 or all there can be: 65536 x 64 fp32, 2 choices 5.5 us and 6.9).
template <int TYPE, int LANES, int VALUES, int LIST>
__global__ __launch_bounds__(kThreads) void row_route_grad_kernel(RouteArgs A)
{
    using T = Score<TYPE>;
    using Row = RouteRow<TYPE, LANES, VALUES>;
    constexpr int kRows = kThreads / LANES, kRounds = (LIST + LANES - 1) / LANES;
    __shared__ float held[kRows][Row::kColumns];
    __shared__ uint32_t listed[kRows][LIST];
    __shared__ float gradient[kRows][LIST];
    const int at = threadIdx.x / LANES;
    const Row R{A.m, (int)(threadIdx.x % LANES)};
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < A.n; row0 += (int64_t)gridDim.x * kRows) {
        const bool there = row0 + at < A.n;
        const int64_t row = there ? row0 + at : A.n - 1;
        const typename T::Raw *const S = static_cast<const typename T::Raw *>(A.S) + row * A.ldS;
        float x[VALUES];
        R.load(S, x);
        uint32_t column[kRounds];
        float g[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = r * LANES + R.l;
            column[r] = i < A.k ? (uint32_t)A.idx_in[row * A.k + i] : 0xffffffffu;
            g[r] = column[r] < A.m ? A.g_weight[row * A.k + i] * A.scale : 0.f;
        }
        float at_listed[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) at_listed[r] = column[r] < A.m ? T::get(S[column[r]]) : 0.f;
        RouteScore score{A.score == REGOT_SIGMOID};
        const bool sigmoid = score.sigmoid;
        const bool nan = is_nan(largest(x));
        float s[VALUES];
        score.template of_row<LANES>(x, s);
        const bool bad = row_any<LANES>(nan || is_nan(score.inv));  // (inv: a softmax with a score of +inf)
        float *const mine = held[at];
        float c[kRounds], Z = 0.f;
        bool any = false;
        score(at_listed, c);
        // sigmoid: s (1 - s), 1 - s being the score of -x (a difference of 1 and a score near it has lost its digits)
        float slope[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) slope[r] = -at_listed[r];
        score(slope, slope);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            slope[r] = sigmoid ? slope[r] : 1.f;
            c[r] = column[r] < A.m ? c[r] : 0.f;
            Z += c[r];
            any |= column[r] < A.m;
        }
        any = row_any<LANES>(any);
        float all = 0.f;
        if (A.renormalise) {
            // the chosen columns' part (g - sum g c / Z) c / Z, with c / Z formed first (g / Z is beyond 32 bits for the smallest sums) and
            // scores 2^40 times as large, so that g c and 1 / Z keep their digits; softmax has nothing elsewhere: the parts add up to 0
            float gs = 0.f;
#pragma unroll
            for (int r = 0; r < kRounds; ++r) {
                c[r] *= 0x1p40f;
                gs += column[r] < A.m ? g[r] * c[r] : 0.f;
            }
            Z = row_all<OpSumF, LANES>(Z) * 0x1p40f;
            const float inv_Z = Z <= 0.f ? 0.f : __builtin_amdgcn_rcpf(Z);
            gs = row_all<OpSumF, LANES>(gs) * inv_Z;
#pragma unroll
            for (int r = 0; r < kRounds; ++r) slope[r] *= c[r] * inv_Z;
#pragma unroll
            for (int r = 0; r < kRounds; ++r) g[r] -= gs;
        } else if (sigmoid) {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) slope[r] *= c[r];
        } else {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) all += column[r] < A.m ? g[r] * c[r] : 0.f;
            all = row_all<OpSumF, LANES>(all);
        }
        if (sigmoid || A.renormalise) {  // what is at a chosen column is all of its gradient
#pragma unroll
            for (int v = 0; v < VALUES; ++v) s[v] = 1.f;
        }
        // each column's part, a column listed twice having the sum of its entries'
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = r * LANES + R.l;
            if (i < A.k) listed[at][i] = column[r], gradient[at][i] = g[r];
        }
        wave_lds();
#pragma unroll
        for (int v = 0; v < VALUES; ++v) mine[v * LANES + R.l] = 0.f;
        wave_lds();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r * LANES >= A.k) continue;
            float sum = 0.f;
            for (int o = 0; o < A.k; ++o) sum += listed[at][o] == column[r] ? gradient[at][o] : 0.f;
            if (column[r] < A.m) mine[column[r]] = sum * slope[r];
        }
        wave_lds();
        typename T::Raw *const out = static_cast<typename T::Raw *>(A.dS) + row * A.ldD;
#pragma unroll
        for (int ch = 0; ch < Row::kChunks; ++ch) {
            const Span<TYPE> span(here((uint32_t)(ch * LANES + R.l) * T::kVec), A.m);  // (R.span(ch), but nothing of it kept since the load: 80 registers, not 85)
            if (!there || span.own >= A.m) continue;
            float d[T::kVec];
#pragma unroll
            for (int e = 0; e < T::kVec; ++e) {
                d[e] = s[ch * T::kVec + e] * (mine[span.first + e] - all);
            }
            if (bad || !any) {
#pragma unroll
                for (int e = 0; e < T::kVec; ++e) d[e] = bad ? kNan : 0.f;
            }
            span.store(out, d);
        }
        wave_lds();
    }
}

}  // namespace regot
