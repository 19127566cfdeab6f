// Products grouped by expert: tiles of a matrix product on the matrix cores (gfx950, wave64).
#pragma once

#include "regot_experts.hpp"

namespace regot {

// What a tile's product becomes: stored; put through the gate; put through the gate's gradient; a weight gradient's (part of a) sum
enum { kPlain = 0, kGate = 1, kGateGrad = 2, kWeightGrad = 3 };

__device__ const uint32_t kNoNumbers[8] = {};  // what is loaded in the place of numbers that are not there: 0

typedef __attribute__((address_space(3))) uint32_t LdsWord;
typedef const __attribute__((address_space(1))) uint32_t GlobalWord;

// One side of a tile: EXT rows (or columns) of a matrix, 128 bytes of each along the sum at a time.  LDS holds them
//   TRANS = false (numbers along the sum are neighbours in memory): row after row, 8 chunks of 16 bytes each
//   TRANS = true (the matrix is read across): for each of the kSum places of the sum its EXT numbers
// with the chunks of a row in an order that depends on the row, so that the lanes that read together meet different banks.
// Row of fragment f (16 rows) that lane i (of 16) reads, from the pair p = f / 2 on:
//   TRANS = false 32 p + 8 (i / 4) + 4 (f % 2) + i % 4 (so that a lane's results are 8 neighbours), TRANS = true 16 f + i
template <int TYPE, int EXT, bool TRANS, int THREADS>
struct Side {
    using Raw = typename Score<TYPE>::Raw;
    static constexpr int kElem = sizeof(Raw), kChunk = 16 / kElem, kSum = 128 / kElem;
    static constexpr int kBytes = EXT * 128, kLoads = kBytes / (16 * THREADS);
    static constexpr int kRowChunks = TRANS ? EXT / kChunk : 8;
    static_assert(kLoads * 16 * THREADS == kBytes, "every thread loads whole chunks");

    static __device__ __forceinline__ int turn(int row)
    {
        if constexpr (TRANS) return (((row & 3) | ((row >> 3) & 1) << 2) << 1) & (kRowChunks - 1);
        return ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
    }
    // place ii of this thread: row of LDS and chunk of it
    static __device__ __forceinline__ int place(int ii)
    {
        const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
        return (wave * kLoads + ii) * kLanes + lane;
    }
    static __device__ __forceinline__ int lds_row(int ii) { return place(ii) / kRowChunks; }
    static __device__ __forceinline__ int chunk(int ii) { return (place(ii) % kRowChunks) ^ turn(lds_row(ii)); }

    // the 16 bytes of a fragment that lane (16 g + i) has at step `step` of 64 bytes along the sum
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int f0, int f, int step)
    {
        const int lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
        if constexpr (!TRANS) {
            const int row = f0 * 16 + (f / 2) * 32 + 8 * (i / 4) + 4 * (f % 2) + i % 4;
            return *reinterpret_cast<const u32x4 *>(lds + row * 128 + ((step * 4 + g) ^ turn(row)) * 16);
        } else if constexpr (kElem == 2) {
            u32x4 v;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = step * 32 + 8 * g + 4 * h + i / 4, at = (f0 + f) * 16 + 4 * (i % 4);
                const char *from = lds + k * (EXT * 2) + ((at / 8) ^ turn(k)) * 16 + (at % 8) * 2;
                const i16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(const_cast<char *>(from)));
                __builtin_memcpy(reinterpret_cast<char *>(&v) + 8 * h, &part, 8);
            }
            return v;
        } else {
            u32x4 v;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = step * 16 + 4 * g + s, at = (f0 + f) * 16 + i;
                v[s] = *reinterpret_cast<const uint32_t *>(lds + k * (EXT * 4) + ((at / 4) ^ turn(k)) * 16 + (at % 4) * 4);
            }
            return v;
        }
    }
};

// Loads of one side, kSum places of the sum at a time.  DIRECT: whole chunks that are 16 bytes aligned, from memory straight into LDS;
// otherwise through registers, at any alignment, numbers beyond the matrix as 0.
template <int TYPE, int EXT, bool TRANS, int THREADS, bool DIRECT, bool GATHER, bool HALVES>
struct Loader {
    using S = Side<TYPE, EXT, TRANS, THREADS>;
    using Raw = typename S::Raw;
    const char *at[S::kLoads];  // of the next chunks
    int64_t step;               // to those after them
    u32x4 kept[DIRECT ? 1 : S::kLoads];
    int next_row[GATHER ? S::kLoads : 1];
    int64_t ld;

    // TRANS = false: row(i) is the address of the i-th row, from the sum's first place on
    template <typename Row>
    __device__ __forceinline__ void rows(Row row)
    {
        step = 128;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) at[ii] = row(S::lds_row(ii)) + S::chunk(ii) * 16;
    }
    // TRANS = true: the matrix at p, numbers first .. extent - 1 of its rows, whose distance is ld_ numbers.  HALVES: half of the tile's are
    // those, and half the numbers of the same places behind extent.
    static __device__ __forceinline__ int column(int ii) { return S::chunk(ii) * S::kChunk % (HALVES ? EXT / 2 : EXT); }
    __device__ __forceinline__ void across(const char *p, int64_t ld_, int64_t first, int64_t extent)
    {
        ld = ld_ * S::kElem;
        step = S::kSum * ld;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) {
            int64_t c = first + column(ii);
            if constexpr (DIRECT) c = min(c, extent - S::kChunk);  // (what is loaded there is not used)
            if (HALVES && S::chunk(ii) * S::kChunk >= EXT / 2) c += extent;
            at[ii] = p + c * S::kElem + (GATHER ? 0 : S::lds_row(ii) * ld);
        }
    }
    // which rows of the matrix the places done .. done + kSum - 1 of a gathered sum are
    __device__ __forceinline__ void gather(const GroupArgs &A, int64_t row, int64_t end)
    {
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) next_row[ii] = (int)source_row(A, min(row + S::lds_row(ii), end - 1));
    }
    // the chunks of places done .. of a sum of `sum` places; first, extent: as for across
    __device__ __forceinline__ void load(char *lds, int64_t done, int64_t sum, int64_t first, int64_t extent)
    {
        const bool last = done + S::kSum > sum;
#pragma unroll
        for (int ii = 0; ii < S::kLoads; ++ii) {
            const char *p = at[ii];
            if constexpr (GATHER) p += (int64_t)next_row[ii] * ld;
            else at[ii] += step;
            const int64_t k = done + (TRANS ? S::lds_row(ii) : S::chunk(ii) * S::kChunk);
            if constexpr (DIRECT) {
                if (last && k >= sum) p = reinterpret_cast<const char *>(kNoNumbers);
                const int wave = threadIdx.x / kLanes;
                __builtin_amdgcn_global_load_lds((GlobalWord *)p, (LdsWord *)(lds + (wave * S::kLoads + ii) * 1024), 16, 0, 0);
            } else {
                const int64_t left = TRANS ? (k < sum ? extent - first - column(ii) : 0) : sum - k;
                u32x4 v = {0, 0, 0, 0};
                if (left >= S::kChunk) {
                    __builtin_memcpy(&v, p, 16);
                } else {
                    Raw part[S::kChunk];
#pragma unroll
                    for (int c = 0; c < S::kChunk; ++c) part[c] = c < left ? reinterpret_cast<const Raw *>(p)[c] : Raw(0.f);
                    __builtin_memcpy(&v, part, 16);
                }
                kept[ii] = v;
            }
        }
    }
    __device__ __forceinline__ void put(char *lds)
    {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int ii = 0; ii < S::kLoads; ++ii) *reinterpret_cast<u32x4 *>(lds + S::place(ii) * 16) = kept[ii];
        }
    }
};

template <int TYPE>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (TYPE == REGOT_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (TYPE == REGOT_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c, 0, 0, 0);
        return c;
    }
}

// COUNT neighbouring results to a row of `left` (or more) numbers, the first of them at p
template <int TYPE, int COUNT, bool WHOLE>
__device__ __forceinline__ void store_run(void *p, const float *v, int64_t left)
{
    using Raw = typename Score<TYPE>::Raw;
    Raw part[COUNT];
#pragma unroll
    for (int c = 0; c < COUNT; ++c) part[c] = Score<TYPE>::put(v[c]);
    if constexpr (WHOLE) {
        if (left > 0) __builtin_memcpy(__builtin_assume_aligned(p, sizeof(part) < 16 ? sizeof(part) : 16), part, sizeof(part));
    } else {
#pragma unroll
        for (int c = 0; c < COUNT; ++c)
            if (c < left) static_cast<Raw *>(p)[c] = part[c];
    }
}

template <int TYPE, int COUNT, bool WHOLE>
__device__ __forceinline__ void load_run(float *v, const void *p, int64_t left)
{
    using Raw = typename Score<TYPE>::Raw;
    Raw part[COUNT];
    if constexpr (WHOLE) {
        __builtin_memcpy(part, __builtin_assume_aligned(p, sizeof(part) < 16 ? sizeof(part) : 16), sizeof(part));
    } else {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) part[c] = c < left ? static_cast<const Raw *>(p)[c] : Raw(0.f);
    }
#pragma unroll
    for (int c = 0; c < COUNT; ++c) v[c] = Score<TYPE>::get(part[c]);
}

// A tile of BM rows and BN columns, WM x WN waves.  Columns come first in the matrix instruction, so that a lane's four results are neighbours
// in a row.  Rows: of X (product), or columns of dY (weight gradient, summed over rows).  Columns: rows of W (of its columns where ACROSS;
// with the gate half of them are g's and half u's), or columns of X.
template <int TYPE, int BM, int BN, int WM, int WN, bool ACROSS, int KIND, bool DIRECT, int OUT, bool GATHER>
__global__ void __launch_bounds__(WM *WN *kLanes) expert_tile_kernel(const GroupArgs A)
{
    constexpr int kThreadsHere = WM * WN * kLanes;
    constexpr bool kAcrossRows = KIND == kWeightGrad;
    using Rows = Side<TYPE, BM, kAcrossRows, kThreadsHere>;
    using Cols = Side<TYPE, BN, ACROSS, kThreadsHere>;
    using Raw = typename Score<TYPE>::Raw;
    constexpr int kElem = sizeof(Raw), kSum = Rows::kSum;
    constexpr int kFragRows = BM / WM / 16, kFragCols = BN / WN / 16;
    static_assert(kFragCols % 2 == 0 && (kAcrossRows || kFragRows % 2 == 0), "fragments come in pairs");
    __shared__ __attribute__((aligned(1024))) char rows0[Rows::kBytes], cols0[Cols::kBytes], rows1[Rows::kBytes], cols1[Cols::kBytes];

    const uint32_t b = die_order(blockIdx.x, A.tiles);
    Loader<TYPE, BM, kAcrossRows, kThreadsHere, DIRECT, false, false> rows;
    Loader<TYPE, BN, ACROSS, kThreadsHere, DIRECT, KIND == kWeightGrad && GATHER, KIND == kGate> cols;
    int64_t first_row, row_end, first_col, col_end, sum, from = 0;
    int expert, part = 0;
    if constexpr (KIND == kWeightGrad) {
        const uint32_t per = A.row_tiles * A.col_tiles, tile = b % per;
        expert = b / per % A.experts;
        part = b / per / A.experts;
        first_row = (int64_t)(tile / A.col_tiles) * BM;
        first_col = (int64_t)(tile % A.col_tiles) * BN;
        row_end = A.m;
        col_end = A.d;
        const int64_t s = run_start(A, expert), count = max(run_start(A, expert + 1) - s, (int64_t)0);
        const int64_t each = ((count + kSum - 1) / kSum + A.splits - 1) / A.splits * kSum;
        from = s + min(part * each, count);
        sum = min(each, count - min(part * each, count));
        rows.across(static_cast<const char *>(A.W) + from * A.ldW * kElem, A.ldW, first_row, row_end);
        cols.across(static_cast<const char *>(A.X) + (GATHER ? 0 : from * A.ldX * kElem), A.ldX, first_col, col_end);
        if constexpr (GATHER)
            if (sum > 0) cols.gather(A, from, from + sum);
    } else {
        const Run run = find_run<BM>(A, b / A.col_tiles);
        if (run.first >= run.end) return;
        expert = run.expert;
        first_row = run.first;
        row_end = run.end;
        first_col = (int64_t)(b % A.col_tiles) * (KIND == kGate ? BN / 2 : BN);
        col_end = A.m;
        sum = A.d;
        const char *W = static_cast<const char *>(A.W) + expert * A.strideW * kElem;
        rows.rows([&](int i) { return static_cast<const char *>(A.X) + source_row(A, min(first_row + i, row_end - 1)) * A.ldX * kElem; });
        if constexpr (ACROSS) {
            cols.across(W, A.ldW, first_col, col_end);
        } else {
            cols.rows([&](int i) {
                const int64_t c = KIND == kGate ? min(first_col + i % (BN / 2), col_end - 1) + (i >= BN / 2 ? col_end : 0) : min(first_col + i, col_end - 1);
                return W + c * A.ldW * kElem;
            });
        }
    }

    const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
    const int wm = wave / WN, wn = wave % WN;
    // with the gate a wave's columns are kFragCols / 2 fragments of g and as many of u
    const auto col_fragment = [&](const char *lds, int f, int step) {
        if constexpr (KIND == kGate) {
            constexpr int kHalf = kFragCols / 2;
            return Cols::fragment(lds, (f < kHalf ? 0 : BN / 32) + wn * kHalf, f % kHalf, step);
        } else {
            return Cols::fragment(lds, wn * kFragCols, f, step);
        }
    };
    f32x4 acc[kFragRows][kFragCols] = {};
    const auto compute = [&](const char *r, const char *c) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            u32x4 fr[kFragRows], fc[kFragCols];
#pragma unroll
            for (int f = 0; f < kFragCols; ++f) fc[f] = col_fragment(c, f, step);
#pragma unroll
            for (int f = 0; f < kFragRows; ++f) fr[f] = Rows::fragment(r, wm * kFragRows, f, step);
#pragma unroll
            for (int x = 0; x < kFragRows; ++x)
#pragma unroll
                for (int y = 0; y < kFragCols; ++y) acc[x][y] = multiply<TYPE>(fc[y], fr[x], acc[x][y]);
        }
    };
    int64_t done = 0;
    const auto load = [&](char *r, char *c) {
        rows.load(r, done, sum, first_row, row_end);
        cols.load(c, done, sum, first_col, col_end);
        done += kSum;
        if constexpr (KIND == kWeightGrad && GATHER)
            if (done < sum) cols.gather(A, from + done, from + sum);
    };
    const auto put = [&](char *r, char *c) {
        rows.put(r);
        cols.put(c);
    };
    const auto all_there = [&] {
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (this wave's loads into LDS; the barrier: everybody's)
        __syncthreads();
    };
    if (sum > 0) {
        load(rows0, cols0);
        put(rows0, cols0);
        for (int64_t t = 0;; t += 2 * kSum) {
            all_there();
            if (t + kSum < sum) load(rows1, cols1);
            compute(rows0, cols0);
            if (t + kSum >= sum) break;
            put(rows1, cols1);
            all_there();
            if (t + 2 * kSum < sum) load(rows0, cols0);
            compute(rows1, cols1);
            if (t + 2 * kSum >= sum) break;
            put(rows0, cols0);
        }
    }

    // results: fragments y and y + 1 of a pair are 8 neighbours of a row, or two runs of 4
    constexpr int kOutElem = sizeof(typename Score<OUT>::Raw);
    const auto row_of = [&](int x) {
        return first_row + (wm * kFragRows + (kAcrossRows ? x : x / 2 * 2)) * 16 + (kAcrossRows ? i : 8 * (i / 4) + 4 * (x % 2) + i % 4);
    };
    constexpr int kRun = ACROSS ? 4 : 8;
    if constexpr (KIND == kGate) {
        constexpr int kHalf = kFragCols / 2;
        static_assert(KIND != kGate || kHalf % 2 == 0, "halves are pairs of fragments");
#pragma unroll
        for (int x = 0; x < kFragRows; ++x) {
            const int64_t r = row_of(x);
            if (r >= row_end) continue;
#pragma unroll
            for (int y = 0; y < kHalf; y += kRun / 4) {
                const int64_t c = first_col + (wn * kHalf + y) * 16 + kRun * g;
                float gate[kRun], up[kRun], h[kRun];
#pragma unroll
                for (int e = 0; e < kRun; ++e) {
                    gate[e] = acc[x][y + e / 4][e % 4];
                    up[e] = acc[x][kHalf + y + e / 4][e % 4];
                    h[e] = gate[e] * sigmoid(gate[e]) * up[e];
                }
                store_run<TYPE, kRun, DIRECT>(static_cast<char *>(A.Y) + (r * A.ldY + c) * kElem, h, col_end - c);
                if (A.saved) {
                    char *s = static_cast<char *>(A.saved) + (r * A.ldSaved + c) * kElem;
                    store_run<TYPE, kRun, DIRECT>(s, gate, col_end - c);
                    store_run<TYPE, kRun, DIRECT>(s + col_end * kElem, up, col_end - c);
                }
            }
        }
    } else {
        char *Y = static_cast<char *>(A.Y);
        if constexpr (KIND == kWeightGrad) Y += ((int64_t)part * A.experts + expert) * A.strideY * kOutElem;
#pragma unroll
        for (int x = 0; x < kFragRows; ++x) {
            const int64_t r = row_of(x);
            if (r >= row_end) continue;
#pragma unroll
            for (int y = 0; y < kFragCols; y += kRun / 4) {
                const int64_t c = first_col + (wn * kFragCols + y) * 16 + kRun * g;
                float v[kRun];
#pragma unroll
                for (int e = 0; e < kRun; ++e) v[e] = acc[x][y + e / 4][e % 4];
                if constexpr (KIND == kGateGrad) {
                    if (c >= col_end) continue;
                    const char *s = static_cast<const char *>(A.saved) + (r * A.ldSaved + c) * kElem;
                    float gate[kRun], up[kRun];
                    load_run<TYPE, kRun, DIRECT>(gate, s, col_end - c);
                    load_run<TYPE, kRun, DIRECT>(up, s + col_end * kElem, col_end - c);
#pragma unroll
                    for (int e = 0; e < kRun; ++e) {
                        const float p = sigmoid(gate[e]), D = v[e];
                        v[e] = D * up[e] * (p * (1.0f + gate[e] * (1.0f - p)));
                        up[e] = D * (gate[e] * p);
                    }
                    store_run<TYPE, kRun, DIRECT>(Y + (r * A.ldY + c) * kElem, v, col_end - c);
                    store_run<TYPE, kRun, DIRECT>(Y + (r * A.ldY + col_end + c) * kElem, up, col_end - c);
                } else {
                    store_run<OUT, kRun, DIRECT>(Y + (r * A.ldY + c) * kOutElem, v, col_end - c);
                }
            }
        }
    }
}

}  // namespace regot
