// Products grouped by expert: what the kernels share (gfx950, wave64).
//
// A product's rows are runs, one for each expert: rows start[e] .. start[e + 1] - 1 of Y belong to expert e.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "regot.h"
#include "regot_rows.hpp"

namespace regot {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// Division by the number k of choices of a token, for numbers below 2^31: with magic = ceil(2^shift / k), shift = 31 + ceil(log2 k), the
// quotient's error is below number * k / 2^shift < 1 of the last place.
struct Divide {
    uint32_t magic, shift;
};

inline Divide divide_by(uint32_t k)
{
    uint32_t shift = 31;
    while ((1ull << (shift - 31)) < k) ++shift;
    return {(uint32_t)(((1ull << shift) + k - 1) / k), shift};
}

struct GroupArgs {
    const int64_t *start;   // [experts + 1]
    int64_t rows;           // what start may reach
    int experts;
    const int32_t *order;   // row r takes row order[r] / k of X; NULL: row r
    Divide by_k;
    int64_t x_rows;
    const void *X;
    int64_t ldX;
    const void *W;          // weights, or the gradient dY of a weight gradient
    int64_t ldW, strideW;
    int64_t m, d;           // product: columns of Y (before the gate: of each half) and length of its sums; weight gradient: dW is m x d
    void *Y;                // product: rows; weight gradient: dW, or parts of it
    int64_t ldY, strideY;
    void *saved;
    int64_t ldSaved;
    uint32_t row_tiles, col_tiles, tiles;
    int splits;
    int groups;             // few rows: stretches of 32 rows of W that a workgroup has
    bool whole;             // results' rows are whole chunks of 16 bytes, and begin at multiples of 16 bytes
    int single;             // tiles are numbered by their first row (fewer rows than experts)
};

// The row of X that row r of the product takes.  (An entry that is none of X's rows is not followed beyond X.)
__device__ __forceinline__ int64_t row_of_slot(const GroupArgs &A, uint32_t slot)
{
    return min((int64_t)((uint64_t)slot * A.by_k.magic >> A.by_k.shift), A.x_rows - 1);
}
__device__ __forceinline__ int64_t source_row(const GroupArgs &A, int64_t r) { return A.order ? row_of_slot(A, A.order[r]) : r; }

// start[e], kept within the rows there are
__device__ __forceinline__ int64_t run_start(const GroupArgs &A, int e) { return min(max(A.start[e], (int64_t)0), A.rows); }

// Which rows tile t of BM rows has.  Tiles are numbered so that no sum over the experts is needed: those of expert e begin at
// start[e] / BM + e, which leaves each at least as many numbers as it has tiles (some of them, at most one an expert, are empty).  Where there
// are fewer rows than experts, tile t is the one that begins at row t, if one does.  A wave counts the experts before the tile, all lanes at once.
struct Run {
    int expert;
    int64_t first, end;  // rows of the tile: first .. min(first + BM, end) - 1; none where first >= end
};

// Whether tile t is behind those of expert i, whose run ends at `end`
template <int BM>
__host__ __device__ constexpr bool tile_is_behind(int end, int i, int64_t t, bool single)
{
    return single ? end <= t : end / BM + i + 1 <= t;
}

// Tile t where it is behind those of e experts: s is where the run of expert e begins, end where it ends
template <int BM>
__host__ __device__ constexpr Run run_of_tile(int e, int s, int end, int64_t t, bool single)
{
    if (single) return {e, t, t < s || (t - s) % BM != 0 ? t : end};
    const int64_t place = t - s / BM - e;  // among the expert's tiles; below 0: in front of the first run, no tile
    return {e, s + place * BM, place < 0 ? 0 : end};
}

template <int BM>
__device__ __forceinline__ Run find_run(const GroupArgs &A, int64_t t)
{
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x % kLanes;
    const int first_start = (int)run_start(A, 0);
    int e = 0, s = 0, end = 0x7fffffff;  // experts before the tile; the largest end of one of those, the smallest of another
    for (int i0 = lane; i0 - lane < A.experts; i0 += kAtOnce * kLanes) {
        int ends[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) ends[j] = (int)run_start(A, min(i0 + j * kLanes + 1, A.experts));
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = i0 + j * kLanes;
            const bool is = i < A.experts, before = is && tile_is_behind<BM>(ends[j], i, t, A.single);
            e += __popcll(__ballot(before));
            s = before ? max(s, ends[j]) : s;
            end = is && !before ? min(end, ends[j]) : end;
        }
    }
    if (e >= A.experts) return {0, 0, 0};
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) {
        s = max(s, __shfl_xor(s, d));
        end = min(end, __shfl_xor(end, d));
    }
    s = __builtin_amdgcn_readfirstlane(e == 0 ? first_start : s);
    end = __builtin_amdgcn_readfirstlane(end);
    e = __builtin_amdgcn_readfirstlane(e);
    return run_of_tile<BM>(e, s, end, t, A.single);
}

// Workgroups that follow each other run on different dies: each die gets a run of tiles, so that the tiles under way on one share
// their rows and their weights in its L2.
__device__ __forceinline__ uint32_t die_order(uint32_t b, uint32_t n)
{
    constexpr uint32_t kDies = 8;
    const uint32_t die = b % kDies, each = n / kDies, more = n % kDies;
    return die * each + min(die, more) + b / kDies;
}

// s(g) = 1 / (1 + exp(-g)).  The fast exponential is that of a rounded product with log2 e, so it is off by about |g| units of the last place: at most 2^-17 of itself before it
// is 0, which 16 bits do not see.  For results of 32 bits it is the exact one to a unit, of -|g|, so that it does not overflow where s(g) still has bits.
template <int TYPE>
__device__ __forceinline__ float sigmoid(float g)
{
    if constexpr (TYPE == REGOT_F32) {
        const float e = expf(-fabsf(g));
        return (g < 0.0f ? e : 1.0f) / (1.0f + e);
    }
    return 1.0f / (1.0f + __expf(-g));
}

}  // namespace regot
