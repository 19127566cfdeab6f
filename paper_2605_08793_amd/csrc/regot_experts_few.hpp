// Products grouped by expert where each has few rows: the weights straight from memory into the matrix instructions (gfx950, wave64).
#pragma once

#include "regot_experts_tile.hpp"

namespace regot {

constexpr int kFewWaves = 8, kFewAhead = 4;  // units of 128 bytes of each of 32 rows that a wave has under way
constexpr int kFewUnits = 16;                // units of a sum that a wave can have

// A workgroup: 16 rows and a stretch of W's rows, 32 at a time (with the gate 16 of g and the 16 of u that belong to them).  What bounds this is the
// reading of the weights, once each, so everything is for keeping loads under way: each wave has its share of the sum, a unit of 128 bytes of each row at a time (so that
// a workgroup reads 1 KB of each of 32 rows), which it loads into its own part of LDS, four units ahead and across the ends of sums, without
// registers and without waiting for another wave.  The rows' numbers stay in registers.  The waves' sums are added up in their order, by each wave in turn.
// Measured: 64 tokens x 4 of 60 experts, 1400 x 2048 fp16 69 us = 5.0 TB/s; one token, 8 of 256, 2048 by 2 x 1024 bf16 14 us = 4.8 TB/s; sums of 3712, 864 rows of 229, 2 x
// 64 bf16 46 us = 4.8 TB/s.  (Loads alone in the same order reach 5.4 TB/s
// on rows of 2800 bytes and 6.0 on rows of whole lines; a workgroup's begin, until its first numbers are there, is what is missing.)
template <int TYPE, bool GATE, int MOST>
__global__ void __launch_bounds__(kFewWaves *kLanes) expert_few_kernel(const GroupArgs A)
{
    using Raw = typename Score<TYPE>::Raw;
    using Cols = Side<TYPE, 32, false, kLanes>;
    constexpr int kElem = sizeof(Raw), kChunk = 16 / kElem, kUnit = 128 / kElem, kLoads = 4, kUnitBytes = kLoads * 1024;
    __shared__ __attribute__((aligned(1024))) char lds[kFewWaves * kFewAhead * kUnitBytes];
    __shared__ f32x4 parts[2][kFewWaves][2][kLanes];
    const uint32_t b = blockIdx.x;  // (neighbours share 16 rows of X alone, and every die gets as many that are not empty)
    const Run run = find_run<16>(A, b / A.col_tiles);
    if (run.first >= run.end) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), lane = threadIdx.x % kLanes, g = lane / 16, i = lane % 16;
    constexpr int kCols = GATE ? 16 : 32;
    const int64_t col0 = (int64_t)(b % A.col_tiles) * A.groups * kCols;
    const int groups = (int)min((int64_t)A.groups, (A.m - col0 + kCols - 1) / kCols);
    const int units = (int)((A.d + kUnit - 1) / kUnit), mine = (units - wave + kFewWaves - 1) / kFewWaves;  // of the sum, and this wave's
    char *const at = lds + wave * kFewAhead * kUnitBytes;
    const uint32_t at_address = lds_address(at);

    // loads j: rows 8 j + lane / 8 of the 32 of W, in the order of Side
    const char *const W = static_cast<const char *>(A.W) + run.expert * A.strideW * kElem;
    const char *w[kLoads];
    int w_chunk[kLoads];
    int group = 0, unit = wave;  // of what is loaded next
    const auto next_group = [&] {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int row = 8 * j + lane / 8;
            w_chunk[j] = (lane % 8) ^ Cols::turn(row);
            const int64_t c = col0 + (int64_t)group * kCols + (GATE ? row / 8 * 4 + row % 4 : row);
            w[j] = W + (min(c, A.m - 1) + (GATE && row & 4 ? A.m : 0)) * A.ldW * kElem + w_chunk[j] * 16;
        }
    };
    const auto load = [&](int slot) {
        const int64_t k = (int64_t)unit * kUnit;
        const bool last = k + kUnit > A.d;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *p = w[j] + k * kElem;
            if (last && k + w_chunk[j] * kChunk >= A.d) p = reinterpret_cast<const char *>(kNoNumbers);
            load_to_lds(p, at_address + slot * kUnitBytes + j * 1024);
        }
        unit += kFewWaves;
        if (unit >= units) {
            unit = wave;
            ++group;
            next_group();
        }
    };
    next_group();
    const int all = groups * mine;
    if (mine > 0) {
#pragma unroll
        for (int s = 0; s < kFewAhead; ++s)
            if (s < all) load(s);
    }
    // row i of X at this wave's units
    u32x4 x[MOST][2];
    const char *const X = static_cast<const char *>(A.X) + source_row(A, min(run.first + i, run.end - 1)) * A.ldX * kElem;
#pragma unroll
    for (int u = 0; u < MOST; ++u)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int64_t k = (int64_t)(wave + u * kFewWaves) * kUnit + (half * 4 + g) * kChunk;
            x[u][half] = u32x4{0, 0, 0, 0};
            if (k < A.d) x[u][half] = *(const __attribute__((address_space(1))) u32x4 *)(X + k * kElem);
        }
#pragma unroll
    for (int u = 0; u < MOST; ++u)
#pragma unroll
        for (int half = 0; half < 2; ++half) asm volatile("" : "+v"(x[u][half]));  // (there before the loop, in which nothing but W is waited for)

    const int64_t r = run.first + i;
    const auto store = [&](void *to, int64_t ld, int64_t c, const float *v, int64_t left) {
        Raw part[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = Score<TYPE>::put(v[e]);
        store_run<TYPE, 4>(static_cast<char *>(to) + (r * ld + c) * kElem, part, left, A.whole);
    };
    int slot = 0, s = 0;
    for (int of = 0; of < groups; ++of) {
        f32x4 acc[2] = {};
#pragma unroll
        for (int u = 0; u < MOST; ++u) {
            if (u >= mine) continue;  // (an exit of the loop would leave it as a loop, and x in memory)
            // (this unit's loads are the oldest)
            const int behind = min(all - 1 - s, kFewAhead - 1);
            if (behind == 3) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
            else if (behind == 2) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
            else if (behind == 1) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const char *from = at + slot * kUnitBytes;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int f = 0; f < 2; ++f) acc[f] = multiply<TYPE>(Cols::fragment(from, 0, f, half), x[u][half], acc[f]);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (s + kFewAhead < all) load(slot);
            slot = slot + 1 < kFewAhead ? slot + 1 : 0;
            ++s;
        }
        // (the place of a sum is written again two sums later, when the wave that added it up has met the others)
        f32x4(&sums)[kFewWaves][2][kLanes] = parts[of & 1];
#pragma unroll
        for (int f = 0; f < 2; ++f) sums[wave][f][lane] = acc[f];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // (a barrier that waits for loads on their way would stop them)
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if (wave != of % kFewWaves || r >= run.end) continue;
        float v[2][4];  // 4 neighbours of row i in each fragment
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            f32x4 sum = sums[0][f][lane];
#pragma unroll
            for (int p = 1; p < kFewWaves; ++p) sum += sums[p][f][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[f][e] = sum[e];
        }
        const int64_t c = col0 + (int64_t)of * kCols + (GATE ? 4 : 8) * g;
        if (c >= A.m) continue;
        if constexpr (GATE) {
            float h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = v[0][e] * sigmoid<TYPE>(v[0][e]) * v[1][e];
            store(A.Y, A.ldY, c, h, A.m - c);
            if (A.saved) {
                store(A.saved, A.ldSaved, c, v[0], A.m - c);
                store(A.saved, A.ldSaved, A.m + c, v[1], A.m - c);
            }
        } else {
            store(A.Y, A.ldY, c, v[0], A.m - c);
            store(A.Y, A.ldY, c + 4, v[1], A.m - c - 4);
        }
    }
}

}  // namespace regot
