// The norm over many tensors, and clipping (gfx950, wave64).
//
// One read for the partial sums, in 64 bits so that no square is lost, and another with the writing, which begins with what was read last (some of it is in the caches).  Memory bounds both: 300
// tensors, 1.2 GB bf16: sums 210 us = 5.7 TB/s, the scaled copy 464 = 5.2; 24 tensors of 12 MB fp32 below the limit 7 and 5 us.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "regot.h"
#include "regot_device.hpp"
#include "regot_rows.hpp"

namespace regot {

constexpr int kListed = 100;  // tensors of a launch: its arguments hold them (4 KB at most), so that no list has to be copied to the device

struct ListedTensor {
    const void *data;
    void *out;
    int64_t count;
    uint32_t first;  // its first workgroup
    int32_t type;
};

struct ClipArgs {
    ListedTensor list[kListed];
    int tensors;
    uint32_t blocks;     // of this launch
    uint32_t part;       // this launch's first partial sum
    uint32_t parts;      // partial sums of all launches
    int64_t each;        // numbers of a workgroup, a multiple of 8 kThreads
    double max_norm;
    double *sums;        // [parts]
    float *norm, *factor;
    int backwards;       // the last workgroup's numbers first
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ int listed(const ClipArgs &A, uint32_t block)
{
    const int lane = threadIdx.x % kLanes;
    int t = -1;
    for (int i = lane; i < (A.tensors + kLanes - 1) / kLanes * kLanes; i += kLanes) t += __popcll(__ballot(i < A.tensors && A.list[min(i, A.tensors - 1)].first <= block));
    return t;
}

template <int TYPE>
__device__ __forceinline__ double sum_of_squares(const ListedTensor &T, int64_t from, int64_t to)
{
    using S = Score<TYPE>;
    using Raw = typename S::Raw;
    typedef u32x4 Any __attribute__((aligned(alignof(uint16_t))));
    const Raw *x = static_cast<const Raw *>(T.data);
    double sum[2] = {0.0, 0.0};
    constexpr int kAtOnce = 4;
    int64_t i = from + (int64_t)threadIdx.x * S::kVec;
    for (; i + (kAtOnce - 1) * kThreads * S::kVec + S::kVec <= to; i += kAtOnce * kThreads * S::kVec) {
        u32x4 raw[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) raw[j] = *reinterpret_cast<const Any *>(x + i + j * kThreads * S::kVec);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            float v[S::kVec];
            S::unpack(raw[j], v);
#pragma unroll
            for (int e = 0; e < S::kVec; ++e) sum[e & 1] = fma((double)v[e], (double)v[e], sum[e & 1]);
        }
    }
    for (; i < to; i += kThreads * S::kVec)
        for (int e = 0; e < S::kVec && i + e < to; ++e) {
            const double v = S::get(x[i + e]);
            sum[0] = fma(v, v, sum[0]);
        }
    return sum[0] + sum[1];
}

__device__ __forceinline__ double block_total(double v)
{
    __shared__ double lds[kWaves];
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) v += __shfl_xor(v, d);
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = v;
    __syncthreads();
    double r = lds[0];
    for (int w = 1; w < kWaves; ++w) r += lds[w];
    __syncthreads();
    return r;
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const ClipArgs A)
{
    const ListedTensor &T = A.list[listed(A, blockIdx.x)];
    const int64_t from = (blockIdx.x - T.first) * A.each, to = min(from + A.each, T.count);
    double v;
    if (T.type == REGOT_F32) v = sum_of_squares<REGOT_F32>(T, from, to);
    else if (T.type == REGOT_BF16) v = sum_of_squares<REGOT_BF16>(T, from, to);
    else v = sum_of_squares<REGOT_F16>(T, from, to);
    v = block_total(v);
    if (threadIdx.x == 0) A.sums[A.part + blockIdx.x] = v;
}

// norm and factor from the partial sums, the same in every workgroup that asks; A.parts of them
__device__ __forceinline__ float clip_factor(const ClipArgs &A, bool tell)
{
    double v = 0.0;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < A.parts; i += kThreads) v += A.sums[i];
    const double norm = sqrt(block_total(v));
    const float told = (float)norm;  // (decided on this one: a norm that a program sees as an infinity has scaled nothing)
    const float factor = norm > A.max_norm && told < __builtin_inff() ? (float)(A.max_norm / norm) : 1.f;
    if (tell && threadIdx.x == 0) {
        A.norm[0] = told;
        if (A.factor) A.factor[0] = factor;
    }
    return factor;
}

__global__ void __launch_bounds__(kThreads) grad_factor_kernel(const ClipArgs A) { clip_factor(A, true); }

template <int TYPE>
__device__ __forceinline__ void scale(const ListedTensor &T, int64_t from, int64_t to, float factor)
{
    using S = Score<TYPE>;
    using Raw = typename S::Raw;
    typedef u32x4 Any __attribute__((aligned(alignof(uint16_t))));
    const Raw *x = static_cast<const Raw *>(T.data);
    Raw *out = static_cast<Raw *>(T.out);
    constexpr int kAtOnce = 4;
    int64_t i = from + (int64_t)threadIdx.x * S::kVec;
    const auto one = [&](u32x4 raw, int64_t at) {
        float v[S::kVec];
        Raw part[S::kVec];
        S::unpack(raw, v);
#pragma unroll
        for (int e = 0; e < S::kVec; ++e) part[e] = S::put(v[e] * factor);
        __builtin_nontemporal_store(S::pack(part), reinterpret_cast<Any *>(out + at));
    };
    for (; i + (kAtOnce - 1) * kThreads * S::kVec + S::kVec <= to; i += kAtOnce * kThreads * S::kVec) {
        u32x4 raw[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) raw[j] = *reinterpret_cast<const Any *>(x + i + j * kThreads * S::kVec);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) one(raw[j], i + j * kThreads * S::kVec);
    }
    for (; i < to; i += kThreads * S::kVec)
        for (int e = 0; e < S::kVec && i + e < to; ++e) out[i + e] = S::put(S::get(x[i + e]) * factor);
}

// SUMS: each workgroup adds the partial sums up itself (few of them); otherwise the factor is there
template <bool SUMS>
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const ClipArgs A)
{
    const uint32_t b = A.backwards ? A.blocks - 1 - blockIdx.x : blockIdx.x;
    const float factor = SUMS ? clip_factor(A, A.part + b == 0) : A.factor[0];
    const ListedTensor &T = A.list[listed(A, b)];
    if (factor == 1.f && T.data == T.out) return;
    const int64_t from = (b - T.first) * A.each, to = min(from + A.each, T.count);
    if (T.type == REGOT_F32) scale<REGOT_F32>(T, from, to, factor);
    else if (T.type == REGOT_BF16) scale<REGOT_BF16>(T, from, to, factor);
    else scale<REGOT_F16>(T, from, to, factor);
}

}  // namespace regot
