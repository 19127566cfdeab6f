// Row operators on scores in fp32, bf16 or fp16: what their kernels share (gfx950, wave64).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "regot.h"
#include "regot_device.hpp"

namespace regot {

constexpr float kInf = __builtin_inff();
constexpr float kNan = __builtin_nanf("");
constexpr float kLn2 = 0.693147180559945309417f;

// A score as a 32-bit number, and back (rounded to nearest even, once).
template <int TYPE>
struct Score;
template <>
struct Score<REGOT_F32> {
    using Raw = float;
    static __device__ __forceinline__ float get(Raw v) { return v; }
    static __device__ __forceinline__ Raw put(float v) { return v; }
};
template <>
struct Score<REGOT_BF16> {
    using Raw = __bf16;
    static __device__ __forceinline__ float get(Raw v) { return (float)v; }
    static __device__ __forceinline__ Raw put(float v) { return (__bf16)v; }
};
template <>
struct Score<REGOT_F16> {
    using Raw = _Float16;
    static __device__ __forceinline__ float get(Raw v) { return (float)v; }
    static __device__ __forceinline__ Raw put(float v) { return (_Float16)v; }
};

// 2^t by the hardware's exponential (within 1 unit in the last place; results below the smallest normal number are 0)
__device__ __forceinline__ float exp2_fast(float t) { return __builtin_amdgcn_exp2f(t); }

struct OpSumF {
    static __device__ __forceinline__ float apply(float a, float b) { return a + b; }
};
struct OpMaxF {
    static __device__ __forceinline__ float apply(float a, float b) { return fmaxf(a, b); }
};

template <typename Op>
__device__ __forceinline__ float wave_all(float v)
{
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) v = Op::apply(v, __shfl_xor(v, d));
    return v;
}

// over the workgroup, in a fixed order; the result in every thread.  lds: one float for each wave.
template <typename Op, int WAVES>
__device__ __forceinline__ float block_all(float v, float *lds)
{
    v = wave_all<Op>(v);
    __syncthreads();
    if ((threadIdx.x & (kLanes - 1)) == 0) lds[threadIdx.x / kLanes] = v;
    __syncthreads();
    float r = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) r = Op::apply(r, lds[w]);
    return r;
}

// (x, column) comes before (y, other) among a row's alternatives
__device__ __forceinline__ bool before(float x, int column, float y, int other) { return x > y || (x == y && column < other); }

}  // namespace regot
