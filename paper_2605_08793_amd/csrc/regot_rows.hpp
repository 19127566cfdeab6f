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
constexpr float kLog2e = 1.44269504088896340736f;

__host__ __device__ constexpr int cbits(int64_t v) { return v > 1 ? 1 + cbits(v / 2) : 0; }  // log2 of a power of two

// orders a wave's accesses to LDS that its lanes share
__device__ __forceinline__ void wave_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A score as a 32-bit number, and back (rounded to nearest even, once); kVec of them are what a lane loads at a time.
// TYPE + kSingle: one score at a time, for rows that are shorter than a load, or give few lanes one.
constexpr int kSingle = 16;
template <int TYPE>
struct Score {
    using Wide = Score<TYPE - kSingle>;
    using Raw = typename Wide::Raw;
    using Chunk = Raw;
    static constexpr int kVec = 1;
    static __device__ __forceinline__ float get(Raw v) { return Wide::get(v); }
    static __device__ __forceinline__ Raw put(float v) { return Wide::put(v); }
    static __device__ __forceinline__ void unpack(Chunk v, float *x) { x[0] = Wide::get(v); }
    static __device__ __forceinline__ Chunk pack(const Raw *v) { return v[0]; }
};
struct WideChunk {
    using Chunk = u32x4;
    template <typename Raw>
    static __device__ __forceinline__ Chunk pack(const Raw *v)
    {
        Chunk c;
        __builtin_memcpy(&c, v, 16);
        return c;
    }
};
template <>
struct Score<REGOT_F32> : WideChunk {
    using Raw = float;
    static constexpr int kVec = 4;
    static __device__ __forceinline__ float get(Raw v) { return v; }
    static __device__ __forceinline__ Raw put(float v) { return v; }
    static __device__ __forceinline__ void unpack(u32x4 v, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
    }
};
template <>
struct Score<REGOT_BF16> : WideChunk {
    using Raw = __bf16;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float get(Raw v) { return (float)v; }
    static __device__ __forceinline__ Raw put(float v) { return (__bf16)v; }
    static __device__ __forceinline__ void unpack(u32x4 v, float *x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(v[i] << 16);
            x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
};
template <>
struct Score<REGOT_F16> : WideChunk {
    using Raw = _Float16;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float get(Raw v) { return (float)v; }
    static __device__ __forceinline__ Raw put(float v) { return (_Float16)v; }
    static __device__ __forceinline__ void unpack(u32x4 v, float *x)
    {
        _Float16 h[8];
        __builtin_memcpy(h, &v, 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
    }
};

// The same number, known from here on only: what is computed from it stays in the branch it is in, instead of taking registers
// beside the common path (the masks of a row's end took up to 200 scalar registers more than there are).
__device__ __forceinline__ uint32_t here(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// What a lane takes of a row at column j, the row having at least kVec.  Where it would reach beyond the row it is moved back
// to end with it, so that every load is whole and unconditional; the columns before j, which another lane has, are then
// forbidden ones here.  (Rows start at any multiple of their element: the load is one instruction whatever the address.)
template <int TYPE>
struct Span {
    using T = Score<TYPE>;
    using Raw = typename T::Raw;
    using Chunk = typename T::Chunk;
    typedef Chunk Any __attribute__((aligned(alignof(uint16_t))));
    uint32_t first, own;  // the columns first .. first + kVec - 1, of which those from `own` on count
    __device__ __forceinline__ Span(uint32_t j, uint32_t m) : first(min(j, m - T::kVec)), own(j) {}
    // ONCE: nothing reads the row again soon
    template <bool ONCE>
    __device__ __forceinline__ Chunk load(const Raw *S) const
    {
        if constexpr (T::kVec == 1) return S[first];
        else if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const Any *>(S + first));
        else return *reinterpret_cast<const Any *>(S + first);
    }
    // x[e] to -inf where column first + e does not count
    __device__ __forceinline__ void mask(float *x) const
    {
        if (__any(first != own)) {  // (the wave at the row's end)
            const uint32_t from = here(first);
#pragma unroll
            for (int e = 0; e < T::kVec; ++e) x[e] = from + e >= own ? x[e] : -kInf;
        }
    }
    __device__ __forceinline__ void load_bias(float *b, const float *bias) const { __builtin_memcpy(b, bias + first, T::kVec * sizeof(float)); }
    __device__ __forceinline__ void add_bias(float *x, const float *bias) const
    {
        float b[T::kVec];
        load_bias(b, bias);
#pragma unroll
        for (int e = 0; e < T::kVec; ++e) x[e] += b[e];
    }
    // what a lane computed from the chunk, to the columns that count: one store where all do
    __device__ __forceinline__ void store(Raw *out, const float *v) const
    {
        Raw part[T::kVec];
#pragma unroll
        for (int e = 0; e < T::kVec; ++e) part[e] = T::put(v[e]);
        if (first == own) {
            if constexpr (T::kVec == 1) out[first] = part[0];
            else __builtin_nontemporal_store(T::pack(part), reinterpret_cast<Any *>(out + first));
        } else {
            const uint32_t from = here(first);
#pragma unroll
            for (int e = 0; e < T::kVec; ++e)
                if (from + e >= own) out[from + e] = part[e];
        }
    }
};

// 2^t by the hardware's exponential (within 1 unit in the last place; results below the smallest normal number are 0)
__device__ __forceinline__ float exp2_fast(float t) { return __builtin_amdgcn_exp2f(t); }

// the larger one, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

struct OpSumF {
    static __device__ __forceinline__ float apply(float a, float b) { return a + b; }
};
struct OpMaxF {
    static __device__ __forceinline__ float apply(float a, float b) { return max_nan(a, b); }
};

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// over the wave, in a fixed order; the result in every lane
template <typename Op>
__device__ __forceinline__ float wave_all(float v)
{
    v = Op::apply(v, dpp_f32<kDppXor1>(v));
    v = Op::apply(v, dpp_f32<kDppXor2>(v));
    v = Op::apply(v, dpp_f32<kDppHalfMirror>(v));
    v = Op::apply(v, dpp_f32<kDppMirror>(v));
    const auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
    return Op::apply(Op::apply(lane(0), lane(16)), Op::apply(lane(32), lane(48)));
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
__device__ __forceinline__ bool before(float x, uint32_t column, float y, uint32_t other) { return x > y || (x == y && column < other); }

// 32 bits that are ordered as the numbers are, and back
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

// max, sum of e^z and sum of e^z z (in units of ln 2) of what a lane has seen of its row, z = (x - max) / eta: one pass, the
// sums brought to a new maximum where one comes.  A NaN makes the maximum NaN, a score of +inf the sum.
struct Softmax {
    float max = -kInf, base = 0.f;  // base: what is subtracted, 0 while there is no maximum
    float sum = 0.f, weighted = 0.f;

    // brings the sums to the maximum `to`, which is no less than max.  From a distance of 150 on nothing is left of them: it is kept
    // finite, so that it is 0 times a number that is left (a mask of the type's lowest value, or no score yet, make it -inf, two
    // maxima of -inf a NaN; where the sums have to be NaN, max or sum is).
    __device__ __forceinline__ void raise(float to, float c)
    {
        const float d = fmaxf((max - to) * c, -1024.f), f = exp2_fast(d);
        weighted = f * fmaf(sum, d, weighted);
        sum *= f;
        max = to;
        base = to == -kInf ? 0.f : to;
    }

    // `count` scores whose largest is `top`; c = log2(e) / eta.  ENTROPY: the weighted sum too
    template <bool ENTROPY = true, int COUNT>
    __device__ __forceinline__ void add(const float (&x)[COUNT], float top, float c)
    {
        const float to = max_nan(max, top);
        if (!(to == max)) raise(to, c);
        float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const float t = (x[i] - base) * c, e = exp2_fast(t);
            s[i & 1] += e;
            if constexpr (ENTROPY) w[i & 1] = fmaf(e, t, w[i & 1]);
        }
        float ws = w[0] + w[1];
        if (ENTROPY && ws != ws) {  // 0 times -inf of a forbidden column, which adds nothing (a NaN among the scores is in the sum)
            ws = 0.f;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const float t = (x[i] - base) * c, e = exp2_fast(t);
                ws += e > 0.f ? e * t : 0.f;
            }
        }
        sum += s[0] + s[1];
        weighted += ws;
    }

    // all lanes' in every lane
    __device__ __forceinline__ void over_wave(float c)
    {
        raise(wave_all<OpMaxF>(max), c);
        sum = wave_all<OpSumF>(sum);
        weighted = wave_all<OpSumF>(weighted);
    }
    // all waves' in every thread.  lds: 3 WAVES floats, not in use by what comes before.  (A barrier inside.)
    template <int WAVES>
    __device__ __forceinline__ void over_block(float c, float *lds)
    {
        over_wave(c);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & (kLanes - 1)) == 0) {
                float *mine = lds + 3 * (threadIdx.x / kLanes);
                mine[0] = max, mine[1] = sum, mine[2] = weighted;
            }
            __syncthreads();
            Softmax all;
            float top = lds[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = max_nan(top, lds[3 * w]);
            all.max = top;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                Softmax one;
                one.max = lds[3 * w], one.sum = lds[3 * w + 1], one.weighted = lds[3 * w + 2];
                one.raise(top, c);
                all.sum += one.sum, all.weighted += one.weighted;
            }
            *this = all;
        }
    }
    __device__ __forceinline__ bool none() const { return max == -kInf; }
    __device__ __forceinline__ bool bad() const { return max != max || sum != sum; }
    __device__ __forceinline__ float log_sum() const { return none() ? -kInf : logf(sum); }
    __device__ __forceinline__ float entropy() const { return none() ? 0.f : logf(sum) - weighted * kLn2 / sum; }
};

template <int COUNT>
__device__ __forceinline__ float largest(const float (&x)[COUNT])
{
    float m = x[0];
#pragma unroll
    for (int i = 1; i < COUNT; ++i) m = max_nan(m, x[i]);
    return m;
}

}  // namespace regot
