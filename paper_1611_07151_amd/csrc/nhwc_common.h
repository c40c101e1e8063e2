// Shared by the kernels on channels-last maps: element types, activations.
#pragma once

#include "sq_internal.h"

#include <type_traits>

namespace sq {

typedef uint16_t bf16_t;      // bfloat16 as the upper half of a binary32 pattern
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
// round to nearest even, NaN stays NaN
template <typename T> __device__ __forceinline__ T from_f32(float v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __builtin_bit_cast(bf16_t, (__bf16)v);
}

// Activations; an infinity or NaN gives what the definition gives (ReLU of a NaN is a NaN, GELU of -inf is -inf * 0).
//   SiLU   x / (1 + exp(-x)) with the exponential as 2^(-x log2 e) and the reciprocal of the hardware (one unit each): within 1.5e-7 |x|
//          of the definition (plain fp32 1.2e-7).  Below -87.3 the reciprocal is no normal number any more and the result -0 (of 1e-36).
//   GELU   x Phi(x), Phi(-t) = Q(t) = erfc(t / sqrt 2) / 2 = exp(-t^2 / 2) q P(q) with q = 1 / (1 + 0.3 t): P of degree 7 fitted
//          here to erfcx on t in [0, 14] (relative error 1.6e-7; behind it exp underflows).  In fp32 the result is within
//          2.6e-7 |x| of the definition (6 million points in [-120, 120]; plain fp32 1.1e-7).  The runtime's erfcf costs four times as many
//          instructions: with it a 16224 x 4096 x 4096 product took 107 us more with GELU and residual than without; now 64.
template <int ACT> __device__ __forceinline__ float activate(float v)
{
    if constexpr (ACT == SQ_ACT_RELU) {
        return v < 0.f ? 0.f : v;
    } else if constexpr (ACT == SQ_ACT_SILU) {
        return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * v));
    } else if constexpr (ACT == SQ_ACT_GELU) {
        const float t = __builtin_fabsf(v), q = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, t, 1.f));
        float s = 0.0356748141348362f;
        s = __builtin_fmaf(s, q, -0.15720324218273163f);
        s = __builtin_fmaf(s, q, 0.20635376870632172f);
        s = __builtin_fmaf(s, q, -0.053683873265981674f);
        s = __builtin_fmaf(s, q, 0.12856173515319824f);
        s = __builtin_fmaf(s, q, 0.09991346299648285f);
        s = __builtin_fmaf(s, q, 0.12075395882129669f);
        s = __builtin_fmaf(s, q, 0.11962930113077164f);
        const float tail = s * q * __builtin_amdgcn_exp2f(-0.72134752044448170f * t * t);
        return v * (v < 0.f ? tail : 1.f - tail);
    } else {
        return v;
    }
}

}  // namespace sq
