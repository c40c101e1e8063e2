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

// Activations by their definitions, so that an infinity or NaN gives what the definition gives (ReLU of a NaN is a NaN).
// GELU is x/2 erfc(-x/sqrt 2): 1 + erf would lose the negative tail to cancellation.
template <int ACT> __device__ __forceinline__ float activate(float v)
{
    if constexpr (ACT == SQ_ACT_RELU) return v < 0.f ? 0.f : v;
    else if constexpr (ACT == SQ_ACT_SILU) return v / (1.f + expf(-v));
    else if constexpr (ACT == SQ_ACT_GELU) return 0.5f * v * erfcf(-0.70710678118654752f * v);
    else return v;
}

}  // namespace sq
