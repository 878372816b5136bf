// The activations of the gated block and their derivatives, fp32.
#pragma once
#include "../../include/molora.h"
#include "common.h"

namespace molora {
namespace {

// Two bf16 bit patterns, rounded to nearest even; what is not finite stays so.
__device__ __forceinline__ uint32_t bf16x2_bits(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ u32x2 bf16x4_bits(f32x4 v) { return u32x2{bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3])}; }

// act(g) = g p(g) with p the logistic function, the normal distribution's, or the latter's logistic form
// p(y), y = 2 sqrt(2 / pi) (g + 0.044715 g^3), which is (1 + tanh(y / 2)) / 2.  Returns p and, where it is
// asked for, its derivative.
template <bool SLOPE>
__device__ __forceinline__ float gate_factor(float g, int act, float &slope) {
    if (act == MOLORA_ACT_GELU) {
        // erfc on the side where 1 + erf would cancel
        const float p = 0.5f * erfcf(-g * 0.70710678118654752f);
        if (SLOPE) slope = 0.3989422804014327f * __expf(-0.5f * g * g);
        return p;
    }
    const float k = 1.5957691216057308f;  // 2 sqrt(2 / pi)
    const float y = act == MOLORA_ACT_SILU ? g : k * (g + 0.044715f * g * g * g);
    const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-y));  // (a step of fp32 off at most)
    // (1 - p would lose what is left of p near 1: q is the same from the other side)
    if (SLOPE) {
        const float q = __builtin_amdgcn_rcpf(1.0f + __expf(y));
        const float d = p * q;
        slope = act == MOLORA_ACT_SILU ? d : d > 0.f ? d * k * (1.0f + 0.134145f * g * g) : 0.f;
    }
    return p;
}

// act(g) u
__device__ __forceinline__ f32x4 gate4(f32x4 g, f32x4 u, int act) {
    f32x4 z;
    float unused;
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = g[i] * gate_factor<false>(g[i], act, unused) * u[i];
    return z;
}

}  // namespace
}  // namespace molora
