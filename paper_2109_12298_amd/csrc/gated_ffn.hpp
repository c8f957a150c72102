// Shared by the kernels of the gated feed-forward block: the activations and
// their derivatives, and element conversions.
#pragma once

#include "common.hpp"

namespace dpg {
namespace ffn {

// sigmoid(2 z) = (1 + tanh z) / 2, so both activations are g * sigmoid(w(g))
// with w = g (SiLU) or w = 2 sqrt(2/pi) (g + 0.044715 g^3) (GELU, tanh form).
// exp overflows to infinity for large -w, where the quotient is a correct 0;
// the product with g is then 0 for every finite g (an infinite g has no
// finite w that would reach it).
constexpr float kGeluA = 1.5957691216057308f;       // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

template <int ACT>
__device__ __forceinline__ float exponent_of(float g)
{
    return ACT == DP_ACT_SILU ? g : kGeluA * (g + kGeluB * g * g * g);
}

template <int ACT>
__device__ __forceinline__ float act(float g)
{
    return g * (1.0f / (1.0f + expf(-exponent_of<ACT>(g))));
}

// The same with the hardware's exp2 and reciprocal (each within about one
// step of fp32; the exponent's product adds |w| half steps to the gate, times
// p (1 - p)): for results that are rounded to bf16, 2^16 times coarser.
template <int ACT>
__device__ __forceinline__ float act_fast(float g)
{
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * exponent_of<ACT>(g)));
}

// for results kept in T
template <int ACT, typename T>
__device__ __forceinline__ float act_for(float g)
{
    return sizeof(T) == 4 ? act<ACT>(g) : act_fast<ACT>(g);
}

// act(g) and act'(g) = p + g p (1 - p) w'(g), p = sigmoid(w(g)).  1 - p is formed
// as e p with p = 1 / (1 + e): the difference would lose its bits where p comes
// near 1 (2^-25 times g w'(g) = 34 at g = 5 in the GELU form, 33 half steps of
// the slope; so 3).  Where e overflows both are 0.  For large |g| in the GELU
// form p (1 - p) is 0 while g w'(g) may be infinite: the term is 0.
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &s)
{
    const float e = expf(-exponent_of<ACT>(g)), p = 1.0f / (1.0f + e);
    const float q = p == 0.0f ? 0.0f : p * (e * p);
    a = g * p;
    if constexpr (ACT == DP_ACT_SILU) s = p + g * q;
    else s = q == 0.0f ? p : p + q * (g * (kGeluA * (1.0f + 3.0f * kGeluB * g * g)));
}

__device__ __forceinline__ uint16_t bf16_bits(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ void store_elem(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t *p, float v) { *p = bf16_bits(v); }

}  // namespace ffn
}  // namespace dpg
