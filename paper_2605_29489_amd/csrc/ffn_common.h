// Device helpers of the kernels that run a block's feed-forward part:
// element access at any alignment, and the activations with their derivatives.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/mergepipe.h"

namespace mp {

// Element types by mp_dtype.
template <int DT>
struct Elem;
template <>
struct Elem<MP_F32> {
    using T = float;
};
template <>
struct Elem<MP_BF16> {
    using T = __bf16;
};

// ---------------------------------------------------------------- activations
// In fp32, from exp and erf only.  1 / (1 + exp(-u)) is taken with the
// hardware's exp2 and reciprocal (both within 1 ulp; exp(-u) = inf gives 0):
// a relative error of a few 2^-24 where |u| is about 1, against the 2^-9 of a
// bf16 output and the 2^-24 * sqrt(k) of the fp32 sum that z is.
__device__ inline float sigmoid_f(float u)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -1.44269504088896f));
}

constexpr float kGeluC = 1.59576912160573f;  // 2 sqrt(2 / pi): (1 + tanh(u)) / 2 = sigmoid(2 u)

template <int ACT>
__device__ inline float act_f(float z)
{
    if constexpr (ACT == MP_ACT_RELU)
        return z > 0.0f ? z : (z != z ? z : 0.0f);
    else if constexpr (ACT == MP_ACT_GELU)
        return 0.5f * z * (1.0f + erff(z * 0.70710678118655f));
    else if constexpr (ACT == MP_ACT_GELU_TANH)
        return z * sigmoid_f(kGeluC * (z + 0.044715f * z * z * z));
    else if constexpr (ACT == MP_ACT_SILU)
        return z * sigmoid_f(z);
    else
        return z;
}

// d act / d z
template <int ACT>
__device__ inline float act_slope_f(float z)
{
    if constexpr (ACT == MP_ACT_RELU)
        return z > 0.0f ? 1.0f : 0.0f;
    else if constexpr (ACT == MP_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678118655f)) +
               z * 0.398942280401433f * __builtin_amdgcn_exp2f(z * z * -0.72134752044448f);
    else if constexpr (ACT == MP_ACT_GELU_TANH) {
        const float p = sigmoid_f(kGeluC * (z + 0.044715f * z * z * z));
        return p + z * p * (1.0f - p) * kGeluC * (1.0f + 0.134145f * z * z);
    } else if constexpr (ACT == MP_ACT_SILU) {
        const float p = sigmoid_f(z);
        return p + z * p * (1.0f - p);
    } else
        return 1.0f;
}

__device__ inline float act_of(int act, float z)
{
    switch (act) {
        case MP_ACT_RELU: return act_f<MP_ACT_RELU>(z);
        case MP_ACT_GELU: return act_f<MP_ACT_GELU>(z);
        case MP_ACT_GELU_TANH: return act_f<MP_ACT_GELU_TANH>(z);
        case MP_ACT_SILU: return act_f<MP_ACT_SILU>(z);
        default: return z;
    }
}

__device__ inline float act_slope_of(int act, float z)
{
    switch (act) {
        case MP_ACT_RELU: return act_slope_f<MP_ACT_RELU>(z);
        case MP_ACT_GELU: return act_slope_f<MP_ACT_GELU>(z);
        case MP_ACT_GELU_TANH: return act_slope_f<MP_ACT_GELU_TANH>(z);
        case MP_ACT_SILU: return act_slope_f<MP_ACT_SILU>(z);
        default: return 1.0f;
    }
}

// Sum over the wave, the same bits in every lane.
__device__ inline float wave_sum(float v)
{
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o, 64);
    return v;
}

}  // namespace mp
