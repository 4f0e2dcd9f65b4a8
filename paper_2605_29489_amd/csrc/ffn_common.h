// Device helpers of the kernels that run a block: element access at any
// alignment, quotients, and the activations with their derivatives.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/mergepipe.h"
#include "device_common.h"

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

// Quotients of n < 2^31 by a divisor the host knows: with 2^(L-1) < d <= 2^L and
// m = ceil(2^(31+L) / d), n m / 2^(31+L) exceeds n / d by less than
// n / 2^31 / d < 1 / d, so that their whole parts agree.
struct Div {
    uint32_t m = 0, shift = 0;
    Div(uint32_t by = 1)
    {
        uint32_t L = 0;
        while (((uint64_t)1 << L) < by)
            ++L;
        shift = 31 + L;
        m = (uint32_t)((((uint64_t)1 << shift) + by - 1) / by);
    }
    __device__ inline uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

// ---------------------------------------------------------------- 16-byte access at element alignment
// Global memory takes 16-byte accesses at any element's alignment, so a row
// that starts off a 16-byte boundary costs no other code, only lines that two
// accesses share.
typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));
__device__ inline uint4 ld16u(const void* p)
{
    const u32x4_t v = *static_cast<const u32x4_a2*>(p);
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ inline void st16u(void* p, uint4 c)
{
    const u32x4_t v = {c.x, c.y, c.z, c.w};
    *static_cast<u32x4_a2*>(p) = v;
}
// The first n (0 <= n < the chunk's elements) elements at p, zeros after them.
template <int DT>
__device__ inline uint4 ld16_head(const void* p, int64_t n)
{
    uint32_t w[4] = {0, 0, 0, 0};
    if constexpr (DT == MP_F32) {
        const uint32_t* q = static_cast<const uint32_t*>(p);
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n)
                w[j] = q[j];
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(p);
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n)
                w[j / 2] |= (uint32_t)q[j] << (16 * (j & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The chunk at p of which `have` elements count (any number; none if it is not
// positive), zeros after them, without a branch: it is read from p, or, where
// that passes the matrix's end, from `last`, its last 16 bytes, and shifted.
template <int DT>
__device__ inline uint4 ld16_edge(const char* p, int64_t have, const char* last)
{
    const char* q = p < last ? p : last;
    const uint4 c = ld16u(q);
    const uint64_t d = (uint64_t)(p - q);
    const uint32_t sh = d < 15 ? (uint32_t)d * 8 : 120;  // bits
    uint64_t lo = c.x | (uint64_t)c.y << 32, hi = c.z | (uint64_t)c.w << 32;
    // (hi << 1) << (63 - n) is hi << (64 - n) for n from 0 on
    const uint32_t n = sh & 63;
    const uint64_t down = lo >> n | (hi << 1) << (63 - n);
    lo = sh < 64 ? down : hi >> n;
    hi = sh < 64 ? hi >> n : 0;
    constexpr int kBits = 8 * Fmt<DT>::esize;
    const int keep = have <= 0 ? 0 : have >= Fmt<DT>::V ? 128 : (int)have * kBits;  // bits
    lo = keep >= 64 ? lo : lo & ((1ull << keep) - 1);
    hi = keep >= 128 ? hi : keep <= 64 ? 0 : hi & ((1ull << (keep - 64)) - 1);
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}
template <int DT>
__device__ inline void st16_head(void* p, uint4 c, int64_t n)
{
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    if constexpr (DT == MP_F32) {
        uint32_t* q = static_cast<uint32_t*>(p);
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n)
                q[j] = w[j];
    } else {
        uint16_t* q = static_cast<uint16_t*>(p);
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n)
                q[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
    }
}

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
        // where z z overflows, p (1 - p) is 0: bounded, so that their product is too
        const float p = sigmoid_f(kGeluC * (z + 0.044715f * z * z * z));
        return p + z * p * (1.0f - p) * kGeluC * (1.0f + 0.134145f * fminf(z * z, 1e30f));
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

}  // namespace mp
