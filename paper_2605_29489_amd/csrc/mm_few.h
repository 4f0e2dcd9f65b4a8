// Products of a weight matrix's rows with a few tokens on the matrix cores,
// straight from memory: what mp_linear with few tokens and mp_moe share.
//
// The weights are read once and by one wave each, so they go from memory to
// registers with no stop in LDS.  A step is 64 bytes of each of 16 rows: lane
// l holds the 16-byte chunk l / 16 of row l % 16, which is the operand layout
// of a 16 x 16 MFMA up to the order of the contraction (bf16: one MFMA of
// depth 32; fp32: four of depth 4, the j-th over element j of every chunk),
// and that order is the tokens' too.  Weight rows are the A operand, tokens
// the B operand: lane l then holds outputs 4 (l / 16) .. + 3 of token l % 16.
#pragma once

#include "ffn_common.h"

namespace mp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int DT>
__device__ inline f32x4 mma16(const uint4& a, const uint4& b, f32x4 c)
{
    if constexpr (DT == MP_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                       c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
}

constexpr int kStepBytes = 64;

// What a lane without a token reads: steps of zeros.
constexpr int kFewUnroll = 8;
__device__ const uint4 g_zero_steps[kFewUnroll * kStepBytes / 16] = {};

// Adds steps [s0, s1) of NA row tiles times TT token tiles to acc.  w[i]: the
// lane's chunk of step 0 in row tile i; x[t]: its chunk of step 0 in token
// tile t, which moves by 64 bytes a step where go[t] is set and else reads
// g_zero_steps.  With XS = 2 each token tile is a sum of two operands, x[t]
// and x[TT + t].  U steps are in flight: each is multiplied when it arrives
// and the step U further on takes its registers.
template <int DT, int NA, int TT, int XS, int U>
__device__ inline void few_steps(f32x4 (&acc)[NA][TT], const char* const (&w0)[NA], const char* const (&x0)[TT * XS],
                                 const bool (&go)[TT], int64_t s0, int64_t s1)
{
    constexpr int XT = TT * XS;
    static_assert(U <= kFewUnroll);
    if (s0 >= s1)
        return;
    const char *w[NA], *x[XT];
    int inc[TT];
#pragma unroll
    for (int i = 0; i < NA; ++i)
        w[i] = w0[i] + s0 * kStepBytes;
#pragma unroll
    for (int t = 0; t < XT; ++t)
        x[t] = x0[t] + (go[t % TT] ? s0 * kStepBytes : 0);
#pragma unroll
    for (int t = 0; t < TT; ++t)
        inc[t] = go[t] ? U * kStepBytes : 0;
    uint4 a[U][NA], b[U][XT];
    auto load = [&](int u) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
            a[u][i] = ld16u(w[i] + u * kStepBytes);
#pragma unroll
        for (int t = 0; t < XT; ++t)
            b[u][t] = ld16u(x[t] + u * kStepBytes);
    };
    auto next = [&]() {
#pragma unroll
        for (int i = 0; i < NA; ++i)
            w[i] += U * kStepBytes;
#pragma unroll
        for (int t = 0; t < XT; ++t)
            x[t] += inc[t % TT];
    };
    auto mul = [&](int u) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int t = 0; t < XT; ++t)
                acc[i][t % TT] = mma16<DT>(a[u][i], b[u][t], acc[i][t % TT]);
    };
    int64_t n = s1 - s0;  // steps not multiplied yet
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n)
            load(u);
    for (; n >= 2 * U; n -= U) {
        next();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mul(u);
            load(u);
        }
    }
    next();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u < n)
            mul(u);
        if (U + u < n)
            load(u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (U + u < n)
            mul(u);
}

// The same for the columns of a row past its last whole step: n elements
// (fewer than a step holds), at step `s`.
template <int DT, int NA, int TT, int XS>
__device__ inline void few_tail(f32x4 (&acc)[NA][TT], const char* const (&w)[NA], const char* const (&x)[TT * XS],
                                const bool (&go)[TT], int64_t s, int n)
{
    constexpr int V = Fmt<DT>::V;
    const int64_t at = s * kStepBytes;
    const int left = n - (int)(threadIdx.x % 64 / 16) * V;  // elements of the lane's chunk
    auto part = [&](const char* p) {
        return left >= V ? ld16u(p) : left > 0 ? ld16_head<DT>(p, left) : make_uint4(0, 0, 0, 0);
    };
#pragma unroll
    for (int t = 0; t < TT * XS; ++t) {
        const uint4 b = go[t % TT] ? part(x[t] + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < NA; ++i)
            acc[i][t % TT] = mma16<DT>(part(w[i] + at), b, acc[i][t % TT]);
    }
}

// Adds the waves' partial tiles over LDS and hands float4 number i of the sum
// (in a wave's lane order, tile by tile) to use(i, sum), spread over `n`
// threads numbered `me`.  Callers put barriers around it.
template <int N, typename F>
__device__ inline void sum_tiles(const float4* red, int waves, int me, int n, F use)
{
    for (int i = me; i < N * 64; i += n) {
        float4 s = red[i];
        for (int w = 1; w < waves; ++w) {
            const float4 v = red[w * N * 64 + i];
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        use(i, s);
    }
}

// Steps in flight for so many operands: about 80 registers of them.
constexpr int few_unroll(int operands) { return operands <= 2 ? 8 : operands == 3 ? 6 : operands <= 5 ? 4 : operands == 6 ? 3 : 2; }

// Whole steps of a row of n elements, and the elements after them.
template <int DT>
__device__ __host__ inline int64_t few_whole(int64_t n)
{
    return n / (kStepBytes / Fmt<DT>::esize);
}
template <int DT>
__device__ __host__ inline int few_rest(int64_t n)
{
    return (int)(n % (kStepBytes / Fmt<DT>::esize));
}

}  // namespace mp
