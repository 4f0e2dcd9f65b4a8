// Products of a weight matrix's rows with a few tokens on the matrix cores,
// straight from memory: what mp_linear with few tokens and mp_moe share.
//
// The weights are read once and by one wave each, so they go from memory to
// registers with no stop in LDS.  A step takes R = 16, 8 or 4 rows and G = 16 / R
// pieces of 64 bytes of each, side by side.  Lane l holds the 16-byte chunk
// l / 16 of piece (l % 16) / R of row (l % 16) % R, which is the A operand of a
// 16 x 16 MFMA whose row p R + r is piece p of row r.  The tokens are the B
// operand, one for each piece; a product with piece p's B operand is right
// in the rows of piece p, which is one lane's 4 accumulators, so each piece has
// accumulators of its own and a lane keeps those of piece (l / 16) * 4 / R: 4
// outputs of token l % 16.  The order of the contraction inside a piece is
// the operands' (bf16: one MFMA of depth 32; fp32: four of depth 4, the j-th
// over element j of every chunk).  Fewer rows a step make more workgroups of
// the same matrix and longer runs in memory, at G times the MFMAs and token
// loads.
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

constexpr int kPieceBytes = 64;

// A wave's operands: NA row tiles, TT token tiles of XS operands each.
template <int DT, int R, int NA, int TT, int XS>
struct Few {
    static constexpr int G = 16 / R, XT = TT * XS, kStep = kPieceBytes * G, kElems = kStep / Fmt<DT>::esize;
    const char* w[NA];  // the lane's chunk of step 0 in a row tile
    const char* x[XT];  // its chunk of piece 0 of step 0 in a token tile: t, and with XS = 2 a second operand at TT + t
    f32x4 acc[NA][TT][G];

    // Byte offset of the lane's chunk in a step, in a row's and in a token's.
    __device__ static inline int row_of(int lane) { return (lane & 15) % R; }
    __device__ static inline int w_off(int lane) { return (lane & 15) / R * kPieceBytes + (lane >> 4) * 16; }
    __device__ static inline int x_off(int lane) { return (lane >> 4) * 16; }

    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    acc[i][t][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Loads of step `at` from the pointers, and the products with them.
    struct Regs {
        uint4 a[NA], b[XT][G];
    };
    __device__ static inline void load(Regs& r, const char* const (&wp)[NA], const char* const (&xp)[XT], int at)
    {
#pragma unroll
        for (int i = 0; i < NA; ++i)
            r.a[i] = ld16u(wp[i] + at * kStep);
#pragma unroll
        for (int t = 0; t < XT; ++t)
#pragma unroll
            for (int g = 0; g < G; ++g)
                r.b[t][g] = ld16u(xp[t] + at * kStep + g * kPieceBytes);
    }
    __device__ inline void mul(const Regs& r)
    {
#pragma unroll
        for (int t = 0; t < XT; ++t)
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
                for (int i = 0; i < NA; ++i)
                    acc[i][t % TT][g] = mma16<DT>(r.a[i], r.b[t][g], acc[i][t % TT][g]);
            }
    }

    // Adds rounds [r0, r1) of kRound steps.  A round is in flight: each step is
    // multiplied when it arrives and the same step of the next round takes its
    // registers.  No load hangs on a branch: the compiler then knows how many
    // are in flight and waits for the oldest alone (with a branch around the
    // tokens' loads it waited for all of them once a round).  Lanes without a
    // token therefore load another's.
    static constexpr int kRound = NA + XT * G <= 3 ? 4 : 2;
    __device__ inline void rounds(int64_t r0, int64_t r1)
    {
        if (r0 >= r1)
            return;
        const char *wp[NA], *xp[XT];
#pragma unroll
        for (int i = 0; i < NA; ++i)
            wp[i] = w[i] + r0 * (kRound * kStep);
#pragma unroll
        for (int t = 0; t < XT; ++t)
            xp[t] = x[t] + r0 * (kRound * kStep);
        Regs r[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u)
            load(r[u], wp, xp, u);
        for (int64_t k = r0 + 1; k < r1; ++k) {
#pragma unroll
            for (int i = 0; i < NA; ++i)
                wp[i] += kRound * kStep;
#pragma unroll
            for (int t = 0; t < XT; ++t)
                xp[t] += kRound * kStep;
#pragma unroll
            for (int u = 0; u < kRound; ++u) {
                mul(r[u]);
                __builtin_amdgcn_sched_barrier(0);  // or a step's loads move up and need registers of their own
                load(r[u], wp, xp, u);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int u = 0; u < kRound; ++u)
            mul(r[u]);
    }

    // What is left of a row of n elements behind its whole rounds: steps, and part of one.
    __device__ inline void rest(int64_t n)
    {
        int64_t s = n / kElems / kRound * kRound;
        const char *wp[NA], *xp[XT];
        for (; s < n / kElems; ++s) {
            Regs r;
#pragma unroll
            for (int i = 0; i < NA; ++i)
                wp[i] = w[i] + s * kStep;
#pragma unroll
            for (int t = 0; t < XT; ++t)
                xp[t] = x[t] + s * kStep;
            load(r, wp, xp, 0);
            mul(r);
        }
        if (n % kElems)
            tail(s, (int)(n % kElems));
    }
    __device__ static inline int64_t whole(int64_t n) { return n / (kElems * kRound); }
    __device__ static inline bool more(int64_t n) { return n % (kElems * kRound) != 0; }

    // The n elements (fewer than a step holds) from step s on.
    __device__ inline void tail(int64_t s, int n)
    {
        constexpr int V = Fmt<DT>::V;
        const int lane = threadIdx.x & 63;
        const int64_t at = s * kStep;
        auto part = [&](const char* p, int left) {
            return left >= V ? ld16u(p) : left > 0 ? ld16_head<DT>(p, left) : make_uint4(0, 0, 0, 0);
        };
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const uint4 a = part(w[i] + at, n - w_off(lane) / Fmt<DT>::esize);
#pragma unroll
            for (int t = 0; t < XT; ++t)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int off = g * kPieceBytes + x_off(lane);
                    const uint4 b = part(x[t] + at + g * kPieceBytes, n - off / Fmt<DT>::esize);
                    acc[i][t % TT][g] = mma16<DT>(a, b, acc[i][t % TT][g]);
                }
        }
    }

    // The lane's outputs: those of its piece, to be added over the pieces (sum_tiles).
    __device__ inline float4 out(int i, int t) const
    {
        const int g = (threadIdx.x & 63) / 16 * 4 / R;
        f32x4 v = acc[i][t][0];
#pragma unroll
        for (int k = 1; k < G; ++k)
            v = g == k ? acc[i][t][k] : v;
        return make_float4(v[0], v[1], v[2], v[3]);
    }
};

// Adds partial tiles over W waves and the pieces: red holds N tiles of 64
// float4 per wave.  use(tile, row, token, sum): one output, spread over `n`
// threads numbered `me`.  Callers put barriers around it.
template <int R, int N, int W, typename F>
__device__ inline void sum_tiles(const float4* red, int me, int n, F use)
{
    constexpr int kOuts = R * 16;  // outputs of a tile
    const float* r = reinterpret_cast<const float*>(red);
    for (int q = me; q < N * kOuts; q += n) {
        const int tile = q / kOuts, o = q % kOuts;
        // float4 o / 4 holds rows 4 (o / 64) .. + 3 of token o / 4 % 16
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int g = 0; g < 16 / R; ++g)
                s += r[(w * N + tile) * 256 + g * kOuts + o];
        use(tile, o / 64 * 4 + (o & 3), o / 4 % 16, s);
    }
}

// ---------------------------------------------------------------- one to four tokens
// With so few tokens the vector ALU keeps up with memory (8 + 8 TT operations
// on 16 bytes of bf16 weights), and it needs no operand layout: a wave reads
// 1 KB runs of RG rows, its lanes' chunks of the TT tokens serve all the rows,
// and the lanes' sums meet at the end.  XF: tokens in fp32 (then a lane's chunk
// is 32 bytes of bf16's 8 columns).
template <int DT, int RG, int TT, bool XF>
struct Gemv {
    static constexpr int V = Fmt<DT>::V, es = Fmt<DT>::esize, kRun = 64 * V;  // columns of a run
    static constexpr int kXs = XF ? 4 : es;                                    // bytes of a token's value
    static constexpr int XC = V * kXs / 16;                                    // 16-byte chunks of a lane's columns
    float acc[RG][TT];

    struct Regs {
        uint4 a[RG], b[TT][XC];
    };
    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < RG; ++i)
#pragma unroll
            for (int t = 0; t < TT; ++t)
                acc[i][t] = 0.0f;
    }
    __device__ inline void fma(const Regs& r)
    {
        float x[TT][V];
#pragma unroll
        for (int t = 0; t < TT; ++t)
            if constexpr (XF && DT == MP_BF16) {
                Fmt<MP_F32>::unpack(r.b[t][0], x[t]);
                Fmt<MP_F32>::unpack(r.b[t][XC - 1], x[t] + 4);
            } else {
                Fmt<DT>::unpack(r.b[t][0], x[t]);
            }
#pragma unroll
        for (int i = 0; i < RG; ++i) {
            float f[V];
            Fmt<DT>::unpack(r.a[i], f);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    acc[i][t] = fmaf(f[j], x[t][j], acc[i][t]);
        }
    }
    // Runs c0, c0 + step, .. (n of them) of the rows w and the tokens x, which are the same for the wave.
    __device__ inline void runs(const char* const (&w)[RG], const char* const (&x)[TT], int64_t c0, int64_t step,
                                int64_t n)
    {
        if (n <= 0)
            return;
        const uint32_t lane = threadIdx.x & 63, wo = lane * 16, xo = lane * (V * kXs);
        auto load = [&](Regs& r, int64_t c) {
#pragma unroll
            for (int i = 0; i < RG; ++i)
                r.a[i] = ld16u(w[i] + c * (kRun * es) + wo);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int k = 0; k < XC; ++k)
                    r.b[t][k] = ld16u(x[t] + c * (kRun * kXs) + k * 16 + xo);
        };
        Regs cur, nxt;
        load(cur, c0);
        for (int64_t i = 1; i < n; ++i) {
            load(nxt, c0 + i * step);
            fma(cur);
            cur = nxt;
        }
        fma(cur);
    }
    // The columns of a row of n behind its whole runs.
    __device__ inline void rest(const char* const (&w)[RG], const char* const (&x)[TT], int64_t n)
    {
        const int64_t at = n / kRun * kRun + (threadIdx.x & 63) * V;
        const int64_t left = n - at;
        Regs r;
#pragma unroll
        for (int i = 0; i < RG; ++i)
            r.a[i] = left >= V ? ld16u(w[i] + at * es) : left > 0 ? ld16_head<DT>(w[i] + at * es, left) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int k = 0; k < XC; ++k) {
                constexpr int kPer = 16 / kXs;  // values of a 16-byte chunk
                const int64_t l = left - k * kPer;
                const char* p = x[t] + at * kXs + k * 16;
                r.b[t][k] = l >= kPer ? ld16u(p)
                                      : l > 0 ? ld16_head<XF ? MP_F32 : DT>(p, l) : make_uint4(0, 0, 0, 0);
            }
        fma(r);
    }
    // All of a row of n, split over W waves.
    __device__ inline void row(const char* const (&w)[RG], const char* const (&x)[TT], int64_t n, int wave, int W)
    {
        const int64_t c = n / kRun;
        runs(w, x, wave, W, (c - wave + W - 1) / W);
        if (wave == (int)(c % W) && n % kRun)
            rest(w, x, n);
    }
    // The wave's sums, into red[RG][TT].
    __device__ inline void put(float* red)
    {
#pragma unroll
        for (int i = 0; i < RG; ++i)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const float s = wave_xor_sum(acc[i][t]);
                if ((threadIdx.x & 63) == (i * TT + t) % 64)
                    red[i * TT + t] = s;
            }
    }
};

}  // namespace mp
