// Products of a weight matrix's rows with a few tokens: what mp_linear with
// few tokens and mp_moe share.  Few: up to 64 tokens on the matrix cores.  Gemv:
// up to four on the vector ALU.
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

// ---------------------------------------------------------------- up to 64 tokens
// A wave multiplies NA tiles of 16 weight rows by the tokens, 128 bytes of every
// row (a block) at a time.  Weights and tokens come from memory in whole lines,
// 8 lanes to a row, into registers, and go through the wave's own LDS into the
// operand layout, where neighbouring lanes hold neighbouring rows: loaded in
// that layout, each of the 64 lanes' chunks is a cache access of its own, and
// the cache takes one a cycle (3.2 TB/s of weights with two token loads per
// weight load).  No barriers: a wave's LDS accesses are in order.  Weight rows
// are the A operand, tokens the B operand: lane l then holds outputs 4 (l / 16)
// .. + 3 of token l % 16.  The order of the contraction inside 64 bytes is the
// operands' (bf16: one MFMA of depth 32; fp32: four of depth 4, the j-th over
// element j of every chunk).  T8: tokens in eights (1, 2, 4 or 8).  With XS = 2
// a token is the sum of two operands.
template <int DT, int NA, int T8, int XS>
struct Few {
    static constexpr int V = Fmt<DT>::V, kElems = 128 / Fmt<DT>::esize, NT = (T8 + 1) / 2;
    static constexpr int kLds = (NA * 16 + T8 * 8) * 128;  // bytes of LDS per wave
    // blocks in flight: about 64 registers of them
    static constexpr int kLoads = 2 * NA + XS * T8;
    static constexpr int kRound = kLoads <= 4 ? 4 : kLoads <= 8 ? 2 : 1;
    const char* w[NA][2];   // the lane's chunk of block 0 in rows row_of(lane, m)
    const char* x[XS][T8];  // and of tokens row_of(lane, m)
    char* lds;              // the wave's kLds bytes
    f32x4 acc[NA][NT];

    struct Regs {
        uint4 a[NA][2], b[XS][T8];
    };
    __device__ static inline int row_of(int lane, int m) { return m * 8 + (lane >> 3); }
    __device__ static inline int off(int lane) { return (lane & 7) * 16; }

    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                acc[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // Block `at`.  PART: the row has `left` more elements, a block's or fewer; the rest reads as zeros.
    template <bool PART>
    __device__ inline void load(Regs& r, int64_t at, int left) const
    {
        const int have = left - (int)(threadIdx.x & 7) * V;
        auto get = [&](const char* p) {
            if constexpr (PART)
                return have >= V ? ld16u(p) : have > 0 ? ld16_head<DT>(p, have) : make_uint4(0, 0, 0, 0);
            else
                return ld16u(p);
        };
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m)
                r.a[i][m] = get(w[i][m] + at * 128);
#pragma unroll
        for (int s = 0; s < XS; ++s)
#pragma unroll
            for (int m = 0; m < T8; ++m)
                r.b[s][m] = get(x[s][m] + at * 128);
    }
    // Chunk c of row `row` in LDS, permuted so that 8 lanes meet 8 different chunks of 128 bytes both ways.
    __device__ static inline int slot(int row, int c) { return row * 128 + ((c ^ (row & 7)) << 4); }
    __device__ inline void mul(const Regs& r)
    {
        const int lane = threadIdx.x & 63, col = lane & 15, q = lane >> 4;
        char* const lx = lds + NA * 16 * 128;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m)
                *reinterpret_cast<uint4*>(lds + slot(i * 16 + row_of(lane, m), lane & 7)) = r.a[i][m];
#pragma unroll
        for (int s = 0; s < XS; ++s) {
#pragma unroll
            for (int m = 0; m < T8; ++m)
                *reinterpret_cast<uint4*>(lx + slot(row_of(lane, m), lane & 7)) = r.b[s][m];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 a[NA];
#pragma unroll
                for (int i = 0; i < NA; ++i)
                    a[i] = *reinterpret_cast<const uint4*>(lds + slot(i * 16 + col, h * 4 + q));
#pragma unroll
                for (int t = 0; t < NT; ++t) {  // with 8 tokens, columns 8 to 15 repeat them
                    const uint4 b = *reinterpret_cast<const uint4*>(lx + slot(T8 == 1 ? col & 7 : t * 16 + col, h * 4 + q));
#pragma unroll
                    for (int i = 0; i < NA; ++i)
                        acc[i][t] = mma16<DT>(a[i], b, acc[i][t]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    // Adds blocks [b0, b1) of a row of n elements; b0 is a multiple of kRound,
    // b1 one too or past the row's last block.  A round of kRound blocks is in
    // flight: each is multiplied when it arrives and the same block of the
    // next round takes its registers.  No load hangs on a branch there: the
    // compiler then knows how many are in flight and waits for the oldest
    // alone.  What is left of a row behind its whole rounds is loaded at once.
    __device__ inline void blocks(int64_t b0, int64_t b1, int64_t n)
    {
        const int64_t full = n / kElems / kRound;  // rounds without an end of the row
        const int64_t r0 = b0 / kRound, r1 = b1 / kRound < full ? b1 / kRound : full;
        Regs r[kRound];
        if (r0 < r1) {
#pragma unroll
            for (int u = 0; u < kRound; ++u)
                load<false>(r[u], r0 * kRound + u, 0);
            for (int64_t k = r0 + 1; k < r1; ++k) {
#pragma unroll
                for (int u = 0; u < kRound; ++u) {
                    mul(r[u]);
                    __builtin_amdgcn_sched_barrier(0);  // or a block's loads move up and need registers of their own
                    load<false>(r[u], k * kRound + u, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int u = 0; u < kRound; ++u)
                mul(r[u]);
        }
        if (b1 > full * kRound && full * kRound * kElems < n) {
#pragma unroll
            for (int u = 0; u < kRound; ++u) {
                const int64_t left = n - (full * kRound + u) * kElems;
                load<true>(r[u], full * kRound + u, (int)(left < 0 ? 0 : left < kElems ? left : kElems));
            }
#pragma unroll
            for (int u = 0; u < kRound; ++u)
                mul(r[u]);
        }
    }
    // Share `part` of `parts` of a row of n elements.
    __device__ inline void row(int64_t n, int part, int parts)
    {
        const int64_t rounds = (n + kElems * kRound - 1) / (kElems * kRound);
        blocks(rounds * part / parts * kRound, rounds * (part + 1) / parts * kRound, n);
    }
    // The lane's 4 outputs of row tile i and token tile t.
    __device__ inline float4 out(int i, int t) const
    {
        return make_float4(acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]);
    }
};

// Adds W waves' partial tiles: wave w's N tiles of 64 float4 are at red + w *
// pitch.  use(tile, row, token, sum): one output, spread over `n` threads
// numbered `me`.  Callers put barriers around it.
template <int N, int W, typename F>
__device__ inline void sum_tiles(const float4* red, int pitch, int me, int n, F use)
{
    const float* r = reinterpret_cast<const float*>(red);
    for (int q = me; q < N * 256; q += n) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            s += r[w * pitch * 4 + q];
        // float4 o / 4 of a tile holds rows 4 (o / 64) .. + 3 of token o / 4 % 16
        const int o = q % 256;
        use(q / 256, o / 64 * 4 + (o & 3), o / 4 % 16, s);
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
    // Runs c0, c0 + step, .. (cnt of them) of the rows w and the tokens x, which
    // are the same for the wave; a row has n columns, and the run that ends it
    // may be a part of one.
    __device__ inline void runs(const char* const (&w)[RG], const char* const (&x)[TT], int64_t c0, int64_t step,
                                int64_t cnt, int64_t n)
    {
        if (cnt <= 0)
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
        const bool part = (c0 + (cnt - 1) * step + 1) * kRun > n;
        const int64_t full = part ? cnt - 1 : cnt;
        Regs cur, nxt;
        if (full > 0)
            load(cur, c0);
        for (int64_t i = 1; i < full; ++i) {
            load(nxt, c0 + i * step);
            fma(cur);
            cur = nxt;
        }
        if (part) {
            const int64_t at = n / kRun * kRun + lane * V, left = n - at;
#pragma unroll
            for (int i = 0; i < RG; ++i)
                nxt.a[i] = left >= V ? ld16u(w[i] + at * es)
                                     : left > 0 ? ld16_head<DT>(w[i] + at * es, left) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int k = 0; k < XC; ++k) {
                    constexpr int kPer = 16 / kXs;  // values of a 16-byte chunk
                    const int64_t l = left - k * kPer;
                    const char* p = x[t] + at * kXs + k * 16;
                    nxt.b[t][k] = l >= kPer ? ld16u(p)
                                            : l > 0 ? ld16_head<XF ? MP_F32 : DT>(p, l) : make_uint4(0, 0, 0, 0);
                }
        }
        if (full > 0)
            fma(cur);
        if (part)
            fma(nxt);
    }
    // All of a row of n, split over W waves.
    __device__ inline void row(const char* const (&w)[RG], const char* const (&x)[TT], int64_t n, int wave, int W)
    {
        const int64_t c = (n + kRun - 1) / kRun;
        runs(w, x, wave, W, (c - wave + W - 1) / W, n);
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
