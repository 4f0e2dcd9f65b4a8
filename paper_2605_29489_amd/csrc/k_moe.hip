// A layer that routes a few tokens among experts, in two kernels: routing with
// the gate and up products, then the down products with the sum over experts.
#include "ffn_common.h"
#include "mm_few.h"
#include "mp_internal.h"

namespace mp {
namespace {

constexpr int kNone = 0xff;  // slot of a token that does not have the expert

// What the first kernel tells the second, at the start of the workspace.
struct Routing {
    uint8_t slot[kMaxK][kMoeMaxTokens];  // choice number of expert e for token t, or kNone
    uint8_t list[kMaxK][kMoeMaxTokens];  // the tokens that have expert e, in order
    uint32_t count[kMaxK];               // how many
    uint32_t unit[2 * kMaxK];            // e + 256 (its first token's number / 32): up to 32 tokens of an expert
    uint32_t units;
    uint32_t pad[3];
};

// Order of the logits with NaN above every number: larger key, larger logit.
__device__ inline uint32_t logit_key(float l)
{
    if (l != l)
        return 0xffffffffu;
    const uint32_t u = __float_as_uint(l + 0.0f);  // -0 counts as 0
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Values of h per row of the workspace's planes.
__host__ __device__ inline int64_t moe_pitch(int64_t ffn) { return (ffn + 31) / 32 * 32; }

// The row of h that token t has for expert e.
template <typename T>
__device__ inline T* h_row(T* h, const MoeArgs& a, const Routing& rt, int e, int t, int64_t pitch)
{
    return h + ((int64_t)t * a.l.top_k + rt.slot[e][t]) * pitch;
}

// Unit u: its expert, its first token's number among the expert's, how many tokens.
struct Unit {
    int e, first, n;
};
__device__ inline Unit unit_of(const Routing& rt, int u)
{
    const uint32_t v = uniform_u32(rt.unit[u]);
    const int e = (int)(v & 255), first = (int)(v >> 8) * 32, c = (int)uniform_u32(rt.count[e]) - first;
    return Unit{e, first, c < 32 ? c : 32};
}

constexpr int kUpWaves = 8, kUpThreads = 64 * kUpWaves;
// Up to so many tokens, the vector ALU multiplies.  8 bf16 experts of 1536 x 8960,
// 2 a token, in us: 1 token 44 (matrix cores 48), 2 tokens 71 (62), 4 tokens 111 (103).
constexpr int kGemvTokens = 4;

// The choices, from the logits without bias in lg[token][32].  32 lanes take a
// token, one expert each; a choice's number is the count of the logits above
// it.  One workgroup also stores the choices for the caller.
template <int DT>
__device__ inline void choose_experts(const MoeArgs& a, Routing* rt, float (*gate)[kMoeMaxTop], const float* lg)
{
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    const int e = lane & 31, E = a.E, top = a.l.top_k;
    const float b = a.router_bias && e < E ? (float)static_cast<const T*>(a.router_bias)[e] : 0.0f;
    for (int t0 = 0; t0 < a.T; t0 += 2 * kUpWaves) {  // the same trips for every lane of a wave
        const int t = t0 + 2 * wave + (lane >> 5);
        const bool on = t < a.T && e < E;
        const float l = on ? lg[t * 32 + e] + b : -INFINITY;
        const uint32_t key = on ? logit_key(l) : 0u;  // below every logit's
        uint32_t bk = key;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            bk = max(bk, (uint32_t)__shfl_xor((int)bk, o, 32));
        // the largest logit, from its key
        const float best = bk == 0xffffffffu ? NAN : __uint_as_float(bk >> 31 ? bk & 0x7fffffffu : ~bk);
        int rank = 0;
        for (int o = 0; o < E; ++o) {
            const uint32_t k2 = __shfl((int)key, o, 32);
            rank += k2 > key || (k2 == key && o < e);
        }
        const bool chosen = on && rank < top;
        float p = on && best != -INFINITY ? expf(l - best) : 0.0f;
        float sum = (a.l.flags & MP_MOE_RENORM) && !chosen ? 0.0f : p;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            sum += __shfl_xor(sum, o, 32);
        p = best != -INFINITY ? p / sum : 0.0f;
        const bool has = chosen && p != 0.0f;  // NaN counts as a gate
        if (t < a.T)
            rt->slot[e][t] = (uint8_t)(has ? rank : kNone);
        if (chosen) {
            gate[t][rank] = p;
            if (blockIdx.x == 0) {
                if (a.ids)
                    a.ids[t * top + rank] = e;
                if (a.gates)
                    a.gates[t * top + rank] = p;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < kMaxK)
        rt->count[threadIdx.x] = 0;
    __syncthreads();
    for (int x = wave; x < E; x += kUpWaves) {
        const bool has = lane < a.T && rt->slot[x][lane] != kNone;
        const unsigned long long m = __ballot(has);
        if (has)
            rt->list[x][__popcll(m & ((1ull << lane) - 1))] = (uint8_t)lane;
        if (lane == 0)
            rt->count[x] = (uint32_t)__popcll(m);
    }
    __syncthreads();
    if (wave == 0) {
        const uint32_t c = lane < kMaxK ? rt->count[lane] : 0;
        const unsigned long long m1 = __ballot(c > 0), m2 = __ballot(c > 32);
        const unsigned long long below = (1ull << lane) - 1;
        const int at = __popcll(m1 & below) + __popcll(m2 & below);
        if (c > 0)
            rt->unit[at] = lane;
        if (c > 32)
            rt->unit[at + 1] = lane + 256;
        if (lane == 0)
            rt->units = (uint32_t)(__popcll(m1) + __popcll(m2));
    }
    __syncthreads();
}

// Routing.  Every workgroup routes all tokens for itself, by the same
// instructions, so that the gate and up products need no launch of their own
// behind it.  lg: 32 floats of LDS per token (of whole token tiles); red: LDS
// for the partial tiles.
template <int DT, int T8>
__device__ inline void logits_tiles(const MoeArgs& a, float* lg, char* lds, int per_wave)
{
    using T = typename Elem<DT>::T;
    using F = Few<DT, 1, T8, 1>;
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    const int64_t D = a.l.hidden;
    F f;
    f.lds = lds + wave * per_wave;
    for (int t0 = 0; t0 < a.T; t0 += T8 * 8)
        for (int e0 = 0; e0 < a.E; e0 += 16) {
            f.clear();
#pragma unroll
            for (int m = 0; m < T8; ++m) {
                const int tok = t0 + F::row_of(lane, m);
                f.x[0][m] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) +
                                                          (int64_t)(tok < a.T ? tok : a.T - 1) * a.ldx) +
                            F::off(lane);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int e = e0 + F::row_of(lane, m);
                f.w[0][m] =
                    reinterpret_cast<const char*>(static_cast<const T*>(a.router) + (e < a.E ? e : a.E - 1) * D) +
                    F::off(lane);
            }
            f.row(D, wave, kUpWaves);
#pragma unroll
            for (int t = 0; t < F::NT; ++t)
                reinterpret_cast<float4*>(f.lds)[t * 64 + lane] = f.out(0, t);
            __syncthreads();
            sum_tiles<F::NT, kUpWaves>(reinterpret_cast<const float4*>(lds), per_wave / 16, threadIdx.x, kUpThreads,
                                       [&](int t, int row, int tok, float v) {
                                           if (t0 + t * 16 + tok < kMoeMaxTokens)
                                               lg[(t0 + t * 16 + tok) * 32 + e0 + row] = v;
                                       });
            __syncthreads();
        }
}

// The same for one to four tokens, a wave per router row.
template <int DT, int TT>
__device__ inline void logits_gemv(const MoeArgs& a, float* lg)
{
    using T = typename Elem<DT>::T;
    const int wave = (int)uniform_u32(threadIdx.x >> 6);
    const char* x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
        x[t] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + (int64_t)(t < a.T ? t : a.T - 1) * a.ldx);
    for (int e = wave; e < a.E; e += kUpWaves) {
        const char* const w[1] = {
            reinterpret_cast<const char*>(static_cast<const T*>(a.router) + (int64_t)e * a.l.hidden)};
        Gemv<DT, 1, TT, false> g;
        g.clear();
        g.row(w, x, a.l.hidden, 0, 1);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float s = wave_xor_sum(g.acc[0][t]);
            if ((threadIdx.x & 63) == 0)
                lg[t * 32 + e] = s;
        }
    }
    __syncthreads();
}

// Routing leaves the workgroup; the second kernel reads what the first workgroup stored.
__device__ inline void pass_on(const Routing& rt, Routing* out)
{
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += kUpThreads)
            reinterpret_cast<uint32_t*>(out)[i] = reinterpret_cast<const uint32_t*>(&rt)[i];
}

template <int DT>
__device__ inline void put_y(const MoeArgs& a, int tok, int64_t d, float y)
{
    using T = typename Elem<DT>::T;
    if (a.residual)
        y += (float)static_cast<const T*>(a.residual)[tok * a.ldr + d];
    static_cast<T*>(a.y)[tok * a.ldy + d] = (T)y;
}

// A workgroup's sums part(tok, row) of the rows from d0 on: into y, or, where
// several workgroups split the contraction, into parts[split][token][hidden].
template <int DT, int ROWS, typename F>
__device__ inline void finish_rows(const MoeArgs& a, int64_t d0, int split, int splits, float* parts, F part)
{
    for (int q = threadIdx.x; q < a.T * ROWS; q += blockDim.x) {
        const int tok = q / ROWS;
        const int64_t d = d0 + q % ROWS;
        if (d >= a.l.hidden)
            continue;
        const float s = part(tok, q % ROWS);
        if (splits > 1)
            parts[((int64_t)split * a.T + tok) * a.l.hidden + d] = s;
        else
            put_y<DT>(a, tok, d, s);
    }
}

// y from the parts: only where hidden is so small that its row groups leave
// CUs without work.
template <int DT>
__global__ __launch_bounds__(256) void k_moe_join(MoeArgs a, const float* parts, int splits)
{
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x, n = a.T * a.l.hidden;
    if (q >= n)
        return;
    float y = 0.0f;
    for (int s = 0; s < splits; ++s)
        y += parts[s * n + q];
    put_y<DT>(a, (int)(q / a.l.hidden), q % a.l.hidden, y);
}

// act(g) * u * gate
__device__ inline float hidden_of(const MoeArgs& a, float g, float u, float gate)
{
    const float h = act_of(a.l.act, g);
    return (a.l.up_off >= 0 ? h * u : h) * gate;
}

// ---------------------------------------------------------------- five tokens and more
// Calls go(eights) for the template value that covers n tokens, up to T8.
template <int T8, typename F>
__device__ inline void with_eights(int n, F go)
{
    if (n <= 8)
        go(std::integral_constant<int, 1>{});
    else if (T8 == 2 || n <= 16)
        go(std::integral_constant<int, T8 < 2 ? 1 : 2>{});
    else
        go(std::integral_constant<int, T8>{});
}

// h = act(gate x) * (up x) times the token's gate for every (unit, 16 rows of
// ffn): WS waves split an item's contraction.  The B operand's columns are the
// unit's tokens.  h is stored as one value (fp32) or as the bf16 rounding and
// the rounded remainder, in two planes.
template <int DT, int T8, int WS>
__global__ __launch_bounds__(kUpThreads, T8 == 4 ? 2 : 4) void k_moe_up(MoeArgs a, ExpertPtrs ex, Routing* out, char* hbuf)
{
    using T = typename Elem<DT>::T;
    constexpr int NT = (T8 + 1) / 2;
    constexpr int kWave = Few<DT, 2, T8, 1>::kLds;  // a wave's operands on the way, then its partial tiles
    static_assert(kWave >= 2 * NT * 1024);
    __shared__ Routing rt;
    __shared__ float gate[kMoeMaxTokens][kMoeMaxTop];
    __shared__ float lg[kMoeMaxTokens * 32];
    __shared__ __attribute__((aligned(16))) char lds[kUpWaves * kWave];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    logits_tiles<DT, T8>(a, lg, lds, kWave);
    choose_experts<DT>(a, &rt, gate, lg);
    pass_on(rt, out);
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F), plane = (int64_t)a.T * a.l.top_k * pitch;
    const int64_t tiles = (F + 15) / 16, items = tiles * uniform_u32(rt.units);
    const int group = wave / WS, part = wave % WS;
    constexpr int kGroups = kUpWaves / WS;
    const bool two = a.l.up_off >= 0;
    // the same trips for the whole workgroup: there are barriers inside
    for (int64_t it0 = (int64_t)blockIdx.x * kGroups; it0 < items; it0 += (int64_t)gridDim.x * kGroups) {
        const int64_t it = it0 + group;
        const bool on = it < items;
        const Unit u = unit_of(rt, on ? (int)(it / tiles) : 0);
        const int64_t f0 = on ? it % tiles * 16 : 0;
        // outputs of token number `pos` of the unit, row f
        auto put = [&](int pos, int64_t f, float g, float up) {
            if (pos >= u.n || f >= F)
                return;
            const int tok = rt.list[u.e][u.first + pos];
            const float h = hidden_of(a, g, up, gate[tok][rt.slot[u.e][tok]]);
            T* p = h_row(reinterpret_cast<T*>(hbuf), a, rt, u.e, tok, pitch) + f;
            *p = (T)h;
            if constexpr (DT == MP_BF16) {
                const float hi = (float)(T)h;
                p[plane] = (T)(fabsf(hi) < INFINITY ? h - hi : 0.0f);  // an infinite or NaN h has no remainder
            }
        };
        float4* const red = reinterpret_cast<float4*>(lds + wave * kWave);  // [token tile][gate, up]
        auto work = [&](auto eights, auto mats) {
            constexpr int NA = decltype(mats)::value;
            using FW = Few<DT, NA, decltype(eights)::value, 1>;
            FW f;
            f.clear();
            f.lds = lds + wave * kWave;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int64_t r = f0 + FW::row_of(lane, m);
                const char* base =
                    static_cast<const char*>(ex.p[u.e]) + (r < F ? r : F - 1) * D * Fmt<DT>::esize + FW::off(lane);
                f.w[0][m] = base + a.l.gate_off * Fmt<DT>::esize;
                if constexpr (NA == 2)
                    f.w[1][m] = base + a.l.up_off * Fmt<DT>::esize;
            }
#pragma unroll
            for (int m = 0; m < decltype(eights)::value; ++m) {  // columns past the last token repeat it
                const int pos = FW::row_of(lane, m), tok = rt.list[u.e][u.first + (pos < u.n ? pos : u.n - 1)];
                f.x[0][m] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + tok * a.ldx) + FW::off(lane);
            }
            f.row(D, part, WS);
#pragma unroll
            for (int t = 0; t < FW::NT; ++t) {
                const float4 g = f.out(0, t), up = NA == 2 ? f.out(NA - 1, t) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if constexpr (WS == 1) {
                    const float gv[4] = {g.x, g.y, g.z, g.w}, uv[4] = {up.x, up.y, up.z, up.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        put(t * 16 + (lane & 15), f0 + (lane >> 4) * 4 + j, gv[j], uv[j]);
                } else {
                    red[(t * 2 + 0) * 64 + lane] = g;
                    red[(t * 2 + 1) * 64 + lane] = up;
                }
            }
        };
        if (on)
            with_eights<T8>(u.n, [&](auto eights) {
                if (two)
                    work(eights, std::integral_constant<int, 2>{});
                else
                    work(eights, std::integral_constant<int, 1>{});
            });
        if constexpr (WS > 1) {
            __syncthreads();
            const float* r = reinterpret_cast<const float*>(lds + group * WS * kWave);
            for (int q = part * 64 + lane; on && q < (u.n + 15) / 16 * 256; q += WS * 64) {  // float q % 256 of a tile
                const int t = q / 256, o = q % 256;
                float s[2] = {0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < WS; ++w)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        s[i] += r[w * (kWave / 4) + (t * 2 + i) * 256 + o];
                put(t * 16 + o / 4 % 16, f0 + o / 64 * 4 + (o & 3), s[0], s[1]);
            }
            __syncthreads();
        }
    }
}

// y = residual + sum over the units of down h: a workgroup takes 16 rows of
// hidden, its waves split the contraction over (unit, ffn).  A unit's columns
// are its tokens; behind its part of a unit a wave adds its sums to its own row
// of LDS per token.
template <int DT, int T8, int W>
__global__ __launch_bounds__(64 * W) void k_moe_down(MoeArgs a, ExpertPtrs ex, const Routing* in, const char* hbuf,
                                                     float* parts, int splits)
{
    using T = typename Elem<DT>::T;
    constexpr int XS = DT == MP_BF16 ? 2 : 1, kTokens = T8 < 4 ? T8 * 8 : kMoeMaxTokens;
    constexpr int kWave = Few<DT, 1, T8, XS>::kLds;
    __shared__ Routing rt;
    __shared__ float4 sums[W][kTokens][4];  // [token][4 of the 16 rows]
    __shared__ __attribute__((aligned(16))) char lds[W * kWave];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += 64 * W)
        reinterpret_cast<uint32_t*>(&rt)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    for (int i = lane; i < kTokens * 4; i += 64)
        sums[wave][i / 4][i % 4] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F);
    const int64_t plane = (int64_t)a.T * a.l.top_k * pitch;
    const int grp = blockIdx.x / splits, split = blockIdx.x % splits;
    const int64_t d0 = (int64_t)grp * 16;
    const int n = (int)uniform_u32(rt.units), me = split * W + wave, all = splits * W;
    // shares of the contraction: 4 blocks, a whole number of rounds for every count of tokens
    constexpr int kShareBlocks = 4, kShare = kShareBlocks * 128 / Fmt<DT>::esize;
    const int64_t shares = (F + kShare - 1) / kShare, s0 = shares * n * me / all, s1 = shares * n * (me + 1) / all;
    for (int k = 0; k < n; ++k) {
        const int64_t lo = s0 > shares * k ? s0 - shares * k : 0;
        const int64_t hi = s1 < shares * (k + 1) ? s1 - shares * k : shares;
        if (lo >= hi)
            continue;
        const Unit u = unit_of(rt, k);
        with_eights<T8>(u.n, [&](auto eights) {
            constexpr int E8 = decltype(eights)::value;
            using FD = Few<DT, 1, E8, XS>;
            static_assert(kShareBlocks % FD::kRound == 0);
            FD f;
            f.clear();
            f.lds = lds + wave * kWave;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int64_t r = d0 + FD::row_of(lane, m);
                f.w[0][m] = static_cast<const char*>(ex.p[u.e]) +
                            (a.l.down_off + (r < D ? r : D - 1) * F) * Fmt<DT>::esize + FD::off(lane);
            }
#pragma unroll
            for (int m = 0; m < E8; ++m) {
                const int pos = FD::row_of(lane, m), tok = rt.list[u.e][u.first + (pos < u.n ? pos : u.n - 1)];
#pragma unroll
                for (int i = 0; i < XS; ++i)
                    f.x[i][m] = reinterpret_cast<const char*>(
                                    h_row(reinterpret_cast<const T*>(hbuf) + i * plane, a, rt, u.e, tok, pitch)) +
                                FD::off(lane);
            }
            f.blocks(lo * kShareBlocks, hi * kShareBlocks, F);
#pragma unroll
            for (int t = 0; t < FD::NT; ++t) {
                const int pos = t * 16 + (lane & 15);
                if (pos < u.n) {
                    const float4 v = f.out(0, t);
                    float4& s = sums[wave][rt.list[u.e][u.first + pos]][lane >> 4];
                    s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
                }
            }
        });
    }
    __syncthreads();
    const float* r = reinterpret_cast<const float*>(sums);
    finish_rows<DT, 16>(a, d0, split, splits, parts, [&](int tok, int row) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            y += r[w * kTokens * 16 + tok * 16 + row];
        return y;
    });
}

// ---------------------------------------------------------------- one to four tokens
constexpr int kUpRows = 4;  // rows of ffn of an item: 4 of gate and 4 of up

// The first kernel: h in fp32.  WS waves split an item's contraction.
template <int DT, int TT, int WS>
__global__ __launch_bounds__(kUpThreads) void k_moe_up_gemv(MoeArgs a, ExpertPtrs ex, Routing* out, float* hbuf)
{
    using T = typename Elem<DT>::T;
    __shared__ Routing rt;
    __shared__ float gate[kMoeMaxTokens][kMoeMaxTop];
    __shared__ float lg[TT * 32];
    __shared__ float red[kUpWaves][2 * kUpRows * TT];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    logits_gemv<DT, TT>(a, lg);
    choose_experts<DT>(a, &rt, gate, lg);
    pass_on(rt, out);
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F);
    const int64_t tiles = (F + kUpRows - 1) / kUpRows, items = tiles * uniform_u32(rt.units);
    const int group = wave / WS, part = wave % WS;
    constexpr int kGroups = kUpWaves / WS;
    const bool two = a.l.up_off >= 0;
    for (int64_t it0 = (int64_t)blockIdx.x * kGroups; it0 < items; it0 += (int64_t)gridDim.x * kGroups) {
        const int64_t it = it0 + group;
        const bool on = it < items;
        const Unit u = unit_of(rt, on ? (int)(it / tiles) : 0);
        const int e = u.e, n = on ? u.n : 0;
        const int64_t f0 = on ? it % tiles * kUpRows : 0;
        auto work = [&](auto nt, auto na) {
            constexpr int NT = decltype(nt)::value, RG = kUpRows * decltype(na)::value;
            using G = Gemv<DT, RG, NT, false>;
            const char *w[RG], *x[NT];
#pragma unroll
            for (int i = 0; i < RG; ++i) {
                const int64_t r = f0 + i % kUpRows < F ? f0 + i % kUpRows : F - 1;
                w[i] = static_cast<const char*>(ex.p[e]) +
                       ((i < kUpRows ? a.l.gate_off : a.l.up_off) + r * D) * Fmt<DT>::esize;
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
                x[t] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) +
                                                     (int64_t)uniform_u32(rt.list[e][t < n ? t : n - 1]) * a.ldx);
            G g;
            g.clear();
            g.row(w, x, D, part, WS);
            g.put(red[wave]);
        };
        auto rows = [&](auto nt) {
            if (two)
                work(nt, std::integral_constant<int, 2>{});
            else
                work(nt, std::integral_constant<int, 1>{});
        };
        int nt = 1;  // token columns of the item's sums
        if (n == 1)
            rows(std::integral_constant<int, 1>{});
        if constexpr (TT > 1)
            if (n == 2) {
                nt = 2;
                rows(std::integral_constant<int, 2>{});
            }
        if constexpr (TT > 2)
            if (n > 2) {
                nt = 4;
                rows(std::integral_constant<int, 4>{});
            }
        if constexpr (WS > 1)
            __syncthreads();
        else
            __builtin_amdgcn_wave_barrier();  // the wave's own LDS, in order
        const int pos = lane % nt, i = lane / nt;
        if (part == 0 && i < kUpRows && pos < n && f0 + i < F) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < WS; ++k) {
                s[0] += red[wave + k][i * nt + pos];
                if (two)
                    s[1] += red[wave + k][(kUpRows + i) * nt + pos];
            }
            const int tok = rt.list[e][pos];
            h_row(hbuf, a, rt, e, tok, pitch)[f0 + i] = hidden_of(a, s[0], s[1], gate[tok][rt.slot[e][tok]]);
        }
        if constexpr (WS > 1)
            __syncthreads();
    }
}

// The second: a workgroup takes RG rows of hidden, its waves split the contraction over (expert, ffn).
template <int DT, int RG, int TT, int W>
__global__ __launch_bounds__(64 * W) void k_moe_down_gemv(MoeArgs a, ExpertPtrs ex, const Routing* in, const float* hbuf,
                                                          float* parts, int splits)
{
    __shared__ Routing rt;
    __shared__ float sums[W][TT][RG];
    __shared__ float red[W][RG * TT];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += 64 * W)
        reinterpret_cast<uint32_t*>(&rt)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    if (lane < RG * TT)
        sums[wave][lane / RG][lane % RG] = 0.0f;
    __syncthreads();
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F);
    const int grp = blockIdx.x / splits, split = blockIdx.x % splits;
    const int64_t d0 = (int64_t)grp * RG;
    const int me = split * W + wave, all = splits * W;
    const int n = (int)uniform_u32(rt.units);
    constexpr int kRun = Gemv<DT, RG, TT, true>::kRun;
    const int64_t runs = (F + kRun - 1) / kRun, s0 = runs * n * me / all, s1 = runs * n * (me + 1) / all;
    for (int k = 0; k < n; ++k) {
        const int64_t lo = s0 > runs * k ? s0 - runs * k : 0;
        const int64_t hi = s1 < runs * (k + 1) ? s1 - runs * k : runs;
        if (lo >= hi)
            continue;
        const Unit u = unit_of(rt, k);
        const int e = u.e, c = u.n;
        auto work = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            using G = Gemv<DT, RG, NT, true>;
            const char *w[RG], *x[NT];
#pragma unroll
            for (int i = 0; i < RG; ++i)
                w[i] = static_cast<const char*>(ex.p[e]) +
                       (a.l.down_off + (d0 + i < D ? d0 + i : D - 1) * F) * Fmt<DT>::esize;
#pragma unroll
            for (int t = 0; t < NT; ++t)
                x[t] = reinterpret_cast<const char*>(
                    h_row(hbuf, a, rt, e, (int)uniform_u32(rt.list[e][t < c ? t : c - 1]), pitch));
            G g;
            g.clear();
            g.runs(w, x, lo, 1, hi - lo, F);
            g.put(red[wave]);
            __builtin_amdgcn_wave_barrier();  // the wave's own LDS, in order
            if (lane < RG * NT && lane % NT < c)
                sums[wave][rt.list[e][lane % NT]][lane / NT] += red[wave][lane];
        };
        if (c == 1)
            work(std::integral_constant<int, 1>{});
        if constexpr (TT > 1)
            if (c == 2)
                work(std::integral_constant<int, 2>{});
        if constexpr (TT > 2)
            if (c > 2)
                work(std::integral_constant<int, 4>{});
    }
    __syncthreads();
    finish_rows<DT, RG>(a, d0, split, splits, parts, [&](int tok, int row) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            y += sums[w][tok][row];
        return y;
    });
}

// ---------------------------------------------------------------- which kernel
// Waves that an item of the first kernel is split over: enough to fill the chip.
// Its workgroups are at most two a CU, since each routes the tokens for itself
// first.  us of a whole call with at most 256, 512 and 1024 of them (bf16 but the last):
//   1 token, 8 experts of 1536 x 8960, 2 a token: 46, 45, 48; 4 tokens: 109, 111, 117
//   16 tokens: 164, 172, 174; 64 tokens: 231, 232, 240
//   24 tokens, 8 experts of 3584 x 18944: 649, 646, 650; 1 token: 150, 152, 150
//   7 tokens, 21 fp32 experts of 515 x 1030: 39, 37, 45
constexpr int kUpGroups = 512;
int up_split(int64_t items) { return items >= 4096 ? 1 : items >= 2048 ? 2 : items >= 1024 ? 4 : 8; }

// Experts reached at most.
int64_t most_experts(const MoeArgs& a) { return a.T * a.l.top_k < a.E ? a.T * a.l.top_k : a.E; }

// Workgroups per row group of the second kernel, with a KB of weight rows for
// each of their waves.  Fewer than 128 row groups are split, into 256 workgroups
// (20 tokens, 16 experts of 256 x 4000: 95 us with 16 workgroups, 46 with 256;
// five tokens through eight of 1536 x 8960: 121 us with 96, 104 with 192).
constexpr int kMaxSplit = 16;
int down_split(const mp_moe_layer& l, int64_t most, int64_t groups, int waves)
{
    const int64_t want = groups < 128 ? 256 / groups : 1;
    const int64_t room = most * l.ffn * (l.dtype == MP_F32 ? 4 : 2) / (1024 * waves);
    const int64_t s = want < room ? want : room;
    return (int)(s < 1 ? 1 : s > kMaxSplit ? kMaxSplit : s);
}

// The workspace: routing, h, the parts of a split second kernel.
struct MoeWs {
    Routing* rt;
    char* h;
    float* parts;
    uint64_t bytes;
};
MoeWs moe_ws(const mp_moe_layer& l, int64_t tokens, void* ws)
{
    char* p = static_cast<char*>(ws);
    const uint64_t h = 4ull * (uint64_t)tokens * (uint64_t)l.top_k * (uint64_t)moe_pitch(l.ffn);  // a plane of 4 bytes or two of 2
    const uint64_t parts = l.hidden < 128 * 16 ? 4ull * kMaxSplit * (uint64_t)tokens * (uint64_t)l.hidden : 0;
    return MoeWs{reinterpret_cast<Routing*>(p), p + sizeof(Routing), reinterpret_cast<float*>(p + sizeof(Routing) + h),
                 sizeof(Routing) + h + parts};
}

template <typename F>
void with_split(int ws, F go)
{
    if (ws == 1)
        go(std::integral_constant<int, 1>{});
    else if (ws == 2)
        go(std::integral_constant<int, 2>{});
    else if (ws == 4)
        go(std::integral_constant<int, 4>{});
    else
        go(std::integral_constant<int, 8>{});
}

template <int DT>
void join(const MoeArgs& a, const MoeWs& m, int splits, hipStream_t st)
{
    if (splits > 1)
        hipLaunchKernelGGL(k_moe_join<DT>, dim3((unsigned)((a.T * a.l.hidden + 255) / 256)), dim3(256), 0, st, a,
                           m.parts, splits);
}

template <int DT, int T8>
hipError_t moe_tiles(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    const MoeWs m = moe_ws(a.l, a.T, ws);
    const int64_t items = (a.l.ffn + 15) / 16 * most_experts(a);
    const int split = up_split(items);
    const int64_t need = (items * split + kUpWaves - 1) / kUpWaves;
    with_split(split, [&](auto s) {
        hipLaunchKernelGGL((k_moe_up<DT, T8, decltype(s)::value>), dim3((unsigned)(need < kUpGroups ? need : kUpGroups)),
                           dim3(kUpThreads), 0, st, a, ex, m.rt, m.h);
    });
    const int64_t groups = (a.l.hidden + 15) / 16;
    constexpr int W = 8;
    const int splits = down_split(a.l, most_experts(a), groups, W);
    hipLaunchKernelGGL((k_moe_down<DT, T8, W>), dim3((unsigned)(groups * splits)), dim3(64 * W), 0, st, a, ex, m.rt,
                       m.h, m.parts, splits);
    join<DT>(a, m, splits, st);
    return hipGetLastError();
}

template <int DT, int TT>
hipError_t moe_gemv(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    const MoeWs m = moe_ws(a.l, a.T, ws);
    float* h = reinterpret_cast<float*>(m.h);
    const int64_t items = (a.l.ffn + kUpRows - 1) / kUpRows * most_experts(a);
    const int split = up_split(items);
    const int64_t need = (items * split + kUpWaves - 1) / kUpWaves;
    with_split(split, [&](auto s) {
        hipLaunchKernelGGL((k_moe_up_gemv<DT, TT, decltype(s)::value>), dim3((unsigned)(need < kUpGroups ? need : kUpGroups)),
                           dim3(kUpThreads), 0, st, a, ex, m.rt, h);
    });
    constexpr int RG = 4, W = 8;
    const int64_t groups = (a.l.hidden + RG - 1) / RG;
    const int splits = down_split(a.l, most_experts(a), groups, W);
    hipLaunchKernelGGL((k_moe_down_gemv<DT, RG, TT, W>), dim3((unsigned)(groups * splits)), dim3(64 * W), 0, st, a, ex,
                       m.rt, h, m.parts, splits);
    join<DT>(a, m, splits, st);
    return hipGetLastError();
}

template <int DT>
hipError_t moe_d(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    if (a.T == 1)
        return moe_gemv<DT, 1>(a, ex, ws, st);
    if (a.T <= kGemvTokens)
        return moe_gemv<DT, 4>(a, ex, ws, st);
    if (a.T <= 8)
        return moe_tiles<DT, 1>(a, ex, ws, st);
    if (a.T <= 16)
        return moe_tiles<DT, 2>(a, ex, ws, st);
    return moe_tiles<DT, 4>(a, ex, ws, st);
}

}  // namespace

hipError_t launch_moe(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    return a.l.dtype == MP_F32 ? moe_d<MP_F32>(a, ex, ws, st) : moe_d<MP_BF16>(a, ex, ws, st);
}

uint64_t moe_ws_bytes(const mp_moe_layer& l, int64_t tokens)
{
    return moe_ws(l, tokens, nullptr).bytes;
}

}  // namespace mp
