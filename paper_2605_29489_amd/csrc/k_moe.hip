// A layer that routes a few tokens among experts, in two kernels: routing with
// the gate and up products, then the down products with the sum over experts.
#include "ffn_common.h"
#include "mm_few.h"
#include "mp_internal.h"
#include <cstdlib>

namespace mp {
namespace {

constexpr int kNone = 0xff;  // slot of a token that does not have the expert

// What the first kernel tells the second, at the start of the workspace.
struct Routing {
    uint8_t slot[kMaxK][kMoeMaxTokens];  // choice number of expert e for token t, or kNone
    uint8_t list[kMaxK][kMoeMaxTokens];  // the tokens that have expert e, in order
    uint32_t count[kMaxK];               // how many
    uint32_t reached;                    // experts that some token has
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

// The expert number k of those reached.
__device__ inline int nth_expert(uint32_t reached, int64_t k)
{
    for (; k > 0; --k)
        reached &= reached - 1;
    return __ffs(reached) - 1;
}

constexpr int kUpWaves = 8, kUpThreads = 64 * kUpWaves;
constexpr int kGemvTokens = 4;  // up to so many, the vector ALU multiplies

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
        const unsigned long long m = __ballot(lane < kMaxK && rt->count[lane & 31] != 0);
        if (lane == 0)
            rt->reached = (uint32_t)m;
    }
    __syncthreads();
}

// Routing.  Every workgroup routes all tokens for itself, by the same
// instructions, so that the gate and up products need no launch of their own
// behind it.  lg: 32 floats of LDS per token (of whole token tiles); red: LDS
// for the partial tiles.
template <int DT, int TT>
__device__ inline void logits_tiles(const MoeArgs& a, float* lg, float4* red)
{
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    using F = Few<DT, 16, 1, TT, 1>;
    const int64_t D = a.l.hidden, whole = F::whole(D);
    F f;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int tok = t * 16 + (lane & 15);
        f.x[t] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + (int64_t)(tok < a.T ? tok : a.T - 1) * a.ldx) +
                 F::x_off(lane);
    }
    for (int e0 = 0; e0 < a.E; e0 += 16) {
        f.clear();
        const int e = e0 + F::row_of(lane);
        f.w[0] = reinterpret_cast<const char*>(static_cast<const T*>(a.router) + (e < a.E ? e : a.E - 1) * D) +
                 F::w_off(lane);
        f.rounds(whole * wave / kUpWaves, whole * (wave + 1) / kUpWaves);
        if (wave == kUpWaves - 1 && F::more(D))
            f.rest(D);
#pragma unroll
        for (int t = 0; t < TT; ++t)
            red[(wave * TT + t) * 64 + lane] = f.out(0, t);
        __syncthreads();
        sum_tiles<16, TT, kUpWaves>(red, threadIdx.x, kUpThreads,
                                    [&](int t, int row, int tok, float v) { lg[(t * 16 + tok) * 32 + e0 + row] = v; });
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

// act(g) * u * gate
__device__ inline float hidden_of(const MoeArgs& a, float g, float u, float gate)
{
    const float h = act_of(a.l.act, g);
    return (a.l.up_off >= 0 ? h * u : h) * gate;
}

// ---------------------------------------------------------------- five tokens and more
// h = act(gate x) * (up x) times the token's gate for every (expert that a
// token has, 16 rows of ffn): WS waves split an item's contraction.  The B
// operand's columns are the expert's tokens, up to 16 TT of them.  h is stored
// as one value (fp32) or as the bf16 rounding and the rounded remainder, in two
// planes.
template <int DT, int TT, int WS>
__global__ __launch_bounds__(kUpThreads, 4) void k_moe_up(MoeArgs a, ExpertPtrs ex, Routing* out, char* hbuf)
{
    using T = typename Elem<DT>::T;
    __shared__ Routing rt;
    __shared__ float gate[kMoeMaxTokens][kMoeMaxTop];
    __shared__ float4 red[kUpWaves * 2 * TT * 64];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    logits_tiles<DT, TT>(a, reinterpret_cast<float*>(red + kUpWaves * TT * 64), red);
    choose_experts<DT>(a, &rt, gate, reinterpret_cast<float*>(red + kUpWaves * TT * 64));
    pass_on(rt, out);
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F), plane = (int64_t)a.T * a.l.top_k * pitch;
    const int64_t tiles = (F + 15) / 16, items = tiles * __popc(rt.reached);
    const int group = wave / WS, part = wave % WS;
    constexpr int kGroups = kUpWaves / WS;
    const bool two = a.l.up_off >= 0;
    // the same trips for the whole workgroup: there are barriers inside
    for (int64_t it0 = (int64_t)blockIdx.x * kGroups; it0 < items; it0 += (int64_t)gridDim.x * kGroups) {
        const int64_t it = it0 + group;
        const bool on = it < items;
        const int e = on ? nth_expert(rt.reached, it / tiles) : 0;
        const int64_t f0 = on ? it % tiles * 16 : 0;
        const int n = on ? (int)uniform_u32(rt.count[e]) : 0;
        // outputs of token number `pos` of the expert, row f
        auto put = [&](int pos, int64_t f, float g, float u) {
            if (pos >= n || f >= F)
                return;
            const int tok = rt.list[e][pos];
            const float h = hidden_of(a, g, u, gate[tok][rt.slot[e][tok]]);
            T* p = h_row(reinterpret_cast<T*>(hbuf), a, rt, e, tok, pitch) + f;
            *p = (T)h;
            if constexpr (DT == MP_BF16) {
                const float hi = (float)(T)h;
                p[plane] = (T)(fabsf(hi) < INFINITY ? h - hi : 0.0f);  // an infinite or NaN h has no remainder
            }
        };
        // the item with NT token tiles
        auto work = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            float4 sum[2][NT];  // gate and up
            const int64_t row = f0 + (lane & 15) < F ? f0 + (lane & 15) : F - 1;
            auto go = [&](auto& f, int na) {
                using FW = std::remove_reference_t<decltype(f)>;
                const char* const base =
                    static_cast<const char*>(ex.p[e]) + row * D * Fmt<DT>::esize + FW::w_off(lane);
                f.clear();
                f.w[0] = base + a.l.gate_off * Fmt<DT>::esize;
                if (na > 1)
                    f.w[na - 1] = base + a.l.up_off * Fmt<DT>::esize;
#pragma unroll
                for (int t = 0; t < NT; ++t) {  // columns past the last token repeat it; their outputs are dropped
                    const int pos = t * 16 + (lane & 15), tok = rt.list[e][pos < n ? pos : n - 1];
                    f.x[t] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + tok * a.ldx) + FW::x_off(lane);
                }
                const int64_t whole = FW::whole(D);
                f.rounds(whole * part / WS, whole * (part + 1) / WS);
                if (part == WS - 1 && FW::more(D))
                    f.rest(D);
            };
            if (two) {
                Few<DT, 16, 2, NT, 1> f;
                go(f, 2);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sum[0][t] = f.out(0, t);
                    sum[1][t] = f.out(1, t);
                }
            } else {
                Few<DT, 16, 1, NT, 1> f;
                go(f, 1);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sum[0][t] = f.out(0, t);
                    sum[1][t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (WS == 1) {
                    const float* g = reinterpret_cast<const float*>(&sum[0][t]);
                    const float* u = reinterpret_cast<const float*>(&sum[1][t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        put(t * 16 + (lane & 15), f0 + (lane >> 4) * 4 + j, g[j], u[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        red[(((group * WS + part) * TT + t) * 2 + i) * 64 + lane] = sum[i][t];
                }
            }
        };
        const int nt = (n + 15) / 16;
        if (nt == 1)
            work(std::integral_constant<int, 1>{});
        if constexpr (TT > 1)
            if (nt == 2)
                work(std::integral_constant<int, 2>{});
        if constexpr (TT > 2)
            if (nt > 2)
                work(std::integral_constant<int, 4>{});
        if constexpr (WS > 1) {
            __syncthreads();
            const float* r = reinterpret_cast<const float*>(red + group * WS * TT * 128);
            for (int q = part * 64 + lane; q < nt * 256; q += WS * 64) {  // float q % 256 of a token tile
                const int t = q / 256, o = q % 256;
                float s[2] = {0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < WS; ++w)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        s[i] += r[((w * TT + t) * 2 + i) * 256 + o];
                put(t * 16 + o / 4 % 16, f0 + o / 64 * 4 + (o & 3), s[0], s[1]);
            }
            __syncthreads();
        }
    }
}

// y = residual + sum over the experts of down h: a workgroup takes 16 rows of
// hidden, its waves split the contraction over (expert, ffn).  An expert's
// columns are its tokens; behind its part of an expert a wave adds its sums to
// its own row of LDS per token.
template <int DT, int TT, int W>
__global__ __launch_bounds__(64 * W) void k_moe_down(MoeArgs a, ExpertPtrs ex, const Routing* in, const char* hbuf)
{
    using T = typename Elem<DT>::T;
    constexpr int XS = DT == MP_BF16 ? 2 : 1;
    __shared__ Routing rt;
    __shared__ float4 sums[W][TT * 16][4];  // [token][4 of the 16 rows]
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += 64 * W)
        reinterpret_cast<uint32_t*>(&rt)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    for (int i = lane; i < TT * 64; i += 64)
        sums[wave][i / 4][i % 4] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F);
    const int64_t plane = (int64_t)a.T * a.l.top_k * pitch;
    const int64_t d0 = (int64_t)blockIdx.x * 16, row = d0 + (lane & 15) < D ? d0 + (lane & 15) : D - 1;
    const uint32_t reached = uniform_u32(rt.reached);
    const int n = __popc(reached);
    // shares of the contraction in 256 bytes of a row
    constexpr int kShare = 256 / Fmt<DT>::esize;
    const int64_t shares = F / kShare, s0 = shares * n * wave / W, s1 = shares * n * (wave + 1) / W;
    uint32_t left = reached;
    for (int k = 0; k < n; ++k, left &= left - 1) {
        const int64_t lo = s0 > shares * k ? s0 - shares * k : 0;
        const int64_t hi = s1 < shares * (k + 1) ? s1 - shares * k : shares;
        const bool rest = F % kShare && k % W == wave;
        if (lo >= hi && !rest)
            continue;
        const int e = __ffs(left) - 1, c = (int)uniform_u32(rt.count[e]);
        auto work = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            using FD = Few<DT, 16, 1, NT, XS>;
            constexpr int kPer = 256 / (FD::kRound * FD::kStep);  // rounds of a share
            static_assert(kPer >= 1);
            FD f;
            f.clear();
            f.w[0] = static_cast<const char*>(ex.p[e]) + (a.l.down_off + row * F) * Fmt<DT>::esize + FD::w_off(lane);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int pos = t * 16 + (lane & 15), tok = rt.list[e][pos < c ? pos : c - 1];
#pragma unroll
                for (int i = 0; i < XS; ++i)
                    f.x[i * NT + t] = reinterpret_cast<const char*>(
                                          h_row(reinterpret_cast<const T*>(hbuf) + i * plane, a, rt, e, tok, pitch)) +
                                      FD::x_off(lane);
            }
            f.rounds(lo * kPer, hi * kPer);
            if (rest) {  // behind the shares: rounds, steps, part of a step
                f.rounds(shares * kPer, FD::whole(F));
                if (FD::more(F))
                    f.rest(F);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int pos = t * 16 + (lane & 15);
                if (pos < c) {
                    const float4 v = f.out(0, t);
                    float4& s = sums[wave][rt.list[e][pos]][lane >> 4];
                    s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
                }
            }
        };
        if (c <= 16)
            work(std::integral_constant<int, 1>{});
        if constexpr (TT > 1)
            if (c > 16 && c <= 32)
                work(std::integral_constant<int, 2>{});
        if constexpr (TT > 2)
            if (c > 32)
                work(std::integral_constant<int, 4>{});
    }
    __syncthreads();
    const float* r = reinterpret_cast<const float*>(sums);
    for (int q = threadIdx.x; q < a.T * 16; q += 64 * W) {
        const int tok = q / 16;
        const int64_t d = d0 + q % 16;
        if (d >= D)
            continue;
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            y += r[w * TT * 256 + q];
        if (a.residual)
            y += (float)static_cast<const T*>(a.residual)[tok * a.ldr + d];
        static_cast<T*>(a.y)[tok * a.ldy + d] = (T)y;
    }
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
    const int64_t tiles = (F + kUpRows - 1) / kUpRows, items = tiles * __popc(uniform_u32(rt.reached));
    const int group = wave / WS, part = wave % WS;
    constexpr int kGroups = kUpWaves / WS;
    const bool two = a.l.up_off >= 0;
    for (int64_t it0 = (int64_t)blockIdx.x * kGroups; it0 < items; it0 += (int64_t)gridDim.x * kGroups) {
        const int64_t it = it0 + group;
        const bool on = it < items;
        const int e = on ? nth_expert(uniform_u32(rt.reached), it / tiles) : 0;
        const int64_t f0 = on ? it % tiles * kUpRows : 0;
        const int n = on ? (int)uniform_u32(rt.count[e]) : 0;
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
__global__ __launch_bounds__(64 * W) void k_moe_down_gemv(MoeArgs a, ExpertPtrs ex, const Routing* in, const float* hbuf)
{
    using T = typename Elem<DT>::T;
    __shared__ Routing rt;
    __shared__ float sums[W][TT][RG];
    __shared__ float red[W][RG * TT];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += 64 * W)
        reinterpret_cast<uint32_t*>(&rt)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    if (lane < RG * TT)
        sums[wave][lane / RG][lane % RG] = 0.0f;
    __syncthreads();
    const int64_t D = a.l.hidden, F = a.l.ffn, pitch = moe_pitch(F), d0 = (int64_t)blockIdx.x * RG;
    const uint32_t reached = uniform_u32(rt.reached);
    const int n = __popc(reached);
    constexpr int kRun = Gemv<DT, RG, TT, true>::kRun;
    const int64_t runs = F / kRun, s0 = runs * n * wave / W, s1 = runs * n * (wave + 1) / W;
    uint32_t left = reached;
    for (int k = 0; k < n; ++k, left &= left - 1) {
        const int64_t lo = s0 > runs * k ? s0 - runs * k : 0;
        const int64_t hi = s1 < runs * (k + 1) ? s1 - runs * k : runs;
        const bool rest = F % kRun && k % W == wave;
        if (lo >= hi && !rest)
            continue;
        const int e = __ffs(left) - 1, c = (int)uniform_u32(rt.count[e]);
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
            g.runs(w, x, lo, 1, hi - lo);
            if (rest)
                g.rest(w, x, F);
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
    const int tok = threadIdx.x / RG;
    const int64_t d = d0 + threadIdx.x % RG;
    if (tok >= a.T || d >= D)
        return;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w)
        y += sums[w][tok][threadIdx.x % RG];
    if (a.residual)
        y += (float)static_cast<const T*>(a.residual)[tok * a.ldr + d];
    static_cast<T*>(a.y)[tok * a.ldy + d] = (T)y;
}

// ---------------------------------------------------------------- which kernel
// Waves that an item of the first kernel is split over: enough to fill the chip.
int up_split(int64_t items) { return items >= 4096 ? 1 : items >= 2048 ? 2 : items >= 1024 ? 4 : 8; }

// Experts reached at most.
int64_t most_experts(const MoeArgs& a) { return a.T * a.l.top_k < a.E ? a.T * a.l.top_k : a.E; }

template <int WS>
using int_c = std::integral_constant<int, WS>;

template <typename F>
void with_split(int ws, F go)
{
    if (ws == 1)
        go(int_c<1>{});
    else if (ws == 2)
        go(int_c<2>{});
    else if (ws == 4)
        go(int_c<4>{});
    else
        go(int_c<8>{});
}

template <int DT, int TT>
hipError_t moe_tiles(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    Routing* rt = static_cast<Routing*>(ws);
    char* h = static_cast<char*>(ws) + sizeof(Routing);
    const int64_t items = (a.l.ffn + 15) / 16 * most_experts(a);
    int split = up_split(items); int G1 = 512;
    if (const char* ev = getenv("MOE_WS")) split = atoi(ev);
    if (const char* ev = getenv("MOE_G1")) G1 = atoi(ev);
    const int64_t need = (items * split + kUpWaves - 1) / kUpWaves;
    with_split(split, [&](auto s) {
        hipLaunchKernelGGL((k_moe_up<DT, TT, decltype(s)::value>), dim3((unsigned)(need < G1 ? need : G1)),
                           dim3(kUpThreads), 0, st, a, ex, rt, h);
    });
    const dim3 g2((unsigned)((a.l.hidden + 15) / 16));
    int W2 = 16;
    if (const char* ev = getenv("MOE_W2")) W2 = atoi(ev);
    if (W2 == 16)
    hipLaunchKernelGGL((k_moe_down<DT, TT, 16>), g2, dim3(1024), 0, st, a, ex, rt, h);
    else
    hipLaunchKernelGGL((k_moe_down<DT, TT, 8>), g2, dim3(512), 0, st, a, ex, rt, h);
    return hipGetLastError();
}

template <int DT, int TT>
hipError_t moe_gemv(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    Routing* rt = static_cast<Routing*>(ws);
    float* h = reinterpret_cast<float*>(static_cast<char*>(ws) + sizeof(Routing));
    const int64_t items = (a.l.ffn + kUpRows - 1) / kUpRows * most_experts(a);
    int split = up_split(items); int G1 = 512;
    if (const char* ev = getenv("MOE_WS")) split = atoi(ev);
    if (const char* ev = getenv("MOE_G1")) G1 = atoi(ev);
    const int64_t need = (items * split + kUpWaves - 1) / kUpWaves;
    with_split(split, [&](auto s) {
        hipLaunchKernelGGL((k_moe_up_gemv<DT, TT, decltype(s)::value>), dim3((unsigned)(need < G1 ? need : G1)),
                           dim3(kUpThreads), 0, st, a, ex, rt, h);
    });
    int W2 = 8;
    if (const char* ev = getenv("MOE_W2")) W2 = atoi(ev);
    constexpr int RG = 4;
    const dim3 g2((unsigned)((a.l.hidden + RG - 1) / RG));
    if (W2 == 8)
    hipLaunchKernelGGL((k_moe_down_gemv<DT, RG, TT, 8>), g2, dim3(512), 0, st, a, ex, rt, h);
    else
    hipLaunchKernelGGL((k_moe_down_gemv<DT, RG, TT, 4>), g2, dim3(256), 0, st, a, ex, rt, h);
    return hipGetLastError();
}

template <int DT>
hipError_t moe_d(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    if (a.T == 1)
        return moe_gemv<DT, 1>(a, ex, ws, st);
    if (a.T <= kGemvTokens)
        return moe_gemv<DT, 4>(a, ex, ws, st);
    if (a.T <= 16)
        return moe_tiles<DT, 1>(a, ex, ws, st);
    if (a.T <= 32)
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
    // fp32: one plane of 4 bytes; bf16: two of 2
    return sizeof(Routing) + 4ull * (uint64_t)tokens * (uint64_t)l.top_k * (uint64_t)moe_pitch(l.ffn);
}

}  // namespace mp
