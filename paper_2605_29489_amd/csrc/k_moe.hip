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

constexpr int kUpWaves = 8, kUpThreads = 64 * kUpWaves;

// Routing.  Every workgroup routes all tokens for itself, by the same
// instructions, so that the gate and up products need no launch of their own
// behind it: the logits are matrix-core products of the router's rows and the
// tokens, split over the waves; then 32 lanes take a token, one expert each,
// and a choice's number is the count of the logits above it.
template <int DT, int TT>
__device__ inline void route(const MoeArgs& a, Routing* rt, float (*gate)[kMoeMaxTop], float* red)
{
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    const int64_t D = a.l.hidden, whole = few_whole<DT>(D);
    const char* x[TT];
    bool go[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int tok = t * 16 + (lane & 15);
        go[t] = true;
        x[t] = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + (int64_t)(tok < a.T ? tok : a.T - 1) * a.ldx) +
               (lane >> 4) * 16;
    }
    float* lg = red + kUpWaves * TT * 256;  // [token][32]
    for (int e0 = 0; e0 < a.E; e0 += 16) {
        f32x4 acc[1][TT] = {};
        const int e = e0 + (lane & 15);
        const char* const w[1] = {
            reinterpret_cast<const char*>(static_cast<const T*>(a.router) + (e < a.E ? e : a.E - 1) * D) +
            (lane >> 4) * 16};
        few_steps<DT, 1, TT, 1, 4>(acc, w, x, go, whole * wave / kUpWaves, whole * (wave + 1) / kUpWaves);
        if (wave == kUpWaves - 1 && few_rest<DT>(D))
            few_tail<DT, 1, TT, 1>(acc, w, x, go, whole, few_rest<DT>(D));
#pragma unroll
        for (int t = 0; t < TT; ++t)
            reinterpret_cast<float4*>(red)[(wave * TT + t) * 64 + lane] =
                make_float4(acc[0][t][0], acc[0][t][1], acc[0][t][2], acc[0][t][3]);
        __syncthreads();
        sum_tiles<TT>(reinterpret_cast<const float4*>(red), kUpWaves, threadIdx.x, kUpThreads,
                      [&](int i, const float4& s) {
                          const int tok = (i >> 6) * 16 + (i & 15), ee = e0 + ((i & 63) >> 4) * 4;
                          *reinterpret_cast<float4*>(lg + tok * 32 + ee) = s;
                      });
        __syncthreads();
    }
    if (threadIdx.x == 0)
        rt->reached = 0;
    __syncthreads();
    const int e = lane & 31, E = a.E, top = a.l.top_k;
    const float b =
        a.router_bias && e < E ? (float)static_cast<const T*>(a.router_bias)[e] : 0.0f;
    uint32_t mine = 0;
    for (int t0 = 0; t0 < a.T; t0 += 2 * kUpWaves) {  // the same trips for every lane of a wave
        const int t = t0 + 2 * wave + (lane >> 5);
        const bool on = t < a.T && e < E;
        const float l = on ? lg[t * 32 + e] + b : -INFINITY;
        const uint32_t key = on ? logit_key(l) : 0u;  // below every logit's
        int rank = 0;
        float best = -INFINITY;
        uint32_t bk = 0;
        for (int o = 0; o < E; ++o) {
            const uint32_t k2 = __shfl(key, o, 32);
            const float l2 = __shfl(l, o, 32);
            rank += k2 > key || (k2 == key && o < e);
            if (k2 > bk) {
                bk = k2;
                best = l2;
            }
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
        mine |= has ? 1u << e : 0u;
    }
    if (mine)
        atomicOr(&rt->reached, mine);
    __syncthreads();
}

// h = act(gate x) * (up x) times the token's gate for every (expert that a
// token has, 16 rows of ffn): WS waves split an item's contraction.  h is
// stored as one value (fp32) or as the bf16 rounding and the rounded
// remainder, in two planes.
template <int DT, int TT, int WS>
__global__ __launch_bounds__(kUpThreads) void k_moe_up(MoeArgs a, ExpertPtrs ex, Routing* out, char* hbuf)
{
    using T = typename Elem<DT>::T;
    __shared__ Routing rt;
    __shared__ float gate[kMoeMaxTokens][kMoeMaxTop];
    __shared__ float4 red4[(kUpWaves * 2 * TT + 2 * TT) * 64];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    route<DT, TT>(a, &rt, gate, reinterpret_cast<float*>(red4));
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += kUpThreads)
            reinterpret_cast<uint32_t*>(out)[i] = reinterpret_cast<const uint32_t*>(&rt)[i];
    const int64_t D = a.l.hidden, F = a.l.ffn, whole = few_whole<DT>(D), pitch = moe_pitch(F);
    const int rest = few_rest<DT>(D);
    const int64_t tiles = (F + 15) / 16, items = tiles * __popc(rt.reached);
    const int group = wave / WS, part = wave % WS;
    constexpr int kGroups = kUpWaves / WS;
    const bool two = a.l.up_off >= 0;
    // the same trips for the whole workgroup: there are barriers inside
    for (int64_t it0 = (int64_t)blockIdx.x * kGroups; it0 < items; it0 += (int64_t)gridDim.x * kGroups) {
        const int64_t it = it0 + group;
        const bool on = it < items;
        uint32_t left = rt.reached;
        for (int64_t k = on ? it / tiles : 0; k > 0; --k)
            left &= left - 1;
        const int e = __ffs(left) - 1;
        const int64_t f0 = on ? it % tiles * 16 : 0;
        f32x4 acc[2][TT] = {};
        if (on) {
            const int64_t row = f0 + (lane & 15) < F ? f0 + (lane & 15) : F - 1;
            const char* const base = static_cast<const char*>(ex.p[e]) + row * D * Fmt<DT>::esize + (lane >> 4) * 16;
            const char* const w[2] = {base + a.l.gate_off * Fmt<DT>::esize,
                                      base + (two ? a.l.up_off : a.l.gate_off) * Fmt<DT>::esize};
            const char* x[TT];
            bool go[TT];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const int tok = t * 16 + (lane & 15);
                go[t] = tok < a.T && rt.slot[e][tok] != kNone;
                x[t] = go[t] ? reinterpret_cast<const char*>(static_cast<const T*>(a.x) + tok * a.ldx) +
                                   (lane >> 4) * 16
                             : reinterpret_cast<const char*>(g_zero_steps);
            }
            const int64_t s0 = whole * part / WS, s1 = whole * (part + 1) / WS;
            if (two) {
                few_steps<DT, 2, TT, 1, few_unroll(2 + TT)>(acc, w, x, go, s0, s1);
                if (part == WS - 1 && rest)
                    few_tail<DT, 2, TT, 1>(acc, w, x, go, whole, rest);
            } else {
                f32x4 one[1][TT] = {};
                const char* const w1[1] = {w[0]};
                few_steps<DT, 1, TT, 1, few_unroll(1 + TT)>(one, w1, x, go, s0, s1);
                if (part == WS - 1 && rest)
                    few_tail<DT, 1, TT, 1>(one, w1, x, go, whole, rest);
#pragma unroll
                for (int t = 0; t < TT; ++t)
                    acc[0][t] = one[0][t];
            }
        }
        auto put = [&](int i, const float4& g4, const float4& u4) {
            const int tok = (i >> 6) * 16 + (i & 15);
            const int64_t f = f0 + ((i & 63) >> 4) * 4;
            if (!on || tok >= a.T || rt.slot[e][tok] == kNone)
                return;
            const int slot = rt.slot[e][tok];
            const float gt = gate[tok][slot];
            const float g[4] = {g4.x, g4.y, g4.z, g4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
            const int64_t at = ((int64_t)tok * a.l.top_k + slot) * pitch + f;
            const int64_t plane = (int64_t)a.T * a.l.top_k * pitch;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (f + j >= F)
                    break;
                float h = act_of(a.l.act, g[j]);
                h = (two ? h * u[j] : h) * gt;
                T* p = reinterpret_cast<T*>(hbuf) + at + j;
                *p = (T)h;
                if constexpr (DT == MP_BF16) {
                    const float hi = (float)(T)h;
                    // an infinite or NaN h has no remainder
                    p[plane] = (T)(fabsf(hi) < INFINITY ? h - hi : 0.0f);
                }
            }
        };
        if constexpr (WS == 1) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
                put(t * 64 + lane, make_float4(acc[0][t][0], acc[0][t][1], acc[0][t][2], acc[0][t][3]),
                    make_float4(acc[1][t][0], acc[1][t][1], acc[1][t][2], acc[1][t][3]));
        } else {
            float4* r = red4 + group * WS * 2 * TT * 64;
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    r[((part * TT + t) * 2 + i) * 64 + lane] =
                        make_float4(acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]);
            __syncthreads();
            // gate and up tiles of a token tile lie next to each other: wave `part` takes token tiles part, part + WS, ..
            for (int t = part; t < TT; t += WS) {
                float4 s[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[i] = r[(t * 2 + i) * 64 + lane];
                    for (int w = 1; w < WS; ++w) {
                        const float4 v = r[((w * TT + t) * 2 + i) * 64 + lane];
                        s[i].x += v.x;
                        s[i].y += v.y;
                        s[i].z += v.z;
                        s[i].w += v.w;
                    }
                }
                put(t * 64 + lane, s[0], s[1]);
            }
            __syncthreads();
        }
    }
}

// y = residual + sum over the experts of down h: a workgroup takes 16 rows of
// hidden, its waves split the contraction over (expert, ffn).  A token without
// the expert is a column of zeros, so the sum over experts stays in the
// accumulators.
template <int DT, int TT, int W>
__global__ __launch_bounds__(64 * W) void k_moe_down(MoeArgs a, ExpertPtrs ex, const Routing* in, const char* hbuf)
{
    using T = typename Elem<DT>::T;
    constexpr int XS = DT == MP_BF16 ? 2 : 1;
    __shared__ Routing rt;
    __shared__ float4 red[W * TT * 64];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < (int)(sizeof(Routing) / 4); i += 64 * W)
        reinterpret_cast<uint32_t*>(&rt)[i] = reinterpret_cast<const uint32_t*>(in)[i];
    __syncthreads();
    const int64_t D = a.l.hidden, F = a.l.ffn, whole = few_whole<DT>(F), pitch = moe_pitch(F);
    const int rest = few_rest<DT>(F), n = __popc(rt.reached);
    const int64_t plane = (int64_t)a.T * a.l.top_k * pitch * Fmt<DT>::esize;
    const int64_t d0 = (int64_t)blockIdx.x * 16, row = d0 + (lane & 15) < D ? d0 + (lane & 15) : D - 1;
    const int64_t s0 = whole * n * wave / W, s1 = whole * n * (wave + 1) / W;
    f32x4 acc[1][TT] = {};
    uint32_t left = rt.reached;
    for (int k = 0; k < n; ++k, left &= left - 1) {
        const int64_t lo = s0 > whole * k ? s0 - whole * k : 0;
        const int64_t hi = s1 < whole * (k + 1) ? s1 - whole * k : whole;
        const bool tail = rest && k % W == wave;
        if (lo >= hi && !tail)
            continue;
        const int e = __ffs(left) - 1;
        const char* const w[1] = {static_cast<const char*>(ex.p[e]) + (a.l.down_off + row * F) * Fmt<DT>::esize +
                                  (lane >> 4) * 16};
        const char* x[TT * XS];
        bool go[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int tok = t * 16 + (lane & 15);
            go[t] = tok < a.T && rt.slot[e][tok] != kNone;
#pragma unroll
            for (int i = 0; i < XS; ++i)
                x[i * TT + t] =
                    go[t] ? hbuf + i * plane +
                                ((int64_t)tok * a.l.top_k + rt.slot[e][tok]) * pitch * Fmt<DT>::esize + (lane >> 4) * 16
                          : reinterpret_cast<const char*>(g_zero_steps);
        }
        few_steps<DT, 1, TT, XS, few_unroll(1 + TT * XS)>(acc, w, x, go, lo, hi);
        if (tail)
            few_tail<DT, 1, TT, XS>(acc, w, x, go, whole, rest);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
        red[(wave * TT + t) * 64 + lane] = make_float4(acc[0][t][0], acc[0][t][1], acc[0][t][2], acc[0][t][3]);
    __syncthreads();
    sum_tiles<TT>(red, W, threadIdx.x, 64 * W, [&](int i, const float4& s) {
        const int tok = (i >> 6) * 16 + (i & 15);
        const int64_t d = d0 + ((i & 63) >> 4) * 4;
        const float v[4] = {s.x, s.y, s.z, s.w};
        if (tok >= a.T)
            return;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) {
                float y = v[j];
                if (a.residual)
                    y += (float)static_cast<const T*>(a.residual)[tok * a.ldr + d + j];
                static_cast<T*>(a.y)[tok * a.ldy + d + j] = (T)y;
            }
    });
}

template <int DT, int TT>
hipError_t moe_t(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    Routing* rt = static_cast<Routing*>(ws);
    char* h = static_cast<char*>(ws) + sizeof(Routing);
    // experts reached at most, and the waves an item of the first kernel is split over: enough waves to fill the chip
    const int most = a.T * a.l.top_k < a.E ? a.T * a.l.top_k : a.E;
    const int64_t items = (a.l.ffn + 15) / 16 * most;
    const int ws_ = items >= 2048 ? 1 : items >= 1024 ? 2 : items >= 512 ? 4 : 8;
    const int64_t need = (items * ws_ + kUpWaves - 1) / kUpWaves;
    const dim3 g1((unsigned)(need < 512 ? need : 512)), b1(kUpThreads);
    if (ws_ == 1)
        hipLaunchKernelGGL((k_moe_up<DT, TT, 1>), g1, b1, 0, st, a, ex, rt, h);
    else if (ws_ == 2)
        hipLaunchKernelGGL((k_moe_up<DT, TT, 2>), g1, b1, 0, st, a, ex, rt, h);
    else if (ws_ == 4)
        hipLaunchKernelGGL((k_moe_up<DT, TT, 4>), g1, b1, 0, st, a, ex, rt, h);
    else
        hipLaunchKernelGGL((k_moe_up<DT, TT, 8>), g1, b1, 0, st, a, ex, rt, h);
    constexpr int W = TT == 1 ? 16 : 8;  // more tokens take more registers than a wave of 16 has
    hipLaunchKernelGGL((k_moe_down<DT, TT, W>), dim3((unsigned)((a.l.hidden + 15) / 16)), dim3(64 * W), 0, st, a, ex,
                       rt, h);
    return hipGetLastError();
}

template <int DT>
hipError_t moe_d(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    if (a.T <= 16)
        return moe_t<DT, 1>(a, ex, ws, st);
    if (a.T <= 32)
        return moe_t<DT, 2>(a, ex, ws, st);
    return moe_t<DT, 4>(a, ex, ws, st);
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
