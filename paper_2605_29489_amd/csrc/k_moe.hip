// A layer that routes a few tokens among experts.
#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

// Order of the logits with NaN above every number: larger key, larger logit.
__device__ inline uint32_t logit_key(float l)
{
    if (l != l)
        return 0xffffffffu;
    const uint32_t u = __float_as_uint(l + 0.0f);  // -0 counts as 0
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// One workgroup per token: logits by waves, then the choice by one thread.
template <typename T>
__global__ __launch_bounds__(256) void k_route(MoeArgs a, int32_t* ids, float* gates)
{
    __shared__ float lg[kMaxK];
    const int t = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const T* x = static_cast<const T*>(a.x) + t * a.ldx;
    for (int e = wave; e < a.E; e += 4) {
        const T* r = static_cast<const T*>(a.router) + (int64_t)e * a.l.hidden;
        float s = 0.0f;
        for (int64_t d = lane; d < a.l.hidden; d += 64)
            s = fmaf((float)x[d], (float)r[d], s);
        s = wave_xor_sum(s);
        if (lane == 0)
            lg[e] = a.router_bias ? s + (float)static_cast<const T*>(a.router_bias)[e] : s;
    }
    __syncthreads();
    if (threadIdx.x != 0)
        return;
    uint32_t taken = 0;
    int pick[kMoeMaxTop];
    for (int k = 0; k < a.l.top_k; ++k) {
        int best = -1;
        for (int e = 0; e < a.E; ++e)
            if (!((taken >> e) & 1) && (best < 0 || logit_key(lg[e]) > logit_key(lg[best])))
                best = e;
        taken |= 1u << best;
        pick[k] = best;
    }
    const float top = lg[pick[0]];
    float sum = 0.0f;
    for (int e = 0; e < a.E; ++e)
        if (!(a.l.flags & MP_MOE_RENORM) || ((taken >> e) & 1))
            sum += expf(lg[e] - top);
    for (int k = 0; k < a.l.top_k; ++k) {
        const float g = top == -INFINITY ? 0.0f : expf(lg[pick[k]] - top) / sum;
        ids[t * a.l.top_k + k] = pick[k];
        gates[t * a.l.top_k + k] = g;
        if (a.ids)
            a.ids[t * a.l.top_k + k] = pick[k];
        if (a.gates)
            a.gates[t * a.l.top_k + k] = g;
    }
}

// h[slot][f]: one wave per (slot, f).
template <typename T>
__global__ __launch_bounds__(256) void k_up(MoeArgs a, ExpertPtrs ex, const int32_t* ids, const float* gates, float* h)
{
    const int slot = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t f = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), D = a.l.hidden;
    if (f >= a.l.ffn || gates[slot] == 0.0f)
        return;
    const T* x = static_cast<const T*>(a.x) + slot / a.l.top_k * a.ldx;
    const T* w = static_cast<const T*>(ex.p[ids[slot]]);
    float g = 0.0f, u = 0.0f;
    for (int64_t d = lane; d < D; d += 64) {
        g = fmaf((float)x[d], (float)w[a.l.gate_off + f * D + d], g);
        if (a.l.up_off >= 0)
            u = fmaf((float)x[d], (float)w[a.l.up_off + f * D + d], u);
    }
    g = act_of(a.l.act, wave_xor_sum(g));
    if (a.l.up_off >= 0)
        g *= wave_xor_sum(u);
    if (lane == 0)
        h[(int64_t)slot * a.l.ffn + f] = g;
}

// y[t][d]: one wave per (t, d).
template <typename T>
__global__ __launch_bounds__(256) void k_down(MoeArgs a, ExpertPtrs ex, const int32_t* ids, const float* gates,
                                              const float* h)
{
    const int t = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t d = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), F = a.l.ffn;
    if (d >= a.l.hidden)
        return;
    float y = 0.0f;
    for (int k = 0; k < a.l.top_k; ++k) {
        const int slot = t * a.l.top_k + k;
        const float g = gates[slot];
        if (g == 0.0f)
            continue;
        const T* w = static_cast<const T*>(ex.p[ids[slot]]) + a.l.down_off + d * F;
        float s = 0.0f;
        for (int64_t f = lane; f < F; f += 64)
            s = fmaf((float)w[f], h[(int64_t)slot * F + f], s);
        y = fmaf(g, wave_xor_sum(s), y);
    }
    if (lane == 0) {
        if (a.residual)
            y += (float)static_cast<const T*>(a.residual)[t * a.ldr + d];
        static_cast<T*>(a.y)[t * a.ldy + d] = (T)y;
    }
}

template <typename T>
hipError_t moe_t(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    const int slots = a.T * a.l.top_k;
    int32_t* ids = static_cast<int32_t*>(ws);
    float* gates = reinterpret_cast<float*>(ids + kMoeMaxTokens * kMoeMaxTop);
    float* h = gates + kMoeMaxTokens * kMoeMaxTop;
    hipLaunchKernelGGL(k_route<T>, dim3(a.T), dim3(256), 0, st, a, ids, gates);
    hipLaunchKernelGGL(k_up<T>, dim3((unsigned)((a.l.ffn + 3) / 4), slots), dim3(256), 0, st, a, ex, ids, gates, h);
    hipLaunchKernelGGL(k_down<T>, dim3((unsigned)((a.l.hidden + 3) / 4), a.T), dim3(256), 0, st, a, ex, ids, gates, h);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_moe(const MoeArgs& a, const ExpertPtrs& ex, void* ws, hipStream_t st)
{
    return a.l.dtype == MP_F32 ? moe_t<float>(a, ex, ws, st) : moe_t<__bf16>(a, ex, ws, st);
}

uint64_t moe_ws_bytes(const mp_moe_layer& l, int64_t tokens)
{
    return 8ull * kMoeMaxTokens * kMoeMaxTop + 4ull * (uint64_t)tokens * (uint64_t)l.top_k * (uint64_t)l.ffn;
}

}  // namespace mp
