// Rotary positions, and new tokens' keys and values into a paged cache.
#include <algorithm>

#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

// cos and sin of pos * f, times the amplitude.  The angle is taken in turns and
// in 64 bits, where subtracting the nearest whole turn is exact: what is left,
// at most half a turn, is off by pos f 2^-54 or so and is then rounded to fp32,
// 2^-26 of a turn at most.
__device__ inline float2 turn_of(int64_t pos, double f, float amp)
{
    double t = (double)pos * (f * 0.15915494309189533577);
    t -= rint(t);
    float s, c;
    sincospif((float)(t + t), &s, &c);
    return make_float2(c * amp, s * amp);
}

// Quotients of n < 2^31 by a divisor the host knows: with 2^(L-1) < d <= 2^L and
// m = ceil(2^(31+L) / d), n m / 2^(31+L) exceeds n / d by less than
// n / 2^31 / d < 1 / d, so that their whole parts agree.
struct Div {
    uint32_t m = 0, shift = 0, d = 1;
    Div(uint32_t by = 1) : d(by)
    {
        uint32_t L = 0;
        while (((uint64_t)1 << L) < by)
            ++L;
        shift = 31 + L;
        m = (uint32_t)((((uint64_t)1 << shift) + by - 1) / by);
    }
    __device__ inline uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

// What one launch turns and copies.  A token's work is a row of items: those of
// its x heads (turned into y), then, with a cache, of its keys (turned) and its
// values (copied).  An item is a 16-byte chunk of a head, or, where pairs lie
// half the turned part apart, two chunks that hold the same pairs; or a single
// pair or value where the chunks do not divide a head.
struct TurnArgs {
    int64_t tokens;
    int tw;             // tokens of a workgroup
    int dim, rot, per;  // items of a turned head
    uint32_t nx, nk, all;  // items of a token: x's, and keys', and all
    Div by_all, by_per, by_copy;
    const int64_t* pos;
    const double* freqs;
    float amplitude, sign;
    const void* x;
    void* y;
    int64_t ldx, hdx, ldy, hdy;
    const void* k;
    const void* v;
    int64_t ldk, ldv;
    const int64_t* slots;
    int64_t pages, page_size, page_stride, slot_stride, head_stride;
    void* ck;
    void* cv;
};

constexpr int kItems = 4;           // of a thread, loaded together
constexpr int64_t kMaxTurns = 4096;  // cos and sin pairs of a workgroup: 32 KB of LDS

// Bound by memory, and where there are few tokens by one launch and one trip to
// memory: a workgroup's first items are on their way while the cos and sin of
// its tokens, one pair a thread, are formed and shared through LDS by all heads.
template <int DT, bool INTER, bool VEC, bool APPEND>
__global__ __launch_bounds__(256) void k_turn(TurnArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int V = VEC ? Fmt<DT>::V : 1;
    extern __shared__ float2 turns[];  // [tw][rot / 2], then the tokens' places in the cache
    const int half = a.rot / 2, tid = threadIdx.x;
    int64_t* place = reinterpret_cast<int64_t*>(turns + a.tw * half);
    const uint32_t turned = (uint32_t)(INTER ? a.rot / (VEC ? V : 2) : half / V);  // turned items of a head

    struct Item {
        uint32_t t, h, j;  // token, head and item of the head; kind: 0 x, 1 key, 2 value, 3 none
        uint32_t kind;
        uint4 lo, hi;
    };
    Item it[kItems];

    for (int64_t t0 = (int64_t)blockIdx.x * a.tw; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.tw) {
        const int nt = (int)(a.tokens - t0 < a.tw ? a.tokens - t0 : a.tw);
        const uint32_t n = (uint32_t)nt * a.all;
        // elements of an item: VEC chunks at [off] (and [off + half]), else single values
        auto offset = [&](const Item& i) -> int {
            if (APPEND && i.kind == 2)
                return (int)i.j * V;
            if constexpr (VEC)
                return INTER || i.j < turned ? (int)i.j * V : (int)(i.j - turned) * V + a.rot;
            else
                return i.j >= turned ? (int)(i.j - turned) + a.rot : INTER ? 2 * (int)i.j : (int)i.j;
        };
        auto load = [&](uint32_t base) {
#pragma unroll
            for (int u = 0; u < kItems; ++u) {
                Item& i = it[u];
                const uint32_t at = base + u * 256 + tid;
                i.kind = 3;
                if (at >= n)
                    continue;
                i.t = a.by_all.of(at);
                uint32_t r = at - i.t * a.all;
                const T* p;
                if (!APPEND || r < a.nx) {
                    i.kind = 0;
                    i.h = a.by_per.of(r);
                    i.j = r - i.h * a.per;
                    p = static_cast<const T*>(a.x) + (t0 + i.t) * a.ldx + i.h * a.hdx;
                } else if (r < a.nk) {
                    r -= a.nx;
                    i.kind = 1;
                    i.h = a.by_per.of(r);
                    i.j = r - i.h * a.per;
                    p = static_cast<const T*>(a.k) + (t0 + i.t) * a.ldk + (int64_t)i.h * a.dim;
                } else {
                    r -= a.nk;
                    i.kind = 2;
                    i.h = a.by_copy.of(r);
                    i.j = r - i.h * a.by_copy.d;
                    p = static_cast<const T*>(a.v) + (t0 + i.t) * a.ldv + (int64_t)i.h * a.dim;
                }
                p += offset(i);
                const bool pair = i.kind != 2 && i.j < turned;
                if constexpr (VEC) {
                    i.lo = ld16u(p);
                    if (!INTER && pair)
                        i.hi = ld16u(p + half);
                } else {
                    const auto bits = [](const T* q) -> uint32_t {
                        if constexpr (DT == MP_F32)
                            return *reinterpret_cast<const uint32_t*>(q);
                        else
                            return *reinterpret_cast<const uint16_t*>(q);
                    };
                    i.lo.x = bits(p);
                    if (pair)
                        i.hi.x = bits(p + (INTER ? 1 : half));
                }
            }
        };
        load(0);
        if (t0 != (int64_t)blockIdx.x * a.tw)
            __syncthreads();  // the group before is done with the turns
        for (int i = tid; i < nt * half; i += 256) {
            const int t = i / half;
            float2 w = turn_of(a.pos[t0 + t], a.freqs[i - t * half], a.amplitude);
            w.y *= a.sign;
            turns[i] = w;
        }
        if constexpr (APPEND)
            for (int t = tid; t < nt; t += 256) {
                const int64_t slot = a.slots[t0 + t];
                const bool in = slot >= 0 && slot < a.pages * a.page_size;
                const int64_t page = in ? slot / a.page_size : 0;
                place[t] = in ? page * a.page_stride + (slot - page * a.page_size) * a.slot_stride : -1;
            }
        __syncthreads();
        for (uint32_t base = 0;;) {
#pragma unroll
            for (int u = 0; u < kItems; ++u) {
                Item& i = it[u];
                if (i.kind == 3)
                    continue;
                T* p;
                if (!APPEND || i.kind == 0) {
                    p = static_cast<T*>(a.y) + (t0 + i.t) * a.ldy + i.h * a.hdy;
                } else {
                    const int64_t at = place[i.t];
                    if (at < 0)
                        continue;
                    p = static_cast<T*>(i.kind == 1 ? a.ck : a.cv) + at + i.h * a.head_stride;
                }
                p += offset(i);
                const bool pair = i.kind != 2 && i.j < turned;
                const float2* w = turns + i.t * half + (pair ? i.j * (INTER && VEC ? V / 2 : V) : 0);
                if constexpr (VEC) {
                    if (pair) {
                        float f[V];
                        Fmt<DT>::unpack(i.lo, f);
                        if constexpr (INTER) {
                            float y[V];
#pragma unroll
                            for (int e = 0; e < V; e += 2) {
                                const float2 c = w[e / 2];
                                y[e] = f[e] * c.x - f[e + 1] * c.y;
                                y[e + 1] = f[e] * c.y + f[e + 1] * c.x;
                            }
                            i.lo = Fmt<DT>::pack(y);
                        } else {
                            float g[V], y[V], z[V];
                            Fmt<DT>::unpack(i.hi, g);
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const float2 c = w[e];
                                y[e] = f[e] * c.x - g[e] * c.y;
                                z[e] = f[e] * c.y + g[e] * c.x;
                            }
                            i.lo = Fmt<DT>::pack(y);
                            st16u(p + half, Fmt<DT>::pack(z));
                        }
                    }
                    st16u(p, i.lo);
                } else {
                    const auto put = [](T* q, uint32_t b) {
                        if constexpr (DT == MP_F32)
                            *reinterpret_cast<uint32_t*>(q) = b;
                        else
                            *reinterpret_cast<uint16_t*>(q) = (uint16_t)b;
                    };
                    if (pair) {
                        const float2 c = *w;
                        constexpr int up = DT == MP_F32 ? 0 : 16;  // a bf16 pattern is the upper half of an fp32 one
                        const float f = __uint_as_float(i.lo.x << up), g = __uint_as_float(i.hi.x << up);
                        p[0] = (T)(f * c.x - g * c.y);
                        p[INTER ? 1 : half] = (T)(f * c.y + g * c.x);
                    } else {
                        put(p, i.lo.x);
                    }
                }
            }
            base += 256 * kItems;
            if (base >= n)
                break;
            load(base);
        }
    }
}

template <int DT, bool INTER, bool VEC>
void launch_turn(const TurnArgs& a, unsigned grid, size_t lds, bool append, hipStream_t st)
{
    if (append)
        k_turn<DT, INTER, VEC, true><<<grid, 256, lds, st>>>(a);
    else
        k_turn<DT, INTER, VEC, false><<<grid, 256, lds, st>>>(a);
}

// heads: turned heads of x; kv: heads of a cache, or 0.
hipError_t launch(TurnArgs& a, int dtype, bool interleaved, int64_t heads, int64_t kv, hipStream_t st)
{
    const int V = dtype == MP_F32 ? 4 : 8, half = a.rot / 2;
    const bool vec = (interleaved ? a.rot : half) % V == 0 && (a.dim - a.rot) % V == 0;
    const int copy = vec ? a.dim / V : a.dim;
    a.per = vec ? (interleaved ? copy : half / V + (a.dim - a.rot) / V) : half + a.dim - a.rot;
    a.nx = (uint32_t)(heads * a.per);
    a.nk = a.nx + (uint32_t)(kv * a.per);
    a.all = a.nk + (uint32_t)(kv * copy);
    a.by_all = Div(a.all);
    a.by_per = Div((uint32_t)a.per);
    a.by_copy = Div((uint32_t)copy);
    // as many tokens as fill a workgroup's threads with items, fewer where that leaves CUs without a workgroup
    int64_t tw = std::max<int64_t>(1, 256 * kItems / a.all);
    tw = std::min(tw, (a.tokens + 511) / 512);
    tw = std::max<int64_t>(1, std::min(tw, kMaxTurns / std::max(half, 1)));
    a.tw = (int)tw;
    const size_t lds = (size_t)(tw * half) * sizeof(float2) + (size_t)tw * sizeof(int64_t);
    const unsigned grid = (unsigned)std::min<int64_t>((a.tokens + tw - 1) / tw, 1 << 20);
    const bool f32 = dtype == MP_F32, append = kv > 0;
    if (f32 && interleaved)
        vec ? launch_turn<MP_F32, true, true>(a, grid, lds, append, st)
            : launch_turn<MP_F32, true, false>(a, grid, lds, append, st);
    else if (f32)
        vec ? launch_turn<MP_F32, false, true>(a, grid, lds, append, st)
            : launch_turn<MP_F32, false, false>(a, grid, lds, append, st);
    else if (interleaved)
        vec ? launch_turn<MP_BF16, true, true>(a, grid, lds, append, st)
            : launch_turn<MP_BF16, true, false>(a, grid, lds, append, st);
    else
        vec ? launch_turn<MP_BF16, false, true>(a, grid, lds, append, st)
            : launch_turn<MP_BF16, false, false>(a, grid, lds, append, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& r, hipStream_t st)
{
    TurnArgs a{};
    a.tokens = r.tokens;
    a.dim = r.dim;
    a.rot = r.rot;
    a.pos = r.pos;
    a.freqs = r.freqs;
    a.amplitude = r.amplitude;
    a.sign = r.sign;
    a.x = r.x;
    a.y = r.y;
    a.ldx = r.ldx;
    a.hdx = r.hdx;
    a.ldy = r.ldy;
    a.hdy = r.hdy;
    return launch(a, r.dtype, r.interleaved, r.heads, 0, st);
}

hipError_t launch_kv_append(const mp_kv_cache& c, const mp_kv_rows& r, const void* k, const void* v,
                            const int64_t* slots, const int64_t* pos, const double* freqs, const void* q, void* q_out,
                            hipStream_t st)
{
    TurnArgs a{};
    a.tokens = r.tokens;
    a.dim = (int)c.head_dim;
    a.rot = (int)r.rot_dim;
    a.pos = pos;
    a.freqs = freqs;
    a.amplitude = r.amplitude;
    a.sign = 1.0f;
    a.x = q;
    a.y = q_out;
    a.ldx = r.ldq;
    a.ldy = r.ldqo;
    a.hdx = a.hdy = c.head_dim;
    a.k = k;
    a.v = v;
    a.ldk = r.ldk;
    a.ldv = r.ldv;
    a.slots = slots;
    a.pages = c.pages;
    a.page_size = c.page_size;
    a.page_stride = c.page_stride;
    a.slot_stride = c.slot_stride;
    a.head_stride = c.head_stride;
    a.ck = c.k;
    a.cv = c.v;
    return launch(a, c.dtype, r.flags & MP_ROPE_INTERLEAVED, r.q_heads, c.heads, st);
}

}  // namespace mp
