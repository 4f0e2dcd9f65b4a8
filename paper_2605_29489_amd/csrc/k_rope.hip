// Rotary positions, and new tokens' keys and values into a paged cache.
#include <algorithm>

#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

// cos and sin of pos * f, times the amplitude.  The angle is taken in turns and
// in 64 bits, where subtracting the nearest whole turn is exact: what is left,
// at most half a turn, is off by 3 |pos f| 2^-53 / 2 pi.  Its fp32 value h is up
// to 2^-25 half turns away; that rest l is added to first order, sin(h + l) =
// sin h + l cos h and so on, whose next term is under 2^-47.  It costs nothing
// that can be measured; sincospi in 64 bits takes 8192 appended tokens of 32 + 8
// heads from 40 us to 48.
__device__ inline float2 turn_of(int64_t pos, double f, float amp)
{
    double t = (double)pos * (f * 0.15915494309189533577);
    t -= rint(t);
    t += t;
    const float h = (float)t, l = (float)(t - h) * 3.14159265358979f;
    float s, c;
    sincospif(h, &s, &c);
    return make_float2(fmaf(-l, s, c) * amp, fmaf(l, c, s) * amp);
}

// Outputs are written once and are more than the caches hold where it counts:
// rotations of 16384 x 32 x 128 bf16 59.8 us with plain stores and 53.3 with
// non-temporal ones, of 8192 x 40 x 128 39.0 and 28.6.  Non-temporal loads as
// well: 51.1 and 33.3.
__device__ inline void st16n(void* p, uint4 c)
{
    const u32x4_t v = {c.x, c.y, c.z, c.w};
    __builtin_nontemporal_store(v, static_cast<u32x4_a2*>(p));
}

// What one launch turns and copies.  A token's work is a row of items: those of
// its x heads (turned into y), then, with a cache, of its keys (turned) and its
// values (copied).  An item is a 16-byte chunk of a head, or, where pairs lie
// half the turned part apart, two chunks that hold the same pairs; or a single
// pair or value of what the chunks leave of a head (WHOLE: nothing).  A head's
// items are its chunks of pairs, single pairs, chunks of copied values and single
// values, in this order.
struct TurnArgs {
    int64_t tokens;
    int tw;             // tokens of a workgroup
    int dim, rot, per, copy;  // items of a turned head, and of a copied one
    uint32_t nx, nk, all;  // items of a token: x's, and keys', and all
    Div by_all, by_per, by_copy, by_page;
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

constexpr int kThreads = 256;
constexpr int64_t kMaxTurns = 4096;  // cos and sin pairs of a workgroup: 32 KB of LDS

// Bound by memory, and where there are few tokens by one launch and one trip to
// memory: a workgroup's first items, one a thread, are on their way while the
// cos and sin of its tokens, one pair a thread, are formed and shared through LDS
// by all heads.  One item at a time keeps reads and writes close together: with
// 1, 2, 4 and 8 of them 16384 x 32 x 128 bf16 take 47.7, 49.3, 53.5 and 65 us (a
// copy 42), 8192 x 40 x 128 26.9, 28.7, 29.1 and 40 (a copy 28).  With a token's
// items in equal parts, each in a workgroup of its own, 47.0 and 27.5, and appends
// of 8192 tokens with 32 + 8 + 8 heads 47.8 for 41.0.
template <int DT, bool INTER, bool WHOLE, bool APPEND>
__global__ __launch_bounds__(kThreads) void k_turn(TurnArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int V = Fmt<DT>::V;
    extern __shared__ float2 turns[];  // [tw][rot / 2], then the tokens' places in the cache
    const int half = a.rot / 2, tid = threadIdx.x;
    int64_t* place = reinterpret_cast<int64_t*>(turns + a.tw * half);
    // a head's chunks and single pairs, and chunks of its copied values and of a value head
    const int pairs_of = INTER ? V / 2 : V, chunks = half / pairs_of, singles = WHOLE ? 0 : half % pairs_of;
    const int copies = (a.dim - a.rot) / V, values = a.dim / V;
    enum { kX, kKey, kValue };

    for (int64_t t0 = (int64_t)blockIdx.x * a.tw; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.tw) {
        const int nt = (int)(a.tokens - t0 < a.tw ? a.tokens - t0 : a.tw);
        const uint32_t end = (uint32_t)nt * a.all;
        // this thread's item: of token t and head h, from value `off` of the head on; a pair's turns at w
        uint32_t t = 0, h = 0;
        int kind = kX, off = 0, w = 0;
        bool pair = false, chunk = true;
        uint4 lo{}, hi{};
        const auto load = [&](uint32_t at) {
            t = a.by_all.of(at);
            uint32_t r = at - t * a.all;
            int j;
            const T* p;
            if (APPEND && r >= a.nk) {
                r -= a.nk;
                kind = kValue;
                h = a.by_copy.of(r);
                j = (int)(r - h * a.copy);
                p = static_cast<const T*>(a.v) + (t0 + t) * a.ldv + (int64_t)h * a.dim;
                pair = false;
                chunk = WHOLE || j < values;
                off = chunk ? j * V : values * V + j - values;
            } else {
                kind = APPEND && r >= a.nx ? kKey : kX;
                r -= kind == kKey ? a.nx : 0;
                h = a.by_per.of(r);
                j = (int)(r - h * a.per);
                p = kind == kKey ? static_cast<const T*>(a.k) + (t0 + t) * a.ldk + (int64_t)h * a.dim
                                 : static_cast<const T*>(a.x) + (t0 + t) * a.ldx + h * a.hdx;
                pair = j < chunks + singles;
                const int c = j - chunks - singles;
                chunk = WHOLE || (pair ? j < chunks : c < copies);
                w = j < chunks ? j * pairs_of : chunks * pairs_of + j - chunks;
                if (pair)
                    off = INTER ? 2 * w : w;
                else
                    off = a.rot + (chunk ? c * V : copies * V + c - copies);
            }
            p += off;
            if (chunk) {
                lo = ld16u(p);
                if (!INTER && pair)
                    hi = ld16u(p + half);
            } else {
                const auto bits = [](const T* q) -> uint32_t {
                    if constexpr (DT == MP_F32)
                        return *reinterpret_cast<const uint32_t*>(q);
                    else
                        return *reinterpret_cast<const uint16_t*>(q);
                };
                lo.x = bits(p);
                if (pair)
                    hi.x = bits(p + (INTER ? 1 : half));
            }
        };
        if (tid < end)
            load(tid);
        if (t0 != (int64_t)blockIdx.x * a.tw)
            __syncthreads();  // the tokens before are done with the turns
        for (int i = tid; i < nt * half; i += kThreads) {
            const int u = i / half;
            float2 w = turn_of(a.pos[t0 + u], a.freqs[i - u * half], a.amplitude);
            w.y *= a.sign;
            turns[i] = w;
        }
        if constexpr (APPEND)
            for (int u = tid; u < nt; u += kThreads) {
                const int64_t slot = a.slots[t0 + u];
                const bool in = slot >= 0 && slot < a.pages * a.page_size;
                const int64_t page = !in ? 0 : slot >> 31 ? slot / a.page_size : a.by_page.of((uint32_t)slot);
                place[u] = in ? page * a.page_stride + (slot - page * a.page_size) * a.slot_stride : -1;
            }
        __syncthreads();
        const auto store = [&]() {
            T* p;
            if (!APPEND || kind == kX) {
                p = static_cast<T*>(a.y) + (t0 + t) * a.ldy + h * a.hdy;
            } else {
                if (place[t] < 0)
                    return;
                p = static_cast<T*>(kind == kKey ? a.ck : a.cv) + place[t] + h * a.head_stride;
            }
            p += off;
            const float2* c = turns + t * half + w;
            if (chunk) {
                if (pair) {
                    float f[V], y[V];
                    Fmt<DT>::unpack(lo, f);
                    if constexpr (INTER) {
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            y[e] = f[e] * c[e / 2].x - f[e + 1] * c[e / 2].y;
                            y[e + 1] = f[e] * c[e / 2].y + f[e + 1] * c[e / 2].x;
                        }
                    } else {
                        float g[V], z[V];
                        Fmt<DT>::unpack(hi, g);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            y[e] = f[e] * c[e].x - g[e] * c[e].y;
                            z[e] = f[e] * c[e].y + g[e] * c[e].x;
                        }
                        st16n(p + half, Fmt<DT>::pack(z));
                    }
                    lo = Fmt<DT>::pack(y);
                }
                st16n(p, lo);
            } else if (pair) {
                constexpr int up = DT == MP_F32 ? 0 : 16;  // a bf16 pattern is the upper half of an fp32 one
                const float f = __uint_as_float(lo.x << up), g = __uint_as_float(hi.x << up);
                p[0] = (T)(f * c->x - g * c->y);
                p[INTER ? 1 : half] = (T)(f * c->y + g * c->x);
            } else if constexpr (DT == MP_F32) {
                *reinterpret_cast<uint32_t*>(p) = lo.x;
            } else {
                *reinterpret_cast<uint16_t*>(p) = (uint16_t)lo.x;
            }
        };
        for (uint32_t at = tid; at < end;) {
            store();
            at += kThreads;
            if (at < end)
                load(at);
        }
    }
}

template <int DT, bool INTER, bool WHOLE>
void launch_turn(const TurnArgs& a, unsigned grid, size_t lds, bool append, hipStream_t st)
{
    if (append)
        k_turn<DT, INTER, WHOLE, true><<<grid, kThreads, lds, st>>>(a);
    else
        k_turn<DT, INTER, WHOLE, false><<<grid, kThreads, lds, st>>>(a);
}

// heads: turned heads of x; kv: heads of a cache, or 0.
hipError_t launch(TurnArgs& a, int dtype, bool interleaved, int64_t heads, int64_t kv, hipStream_t st)
{
    const int V = dtype == MP_F32 ? 4 : 8, half = a.rot / 2, pairs = interleaved ? V / 2 : V, rest = a.dim - a.rot;
    const bool whole = half % pairs == 0 && rest % V == 0;
    a.copy = a.dim / V + a.dim % V;
    a.per = half / pairs + half % pairs + rest / V + rest % V;
    a.nx = (uint32_t)(heads * a.per);
    a.nk = a.nx + (uint32_t)(kv * a.per);
    a.all = a.nk + (uint32_t)(kv * a.copy);
    a.by_all = Div(a.all);
    a.by_per = Div((uint32_t)a.per);
    a.by_copy = Div((uint32_t)a.copy);
    // as many tokens as there are threads for
    const int64_t tw = std::max<int64_t>(1, std::min<int64_t>(kThreads / a.all, kMaxTurns / std::max(half, 1)));
    a.tw = (int)tw;
    const size_t lds = (size_t)(tw * half) * sizeof(float2) + (size_t)tw * sizeof(int64_t);
    const unsigned grid = (unsigned)std::min<int64_t>((a.tokens + tw - 1) / tw, 1 << 20);
    const bool f32 = dtype == MP_F32, append = kv > 0;
    if (f32 && interleaved)
        whole ? launch_turn<MP_F32, true, true>(a, grid, lds, append, st)
              : launch_turn<MP_F32, true, false>(a, grid, lds, append, st);
    else if (f32)
        whole ? launch_turn<MP_F32, false, true>(a, grid, lds, append, st)
              : launch_turn<MP_F32, false, false>(a, grid, lds, append, st);
    else if (interleaved)
        whole ? launch_turn<MP_BF16, true, true>(a, grid, lds, append, st)
              : launch_turn<MP_BF16, true, false>(a, grid, lds, append, st);
    else
        whole ? launch_turn<MP_BF16, false, true>(a, grid, lds, append, st)
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
    a.by_page = Div((uint32_t)c.page_size);
    a.page_stride = c.page_stride;
    a.slot_stride = c.slot_stride;
    a.head_stride = c.head_stride;
    a.ck = c.k;
    a.cv = c.v;
    return launch(a, c.dtype, r.flags & MP_ROPE_INTERLEAVED, r.q_heads, c.heads, st);
}

}  // namespace mp
