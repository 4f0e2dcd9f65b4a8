// Rotary positions, and new tokens' keys and values into a paged cache.
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

// A thread per pair and per value that is only copied.
template <int DT>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a)
{
    using T = typename Elem<DT>::T;
    const int half = a.rot / 2, items = half + a.dim - a.rot;
    const int64_t all = a.tokens * a.heads * items, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int j = (int)(i % items);
        const int64_t th = i / items, t = th / a.heads, h = th % a.heads;
        const T* x = static_cast<const T*>(a.x) + t * a.ldx + h * a.hdx;
        T* y = static_cast<T*>(a.y) + t * a.ldy + h * a.hdy;
        if (j >= half) {
            y[j + half] = x[j + half];
            continue;
        }
        const float2 w = turn_of(a.pos[t], a.freqs[j], a.amplitude);
        const float s = a.sign * w.y;
        const int p = a.interleaved ? 2 * j : j, q = a.interleaved ? 2 * j + 1 : j + half;
        const float u = (float)x[p], v = (float)x[q];
        y[p] = (T)(u * w.x - v * s);
        y[q] = (T)(u * s + v * w.x);
    }
}

struct Copy {
    const void* v;
    const int64_t* slots;
    int64_t tokens, ldv, pages, page_size, page_stride, slot_stride, head_stride;
    int heads, dim;
    void* out;
};

// Values (or keys that nothing turns) into their slots.
template <int DT>
__global__ __launch_bounds__(256) void k_store(Copy a)
{
    using T = typename Elem<DT>::T;
    const int row = a.heads * a.dim;
    const int64_t all = a.tokens * row, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int64_t t = i / row, slot = a.slots[t];
        const int c = (int)(i % row);
        if (slot < 0 || slot >= a.pages * a.page_size)
            continue;
        static_cast<T*>(a.out)[slot / a.page_size * a.page_stride + slot % a.page_size * a.slot_stride +
                               c / a.dim * a.head_stride + c % a.dim] = static_cast<const T*>(a.v)[t * a.ldv + c];
    }
}

template <int DT>
__global__ __launch_bounds__(256) void k_store_turned(Copy a, RopeArgs r)
{
    using T = typename Elem<DT>::T;
    const int half = r.rot / 2, items = half + a.dim - r.rot;
    const int64_t all = a.tokens * a.heads * items, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int j = (int)(i % items);
        const int64_t th = i / items, t = th / a.heads, h = th % a.heads, slot = a.slots[t];
        if (slot < 0 || slot >= a.pages * a.page_size)
            continue;
        const T* x = static_cast<const T*>(a.v) + t * a.ldv + h * a.dim;
        T* y = static_cast<T*>(a.out) + slot / a.page_size * a.page_stride + slot % a.page_size * a.slot_stride +
               h * a.head_stride;
        if (j >= half) {
            y[j + half] = x[j + half];
            continue;
        }
        const float2 w = turn_of(r.pos[t], r.freqs[j], r.amplitude);
        const int p = r.interleaved ? 2 * j : j, q = r.interleaved ? 2 * j + 1 : j + half;
        const float u = (float)x[p], v = (float)x[q];
        y[p] = (T)(u * w.x - v * w.y);
        y[q] = (T)(u * w.y + v * w.x);
    }
}

unsigned grid(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 65536); }

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t st)
{
    const unsigned g = grid(a.tokens * a.heads * (a.dim - a.rot / 2));
    if (a.dtype == MP_F32)
        k_rope<MP_F32><<<g, 256, 0, st>>>(a);
    else
        k_rope<MP_BF16><<<g, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_append(const mp_kv_cache& c, const mp_kv_rows& r, const void* k, const void* v,
                            const int64_t* slots, const int64_t* pos, const double* freqs, const void* q, void* q_out,
                            hipStream_t st)
{
    Copy a{k,           slots,        r.tokens,      r.ldk,        c.pages,         c.page_size, c.page_stride,
           c.slot_stride, c.head_stride, (int)c.heads, (int)c.head_dim, c.k};
    RopeArgs t{};
    t.dtype = c.dtype;
    t.interleaved = r.flags & MP_ROPE_INTERLEAVED;
    t.tokens = r.tokens;
    t.heads = (int)r.q_heads;
    t.dim = (int)c.head_dim;
    t.rot = (int)r.rot_dim;
    t.x = q;
    t.ldx = r.ldq;
    t.y = q_out;
    t.ldy = r.ldqo;
    t.hdx = t.hdy = c.head_dim;
    t.pos = pos;
    t.freqs = freqs;
    t.amplitude = r.amplitude;
    t.sign = 1.0f;
    const unsigned g = grid(r.tokens * c.heads * c.head_dim);
    const bool f32 = c.dtype == MP_F32;
    if (f32)
        k_store_turned<MP_F32><<<g, 256, 0, st>>>(a, t);
    else
        k_store_turned<MP_BF16><<<g, 256, 0, st>>>(a, t);
    a.v = v;
    a.ldv = r.ldv;
    a.out = c.v;
    if (f32)
        k_store<MP_F32><<<g, 256, 0, st>>>(a);
    else
        k_store<MP_BF16><<<g, 256, 0, st>>>(a);
    if (r.q_heads)
        return launch_rope(t, st);
    return hipGetLastError();
}

}  // namespace mp
