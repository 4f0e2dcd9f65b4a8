// Attention of one new token per row over a paged cache of keys and values.
#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

struct AttendArgs {
    const void* k;
    const void* v;
    const void* q;
    const int32_t* table;
    const int32_t* lens;
    void* out;
    float* lse;  // or null
    int64_t pages, page_stride, slot_stride, head_stride, ldq, ldo, ldt;
    int64_t most;    // keys that a table row has room for
    int64_t window;  // keys, INT64_MAX: all
    int page_size, heads, group, dim;
    float scale;
};

// A wave per row and query head, a key at a time; lane l holds the values l,
// l + 64, ... of the head.
template <int DT>
__global__ __launch_bounds__(64) void k_attend(AttendArgs a)
{
    using T = typename Elem<DT>::T;
    const int row = blockIdx.x, head = blockIdx.y, l = threadIdx.x;
    float q[4], o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const T* qp = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)head * a.dim;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q[i] = l + 64 * i < a.dim ? (float)qp[l + 64 * i] : 0.0f;
    const int64_t n = a.lens[row] < 0 ? 0 : a.lens[row] < a.most ? a.lens[row] : a.most;
    float m = -INFINITY, sum = 0.0f;
    for (int64_t j = n > a.window ? n - a.window : 0; j < n; ++j) {
        const int64_t page = a.table[row * a.ldt + j / a.page_size];
        if (page < 0 || page >= a.pages)
            continue;
        const int64_t at = page * a.page_stride + j % a.page_size * a.slot_stride + head / a.group * a.head_stride;
        const T* k = static_cast<const T*>(a.k) + at;
        const T* v = static_cast<const T*>(a.v) + at;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (l + 64 * i < a.dim)
                s += q[i] * (float)k[l + 64 * i];
        s = wave_xor_sum(s) * a.scale;
        const float top = fmaxf(m, s);
        const float base = top == -INFINITY ? 0.0f : top;
        const float p = s != s ? s : expf(s - base), keep = expf(m - base);
        m = top;
        sum = sum * keep + p;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (l + 64 * i < a.dim)
                o[i] = o[i] * keep + p * (float)v[l + 64 * i];
    }
    const float r = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* op = static_cast<T*>(a.out) + row * a.ldo + (int64_t)head * a.dim;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (l + 64 * i < a.dim)
            op[l + 64 * i] = (T)(sum == 0.0f ? 0.0f : o[i] * r);
    if (a.lse && l == 0)
        a.lse[(int64_t)row * a.heads * a.group + head] = sum == 0.0f ? -INFINITY : m + logf(sum);
}

}  // namespace

uint64_t kv_attend_ws_bytes(const mp_kv_cache& c, const mp_kv_attend_shape& s) { return 0; }

hipError_t launch_kv_attend(const mp_kv_cache& c, const mp_kv_attend_shape& s, const void* q, const int32_t* table,
                            const int32_t* lens, void* out, float* lse, void* ws, hipStream_t st)
{
    AttendArgs a{c.k,   c.v,   q,     table, lens, out, lse, c.pages, c.page_stride, c.slot_stride, c.head_stride,
                 s.ldq, s.ldo, s.ldt};
    a.most = s.width * c.page_size;
    a.window = s.window ? s.window : INT64_MAX;
    a.page_size = (int)c.page_size;
    a.heads = (int)c.heads;
    a.group = (int)(s.q_heads / c.heads);
    a.dim = (int)c.head_dim;
    a.scale = s.scale;
    const dim3 g((unsigned)s.rows, (unsigned)s.q_heads);
    if (c.dtype == MP_F32)
        k_attend<MP_F32><<<g, 64, 0, st>>>(a);
    else
        k_attend<MP_BF16><<<g, 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace mp
