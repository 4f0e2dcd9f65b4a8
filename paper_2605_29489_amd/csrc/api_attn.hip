// The entry points of attention over a paged cache: argument checks, dispatch
// and the rotary frequencies.  They keep no state, so they take no lock.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_check.h"

namespace mp {
namespace {

constexpr double kPi = 3.14159265358979323846;
constexpr int64_t kMaxHeads = 65536, kMaxCacheHeads = 4096, kMaxCacheStride = (int64_t)1 << 24;

// A buffer of `rows` rows of `cols` elements, ld apart, in bytes: packed
// projections hold queries, keys and values side by side in one row, so two
// buffers may interleave without sharing an element.
struct Rows {
    Span s;
    size_t width = 0, pitch = 0;  // bytes; pitch 0: a single row
};

// Whether two buffers' rows, equally far apart, pass between each other.
bool interleaved(const Rows& a, const Rows& b)
{
    if (a.pitch == 0 || a.pitch != b.pitch)
        return false;
    const int64_t pitch = (int64_t)a.pitch;
    const int64_t d = (((int64_t)(b.s.p - a.s.p)) % pitch + pitch) % pitch;
    return (size_t)d >= a.width && (size_t)d + b.width <= a.pitch;
}

int check_apart(const Rows& out, const Rows& in, bool same)
{
    if (same && out.s.p == in.s.p && out.pitch == in.pitch && out.width == in.width)
        return MP_OK;
    if (meet(out.s, in.s) && !interleaved(out, in))
        return fail(MP_E_ARG, "%s overlaps %s", out.s.name, in.s.name);
    return MP_OK;
}

int check_rows(Seen& seen, const void* p, int64_t rows, int64_t cols, int64_t ld, int es, const char* name, Rows* out)
{
    out->width = (size_t)cols * (size_t)es;
    out->pitch = rows > 1 ? (size_t)ld * (size_t)es : 0;
    return check_matrix(seen, p, rows, cols, ld, es, name, &out->s);
}

// Device int32, int64, float or double values.
int check_values(Seen& seen, const void* p, int64_t n, int size, const char* name, Rows* out)
{
    return check_rows(seen, p, 1, n, n, size, name, out);
}

// Extents and strides (elements) of an array of heads, from the innermost on;
// those of one place only are left out.
struct Nest {
    int64_t n[3], stride[3];
    int k = 0;
};

Nest nest(const int64_t* n, const int64_t* stride, int count)
{
    Nest r;
    for (int i = 0; i < count; ++i)
        if (n[i] > 1) {
            r.n[r.k] = n[i];
            r.stride[r.k++] = stride[i];
        }
    for (int i = 1; i < r.k; ++i)
        for (int j = i; j > 0 && r.stride[j] < r.stride[j - 1]; --j) {
            std::swap(r.stride[j], r.stride[j - 1]);
            std::swap(r.n[j], r.n[j - 1]);
        }
    return r;
}

// Whether heads of dim elements meet where one array starts d elements behind
// the other: some difference of two places is less than dim from d.
bool places_meet(const Nest& r, int k, __int128 d, int64_t dim)
{
    if (k == 0)
        return d > -dim && d < dim;
    // the strides inside this one, and a head, reach less far than it, so that
    // only the two multiples beside d can come near it
    const __int128 st = r.stride[k - 1], most = r.n[k - 1] - 1;
    __int128 q = d / st;
    for (__int128 m = q - 1; m <= q + 1; ++m)
        if (m >= -most && m <= most && places_meet(r, k - 1, d - m * st, dim))
            return true;
    return false;
}

// ---------------------------------------------------------------- rotary positions
int check_turn(int64_t dim, int64_t rot, int32_t flags, float amplitude)
{
    if (rot < 0 || rot > dim || rot % 2 != 0)
        return fail(MP_E_ARG, "rot_dim = %lld must be even and in [0, %lld]", (long long)rot, (long long)dim);
    if (flags & ~(int32_t)MP_ROPE_INTERLEAVED)
        return fail(MP_E_ARG, "flags %d: unknown bits", flags);
    if (!std::isfinite(amplitude))
        return fail(MP_E_ARG, "amplitude must be finite");
    return MP_OK;
}

// Strides of tokens x heads x dim, one of them outside the other.
int check_strides(const mp_rope_shape& s, int64_t ld, int64_t hd, const char* which)
{
    const bool one_t = s.tokens <= 1, one_h = s.heads <= 1;
    if ((!one_t && (ld < 1 || ld > kMaxLd)) || (!one_h && (hd < 1 || hd > kMaxLd)))
        return fail(MP_E_ARG, "ld%s or hd%s is not in [1, 2^40]", which, which);
    const bool heads_in = (one_h || hd >= s.head_dim) &&
                          (one_t || (one_h ? ld >= s.head_dim : ld >= (s.heads - 1) * hd + s.head_dim));
    const unsigned __int128 run = one_t ? 0 : (unsigned __int128)(s.tokens - 1) * (uint64_t)ld;
    const bool tokens_in = (one_t || ld >= s.head_dim) &&
                           (one_h || (unsigned __int128)(uint64_t)hd >= run + (uint64_t)s.head_dim);
    if (!heads_in && !tokens_in)
        return fail(MP_E_ARG, "ld%s = %lld, hd%s = %lld: heads share memory", which, (long long)ld, which,
                    (long long)hd);
    return MP_OK;
}

int check_rope_shape(const mp_rope_shape* s, int* es)
{
    if (s == nullptr)
        return fail(MP_E_ARG, "shape is NULL");
    int rc;
    if ((rc = check_dtype(s->dtype, es)) || (rc = check_size(s->tokens, 0, kMaxRows, "tokens")) ||
        (rc = check_size(s->heads, 0, kMaxHeads, "heads")) || (rc = check_size(s->head_dim, 1, 4096, "head_dim")) ||
        (rc = check_turn(s->head_dim, s->rot_dim, s->flags, s->amplitude)))
        return rc;
    if (s->tokens == 0 || s->heads == 0)
        return MP_OK;
    if ((rc = check_strides(*s, s->ldx, s->hdx, "x")) || (rc = check_strides(*s, s->ldy, s->hdy, "y")))
        return rc;
    return MP_OK;
}

// Tokens of heads as rows, whichever stride is the outer one.
int check_heads(Seen& seen, const void* p, const mp_rope_shape& s, int64_t ld, int64_t hd, int es, const char* name,
                Rows* out)
{
    ld = s.tokens > 1 ? ld : 0;
    hd = s.heads > 1 ? hd : 0;
    const bool outer_t = ld >= hd;
    const int64_t rows = outer_t ? s.tokens : s.heads, in = outer_t ? s.heads : s.tokens;
    // an inner extent is less than the outer stride, unless there is one row only
    const size_t inner = span_bytes(in, s.head_dim, outer_t ? hd : ld, 1);
    if (inner > (size_t)1 << 50)
        return fail(MP_E_ARG, "%s: allocation too small", name);
    return check_rows(seen, p, rows, (int64_t)inner, outer_t ? ld : hd, es, name, out);
}

// Whether heads of a tensor share memory with those of one that starts d elements behind it.
bool heads_meet(const mp_rope_shape& s, int64_t ld, int64_t hd, int64_t d)
{
    const int64_t n[2] = {s.tokens, s.heads}, st[2] = {ld, hd};
    const Nest r = nest(n, st, 2);
    return places_meet(r, r.k, d, s.head_dim);
}

int rope(const mp_rope_shape* shape, const void* in, const int64_t* positions, const double* freqs, void* out,
         bool back, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_rope_shape(shape, &es)))
        return rc;
    const mp_rope_shape& s = *shape;
    if (s.tokens == 0 || s.heads == 0)
        return MP_OK;
    RopeArgs a{};
    a.dtype = s.dtype;
    a.interleaved = s.flags & MP_ROPE_INTERLEAVED;
    a.tokens = s.tokens;
    a.heads = (int)s.heads;
    a.dim = (int)s.head_dim;
    a.rot = (int)s.rot_dim;
    a.x = in;
    a.ldx = s.tokens > 1 ? (back ? s.ldy : s.ldx) : 0;
    a.hdx = s.heads > 1 ? (back ? s.hdy : s.hdx) : 0;
    a.y = out;
    a.ldy = s.tokens > 1 ? (back ? s.ldx : s.ldy) : 0;
    a.hdy = s.heads > 1 ? (back ? s.hdx : s.hdy) : 0;
    a.pos = s.rot_dim ? positions : nullptr;
    a.freqs = s.rot_dim ? freqs : nullptr;
    a.amplitude = s.amplitude;
    a.sign = back ? -1.0f : 1.0f;
    Seen seen;
    Rows X, Y, P, F;
    if ((rc = check_heads(seen, in, s, a.ldx, a.hdx, es, back ? "dy" : "x", &X)) ||
        (rc = check_heads(seen, out, s, a.ldy, a.hdy, es, back ? "dx" : "y", &Y)) ||
        (s.rot_dim && (rc = check_values(seen, positions, s.tokens, 8, "positions", &P))) ||
        (s.rot_dim && (rc = check_values(seen, freqs, s.rot_dim / 2, 8, "freqs", &F))))
        return rc;
    // where the strides are equal, heads of one may lie between those of the other
    const bool alike = a.ldx == a.ldy && a.hdx == a.hdy;
    const bool between = alike && X.s.p != Y.s.p && meet(Y.s, X.s) &&
                         !heads_meet(s, a.ldx, a.hdx, (Y.s.p - X.s.p) / es);
    if (!between && (rc = check_apart(Y, X, alike)))
        return rc;
    if ((rc = check_apart(Y, P, false)) || (rc = check_apart(Y, F, false)))
        return rc;
    const hipError_t e = launch_rope(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "rope launch");
}

// ---------------------------------------------------------------- the cache
Nest nest(const mp_kv_cache& c)
{
    const int64_t n[3] = {c.pages, c.page_size, c.heads}, st[3] = {c.page_stride, c.slot_stride, c.head_stride};
    return nest(n, st, 3);
}

int check_cache(const mp_kv_cache* c, int* es)
{
    if (c == nullptr)
        return fail(MP_E_ARG, "cache is NULL");
    int rc;
    if ((rc = check_dtype(c->dtype, es)))
        return rc;
    if (c->flags != 0)
        return fail(MP_E_ARG, "flags %d: unknown bits", c->flags);
    if ((rc = check_size(c->pages, 0, (int64_t)1 << 40, "pages")) ||
        (rc = check_size(c->page_size, 1, (int64_t)1 << 30, "page_size")) ||
        (rc = check_size(c->heads, 1, kMaxCacheHeads, "heads")) ||
        (rc = check_size(c->head_dim, 1, (int64_t)1 << 20, "head_dim")))
        return rc;
    if (c->head_dim > 256)
        return fail(MP_E_UNSUPPORTED, "head_dim = %lld: at most 256 is taken", (long long)c->head_dim);
    if ((unsigned __int128)c->pages * (uint64_t)c->page_size > (unsigned __int128)1 << 40)
        return fail(MP_E_ARG, "pages * page_size exceeds 2^40");
    if ((c->pages > 1 && (rc = check_size(c->page_stride, 1, kMaxLd, "page_stride"))) ||
        (c->page_size > 1 && (rc = check_size(c->slot_stride, 1, kMaxCacheStride, "slot_stride"))) ||
        (c->heads > 1 && (rc = check_size(c->head_stride, 1, (int64_t)1 << 38, "head_stride"))))
        return rc;
    const Nest r = nest(*c);
    __int128 reach = c->head_dim;  // elements of what lies inside the next stride
    for (int i = 0; i < r.k; ++i) {
        if (r.stride[i] < reach)
            return fail(MP_E_ARG, "the cache's strides let heads share memory");
        reach += (__int128)(r.n[i] - 1) * r.stride[i];
    }
    return MP_OK;
}

// The buffers of a cache that has pages.
int check_cache_buffers(Seen& seen, const mp_kv_cache& c, int es, Rows* K, Rows* V)
{
    const Nest r = nest(c);
    unsigned __int128 reach = (uint64_t)c.head_dim;
    for (int i = 0; i < r.k; ++i)
        reach += (unsigned __int128)(r.n[i] - 1) * (uint64_t)r.stride[i];
    const int64_t n = c.pages == 0 ? 0 : reach >> 58 ? (int64_t)1 << 58 : (int64_t)reach;
    int rc;
    if ((rc = check_rows(seen, c.k, 1, n, n, es, "the cache's k", K)) ||
        (rc = check_rows(seen, c.v, 1, n, n, es, "the cache's v", V)))
        return rc;
    if (meet(K->s, V->s)) {
        const int64_t d = V->s.p - K->s.p;
        if (d % es != 0 || places_meet(r, r.k, d / es, c.head_dim))
            return fail(MP_E_ARG, "the cache's k and v share memory");
    }
    return MP_OK;
}

int check_attend(const mp_kv_cache* c, const mp_kv_attend_shape* s, int* es)
{
    int rc;
    if ((rc = check_cache(c, es)))
        return rc;
    if (s == nullptr)
        return fail(MP_E_ARG, "shape is NULL");
    if ((rc = check_size(s->rows, 0, (int64_t)1 << 20, "rows")) ||
        (rc = check_size(s->q_heads, 1, (int64_t)1 << 23, "q_heads")) ||
        (rc = check_size(s->width, 0, kMaxRows, "width")) ||
        (rc = check_size(s->window, 0, (int64_t)1 << 40, "window")))
        return rc;
    if (s->q_heads % c->heads != 0)
        return fail(MP_E_ARG, "q_heads = %lld is not a multiple of the cache's %lld heads", (long long)s->q_heads,
                    (long long)c->heads);
    if (s->rows * s->q_heads > (int64_t)1 << 23)
        return fail(MP_E_ARG, "rows * q_heads exceeds 2^23");
    if (s->width * c->page_size > (int64_t)1 << 29)  // <= 2^61
        return fail(MP_E_ARG, "width * page_size exceeds 2^29");
    return MP_OK;
}

}  // namespace
}  // namespace mp

using namespace mp;

extern "C" {

int mp_rope(const mp_rope_shape* shape, const void* x, const int64_t* positions, const double* freqs, void* y,
            void* stream)
{
    return rope(shape, x, positions, freqs, y, false, stream);
}

int mp_rope_backward(const mp_rope_shape* shape, const void* dy, const int64_t* positions, const double* freqs,
                     void* dx, void* stream)
{
    return rope(shape, dy, positions, freqs, dx, true, stream);
}

int mp_rope_frequencies(const mp_rope_scaling* scaling, int64_t rot_dim, double* freqs, float* amplitude)
{
    clear_error();
    if (scaling == nullptr || (freqs == nullptr && rot_dim > 0))
        return fail(MP_E_ARG, "scaling or freqs is NULL");
    const mp_rope_scaling& s = *scaling;
    if (s.kind < MP_ROPE_PLAIN || s.kind > MP_ROPE_YARN)
        return fail(MP_E_ARG, "kind %d is not an mp_rope_kind", s.kind);
    if (rot_dim < 0 || rot_dim > 4096 || rot_dim % 2 != 0)
        return fail(MP_E_ARG, "rot_dim = %lld must be even and in [0, 4096]", (long long)rot_dim);
    if (!(s.base > 1.0) || !std::isfinite(s.base))
        return fail(MP_E_ARG, "base must be finite and over 1");
    if (s.kind != MP_ROPE_PLAIN && (!(s.factor >= 1.0) || !std::isfinite(s.factor)))
        return fail(MP_E_ARG, "factor must be finite and at least 1");
    const bool ramp = s.kind == MP_ROPE_PARTS || s.kind == MP_ROPE_YARN;
    if (ramp && (!(s.original > 0.0) || !std::isfinite(s.original) || !(s.low > 0.0) || !(s.high > s.low) ||
                 !std::isfinite(s.high)))
        return fail(MP_E_ARG, "original must be over 0, and 0 < low < high, all finite");
    const int64_t half = rot_dim / 2;
    const double R = (double)rot_dim;
    double base = s.base, lo = 0.0, hi = 0.0;
    if (s.kind == MP_ROPE_NTK && rot_dim > 2)  // a single pair turns by 1 whatever the base
        base *= std::pow(s.factor, R / (R - 2.0));
    if (s.kind == MP_ROPE_YARN) {
        // base^(-2 i / R) original / (2 pi) = r at i = R ln(original / (2 pi r)) / (2 ln base)
        const auto pair = [&](double r) { return R * std::log(s.original / (2.0 * kPi * r)) / (2.0 * std::log(base)); };
        lo = std::max(std::floor(pair(s.high)), 0.0);
        hi = std::min(std::ceil(pair(s.low)), R - 1.0);
    }
    for (int64_t i = 0; i < half; ++i) {
        const double f = std::pow(base, -2.0 * (double)i / R);
        if (s.kind == MP_ROPE_LINEAR) {
            freqs[i] = f / s.factor;
        } else if (s.kind == MP_ROPE_PARTS) {
            const double k = std::clamp((s.original * f / (2.0 * kPi) - s.low) / (s.high - s.low), 0.0, 1.0);
            freqs[i] = f * k + f / s.factor * (1.0 - k);
        } else if (s.kind == MP_ROPE_YARN) {
            const double k = std::clamp(((double)i - lo) / std::max(hi - lo, 1e-3), 0.0, 1.0);
            freqs[i] = f * (1.0 - k) + f / s.factor * k;
        } else {
            freqs[i] = f;
        }
    }
    if (amplitude != nullptr)
        *amplitude = s.kind == MP_ROPE_YARN ? (float)(0.1 * std::log(s.factor) + 1.0) : 1.0f;
    return MP_OK;
}

int mp_kv_append(const mp_kv_cache* cache, const mp_kv_rows* rows, const void* k, const void* v,
                 const int64_t* slots, const int64_t* positions, const double* freqs, const void* q, void* q_out,
                 void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_cache(cache, &es)))
        return rc;
    if (rows == nullptr)
        return fail(MP_E_ARG, "rows is NULL");
    const mp_kv_cache& c = *cache;
    mp_kv_rows r = *rows;
    if (q == nullptr)
        r.q_heads = 0;
    if ((rc = check_size(r.tokens, 0, kMaxRows, "tokens")) || (rc = check_size(r.q_heads, 0, kMaxHeads, "q_heads")) ||
        (rc = check_turn(c.head_dim, r.rot_dim, r.flags, r.amplitude)))
        return rc;
    const int64_t kw = c.heads * c.head_dim, qw = r.q_heads * c.head_dim;
    if ((rc = check_ld(r.ldk, kw, "ldk")) || (rc = check_ld(r.ldv, kw, "ldv")) ||
        (qw && ((rc = check_ld(r.ldq, qw, "ldq")) || (rc = check_ld(r.ldqo, qw, "ldqo")))))
        return rc;
    if (r.tokens == 0)
        return MP_OK;
    Seen seen;
    Rows CK, CV, K, V, Q, QO, S, P, F;
    if ((rc = check_cache_buffers(seen, c, es, &CK, &CV)) ||
        (rc = check_rows(seen, k, r.tokens, kw, r.ldk, es, "k", &K)) ||
        (rc = check_rows(seen, v, r.tokens, kw, r.ldv, es, "v", &V)) ||
        (rc = check_values(seen, slots, r.tokens, 8, "slots", &S)) ||
        (r.rot_dim && (rc = check_values(seen, positions, r.tokens, 8, "positions", &P))) ||
        (r.rot_dim && (rc = check_values(seen, freqs, r.rot_dim / 2, 8, "freqs", &F))) ||
        (qw && (rc = check_rows(seen, q, r.tokens, qw, r.ldq, es, "q", &Q))) ||
        (qw && (rc = check_rows(seen, q_out, r.tokens, qw, r.ldqo, es, "q_out", &QO))))
        return rc;
    for (const Rows* i : {&K, &V, &Q, &QO, &S, &P, &F})
        if ((rc = check_apart(CK, *i, false)) || (rc = check_apart(CV, *i, false)))
            return rc;
    if ((rc = check_apart(QO, Q, true)))
        return rc;
    for (const Rows* i : {&K, &V, &S, &P, &F})
        if ((rc = check_apart(QO, *i, false)))
            return rc;
    const hipError_t e =
        launch_kv_append(c, r, k, v, slots, positions, freqs, q, q_out, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "kv append launch");
}

int mp_kv_attend_workspace(const mp_kv_cache* cache, const mp_kv_attend_shape* shape, uint64_t* bytes)
{
    clear_error();
    int es, rc;
    if ((rc = check_attend(cache, shape, &es)))
        return rc;
    if (bytes == nullptr)
        return fail(MP_E_ARG, "bytes is NULL");
    *bytes = kv_attend_ws_bytes(*cache, *shape);
    return MP_OK;
}

int mp_kv_attend(const mp_kv_cache* cache, const mp_kv_attend_shape* shape, const void* q, const int32_t* table,
                 const int32_t* lens, void* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_attend(cache, shape, &es)))
        return rc;
    const mp_kv_cache& c = *cache;
    const mp_kv_attend_shape& s = *shape;
    const int64_t qw = s.q_heads * c.head_dim;
    if ((rc = check_ld(s.ldq, qw, "ldq")) || (rc = check_ld(s.ldo, qw, "ldo")) ||
        (s.ldt != 0 && (rc = check_ld(s.ldt, s.width, "ldt"))))
        return rc;
    if (!(std::fabs(s.scale) <= 1e30f))
        return fail(MP_E_ARG, "scale must be in [-1e30, 1e30]");
    if (s.rows == 0)
        return MP_OK;
    Seen seen;
    Rows CK, CV, Q, O, T, L, E, W;
    if ((rc = check_workspace(seen, workspace, workspace_bytes, kv_attend_ws_bytes(c, s), &W.s)) ||
        (rc = check_cache_buffers(seen, c, es, &CK, &CV)) ||
        (rc = check_rows(seen, q, s.rows, qw, s.ldq, es, "q", &Q)) ||
        (rc = check_rows(seen, out, s.rows, qw, s.ldo, es, "out", &O)) ||
        (rc = check_rows(seen, table, s.ldt ? s.rows : 1, s.width, s.ldt ? s.ldt : s.width, 4, "table", &T)) ||
        (rc = check_values(seen, lens, s.rows, 4, "lens", &L)) ||
        (lse && (rc = check_values(seen, lse, s.rows * s.q_heads, 4, "lse", &E))))
        return rc;
    if ((rc = check_apart(O, Q, true)))
        return rc;
    for (const Rows* i : {&CK, &CV, &T, &L, &E})
        if ((rc = check_apart(O, *i, false)))
            return rc;
    for (const Rows* i : {&CK, &CV, &Q, &T, &L})
        if ((rc = check_apart(E, *i, false)))
            return rc;
    for (const Rows* i : {&CK, &CV, &Q, &O, &T, &L, &E})
        if ((rc = check_apart(W, *i, false)))
            return rc;
    const hipError_t e =
        launch_kv_attend(c, s, q, table, lens, out, lse, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "kv attend launch");
}

}  // extern "C"
