// The entry points that run a block's feed-forward part: argument checks and
// dispatch.  They keep no state, so they take no lock.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "api_check.h"

namespace mp {
namespace {

int check_linear_shape(const mp_linear_shape* s, int* es)
{
    if (s == nullptr)
        return fail(MP_E_ARG, "shape is NULL");
    int rc;
    if ((rc = check_dtype(s->dtype, es)) || (rc = check_size(s->m, 0, kMaxSize, "m")) ||
        (rc = check_size(s->n, 0, kMaxSize, "n")) || (rc = check_size(s->k, 0, kMaxSize, "k")))
        return rc;
    if (s->act < MP_ACT_NONE || s->act > MP_ACT_SILU)
        return fail(MP_E_ARG, "act %d is not an mp_act", s->act);
    return MP_OK;
}

int check_norm_shape(const mp_norm_shape* s, int* es)
{
    if (s == nullptr)
        return fail(MP_E_ARG, "shape is NULL");
    int rc;
    if ((rc = check_dtype(s->dtype, es)) || (rc = check_size(s->rows, 0, kMaxRows, "rows")) ||
        (rc = check_size(s->cols, 0, kMaxSize, "cols")))
        return rc;
    if (s->flags & ~(int32_t)MP_NORM_RMS)
        return fail(MP_E_ARG, "flags %d: unknown bits", s->flags);
    if (!(s->eps >= 0.0f) || std::isinf(s->eps))
        return fail(MP_E_ARG, "eps must be finite and >= 0");
    return MP_OK;
}

int check_moe_layer(const mp_moe_layer* l, int64_t tokens, int* es)
{
    if (l == nullptr)
        return fail(MP_E_ARG, "layer is NULL");
    int rc;
    if ((rc = check_dtype(l->dtype, es)) || (rc = check_size(l->hidden, 1, kMaxHidden, "hidden")) ||
        (rc = check_size(l->ffn, 1, kMaxHidden, "ffn")) || (rc = check_size(tokens, 0, kMaxRows, "tokens")))
        return rc;
    if (l->act < MP_ACT_NONE || l->act > MP_ACT_SILU)
        return fail(MP_E_ARG, "act %d is not an mp_act", l->act);
    if (l->flags & ~(int32_t)MP_MOE_RENORM)
        return fail(MP_E_ARG, "flags %d: unknown bits", l->flags);
    if (l->top_k < 1 || l->top_k > kMoeMaxTop)
        return fail(MP_E_ARG, "top_k = %d must be in [1, %d]", l->top_k, kMoeMaxTop);
    const int64_t lim = (int64_t)1 << 48;
    if (l->gate_off < 0 || l->gate_off > lim || l->down_off < 0 || l->down_off > lim || l->up_off > lim)
        return fail(MP_E_ARG, "an offset is out of range");
    if (tokens > kMoeMaxTokens)
        return fail(MP_E_UNSUPPORTED, "%lld tokens: at most %d are taken", (long long)tokens, kMoeMaxTokens);
    return MP_OK;
}

}  // namespace
}  // namespace mp

using namespace mp;

extern "C" {

int mp_linear_workspace(const mp_linear_shape* shape, int32_t backward, uint64_t* bytes)
{
    clear_error();
    int es, rc;
    if ((rc = check_linear_shape(shape, &es)))
        return rc;
    if (bytes == nullptr)
        return fail(MP_E_ARG, "bytes is NULL");
    if (backward != 0 && backward != 1)
        return fail(MP_E_ARG, "backward must be 0 or 1");
    *bytes = backward ? linear_backward_ws_bytes(*shape) : linear_ws_bytes(*shape);
    return MP_OK;
}

int mp_linear(const mp_linear_shape* shape, const void* x, const void* w, const void* bias, const void* residual,
              void* y, void* z, void* workspace, uint64_t workspace_bytes, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_linear_shape(shape, &es)))
        return rc;
    const mp_linear_shape& s = *shape;
    Seen seen;
    Span X, W, B, R, Y, Z, S;
    if ((rc = check_ld(s.ldx, s.k, "ldx")) || (rc = check_ld(s.ldw, s.k, "ldw")) || (rc = check_ld(s.ldy, s.n, "ldy")) ||
        (z && (rc = check_ld(s.ldz, s.n, "ldz"))) || (residual && (rc = check_ld(s.ldr, s.n, "ldr"))))
        return rc;
    if (s.m == 0 || s.n == 0)
        return MP_OK;
    if ((rc = check_workspace(seen, workspace, workspace_bytes, linear_ws_bytes(s), &S)) ||
        (rc = check_matrix(seen, x, s.m, s.k, s.ldx, es, "x", &X)) || (rc = check_matrix(seen, w, s.n, s.k, s.ldw, es, "w", &W)) ||
        (rc = check_matrix(seen, y, s.m, s.n, s.ldy, es, "y", &Y)) ||
        (bias && (rc = check_matrix(seen, bias, 1, s.n, s.n, es, "bias", &B))) ||
        (residual && (rc = check_matrix(seen, residual, s.m, s.n, s.ldr, es, "residual", &R))) ||
        (z && (rc = check_matrix(seen, z, s.m, s.n, s.ldz, es, "z", &Z))))
        return rc;
    if ((rc = check_apart(Y, X, false)) || (rc = check_apart(Y, W, false)) || (rc = check_apart(Y, B, false)) ||
        (rc = check_apart(Y, R, true)) || (rc = check_apart(Y, Z, false)) || (rc = check_apart(Z, X, false)) ||
        (rc = check_apart(Z, W, false)) || (rc = check_apart(Z, B, false)) || (rc = check_apart(Z, R, false)))
        return rc;
    for (const Span* o : {&X, &W, &B, &R, &Y, &Z})
        if ((rc = check_apart(S, *o, false)))
            return rc;
    hipError_t e = launch_linear(s, x, w, bias, residual, y, z, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "linear launch");
}

int mp_linear_backward(const mp_linear_shape* shape, const void* dy, const void* x, const void* w, const void* z,
                       void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias, void* workspace,
                       uint64_t workspace_bytes, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_linear_shape(shape, &es)))
        return rc;
    const mp_linear_shape& s = *shape;
    const bool act = s.act != MP_ACT_NONE;
    if ((rc = check_ld(s.ldy, s.n, "ldy")) || (act && (rc = check_ld(s.ldz, s.n, "ldz"))) ||
        (dx && ((rc = check_ld(lddx, s.k, "lddx")) || (rc = check_ld(s.ldw, s.k, "ldw")))) ||
        (dw && ((rc = check_ld(lddw, s.k, "lddw")) || (rc = check_ld(s.ldx, s.k, "ldx")))))
        return rc;
    Seen seen;
    Span DY, X, W, Z, DX, DW, DB, S;
    if ((rc = check_workspace(seen, workspace, workspace_bytes, linear_backward_ws_bytes(s), &S)) ||
        (rc = check_matrix(seen, dy, s.m, s.n, s.ldy, es, "dy", &DY)) ||
        (act && (rc = check_matrix(seen, z, s.m, s.n, s.ldz, es, "z", &Z))) ||
        (dw && (rc = check_matrix(seen, x, s.m, s.k, s.ldx, es, "x", &X))) ||
        (dx && (rc = check_matrix(seen, w, s.n, s.k, s.ldw, es, "w", &W))) ||
        (dx && (rc = check_matrix(seen, dx, s.m, s.k, lddx, es, "dx", &DX))) ||
        (dw && (rc = check_matrix(seen, dw, s.n, s.k, lddw, es, "dw", &DW))) ||
        (dbias && (rc = check_matrix(seen, dbias, 1, s.n, s.n, es, "dbias", &DB))))
        return rc;
    for (const Span* o : {&DX, &DW, &DB, &S})
        for (const Span* i : {&DY, &X, &W, &Z})
            if ((rc = check_apart(*o, *i, false)))
                return rc;
    if ((rc = check_apart(DX, DW, false)) || (rc = check_apart(DX, DB, false)) || (rc = check_apart(DW, DB, false)) ||
        (rc = check_apart(S, DX, false)) || (rc = check_apart(S, DW, false)) || (rc = check_apart(S, DB, false)))
        return rc;
    hipError_t e = launch_linear_backward(s, dy, x, w, z, dx, lddx, dw, lddw, dbias, workspace,
                                          static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "linear backward launch");
}

int mp_norm(const mp_norm_shape* shape, const void* x, const void* weight, const void* bias, void* y, float* mean,
            float* rstd, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_norm_shape(shape, &es)))
        return rc;
    const mp_norm_shape& s = *shape;
    if ((rc = check_ld(s.ldx, s.cols, "ldx")) || (rc = check_ld(s.ldy, s.cols, "ldy")))
        return rc;
    if (s.rows == 0 || s.cols == 0)
        return MP_OK;
    if (s.flags & MP_NORM_RMS)
        mean = nullptr;
    Seen seen;
    Span X, W, B, Y, M, R;
    if ((rc = check_matrix(seen, x, s.rows, s.cols, s.ldx, es, "x", &X)) ||
        (rc = check_matrix(seen, y, s.rows, s.cols, s.ldy, es, "y", &Y)) ||
        (weight && (rc = check_matrix(seen, weight, 1, s.cols, s.cols, es, "weight", &W))) ||
        (bias && (rc = check_matrix(seen, bias, 1, s.cols, s.cols, es, "bias", &B))) ||
        (mean && (rc = check_matrix(seen, mean, 1, s.rows, s.rows, 4, "mean", &M))) ||
        (rstd && (rc = check_matrix(seen, rstd, 1, s.rows, s.rows, 4, "rstd", &R))))
        return rc;
    if ((rc = check_apart(Y, X, true)) || (rc = check_apart(Y, W, false)) || (rc = check_apart(Y, B, false)))
        return rc;
    for (const Span* i : {&X, &W, &B, &Y})
        if ((rc = check_apart(M, *i, false)) || (rc = check_apart(R, *i, false)))
            return rc;
    if ((rc = check_apart(M, R, false)))
        return rc;
    hipError_t e = launch_norm(s, x, weight, bias, y, mean, rstd, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "norm launch");
}

int mp_norm_workspace(const mp_norm_shape* shape, uint64_t* bytes)
{
    clear_error();
    int es, rc;
    if ((rc = check_norm_shape(shape, &es)))
        return rc;
    if (bytes == nullptr)
        return fail(MP_E_ARG, "bytes is NULL");
    *bytes = norm_ws_bytes(*shape);
    return MP_OK;
}

int mp_norm_backward(const mp_norm_shape* shape, const void* dy, const void* x, const void* weight, const float* mean,
                     const float* rstd, void* dx, int64_t lddx, void* dweight, void* dbias, void* workspace,
                     uint64_t workspace_bytes, void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_norm_shape(shape, &es)))
        return rc;
    const mp_norm_shape& s = *shape;
    if ((rc = check_ld(s.ldx, s.cols, "ldx")) || (rc = check_ld(s.ldy, s.cols, "ldy")) ||
        (dx && (rc = check_ld(lddx, s.cols, "lddx"))))
        return rc;
    if (s.cols == 0)
        return MP_OK;
    if (s.flags & MP_NORM_RMS)
        mean = nullptr;
    Seen seen;
    Span DY, X, W, M, R, DX, DW, DB, S;
    if ((rc = check_workspace(seen, workspace, workspace_bytes, norm_ws_bytes(s), &S)) ||
        (rc = check_matrix(seen, dy, s.rows, s.cols, s.ldy, es, "dy", &DY)) ||
        (rc = check_matrix(seen, x, s.rows, s.cols, s.ldx, es, "x", &X)) ||
        (weight && (rc = check_matrix(seen, weight, 1, s.cols, s.cols, es, "weight", &W))) ||
        (!(s.flags & MP_NORM_RMS) && (rc = check_matrix(seen, mean, 1, s.rows, s.rows, 4, "mean", &M))) ||
        (rc = check_matrix(seen, rstd, 1, s.rows, s.rows, 4, "rstd", &R)) ||
        (dx && (rc = check_matrix(seen, dx, s.rows, s.cols, lddx, es, "dx", &DX))) ||
        (dweight && (rc = check_matrix(seen, dweight, 1, s.cols, s.cols, es, "dweight", &DW))) ||
        (dbias && (rc = check_matrix(seen, dbias, 1, s.cols, s.cols, es, "dbias", &DB))))
        return rc;
    for (const Span* o : {&DX, &DW, &DB, &S})
        for (const Span* i : {&DY, &X, &W, &M, &R})
            if ((rc = check_apart(*o, *i, o == &DX && i == &DY)))
                return rc;
    if ((rc = check_apart(DX, DW, false)) || (rc = check_apart(DX, DB, false)) || (rc = check_apart(DW, DB, false)) ||
        (rc = check_apart(S, DX, false)) || (rc = check_apart(S, DW, false)) || (rc = check_apart(S, DB, false)))
        return rc;
    hipError_t e = launch_norm_backward(s, dy, x, weight, mean, rstd, dx, lddx, dweight, dbias, workspace,
                                        static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "norm backward launch");
}

int mp_moe_workspace(const mp_moe_layer* layer, int64_t tokens, uint64_t* bytes)
{
    clear_error();
    int es, rc;
    if ((rc = check_moe_layer(layer, tokens, &es)))
        return rc;
    if (bytes == nullptr)
        return fail(MP_E_ARG, "bytes is NULL");
    *bytes = moe_ws_bytes(*layer, tokens);
    return MP_OK;
}

int mp_moe(const mp_moe_layer* layer, int64_t tokens, const void* x, int64_t ldx, const void* router,
           const void* router_bias, const void* const* experts, int32_t E, int32_t residency, const void* residual,
           int64_t ldr, void* y, int64_t ldy, int32_t* ids, float* gates, void* workspace, uint64_t workspace_bytes,
           void* stream)
{
    clear_error();
    int es, rc;
    if ((rc = check_moe_layer(layer, tokens, &es)))
        return rc;
    const mp_moe_layer& l = *layer;
    if (E < 1 || E > kMaxK)
        return fail(MP_E_ARG, "E = %d must be in [1, 32]", E);
    if (l.top_k > E)
        return fail(MP_E_ARG, "top_k = %d exceeds E = %d", l.top_k, E);
    if (residency != MP_DEVICE && residency != MP_HOST_PINNED)
        return fail(residency == MP_HOST_PAGEABLE || residency == MP_HOST_FILE ? MP_E_UNSUPPORTED : MP_E_ARG,
                    "residency %d is not MP_DEVICE or MP_HOST_PINNED", residency);
    if (experts == nullptr)
        return fail(MP_E_ARG, "experts is NULL");
    if ((rc = check_ld(ldx, l.hidden, "ldx")) || (rc = check_ld(ldy, l.hidden, "ldy")) ||
        (residual && (rc = check_ld(ldr, l.hidden, "ldr"))))
        return rc;
    if (tokens == 0)
        return MP_OK;
    Seen seen;
    Span X, RT, RB, R, Y, I, G, S;
    if ((rc = check_workspace(seen, workspace, workspace_bytes, moe_ws_bytes(l, tokens), &S)) ||
        (rc = check_matrix(seen, x, tokens, l.hidden, ldx, es, "x", &X)) ||
        (rc = check_matrix(seen, router, E, l.hidden, l.hidden, es, "router", &RT)) ||
        (router_bias && (rc = check_matrix(seen, router_bias, 1, E, E, es, "router_bias", &RB))) ||
        (residual && (rc = check_matrix(seen, residual, tokens, l.hidden, ldr, es, "residual", &R))) ||
        (rc = check_matrix(seen, y, tokens, l.hidden, ldy, es, "y", &Y)) ||
        (ids && (rc = check_matrix(seen, ids, tokens, l.top_k, l.top_k, 4, "ids", &I))) ||
        (gates && (rc = check_matrix(seen, gates, tokens, l.top_k, l.top_k, 4, "gates", &G))))
        return rc;
    const int64_t df = l.hidden * l.ffn;  // <= 2^48
    int64_t last = l.gate_off > l.down_off ? l.gate_off : l.down_off;
    last = l.up_off > last ? l.up_off : last;
    const size_t ebytes = (size_t)(last + df) * (size_t)es;
    MoeArgs a{l, (int)tokens, E, x, ldx, router, router_bias, residual, ldr, y, ldy, ids, gates};
    ExpertPtrs ex{};
    Span ES[kMaxK];
    for (int i = 0; i < E; ++i) {
        char nm[32];
        std::snprintf(nm, sizeof nm, "experts[%d]", i);
        if (reinterpret_cast<uintptr_t>(experts[i]) % (uintptr_t)es != 0)
            return fail(MP_E_ARG, "%s is not aligned to its elements", nm);
        ex.p[i] = experts[i];
        rc = residency == MP_DEVICE ? seen.check(experts[i], ebytes, nm)
                                    : check_pinned_buffer(experts[i], ebytes, nm, &ex.p[i]);
        if (rc)
            return rc;
        ES[i] = Span{static_cast<const char*>(experts[i]), ebytes, 0, "an expert"};
    }
    if ((rc = check_apart(Y, X, true)) || (rc = check_apart(Y, R, true)) || (rc = check_apart(Y, RT, false)) ||
        (rc = check_apart(Y, RB, false)))
        return rc;
    for (const Span* o : {&I, &G, &S})
        for (const Span* i : {&X, &RT, &RB, &R, &Y})
            if ((rc = check_apart(*o, *i, false)))
                return rc;
    if ((rc = check_apart(I, G, false)) || (rc = check_apart(S, I, false)) || (rc = check_apart(S, G, false)))
        return rc;
    for (int i = 0; i < E; ++i)
        for (const Span* o : {&Y, &I, &G, &S})
            if ((rc = check_apart(*o, ES[i], false)))
                return rc;
    hipError_t e = launch_moe(a, ex, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MP_OK : hip_fail(e, "moe launch");
}

}  // extern "C"
