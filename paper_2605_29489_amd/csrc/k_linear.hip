// A linear layer with bias, activation and residual, and its backward pass.
#include "ffn_common.h"
#include "mm_few.h"
#include "mp_internal.h"

namespace mp {
namespace {

struct Epi {
    const void* bias;
    const void* r;
    void* z;
    int64_t ldr, ldz;
    int act;
};

// C[i][j] = epilogue(sum over p of A(i, p) B(j, p)), A(i, p) = a[i * ai + p * ap], B(j, p) = b[j * bj + p * bp]:
// a 64 x 64 tile per workgroup, 4 x 4 outputs per thread, 16 steps of p through LDS at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_gemm(const T* a, int64_t ai, int64_t ap, const T* b, int64_t bj, int64_t bp,
                                              T* c, int64_t ldc, int64_t I, int64_t J, int64_t P, Epi e)
{
    __shared__ float sa[16][65], sb[16][65];
    const int64_t i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int64_t p0 = 0; p0 < P; p0 += 16) {
        __syncthreads();
        for (int q = threadIdx.x; q < 1024; q += 256) {
            const int l = ap == 1 ? q >> 4 : q & 63, p = ap == 1 ? q & 15 : q >> 6;
            sa[p][l] = i0 + l < I && p0 + p < P ? (float)a[(i0 + l) * ai + (p0 + p) * ap] : 0.0f;
        }
        for (int q = threadIdx.x; q < 1024; q += 256) {
            const int l = bp == 1 ? q >> 4 : q & 63, p = bp == 1 ? q & 15 : q >> 6;
            sb[p][l] = j0 + l < J && p0 + p < P ? (float)b[(j0 + l) * bj + (p0 + p) * bp] : 0.0f;
        }
        __syncthreads();
        for (int p = 0; p < 16; ++p)
            for (int u = 0; u < 4; ++u)
                for (int v = 0; v < 4; ++v)
                    acc[u][v] = fmaf(sa[p][ty + 16 * u], sb[p][tx + 16 * v], acc[u][v]);
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ty + 16 * u, j = j0 + tx + 16 * v;
            if (i >= I || j >= J)
                continue;
            float z = acc[u][v];
            if (e.bias)
                z += (float)static_cast<const T*>(e.bias)[j];
            if (e.z)
                static_cast<T*>(e.z)[i * e.ldz + j] = (T)z;
            float y = act_of(e.act, z);
            if (e.r)
                y += (float)static_cast<const T*>(e.r)[i * e.ldr + j];
            c[i * ldc + j] = (T)y;
        }
}

// ---------------------------------------------------------------- a few tokens
// A workgroup takes NA tiles of 16 weight rows, its W waves split k, and the
// partial tiles meet in LDS.
template <int DT, int NA, int TT, int W>
__global__ __launch_bounds__(64 * W) void k_linear_few(const char* x, int64_t ldx, const char* w, int64_t ldw,
                                                       typename Elem<DT>::T* y, int64_t ldy, int M, int64_t N,
                                                       int64_t K, Epi e)
{
    using T = typename Elem<DT>::T;
    constexpr int es = Fmt<DT>::esize;
    __shared__ float4 red[W * NA * TT * 64];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NA), whole = few_whole<DT>(K);
    const char *wp[NA], *xp[TT];
    bool go[TT];
#pragma unroll
    for (int i = 0; i < NA; ++i) {  // rows past the last repeat it; their outputs are dropped
        const int64_t r = n0 + i * 16 + (lane & 15);
        wp[i] = w + (r < N ? r : N - 1) * ldw * es + (lane >> 4) * 16;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int r = t * 16 + (lane & 15);
        go[t] = r < M;
        xp[t] = go[t] ? x + (int64_t)r * ldx * es + (lane >> 4) * 16 : reinterpret_cast<const char*>(g_zero_steps);
    }
    f32x4 acc[NA][TT] = {};
    few_steps<DT, NA, TT, 1, few_unroll(NA + TT)>(acc, wp, xp, go, whole * wave / W, whole * (wave + 1) / W);
    if (wave == W - 1 && few_rest<DT>(K))
        few_tail<DT, NA, TT, 1>(acc, wp, xp, go, whole, few_rest<DT>(K));
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int t = 0; t < TT; ++t)
            red[((wave * NA + i) * TT + t) * 64 + lane] =
                make_float4(acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]);
    __syncthreads();
    sum_tiles<NA * TT>(red, W, threadIdx.x, 64 * W, [&](int q, const float4& s) {
        const int t = (q >> 6) % TT * 16 + (q & 15);
        const int64_t j0 = n0 + (q >> 6) / TT * 16 + ((q & 63) >> 4) * 4;
        const float v[4] = {s.x, s.y, s.z, s.w};
        if (t >= M)
            return;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t j = j0 + u;
            if (j >= N)
                break;
            float z = v[u];
            if (e.bias)
                z += (float)static_cast<const T*>(e.bias)[j];
            if (e.z)
                static_cast<T*>(e.z)[t * e.ldz + j] = (T)z;
            float a = act_of(e.act, z);
            if (e.r)
                a += (float)static_cast<const T*>(e.r)[t * e.ldr + j];
            y[t * ldy + j] = (T)a;
        }
    });
}

constexpr int kFewTokens = 64;

template <int DT, int NA, int TT>
hipError_t few_go(const mp_linear_shape& s, const void* x, const void* w, void* y, const Epi& e, hipStream_t st)
{
    // waves to fill the chip, with 8 steps each at least
    const int64_t tiles = (s.n + 16 * NA - 1) / (16 * NA), whole = few_whole<DT>(s.k);
    const int64_t most = whole / 8, want = 4096 / tiles;
    const int64_t W = want < most ? want : most;
    const dim3 g((unsigned)tiles);
    using T = typename Elem<DT>::T;
#define MP_FEW(w_)                                                                                              \
    hipLaunchKernelGGL((k_linear_few<DT, NA, TT, w_>), g, dim3(64 * w_), 0, st, (const char*)x, s.ldx,            \
                       (const char*)w, s.ldw, (T*)y, s.ldy, (int)s.m, s.n, s.k, e)
    if (W >= 16)
        MP_FEW(16);
    else if (W >= 8)
        MP_FEW(8);
    else
        MP_FEW(4);
#undef MP_FEW
    return hipGetLastError();
}

template <int DT>
hipError_t linear_few(const mp_linear_shape& s, const void* x, const void* w, void* y, const Epi& e, hipStream_t st)
{
    if (s.m <= 16)
        return few_go<DT, 1, 1>(s, x, w, y, e, st);
    if (s.m <= 32)
        return few_go<DT, 2, 2>(s, x, w, y, e, st);
    return few_go<DT, 2, 4>(s, x, w, y, e, st);
}

template <typename T>
hipError_t gemm(const void* a, int64_t ai, int64_t ap, const void* b, int64_t bj, int64_t bp, void* c, int64_t ldc,
                int64_t I, int64_t J, int64_t P, const Epi& e, hipStream_t st)
{
    const dim3 g((unsigned)((J + 63) / 64), (unsigned)((I + 63) / 64));
    hipLaunchKernelGGL(k_gemm<T>, g, dim3(256), 0, st, (const T*)a, ai, ap, (const T*)b, bj, bp, (T*)c, ldc, I, J, P,
                       e);
    return hipGetLastError();
}

// dz = dy * act'(z), and its column sums: one thread per column.
template <typename T>
__global__ __launch_bounds__(256) void k_dz(const T* dy, int64_t lddy, const T* z, int64_t ldz, int act, T* dz, T* db,
                                            int64_t M, int64_t N)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= N)
        return;
    float s = 0.0f;
    for (int64_t i = 0; i < M; ++i) {
        float v = (float)dy[i * lddy + j];
        if (act != MP_ACT_NONE)
            v *= act_slope_of(act, (float)z[i * ldz + j]);
        s += v;
        if (dz)
            dz[i * N + j] = (T)v;
    }
    if (db)
        db[j] = (T)s;
}

template <typename T>
hipError_t back_t(const mp_linear_shape& s, const void* dy, const void* x, const void* w, const void* z, void* dx,
                  int64_t lddx, void* dw, int64_t lddw, void* db, void* ws, hipStream_t st)
{
    const bool act = s.act != MP_ACT_NONE;
    hipError_t e = hipSuccess;
    if (s.n > 0 && (act || db))
        hipLaunchKernelGGL(k_dz<T>, dim3((unsigned)((s.n + 255) / 256)), dim3(256), 0, st, (const T*)dy, s.ldy,
                           (const T*)z, s.ldz, s.act, act ? (T*)ws : nullptr, (T*)db, s.m, s.n);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    const void* dz = act ? ws : dy;
    const int64_t lddz = act ? s.n : s.ldy;
    const Epi none{};
    if (dx && s.m > 0 && s.k > 0 &&
        (e = gemm<T>(dz, lddz, 1, w, 1, s.ldw, dx, lddx, s.m, s.k, s.n, none, st)) != hipSuccess)
        return e;
    if (dw && s.n > 0 && s.k > 0)
        e = gemm<T>(dz, 1, lddz, x, 1, s.ldx, dw, lddw, s.n, s.k, s.m, none, st);
    return e;
}

}  // namespace

hipError_t launch_linear(const mp_linear_shape& s, const void* x, const void* w, const void* bias,
                         const void* residual, void* y, void* z, void* ws, hipStream_t st)
{
    const Epi e{bias, residual, z, s.ldr, s.ldz, s.act};
    if (s.m <= kFewTokens)
        return s.dtype == MP_F32 ? linear_few<MP_F32>(s, x, w, y, e, st) : linear_few<MP_BF16>(s, x, w, y, e, st);
    return s.dtype == MP_F32 ? gemm<float>(x, s.ldx, 1, w, s.ldw, 1, y, s.ldy, s.m, s.n, s.k, e, st)
                             : gemm<__bf16>(x, s.ldx, 1, w, s.ldw, 1, y, s.ldy, s.m, s.n, s.k, e, st);
}

uint64_t linear_ws_bytes(const mp_linear_shape& s) { return 0; }

hipError_t launch_linear_backward(const mp_linear_shape& s, const void* dy, const void* x, const void* w,
                                  const void* z, void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias,
                                  void* ws, hipStream_t st)
{
    return s.dtype == MP_F32 ? back_t<float>(s, dy, x, w, z, dx, lddx, dw, lddw, dbias, ws, st)
                             : back_t<__bf16>(s, dy, x, w, z, dx, lddx, dw, lddw, dbias, ws, st);
}

uint64_t linear_backward_ws_bytes(const mp_linear_shape& s)
{
    if (s.act == MP_ACT_NONE)
        return 0;
    return ((uint64_t)s.m * (uint64_t)s.n * (s.dtype == MP_F32 ? 4 : 2) + 15) / 16 * 16;
}

}  // namespace mp
