// A linear layer with bias, activation and residual, and its backward pass.
#include "ffn_common.h"
#include "gemm.h"
#include "mm_few.h"
#include "mp_internal.h"

namespace mp {
namespace {

// ---------------------------------------------------------------- a few tokens
// A workgroup takes 16 weight rows, its W waves split k, and the partial tiles
// meet in LDS.
template <int DT, int T8, int W>
__global__ __launch_bounds__(64 * W) void k_linear_few(const char* x, int64_t ldx, const char* w, int64_t ldw,
                                                       typename Elem<DT>::T* y, int64_t ldy, int M, int64_t N,
                                                       int64_t K, Epi e)
{
    using T = typename Elem<DT>::T;
    using F = Few<DT, 1, T8, 1>;
    constexpr int es = Fmt<DT>::esize;
    // a wave's operands on the way, then its partial tiles
    constexpr int kWave = F::kLds > F::NT * 1024 ? F::kLds : F::NT * 1024;
    __shared__ __attribute__((aligned(16))) char lds[W * kWave];
    const int lane = threadIdx.x & 63, wave = (int)uniform_u32(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    F f;
    f.clear();
    f.lds = lds + wave * kWave;
#pragma unroll
    for (int m = 0; m < 2; ++m) {  // rows and tokens past the last repeat it; their outputs are dropped
        const int64_t r = n0 + F::row_of(lane, m);
        f.w[0][m] = w + (r < N ? r : N - 1) * ldw * es + F::off(lane);
    }
#pragma unroll
    for (int m = 0; m < T8; ++m) {
        const int r = F::row_of(lane, m);
        f.x[0][m] = x + (int64_t)(r < M ? r : M - 1) * ldx * es + F::off(lane);
    }
    f.row(K, wave, W);
    float4* red = reinterpret_cast<float4*>(f.lds);
#pragma unroll
    for (int t = 0; t < F::NT; ++t)
        red[t * 64 + lane] = f.out(0, t);
    __syncthreads();
    sum_tiles<F::NT, W>(reinterpret_cast<const float4*>(lds), kWave / 16, threadIdx.x, 64 * W,
                        [&](int tile, int row, int tok, float v) {
                            const int t = tile * 16 + tok;
                            const int64_t j = n0 + row;
                            if (t >= M || j >= N)
                                return;
                            if (e.bias)
                                v += (float)static_cast<const T*>(e.bias)[j];
                            if (e.z)
                                static_cast<T*>(e.z)[t * e.ldz + j] = (T)v;
                            v = act_of(e.act, v);
                            if (e.r)
                                v += (float)static_cast<const T*>(e.r)[t * e.ldr + j];
                            y[t * ldy + j] = (T)v;
                        });
}

// Up to so many tokens go to k_linear_few, more to the tiled products.  us through
// 8960 x 1536, here and there: 33 tokens bf16 11.7 and 12.9, 64 tokens 12.9 and
// 12.8; fp32, bound by the matrix cores, 34 and 26, 35 and 28.
constexpr int kFewTokens = 64;

// One to four tokens: a workgroup takes RG rows, its W waves split k.  us through
// 1536 x 8960, with k_linear_few in brackets: fp32 1 token 10.1 (16.2), 4 tokens 11.9
// (16.4); bf16 1 and 2 tokens 7.9 (7.9), 4 tokens 9.3 (8.2).
template <int DT, int RG, int TT, int W>
__global__ __launch_bounds__(64 * W) void k_linear_gemv(const char* x, int64_t ldx, const char* w, int64_t ldw,
                                                        typename Elem<DT>::T* y, int64_t ldy, int M, int64_t N,
                                                        int64_t K, Epi e)
{
    using T = typename Elem<DT>::T;
    using G = Gemv<DT, RG, TT, false>;
    __shared__ float red[W][RG * TT];
    const int wave = (int)uniform_u32(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * RG;
    const char *wp[RG], *xp[TT];
#pragma unroll
    for (int i = 0; i < RG; ++i)  // rows and tokens past the last repeat it; their outputs are dropped
        wp[i] = w + (n0 + i < N ? n0 + i : N - 1) * ldw * G::es;
#pragma unroll
    for (int t = 0; t < TT; ++t)
        xp[t] = x + (int64_t)(t < M ? t : M - 1) * ldx * G::es;
    G g;
    g.clear();
    g.row(wp, xp, K, wave, W);
    g.put(red[wave]);
    __syncthreads();
    const int t = threadIdx.x % TT;
    const int64_t j = n0 + threadIdx.x / TT;
    if (threadIdx.x >= RG * TT || t >= M || j >= N)
        return;
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k)
        v += red[k][threadIdx.x];
    if (e.bias)
        v += (float)static_cast<const T*>(e.bias)[j];
    if (e.z)
        static_cast<T*>(e.z)[t * e.ldz + j] = (T)v;
    v = act_of(e.act, v);
    if (e.r)
        v += (float)static_cast<const T*>(e.r)[t * e.ldr + j];
    y[t * ldy + j] = (T)v;
}

template <int DT, int RG, int TT>
hipError_t gemv_go(const mp_linear_shape& s, const void* x, const void* w, void* y, const Epi& e, hipStream_t st)
{
    const int64_t groups = (s.n + RG - 1) / RG, runs = s.k / Gemv<DT, RG, TT, false>::kRun, want = 4096 / groups;
    const int64_t W = want < runs / 2 ? want : runs / 2;
    using T = typename Elem<DT>::T;
#define MP_GEMV(w_)                                                                                               \
    hipLaunchKernelGGL((k_linear_gemv<DT, RG, TT, w_>), dim3((unsigned)groups), dim3(64 * w_), 0, st,             \
                       (const char*)x, s.ldx, (const char*)w, s.ldw, (T*)y, s.ldy, (int)s.m, s.n, s.k, e)
    if (W >= 8)
        MP_GEMV(8);
    else if (W >= 4)
        MP_GEMV(4);
    else if (W >= 2)
        MP_GEMV(2);
    else
        MP_GEMV(1);
#undef MP_GEMV
    return hipGetLastError();
}


template <int DT, int T8>
hipError_t few_go(const mp_linear_shape& s, const void* x, const void* w, void* y, const Epi& e, hipStream_t st)
{
    // waves to fill the chip, with 512 bytes of each row at least
    const int64_t tiles = (s.n + 15) / 16, most = s.k * Fmt<DT>::esize / 512, want = 4096 / tiles;
    const int64_t W = want < most ? want : most;
    const dim3 g((unsigned)tiles);
    using T = typename Elem<DT>::T;
#define MP_FEW(w_)                                                                                                \
    hipLaunchKernelGGL((k_linear_few<DT, T8, w_>), g, dim3(64 * w_), 0, st, (const char*)x, s.ldx,            \
                       (const char*)w, s.ldw, (T*)y, s.ldy, (int)s.m, s.n, s.k, e)
    if constexpr (T8 < 8)
        if (W >= 16) {
            MP_FEW(16);
            return hipGetLastError();
        }
    if (W >= 8)
        MP_FEW(8);
    else
        MP_FEW(4);
#undef MP_FEW
    return hipGetLastError();
}

template <int DT>
hipError_t linear_few(const mp_linear_shape& s, const void* x, const void* w, void* y, const Epi& e, hipStream_t st)
{
    if (s.m == 1)
        return gemv_go<DT, 4, 1>(s, x, w, y, e, st);
    if (s.m == 2)
        return gemv_go<DT, 4, 2>(s, x, w, y, e, st);
    if (s.m <= 4)
        return gemv_go<DT, 4, 4>(s, x, w, y, e, st);
    if (s.m <= 8)
        return few_go<DT, 1>(s, x, w, y, e, st);
    if (s.m <= 16)
        return few_go<DT, 2>(s, x, w, y, e, st);
    if (s.m <= 32)
        return few_go<DT, 4>(s, x, w, y, e, st);
    return few_go<DT, 8>(s, x, w, y, e, st);
}

// ---------------------------------------------------------------- dz
// dz = dy * act'(z) in the dtype, and the columns' sums of the unrounded values.
// In bf16 the rounding is that of the type the matrix cores multiply: dx and dw
// are 2.3e-3 of their norm from the definition (up to 2.8e-3 where few terms are
// added), 1.7e-3 (2.0e-3) with dz in fp32.  A second bf16 value for what the
// rounding leaves would double both products, 410 of 8192 x 8960 x 1536's 461 us.
// Bound by memory (8192 x 8960 bf16: 79 us, 5.6 TB/s): a workgroup takes 512 (bf16)
// or 256 (fp32) columns of every gridDim.y-th band of 4 rows, a chunk per thread,
// and writes one partial row.
template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_dz(const typename Elem<DT>::T* dy, int64_t lddy,
                                            const typename Elem<DT>::T* z, int64_t ldz, typename Elem<DT>::T* dz,
                                            int64_t lddz, float* part, int64_t pitch, int64_t M, int64_t N)
{
    constexpr int V = Fmt<DT>::V;
    __shared__ float4 red[3][V / 4][64];
    const int lane = threadIdx.x & 63, band = threadIdx.x >> 6;
    const int64_t j = ((int64_t)blockIdx.x * 64 + lane) * V, have = N - j;
    float s[V];
#pragma unroll
    for (int u = 0; u < V; ++u)
        s[u] = 0.0f;
    auto get = [&](const typename Elem<DT>::T* p) {
        return have >= V ? ld16u(p) : have > 0 ? ld16_head<DT>(p, have) : make_uint4(0, 0, 0, 0);
    };
    const int64_t step = (int64_t)gridDim.y * 4;
    for (int64_t i = (int64_t)blockIdx.y * 4 + band; i < M; i += step) {
        float d[V];
        const uint4 dc = get(dy + i * lddy + j);
        if constexpr (ACT != MP_ACT_NONE) {
            float f[V];
            const uint4 zc = get(z + i * ldz + j);
            Fmt<DT>::unpack(dc, d);
            Fmt<DT>::unpack(zc, f);
#pragma unroll
            for (int u = 0; u < V; ++u)
                d[u] *= act_slope_f<ACT>(f[u]);
            if (dz) {  // rows of whole chunks; the columns past N are not read
                if (have > 0)
                    st16u(dz + i * lddz + j, Fmt<DT>::pack(d));
            }
        } else {
            Fmt<DT>::unpack(dc, d);
        }
#pragma unroll
        for (int u = 0; u < V; ++u)
            s[u] += d[u];
    }
    if (!part)
        return;
    if (band > 0)
#pragma unroll
        for (int u = 0; u < V / 4; ++u)
            red[band - 1][u][lane] = make_float4(s[4 * u], s[4 * u + 1], s[4 * u + 2], s[4 * u + 3]);
    __syncthreads();
    if (band == 0 && have > 0) {
#pragma unroll
        for (int u = 0; u < V / 4; ++u) {
            float4 v = make_float4(s[4 * u], s[4 * u + 1], s[4 * u + 2], s[4 * u + 3]);
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const float4 r = red[k][u][lane];
                v.x += r.x;
                v.y += r.y;
                v.z += r.z;
                v.w += r.w;
            }
            *reinterpret_cast<float4*>(part + blockIdx.y * pitch + j + 4 * u) = v;
        }
    }
}

// Bands of k_dz: enough workgroups to fill the chip, 2 rows a thread at least; 1 where there are no columns.
int dz_bands(const mp_linear_shape& s)
{
    if (s.n == 0)
        return 1;
    const int V = s.dtype == MP_F32 ? 4 : 8;
    const int64_t across = (s.n + 64 * V - 1) / (64 * V), want = (2048 + across - 1) / across, most = (s.m + 7) / 8;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 512 ? 512 : n);
}

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The workspace of a backward pass: dz, the partial rows of dbias, and what the products need, one after the other.
struct BackWs {
    uint64_t dz, part, gemm, bytes;
    int64_t lddz;
};
BackWs back_ws(const mp_linear_shape& s)
{
    BackWs w{};
    const uint64_t es = s.dtype == MP_F32 ? 4 : 2;
    w.lddz = up(s.n, 8);
    w.part = s.act != MP_ACT_NONE ? up((int64_t)((uint64_t)s.m * (uint64_t)w.lddz * es), 16) : 0;
    w.gemm = w.part + (uint64_t)dz_bands(s) * (uint64_t)w.lddz * 4;
    uint64_t g = 0;
    if (s.m > 0 && s.n > 0 && s.k > 0) {
        const uint64_t a = gemm_ws_bytes(s.dtype, s.m, s.k, s.n);
        const uint64_t b = gemm_ws_bytes(s.dtype, s.n, s.k, s.m);
        g = a > b ? a : b;
    }
    w.bytes = w.gemm + g;
    return w;
}

template <int DT>
hipError_t dz_go(const mp_linear_shape& s, const void* dy, const void* z, void* dz, float* part, const BackWs& w,
                 hipStream_t st)
{
    using T = typename Elem<DT>::T;
    const dim3 g((unsigned)((s.n + 64 * Fmt<DT>::V - 1) / (64 * Fmt<DT>::V)), dz_bands(s));
    auto go = [&](auto act) {
        hipLaunchKernelGGL((k_dz<DT, decltype(act)::value>), g, dim3(256), 0, st, (const T*)dy, s.ldy, (const T*)z,
                           s.ldz, (T*)dz, w.lddz, part, w.lddz, s.m, s.n);
    };
    switch (s.act) {
        case MP_ACT_RELU: go(std::integral_constant<int, MP_ACT_RELU>{}); break;
        case MP_ACT_GELU: go(std::integral_constant<int, MP_ACT_GELU>{}); break;
        case MP_ACT_GELU_TANH: go(std::integral_constant<int, MP_ACT_GELU_TANH>{}); break;
        case MP_ACT_SILU: go(std::integral_constant<int, MP_ACT_SILU>{}); break;
        default: go(std::integral_constant<int, MP_ACT_NONE>{}); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const mp_linear_shape& s, const void* x, const void* w, const void* bias,
                         const void* residual, void* y, void* z, void* ws, hipStream_t st)
{
    const Epi e{bias, residual, z, s.ldr, s.ldz, s.act};
    if (s.m <= kFewTokens)
        return s.dtype == MP_F32 ? linear_few<MP_F32>(s, x, w, y, e, st) : linear_few<MP_BF16>(s, x, w, y, e, st);
    const Gemm g{s.dtype, Form::NT, x, w, y, s.ldx, s.ldw, s.ldy, s.m, s.n, s.k, e};
    return launch_gemm(g, ws, st);
}

uint64_t linear_ws_bytes(const mp_linear_shape& s)
{
    if (s.m <= kFewTokens || s.n == 0)
        return 0;
    return gemm_ws_bytes(s.dtype, s.m, s.n, s.k);
}

hipError_t launch_linear_backward(const mp_linear_shape& s, const void* dy, const void* x, const void* w,
                                  const void* z, void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias,
                                  void* ws, hipStream_t st)
{
    const bool act = s.act != MP_ACT_NONE;
    const BackWs l = back_ws(s);
    char* base = static_cast<char*>(ws);
    hipError_t e = hipSuccess;
    if (s.n > 0 && ((act && (dx || dw)) || dbias)) {
        float* part = dbias ? reinterpret_cast<float*>(base + l.part) : nullptr;
        void* to = act && (dx || dw) ? base + l.dz : nullptr;
        e = s.dtype == MP_F32 ? dz_go<MP_F32>(s, dy, z, to, part, l, st) : dz_go<MP_BF16>(s, dy, z, to, part, l, st);
        if (e == hipSuccess && dbias)
            e = launch_sum_rows(s.dtype, part, dz_bands(s), l.lddz, s.n, dbias, st);
        if (e != hipSuccess)
            return e;
    }
    const void* dz = act ? static_cast<const void*>(base + l.dz) : dy;
    const int64_t lddz = act ? l.lddz : s.ldy;
    if (dx && s.m > 0 && s.k > 0) {
        const Gemm g{s.dtype, Form::NN, dz, w, dx, lddz, s.ldw, lddx, s.m, s.k, s.n, Epi{}};
        if ((e = launch_gemm(g, base + l.gemm, st)) != hipSuccess)
            return e;
    }
    if (dw && s.n > 0 && s.k > 0) {
        const Gemm g{s.dtype, Form::TN, dz, x, dw, lddz, s.ldx, lddw, s.n, s.k, s.m, Epi{}};
        e = launch_gemm(g, base + l.gemm, st);
    }
    return e;
}

uint64_t linear_backward_ws_bytes(const mp_linear_shape& s) { return back_ws(s).bytes; }

}  // namespace mp
