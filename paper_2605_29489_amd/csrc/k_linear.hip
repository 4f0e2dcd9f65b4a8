// A linear layer with bias, activation and residual, and its backward pass.
#include "ffn_common.h"
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
