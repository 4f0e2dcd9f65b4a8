// Layer norm and RMS norm, forward and backward.
#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

__device__ inline float block_sum(float v, float* tmp)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    return tmp[0] + tmp[1] + tmp[2] + tmp[3];
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm(const T* x, const T* w, const T* b, T* y, float* mean, float* rstd,
                                              int64_t cols, int64_t ldx, int64_t ldy, float eps, bool rms)
{
    __shared__ float tmp[4];
    const int64_t r = blockIdx.x;
    x += r * ldx;
    y += r * ldy;
    float s = 0.0f;
    if (!rms) {
        for (int64_t c = threadIdx.x; c < cols; c += 256)
            s += (float)x[c];
        s = block_sum(s, tmp) / (float)cols;
    }
    float q = 0.0f;
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
        const float d = (float)x[c] - s;
        q = fmaf(d, d, q);
    }
    const float rs = 1.0f / sqrtf(block_sum(q, tmp) / (float)cols + eps);
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
        float v = ((float)x[c] - s) * rs;
        v = v * (w ? (float)w[c] : 1.0f) + (b ? (float)b[c] : 0.0f);
        y[c] = (T)v;
    }
    if (threadIdx.x == 0) {
        if (mean)
            mean[r] = s;
        if (rstd)
            rstd[r] = rs;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_dx(const T* dy, const T* x, const T* w, const float* mean,
                                                 const float* rstd, T* dx, int64_t cols, int64_t lddy, int64_t ldx,
                                                 int64_t lddx)
{
    __shared__ float tmp[4];
    const int64_t r = blockIdx.x;
    x += r * ldx;
    dy += r * lddy;
    dx += r * lddx;
    const float m = mean ? mean[r] : 0.0f, rs = rstd[r];
    float sg = 0.0f, sgn = 0.0f;
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
        const float g = (float)dy[c] * (w ? (float)w[c] : 1.0f);
        sg += g;
        sgn = fmaf(g, ((float)x[c] - m) * rs, sgn);
    }
    sg = mean ? block_sum(sg, tmp) / (float)cols : 0.0f;
    sgn = block_sum(sgn, tmp) / (float)cols;
    for (int64_t c = threadIdx.x; c < cols; c += 256) {
        const float g = (float)dy[c] * (w ? (float)w[c] : 1.0f);
        const float n = ((float)x[c] - m) * rs;
        dx[c] = (T)(rs * (g - sg - n * sgn));
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_dw(const T* dy, const T* x, const float* mean, const float* rstd, T* dw,
                                                 T* db, int64_t rows, int64_t cols, int64_t lddy, int64_t ldx)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= cols)
        return;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t r = 0; r < rows; ++r) {
        const float d = (float)dy[r * lddy + c];
        sb += d;
        sw = fmaf(d, ((float)x[r * ldx + c] - (mean ? mean[r] : 0.0f)) * rstd[r], sw);
    }
    if (dw)
        dw[c] = (T)sw;
    if (db)
        db[c] = (T)sb;
}

template <typename T>
hipError_t norm_t(const mp_norm_shape& s, const void* x, const void* w, const void* b, void* y, float* mean,
                  float* rstd, hipStream_t st)
{
    hipLaunchKernelGGL(k_norm<T>, dim3((unsigned)s.rows), dim3(256), 0, st, (const T*)x, (const T*)w, (const T*)b,
                       (T*)y, mean, rstd, s.cols, s.ldx, s.ldy, s.eps, (s.flags & MP_NORM_RMS) != 0);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_back_t(const mp_norm_shape& s, const void* dy, const void* x, const void* w, const float* mean,
                       const float* rstd, void* dx, int64_t lddx, void* dw, void* db, hipStream_t st)
{
    if (dx && s.rows)
        hipLaunchKernelGGL(k_norm_dx<T>, dim3((unsigned)s.rows), dim3(256), 0, st, (const T*)dy, (const T*)x,
                           (const T*)w, mean, rstd, (T*)dx, s.cols, s.ldy, s.ldx, lddx);
    if (dw || db)
        hipLaunchKernelGGL(k_norm_dw<T>, dim3((unsigned)((s.cols + 255) / 256)), dim3(256), 0, st, (const T*)dy,
                           (const T*)x, mean, rstd, (T*)dw, (T*)db, s.rows, s.cols, s.ldy, s.ldx);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const mp_norm_shape& s, const void* x, const void* weight, const void* bias, void* y,
                       float* mean, float* rstd, hipStream_t st)
{
    return s.dtype == MP_F32 ? norm_t<float>(s, x, weight, bias, y, mean, rstd, st)
                             : norm_t<__bf16>(s, x, weight, bias, y, mean, rstd, st);
}

hipError_t launch_norm_backward(const mp_norm_shape& s, const void* dy, const void* x, const void* weight,
                                const float* mean, const float* rstd, void* dx, int64_t lddx, void* dweight,
                                void* dbias, void* ws, hipStream_t st)
{
    return s.dtype == MP_F32 ? norm_back_t<float>(s, dy, x, weight, mean, rstd, dx, lddx, dweight, dbias, st)
                             : norm_back_t<__bf16>(s, dy, x, weight, mean, rstd, dx, lddx, dweight, dbias, st);
}

uint64_t norm_ws_bytes(const mp_norm_shape& s) { return 0; }

}  // namespace mp
