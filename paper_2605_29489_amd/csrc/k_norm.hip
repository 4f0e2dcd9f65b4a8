// Layer norm and RMS norm, forward and backward.
#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

// ---------------------------------------------------------------- rows in registers
// A row is held by TPR threads (8, a wave of 64, or a workgroup's 256 or
// 1024), NV chunks of 16 bytes each: chunk i of thread l starts at column
// (i * TPR + l) * V, so a load instruction covers adjacent chunks, and all but
// the last chunk of a thread are whole.
template <int DT, int TPR, int NV>
struct Row {
    static constexpr int V = Fmt<DT>::V;
    using T = typename Elem<DT>::T;
    uint4 c[NV];

    __device__ inline void load(const T* p, int l, int cols)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * TPR + l) * V;
            if (i < NV - 1 || at + V <= cols)
                c[i] = ld16u(p + at);
            else
                c[i] = at < cols ? ld16_head<DT>(p + at, cols - at) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            c[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ static inline void store(T* p, int i, int l, int cols, const float* f)
    {
        const int at = (i * TPR + l) * V;
        const uint4 v = Fmt<DT>::pack(f);
        if (i < NV - 1 || at + V <= cols)
            st16u(p + at, v);
        else if (at < cols)
            st16_head<DT>(p + at, v, cols - at);
    }
};

// Sum over a row's TPR threads, the same bits in each.  tmp: 16 floats of LDS
// that no thread still reads from an earlier call (rows of more than a wave;
// callers alternate between two).
template <int TPR>
__device__ inline float row_sum(float v, float* tmp)
{
    if constexpr (TPR < 64) {
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1)
            v += __shfl_xor(v, o, TPR);
        return v;
    }
    v = wave_xor_sum(v);
    if constexpr (TPR > 64) {
        const int w = (threadIdx.x % TPR) >> 6;
        if ((threadIdx.x & 63) == 0)
            tmp[w] = v;
        __syncthreads();
        v = tmp[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i)
            v += tmp[i];
    }
    return v;
}

template <int DT>
struct NormArgs {
    using T = typename Elem<DT>::T;
    const T* x;
    const T* w;
    const T* b;
    T* y;
    float* mean;
    float* rstd;
    int64_t rows, ldx, ldy;
    int cols;
    float eps;
    int rms;
};

// Rows that need barriers have a workgroup each.
constexpr int norm_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }

// y = (x - mean) rstd w + b.  The row is read once and stays in registers;
// the sum of squares is taken of the differences from the mean, so that a
// large mean costs no digits.  Bound by memory, and by w and b, which come
// through L2 for every row: 16384 x 3584 bf16 in 52 us (4.5 TB/s; RMS norm
// without b 47), 16384 x 1536 in 20 us.  Rows of 512 threads and more go to the
// workgroups that the chip holds, which keep w and b and load the next row
// before the present one is reduced.  us with w and b kept and with a workgroup
// per row, layer norm with bias:
//   128 and 256 threads, bf16  16384 x 3584: 60, 56; 8192 x 4104: 41, 35; 8192 x 8192: 49, 52
//   256 threads, fp32          8192 x 3200: 42, 44; 8192 x 4096: 50, 51
//   512 threads, bf16          4096 x 8200: 44, 34; 4096 x 12288: 39, 46; 2048 x 16384: 28, 36
//   512 threads, fp32          4096 x 4104: 27, 31; 3000 x 8192: 39, 42
//   1024 threads               2048 x 18944 bf16: 41, 49; 3000 x 8961 fp32: 50, 56
// Up to 256 threads it gains 2 to 6 % in full rows and costs up to 17 % elsewhere.
constexpr bool norm_stays(int tpr) { return tpr >= 512; }
template <int DT, int TPR, int NV>
__global__ __launch_bounds__(norm_threads(TPR)) void k_norm(NormArgs<DT> a)
{
    constexpr int kRows = norm_threads(TPR) / TPR, V = Fmt<DT>::V;
    __shared__ float tmp[2][TPR > 64 ? TPR / 64 : 1];
    const int l = threadIdx.x % TPR, cols = a.cols;
    using R = Row<DT, TPR, NV>;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    R x, w, b, x1;
    auto fetch = [&]() {
        x.load(a.x + r * a.ldx, l, cols);
        if (a.w)
            w.load(a.w, l, cols);
        if (a.b)
            b.load(a.b, l, cols);
    };
    if constexpr (norm_stays(TPR))
        if (r < a.rows)
            fetch();
    // rows of one wave or less need no barrier, so their threads may leave the loop early
    for (; r < a.rows; r += step) {
        if constexpr (!norm_stays(TPR))
            fetch();
        else if (r + step < a.rows)
            x1.load(a.x + (r + step) * a.ldx, l, cols);
        float m = 0.0f, f[V];
        if (!a.rms) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                Fmt<DT>::unpack(x.c[i], f);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    s += f[j];
            }
            m = row_sum<TPR>(s, tmp[0]) / (float)cols;
        }
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Fmt<DT>::unpack(x.c[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float d = f[j] - m;
                if (i == NV - 1)
                    d = (i * TPR + l) * V + j < cols ? d : 0.0f;
                q = fmaf(d, d, q);
            }
        }
        const float rs = 1.0f / sqrtf(row_sum<TPR>(q, tmp[1]) / (float)cols + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float g[V];
            Fmt<DT>::unpack(x.c[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                f[j] = (f[j] - m) * rs;
            if (a.w) {
                Fmt<DT>::unpack(w.c[i], g);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    f[j] *= g[j];
            }
            if (a.b) {
                Fmt<DT>::unpack(b.c[i], g);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    f[j] += g[j];
            }
            R::store(a.y + r * a.ldy, i, l, cols, f);
        }
        if (l == 0) {
            if (a.mean)
                a.mean[r] = m;
            if (a.rstd)
                a.rstd[r] = rs;
        }
        if constexpr (norm_stays(TPR))
            x = x1;
        if constexpr (TPR > 64)
            __syncthreads();  // tmp is free again
    }
}

// Rows longer than a workgroup's registers (over 32768 bf16 or 16384 fp32
// columns, wider than the hidden sizes that norms meet): read three times, an
// element per thread.  RMS norm of 1000 x 40000 bf16 86 us, 1000 x 20000 fp32 55 us.
template <int DT>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs<DT> a)
{
    using T = typename Elem<DT>::T;
    __shared__ float tmp[2][16];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = a.x + r * a.ldx;
        float m = 0.0f, s = 0.0f, q = 0.0f;
        if (!a.rms) {
            for (int c = threadIdx.x; c < a.cols; c += 1024)
                s += (float)x[c];
            m = row_sum<1024>(s, tmp[0]) / (float)a.cols;
        }
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
            const float d = (float)x[c] - m;
            q = fmaf(d, d, q);
        }
        const float rs = 1.0f / sqrtf(row_sum<1024>(q, tmp[1]) / (float)a.cols + a.eps);
        for (int c = threadIdx.x; c < a.cols; c += 1024)
            a.y[r * a.ldy + c] =
                (T)(((float)x[c] - m) * rs * (a.w ? (float)a.w[c] : 1.0f) + (a.b ? (float)a.b[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (a.mean)
                a.mean[r] = m;
            if (a.rstd)
                a.rstd[r] = rs;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- backward
template <int DT>
struct NormBackArgs {
    using T = typename Elem<DT>::T;
    const T* dy;
    const T* x;
    const T* w;
    const float* mean;  // null: RMS norm
    const float* rstd;
    T* dx;        // or null
    float* part;  // [workgroup][2][pitch]: each workgroup's sums of dy n and of dy; or null
    int64_t rows, lddy, ldx, lddx;
    int cols, pitch;
};

// Workgroup size of the one-pass backward kernel.
constexpr int back_threads(int tpr) { return tpr < 512 ? 512 : tpr; }

// dx, and the columns' sums of dy n and dy, in one reading of dy and x.  A
// workgroup takes every gridDim-th band of rows; a thread keeps the sums of its
// columns in registers (NV * V <= 24 columns, so that two rows and the sums
// fit; 16384 x 1536 bf16 41 us with the sum of the partial rows, 1001 x 8961 fp32
// 33 us, a wait for every row and the second launch included), the workgroup
// adds its bands' sums through LDS and writes one partial row, which k_sum_rows
// adds.  The next row is loaded before the present one is reduced.
template <int DT, int TPR, int NV>
__global__ __launch_bounds__(back_threads(TPR)) void k_norm_back(NormBackArgs<DT> a)
{
    constexpr int kT = back_threads(TPR), kRows = kT / TPR, V = Fmt<DT>::V;
    using R = Row<DT, TPR, NV>;
    constexpr bool kAhead = TPR < 1024;  // a workgroup of 1024 has 128 registers a thread
    __shared__ float tmp[2][kRows][2][TPR > 64 ? TPR / 64 : 1];
    constexpr int kHalf = kRows > 1 ? kRows / 2 : 1;
    __shared__ float4 sum[kHalf][NV * V / 4][TPR];
    const int l = threadIdx.x % TPR, band = threadIdx.x / TPR, cols = a.cols;
    const float inv = 1.0f / (float)cols;
    float sw[NV * V], sb[NV * V];
#pragma unroll
    for (int i = 0; i < NV * V; ++i)
        sw[i] = sb[i] = 0.0f;
    R w;
    w.clear();
    if (a.w)
        w.load(a.w, l, cols);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + band;
    R x, d, x1, d1;
    float m = 0.0f, rs = 0.0f, m1 = 0.0f, rs1 = 0.0f;
    // a band past the last row works on zeros, so that every thread of the workgroup meets its barriers
    auto fetch = [&](int64_t row, R& xx, R& dd, float& mm, float& rr) {
        if (row < a.rows) {
            xx.load(a.x + row * a.ldx, l, cols);
            dd.load(a.dy + row * a.lddy, l, cols);
            mm = a.mean ? a.mean[row] : 0.0f;
            rr = a.rstd[row];
        } else {
            xx.clear();
            dd.clear();
            mm = rr = 0.0f;
        }
    };
    fetch(r, x, d, m, rs);
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.rows; r0 += step, r += step, turn ^= 1) {
        if constexpr (kAhead)
            fetch(r + step, x1, d1, m1, rs1);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float xf[V], df[V], wf[V];
            Fmt<DT>::unpack(x.c[i], xf);
            Fmt<DT>::unpack(d.c[i], df);
            if (a.w)
                Fmt<DT>::unpack(w.c[i], wf);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float n = (xf[j] - m) * rs, g = a.w ? df[j] * wf[j] : df[j];
                sw[i * V + j] = fmaf(df[j], n, sw[i * V + j]);
                sb[i * V + j] += df[j];
                s1 += g;
                s2 = fmaf(g, n, s2);
            }
        }
        if (a.dx) {
            if constexpr (TPR <= 64) {
                s1 = row_sum<TPR>(s1, nullptr);
                s2 = row_sum<TPR>(s2, nullptr);
            } else {  // both sums over one barrier
                s1 = wave_xor_sum(s1);
                s2 = wave_xor_sum(s2);
                const int wv = l >> 6;
                if ((threadIdx.x & 63) == 0) {
                    tmp[turn][band][0][wv] = s1;
                    tmp[turn][band][1][wv] = s2;
                }
                __syncthreads();
                s1 = tmp[turn][band][0][0];
                s2 = tmp[turn][band][1][0];
#pragma unroll
                for (int i = 1; i < TPR / 64; ++i) {
                    s1 += tmp[turn][band][0][i];
                    s2 += tmp[turn][band][1][i];
                }
            }
            s1 = a.mean ? s1 * inv : 0.0f;
            s2 *= inv;
            if (r < a.rows) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float xf[V], df[V], wf[V];
                    Fmt<DT>::unpack(x.c[i], xf);
                    Fmt<DT>::unpack(d.c[i], df);
                    if (a.w)
                        Fmt<DT>::unpack(w.c[i], wf);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float n = (xf[j] - m) * rs, g = a.w ? df[j] * wf[j] : df[j];
                        df[j] = rs * (g - s1 - n * s2);
                    }
                    R::store(a.dx + r * a.lddx, i, l, cols, df);
                }
            }
        }
        if constexpr (kAhead) {
            x = x1;
            d = d1;
            m = m1;
            rs = rs1;
        } else {
            fetch(r + step, x, d, m, rs);
        }
    }
    if (!a.part)
        return;
    // the bands' sums, halving the bands each time
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* s = which ? sb : sw;
#pragma unroll
        for (int h = kRows / 2; h > 0; h >>= 1) {
            __syncthreads();
            if (band >= h && band < 2 * h) {
#pragma unroll
                for (int i = 0; i < NV * V / 4; ++i)
                    sum[band - h][i][l] = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
            }
            __syncthreads();
            if (band < h) {
#pragma unroll
                for (int i = 0; i < NV * V / 4; ++i) {
                    const float4 v = sum[band][i][l];
                    s[4 * i] += v.x;
                    s[4 * i + 1] += v.y;
                    s[4 * i + 2] += v.z;
                    s[4 * i + 3] += v.w;
                }
            }
        }
        if (band == 0) {  // pitch covers whole chunks: the columns past the last one hold zeros
            float* p = a.part + ((int64_t)blockIdx.x * 2 + which) * a.pitch;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int at = (i * TPR + l) * V;
                if (at < cols)
#pragma unroll
                    for (int j = 0; j < V; j += 4)
                        *reinterpret_cast<float4*>(p + at + j) =
                            make_float4(s[i * V + j], s[i * V + j + 1], s[i * V + j + 2], s[i * V + j + 3]);
            }
        }
    }
}

// Sum of n partial rows, `next` floats apart: 32 columns by 32 parts of the
// rows per workgroup.  blockIdx.y picks the output, whose rows start y * pitch in.
template <int DT>
__global__ __launch_bounds__(1024) void k_sum_rows(const float* part, int n, int64_t next, int64_t pitch, int64_t cols,
                                                   typename Elem<DT>::T* o0, typename Elem<DT>::T* o1)
{
    __shared__ float t[32][33];
    typename Elem<DT>::T* out = blockIdx.y ? o1 : o0;
    if (!out)
        return;
    const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
    const int64_t at = (int64_t)blockIdx.x * 32 + c;
    float s = 0.0f;
    if (at < cols)
        for (int k = g; k < n; k += 32)
            s += part[k * next + blockIdx.y * pitch + at];
    t[g][c] = s;
    __syncthreads();
    s = t[c][g];  // the parts of column g
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        s += __shfl_xor(s, o, 32);
    if (c == 0 && (int64_t)blockIdx.x * 32 + g < cols)
        out[(int64_t)blockIdx.x * 32 + g] = (typename Elem<DT>::T)s;
}

// Rows longer than the one-pass kernel holds (over 16384 columns): dx, a
// workgroup per row, which reads x and dy twice; the column sums read them once
// more.  RMS norm, all gradients: 1000 x 18944 fp32 97 us, 2048 x 18944 bf16 176 us.
template <int DT>
__global__ __launch_bounds__(1024) void k_norm_back_long(NormBackArgs<DT> a)
{
    using T = typename Elem<DT>::T;
    __shared__ float tmp[2][16];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = a.x + r * a.ldx, *dy = a.dy + r * a.lddy;
        const float m = a.mean ? a.mean[r] : 0.0f, rs = a.rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = (float)dy[c] * (a.w ? (float)a.w[c] : 1.0f);
            s1 += g;
            s2 = fmaf(g, ((float)x[c] - m) * rs, s2);
        }
        s1 = row_sum<1024>(s1, tmp[0]) / (float)a.cols;
        s2 = row_sum<1024>(s2, tmp[1]) / (float)a.cols;
        if (!a.mean)
            s1 = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = (float)dy[c] * (a.w ? (float)a.w[c] : 1.0f);
            a.dx[r * a.lddx + c] = (T)(rs * (g - s1 - ((float)x[c] - m) * rs * s2));
        }
        __syncthreads();
    }
}

// and the column sums: a thread per column, a part of the rows per workgroup.
template <int DT>
__global__ __launch_bounds__(256) void k_norm_cols_long(NormBackArgs<DT> a)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols)
        return;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float d = (float)a.dy[r * a.lddy + c];
        sb += d;
        sw = fmaf(d, ((float)a.x[r * a.ldx + c] - (a.mean ? a.mean[r] : 0.0f)) * a.rstd[r], sw);
    }
    a.part[(int64_t)blockIdx.y * 2 * a.pitch + c] = sw;
    a.part[((int64_t)blockIdx.y * 2 + 1) * a.pitch + c] = sb;
}

// ---------------------------------------------------------------- which kernel
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a launch; the kernels loop over the rest

int norm_chunks(int64_t cols, int V) { return (int)((cols + V - 1) / V); }

template <int DT, int TPR, int NV>
void norm_go(const NormArgs<DT>& a, hipStream_t st)
{
    // rows to as few workgroups as `most` allows, as many to each
    constexpr int kT = norm_threads(TPR);
    const int64_t per = kT / TPR, n = (a.rows + per - 1) / per;
    const int64_t most = norm_stays(TPR) ? 256 * 1024 / kT : kMaxGrid;
    const int64_t turns = (n + most - 1) / most;
    hipLaunchKernelGGL((k_norm<DT, TPR, NV>), dim3((unsigned)((n + turns - 1) / turns)), dim3(kT), 0, st, a);
}

template <int DT, int TPR>
void norm_nv(const NormArgs<DT>& a, int nv, hipStream_t st)
{
    switch (nv) {
        case 1: return norm_go<DT, TPR, 1>(a, st);
        case 2: return norm_go<DT, TPR, 2>(a, st);
        case 3: return norm_go<DT, TPR, 3>(a, st);
        default: return norm_go<DT, TPR, 4>(a, st);
    }
}

template <int DT>
hipError_t norm_t(const mp_norm_shape& s, const void* x, const void* w, const void* b, void* y, float* mean,
                  float* rstd, hipStream_t st)
{
    using T = typename Elem<DT>::T;
    NormArgs<DT> a{(const T*)x, (const T*)w, (const T*)b, (T*)y,  mean,  rstd, s.rows, s.ldx,
                   s.ldy,       (int)s.cols, s.eps,       (s.flags & MP_NORM_RMS) != 0};
    const int n = norm_chunks(s.cols, Fmt<DT>::V);
    int tpr = n <= 8 * 4 ? 8 : 64;
    while (tpr >= 64 && n > tpr * 4 && tpr <= 1024)
        tpr *= 2;
    const int nv = (n + tpr - 1) / tpr;
    switch (tpr) {
        case 8: norm_nv<DT, 8>(a, nv, st); break;
        case 64: norm_nv<DT, 64>(a, nv, st); break;
        case 128: norm_nv<DT, 128>(a, nv, st); break;
        case 256: norm_nv<DT, 256>(a, nv, st); break;
        case 512: norm_nv<DT, 512>(a, nv, st); break;
        case 1024: norm_nv<DT, 1024>(a, nv, st); break;
        default:
            hipLaunchKernelGGL(k_norm_long<DT>, dim3((unsigned)(s.rows < kMaxGrid ? s.rows : kMaxGrid)), dim3(1024),
                               0, st, a);
    }
    return hipGetLastError();
}

// Threads per row of the one-pass backward kernel, as few as hold it at 16
// columns each; 24 columns in bf16 where that makes it one wave, whose rows need
// no barrier; 0: longer rows.  16384 bf16 rows of RMS norm in us, one wave and two:
//   1032 columns 41, 52; 1280: 43, 54; 1536: 41, 54
//   1544 columns 50, 56; 1792: 53, 57; 2048: 51, 47 (one wave at 32 columns a thread)
// 24 columns with more waves gain nothing (1001 x 8961 fp32: 38 us with 512
// threads, 33 with 1024).
int back_tpr(int dtype, int64_t cols)
{
    if (cols <= 8 * 16)
        return 8;
    if (dtype == MP_BF16 && cols <= 64 * 24)
        return 64;
    for (int t = 64; t <= 1024; t *= 2)
        if (cols <= t * 16)
            return t;
    return 0;
}

// Workgroups of the backward kernel, one partial row each.
int back_groups(int dtype, int64_t rows, int64_t cols)
{
    const int tpr = back_tpr(dtype, cols);
    if (tpr == 0)
        return (int)(rows < 64 ? rows : 64);
    const int64_t per = back_threads(tpr) / tpr, n = (rows + per - 1) / per, most = tpr == 1024 ? 256 : 512;
    return (int)(n < most ? n : most);
}

int norm_pitch(int64_t cols) { return (int)((cols + 7) / 8 * 8); }

template <int DT, int TPR, int NV>
void back_go(const NormBackArgs<DT>& a, int groups, hipStream_t st)
{
    hipLaunchKernelGGL((k_norm_back<DT, TPR, NV>), dim3(groups), dim3(back_threads(TPR)), 0, st, a);
}

template <int DT, int TPR>
void back_nv(const NormBackArgs<DT>& a, int nv, int groups, hipStream_t st)
{
    if (nv == 1)
        return back_go<DT, TPR, 1>(a, groups, st);
    if constexpr (DT == MP_F32 || TPR == 64)
        if (nv == 3)
            return back_go<DT, TPR, 3>(a, groups, st);
    if constexpr (DT == MP_F32)  // chunks of 4 columns
        if (nv == 4)
            return back_go<DT, TPR, 4>(a, groups, st);
    return back_go<DT, TPR, 2>(a, groups, st);
}

template <int DT>
hipError_t norm_back_t(const mp_norm_shape& s, const void* dy, const void* x, const void* w, const float* mean,
                       const float* rstd, void* dx, int64_t lddx, void* dw, void* db, void* ws, hipStream_t st)
{
    using T = typename Elem<DT>::T;
    const int groups = back_groups(s.dtype, s.rows, s.cols), pitch = norm_pitch(s.cols);
    const bool cols = dw || db;
    NormBackArgs<DT> a{(const T*)dy, (const T*)x, (const T*)w, mean,  rstd, (T*)dx,      cols ? (float*)ws : nullptr,
                       s.rows,       s.ldy,       s.ldx,       lddx,  (int)s.cols, pitch};
    const int tpr = back_tpr(DT, s.cols), n = norm_chunks(s.cols, Fmt<DT>::V);
    if (s.rows > 0) {
        const int nv = tpr ? (n + tpr - 1) / tpr : 0;
        if (tpr == 8)
            back_nv<DT, 8>(a, nv, groups, st);
        else if (tpr == 64)
            back_nv<DT, 64>(a, nv, groups, st);
        else if (tpr == 128)
            back_nv<DT, 128>(a, nv, groups, st);
        else if (tpr == 256)
            back_nv<DT, 256>(a, nv, groups, st);
        else if (tpr == 512)
            back_nv<DT, 512>(a, nv, groups, st);
        else if (tpr == 1024)
            back_nv<DT, 1024>(a, nv, groups, st);
        else {
            // the column sums first: dx may be dy itself
            if (cols)
                hipLaunchKernelGGL(k_norm_cols_long<DT>, dim3((unsigned)((s.cols + 255) / 256), groups), dim3(256), 0,
                                   st, a);
            if (dx)
                hipLaunchKernelGGL(k_norm_back_long<DT>, dim3((unsigned)(s.rows < kMaxGrid ? s.rows : kMaxGrid)),
                                   dim3(1024), 0, st, a);
        }
    }
    if (cols)
        hipLaunchKernelGGL(k_sum_rows<DT>, dim3((unsigned)((s.cols + 31) / 32), 2), dim3(1024), 0, st,
                           (const float*)ws, groups, (int64_t)2 * pitch, (int64_t)pitch, s.cols, (T*)dw, (T*)db);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const mp_norm_shape& s, const void* x, const void* weight, const void* bias, void* y,
                       float* mean, float* rstd, hipStream_t st)
{
    return s.dtype == MP_F32 ? norm_t<MP_F32>(s, x, weight, bias, y, mean, rstd, st)
                             : norm_t<MP_BF16>(s, x, weight, bias, y, mean, rstd, st);
}

hipError_t launch_norm_backward(const mp_norm_shape& s, const void* dy, const void* x, const void* weight,
                                const float* mean, const float* rstd, void* dx, int64_t lddx, void* dweight,
                                void* dbias, void* ws, hipStream_t st)
{
    return s.dtype == MP_F32
               ? norm_back_t<MP_F32>(s, dy, x, weight, mean, rstd, dx, lddx, dweight, dbias, ws, st)
               : norm_back_t<MP_BF16>(s, dy, x, weight, mean, rstd, dx, lddx, dweight, dbias, ws, st);
}

hipError_t launch_sum_rows(int dtype, const float* part, int n, int64_t pitch, int64_t cols, void* out, hipStream_t st)
{
    const dim3 g((unsigned)((cols + 31) / 32), 1);
    if (dtype == MP_F32)
        hipLaunchKernelGGL(k_sum_rows<MP_F32>, g, dim3(1024), 0, st, part, n, pitch, (int64_t)0, cols, (float*)out,
                           nullptr);
    else
        hipLaunchKernelGGL(k_sum_rows<MP_BF16>, g, dim3(1024), 0, st, part, n, pitch, (int64_t)0, cols, (__bf16*)out,
                           nullptr);
    return hipGetLastError();
}

uint64_t norm_ws_bytes(const mp_norm_shape& s)
{
    return 8ull * (uint64_t)back_groups(s.dtype, s.rows, s.cols) * (uint64_t)norm_pitch(s.cols);
}

}  // namespace mp
