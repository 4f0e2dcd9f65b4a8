// Tiled matrix products on the matrix cores, with bias, activation and residual
// applied to the accumulators.
#include "ffn_common.h"
#include "gemm.h"
#include "gemm_edge.h"
#include "mm_few.h"

#include <algorithm>

namespace mp {
namespace {

struct TileArgs {
    const char* a;
    const char* b;
    const char* a_end;  // behind the operands' last elements
    const char* b_end;
    void* c;
    int64_t lda, ldb, ldc;
    int64_t I, J, P;
    int ti, tj;      // tiles along i and j
    int splits;      // parts of p, each k_tiles long but the last
    int k_tiles;     // K tiles of a part
    int whole;       // K tiles, of all of p, that are read in whole chunks
    int64_t pitch;   // of a partial result's rows
    Epi e;
};

enum { EPI_STORE = 0, EPI_FULL = 1, EPI_PART = 2 };

constexpr int kRowBytes = 128;  // of p in a tile: 64 bf16 or 32 fp32

template <int DT, Form F, int BM, int BN>
struct Tile {
    static constexpr int es = Fmt<DT>::esize, V = Fmt<DT>::V, BK = kRowBytes / es;
    static constexpr bool AR = F == Form::TN, BR = F != Form::NT;  // operands whose rows are p
    static constexpr int WJ = BN / 64, kThreads = 2 * WJ * 64;     // waves: 2 along i, WJ along j
    static constexpr int FI = BM / 32, FJ = 4;                     // 16 x 16 pieces of a wave's BM/2 x 64
    static constexpr int kBufA = BM * kRowBytes, kBufB = BN * kRowBytes;
    static constexpr int LA = BM * 8 / kThreads, LB = BN * 8 / kThreads;  // 16-byte chunks per thread
    // K tiles on their way in registers.  One in a 256 x 256 tile, whose K tile
    // takes as long as a trip to memory; where few, small tiles share the chip
    // the trip is what a K tile costs (1.1 us with one set, 128 x 128)
    static constexpr int SETS = BM == 256 ? 1 : BM == 128 ? 2 : 4, UNROLL = SETS < 2 ? 2 : SETS;
};

// Byte offset of a chunk in an operand's LDS tile.  Rows of p side by side: 8
// chunks a row, permuted by bits of the row so that the 8 lanes of a phase
// of ds_read_b128, which read one chunk of 8 rows, meet 8 different chunks of
// the 128 bytes that a cycle serves.  perm: the lanes' rows are 0-3, 16-19,
// .. (see the epilogue), else 16 in a row.
__device__ inline int lds_row(int row, int c, bool perm)
{
    const int key = perm ? (row & 3) | ((row >> 2) & 4) : row & 7;
    return row * kRowBytes + ((c ^ key) << 4);
}
// Rows that are p: bf16 reads 4 rows of 32 bytes per 16 lanes (ds_read_b64_tr_b16),
// fp32 4 rows of 64 bytes per wave: the same idea over 32- and 64-byte pieces.
template <int DT, int CPR>
__device__ inline int lds_col(int k, int c)
{
    return (k * CPR + (DT == MP_BF16 ? c ^ ((k & 3) << 1) : c ^ (((k >> 2) & 3) << 2))) << 4;
}

// The address of a 64-bit base that is the same for the workgroup plus a 32-bit offset per lane.
__device__ inline const char* at32(const char* base, uint32_t off) { return base + off; }

// One operand's part of loading a K tile: which chunks a thread takes, global
// memory to registers, registers to LDS.  Rows past the last repeat it, columns
// of p-rows past the last are whatever follows them: their outputs are
// dropped.  Only p past the end has to be zero, for both operands, which
// concerns the last K tile alone, and the matrix's end must not be passed, which
// concerns the one before it too where p-rows are shorter than a chunk.
template <int DT, int B, int N, int kThreads, bool ROWS, bool PERM, int SETS>
struct Loader {
    static constexpr int es = Fmt<DT>::esize, V = Fmt<DT>::V, BK = kRowBytes / es, CPR = B * es / 16;
    const char* base;   // of the tile's first element at p = 0
    const char* last;   // the matrix's last 16 bytes
    int64_t step;       // bytes from one K tile to the next
    uint32_t off[N];
    uint4 r[SETS][N];

    // p: the operand at the part's first p; first, count: the tile's first row (column) and how many there are
    __device__ inline void init(const char* p, int64_t ld, int64_t first, int64_t count, const char* end)
    {
        last = end - 16;
        if constexpr (!ROWS) {
            base = p + first * ld * es;
            step = kRowBytes;
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const int idx = t * kThreads + threadIdx.x, row = idx >> 3;
                const int64_t left = count - 1 - first;
                off[t] = (uint32_t)((row < left ? row : left) * ld * es) + (idx & 7) * 16;
            }
        } else {
            base = p + first * es;
            step = ld * BK * es;
            const int chunks = (int)((count - first + V - 1) / V < CPR ? (count - first + V - 1) / V : CPR);
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const int idx = t * kThreads + threadIdx.x, c = idx % CPR;
                off[t] = (uint32_t)((idx / CPR) * ld * es) + (c < chunks ? c : chunks - 1) * 16;
            }
        }
    }
    // K tile kt, one of the whole ones, into register set `set`
    __device__ inline void load(int set, int64_t kt)
    {
        const char* p = base + kt * step;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            // as a value that may have changed, the offset stays 32 bits wide and
            // goes into the load; else it is kept as 64 bits, in two registers
            asm volatile("" : "+v"(off[t]));
            r[set][t] = ld16u(at32(p, off[t]));
        }
    }
    // one with edges, from whose first on p has `left` elements
    __device__ inline void load_edge(int set, int64_t kt, int64_t left)
    {
        const char* p = base + kt * step;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int idx = t * kThreads + threadIdx.x;
            r[set][t] = ld16_edge<DT>(at32(p, off[t]), ROWS ? (idx / CPR < left ? V : 0) : left - (idx & 7) * V, last);
        }
    }
    __device__ inline void store(int set, char* lds) const
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int idx = t * kThreads + threadIdx.x;
            const int o = ROWS ? lds_col<DT, CPR>(idx / CPR, idx % CPR) : lds_row(idx >> 3, idx & 7, PERM);
            *reinterpret_cast<uint4*>(lds + o) = r[set][t];
        }
    }
};

// A 16-row piece of an operand for half a K tile (ks), from LDS.
template <int DT, int B, bool ROWS, bool PERM>
__device__ inline uint4 piece(const char* lds, int first, int f, int ks)
{
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    constexpr int CPR = B * Fmt<DT>::esize / 16;
    if constexpr (!ROWS) {
        const int row = PERM ? first + (r >> 2) * 16 + f * 4 + (r & 3) : first + f * 16 + r;
        return *reinterpret_cast<const uint4*>(lds + lds_row(row, ks * 4 + q, PERM));
    } else if constexpr (DT == MP_BF16) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        s16x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = ks * 32 + q * 8 + h * 4 + (r >> 2), col = first + f * 16 + (r & 3) * 4;
            const char* p = lds + lds_col<DT, CPR>(k, col >> 3) + (r & 1) * 8;
            v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
        }
        const uint2 a = __builtin_bit_cast(uint2, v[0]), b = __builtin_bit_cast(uint2, v[1]);
        return make_uint4(a.x, a.y, b.x, b.y);
    } else {
        const int col = first + f * 16 + r;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = *reinterpret_cast<const uint32_t*>(lds + lds_col<DT, CPR>(ks * 16 + q * 4 + e, col >> 2) +
                                                      (col & 3) * 4);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// n adjacent values of a row of T: all of them, or the first `have`.
template <int DT, int N>
__device__ inline void load_n(const void* p, int64_t have, float* f)
{
    using T = typename Elem<DT>::T;
    constexpr int V = Fmt<DT>::V;
    if (have >= N && N >= V) {
#pragma unroll
        for (int i = 0; i < N / V; ++i)
            Fmt<DT>::unpack(ld16u(static_cast<const T*>(p) + i * V), f + i * V);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        f[i] = i < have ? (float)static_cast<const T*>(p)[i] : 0.0f;
}
template <int DT, int N>
__device__ inline void store_n(void* p, int64_t have, const float* f)
{
    using T = typename Elem<DT>::T;
    constexpr int V = Fmt<DT>::V;
    if (have >= N) {
        if constexpr (N >= V) {
#pragma unroll
            for (int i = 0; i < N / V; ++i)
                st16u(static_cast<T*>(p) + i * V, Fmt<DT>::pack(f + i * V));
        } else {  // 4 bf16
            typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
            typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
            const u32x2 v = {Fmt<MP_BF16>::pack2(f[0], f[1]), Fmt<MP_BF16>::pack2(f[2], f[3])};
            *static_cast<u32x2_a2*>(p) = v;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have)
            static_cast<T*>(p)[i] = (T)f[i];
}

// N adjacent outputs of row i from column j on.
template <int DT, int ACT, int N>
__device__ inline void finish(const Epi& e, void* c, int64_t ldc, int64_t i, int64_t j, int64_t have,
                              const float* bias, float* v)
{
    using T = typename Elem<DT>::T;
    if (e.bias)
#pragma unroll
        for (int u = 0; u < N; ++u)
            v[u] += bias[u];
    if (e.z)
        store_n<DT, N>(static_cast<T*>(e.z) + i * e.ldz + j, have, v);
#pragma unroll
    for (int u = 0; u < N; ++u)
        v[u] = act_f<ACT>(v[u]);
    if (e.r) {
        float r[N];
        load_n<DT, N>(static_cast<const T*>(e.r) + i * e.ldr + j, have, r);
#pragma unroll
        for (int u = 0; u < N; ++u)
            v[u] += r[u];
    }
    store_n<DT, N>(static_cast<T*>(c) + i * ldc + j, have, v);
}

// Which tile a workgroup takes.  Workgroups go to the 8 XCDs in turn; each XCD
// gets a run of consecutive tiles, and tiles are numbered down bands of 8 rows
// of tiles, so that the tiles an XCD works on together share panels in its L2.
__device__ inline void which_tile(int id, int n, int ti, int tj, int* i, int* j)
{
    const int xcd = id & 7, pos = id >> 3, q = n >> 3, r = n & 7;
    id = xcd * q + (xcd < r ? xcd : r) + pos;
    const int per = 8 * tj, band = id / per, in = id - band * per;
    const int h = ti - band * 8 < 8 ? ti - band * 8 : 8;
    *i = band * 8 + in % h;
    *j = in / h;
}

template <int DT, Form F, int BM, int BN, int EPI>
__global__ __launch_bounds__((Tile<DT, F, BM, BN>::kThreads), BM == 64 ? 1 : 2) void k_gemm(TileArgs g)
{
    using C = Tile<DT, F, BM, BN>;
    constexpr bool PERM = !C::BR, kPong = BM == 256;
    constexpr bool kShort = BM == 64 && (C::AR || C::BR);  // p-rows shorter than a chunk come here
    __shared__ __attribute__((aligned(16))) char lds[2 * (C::kBufA + C::kBufB)];
    int bi, bj;
    const int tiles = g.ti * g.tj, split = blockIdx.x / tiles;
    which_tile(blockIdx.x - split * tiles, tiles, g.ti, g.tj, &bi, &bj);
    const int64_t i0 = (int64_t)bi * BM, j0 = (int64_t)bj * BN;
    const int wave = (int)uniform_u32(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wi = wave / C::WJ * (BM / 2), wj = wave % C::WJ * 64;
    const int64_t p0 = (int64_t)split * g.k_tiles * C::BK;
    const int64_t pn = g.P - p0 < (int64_t)g.k_tiles * C::BK ? g.P - p0 : (int64_t)g.k_tiles * C::BK;
    const int nk = (int)((pn + C::BK - 1) / C::BK);

    Loader<DT, BM, C::LA, C::kThreads, C::AR, false, C::SETS> la;
    Loader<DT, BN, C::LB, C::kThreads, C::BR, PERM, C::SETS> lb;
    la.init(g.a + p0 * C::es * (C::AR ? g.lda : 1), g.lda, i0, g.I, g.a_end);
    lb.init(g.b + p0 * C::es * (C::BR ? g.ldb : 1), g.ldb, j0, g.J, g.b_end);

    f32x4 acc[C::FI][C::FJ];
#pragma unroll
    for (int f = 0; f < C::FI; ++f)
#pragma unroll
        for (int h = 0; h < C::FJ; ++h)
            acc[f][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // [A of the even K tiles][A of the odd ones][B even][B odd]
    char* const sa = lds;
    char* const sb = lds + 2 * C::kBufA;
    auto half = [&](int buf, int ks) {
        uint4 b[C::FJ];
#pragma unroll
        for (int h = 0; h < C::FJ; ++h)
            b[h] = piece<DT, BN, C::BR, PERM>(sb + buf * C::kBufB, wj, h, ks);
#pragma unroll
        for (int f = 0; f < C::FI; ++f) {
            const uint4 a = piece<DT, BM, C::AR, false>(sa + buf * C::kBufA, wi, f, ks);
#pragma unroll
            for (int h = 0; h < C::FJ; ++h)
                acc[f][h] = mma16<DT>(b[h], a, acc[f][h]);
        }
    };
    // The matrix's last K tile, and where kShort the one before it, have edges
    // and come behind the loop over the tiles below `end`.  There, loads past
    // them repeat the last one, so that no load hangs on a branch: the compiler
    // then counts those in flight and waits for the oldest set alone.
    int end = split == g.splits - 1 ? nk - 1 : nk;
    if constexpr (kShort) {
        const int whole = g.whole - split * g.k_tiles;  // below 0 in a part of edges alone
        end = whole < 0 ? 0 : whole < end ? whole : end;
    }
    auto next = [&](int kt) { return kt < end ? kt : end - 1; };
    // K tile kt is multiplied from one buffer while tile kt + 1 goes from its
    // register set to the other and tile kt + 1 + SETS from memory to that set.
    [[maybe_unused]] auto turn = [&](int kt, int buf, int set) {
        half(buf, 0);
        la.store(set, sa + (buf ^ 1) * C::kBufA);
        lb.store(set, sb + (buf ^ 1) * C::kBufB);
        la.load(set, next(kt + 1 + C::SETS));
        lb.load(set, next(kt + 1 + C::SETS));
        half(buf, 1);
        __syncthreads();
    };
    // The same with the two waves of a SIMD half a turn apart: while one reads
    // its operands from LDS (and moves its part of the next tiles along), the
    // other multiplies, and at the barrier they change over.  Without it the
    // LDS and the matrix cores, each busy 2048 cycles a K tile, took turns.  A
    // buffer is written while neither group reads it: the slower group's last
    // reads of it are a barrier behind the faster one's first write, and the
    // slower one's last write a barrier ahead of the faster one's first read.
    [[maybe_unused]] auto step = [&](int kt, int buf, int ks) {
        uint4 a[C::FI], b[C::FJ];
#pragma unroll
        for (int h = 0; h < C::FJ; ++h)
            b[h] = piece<DT, BN, C::BR, PERM>(sb + buf * C::kBufB, wj, h, ks);
#pragma unroll
        for (int f = 0; f < C::FI; ++f)
            a[f] = piece<DT, BM, C::AR, false>(sa + buf * C::kBufA, wi, f, ks);
        if (ks == 0) {
            la.store(0, sa + (buf ^ 1) * C::kBufA);
            la.load(0, next(kt + 2));
        } else {
            lb.store(0, sb + (buf ^ 1) * C::kBufB);
            lb.load(0, next(kt + 2));
        }
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int f = 0; f < C::FI; ++f)
#pragma unroll
            for (int h = 0; h < C::FJ; ++h)
                acc[f][h] = mma16<DT>(b[h], a[f], acc[f][h]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
    };
    if (end > 0) {
#pragma unroll
        for (int u = 0; u < C::SETS; ++u) {
            la.load(u, next(u));
            lb.load(u, next(u));
        }
        la.store(0, sa);
        lb.store(0, sb);
        la.load(0, next(C::SETS));
        lb.load(0, next(C::SETS));
        __syncthreads();
        int kt = 0;
        if constexpr (kPong) {
            if (wave >= C::kThreads / 128)
                __syncthreads();
            for (; kt + 1 < end; kt += 2) {
                step(kt, 0, 0);
                step(kt, 0, 1);
                step(kt + 1, 1, 0);
                step(kt + 1, 1, 1);
            }
            if (kt < end) {
                step(kt, 0, 0);
                step(kt, 0, 1);
            }
            if (wave < C::kThreads / 128)
                __syncthreads();
        } else {
            for (; kt + C::UNROLL <= end; kt += C::UNROLL)
#pragma unroll
                for (int u = 0; u < C::UNROLL; ++u)
                    turn(kt + u, u & 1, (u + 1) % C::SETS);
#pragma unroll
            for (int u = 0; u < C::UNROLL - 1; ++u)
                if (kt + u < end)
                    turn(kt + u, u & 1, (u + 1) % C::SETS);
        }
    }
    auto edge = [&](int kt) {
        la.load_edge(0, kt, pn - (int64_t)kt * C::BK);
        lb.load_edge(0, kt, pn - (int64_t)kt * C::BK);
        la.store(0, sa);
        lb.store(0, sb);
        __syncthreads();
        half(0, 0);
        half(0, 1);
    };
    if (end < nk)
        edge(end);
    if constexpr (kShort)
        if (end + 1 < nk) {
            __syncthreads();  // the buffer has been read
            edge(end + 1);
        }

    // lane: row i0 + wi + f * 16 + lane % 16, and with PERM 16 adjacent columns
    // (pieces are 4 columns of each of the wave's four 16s), else 4 of each piece
    const int q = lane >> 4;
    constexpr int N = PERM ? 16 : 4;
    constexpr int NG = 16 / N;
#pragma unroll
    for (int gI = 0; gI < NG; ++gI) {
        const int64_t j = j0 + wj + (PERM ? q * 16 : gI * 16 + q * 4);
        const int64_t have = g.J - j;
        if (have <= 0)
            continue;
        float bias[N] = {};
        if (EPI == EPI_FULL && g.e.bias)
            load_n<DT, N>(static_cast<const typename Elem<DT>::T*>(g.e.bias) + j, have, bias);
        auto rows = [&](auto act) {
#pragma unroll
            for (int f = 0; f < C::FI; ++f) {
                const int64_t i = i0 + wi + f * 16 + (lane & 15);
                if (i >= g.I)
                    continue;
                float v[N];
#pragma unroll
                for (int h = 0; h < N / 4; ++h)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        v[h * 4 + u] = acc[f][PERM ? h : gI][u];
                if constexpr (EPI == EPI_FULL) {
                    finish<DT, decltype(act)::value, N>(g.e, g.c, g.ldc, i, j, have, bias, v);
                } else if constexpr (EPI == EPI_STORE) {
                    store_n<DT, N>(static_cast<typename Elem<DT>::T*>(g.c) + i * g.ldc + j, have, v);
                } else {  // rows of whole chunks: nothing past the pitch
                    float* p = static_cast<float*>(g.c) + ((int64_t)split * g.I + i) * g.pitch + j;
#pragma unroll
                    for (int u = 0; u < N; u += 4)
                        if (u < have)
                            *reinterpret_cast<float4*>(p + u) = make_float4(v[u], v[u + 1], v[u + 2], v[u + 3]);
                }
            }
        };
        if constexpr (EPI == EPI_FULL) {
            switch (g.e.act) {
                case MP_ACT_RELU: rows(std::integral_constant<int, MP_ACT_RELU>{}); break;
                case MP_ACT_GELU: rows(std::integral_constant<int, MP_ACT_GELU>{}); break;
                case MP_ACT_GELU_TANH: rows(std::integral_constant<int, MP_ACT_GELU_TANH>{}); break;
                case MP_ACT_SILU: rows(std::integral_constant<int, MP_ACT_SILU>{}); break;
                default: rows(std::integral_constant<int, MP_ACT_NONE>{}); break;
            }
        } else {
            rows(std::integral_constant<int, MP_ACT_NONE>{});
        }
    }
}

// The sum of a split product's parts, and the epilogue: 4 adjacent outputs per thread.
template <int DT>
__global__ __launch_bounds__(256) void k_gemm_join(const float* part, int splits, int64_t pitch, void* c, int64_t ldc,
                                                   int64_t I, int64_t J, Epi e)
{
    using T = typename Elem<DT>::T;
    const int64_t per = pitch / 4, n = I * per;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < n; q += (int64_t)gridDim.x * 256) {
        const int64_t i = q / per, j = (q - i * per) * 4;
        const float* p = part + i * pitch + j;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k0 = 0; k0 < splits; k0 += 4) {  // four loads at once
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = k0 + u < splits ? *reinterpret_cast<const float4*>(p + (int64_t)(k0 + u) * I * pitch)
                                       : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                s.x += v[u].x;
                s.y += v[u].y;
                s.z += v[u].z;
                s.w += v[u].w;
            }
        }
        float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (j + u >= J)
                break;
            float z = v[u];
            if (e.bias)
                z += (float)static_cast<const T*>(e.bias)[j + u];
            if (e.z)
                static_cast<T*>(e.z)[i * e.ldz + j + u] = (T)z;
            z = act_of(e.act, z);
            if (e.r)
                z += (float)static_cast<const T*>(e.r)[i * e.ldr + j + u];
            static_cast<T*>(c)[i * ldc + j + u] = (T)z;
        }
    }
}

// Rows so far apart that the offsets inside a tile pass 32 bits, and operands of
// a few bytes: a 64 x 64 tile
// per workgroup on the vector ALU, 16 steps of p at a time, any strides.
template <int DT>
__global__ __launch_bounds__(256) void k_gemm_any(const typename Elem<DT>::T* a, int64_t ai, int64_t ap,
                                                  const typename Elem<DT>::T* b, int64_t bj, int64_t bp, void* c,
                                                  int64_t ldc, int64_t I, int64_t J, int64_t P, int tj, Epi e)
{
    using T = typename Elem<DT>::T;
    __shared__ float sa[16][65], sb[16][65];
    const int64_t i0 = (int64_t)(blockIdx.x / tj) * 64, j0 = (int64_t)(blockIdx.x % tj) * 64;
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
            z = act_of(e.act, z);
            if (e.r)
                z += (float)static_cast<const T*>(e.r)[i * e.ldr + j];
            static_cast<T*>(c)[i * ldc + j] = (T)z;
        }
}

// ---------------------------------------------------------------- which kernel
struct Choice {
    int tile;     // 256, 128 or 64
    int splits, k_tiles;
    int64_t ti, tj, pitch;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of 256 (bf16) where they give half the CUs one, of 128 where they give
// every CU one, else of 64, with p split into parts of 16 K tiles and more
// (fp32, whose K tile is 2048 cycles of matrix cores: 4) until there are 512
// workgroups: the sum of the parts is a launch and 5 us.
// us at one layer of m x n x k in bf16, by tile (parts):
//   2048 4096 4096: 77-84 (256), 77 (128), 126 (64)
//   1024 4096 4096: 73 (256), 46 (128), 64 (64)
//    512 4096 4096: 40 (128), 32 (64), 43 (64, 2)
//    128 1536 8960: 79 (128), 51 (64), 18 (64, 8)
//    300 1000  700: 11.9 (128), 8.4 (64), 12.0 (64, 2)
// and in fp32 with tiles of 64, parts of 16 and of 4 K tiles at least:
//    777  515 1029: 26, 22
//    300  300 2000: 28, 18
//    128 1536 1536: 25, 19
//     90  200  300: 14.5, 12.1
Choice choose(int dtype, int64_t I, int64_t J, int64_t P)
{
    const int BK = kRowBytes / (dtype == MP_F32 ? 4 : 2);
    const int64_t nk = P > 0 ? ceil_div(P, BK) : 1;
    Choice c{};
    c.tile = dtype == MP_BF16 && ceil_div(I, 256) * ceil_div(J, 256) >= 128 ? 256
             : ceil_div(I, 128) * ceil_div(J, 128) >= 256                  ? 128
                                                                           : 64;
    c.ti = ceil_div(I, c.tile);
    c.tj = ceil_div(J, c.tile);
    int64_t s = 1;
    if (c.tile == 64) {
        const int64_t want = 512 / (c.ti * c.tj), most = nk / (dtype == MP_F32 ? 4 : 16);
        s = want < most ? want : most;
        s = s > 1 ? s : 1;
    }
    c.k_tiles = (int)ceil_div(nk, s);
    c.splits = (int)ceil_div(nk, c.k_tiles);
    c.pitch = (J + 3) / 4 * 4;
    return c;
}

// Bytes from an operand's first element to behind its last.
int64_t span(const Gemm& g, bool a)
{
    const bool rows = a ? g.form == Form::TN : g.form != Form::NT;  // its rows are p
    const int64_t free = a ? g.I : g.J, n = rows ? g.P : free, cols = rows ? free : g.P;
    return n == 0 || cols == 0 ? 0 : ((n - 1) * (a ? g.lda : g.ldb) + cols) * (g.dtype == MP_F32 ? 4 : 2);
}

// K tiles that both operands' loads may take whole.
int64_t whole_of(const Gemm& g)
{
    const int V = g.dtype == MP_F32 ? 4 : 8, BK = kRowBytes / (g.dtype == MP_F32 ? 4 : 2);
    int64_t n = whole_k_tiles(g.P, V, V, V, BK);  // operands of rows of p: all but the last
    if (g.form == Form::TN)
        n = std::min(n, whole_k_tiles(g.P, g.I, g.lda, V, BK));
    if (g.form != Form::NT)
        n = std::min(n, whole_k_tiles(g.P, g.J, g.ldb, V, BK));
    return n;
}

// The tiled kernel takes 32-bit offsets inside a tile, and operands of 16 bytes at least.
bool untiled(const Gemm& g)
{
    const int64_t lim = (int64_t)1 << 31, es = g.dtype == MP_F32 ? 4 : 2;
    return g.lda * es * 256 >= lim || g.ldb * es * 256 >= lim || span(g, true) < 16 || span(g, false) < 16;
}

template <int DT, Form F, int B, int EPI>
void tile_go(const TileArgs& t, hipStream_t st)
{
    using C = Tile<DT, F, B, B>;
    hipLaunchKernelGGL((k_gemm<DT, F, B, B, EPI>), dim3((unsigned)(t.ti * t.tj * t.splits)), dim3(C::kThreads), 0, st,
                       t);
}

template <int DT, Form F>
hipError_t gemm_go(const Gemm& g, const Choice& c, void* ws, hipStream_t st)
{
    const char *a = (const char*)g.a, *b = (const char*)g.b;
    TileArgs t{a,
               b,
               a + span(g, true),
               b + span(g, false),
               g.c,
               g.lda,
               g.ldb,
               g.ldc,
               g.I,
               g.J,
               g.P,
               (int)c.ti,
               (int)c.tj,
               c.splits,
               c.k_tiles,
               (int)whole_of(g),
               c.pitch,
               g.epi};
    constexpr int kEpi = F == Form::NT ? EPI_FULL : EPI_STORE;
    if (c.splits > 1) {
        t.c = ws;
        tile_go<DT, F, 64, EPI_PART>(t, st);
        const int64_t n = ceil_div(g.I * c.pitch / 4, 256);
        hipLaunchKernelGGL(k_gemm_join<DT>, dim3((unsigned)(n < 4096 ? n : 4096)), dim3(256), 0, st, (const float*)ws,
                           c.splits, c.pitch, g.c, g.ldc, g.I, g.J, g.epi);
    } else if (c.tile == 256) {
        if constexpr (DT == MP_BF16)
            tile_go<DT, F, 256, kEpi>(t, st);
    } else if (c.tile == 128) {
        tile_go<DT, F, 128, kEpi>(t, st);
    } else {
        tile_go<DT, F, 64, kEpi>(t, st);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t gemm_d(const Gemm& g, void* ws, hipStream_t st)
{
    using T = typename Elem<DT>::T;
    if (untiled(g)) {
        const bool ar = g.form == Form::TN, br = g.form != Form::NT;
        const int64_t ti = ceil_div(g.I, 64), tj = ceil_div(g.J, 64);
        hipLaunchKernelGGL(k_gemm_any<DT>, dim3((unsigned)(ti * tj)), dim3(256), 0, st, (const T*)g.a,
                           ar ? 1 : g.lda, ar ? g.lda : 1, (const T*)g.b, br ? 1 : g.ldb, br ? g.ldb : 1, g.c, g.ldc,
                           g.I, g.J, g.P, (int)tj, g.epi);
        return hipGetLastError();
    }
    Choice c = choose(DT, g.I, g.J, g.P);
    if (whole_of(g) + 1 < ceil_div(g.P, kRowBytes / Fmt<DT>::esize)) {
        // p-rows shorter than a chunk (three columns at most): larger tiles would be
        // nearly empty, and their kernels know one K tile with edges.  Whether p is
        // split stays as it was, and so does the workspace.
        c.tile = 64;
        c.ti = ceil_div(g.I, 64);
        c.tj = ceil_div(g.J, 64);
    }
    switch (g.form) {
        case Form::NT: return gemm_go<DT, Form::NT>(g, c, ws, st);
        case Form::NN: return gemm_go<DT, Form::NN>(g, c, ws, st);
        default: return gemm_go<DT, Form::TN>(g, c, ws, st);
    }
}

}  // namespace

hipError_t launch_gemm(const Gemm& g, void* ws, hipStream_t st)
{
    return g.dtype == MP_F32 ? gemm_d<MP_F32>(g, ws, st) : gemm_d<MP_BF16>(g, ws, st);
}

uint64_t gemm_ws_bytes(int dtype, int64_t I, int64_t J, int64_t P)
{
    const Choice c = choose(dtype, I, J, P);
    return c.splits > 1 ? 4ull * (uint64_t)c.splits * (uint64_t)I * (uint64_t)c.pitch : 0;
}

}  // namespace mp
