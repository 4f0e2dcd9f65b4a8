// Attention of one new token per row over a paged cache of keys and values.
//
// One pass over the keys with a running maximum and sum.  A workgroup of four
// waves takes a chunk of one row's keys for one head of the cache and up to 16
// (or 32) of the query heads that share it, on the matrix cores:
//   S^T (keys x heads) = K Q^T      a lane's scores belong to one query head
//   O^T (dims x heads) += V^T P^T   and so do its outputs,
// so that the softmax needs no data of other lanes but the maximum's, and P
// goes from the accumulators of the first product straight into the operand of
// the second: the order of keys within a product is free, and is taken as the
// first product leaves them.  V^T's operand is formed in registers too: a lane
// holds the same 8 dims of 8 keys, as 16-byte chunks, and turns them with byte
// permutes.  No key or value passes through LDS.
//
// Bound by memory: every key and value is read once, by a group of 16 lanes
// each 16-byte chunks of a row.  A chunk is as long as makes about 1024 of
// equal work of the whole call, whatever the lengths are, so that ragged rows
// fill the chip evenly; the parts of a row are joined by a second kernel.
#include <algorithm>

#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTarget = 1024;   // chunks that a call is divided into, about
constexpr int kMinTiles = 4;    // tiles of a chunk at least: one for each wave

// Quotients of n < 2^31 by a divisor the host knows: with 2^(L-1) < d <= 2^L and
// m = ceil(2^(31+L) / d), n m / 2^(31+L) exceeds n / d by less than
// n / 2^31 / d < 1 / d, so that their whole parts agree.
struct Div {
    uint32_t m = 0, shift = 0;
    Div(uint32_t by = 1)
    {
        uint32_t L = 0;
        while (((uint64_t)1 << L) < by)
            ++L;
        shift = 31 + L;
        m = (uint32_t)((((uint64_t)1 << shift) + by - 1) / by);
    }
    __device__ inline uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

struct AttendArgs {
    const char* k;
    const char* v;
    const void* q;
    const int32_t* table;
    const int32_t* lens;
    void* out;
    float* lse;   // or null
    int2* split;  // [rows]: first slot and parts of a row in more than one chunk, else parts 0 or 1
    float2* stat;  // [slots][heads of a unit]: maximum (log2) and sum
    float* part;   // [slots][heads of a unit][dim]: sums relative to it
    int64_t pages, page_stride, slot_stride, head_stride, ldq, ldo, ldt;  // elements
    int64_t window;
    int32_t most;  // keys that a table row has room for
    int32_t rows, page_size, heads, group, dim;
    int32_t tiles_of_group;  // head tiles of the query heads that share a head of the cache
    int32_t unit_heads;      // query heads of a unit, at most
    Div by_page;
    float scale;  // times log2(e)
};

// A lane's keys of a row: [lo, n).
struct Range {
    int32_t lo, n;
};
__device__ inline Range range_of(const AttendArgs& a, int row)
{
    const int32_t len = a.lens[row];
    const int32_t n = len < 0 ? 0 : len < a.most ? len : a.most;
    return {n > a.window ? n - (int32_t)a.window : 0, n};
}
template <int KT>
__device__ inline int32_t tiles_of(Range r)
{
    return r.n > r.lo ? (r.n + KT - 1) / KT - r.lo / KT : 0;
}

// Which chunk of which row a workgroup takes.
struct Unit {
    int row, chunk, chunks, slot;  // slot: of the row's first chunk
};

// Chunk number `at` of all rows' chunks, counted in the order of the rows.  A row
// of t tiles has max(1, ceil(t / C)) of them, C so that there are about kTarget
// units of it.  False if there are fewer chunks.
template <int KT>
__device__ inline bool find_unit(const AttendArgs& a, uint32_t at, uint32_t per_chunk, Unit* out)
{
    __shared__ uint64_t sums[4];
    __shared__ Unit found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t total = 0;
    int32_t first = 0;
    for (int r = tid; r < a.rows; r += 256) {
        const int32_t t = tiles_of<KT>(range_of(a, r));
        first = r == tid ? t : first;
        total += (uint32_t)t;
    }
    if (a.rows > 1) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1)
            total += __shfl_xor(total, o);
        if (lane == 0)
            sums[wave] = total;
        if (tid == 0)
            found.row = -1;
        __syncthreads();
        total = sums[0] + sums[1] + sums[2] + sums[3];
    } else {
        total = (uint32_t)tiles_of<KT>(range_of(a, 0));
    }
    const uint64_t even = (total * per_chunk + kTarget - 1) / kTarget;
    const uint32_t C = even < kMinTiles ? kMinTiles : even < 0x7fffffff ? (uint32_t)even : 0x7fffffffu;
    if (a.rows == 1) {
        const uint32_t c = max(1u, ((uint32_t)total + C - 1) / C);
        *out = {0, (int)at, (int)c, 0};
        return at < c;
    }
    // chunks in the low half, slots of split rows in the high half
    uint64_t before = 0;
    for (int r0 = 0; r0 < a.rows; r0 += 256) {
        const int r = r0 + tid;
        const uint32_t t = r0 == 0 ? first : r < a.rows ? tiles_of<KT>(range_of(a, r)) : 0;
        const uint32_t c = r < a.rows ? max(1u, (t + C - 1) / C) : 0;
        const uint64_t own = c | (uint64_t)(c > 1 ? c : 0) << 32;
        uint64_t scan = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint64_t up = __shfl_up(scan, o);
            scan += lane >= o ? up : 0;
        }
        __syncthreads();  // sums is read
        if (lane == 63)
            sums[wave] = scan;
        __syncthreads();
        uint64_t mine = before + scan - own;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mine += w < wave ? sums[w] : 0;
            before += sums[w];
        }
        const uint32_t lo = (uint32_t)mine;
        if (c != 0 && at >= lo && at - lo < c)
            found = {r, (int)(at - lo), (int)c, (int)(mine >> 32)};
        if (at < (uint32_t)before)  // the same in every thread
            break;
    }
    __syncthreads();
    *out = found;
    return out->row >= 0;
}

// ---------------------------------------------------------------- chunks of rows
// PAGES: how a tile's rows are found and read.
enum { kWhole = 0, kEven = 1, kOdd = 2 };
// kWhole: pages hold whole groups of 16 keys and heads fill the registers'
// dims, so that a group's address is one for the wave.  kEven: any page size,
// heads of whole 16-byte chunks.  kOdd: any heads.

// N (8 or 16) bytes at p, d elements in a row of dim elements; elements past it are 0.
template <int DT, int PAGES, int N>
__device__ inline uint4 ld_dims(const char* row, int d, int dim)
{
    constexpr int es = Fmt<DT>::esize, E = N / es;
    typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
    typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
    const auto whole = [](const char* p) -> uint4 {
        if constexpr (N == 16)
            return ld16u(p);
        const u32x2_t v = *reinterpret_cast<const u32x2_a2*>(p);
        return make_uint4(v.x, v.y, 0, 0);
    };
    if constexpr (PAGES == kWhole) {
        return whole(row + d * es);
    } else if constexpr (PAGES == kEven) {
        const uint4 c = whole(row + (d < dim ? d : 0) * es);
        return d < dim ? c : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (d + j < dim) {
                if constexpr (DT == MP_F32)
                    w[j] = reinterpret_cast<const uint32_t*>(row)[d + j];
                else
                    w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[d + j] << (16 * (j & 1));
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ inline uint32_t word(const uint4& c, int i) { return i == 0 ? c.x : i == 1 ? c.y : i == 2 ? c.z : c.w; }

// Maximum over the four lanes that hold a query head.
__device__ inline float quad_max(float p)
{
    typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
    u32x2_t w = __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(p), false, false);
    p = fmaxf(__uint_as_float(w.x), __uint_as_float(w.y));
    w = __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(p), false, false);
    return fmaxf(__uint_as_float(w.x), __uint_as_float(w.y));
}
__device__ inline float quad_sum(float p)
{
    typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
    u32x2_t w = __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(p), false, false);
    p = __uint_as_float(w.x) + __uint_as_float(w.y);
    w = __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(p), false, false);
    return __uint_as_float(w.x) + __uint_as_float(w.y);
}

__device__ inline f32x4 mfma_bf16(uint4 a, uint4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// Two bf16 values, 0 in the place of one that is not finite.
__device__ inline uint32_t finite2(uint32_t w)
{
    w = (w & 0x7f80u) == 0x7f80u ? w & 0xffff0000u : w;
    return (w & 0x7f800000u) == 0x7f800000u ? w & 0xffffu : w;
}

// DP: dims that the registers hold (64, 128, 256); HT: tiles of 16 query heads.
// Lane l = 16 g + m.  First product: m is a key of a group of 16 (operand A) and
// a query head (B), dims 4 V s + V g + e of step s.  Its result: query head m,
// keys 4 g + r.  Second product: m is a dim (A) and the query head (B).
template <int DT, int DP, int HT, int PAGES>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a)
{
    constexpr bool kBf16 = DT == MP_BF16;
    constexpr int es = Fmt<DT>::esize, V = Fmt<DT>::V;
    constexpr int KG = kBf16 ? 2 : 1, KT = 16 * KG;  // groups of 16 keys, keys of a tile
    constexpr int S = DP / (4 * V);                  // steps of the first product
    constexpr int W = kBf16 && DP >= 128 ? 8 : 4;    // adjacent dims of a lane
    constexpr int NC = DP / (16 * W);                // chunks of them: dims 16 W c + W m + j
    constexpr int WB = W * es;                       // their bytes, 8 or 16
    constexpr int PD = DP + 4;                       // a head's outputs in LDS, off the banks of the next head's

    __shared__ float sm[4][16 * HT], sl[4][16 * HT];
    __shared__ float4 so[4 * 16 * HT * PD / 4];

    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t per_chunk = (uint32_t)(a.heads * a.tiles_of_group);
    const uint32_t at = blockIdx.x / per_chunk, ht = blockIdx.x - at * per_chunk;
    Unit u;
    if (!find_unit<KT>(a, at, per_chunk, &u))
        return;
    // the same in all lanes, which the compiler is told: addresses then are the wave's
    u.row = __builtin_amdgcn_readfirstlane(u.row);
    u.chunk = __builtin_amdgcn_readfirstlane(u.chunk);
    u.chunks = __builtin_amdgcn_readfirstlane(u.chunks);
    u.slot = __builtin_amdgcn_readfirstlane(u.slot);
    const int kvh = (int)ht / a.tiles_of_group, gh0 = ((int)ht - kvh * a.tiles_of_group) * 16 * HT;
    const int nh = min(a.group - gh0, 16 * HT);  // query heads of this unit
    const Range r = range_of(a, u.row);
    // the row's tiles, divided evenly
    const int tiles = tiles_of<KT>(r), tile0 = r.lo / KT;
    const int begin = tile0 + (int)((int64_t)tiles * u.chunk / u.chunks);
    const int end = tile0 + (int)((int64_t)tiles * (u.chunk + 1) / u.chunks);
    if (u.chunk == 0 && ht == 0 && tid == 0 && a.split != nullptr)
        a.split[u.row] = make_int2(u.slot, u.chunks);

    // the query heads' operand
    uint4 q[HT][S];
#pragma unroll
    for (int h = 0; h < HT; ++h) {
        const char* qp = static_cast<const char*>(a.q) +
                         (u.row * a.ldq + (int64_t)(kvh * a.group + gh0 + (16 * h + m < nh ? 16 * h + m : 0)) * a.dim) * es;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const uint4 c = ld_dims<DT, PAGES, 16>(qp, 4 * V * s + V * g, a.dim);
            q[h][s] = 16 * h + m < nh ? c : make_uint4(0, 0, 0, 0);
        }
    }

    const int32_t* table = a.table + u.row * a.ldt;
    const int64_t head_off = (int64_t)kvh * a.head_stride;

    // Pages of this wave's tiles (begin + wave + 4 i): lane 2 i + j (i with one
    // group a tile) holds that of group j of tile i, 64 / KG tiles ahead.  -1: no
    // key of the group counts.
    const auto pages_from = [&](int tile) -> int32_t {
        const int t = tile + 4 * (lane / KG), key = t * KT + 16 * (lane % KG);
        int32_t p = -1;
        if (t < end && key < r.n) {
            p = table[a.by_page.of((uint32_t)key)];
            p = (uint64_t)(int64_t)p < (uint64_t)a.pages ? p : -1;
        }
        return p;
    };

    uint4 kr[KG][S], vr[4 * KG][NC];
    uint32_t seen = 0;  // kWhole: bit j: group j's page is there; else bit 4 j + r: key 4 g + r of group j
    const uint32_t k_off = (uint32_t)(m * (int32_t)a.slot_stride + V * g) * es;
    const uint32_t v_off = (uint32_t)(4 * g * (int32_t)a.slot_stride + W * m) * es;
    // where a key lies, for pages that end anywhere; -1: nowhere
    const auto key_at = [&](int key) -> int64_t {
        if (key >= r.n || key < r.lo)
            return -1;
        const uint32_t p = a.by_page.of((uint32_t)key);
        const int64_t page = table[p];
        if ((uint64_t)page >= (uint64_t)a.pages)
            return -1;
        return page * a.page_stride + (int64_t)(key - (int32_t)(p * (uint32_t)a.page_size)) * a.slot_stride + head_off;
    };
    const auto group_at = [&](int key, int32_t page) -> int64_t {
        const int32_t slot = key - (int32_t)(a.by_page.of((uint32_t)key) * (uint32_t)a.page_size);
        return ((int64_t)page * a.page_stride + (int64_t)slot * a.slot_stride + head_off) * es;
    };
    const auto load_k = [&](int tile, const int32_t* pg) {
#pragma unroll
        for (int j = 0; j < KG; ++j) {
            if constexpr (PAGES == kWhole) {
                const char* base = a.k + group_at(tile * KT + 16 * j, pg[j] < 0 ? 0 : pg[j]);
#pragma unroll
                for (int s = 0; s < S; ++s)
                    kr[j][s] = ld16u(base + k_off + 4 * V * es * s);
            } else {
                const int64_t p = key_at(tile * KT + 16 * j + m);
                const char* row = a.k + (p < 0 ? 0 : p) * es;
#pragma unroll
                for (int s = 0; s < S; ++s)
                    kr[j][s] = ld_dims<DT, PAGES, 16>(row, 4 * V * s + V * g, a.dim);
            }
        }
    };
    const auto load_v = [&](int tile, const int32_t* pg) {
        seen = 0;
#pragma unroll
        for (int j = 0; j < KG; ++j) {
            if constexpr (PAGES == kWhole) {
                seen |= pg[j] < 0 ? 0u : 1u << j;
                const char* base = a.v + group_at(tile * KT + 16 * j, pg[j] < 0 ? 0 : pg[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        vr[4 * j + i][c] = ld_dims<DT, kWhole, WB>(base + i * a.slot_stride * es + v_off, 16 * W * c, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t p = key_at(tile * KT + 16 * j + 4 * g + i);
                    seen |= p < 0 ? 0u : 1u << (4 * j + i);
                    const char* row = a.v + (p < 0 ? 0 : p) * es;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        vr[4 * j + i][c] = ld_dims<DT, PAGES, WB>(row, 16 * W * c + W * m, a.dim);
                }
            }
        }
    };

    f32x4 o[HT][NC * W];
    float top[HT], sum[HT];
    constexpr int kAhead = 64 / KG;  // tiles whose pages a wave holds
    int32_t held, next = 0;
    const auto page_of = [&](int i, int32_t* pg) {
#pragma unroll
        for (int j = 0; j < KG; ++j)
            pg[j] = PAGES == kWhole ? __builtin_amdgcn_readlane(held, i * KG + j) : 0;
    };
    // In bf16 an infinite value gives NaN with p's remainder, which may be 0 or
    // negative.  A wave that ends with NaN goes through its keys once more, now
    // leaving values that are not finite out of the remainder's product.
    bool again = false;
pass:
#pragma unroll
    for (int h = 0; h < HT; ++h) {
        top[h] = -INFINITY;
        sum[h] = 0.0f;
#pragma unroll
        for (int j = 0; j < NC * W; ++j)
            o[h][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    held = PAGES == kWhole ? pages_from(begin + wave) : 0;
    int32_t pg[KG];
    page_of(0, pg);
    if (begin + wave < end)
        load_k(begin + wave, pg);
    int i = 0;
    for (int tile = begin + wave; tile < end; tile += 4) {
        if (PAGES == kWhole && i == 0)
            next = pages_from(tile + 4 * kAhead);
        load_v(tile, pg);
        // scores
        f32x4 s[HT][KG];
#pragma unroll
        for (int h = 0; h < HT; ++h)
#pragma unroll
            for (int j = 0; j < KG; ++j) {
                s[h][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < S; ++t) {
                    if constexpr (kBf16) {
                        s[h][j] = mfma_bf16(kr[j][t], q[h][t], s[h][j]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(kr[j][t], e)),
                                                                          __uint_as_float(word(q[h][t], e)), s[h][j], 0,
                                                                          0, 0);
                    }
                }
            }
        // the next tile's keys, in the registers that these left
        if (++i == kAhead) {
            i = 0;
            held = next;
        }
        page_of(i, pg);
        const uint32_t have = seen;
        if (tile + 4 < end)
            load_k(tile + 4, pg);
        // masks: keys outside [lo, n) and of pages that are not there
        const bool full = PAGES == kWhole && tile * KT >= r.lo && tile * KT + KT <= r.n && have == (1u << KG) - 1;
        uint32_t in = (1u << (4 * KG)) - 1;  // bit 4 j + r: key 4 g + r of group j
        if (!full) {
            if constexpr (PAGES == kWhole) {
                in = 0;
#pragma unroll
                for (int j = 0; j < KG; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = tile * KT + 16 * j + 4 * g + e;
                        in |= (have >> j & 1) != 0 && key >= r.lo && key < r.n ? 1u << (4 * j + e) : 0u;
                    }
            } else {
                in = have;
            }
            // what lies there may be NaN, which p = 0 would not hide
#pragma unroll
            for (int e = 0; e < 4 * KG; ++e)
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    if (!(in >> e & 1))
                        vr[e][c] = make_uint4(0, 0, 0, 0);
        }
        float p[HT][4 * KG];
#pragma unroll
        for (int h = 0; h < HT; ++h) {
            float best = top[h];
#pragma unroll
            for (int e = 0; e < 4 * KG; ++e) {
                const float x = s[h][e / 4][e % 4] * a.scale;
                p[h][e] = in >> e & 1 ? x : -INFINITY;
                best = fmaxf(best, p[h][e]);
            }
            best = quad_max(best);
            if (__any(best > top[h])) {
                const float keep = best > top[h] ? __builtin_amdgcn_exp2f(top[h] - best) : 1.0f;
                sum[h] *= keep;
#pragma unroll
                for (int j = 0; j < NC * W; ++j)
                    o[h][j] *= keep;
                top[h] = best;
            }
            const float zero = best == -INFINITY ? 0.0f : best;  // no score above -inf yet
#pragma unroll
            for (int e = 0; e < 4 * KG; ++e) {
                p[h][e] = __builtin_amdgcn_exp2f(p[h][e] - zero);
                sum[h] += p[h][e];
            }
        }
        // outputs
        if constexpr (kBf16) {
            uint4 hi[HT], lo[HT];
#pragma unroll
            for (int h = 0; h < HT; ++h) {
                float f[8], back[8];
                hi[h] = Fmt<DT>::pack(p[h]);
                Fmt<DT>::unpack(hi[h], back);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    f[e] = p[h][e] - back[e];
                lo[h] = Fmt<DT>::pack(f);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int w = 0; w < W / 2; ++w)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        // dim 2 w + half of the lane's chunk, keys in pairs
                        const uint32_t sel = half ? 0x07060302u : 0x05040100u;
                        uint4 t;
                        t.x = __builtin_amdgcn_perm(word(vr[1][c], w), word(vr[0][c], w), sel);
                        t.y = __builtin_amdgcn_perm(word(vr[3][c], w), word(vr[2][c], w), sel);
                        t.z = __builtin_amdgcn_perm(word(vr[5][c], w), word(vr[4][c], w), sel);
                        t.w = __builtin_amdgcn_perm(word(vr[7][c], w), word(vr[6][c], w), sel);
#pragma unroll
                        for (int h = 0; h < HT; ++h)
                            o[h][c * W + 2 * w + half] = mfma_bf16(t, hi[h], o[h][c * W + 2 * w + half]);
                        if (again)
                            t = make_uint4(finite2(t.x), finite2(t.y), finite2(t.z), finite2(t.w));
#pragma unroll
                        for (int h = 0; h < HT; ++h)
                            o[h][c * W + 2 * w + half] = mfma_bf16(t, lo[h], o[h][c * W + 2 * w + half]);
                    }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int h = 0; h < HT; ++h)
                            o[h][c * W + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(vr[e][c], j)),
                                                                                  p[h][e], o[h][c * W + j], 0, 0, 0);
        }
    }

    if constexpr (kBf16)
        if (!again) {
            bool nan = false;
#pragma unroll
            for (int h = 0; h < HT; ++h)
#pragma unroll
                for (int j = 0; j < NC * W; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        nan |= 16 * h + m < nh && o[h][j][e] != o[h][j][e];
            if (__any(nan)) {
                again = true;
                goto pass;
            }
        }

    // The four waves' parts, in LDS.
#pragma unroll
    for (int h = 0; h < HT; ++h) {
        sum[h] = quad_sum(sum[h]);
        if (g == 0) {
            sm[wave][16 * h + m] = top[h];
            sl[wave][16 * h + m] = sum[h];
        }
    }
    __syncthreads();
    float all_top[HT], all_sum[HT];
#pragma unroll
    for (int h = 0; h < HT; ++h) {
        float t = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            t = fmaxf(t, sm[w][16 * h + m]);
        const float zero = t == -INFINITY ? 0.0f : t;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            l += sl[w][16 * h + m] * __builtin_amdgcn_exp2f(sm[w][16 * h + m] - zero);
        all_top[h] = t;
        all_sum[h] = l;
        const float f = __builtin_amdgcn_exp2f(top[h] - zero);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < W; j += 4)
                    so[((wave * 16 * HT + 16 * h + m) * PD + 16 * W * c + W * (4 * g + e) + j) / 4] =
                        make_float4(o[h][c * W + j][e] * f, o[h][c * W + j + 1][e] * f, o[h][c * W + j + 2][e] * f,
                                    o[h][c * W + j + 3][e] * f);
    }
    // the sums of all waves, for the threads that write the outputs
    __syncthreads();
    if (wave == 0 && g == 0)
#pragma unroll
        for (int h = 0; h < HT; ++h) {
            sm[0][16 * h + m] = all_top[h];
            sl[0][16 * h + m] = all_sum[h];
        }
    __syncthreads();
    const float* sof = reinterpret_cast<const float*>(so);
    const auto total_of = [&](int h, int d) {
        return sof[h * PD + d] + sof[(16 * HT + h) * PD + d] + sof[(32 * HT + h) * PD + d] +
               sof[(48 * HT + h) * PD + d];
    };
    const int64_t head0 = (int64_t)kvh * a.group + gh0;
    using T = typename Elem<DT>::T;
    if (u.chunks == 1) {
        T* out = static_cast<T*>(a.out) + u.row * a.ldo + head0 * a.dim;
        for (int d = tid % DP, h = tid / DP; h < nh; h += 256 / DP)
            if (d < a.dim) {
                const float l = sl[0][h];
                out[h * a.dim + d] = (T)(l == 0.0f ? 0.0f : total_of(h, d) / l);
            }
        if (a.lse != nullptr && tid < nh) {
            const float l = sl[0][tid];
            a.lse[u.row * (int64_t)(a.heads * a.group) + head0 + tid] =
                l == 0.0f ? -INFINITY : (sm[0][tid] + __builtin_amdgcn_logf(l)) * 0.693147180559945f;
        }
        return;
    }
    const int64_t slot = (int64_t)(u.slot + u.chunk) * per_chunk + ht;
    float* part = a.part + slot * a.unit_heads * a.dim;
    for (int d = tid % DP, h = tid / DP; h < nh; h += 256 / DP)
        if (d < a.dim)
            part[h * a.dim + d] = total_of(h, d);
    if (tid < nh)
        a.stat[slot * a.unit_heads + tid] = make_float2(sm[0][tid], sl[0][tid]);
}

// A workgroup per row and query head joins the row's parts: sums relative to the
// largest of their maxima.
template <int DT>
__global__ __launch_bounds__(256) void k_join(AttendArgs a)
{
    const uint32_t heads = (uint32_t)(a.heads * a.group);
    const int row = (int)(blockIdx.x / heads), head = (int)(blockIdx.x - (uint32_t)row * heads);
    const int2 split = a.split[row];
    if (split.y <= 1)
        return;
    const int tid = threadIdx.x, kvh = head / a.group, gh = head - kvh * a.group;
    const uint32_t per_chunk = (uint32_t)(a.heads * a.tiles_of_group);
    const int ht = kvh * a.tiles_of_group + gh / a.unit_heads, h = gh % a.unit_heads;
    // part c of the row is slot0 + c * per_chunk
    const int64_t slot0 = (int64_t)split.x * per_chunk + ht;
    const auto stat = [&](int c) { return a.stat[(slot0 + (int64_t)c * per_chunk) * a.unit_heads + h]; };
    __shared__ float tmp[8];
    __shared__ float acc[256];
    float t = -INFINITY;
    for (int c = tid; c < split.y; c += 256)
        t = fmaxf(t, stat(c).x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t = fmaxf(t, __shfl_xor(t, o));
    if ((tid & 63) == 0)
        tmp[tid >> 6] = t;
    __syncthreads();
    t = fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
    const float zero = t == -INFINITY ? 0.0f : t;
    float l = 0.0f;
    for (int c = tid; c < split.y; c += 256) {
        const float2 s = stat(c);
        l += s.y * __builtin_amdgcn_exp2f(s.x - zero);
    }
    l = wave_xor_sum(l);
    if ((tid & 63) == 0)
        tmp[4 + (tid >> 6)] = l;
    __syncthreads();
    l = tmp[4] + tmp[5] + tmp[6] + tmp[7];
    // `lanes` threads side by side on the dims, the others on further parts
    const int lanes = a.dim <= 64 ? 64 : a.dim <= 128 ? 128 : 256, groups = 256 / lanes;
    const int d = tid % lanes, first = tid / lanes;
    float sum = 0.0f;
    if (d < a.dim)
        for (int c = first; c < split.y; c += groups)
            sum += a.part[((slot0 + (int64_t)c * per_chunk) * a.unit_heads + h) * a.dim + d] *
                   __builtin_amdgcn_exp2f(stat(c).x - zero);
    acc[tid] = sum;
    __syncthreads();
    using T = typename Elem<DT>::T;
    if (first == 0 && d < a.dim) {
        for (int i = 1; i < groups; ++i)
            sum += acc[i * lanes + d];
        static_cast<T*>(a.out)[row * a.ldo + (int64_t)head * a.dim + d] = (T)(l == 0.0f ? 0.0f : sum / l);
    }
    if (a.lse != nullptr && tid == 0)
        a.lse[(int64_t)row * heads + head] = l == 0.0f ? -INFINITY : (t + __builtin_amdgcn_logf(l)) * 0.693147180559945f;
}

// ---------------------------------------------------------------- the host's side
struct Plan {
    int ht = 1, tile = 32;
    int64_t per_chunk = 1, units = 0, slots = 0, unit_heads = 1;
    bool joins = false;
};

Plan plan_of(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    Plan p;
    const int64_t group = s.q_heads / c.heads;
    p.tile = c.dtype == MP_F32 ? 16 : 32;
    p.ht = group > 16 && c.head_dim <= 128 ? 2 : 1;
    const int64_t tiles_of_group = (group + 16 * p.ht - 1) / (16 * p.ht);
    p.per_chunk = c.heads * tiles_of_group;
    p.unit_heads = std::min<int64_t>(group, 16 * p.ht);
    int64_t most = s.width * c.page_size;
    if (s.window > 0 && s.window < most)
        most = s.window;
    const int64_t tiles = (most + p.tile - 1) / p.tile + 1;  // a window may begin inside a tile
    // chunks of C tiles: rows * per_chunk of them for the rows' first, and as many more as kTarget
    p.joins = (s.window > 0 ? tiles : tiles - 1) > kMinTiles;
    p.units = s.rows * p.per_chunk;
    if (p.joins) {
        const int64_t longest = (tiles + kMinTiles - 1) / kMinTiles;  // chunks of a row
        p.units = std::min(p.units + kTarget, p.units * longest);
        // a row of more than one chunk has less than twice its tiles' share of kTarget
        p.slots = std::min<int64_t>(2 * kTarget + 2 * p.per_chunk, p.units);
    }
    return p;
}

uint64_t up16(uint64_t n) { return (n + 15) / 16 * 16; }

template <int DT, int DP>
void launch_dims(const AttendArgs& a, const Plan& p, int pages, hipStream_t st)
{
    const unsigned grid = (unsigned)p.units;
    if constexpr (DP <= 128)
        if (p.ht == 2) {
            if (pages == kWhole)
                k_attend<DT, DP, 2, kWhole><<<grid, 256, 0, st>>>(a);
            else if (pages == kEven)
                k_attend<DT, DP, 2, kEven><<<grid, 256, 0, st>>>(a);
            else
                k_attend<DT, DP, 2, kOdd><<<grid, 256, 0, st>>>(a);
            return;
        }
    if (pages == kWhole)
        k_attend<DT, DP, 1, kWhole><<<grid, 256, 0, st>>>(a);
    else if (pages == kEven)
        k_attend<DT, DP, 1, kEven><<<grid, 256, 0, st>>>(a);
    else
        k_attend<DT, DP, 1, kOdd><<<grid, 256, 0, st>>>(a);
}

template <int DT>
void launch_type(const AttendArgs& a, const Plan& p, hipStream_t st)
{
    const int dp = a.dim <= 64 ? 64 : a.dim <= 128 ? 128 : 256;
    const int pages = a.dim % Fmt<DT>::V != 0 ? kOdd : a.dim == dp && a.page_size % 16 == 0 ? kWhole : kEven;
    if (dp == 64)
        launch_dims<DT, 64>(a, p, pages, st);
    else if (dp == 128)
        launch_dims<DT, 128>(a, p, pages, st);
    else
        launch_dims<DT, 256>(a, p, pages, st);
    if (p.joins)
        k_join<DT><<<(unsigned)(a.rows * a.heads * a.group), 256, 0, st>>>(a);
}

}  // namespace

uint64_t kv_attend_ws_bytes(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    const Plan p = plan_of(c, s);
    if (s.rows == 0 || !p.joins)
        return 0;
    const uint64_t heads = (uint64_t)(p.slots * p.unit_heads);
    return up16((uint64_t)s.rows * sizeof(int2)) + up16(heads * sizeof(float2)) +
           heads * (uint64_t)c.head_dim * sizeof(float);
}

hipError_t launch_kv_attend(const mp_kv_cache& c, const mp_kv_attend_shape& s, const void* q, const int32_t* table,
                            const int32_t* lens, void* out, float* lse, void* ws, hipStream_t st)
{
    const Plan p = plan_of(c, s);
    AttendArgs a{};
    a.k = static_cast<const char*>(c.k);
    a.v = static_cast<const char*>(c.v);
    a.q = q;
    a.table = table;
    a.lens = lens;
    a.out = out;
    a.lse = lse;
    if (p.joins) {
        char* w = static_cast<char*>(ws);
        a.split = reinterpret_cast<int2*>(w);
        w += up16((uint64_t)s.rows * sizeof(int2));
        a.stat = reinterpret_cast<float2*>(w);
        w += up16((uint64_t)(p.slots * p.unit_heads) * sizeof(float2));
        a.part = reinterpret_cast<float*>(w);
    }
    a.pages = c.pages;
    a.page_stride = c.pages > 1 ? c.page_stride : 0;
    a.slot_stride = c.page_size > 1 ? c.slot_stride : 0;
    a.head_stride = c.heads > 1 ? c.head_stride : 0;
    a.ldq = s.ldq;
    a.ldo = s.ldo;
    a.ldt = s.ldt;
    a.window = s.window ? s.window : INT64_MAX;
    a.most = c.pages ? (int32_t)(s.width * c.page_size) : 0;  // without pages there are no keys
    a.rows = (int32_t)s.rows;
    a.page_size = (int32_t)c.page_size;
    a.heads = (int32_t)c.heads;
    a.group = (int32_t)(s.q_heads / c.heads);
    a.dim = (int32_t)c.head_dim;
    a.tiles_of_group = (int32_t)(p.per_chunk / c.heads);
    a.unit_heads = (int32_t)p.unit_heads;
    a.by_page = Div((uint32_t)c.page_size);
    a.scale = (float)((double)s.scale * 1.4426950408889634);
    if (c.dtype == MP_F32)
        launch_type<MP_F32>(a, p, st);
    else
        launch_type<MP_BF16>(a, p, st);
    return hipGetLastError();
}

}  // namespace mp
