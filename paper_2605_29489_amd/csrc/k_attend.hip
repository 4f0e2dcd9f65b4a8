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
#include <type_traits>

#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMinTiles = 4;  // tiles of a share at least: one for each wave
constexpr int kMostShares = 768;

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
    int2* split;   // [rows][head sets]: first share and parts of what is in more than one share, else parts 1
    float2* stat;  // [slots][head tiles of a workgroup][unit_heads]: maximum (log2) and sum
    float* part;   // [slots][head tiles of a workgroup][unit_heads][dim]: sums relative to it
    int64_t page_stride, head_stride, ldq, ldo, ldt;  // elements
    int64_t window;
    uint32_t pages;
    int32_t slot_stride;
    int32_t most;  // keys that a table row has room for
    int32_t rows, page_size, heads, group, dim;
    int32_t tiles_of_group;  // head tiles of the query heads that share a head of the cache
    int32_t unit_heads;      // query heads of a head tile, at most
    int32_t split_waves;     // waves of a workgroup that share a head tile's keys: 1, 2 or 4
    int32_t head_sets;       // workgroups that the head tiles of a row take
    int32_t shares;          // 0: a workgroup per row and head set
    Div by_page, by_tiles;  // by_tiles: tiles_of_group
    float scale;  // times log2(e)
};

// A lane's keys of a row: [lo, n).
struct Range {
    int32_t lo, n;
};
__device__ inline Range range_of(const AttendArgs& a, int row)
{
    // the kernel writes no length: read so, a wave's own row comes through the scalar cache
    const int32_t len = *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
        reinterpret_cast<uintptr_t>(a.lens + row));
    const int32_t n = len < 0 ? 0 : len < a.most ? len : a.most;
    return {n > a.window ? n - (int32_t)a.window : 0, n};
}
template <int KT>
__device__ inline int32_t tiles_of(Range r)
{
    return r.n > r.lo ? (r.n + KT - 1) / KT - r.lo / KT : 0;
}

// Every row counts for a tile at least, so that one without keys is someone's.
template <int KT>
__device__ inline uint32_t work_of(const AttendArgs& a, int row)
{
    return max(1, tiles_of<KT>(range_of(a, row)));
}

// The call's tiles are the sequence (row, head set, tile), and a share is a run
// of it, of `per` tiles from `at` on; it begins in `row`, whose first tile is at
// row_at.
struct Share {
    uint64_t at, end, row_at;
    uint32_t per;
    int row;
};

// False where the shares before hold everything.
template <int KT>
__device__ inline bool find_share(const AttendArgs& a, uint32_t number, Share* out)
{
    __shared__ uint64_t sums[4];
    __shared__ uint64_t found_at;
    __shared__ int found_row;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t sets = (uint32_t)a.head_sets;
    uint64_t total = 0;
    uint32_t first = 0;
    for (int r = tid; r < a.rows; r += 256) {
        const uint32_t t = work_of<KT>(a, r);
        first = r == tid ? t : first;
        total += t;
    }
    if (a.rows > 1) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1)
            total += __shfl_xor(total, o);
        if (lane == 0)
            sums[wave] = total;
        __syncthreads();
        total = sums[0] + sums[1] + sums[2] + sums[3];
    } else {
        total = work_of<KT>(a, 0);
    }
    const uint64_t all = total * sets, even = (all + a.shares - 1) / (uint32_t)a.shares;
    out->per = even < kMinTiles ? (uint32_t)kMinTiles : even < 0x7fffffff ? (uint32_t)even : 0x7fffffffu;
    out->at = (uint64_t)number * out->per;
    out->end = min(all, out->at + out->per);
    out->row = 0;
    out->row_at = 0;
    if (out->at >= all)
        return false;
    if (a.rows == 1)
        return true;
    // the row r with before(r) <= at / sets < before(r + 1)
    const uint64_t at = out->at / sets;
    uint64_t before = 0;
    for (int r0 = 0; r0 < a.rows; r0 += 256) {
        const int r = r0 + tid;
        const uint32_t own = r0 == 0 ? first : r < a.rows ? work_of<KT>(a, r) : 0;
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
        if (at >= mine && at - mine < own) {
            found_row = r;
            found_at = mine * sets;
        }
        if (at < before)  // the same in every thread
            break;
    }
    __syncthreads();
    out->row = found_row;
    out->row_at = found_at;
    return true;
}

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline uint64_t uniform(uint64_t x)
{
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// ---------------------------------------------------------------- shares of the tiles
// MODE: how keys and values are found and read.
enum { kWhole = 0, kRows = 1, kEven = 2, kOdd = 3 };
// kWhole: pages hold whole groups of 16 keys, so that a group's address is one
// for the wave, and heads fill the registers' dims.  kRows: the same pages, heads
// of at least a 16-byte chunk.  kEven: any page size.  kOdd: any heads as well.

// Workgroups that a CU's registers hold.
constexpr int resident(int dp, int ht) { return dp * ht <= 64 ? 3 : dp * ht <= 128 ? 2 : 1; }

// The chunk at dim d of a row of few dims, one value at a time, zeros behind it.
template <int DT>
__device__ inline uint4 ld16_few(const char* row, int d, int dim)
{
    return d < dim ? ld16_head<DT>(row + d * Fmt<DT>::esize, dim - d) : make_uint4(0, 0, 0, 0);
}

// N (8 or 16) bytes of a row of values.  A load instruction takes whole rows of
// up to 256 bytes, which no other reads, so that they need not stay in the
// caches; rows of keys are read in pieces of 64 bytes by several, and do.  64
// rows of up to 8192 keys: 211 us without non-temporal loads, 193 with them for
// the values, 192 for both; rows of 128 bytes: 86.6, 86.8 and 88.5 us.
template <int N>
__device__ inline uint4 ld_values(const char* p)
{
    if constexpr (N == 16) {
        const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p));
        return make_uint4(v.x, v.y, v.z, v.w);
    } else {
        typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
        typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
        const u32x2_t v = *reinterpret_cast<const u32x2_a2*>(p);
        return make_uint4(v.x, v.y, 0, 0);
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

// W dims of an output.
template <int DT, int W>
__device__ inline void st_dims(void* p, const float* x)
{
    if constexpr (DT == MP_F32) {
        st16u(p, Fmt<DT>::pack(x));
    } else if constexpr (W == 8) {
        st16u(p, Fmt<DT>::pack(x));
    } else {
        typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
        typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
        *static_cast<u32x2_a2*>(p) = u32x2_t{Fmt<DT>::pack2(x[0], x[1]), Fmt<DT>::pack2(x[2], x[3])};
    }
}

// log of a sum l relative to 2^t.
__device__ inline float lse_of(float t, float l)
{
    return l == 0.0f ? -INFINITY : (t + __builtin_amdgcn_logf(l)) * 0.693147180559945f;
}

// DP: dims that the registers hold (64, 128, 256); HT: tiles of 16 query heads.
// Lane l = 16 g + m.  First product: m is a key of a group of 16 (operand A) and
// a query head (B), dims 4 V s + V g + e of step s.  Its result: query head m,
// keys 4 g + r.  Second product: m is a dim (A) and the query head (B).
//
// A wave's loads run ahead of it, from one row's tiles into the next row's: keys
// are asked for when the first product is done with those before, values when
// the second is, and pages of the cache a tile before that, through the scalar
// cache.  (Under load a trip to memory takes some 4 us; a row's start would be
// three, one after the other.)  No branch lies around these loads, so that a
// wait for keys leaves the values behind them in flight, and the other way
// round; at a share's end they fetch its last tile again, from the caches.
template <int DT, int DP, int HT, int MODE>
__global__ __launch_bounds__(256, resident(DP, HT)) void k_attend(AttendArgs a)
{
    constexpr bool kBf16 = DT == MP_BF16, kUni = MODE == kWhole || MODE == kRows;
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
    const int wave = uniform(tid >> 6);
    const uint32_t head_tiles = (uint32_t)(a.heads * a.tiles_of_group), sets = (uint32_t)a.head_sets;
    const int step = a.split_waves, wt = 4 / step;  // head tiles of a workgroup
    // the wave's place among those that share its head tile
    const int mine = wave / step, place = wave % step;

    // The tiles of one row and head set that a share takes.
    struct Run {
        int row;
        uint32_t set, off, n_tiles, work;  // the first one's number, how many, and how many the row has
        int lo, n;                         // the row's keys
        int begin, end;                    // this wave's tiles, `step` apart
    };
    const auto run_of = [&](int row, uint32_t set, uint32_t off, uint32_t left, Range keys) {
        Run r;
        r.row = row;
        r.set = set;
        r.off = off;
        r.work = max(1, tiles_of<KT>(keys));
        r.n_tiles = min(r.work - off, left);
        r.lo = keys.lo;
        r.n = keys.n;
        const int tile0 = keys.lo / KT + (int)off;
        r.begin = tile0 + place;
        // no tiles: a row without keys, and a head tile that is not there
        r.end = set * wt + mine >= head_tiles || keys.n <= keys.lo ? r.begin : tile0 + (int)r.n_tiles;
        return r;
    };
    // The run behind r, if `left` tiles of the share lie behind it.
    const auto behind = [&](const Run& r, uint32_t left) {
        if (r.set + 1 < sets)
            return run_of(r.row, r.set + 1, 0, left, Range{r.lo, r.n});
        return run_of(r.row + 1, 0, 0, left, range_of(a, r.row + 1));
    };
    // Head tile of a set for this wave: head of the cache, first query head of it, query heads.
    struct Heads {
        int kvh, gh0, nh;
    };
    const auto heads_of = [&](uint32_t tile) {
        Heads h;
        h.kvh = (int)a.by_tiles.of(tile);
        h.gh0 = ((int)tile - h.kvh * a.tiles_of_group) * 16 * HT;
        h.nh = min(a.group - h.gh0, 16 * HT);
        return h;
    };

    Run cur;
    uint32_t left, before = 0, per = 0;  // tiles of the share from cur on, and before it; tiles of a share
    if (a.shares == 0) {
        const int row = (int)(blockIdx.x / sets);
        cur = run_of(row, blockIdx.x - (uint32_t)row * sets, 0, 0x7fffffff, range_of(a, row));
        left = cur.n_tiles;
    } else {
        Share share;
        if (!find_share<KT>(a, blockIdx.x, &share))
            return;
        // the same in all lanes, which the compiler is told: addresses then are the wave's
        per = (uint32_t)uniform((int)share.per);
        left = (uint32_t)uniform((int)(uint32_t)(share.end - share.at));
        const uint64_t in = uniform(share.at - share.row_at);
        const int row = uniform(share.row);
        const Range keys = range_of(a, row);
        const uint32_t work = max(1, tiles_of<KT>(keys)), set = (uint32_t)(in / work);
        cur = run_of(row, set, (uint32_t)(in - (uint64_t)set * work), left, keys);
    }

    // The tile that is loaded next.
    struct Cursor {
        Run run;
        uint32_t left;
        int tile;
        bool none;  // behind the share's last one, at which it stays
    };
    const auto seek = [&](Cursor& c) {  // from a run's end to the next tile
        Run r = c.run;
        uint32_t n = c.left;
        do {
            n -= r.n_tiles;
            if (n == 0) {
                c.none = true;
                return;
            }
            r = behind(r, n);
        } while (r.begin >= r.end);
        c.run = r;
        c.left = n;
        c.tile = r.begin;
    };
    const auto advance = [&](Cursor& c) {
        if (c.none)
            return;
        if (c.tile + step < c.run.end)
            c.tile += step;
        else
            seek(c);
    };

    uint4 q[HT][S], kr[KG][S], vr[4 * KG][NC];
    // where a lane's chunks begin in a head, and the dims of a chunk that the one before holds: with heads that do
    // not fill the registers the last chunks lie over each other
    const auto chunk_at = [&](int s) {
        const int d = 4 * V * s + V * g;
        return MODE == kWhole ? d : min(d, max(a.dim - V, 0));
    };
    const auto clear = [&](uint4 c, int s) {
        if constexpr (MODE != kRows && MODE != kEven)
            return c;
        constexpr int bits = 8 * es;
        const int drop = (4 * V * s + V * g - chunk_at(s)) * bits;
        const auto keep = [&](int w) { return drop <= 32 * w ? ~0u : drop >= 32 * w + 32 ? 0u : ~0u << (drop - 32 * w); };
        return make_uint4(c.x & keep(0), c.y & keep(1), c.z & keep(2), c.w & keep(3));
    };
    const auto value_at = [&](int c, int mm) {
        const int d = 16 * W * c + W * mm;
        return MODE == kWhole || MODE == kOdd ? d : min(d, a.dim - W);
    };
    const auto load_q = [&](const Run& r) {
        const Heads hd = heads_of(r.set * wt + mine);
#pragma unroll
        for (int h = 0; h < HT; ++h) {
            // heads that are not there take the last one's place: their results are not used
            const char* qp = static_cast<const char*>(a.q) +
                             (r.row * a.ldq + (int64_t)(hd.kvh * a.group + hd.gh0 + min(16 * h + m, hd.nh - 1)) * a.dim) * es;
#pragma unroll
            for (int s = 0; s < S; ++s)
                q[h][s] = MODE == kOdd ? ld16_few<DT>(qp, 4 * V * s + V * g, a.dim) : ld16u(qp + chunk_at(s) * es);
        }
    };

    // kUni: the pages of a tile's groups; else the page of a lane's key (lane % KT).  Not looked at before their use.
    int32_t page[kUni ? KG : 1];
    const auto load_pages = [&](const Cursor& c) {
        const int32_t* table = a.table + c.run.row * a.ldt;
        if constexpr (kUni) {
#pragma unroll
            for (int j = 0; j < KG; ++j)
                page[j] = *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(
                    table + a.by_page.of((uint32_t)min(c.tile * KT + 16 * j, c.run.n - 1))));
        } else {
            page[0] = table[a.by_page.of((uint32_t)min(c.tile * KT + lane % KT, c.run.n - 1))];
        }
    };
    const uint32_t row_bytes = (uint32_t)a.slot_stride * es;
    uint32_t seen = 0, seen_next = 0;  // kUni: bit j: group j's page is there; else bit 4 j + r: key 4 g + r of it
    int64_t where[KG];  // kUni: the groups' offsets; else where[0]: that of the lane's key, -1 if it does not count
    const auto load_k = [&](const Cursor& c) {
        const int64_t head = heads_of(c.run.set * wt + mine).kvh * a.head_stride * es;
        if constexpr (kUni) {
            seen_next = 0;
#pragma unroll
            for (int j = 0; j < KG; ++j) {
                const int key = c.tile * KT + 16 * j;
                const bool there = key < c.run.n && (uint32_t)page[j] < a.pages;
                const int32_t slot = key - (int32_t)(a.by_page.of((uint32_t)key) * (uint32_t)a.page_size);
                seen_next |= there ? 1u << j : 0u;
                where[j] = (there ? page[j] : 0) * (a.page_stride * es) + (int64_t)slot * row_bytes + head;
                const char* base = a.k + where[j];
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if constexpr (MODE == kWhole)
                        kr[j][s] = ld16u(base + (uint32_t)(m * row_bytes + V * g * es) + 4 * V * es * s);
                    else
                        kr[j][s] = ld16u(base + (uint32_t)(m * row_bytes + chunk_at(s) * es));
            }
        } else {
            const int key = c.tile * KT + lane % KT;
            const int32_t slot = key - (int32_t)(a.by_page.of((uint32_t)key) * (uint32_t)a.page_size);
            const bool there = key >= c.run.lo && key < c.run.n && (uint32_t)page[0] < a.pages;
            where[0] = there ? page[0] * (a.page_stride * es) + (int64_t)slot * row_bytes + head : -1;
#pragma unroll
            for (int j = 0; j < KG; ++j) {
                const char* row = a.k + max((int64_t)__shfl(where[0], 16 * j + m), (int64_t)0);
#pragma unroll
                for (int s = 0; s < S; ++s)
                    kr[j][s] = MODE == kOdd ? ld16_few<DT>(row, 4 * V * s + V * g, a.dim) : ld16u(row + chunk_at(s) * es);
            }
        }
    };
    const auto load_v = [&]() {
        if constexpr (kUni) {
            seen = seen_next;
#pragma unroll
            for (int j = 0; j < KG; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        if constexpr (MODE == kWhole)
                            vr[4 * j + e][c] = ld_values<WB>(a.v + where[j] + e * (int64_t)row_bytes +
                                                             (uint32_t)(4 * g * row_bytes + WB * m) + 16 * WB * c);
                        else
                            vr[4 * j + e][c] = ld_values<WB>(a.v + where[j] + e * (int64_t)row_bytes +
                                                             (uint32_t)(4 * g * row_bytes + value_at(c, m) * es));
        } else {
            seen = 0;
#pragma unroll
            for (int j = 0; j < KG; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t p = __shfl(where[0], 16 * j + 4 * g + e);
                    seen |= p < 0 ? 0u : 1u << (4 * j + e);
                    const char* row = a.v + max(p, (int64_t)0);
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        if constexpr (MODE == kOdd)
                            vr[4 * j + e][c] = ld16_few<DT>(row, 16 * W * c + W * m, min(a.dim, 16 * W * c + W * m + W));
                        else
                            vr[4 * j + e][c] = ld_values<WB>(row + value_at(c, m) * es);
                }
        }
    };

    Cursor ahead;
    const auto begin_at = [&]() {
        ahead = Cursor{cur, left, cur.begin, false};
        if (cur.begin >= cur.end)
            seek(ahead);
        if (ahead.none)
            return;
        load_pages(ahead);
        load_q(ahead.run);
        load_k(ahead);
        advance(ahead);
        load_pages(ahead);
        load_v();
    };
    begin_at();

    for (;;) {
        const bool whole = cur.n_tiles == cur.work;
        if (cur.off == 0 && tid == 0 && a.split != nullptr)
            a.split[(int64_t)cur.row * sets + cur.set] =
                make_int2((int)blockIdx.x, whole ? 1 : (int)((before + cur.work - 1) / per) + 1);

        f32x4 o[HT][NC * W];
        float top[HT], sum[HT];
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
        for (int tile = cur.begin; tile < cur.end; tile += step) {
            if (MODE != kWhole && tile == cur.begin)
#pragma unroll
                for (int h = 0; h < HT; ++h)
#pragma unroll
                    for (int s = 0; s < S; ++s)
                        q[h][s] = clear(q[h][s], s);
            // scores
            f32x4 s[HT][KG];
#pragma unroll
            for (int j = 0; j < KG; ++j) {
#pragma unroll
                for (int h = 0; h < HT; ++h)
                    s[h][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < S; ++t) {
                    const uint4 k = clear(kr[j][t], t);
#pragma unroll
                    for (int h = 0; h < HT; ++h) {
                        if constexpr (kBf16) {
                            s[h][j] = mfma_bf16(k, q[h][t], s[h][j]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                s[h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                    __uint_as_float(word(k, e)), __uint_as_float(word(q[h][t], e)), s[h][j], 0, 0, 0);
                        }
                    }
                }
            }
            if (ahead.tile == ahead.run.begin)  // of another run
                load_q(ahead.run);
            load_k(ahead);
            advance(ahead);
            load_pages(ahead);
            // masks: keys outside [lo, n) and of pages that are not there
            const bool full = kUni && tile * KT >= cur.lo && tile * KT + KT <= cur.n && seen == (1u << KG) - 1;
            uint32_t in = (1u << (4 * KG)) - 1;  // bit 4 j + r: key 4 g + r of group j
            if (!full) {
                if constexpr (kUni) {
                    in = 0;
#pragma unroll
                    for (int j = 0; j < KG; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = tile * KT + 16 * j + 4 * g + e;
                            in |= (seen >> j & 1) != 0 && key >= cur.lo && key < cur.n ? 1u << (4 * j + e) : 0u;
                        }
                } else {
                    in = seen;
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
                                o[h][c * W + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                    __uint_as_float(word(vr[e][c], j)), p[h][e], o[h][c * W + j], 0, 0, 0);
            }
            load_v();
        }
        const Heads hd = heads_of(min(cur.set * wt + mine, head_tiles - 1));
        if constexpr (kBf16)
            if (!again) {
                bool nan = false;
#pragma unroll
                for (int h = 0; h < HT; ++h)
#pragma unroll
                    for (int j = 0; j < NC * W; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            nan |= 16 * h + m < hd.nh && o[h][j][e] != o[h][j][e];
                if (__any(nan)) {
                    again = true;
                    begin_at();
                    goto pass;
                }
            }

        using T = typename Elem<DT>::T;
        // a share holds the end of a row that began before, or the beginning of one that goes on, or both
        const int64_t slot = (2 * (int64_t)blockIdx.x + (cur.off == 0 ? 1 : 0)) * wt;
#pragma unroll
        for (int h = 0; h < HT; ++h)
            sum[h] = quad_sum(sum[h]);
        if (step == 1) {
            // a head tile a wave: from its registers, W dims at a time
            const int64_t head0 = (int64_t)hd.kvh * a.group + hd.gh0, at = (slot + mine) * a.unit_heads;
#pragma unroll
            for (int h = 0; h < HT; ++h) {
                const int head = 16 * h + m;
                if (cur.set * wt + mine >= head_tiles || head >= hd.nh)
                    continue;
                const float r = sum[h] == 0.0f ? 0.0f : whole ? 1.0f / sum[h] : 1.0f;
                T* out = static_cast<T*>(a.out) + cur.row * a.ldo + (head0 + head) * a.dim;
                float* part = a.part + (at + head) * a.dim;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int d = value_at(c, 4 * g + e);
                        float x[W];
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            x[j] = sum[h] == 0.0f ? 0.0f : o[h][c * W + j][e] * r;
                        if (MODE != kOdd && whole)
                            st_dims<DT, W>(out + d, x);
                        else if (MODE == kWhole)
                            for (int j = 0; j < W; j += 4)
                                *reinterpret_cast<float4*>(part + d + j) =
                                    make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                        else
                            for (int j = 0; j < W; ++j)
                                if (MODE != kOdd || d + j < a.dim) {
                                    if (whole)
                                        out[d + j] = (T)x[j];
                                    else
                                        part[d + j] = x[j];
                                }
                    }
                if (g == 0) {
                    if (!whole)
                        a.stat[at + head] = make_float2(top[h], sum[h]);
                    else if (a.lse != nullptr)
                        a.lse[cur.row * (int64_t)(a.heads * a.group) + head0 + head] = lse_of(top[h], sum[h]);
                }
            }
        } else {
            // The waves' parts, in LDS.
#pragma unroll
            for (int h = 0; h < HT; ++h)
                if (g == 0) {
                    sm[wave][16 * h + m] = top[h];
                    sl[wave][16 * h + m] = sum[h];
                }
            __syncthreads();
            float all_top[HT], all_sum[HT];
#pragma unroll
            for (int h = 0; h < HT; ++h) {
                float t = -INFINITY, l = 0.0f;
                for (int w = wave - place; w < wave - place + step; ++w)
                    t = fmaxf(t, sm[w][16 * h + m]);
                const float zero = t == -INFINITY ? 0.0f : t;
                for (int w = wave - place; w < wave - place + step; ++w)
                    l += sl[w][16 * h + m] * __builtin_amdgcn_exp2f(sm[w][16 * h + m] - zero);
                all_top[h] = t;
                all_sum[h] = l;
                const float f = __builtin_amdgcn_exp2f(top[h] - zero);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < W; j += 4) {
                            const int at = (wave * 16 * HT + 16 * h + m) * PD + value_at(c, 4 * g + e) + j;
                            const float4 x = make_float4(o[h][c * W + j][e] * f, o[h][c * W + j + 1][e] * f,
                                                         o[h][c * W + j + 2][e] * f, o[h][c * W + j + 3][e] * f);
                            float* to = reinterpret_cast<float*>(so) + at;
                            if constexpr (MODE == kWhole || MODE == kOdd) {
                                *reinterpret_cast<float4*>(to) = x;
                            } else {  // two lanes may hold a dim, with the same value
                                to[0] = x.x;
                                to[1] = x.y;
                                to[2] = x.z;
                                to[3] = x.w;
                            }
                        }
            }
            __syncthreads();  // sm and sl are read
            if (place == 0 && g == 0)
#pragma unroll
                for (int h = 0; h < HT; ++h) {
                    sm[wave][16 * h + m] = all_top[h];
                    sl[wave][16 * h + m] = all_sum[h];
                }
            __syncthreads();
            // The sums of a head tile's waves, by all threads.
            const float* sof = reinterpret_cast<const float*>(so);
            for (int w = 0; w < 4; w += step) {
                const uint32_t tile = cur.set * wt + w / step;
                if (tile >= head_tiles)
                    break;
                const Heads of = heads_of(tile);
                const int heads = of.nh;
                const int64_t head0 = (int64_t)of.kvh * a.group + of.gh0, at = (slot + w / step) * a.unit_heads;
                T* out = static_cast<T*>(a.out) + cur.row * a.ldo + head0 * a.dim;
                float* part = a.part + at * a.dim;
                for (int d = tid % DP, h = tid / DP; h < heads; h += 256 / DP)
                    if (d < a.dim) {
                        float x = sof[(w * 16 * HT + h) * PD + d];
                        for (int v = w + 1; v < w + step; ++v)
                            x += sof[(v * 16 * HT + h) * PD + d];
                        if (whole) {
                            const float l = sl[w][h];
                            out[h * a.dim + d] = (T)(l == 0.0f ? 0.0f : x / l);
                        } else {
                            part[h * a.dim + d] = x;
                        }
                    }
                if (tid < heads) {
                    const float t = sm[w][tid], l = sl[w][tid];
                    if (!whole)
                        a.stat[at + tid] = make_float2(t, l);
                    else if (a.lse != nullptr)
                        a.lse[cur.row * (int64_t)(a.heads * a.group) + head0 + tid] = lse_of(t, l);
                }
            }
            __syncthreads();  // LDS is read
        }
        left -= cur.n_tiles;
        before += cur.n_tiles;
        if (left == 0)
            return;
        cur = behind(cur, left);
    }
}

// Joins the parts of a row: their sums relative to the largest of their maxima.
// A workgroup takes 4 `lanes` dims of one query head, a float4 a thread, the
// other threads further parts.
template <int DT>
__global__ __launch_bounds__(256) void k_join(AttendArgs a, int lanes)
{
    const uint32_t heads = (uint32_t)(a.heads * a.group);
    const int row = (int)(blockIdx.x / heads), head = (int)(blockIdx.x - (uint32_t)row * heads);
    const int kvh = head / a.group, gh = head - kvh * a.group;
    const int ht = kvh * a.tiles_of_group + gh / a.unit_heads, wt = 4 / a.split_waves;
    const int2 split = a.split[(int64_t)row * a.head_sets + ht / wt];
    const int n = split.y;
    if (n <= 1)
        return;
    __shared__ float weight[kMostShares];
    __shared__ float tmp[8];
    __shared__ float4 acc[256];
    const int tid = threadIdx.x;
    // part c of the row, in the first place of a share but for part 0
    const auto place = [&](int c) {
        return ((2 * (int64_t)(split.x + c) + (c == 0 ? 1 : 0)) * wt + ht % wt) * a.unit_heads + gh % a.unit_heads;
    };
    float t = -INFINITY;
    for (int c = tid; c < n; c += 256)
        t = fmaxf(t, a.stat[place(c)].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t = fmaxf(t, __shfl_xor(t, o));
    if ((tid & 63) == 0)
        tmp[tid >> 6] = t;
    __syncthreads();
    t = fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
    const float zero = t == -INFINITY ? 0.0f : t;
    float l = 0.0f;
    for (int c = tid; c < n; c += 256) {
        const float2 s = a.stat[place(c)];
        const float w = __builtin_amdgcn_exp2f(s.x - zero);
        weight[c] = w;
        l += s.y * w;
    }
    l = wave_xor_sum(l);
    if ((tid & 63) == 0)
        tmp[4 + (tid >> 6)] = l;
    __syncthreads();
    l = tmp[4] + tmp[5] + tmp[6] + tmp[7];
    const int groups = 256 / lanes, mine = tid / lanes, d = (int)(blockIdx.y * lanes + tid % lanes) * 4;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const auto add = [&](float4 v, float w) {
        sum.x += v.x * w;
        sum.y += v.y * w;
        sum.z += v.z * w;
        sum.w += v.w * w;
    };
    const auto part = [&](int c) {
        const float* q = a.part + place(c) * a.dim + d;
        if (a.dim % 4 == 0)
            return *reinterpret_cast<const float4*>(q);
        const int k = a.dim - d;
        return make_float4(q[0], k > 1 ? q[1] : 0.0f, k > 2 ? q[2] : 0.0f, k > 3 ? q[3] : 0.0f);
    };
    if (d < a.dim) {
        int c = mine;
        for (; c + 3 * groups < n; c += 4 * groups) {
            const float4 v0 = part(c), v1 = part(c + groups), v2 = part(c + 2 * groups), v3 = part(c + 3 * groups);
            add(v0, weight[c]);
            add(v1, weight[c + groups]);
            add(v2, weight[c + 2 * groups]);
            add(v3, weight[c + 3 * groups]);
        }
        for (; c < n; c += groups)
            add(part(c), weight[c]);
    }
    acc[tid] = sum;
    // halves onto halves; the number of groups is a power of two
    for (int k = groups / 2; k > 0; k /= 2) {
        __syncthreads();
        if (mine < k) {
            const float4 v = acc[tid + k * lanes];
            add(v, 1.0f);
            acc[tid] = sum;
        }
    }
    using T = typename Elem<DT>::T;
    if (mine == 0 && d < a.dim) {
        T* out = static_cast<T*>(a.out) + row * a.ldo + (int64_t)head * a.dim + d;
        const float x[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < a.dim)
                out[j] = (T)(l == 0.0f ? 0.0f : x[j] / l);
    }
    if (a.lse != nullptr && tid == 0 && blockIdx.y == 0)
        a.lse[(int64_t)row * heads + head] = lse_of(t, l);
}

// ---------------------------------------------------------------- the host's side
struct Plan {
    int ht = 1, split_waves = 4;
    int64_t head_tiles = 1, sets = 1, unit_heads = 1;
    int64_t shares = 0;  // 0: no row is split
};

int split_waves_of(int64_t rows, int64_t head_tiles)
{
    return rows * head_tiles < 256 ? 4 : head_tiles % 4 == 0 ? 1 : head_tiles % 2 == 0 ? 2 : 4;
}

Plan plan_of(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    Plan p;
    const int64_t group = s.q_heads / c.heads, tile = c.dtype == MP_F32 ? 16 : 32;
    p.ht = group > 16 && c.head_dim <= 128 ? 2 : 1;
    p.head_tiles = c.heads * ((group + 16 * p.ht - 1) / (16 * p.ht));
    p.unit_heads = std::min<int64_t>(group, 16 * p.ht);
    p.split_waves = split_waves_of(s.rows, p.head_tiles);
    const int64_t wt = 4 / p.split_waves;
    p.sets = (p.head_tiles + wt - 1) / wt;
    int64_t most = s.width * c.page_size;
    const bool slides = s.window > 0 && s.window < most;
    most = slides ? s.window : most;
    const int64_t tiles = (most + tile - 1) / tile + (slides ? 1 : 0);  // a window may begin inside a tile
    if (tiles > kMinTiles) {
        const int64_t needed = (s.rows * p.sets * tiles + kMinTiles - 1) / kMinTiles;  // < 2^50
        const int dp = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
        p.shares = std::min<int64_t>(256 * resident(dp, p.ht), needed);
    }
    return p;
}

uint64_t up16(uint64_t n) { return (n + 15) / 16 * 16; }
// query heads of all parts: two of a share, of 4 / split_waves head tiles
uint64_t slot_heads(const Plan& p) { return (uint64_t)(2 * p.shares * (4 / p.split_waves) * p.unit_heads); }

template <int DT, int DP, int HT>
void launch_tiles(const AttendArgs& a, unsigned grid, int mode, hipStream_t st)
{
    if (mode == kWhole)
        k_attend<DT, DP, HT, kWhole><<<grid, 256, 0, st>>>(a);
    else if (mode == kRows)
        k_attend<DT, DP, HT, kRows><<<grid, 256, 0, st>>>(a);
    else if (mode == kEven)
        k_attend<DT, DP, HT, kEven><<<grid, 256, 0, st>>>(a);
    else if constexpr (DP == 64)
        k_attend<DT, DP, HT, kOdd><<<grid, 256, 0, st>>>(a);
}

template <int DT>
void launch_type(const AttendArgs& a, const Plan& p, hipStream_t st)
{
    const int dp = a.dim <= 64 ? 64 : a.dim <= 128 ? 128 : 256;
    const int mode = a.dim < Fmt<DT>::V ? kOdd : a.page_size % 16 != 0 ? kEven : a.dim == dp ? kWhole : kRows;
    const unsigned grid = (unsigned)(p.shares ? p.shares : a.rows * p.sets);
    if (dp == 64)
        p.ht == 2 ? launch_tiles<DT, 64, 2>(a, grid, mode, st) : launch_tiles<DT, 64, 1>(a, grid, mode, st);
    else if (dp == 128)
        p.ht == 2 ? launch_tiles<DT, 128, 2>(a, grid, mode, st) : launch_tiles<DT, 128, 1>(a, grid, mode, st);
    else
        launch_tiles<DT, 256, 1>(a, grid, mode, st);
    if (p.shares) {
        // few heads: their dims in slices of 32, so that more workgroups share the parts
        const unsigned heads = (unsigned)(a.rows * a.heads * a.group);
        const int lanes = heads < 512 ? 8 : dp / 4;
        k_join<DT><<<dim3(heads, (unsigned)((a.dim + 4 * lanes - 1) / (4 * lanes))), 256, 0, st>>>(a, lanes);
    }
}

}  // namespace

uint64_t kv_attend_ws_bytes(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    const Plan p = plan_of(c, s);
    if (s.rows == 0 || p.shares == 0)
        return 0;
    return up16((uint64_t)(s.rows * p.sets) * sizeof(int2)) + up16(slot_heads(p) * sizeof(float2)) +
           slot_heads(p) * (uint64_t)c.head_dim * sizeof(float);
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
    if (p.shares) {
        char* w = static_cast<char*>(ws);
        a.split = reinterpret_cast<int2*>(w);
        w += up16((uint64_t)(s.rows * p.sets) * sizeof(int2));
        a.stat = reinterpret_cast<float2*>(w);
        w += up16(slot_heads(p) * sizeof(float2));
        a.part = reinterpret_cast<float*>(w);
    }
    a.pages = (uint32_t)std::min<int64_t>(c.pages, INT32_MAX);  // of those that a table can name
    a.page_stride = c.pages > 1 ? c.page_stride : 0;
    a.slot_stride = c.page_size > 1 ? (int32_t)c.slot_stride : 0;
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
    a.tiles_of_group = (int32_t)(p.head_tiles / c.heads);
    a.split_waves = p.split_waves;
    a.head_sets = (int32_t)p.sets;
    a.shares = (int32_t)p.shares;
    a.unit_heads = (int32_t)p.unit_heads;
    a.by_page = Div((uint32_t)c.page_size);
    a.by_tiles = Div((uint32_t)a.tiles_of_group);
    a.scale = (float)((double)s.scale * 1.4426950408889634);
    if (c.dtype == MP_F32)
        launch_type<MP_F32>(a, p, st);
    else
        launch_type<MP_BF16>(a, p, st);
    return hipGetLastError();
}

}  // namespace mp
