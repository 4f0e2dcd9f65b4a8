// Attention of one new token per row over a paged cache of keys and values.
//
// One pass over the keys with a running maximum and sum.  A wave takes tiles of
// 32 keys (fp32: 16) of one head of the cache for up to 16 (or 32) of the query
// heads that share it, on the matrix cores:
//   S^T (keys x heads) = K Q^T      a lane's scores belong to one query head
//   O^T (dims x heads) += V^T P^T   and so do its outputs,
// so that the softmax needs nothing of other lanes but the maximum, and P goes
// from the accumulators of the first product straight into the operand of the
// second: the order of keys within a product is free, and is taken as the first
// product leaves them.  V^T's operand is formed in registers too: a lane holds
// the same 8 dims of 8 keys, as 16-byte chunks, and turns them with byte
// permutes.  No key or value passes through LDS.
//
// Bound by memory: every key and value is read once.  The keys of all rows are
// divided into as many equal shares as there are CUs, whatever the lengths are,
// so that ragged rows fill the chip evenly; a second kernel joins the parts of a
// row.  bf16, 128 dims: 64 rows of 1 to 8192 keys of 8 heads (1.11 GB) 180 us, 172 of them
// here (6.4 TB/s); the same rows of 4096 keys 173 us; one row of 131072 keys of
// 4 heads (268 MB) 54 us, 6 of them in the second kernel; of the first one's 48 the
// keys take 40 at 6.7 TB/s, 2 pass before the first of them arrives and 3 in joining
// the waves.
#include <algorithm>
#include <type_traits>

#include "ffn_common.h"
#include "mp_internal.h"

namespace mp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Tiles of a share at least.  One row of 4096 or 32768 keys (4 heads of 128 bf16
// dims) 14.8 and 23.8 us, with 2 tiles the same, with 8 16.6 and 25.2; 8 rows of up
// to 300 keys 27.7, with 8 32.2, with 2 14.6, as their shares then are enough for
// equal parts of each row.
constexpr int kMinTiles = 4;
constexpr int kShares = 256;  // one for each CU
// Tiles that the waves of a workgroup are apart at most.  64 ragged rows of up to
// 8192 keys / 256 of up to 700: 180 / 80 us; 1 apart 182 / 81, 4 180 / 81, 8 180 / 81.
constexpr int kInStep = 2;

struct AttendArgs {
    const char* k;
    const char* v;
    const void* q;
    const int32_t* table;
    const int32_t* lens;
    void* out;
    float* lse;   // or null
    int2* split;   // [rows][head tiles]: first share; number of parts, and above them the head tiles of a set
    float2* stat;  // [slots][set_tiles][unit_heads]: maximum (log2) and sum
    float* part;   // [slots][set_tiles][unit_heads][dim]: sums relative to it
    int64_t page_stride, head_stride, ldq, ldo, ldt;  // elements
    int64_t window;
    uint32_t pages;
    int32_t slot_stride;
    int32_t most;  // keys that a table row has room for
    int32_t rows, page_size, heads, group, dim;
    int32_t tiles_of_group;  // head tiles of the query heads that share a head of the cache
    int32_t unit_heads;      // query heads of a head tile, at most
    int32_t set_tiles;       // head tiles of a workgroup, a head set: a power of two; a row's last set may have fewer
    int32_t one_if_few;      // or one, where the call's tiles are few
    int32_t shares;          // 0: a workgroup per row and head set
    Div by_page, by_tiles, by_heads;  // page_size, tiles_of_group, unit_heads
    float scale;  // times log2(e)
};

// A length or a page, which no kernel here writes: where the address is one for
// the wave it comes through the scalar cache.
__device__ inline int32_t ld_constant(const int32_t* p)
{
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p));
}

// The keys of a row: [lo, n).
struct Range {
    int32_t lo, n;
};
__device__ inline Range range_of(const AttendArgs& a, int row)
{
    const int32_t len = ld_constant(a.lens + row);
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
// Where the tiles are few, a run is instead one of the equal parts of a row and
// head set, so that no share holds two: 7 rows of up to 2000 fp32 keys 25.7 us
// cut evenly, 21.3 so.  That is done up to a quarter of the shares in rows and head
// sets: up to an eighth, 16 rows of up to 500 bf16 keys take 28.7 us for 15.9.
struct Share {
    uint64_t at, end, row_at;
    uint32_t per, set_tiles;
    int row;
    uint32_t parts;  // of the row and head set; 0: as `per` says
};

// Inclusive sum over the lanes before, and its own.
__device__ inline uint32_t wave_scan(uint32_t v)
{
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);  // row_bcast:15, 31
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
    return v;
}

__device__ inline uint64_t quotient(uint64_t n, uint32_t d)
{
    return n >> 32 ? n / d : (uint32_t)n / d;  // the same, but 32 bits take a tenth of the instructions
}

// False where the shares before hold everything.  64 rows' tiles fit 32 bits.
template <int KT, int NW>
__device__ inline bool find_share(const AttendArgs& a, uint32_t number, Share* out)
{
    __shared__ uint32_t sums[2][NW];
    __shared__ uint64_t found_at;
    __shared__ int found_row;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int turn = 0;
    // tiles of the thread's row among NW * 64, those of the rows before it from r0 on, and all of them
    uint32_t own = 0;
    uint64_t mine = 0, total = 0;
    const auto scan_from = [&](int r0) {
        own = r0 + tid < a.rows ? work_of<KT>(a, r0 + tid) : 0;
        const uint32_t scan = wave_scan(own);
        if (lane == 63)
            sums[turn][wave] = scan;
        __syncthreads();
        mine = scan - own;
        uint64_t n = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const uint32_t x = sums[turn][w];
            mine += w < wave ? x : 0;
            n += x;
        }
        turn ^= 1;  // the next scan's barrier is behind every read of this one's sums
        return n;
    };
    if (a.rows == 1)
        total = work_of<KT>(a, 0);
    else
        for (int r0 = 0; r0 < a.rows; r0 += 64 * NW)
            total += scan_from(r0);
    // Whole sets read the heads of a token together, whose places in memory follow
    // each other; one head tile is divided among a workgroup's waves more finely,
    // which counts below two tiles a wave: one row of 4096 keys 14.6 and 17.7 us,
    // of 32768 23.6 and 23.6, of 131072 59 and 55.
    const uint32_t head_tiles = (uint32_t)(a.heads * a.tiles_of_group);
    const bool few = total * head_tiles < 2 * kShares * NW;
    out->set_tiles = a.one_if_few && few ? 1 : (uint32_t)a.set_tiles;
    const uint32_t sets = (head_tiles + out->set_tiles - 1) / out->set_tiles;
    const uint64_t all = total * sets, even = quotient(all + a.shares - 1, (uint32_t)a.shares);
    // a share holds kMinTiles at least, but no more than a row has where rows are
    // short: 132 of 1 tile (fp32) 21.5 us in shares of 4 and 9.6 of 1
    const uint32_t row = (uint32_t)min(quotient(total + a.rows - 1, (uint32_t)a.rows), (uint64_t)kMinTiles);
    out->per = max((uint32_t)even, row);  // all < 2^38
    out->at = (uint64_t)number * out->per;
    out->end = min(all, out->at + out->per);
    out->row = 0;
    out->row_at = 0;
    out->parts = 0;
    const uint32_t runs = (uint32_t)a.rows * sets;
    if (few && 4 * runs <= (uint32_t)a.shares) {
        // all / C + runs parts of at most C tiles: no more than the shares
        const uint32_t room = (uint32_t)a.shares - runs;
        const uint32_t C = max((uint32_t)kMinTiles, ((uint32_t)all + room - 1) / room);
        const auto take = [&](int row, uint32_t before, uint32_t work, uint32_t row_at) {
            // the part `number` among this row's, counted from `before` on
            const uint32_t parts = (work + C - 1) / C, in = number - before, set = in / parts, j = in - set * parts;
            out->row = row;
            out->row_at = row_at;
            out->parts = parts;
            out->at = row_at + (uint64_t)set * work + work * j / parts;
            out->end = row_at + (uint64_t)set * work + work * (j + 1) / parts;
        };
        if (a.rows == 1) {
            if (number >= ((uint32_t)total + C - 1) / C * sets)
                return false;
            take(0, 0, (uint32_t)total, 0);
            return true;
        }
        // the rows are those of the first wave's lanes
        __shared__ uint32_t found[3];
        const uint32_t parts = (own + C - 1) / C * sets, before = wave_scan(parts) - parts;
        if (tid == 0)
            found_row = -1;
        __syncthreads();
        if (wave == 0 && number >= before && number - before < parts) {
            found_row = tid;
            found[0] = before;
            found[1] = own;
            found[2] = (uint32_t)mine * sets;
        }
        __syncthreads();
        if (found_row < 0)
            return false;
        take(found_row, found[0], found[1], found[2]);
        return true;
    }
    if (out->at >= all)
        return false;
    if (a.rows == 1)
        return true;
    // the row r with before(r) <= at / sets < before(r + 1)
    const uint64_t at = quotient(out->at, sets);
    uint64_t before = 0;
    for (int r0 = 0;; r0 += 64 * NW) {
        const uint64_t n = a.rows > 64 * NW ? scan_from(r0) : total;
        if (at < before + n) {  // the same in every thread
            if (at >= before + mine && at - before - mine < own) {
                found_row = r0 + tid;
                found_at = (before + mine) * sets;
            }
            break;
        }
        before += n;
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

// Waves of a workgroup: as many as a CU's registers hold, so that each CU has one
// workgroup.  Of two workgroups on a CU one is served before the other: with
// equal shares of one row of 131072 keys they ended after 28 and 49 us.
constexpr int waves_of(int dp, int ht, int mode)
{
    return dp * ht <= 64 && mode == kWhole ? 16 : dp * ht <= 128 ? 8 : 4;
}

// The chunk at dim d of a row of few dims, one value at a time, zeros behind it.
template <int DT>
__device__ inline uint4 ld16_few(const char* row, int d, int dim)
{
    return d < dim ? ld16_head<DT>(row + d * Fmt<DT>::esize, dim - d) : make_uint4(0, 0, 0, 0);
}

// N (8 or 16) bytes of a row of values.  A load instruction takes whole rows of
// up to 256 bytes, which, where a sequence has pages of its own and a head of the
// cache one head tile, no other reads, so that they need not stay in the caches;
// rows of keys are read in pieces of 64 bytes by several, and do.  64 rows of up
// to 8192 keys (128 bf16 dims) 180 us, with plain loads 196; of 256 dims 183 and
// 202; of 64 fp32 dims 186 and 204; one row of 131072 keys 55.4 and 59.5; rows of
// 128 bytes 80 and 80.  Values that several read lose by it: three head tiles of a group of 48
// of 256 dims 227 us, with plain loads 214; 8 rows of the same 65536 keys 99 and 88;
// a prompt of 2048 tokens, a row each, 770 and 751.
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
__global__ __launch_bounds__(64 * waves_of(DP, HT, MODE)) void k_attend(AttendArgs a)
{
    constexpr int NW = waves_of(DP, HT, MODE);
    constexpr bool kBf16 = DT == MP_BF16, kUni = MODE == kWhole || MODE == kRows;
    constexpr int es = Fmt<DT>::esize, V = Fmt<DT>::V;
    constexpr int KG = kBf16 ? 2 : 1, KT = 16 * KG;  // groups of 16 keys, keys of a tile
    constexpr int S = DP / (4 * V);                  // steps of the first product
    constexpr int W = kBf16 && DP >= 128 ? 8 : 4;    // adjacent dims of a lane
    constexpr int NC = DP / (16 * W);                // chunks of them: dims 16 W c + W m + j
    constexpr int WB = W * es;                       // their bytes, 8 or 16
    constexpr int PD = DP + 4;                       // a head's outputs in LDS, off the banks of the next head's

    __shared__ float sm[NW][16 * HT], sl[NW][16 * HT];
    __shared__ float4 so[NW * 16 * HT * PD / 4];

    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int wave = uniform(tid >> 6);
    const uint32_t head_tiles = (uint32_t)(a.heads * a.tiles_of_group);

    Share share{};
    share.set_tiles = (uint32_t)a.set_tiles;
    if (a.shares != 0 && !find_share<KT, NW>(a, blockIdx.x, &share))
        return;
    // what is the same in all lanes the compiler is told: addresses then are the wave's
    const int wt = uniform((int)share.set_tiles);
    // waves that share a head tile, and this one's head tile and place among them
    const int step = NW / wt, mine = wave / step, place = wave % step;
    const uint32_t sets = (head_tiles + wt - 1) / (uint32_t)wt;

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
        r.end = keys.n <= keys.lo || set * wt + mine >= head_tiles ? r.begin : tile0 + (int)r.n_tiles;
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
    int parts = 0;                       // of the run's row and head set, where that is known
    if (a.shares == 0) {
        const int row = (int)(blockIdx.x / sets);
        cur = run_of(row, blockIdx.x - (uint32_t)row * sets, 0, 0x7fffffff, range_of(a, row));
        left = cur.n_tiles;
    } else {
        per = (uint32_t)uniform((int)share.per);
        parts = uniform((int)share.parts);
        left = (uint32_t)uniform((int)(uint32_t)(share.end - share.at));
        const uint64_t in = uniform(share.at - share.row_at);
        const int row = uniform(share.row);
        const Range keys = range_of(a, row);
        const uint32_t work = max(1, tiles_of<KT>(keys)), set = (uint32_t)quotient(in, work);
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
        const auto keep = [&](int w) {
            return drop <= 32 * w ? ~0u : drop >= 32 * w + 32 ? 0u : ~0u << (drop - 32 * w);
        };
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
            const int64_t head = hd.kvh * a.group + hd.gh0 + min(16 * h + m, hd.nh - 1);
            const char* qp = static_cast<const char*>(a.q) + (r.row * a.ldq + head * a.dim) * es;
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
                page[j] = ld_constant(table + a.by_page.of((uint32_t)min(c.tile * KT + 16 * j, c.run.n - 1)));
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
                    if constexpr (MODE == kOdd)
                        kr[j][s] = ld16_few<DT>(row, 4 * V * s + V * g, a.dim);
                    else
                        kr[j][s] = ld16u(row + chunk_at(s) * es);
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
                            vr[4 * j + e][c] = ld16_few<DT>(row, value_at(c, m), min(a.dim, value_at(c, m) + W));
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
        if (cur.off == 0 && tid < wt && cur.set * wt + tid < head_tiles && a.split != nullptr) {
            const int n = whole ? 1 : parts ? parts : (int)((before + cur.work - 1) / per) + 1;
            a.split[(int64_t)cur.row * head_tiles + cur.set * wt + tid] = make_int2((int)blockIdx.x, n | wt << 16);
        }

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
        // The waves keep step, or those that are served first would leave the
        // others to end alone: a barrier every kInStep tiles, as many in each wave.
        int barriers = again ? 0 : (int)(cur.n_tiles / (uint32_t)step / kInStep), until = kInStep;
        for (int tile = cur.begin; tile < cur.end; tile += step) {
            if (--until == 0 && barriers > 0) {
                __builtin_amdgcn_s_barrier();
                --barriers;
                until = kInStep;
            }
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
            // Outputs.  In bf16 p enters as its rounding and the rounded remainder, two products, which keep 16 of its
            // bits: 2^-16 of sum p |v| beside 2^-8 of the result when that is rounded.
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
        for (; barriers > 0; --barriers)
            __builtin_amdgcn_s_barrier();
        const bool there = cur.set * wt + mine < head_tiles;
        const Heads hd = heads_of(there ? cur.set * wt + mine : 0);
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
                if (head >= hd.nh || !there)
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
            // The sums of each head tile's waves, by all threads, four dims each.
            constexpr int D4 = DP / 4;
            for (int i = tid / D4, d = tid % D4 * 4; i < wt * a.unit_heads; i += 64 * NW / D4) {
                const int t = (int)a.by_heads.of((uint32_t)i), h = i - t * a.unit_heads;
                if (cur.set * wt + t >= head_tiles)
                    break;
                const Heads of = heads_of(cur.set * wt + t);
                if (h >= of.nh || d >= a.dim)
                    continue;
                const int w = t * step;  // the tile's first wave
                float4 x = so[((w * 16 * HT + h) * PD + d) / 4];
                for (int v = w + 1; v < w + step; ++v) {
                    const float4 y = so[((v * 16 * HT + h) * PD + d) / 4];
                    x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                }
                const float l = sl[w][h];
                const int64_t head = (int64_t)of.kvh * a.group + of.gh0 + h, at = (slot + t) * a.unit_heads + h;
                if (whole) {
                    const float r = l == 0.0f ? 0.0f : 1.0f / l;
                    const float f[4] = {l == 0.0f ? 0.0f : x.x * r, l == 0.0f ? 0.0f : x.y * r,
                                        l == 0.0f ? 0.0f : x.z * r, l == 0.0f ? 0.0f : x.w * r};
                    T* out = static_cast<T*>(a.out) + cur.row * a.ldo + head * a.dim + d;
                    if (d + 4 <= a.dim)
                        st_dims<DT, 4>(out, f);
                    else
                        for (int k = 0; d + k < a.dim; ++k)
                            out[k] = (T)f[k];
                    if (d == 0 && a.lse != nullptr)
                        a.lse[cur.row * (int64_t)(a.heads * a.group) + head] = lse_of(sm[w][h], l);
                } else {
                    float* part = a.part + at * a.dim + d;
                    if (a.dim % 4 == 0) {
                        *reinterpret_cast<float4*>(part) = x;
                    } else {
                        const float f[4] = {x.x, x.y, x.z, x.w};
                        for (int k = 0; k < 4 && d + k < a.dim; ++k)
                            part[k] = f[k];
                    }
                    if (d == 0)
                        a.stat[at] = make_float2(sm[w][h], l);
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

// ---------------------------------------------------------------- the parts of a row
// A query head's parts: n of them, at most kShares.
struct Parts {
    int row, head, n;
    int64_t first, next, share;  // places of part 0 and of part 1, and from one share's to the next's
    __device__ inline Parts(const AttendArgs& a, int row_, int head_) : row(row_), head(head_)
    {
        const int kvh = head / a.group, gh = head - kvh * a.group;
        const int ht = kvh * a.tiles_of_group + gh / a.unit_heads;
        const int2 split = a.split[(int64_t)row * (a.heads * a.tiles_of_group) + ht];
        const int wt = split.y >> 16;
        n = split.y & 0xffff;
        // part 0 is in the second place of its share, the others in the first
        const auto place = [&](int share, int second) {
            return ((2 * (int64_t)share + second) * wt + ht % wt) * a.unit_heads + gh % a.unit_heads;
        };
        first = place(split.x, 1);
        next = place(split.x + 1, 0);
        share = 2 * (int64_t)wt * a.unit_heads;
    }
    __device__ inline int64_t at(int c) const { return c == 0 ? first : next + (c - 1) * share; }
};

// Four dims of part c from d on; zeros where there is no such part or dim.
__device__ inline float4 part_at(const AttendArgs& a, const Parts& p, int c, int d)
{
    if (c >= p.n || d >= a.dim)
        return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float* q = a.part + p.at(c) * a.dim + d;
    if (a.dim % 4 == 0)
        return *reinterpret_cast<const float4*>(q);
    const int k = a.dim - d;
    return make_float4(q[0], k > 1 ? q[1] : 0.0f, k > 2 ? q[2] : 0.0f, k > 3 ? q[3] : 0.0f);
}

__device__ inline void add_to(float (&x)[4], float4 p, float f)
{
    x[0] += p.x * f;
    x[1] += p.y * f;
    x[2] += p.z * f;
    x[3] += p.w * f;
}

template <int DT>
__device__ inline void put_joined(const AttendArgs& a, const Parts& p, int d, const float* x, float l)
{
    using T = typename Elem<DT>::T;
    T* out = static_cast<T*>(a.out) + p.row * a.ldo + (int64_t)p.head * a.dim + d;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (d + k < a.dim)
            out[k] = (T)(l == 0.0f ? 0.0f : x[k] / l);
}

__device__ inline float wave_max(float t)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t = fmaxf(t, __shfl_xor(t, o));
    return t;
}

// The sums relative to the largest of the parts' maxima, by a workgroup: a float4
// of the dims from d0 on a thread, the other threads further parts; what a thread
// adds first is on its way while the statistics come in.
template <int DT, int LANES>
__device__ inline void join_by_group(const AttendArgs& a, const Parts& p, int d0)
{
    constexpr int kGroups = 256 / LANES, kFirst = 4;
    __shared__ float weight[kShares];
    __shared__ float tmp[8];
    __shared__ float4 acc[4][LANES];
    const int tid = threadIdx.x, wave = tid >> 6, mine = tid / LANES, d = d0 + tid % LANES * 4;
    const float2 s = tid < p.n ? a.stat[p.at(tid)] : make_float2(-INFINITY, 0.0f);
    float4 v[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; ++i)
        v[i] = part_at(a, p, mine + i * kGroups, d);
    float t = wave_max(s.x);
    if ((tid & 63) == 0)
        tmp[wave] = t;
    __syncthreads();
    t = fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
    const float w = __builtin_amdgcn_exp2f(s.x - (t == -INFINITY ? 0.0f : t));
    weight[tid] = w;
    float l = wave_xor_sum(s.y * w);
    if ((tid & 63) == 0)
        tmp[4 + wave] = l;
    __syncthreads();
    l = tmp[4] + tmp[5] + tmp[6] + tmp[7];
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kFirst; ++i)
        if (mine + i * kGroups < p.n)
            add_to(x, v[i], weight[mine + i * kGroups]);
    for (int c = mine + kFirst * kGroups; c < p.n; c += kFirst * kGroups) {
#pragma unroll
        for (int i = 0; i < kFirst; ++i)
            v[i] = part_at(a, p, c + i * kGroups, d);
#pragma unroll
        for (int i = 0; i < kFirst; ++i)
            if (c + i * kGroups < p.n)
                add_to(x, v[i], weight[c + i * kGroups]);
    }
    // over the groups of a wave, then over the waves
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] += __shfl_xor(x[k], o);
    if ((tid & 63) < LANES)
        acc[wave][tid % LANES] = make_float4(x[0], x[1], x[2], x[3]);
    __syncthreads();
    if (tid < LANES) {
        const float4 p0 = acc[0][tid], p1 = acc[1][tid], p2 = acc[2][tid], p3 = acc[3][tid];
        const float y[4] = {p0.x + p1.x + p2.x + p3.x, p0.y + p1.y + p2.y + p3.y, p0.z + p1.z + p2.z + p3.z,
                            p0.w + p1.w + p2.w + p3.w};
        put_joined<DT>(a, p, d, y, l);
    }
    if (a.lse != nullptr && tid == 0 && d0 == 0)
        a.lse[(int64_t)p.row * (a.heads * a.group) + p.head] = lse_of(t, l);
}

// A query head, or 4 LANES dims of it, a workgroup.
template <int DT, int LANES>
__global__ __launch_bounds__(256) void k_join(AttendArgs a)
{
    const uint32_t heads = (uint32_t)(a.heads * a.group);
    const int row = (int)(blockIdx.x / heads);
    const Parts p(a, row, (int)(blockIdx.x - (uint32_t)row * heads));
    if (p.n > 1)
        join_by_group<DT, LANES>(a, p, (int)blockIdx.y * 4 * LANES);
}

// Four query heads a workgroup: a wave each where no head has more than kByWave
// parts, else one after the other.  256 rows of 16 heads, few of them split: 8.9
// us with a workgroup a head, 6.5 so.  With 4, 8, 16 and 32 parts a wave, the whole
// attention of 64 rows of 32 heads and up to 8192 keys takes 185, 184, 180 and 180
// us, of 24 such rows 84, 84, 84 and 80.
constexpr int kByWave = 16;
template <int DT, int LANES>
__global__ __launch_bounds__(256) void k_join4(AttendArgs a)
{
    const int heads = a.heads * a.group, fours = (heads + 3) / 4;
    const int row = (int)(blockIdx.x / (uint32_t)fours);
    const int head0 = 4 * (int)(blockIdx.x - (uint32_t)row * (uint32_t)fours);
    const int there = min(heads - head0, 4), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int most = 0;
    for (int i = 0; i < there; ++i)
        most = max(most, Parts(a, row, head0 + i).n);
    if (most <= 1)
        return;
    if (most > kByWave) {
        for (int i = 0; i < there; ++i) {
            const Parts p(a, row, head0 + i);
            if (p.n > 1)
                join_by_group<DT, LANES>(a, p, 0);
            __syncthreads();  // LDS is read
        }
        return;
    }
    if (wave >= there)
        return;
    const Parts p(a, row, head0 + wave);
    if (p.n <= 1)
        return;
    constexpr int kGroups = 64 / LANES;
    const int mine = lane / LANES, d = lane % LANES * 4;
    float4 v[kByWave / kGroups];
#pragma unroll
    for (int i = 0; i < kByWave / kGroups; ++i)
        v[i] = part_at(a, p, mine + i * kGroups, d);
    const float2 s = lane < p.n ? a.stat[p.at(lane)] : make_float2(-INFINITY, 0.0f);
    const float t = wave_max(s.x), w = __builtin_amdgcn_exp2f(s.x - (t == -INFINITY ? 0.0f : t));
    const float l = wave_xor_sum(s.y * w);
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kByWave / kGroups; ++i) {
        const int c = mine + i * kGroups;
        const float f = __shfl(w, c);
        if (c < p.n)
            add_to(x, v[i], f);
    }
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] += __shfl_xor(x[k], o);
    if (lane < LANES)
        put_joined<DT>(a, p, d, x, l);
    if (a.lse != nullptr && lane == 0)
        a.lse[(int64_t)row * heads + p.head] = lse_of(t, l);
}

// ---------------------------------------------------------------- the host's side
struct Plan {
    int dp = 64, ht = 1, mode = kWhole;
    int64_t head_tiles = 1, set_tiles = 1, unit_heads = 1;
    bool one_if_few = false;
    int64_t shares = 0;  // 0: no row is split
};

Plan plan_of(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    Plan p;
    const int V = c.dtype == MP_F32 ? 4 : 8, dim = (int)c.head_dim;
    const int64_t group = s.q_heads / c.heads, tile = c.dtype == MP_F32 ? 16 : 32;
    p.dp = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
    p.mode = dim < V ? kOdd : c.page_size % 16 != 0 ? kEven : dim == p.dp ? kWhole : kRows;
    // Groups of more than 16 heads read their keys once for 32, with half the waves: 32 rows of up to 8192 keys, 8
    // heads for 32 each, 128 dims, 117 us; 16 at a time 144.  256 dims leave no registers for it.
    p.ht = group > 16 && dim <= 128 ? 2 : 1;
    p.head_tiles = c.heads * ((group + 16 * p.ht - 1) / (16 * p.ht));
    p.unit_heads = std::min<int64_t>(group, 16 * p.ht);
    // The largest set that leaves no more than a quarter of the waves idle in a row's sets: the heads of a token are
    // read together, and waves with a head tile of their own need not be joined.  Sets of one: 64 rows of 8 heads
    // 199 us for 180, 256 of 16 heads 327 for 80.
    const auto waste = [&](int64_t n) { return (p.head_tiles + n - 1) / n * n - p.head_tiles; };
    p.set_tiles = waves_of(p.dp, p.ht, p.mode);
    while (4 * waste(p.set_tiles) > p.head_tiles + waste(p.set_tiles))
        p.set_tiles /= 2;
    p.one_if_few = s.rows * p.head_tiles < kShares;
    const auto tiles_in = [&](int64_t keys) { return (keys + tile - 1) / tile; };
    const int64_t most = s.width * c.page_size;
    // a window may begin inside a tile, but a row has no more than its table has room for
    const bool slides = s.window > 0 && s.window < most;
    const int64_t tiles = slides ? std::min(tiles_in(s.window) + 1, tiles_in(most)) : tiles_in(most);
    // Rows of few tiles are a workgroup each and head set, but for very many of them: 2^20 rows of up to 32 keys, 7
    // heads of 64 dims, 29.1 ms in shares and 34.2 unsplit; of up to 64 keys, 8 heads of 128, 26.7 and 34.8.  (From
    // 2^12 such rows on shares are the faster ones, 118 us for 136 and 115 for 137; at 1000 rows they are the same, at
    // 64 16 us for 11; 20000 rows of 2 heads 565 for 528.)  The launch would hold either: rows <= 2^20 and rows *
    // head_tiles <= rows * q_heads <= 2^23, and a set holds all head tiles or 4 of them at least, or 2 of 5, so that
    // there are 3 * 2^20 workgroups of 1024 threads at most.
    const int64_t waves = s.rows * p.head_tiles * waves_of(p.dp, p.ht, p.mode);
    // A share counts its tiles in 31 bits.  Tables with room for more have 2^13 rows and head sets or more, which
    // fill the chip unsplit.
    const int64_t all = s.rows * ((p.head_tiles + p.set_tiles - 1) / p.set_tiles) * tiles;
    if (all < (int64_t)1 << 38 && (tiles > kMinTiles || waves >= (int64_t)1 << 26))
        p.shares = std::min<int64_t>(kShares, (s.rows * p.head_tiles * tiles + kMinTiles - 1) / kMinTiles);
    else if (p.one_if_few)
        p.set_tiles = 1;
    return p;
}

uint64_t up16(uint64_t n) { return (n + 15) / 16 * 16; }
// query heads of all parts: two of a share
uint64_t slot_heads(const Plan& p) { return (uint64_t)(2 * p.shares * p.set_tiles * p.unit_heads); }

template <int DT, int DP, int HT, int MODE>
void launch_mode(const AttendArgs& a, unsigned grid, hipStream_t st)
{
    k_attend<DT, DP, HT, MODE><<<grid, 64 * waves_of(DP, HT, MODE), 0, st>>>(a);
}

template <int DT, int DP, int HT>
void launch_tiles(const AttendArgs& a, unsigned grid, int mode, hipStream_t st)
{
    if (mode == kWhole)
        launch_mode<DT, DP, HT, kWhole>(a, grid, st);
    else if (mode == kRows)
        launch_mode<DT, DP, HT, kRows>(a, grid, st);
    else if (mode == kEven)
        launch_mode<DT, DP, HT, kEven>(a, grid, st);
    else if constexpr (DP == 64)
        launch_mode<DT, DP, HT, kOdd>(a, grid, st);
}

template <int DT>
void launch_type(const AttendArgs& a, const Plan& p, hipStream_t st)
{
    const unsigned grid = (unsigned)(p.shares ? p.shares : a.rows * ((p.head_tiles + p.set_tiles - 1) / p.set_tiles));
    if (p.dp == 64)
        p.ht == 2 ? launch_tiles<DT, 64, 2>(a, grid, p.mode, st) : launch_tiles<DT, 64, 1>(a, grid, p.mode, st);
    else if (p.dp == 128)
        p.ht == 2 ? launch_tiles<DT, 128, 2>(a, grid, p.mode, st) : launch_tiles<DT, 128, 1>(a, grid, p.mode, st);
    else
        launch_tiles<DT, 256, 1>(a, grid, p.mode, st);
    if (p.shares) {
        // Few heads: their dims in slices of 32, so that more workgroups share the parts.  One row of 28 heads 55 us,
        // by k_join4 85.  Rows of up to 8192 keys in slices / by k_join4, 128 dims: 256 heads 35 / 44, 512 58 / 63,
        // 768 81 / 84, 1024 102 / 99, 1536 142 / 136; 64 dims: 384 heads 83 / 89, 640 125 / 125.
        const unsigned heads = (unsigned)(a.rows * a.heads * a.group);
        const unsigned fours = (unsigned)(a.rows * ((a.heads * a.group + 3) / 4));
        if (heads < 512)
            k_join<DT, 8><<<dim3(heads, (unsigned)((a.dim + 31) / 32)), 256, 0, st>>>(a);
        else if (p.dp == 64)
            k_join4<DT, 16><<<fours, 256, 0, st>>>(a);
        else if (p.dp == 128)
            k_join4<DT, 32><<<fours, 256, 0, st>>>(a);
        else
            k_join4<DT, 64><<<fours, 256, 0, st>>>(a);
    }
}

}  // namespace

uint64_t kv_attend_ws_bytes(const mp_kv_cache& c, const mp_kv_attend_shape& s)
{
    const Plan p = plan_of(c, s);
    if (s.rows == 0 || p.shares == 0)
        return 0;
    return up16((uint64_t)(s.rows * p.head_tiles) * sizeof(int2)) + up16(slot_heads(p) * sizeof(float2)) +
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
        w += up16((uint64_t)(s.rows * p.head_tiles) * sizeof(int2));
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
    a.set_tiles = (int32_t)p.set_tiles;
    a.one_if_few = p.one_if_few;
    a.shares = (int32_t)p.shares;
    a.unit_heads = (int32_t)p.unit_heads;
    a.by_page = Div((uint32_t)c.page_size);
    a.by_tiles = Div((uint32_t)a.tiles_of_group);
    a.by_heads = Div((uint32_t)p.unit_heads);
    a.scale = (float)((double)s.scale * 1.4426950408889634);
    if (c.dtype == MP_F32)
        launch_type<MP_F32>(a, p, st);
    else
        launch_type<MP_BF16>(a, p, st);
    return hipGetLastError();
}

}  // namespace mp
