// Argument checks that the operators' entry points share (api_ffn.hip,
// api_attn.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mp_internal.h"

namespace mp {

// A launch takes fewer than 2^32 threads along x: up to kMaxSize rows or
// columns of an operand, the kernels' grids stay below that.
constexpr int64_t kMaxRows = 0x7fffffff, kMaxSize = (int64_t)1 << 26, kMaxHidden = (int64_t)1 << 24;
constexpr int64_t kMaxLd = (int64_t)1 << 40;

// A buffer of a call: n bytes from p on.
struct Span {
    const char* p = nullptr;
    size_t n = 0;
    int64_t ld = 0;
    const char* name = "";
};

// Bytes from a matrix's first element to behind its last, (rows - 1) * ld +
// cols elements; 2^62, more than any buffer holds, where that is beyond it.
inline size_t span_bytes(int64_t rows, int64_t cols, int64_t ld, int es)
{
    if (rows == 0 || cols == 0)
        return 0;
    const unsigned __int128 n = ((unsigned __int128)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * (uint32_t)es;
    return n >> 62 ? (size_t)1 << 62 : (size_t)n;
}

inline int check_dtype(int32_t dtype, int* es)
{
    if (dtype != MP_F32 && dtype != MP_BF16)
        return fail(MP_E_ARG, "dtype %d is not MP_F32 or MP_BF16", dtype);
    *es = dtype == MP_F32 ? 4 : 2;
    return MP_OK;
}

inline int check_size(int64_t v, int64_t lo, int64_t hi, const char* name)
{
    if (v < lo || v > hi)
        return fail(MP_E_ARG, "%s = %lld must be in [%lld, %lld]", name, (long long)v, (long long)lo, (long long)hi);
    return MP_OK;
}

inline int check_ld(int64_t ld, int64_t cols, const char* name)
{
    if (ld < cols || ld > kMaxLd)
        return fail(MP_E_ARG, "%s = %lld must be in [%lld, 2^40]", name, (long long)ld, (long long)cols);
    return MP_OK;
}

// The device allocations that the present call has looked up: its buffers often
// share one, and asking the runtime for a pointer's costs 0.3 us.
class Seen {
public:
    int check(const void* p, size_t bytes, const char* name)
    {
        const char* q = static_cast<const char*>(p);
        for (int i = 0; i < k_; ++i)
            if (q >= a_[i].p && q < a_[i].p + a_[i].n && bytes <= (size_t)(a_[i].p + a_[i].n - q))
                return MP_OK;
        Allocation found;
        const int rc = check_device_buffer(p, bytes, name, &found);
        if (rc == MP_OK && found.n != 0 && k_ < kMost)
            a_[k_++] = found;
        return rc;
    }

private:
    static constexpr int kMost = 8;
    Allocation a_[kMost];
    int k_ = 0;
};

// A rows x cols matrix in device memory, aligned to its elements.
inline int check_matrix(Seen& seen, const void* p, int64_t rows, int64_t cols, int64_t ld, int es, const char* name, Span* out)
{
    *out = Span{static_cast<const char*>(p), span_bytes(rows, cols, ld, es), ld, name};
    if (out->n == 0)  // nothing of it is read or written
        return MP_OK;
    if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)es != 0)
        return fail(MP_E_ARG, "%s is not aligned to its elements", name);
    return seen.check(p, out->n, name);
}

inline bool meet(const Span& a, const Span& b) { return a.n && b.n && a.p < b.p + b.n && b.p < a.p + a.n; }

// An output against a buffer that it may not share, or may share only exactly (same).
inline int check_apart(const Span& out, const Span& in, bool same)
{
    if (meet(out, in) && !(same && out.p == in.p && out.ld == in.ld))
        return fail(MP_E_ARG, "%s overlaps %s", out.name, in.name);
    return MP_OK;
}

inline int check_workspace(Seen& seen, const void* ws, uint64_t have, uint64_t need, Span* out)
{
    *out = Span{static_cast<const char*>(ws), (size_t)need, 0, "workspace"};
    if (need == 0)
        return MP_OK;
    if (ws == nullptr || have < need)
        return fail(MP_E_ARG, "workspace holds %llu bytes, %llu needed", (unsigned long long)(ws ? have : 0),
                    (unsigned long long)need);
    if (reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return fail(MP_E_ARG, "workspace is not 16-byte aligned");
    return seen.check(ws, (size_t)need, "workspace");
}

}  // namespace mp
