// Tiled matrix products with an epilogue (k_gemm.hip), for k_linear.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mp_internal.h"

namespace mp {

// What follows z = sum + bias: z stored, y = act(z) + r stored.
struct Epi {
    const void* bias;  // or null
    const void* r;     // or null
    void* z;           // or null
    int64_t ldr, ldz;
    int act;
};

// C[i][j] = sum over p of A(i, p) B(j, p).  An operand's rows are its i (or j)
// and hold p side by side, or its rows are p: NT has both of the first kind
// (x w^T), NN has B's rows p (dz w), TN both (dz^T x).
enum class Form { NT, NN, TN };

struct Gemm {
    int dtype;
    Form form;
    const void* a;
    const void* b;
    void* c;
    int64_t lda, ldb, ldc;
    int64_t I, J, P;  // > 0, except P
    Epi epi;          // used by NT only
};

// ws: gemm_ws_bytes(dtype, I, J, P) bytes, 16-byte aligned.
hipError_t launch_gemm(const Gemm& g, void* ws, hipStream_t st);
uint64_t gemm_ws_bytes(int dtype, int64_t I, int64_t J, int64_t P);

}  // namespace mp
