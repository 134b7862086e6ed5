// What the fp4 GEMM's files share.
#pragma once

#include "ptx.cuh"
#include "quant.cuh"

namespace wdc {

// C = epilogue((A W^T) row_a row_w), or, gated, act(that + bias) * ((A U^T) row_a row_u + up_bias).
struct Gemm4Args {
    int M, N, K, pieces;                // pieces: K / 64
    const uint8_t *A, *W, *U;           // codes; U: the second weights, null unless gated
    const uint8_t *sa, *sw, *su;        // scales
    const float *ra, *rw, *ru;          // the rows' scales
    const float *bias, *up_bias, *gate;
    const void* res;
    void* out;
    int gelu;
    unsigned* err;
};

__device__ __forceinline__ float silu_f(float x) { return __fdividef(x, 1.0f + __expf(-x)); }

}  // namespace wdc
