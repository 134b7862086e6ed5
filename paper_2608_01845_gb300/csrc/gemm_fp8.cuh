// What the two fp8 GEMM kernels share (gemm_fp8.cu, gemm_fp8_pair.cu).
#pragma once

#include "dit_kernels.cuh"
#include "ptx.cuh"

namespace wdc {

constexpr int kBlock8 = 128;            // of K: a scale's columns, the bytes of a tile row

struct Gemm8Args {
    int M, N, K, kb;                    // kb: blocks of K
    int m_tiles, n_tiles;
    int split, stages, bufs;            // narrow kernel: CTAs a tile, tiles of its ring, TMEM buffers
    int group_n;                        // pair kernel: column blocks of a raster group
    int sw_rows;                        // rows of w_scale
    const float *sa, *sw, *bias, *gate;
    const void* res;
    void* out;
    int gelu;
    unsigned* err;
};

__device__ __forceinline__ void cp_async4(float* dst, const float* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16(float* dst, const float* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// gemm_fp8_pair.cu
wdc_status launch_gemm8_pair(Ctx* c, const void* A, const void* W, Gemm8Args g, int bn, cudaStream_t s);

}  // namespace wdc
