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
    int m_tiles, n_tiles;
    int kb;                             // tiles of K (kTileK4)
    int split;                          // narrow kernel: CTAs a tile
    // pair kernel: column blocks of a raster group; tiles that a pair takes whole, the tiles
    // behind them and the parts of K those are split in; the parts' sums and counters
    int group_n, whole, tail, parts;
    float* work;
    unsigned* counters;
};

constexpr int kTileK4 = 256;            // of K: 128 bytes of codes, a row of the swizzled tiles, and four pieces of scales

// Tensor maps of codes [rows][K / 2] in boxes of `box` rows by 128 bytes, and of scales in
// boxes of four pieces.
inline bool encode_codes(CUtensorMap* m, const void* codes, int rows, int K, int box, std::string* why) {
    return encode_tmap_2d(m, codes, (uint64_t)K / 2, (uint64_t)rows, (uint64_t)K / 2, kTileK4 / 2, box, why,
                          CU_TENSOR_MAP_DATA_TYPE_UINT8);
}
inline bool encode_scales(CUtensorMap* m, const void* scale, int rows, int pieces, std::string* why) {
    return encode_tmap_3d(m, scale, kPiece4 / 2, pieces, (uint64_t)(rows - 1) / 128 + 1, kPiece4, (uint64_t)pieces * kPiece4,
                          kPiece4 / 2, 4, 1, why, false, CU_TENSOR_MAP_SWIZZLE_NONE);
}

__device__ __forceinline__ float silu_f(float x) { return __fdividef(x, 1.0f + __expf(-x)); }

// gemm_fp4_pair.cu
bool plan_gemm4_pair(const Ctx* c, Gemm4Args& g);   // its tiles (from M, N, K and whether there is a U); false: it cannot
wdc_status launch_gemm4_pair(Ctx* c, const Gemm4Args& g, cudaStream_t s);

}  // namespace wdc
