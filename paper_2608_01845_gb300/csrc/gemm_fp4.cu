// Product of e2m1 matrices with e4m3 scales of 16 columns and fp32 scales of rows:
//   C[m, n] = epilogue( ra[m] rw[n] sum_k (a s_a)[m, k] (w s_w)[n, k] ),
// and of two such products the gated form act(A W^T) * (A U^T).
#include "gemm_fp4.cuh"

namespace wdc {

namespace {

constexpr int kTile = 64;

__device__ __forceinline__ void decode_tile(float (*dst)[kTile + 1], const uint8_t* codes, const uint8_t* scale, int row0,
                                            int rows, int K, int piece, int pieces) {
    const int r = threadIdx.x >> 2, part = threadIdx.x & 3, row = row0 + r;
    uint2 q = make_uint2(0u, 0u);
    float s = 0.f;
    if (row < rows) {
        q = *reinterpret_cast<const uint2*>(codes + ((size_t)row * K + piece * 64 + part * 16) / 2);
        const uint8_t b = scale[4 * piece_word4(row, piece, pieces) + part];
        s = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3)));
    }
    float v[8];
    e2m1_values(q.x, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[r][part * 16 + i] = v[i] * s;
    e2m1_values(q.y, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[r][part * 16 + 8 + i] = v[i] * s;
}

template <typename T, bool GATED>
__global__ void __launch_bounds__(256) gemm4_plain_kernel(const __grid_constant__ Gemm4Args g) {
    __shared__ float a[kTile][kTile + 1], w[kTile][kTile + 1];
    chain_release();
    chain_wait();
    const int n_tiles = (g.N + kTile - 1) / kTile;
    const int m0 = (int)(blockIdx.x / n_tiles) * kTile, n0 = (int)(blockIdx.x % n_tiles) * kTile;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    float acc[2][4][4] = {};
    for (int p = 0; p < g.pieces; ++p) {
        decode_tile(a, g.A, g.sa, m0, g.M, g.K, p, g.pieces);
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            decode_tile(w, h ? g.U : g.W, h ? g.su : g.sw, n0, g.N, g.K, p, g.pieces);
            __syncthreads();
            for (int k = 0; k < kTile; ++k) {
                float x[4], y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = a[ty + 16 * i][k];
                    y[i] = w[tx + 16 * i][k];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[h][i][j] = fmaf(x[i], y[j], acc[h][i][j]);
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= g.M || n >= g.N) continue;
            float v = acc[0][i][j] * g.ra[m] * g.rw[n] + (g.bias ? g.bias[n] : 0.f);
            T* out = reinterpret_cast<T*>(g.out) + (size_t)m * g.N + n;
            if constexpr (GATED) {
                const float u = acc[1][i][j] * g.ra[m] * g.ru[n] + (g.up_bias ? g.up_bias[n] : 0.f);
                *out = to_act<T>((g.gelu ? gelu_tanh_f(v) : silu_f(v)) * u);
            } else {
                if (g.gelu) v = gelu_tanh_f(v);
                if (g.res) v = fmaf(g.gate ? g.gate[n] : 1.f, v, ld_act<T>(reinterpret_cast<const T*>(g.res) + (size_t)m * g.N + n));
                *out = to_act<T>(v);
            }
        }
}

wdc_status launch(Ctx* c, const Gemm4Args& g, cudaStream_t s) {
    const long long tiles = ((long long)(g.M - 1) / kTile + 1) * ((g.N - 1) / kTile + 1);
    if (tiles > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM: more than 2^31 - 1 thread blocks");
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_GEMM, s);
        const bool bf16 = c->cfg.dtype == WDC_BF16;
        auto k = g.U ? (bf16 ? gemm4_plain_kernel<__nv_bfloat16, true> : gemm4_plain_kernel<float, true>)
                     : (bf16 ? gemm4_plain_kernel<__nv_bfloat16, false> : gemm4_plain_kernel<float, false>);
        launch_kernel(k, dim3((unsigned)tiles), 256, 0, s, 1, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 GEMM launch: ") + cudaGetErrorString(e));
    return WDC_OK;
}

// What both products check; WDC_OK with *none: there is nothing to do.
wdc_status check(Ctx* c, const wdc_fp4* A, const wdc_fp4* W, const void* C, int M, int N, int K, uintptr_t rest, bool* none) {
    *none = false;
    if (M < 0 || N <= 0 || K <= 0) return fail(c, WDC_ERR_INVALID_ARG, "fp4 GEMM: M >= 0, N > 0 and K > 0 wanted");
    if (N > kMaxWidth4 || K > kMaxWidth4) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM: N or K above 2^31 - 512");
    if (M > kMaxRows4) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM: more than 2^31 - 128 rows");
    if (N % 8 || K % 64) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM needs N % 8 == 0 and K % 64 == 0");
    if ((*none = M == 0)) return WDC_OK;
    if (wdc_status st = check_fp4(c, A)) return st;
    if (wdc_status st = check_fp4(c, W)) return st;
    if (!C) return fail(c, WDC_ERR_INVALID_ARG, "fp4 GEMM: null pointer");
    if (((uintptr_t)C | rest) & 15) return fail(c, WDC_ERR_INVALID_ARG, "fp4 GEMM: pointers must be 16-byte aligned");
    return WDC_OK;
}

Gemm4Args args(Ctx* c, const wdc_fp4* A, const wdc_fp4* W, const float* bias, void* C, int M, int N, int K, int gelu) {
    Gemm4Args g{};
    g.M = M; g.N = N; g.K = K; g.pieces = K / kPieceCols4;
    g.A = (const uint8_t*)A->codes; g.sa = (const uint8_t*)A->scale; g.ra = A->row_scale;
    g.W = (const uint8_t*)W->codes; g.sw = (const uint8_t*)W->scale; g.rw = W->row_scale;
    g.bias = bias; g.out = C; g.gelu = gelu; g.err = c->err;
    return g;
}

}  // namespace

wdc_status op_gemm_fp4(Ctx* c, const wdc_fp4* A, const wdc_fp4* W, const float* bias, void* C, int M, int N, int K, int gelu,
                       const void* res, const float* gate, cudaStream_t s) {
    bool none;
    if (wdc_status st = check(c, A, W, C, M, N, K, (uintptr_t)bias | (uintptr_t)res | (uintptr_t)gate, &none)) return st;
    if (none) return WDC_OK;
    Gemm4Args g = args(c, A, W, bias, C, M, N, K, gelu);
    g.res = res;
    g.gate = res ? gate : nullptr;
    return launch(c, g, s);
}

wdc_status op_gated_fp4(Ctx* c, const wdc_fp4* A, const wdc_fp4* W, const wdc_fp4* U, const float* gate_bias,
                        const float* up_bias, void* C, int M, int N, int K, int gelu, cudaStream_t s) {
    bool none;
    if (wdc_status st = check(c, A, W, C, M, N, K, (uintptr_t)gate_bias | (uintptr_t)up_bias, &none)) return st;
    if (none) return WDC_OK;
    if (wdc_status st = check_fp4(c, U)) return st;
    Gemm4Args g = args(c, A, W, gate_bias, C, M, N, K, gelu);
    g.U = (const uint8_t*)U->codes; g.su = (const uint8_t*)U->scale; g.ru = U->row_scale;
    g.up_bias = up_bias;
    return launch(c, g, s);
}

}  // namespace wdc
