// Rows to e2m1 with an e4m3 scale for 16 columns and an fp32 scale for the row, and
// back:
//   row   = max |x| / 2688 over the row,
//   s     = e4m3(max |x| / (6 row)) over 16 columns,  code = e2m1(x / (s row)),
//   value = code * (s * row).
// The row's scale needs the whole row before the first code: a row stays in the
// registers of its warps between the two, so x is read once.  Bound by memory: 2.56
// bytes an element for bf16, 4.56 for fp32.
#include "quant.cuh"

namespace wdc {

namespace {

struct Quant4Args {
    const void* x;
    long long ldx;
    uint8_t* codes;
    uint32_t* scale;                   // words of four scales (piece_word4)
    float* row_scale;
    int M, K, pieces;                  // pieces: K / 64
};

// The largest magnitude of a row over its W warps (blockDim.x threads), NaN kept.
// `part`: [rows of the block][32]; every thread of the block calls it.
__device__ __forceinline__ float row_max(float a, float (*part)[32]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    if (blockDim.x == 32) return a;
    if ((threadIdx.x & 31) == 0) part[threadIdx.y][threadIdx.x >> 5] = a;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    a = lane < (int)(blockDim.x >> 5) ? part[threadIdx.y][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}

// A row of blockDim.x threads, V pieces of 8 columns a thread; rows past M (of the
// last 128) get scales of zero.
template <typename T, int V>
__global__ void __launch_bounds__(512) quantize4_kernel(const __grid_constant__ Quant4Args a) {
    __shared__ float part[16][32];
    chain_release();
    chain_wait();
    const int m = (int)(blockIdx.x * blockDim.y + threadIdx.y);
    const T* x = reinterpret_cast<const T*>(a.x) + (size_t)m * a.ldx;
    float v[V][8], top = 0.f;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int k = (u * (int)blockDim.x + (int)threadIdx.x) * 8;
        if (m < a.M && k < a.K) {
            load8(x + k, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < V; ++u) top = max_nan(top, absmax8(v[u]));
    const float row = row_scale4(row_max(top, part)), six = 6.f * row;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int k = (u * (int)blockDim.x + (int)threadIdx.x) * 8;
        uint32_t* codes = m < a.M && k < a.K ? reinterpret_cast<uint32_t*>(a.codes + ((size_t)m * a.K + k) / 2) : nullptr;
        uint32_t* word = k < a.K && k % kPieceCols4 == 0 ? a.scale + piece_word4(m, k / kPieceCols4, a.pieces) : nullptr;
        store_fp4(v[u], row, six, codes, word);
        if (m >= a.M && word) *word = 0u;
    }
    if (m < a.M && threadIdx.x == 0) a.row_scale[m] = row;
}

// Rows wider than a block's registers: read twice, the second time from L2.
template <typename T>
__global__ void __launch_bounds__(512) quantize4_wide_kernel(const __grid_constant__ Quant4Args a) {
    __shared__ float part[1][32];
    chain_release();
    chain_wait();
    const int m = (int)blockIdx.x;
    if (m >= a.M) {
        for (int p = threadIdx.x; p < a.pieces; p += blockDim.x) a.scale[piece_word4(m, p, a.pieces)] = 0u;
        return;
    }
    const T* x = reinterpret_cast<const T*>(a.x) + (size_t)m * a.ldx;
    float v[8], top = 0.f;
    for (long long k = threadIdx.x * 8; k < a.K; k += blockDim.x * 8) {
        load8(x + k, v);
        top = max_nan(top, absmax8(v));
    }
    const float row = row_scale4(row_max(top, part)), six = 6.f * row;
    for (long long k0 = 0; k0 < a.K; k0 += blockDim.x * 8) {        // (whole warps: the lanes trade scales)
        const long long k = k0 + threadIdx.x * 8;
        if (k < a.K) {
            load8(x + k, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        }
        uint32_t* codes = k < a.K ? reinterpret_cast<uint32_t*>(a.codes + ((size_t)m * a.K + k) / 2) : nullptr;
        uint32_t* word =
            k < a.K && k % kPieceCols4 == 0 ? a.scale + piece_word4(m, (int)(k / kPieceCols4), a.pieces) : nullptr;
        store_fp4(v, row, six, codes, word);
    }
    if (threadIdx.x == 0) a.row_scale[m] = row;
}

// Eight columns a thread.
template <typename T>
__global__ void __launch_bounds__(256) dequantize4_kernel(const uint8_t* codes, const uint8_t* scale, const float* row_scale,
                                                          T* x, long long ldx, int M, int K, int pieces) {
    chain_release();
    chain_wait();
    const int per = K / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = i / per;
    if (row >= M) return;
    const int m = (int)row, k = (int)(i - row * per) * 8;
    const uint32_t q = *reinterpret_cast<const uint32_t*>(codes + ((size_t)m * K + k) / 2);
    const uint8_t s = scale[4 * piece_word4(m, k / kPieceCols4, pieces) + (k / 16) % 4];
    const float step = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)s, __NV_E4M3))) * row_scale[m];
    float v[8];
    e2m1_values(q, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= step;
    put8(x + (size_t)m * ldx + k, v);
}

constexpr int kHeld = 4;                           // pieces of 8 columns a thread holds at most
constexpr int kMaxThreads = 512;

template <typename T>
wdc_status launch(Ctx* c, const Quant4Args& a, cudaStream_t s) {
    const long long rows = ((long long)(a.M - 1) / 128 + 1) * 128;      // those behind M: scales of zero
    const int eights = a.K / 8;
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_OTHER, s);
        if (eights > kHeld * kMaxThreads) {
            launch_kernel(quantize4_wide_kernel<T>, dim3((unsigned)rows), 512, 0, s, 1, a);
        } else {
            const int v = eights <= 32 ? 1 : (eights <= 128 ? 2 : kHeld);
            const int warps = (eights + 32 * v - 1) / (32 * v);
            const int per = warps >= 8 ? 1 : (warps >= 4 ? 2 : (warps >= 2 ? 4 : 8));
            const dim3 block(32 * warps, per), grid((unsigned)(rows / per));
            if (v == 1) launch_kernel(quantize4_kernel<T, 1>, grid, block, 0, s, 1, a);
            else if (v == 2) launch_kernel(quantize4_kernel<T, 2>, grid, block, 0, s, 1, a);
            else launch_kernel(quantize4_kernel<T, kHeld>, grid, block, 0, s, 1, a);
        }
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 quantize: ") + cudaGetErrorString(e));
    return WDC_OK;
}

template <typename T>
wdc_status launch_back(Ctx* c, const wdc_fp4& q, T* x, long long ldx, int M, int K, cudaStream_t s) {
    const long long blocks = ((long long)M * (K / 8) + 255) / 256;
    if (blocks > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 dequantize: more than 2^31 - 1 thread blocks");
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_OTHER, s);
        launch_kernel(dequantize4_kernel<T>, dim3((unsigned)blocks), 256, 0, s, 1, (const uint8_t*)q.codes,
                      (const uint8_t*)q.scale, (const float*)q.row_scale, x, ldx, M, K, K / kPieceCols4);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 dequantize: ") + cudaGetErrorString(e));
    return WDC_OK;
}

// What both directions check.
wdc_status check(Ctx* c, const void* x, long long ldx, const wdc_fp4* q, int M, int K) {
    if (!q) return fail(c, WDC_ERR_INVALID_ARG, "fp4: no wdc_fp4");
    if (M < 0 || K <= 0) return fail(c, WDC_ERR_INVALID_ARG, "fp4: M >= 0 and K > 0 wanted");
    if (ldx < K) return fail(c, WDC_ERR_INVALID_ARG, "fp4: row stride below K");
    if (K > kMaxWidth4) return fail(c, WDC_ERR_UNSUPPORTED, "fp4: more than 2^31 - 512 columns");
    if (M > kMaxRows4) return fail(c, WDC_ERR_UNSUPPORTED, "fp4: more than 2^31 - 128 rows");
    if (K % 64 || ldx % 8) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 needs K % 64 == 0 and ldx % 8 == 0");
    if (M == 0) return WDC_OK;
    if (!x) return fail(c, WDC_ERR_INVALID_ARG, "fp4: null pointer");
    if ((uintptr_t)x & 15) return fail(c, WDC_ERR_INVALID_ARG, "fp4: pointers must be 16-byte aligned");
    return check_fp4(c, q);
}

}  // namespace

wdc_status check_fp4(Ctx* c, const wdc_fp4* q) {
    if (!q || !q->codes || !q->scale || !q->row_scale) return fail(c, WDC_ERR_INVALID_ARG, "fp4: null pointer");
    if (((uintptr_t)q->codes | (uintptr_t)q->scale | (uintptr_t)q->row_scale) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "fp4: pointers must be 16-byte aligned");
    return WDC_OK;
}

wdc_status op_quantize_fp4(Ctx* c, const void* x, long long ldx, const wdc_fp4* q, int M, int K, cudaStream_t s) {
    if (wdc_status st = check(c, x, ldx, q, M, K)) return st;
    if (M == 0) return WDC_OK;
    Quant4Args a{x, ldx, (uint8_t*)q->codes, (uint32_t*)q->scale, q->row_scale, M, K, K / kPieceCols4};
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, a, s) : launch<float>(c, a, s);
}

wdc_status op_dequantize_fp4(Ctx* c, const wdc_fp4* q, void* x, long long ldx, int M, int K, cudaStream_t s) {
    if (wdc_status st = check(c, x, ldx, q, M, K)) return st;
    if (M == 0) return WDC_OK;
    return c->cfg.dtype == WDC_BF16 ? launch_back(c, *q, (__nv_bfloat16*)x, ldx, M, K, s)
                                    : launch_back(c, *q, (float*)x, ldx, M, K, s);
}

}  // namespace wdc
