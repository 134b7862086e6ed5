// Rows or 128 x 128 blocks to e4m3 with a scale for each block:
//   s = max |x| / 448,  q = e4m3(x / s).
// One pass over x: a block's elements stay in registers between its maximum
// and its quotients.  Bound by memory: 3 bytes an element for bf16, 5 for fp32.
#include "dit_kernels.cuh"

namespace wdc {

namespace {

constexpr int kBlock = 128;             // columns (and, for weights, rows) of a block
constexpr float kE4m3Max = 448.0f;

// Maximum that keeps a NaN (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Four quotients to e4m3, to nearest even; beyond 448 saturated, NaN kept.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        " mov.b32 %0, {lo, hi};\n}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// A lane's 8 elements in fp32.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ float absmax8(const float (&v)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max_nan(m, fabsf(v[i]));
    return m;
}

// The eight quotients by a scale outside the range of store8's shorter way.
__device__ __noinline__ uint2 quotients(float4 a, float4 b, float s) {
    return make_uint2(e4m3x4(a.x / s, a.y / s, a.z / s, a.w / s), e4m3x4(b.x / s, b.y / s, b.z / s, b.w / s));
}

// The eight quotients by s, in e4m3.  With r the correctly rounded reciprocal of s,
// t = x r corrected once by its remainder, t + (x - t s) r, is the correctly rounded
// quotient (Markstein, "Computation of elementary functions on the IBM RISC
// System/6000 processor", 1990) as long as nothing underflows that matters.  Three
// instructions an element and little code: eight divisions a lane were what the
// kernel waited for, and their code what a short call fetched (1576 x 3072 bf16 8.2
// us, now 4.2).
__device__ __forceinline__ void store8(uint8_t* q, const float (&v)[8], float s) {
    uint2 w;
    const float by = s == 0.f ? 1.f : s;           // a block of zeros (or one so small that its scale is)
    if (by >= 0x1p-100f && by < INFINITY) {
        const float r = 1.0f / by;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = v[i] * r;
            y[i] = fmaf(fmaf(-t, by, v[i]), r, t);
        }
        w = make_uint2(e4m3x4(y[0], y[1], y[2], y[3]), e4m3x4(y[4], y[5], y[6], y[7]));
    } else {
        w = quotients(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]), s);
    }
    *reinterpret_cast<uint2*>(q) = w;
}

// Scales along rows.  Sixteen lanes hold a block, a warp kSpan neighbouring
// pairs of blocks of one row (all loaded before the first is reduced), and the
// eight warps of a CTA take successive rows, whose scales lie side by side.
constexpr int kSpan = 2;
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* x, long long ldx, uint8_t* q, float* scale, int M,
                                                            int K, int spans) {
    chain_release();
    chain_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int span = blockIdx.x % spans;
    const int m = (int)(blockIdx.x / spans) * 8 + warp;
    if (m >= M) return;
    const int k0 = span * (kSpan * 2 * kBlock) + lane * 8;
    float v[kSpan][8];
#pragma unroll
    for (int u = 0; u < kSpan; ++u) {
        const int k = k0 + u * 2 * kBlock;
        if (k < K) {
            load8(x + (size_t)m * ldx + k, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < kSpan; ++u) {
        const int k = k0 + u * 2 * kBlock;
        float a = absmax8(v[u]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
        const float s = a / kE4m3Max;
        if (k < K) {
            store8(q + (size_t)m * K + k, v[u], s);
            if ((lane & 15) == 0) scale[(size_t)(k / kBlock) * M + m] = s;
        }
    }
}

// One 128 x 128 block a CTA: sixteen lanes a row, sixteen rows at a time.
template <typename T>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const T* x, long long ldx, uint8_t* q, float* scale, int M,
                                                              int K, int kb) {
    __shared__ float part[8];
    chain_release();
    chain_wait();
    const int row0 = (int)(blockIdx.x / kb) * kBlock + (threadIdx.x >> 4);
    const int k = (int)(blockIdx.x % kb) * kBlock + (threadIdx.x & 15) * 8;
    float v[8][8], a = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int m = row0 + u * 16;
        if (m < M && k < K) {
            load8(x + (size_t)m * ldx + k, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) a = max_nan(a, absmax8(v[u]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) a = max_nan(a, part[i]);
    const float s = a / kE4m3Max;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int m = row0 + u * 16;
        if (m < M && k < K) store8(q + (size_t)m * K + k, v[u], s);
    }
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
}

template <typename T>
wdc_status launch(Ctx* c, const void* x, long long ldx, void* q, float* scale, int M, int K, int block_rows, cudaStream_t s) {
    const int kb = (K + kBlock - 1) / kBlock;
    const T* xt = reinterpret_cast<const T*>(x);
    uint8_t* qt = reinterpret_cast<uint8_t*>(q);
    const int spans = (K + kSpan * 2 * kBlock - 1) / (kSpan * 2 * kBlock);
    const long long grid = block_rows == 1 ? (long long)((M - 1) / 8 + 1) * spans : (long long)((M - 1) / kBlock + 1) * kb;
    if (grid > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "quantize: more than 2^31 - 1 thread blocks");
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_OTHER, s);
        if (block_rows == 1)
            launch_kernel(quantize_rows_kernel<T>, dim3((unsigned)grid), 256, 0, s, 1, xt, ldx, qt, scale, M, K, spans);
        else
            launch_kernel(quantize_blocks_kernel<T>, dim3((unsigned)grid), 256, 0, s, 1, xt, ldx, qt, scale, M, K, kb);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("quantize: ") + cudaGetErrorString(e));
    return WDC_OK;
}

}  // namespace

wdc_status op_quantize_fp8(Ctx* c, const void* x, long long ldx, void* q, float* scale, int M, int K, int block_rows,
                           cudaStream_t s) {
    if (M < 0 || K <= 0) return fail(c, WDC_ERR_INVALID_ARG, "quantize: M >= 0 and K > 0 wanted");
    if (block_rows != 1 && block_rows != kBlock) return fail(c, WDC_ERR_INVALID_ARG, "quantize: block_rows must be 1 or 128");
    if (ldx < K) return fail(c, WDC_ERR_INVALID_ARG, "quantize: row stride below K");
    if (K > kMaxWidth8) return fail(c, WDC_ERR_UNSUPPORTED, "quantize: more than 2^31 - 512 columns");
    if (K % 16 || ldx % 8) return fail(c, WDC_ERR_UNSUPPORTED, "quantize needs K % 16 == 0 and ldx % 8 == 0");
    if (M == 0) return WDC_OK;
    if (!x || !q || !scale) return fail(c, WDC_ERR_INVALID_ARG, "quantize: null pointer");
    if (((uintptr_t)x | (uintptr_t)q | (uintptr_t)scale) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "quantize: pointers must be 16-byte aligned");
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, x, ldx, q, scale, M, K, block_rows, s)
                                    : launch<float>(c, x, ldx, q, scale, M, K, block_rows, s);
}

}  // namespace wdc
