// Rows to e2m1 with an e4m3 scale for 16 columns and an fp32 scale for the row, and
// back:
//   row   = max |x| / 2688 over the row,
//   s     = e4m3(max |x| / (6 row)) over 16 columns,  code = e2m1(x / (s row)),
//   value = code * (s * row).
// The row's scale needs the whole row before the first code: a row stays in the
// registers of its warps between the two, so x is read once.  Bound by memory (2.56
// bytes an element for bf16, 4.56 for fp32) where rows are fp32: 4276 x 12288 to codes 44
// us (5.5 TB/s; 48 with 4 pieces of 8 columns a thread) and back 38 (6.3).  bf16 rows are bound by their instructions, about
// 130 for 8 columns, 50 of them the conversions (two lanes work out each scale; 68% of the issue slots):
// 17776 x 4096 to codes 45 to 49 us (3.8 to 4.1 TB/s), back 29 (6.4); with 4 pieces of 8 columns a thread instead of 2, a row of fewer threads, 54 ->
// 49.  4 x 5120: 1.8 us either way, a launch.
#include <type_traits>

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

constexpr int kHeld = 4;                           // pieces of 8 columns a thread holds at most
constexpr int kMaxThreads = 512;                   // of a row of bf16; of fp32, twice as many with half the pieces
template <typename T>
constexpr int kRowThreads = sizeof(T) == 2 ? kMaxThreads : 2 * kMaxThreads;
constexpr int kRowsAtOnce = 8;                     // of a block whose rows have a warp each

__device__ __forceinline__ float warp_max(float a) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}

// A block takes rows a grid apart: one at a time with all its threads, or (blockDim.y ==
// kRowsAtOnce) one a warp; a thread has V pieces of 8 columns, and the next row's loads
// are under way while one is worked on.  Rows past M (of the last 128) get scales of zero.
template <typename T, int V>
__global__ void __launch_bounds__(kRowThreads<T>) quantize4_kernel(const __grid_constant__ Quant4Args a) {
    __shared__ float tops[2][32];
    chain_release();
    chain_wait();
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const unsigned step = gridDim.x * blockDim.y, M = a.M, rows = (M + 127) / 128 * 128;   // (a row and a step: below 2^32)
    int col[V];
#pragma unroll
    for (int u = 0; u < V; ++u) col[u] = (u * (int)blockDim.x + (int)threadIdx.x) * 8;
    const bool wide = is_wide(a.x);
    Raw8<T> raw[V];
    auto load = [&](unsigned m) {
        if (m >= M) return;
        const T* x = reinterpret_cast<const T*>(a.x) + (size_t)m * a.ldx;
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (col[u] < a.K) load_raw(x + col[u], raw[u], wide);
    };
    unsigned m = blockIdx.x * blockDim.y + threadIdx.y;
    int parity = 0;
    load(m);
    for (; m < M; m += step, parity ^= 1) {
        float v[V][8], top8[V], top = 0.f;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if (col[u] < a.K) {
                widen8(raw[u], v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
            }
        }
        load(m + step);
#pragma unroll
        for (int u = 0; u < V; ++u) top = max_nan(top, top8[u] = absmax8(v[u]));
        top = warp_max(top);
        if (warps > 1) {
            if (lane == 0) tops[parity][threadIdx.x >> 5] = top;
            __syncthreads();
            top = warp_max(lane < warps ? tops[parity][lane] : 0.f);
        }
        const Row4 row(top);
        uint8_t* codes = a.codes + (size_t)m * (unsigned)a.K / 2;
        uint32_t* words = a.scale + piece_word4((int)m, 0, a.pieces);
#pragma unroll
        for (int u = 0; u < V; ++u)
            store_fp4(v[u], top8[u], row, col[u] < a.K, reinterpret_cast<uint32_t*>(codes + col[u] / 2),
                      words + (size_t)(col[u] / kPieceCols4) * (kPiece4 / 4));
        if (threadIdx.x == 0) a.row_scale[m] = row.row;
    }
    for (; m < rows; m += step)
        for (int p = threadIdx.x; p < a.pieces; p += blockDim.x) a.scale[piece_word4((int)m, p, a.pieces)] = 0u;
}

// Rows wider than a block's registers: read twice, the second time from L2.
template <typename T>
__global__ void __launch_bounds__(512) quantize4_wide_kernel(const __grid_constant__ Quant4Args a) {
    __shared__ float tops[16];
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
    top = warp_max(top);
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    for (int w = 0; w < 16; ++w) top = max_nan(top, tops[w]);
    const Row4 row(top);
    for (long long k0 = 0; k0 < a.K; k0 += blockDim.x * 8) {        // (whole warps: the lanes trade scales)
        const long long k = k0 + threadIdx.x * 8;
        if (k < a.K) {
            load8(x + k, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        }
        store_fp4(v, absmax8(v), row, k < a.K, reinterpret_cast<uint32_t*>(a.codes + ((size_t)m * a.K + k) / 2),
                  a.scale + piece_word4(m, (int)(k / kPieceCols4), a.pieces));
    }
    if (threadIdx.x == 0) a.row_scale[m] = row.row;
}

// 16 bytes of x a thread, in kBackRows rows blockDim.y apart.
constexpr int kBackRows = 4;
template <typename T>
__global__ void __launch_bounds__(256) dequantize4_kernel(const uint8_t* codes, const uint8_t* scale, const float* row_scale,
                                                          T* x, long long ldx, int M, int K, int pieces, int segments) {
    constexpr int E = 16 / (int)sizeof(T);
    using Codes = typename std::conditional<E == 8, uint32_t, uint16_t>::type;
    chain_release();
    chain_wait();
    const int k = ((int)(blockIdx.x % segments) * (int)blockDim.x + (int)threadIdx.x) * E;
    if (k >= K) return;
    const unsigned m0 = blockIdx.x / segments * (blockDim.y * kBackRows) + threadIdx.y;
    Codes q[kBackRows];
    uint8_t s[kBackRows];
    float r[kBackRows];
#pragma unroll
    for (int i = 0; i < kBackRows; ++i) {
        const unsigned m = m0 + i * blockDim.y;
        if (m >= (unsigned)M) continue;
        q[i] = *reinterpret_cast<const Codes*>(codes + ((size_t)m * K + k) / 2);
        s[i] = scale[4 * piece_word4((int)m, k / kPieceCols4, pieces) + (k / 16) % 4];
        r[i] = row_scale[m];
    }
#pragma unroll
    for (int i = 0; i < kBackRows; ++i) {
        const unsigned m = m0 + i * blockDim.y;
        if (m >= (unsigned)M) continue;
        const float step = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)s[i], __NV_E4M3))) * r[i];
        float v[8];
        e2m1_values(q[i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= step;
        T* to = x + (size_t)m * ldx + k;
        if constexpr (E == 8) put8(to, v);
        else *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    }
}

template <typename T, int V>
void launch_held(Ctx* c, const Quant4Args& a, int warps, cudaStream_t s) {
    const int per = warps == 1 ? kRowsAtOnce : 1;
    const long long rows = ((long long)(a.M - 1) / 128 + 1) * 128, blocks = (rows + per - 1) / per;
    static PerDevice<int> held[33];
    const int most = held[warps].get(c->device, [&](int& n) {
        n = resident_blocks(c, quantize4_kernel<T, V>, 32 * warps * per);
        return true;
    });
    launch_kernel(quantize4_kernel<T, V>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(32 * warps, per), 0, s, 1, a);
}

template <typename T>
wdc_status launch(Ctx* c, const Quant4Args& a, cudaStream_t s) {
    const int eights = a.K / 8;                    // (bf16: wide threads, see above; fp32's hold twice the registers)
    const int most = sizeof(T) == 2 ? kHeld : 2;
    const int v = eights <= 32 ? 1 : (eights <= 64 ? 2 : most), warps = (eights + 32 * v - 1) / (32 * v);
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_OTHER, s);
        if (eights > most * kRowThreads<T>)                  // (a block a row, those behind M of the last 128 too)
            launch_kernel(quantize4_wide_kernel<T>, dim3(((unsigned)a.M + 127) / 128 * 128), 512, 0, s, 1, a);
        else if (v == 1) launch_held<T, 1>(c, a, warps, s);
        else if (v == 2) launch_held<T, 2>(c, a, warps, s);
        else if constexpr (sizeof(T) == 2) launch_held<T, kHeld>(c, a, warps, s);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 quantize: ") + cudaGetErrorString(e));
    return WDC_OK;
}

template <typename T>
wdc_status launch_back(Ctx* c, const wdc_fp4& q, T* x, long long ldx, int M, int K, cudaStream_t s) {
    const int across = K / (16 / (int)sizeof(T));
    int tx = 8;
    while (tx < across && tx < 256) tx *= 2;
    const int ty = 256 / tx, segments = (across + tx - 1) / tx;
    const long long blocks = ((long long)(M - 1) / (ty * kBackRows) + 1) * segments;
    if (blocks > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 dequantize: more than 2^31 - 1 thread blocks");
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_OTHER, s);
        launch_kernel(dequantize4_kernel<T>, dim3((unsigned)blocks), dim3(tx, ty), 0, s, 1, (const uint8_t*)q.codes,
                      (const uint8_t*)q.scale, (const float*)q.row_scale, x, ldx, M, K, K / kPieceCols4, segments);
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
