// The step between a block's halves, one pass over the rows:
//   r = x + gate * delta,   y = (r [- mean r]) / sqrt(mean (.)^2 + eps) * (weight + offset) + shift,
// with y in the model's type, in e4m3 with a scale for 128 columns, or in e2m1 with
// scales for 16 columns and the row.  A row's fp32 values stay in the registers of its
// warps from the sum to the last conversion (a layer norm's variance is that of the
// centred values), so that x and delta are read once.  Bound by memory: for bf16 6
// bytes an element and those of y (2, 1.03 or 0.56).
#include "quant.cuh"

namespace wdc {

namespace {

enum Out { kSame = 0, kE4m3 = 1, kE2m1 = 2 };

struct AddNormArgs {
    const void *x, *delta;
    void *total, *out;
    long long ldx, ldd, ldt, ldo;
    const float *weight, *shift, *gate;            // [sets][D]
    float offset, eps, by;                         // by: 1 / D
    int M, D, rows_per_set, center;
    float* scale;                                  // e4m3: [ceil(D / 128)][M]
    uint32_t* words;                               // e2m1: words of four scales
    float* row_scale;
};

constexpr int kHeld = 4;                           // pieces of 8 columns a thread holds at most
constexpr int kMaxThreads = 512;
constexpr int kMaxD = 8 * kHeld * kMaxThreads;

struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); }
};
// Over the blockDim.x threads of a row; every thread of the block calls it.  `part` is
// not in use by an earlier call any more.
template <class Op>
__device__ __forceinline__ float over_row(float a, float (*part)[16], Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = op(a, __shfl_xor_sync(0xffffffffu, a, o));
    if (blockDim.x == 32) return a;
    if ((threadIdx.x & 31) == 0) part[threadIdx.y][threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[threadIdx.y][0];
    for (int i = 1; i < (int)(blockDim.x >> 5); ++i) a = op(a, part[threadIdx.y][i]);
    return a;
}

template <typename T, int OUT, int V>
__global__ void __launch_bounds__(kMaxThreads) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
    __shared__ float part[3][8][16];
    chain_release();
    chain_wait();
    const int m = (int)(blockIdx.x * blockDim.y + threadIdx.y);
    const bool live = m < a.M;
    const size_t set = live && a.rows_per_set ? (size_t)(m / a.rows_per_set) * a.D : 0;
    auto column = [&](int u) { return (u * (int)blockDim.x + (int)threadIdx.x) * 8; };
    float v[V][8];
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int k = column(u);
        if (live && k < a.D) {
            load8(reinterpret_cast<const T*>(a.x) + (size_t)m * a.ldx + k, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        }
    }
    if (a.delta) {
        float d[V][8];
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (live && column(u) < a.D) load8(reinterpret_cast<const T*>(a.delta) + (size_t)m * a.ldd + column(u), d[u]);
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int k = column(u);
            if (!live || k >= a.D) continue;
            float g[8];
            if (a.gate) {
                load8(a.gate + set + k, g);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = 1.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = fmaf(g[i], d[u][i], v[u][i]);
        }
    }
    if (a.total) {
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (live && column(u) < a.D) put8(reinterpret_cast<T*>(a.total) + (size_t)m * a.ldt + column(u), v[u]);
    }
    if (a.center) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[u][i];
        const float mean = over_row(s, part[0], Sum()) * a.by;
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (column(u) < a.D) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] -= mean;
            }
    }
    float ss = 0.f;
#pragma unroll
    for (int u = 0; u < V; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(v[u][i], v[u][i], ss);
    const float inv = rsqrtf(over_row(ss, part[1], Sum()) * a.by + a.eps);
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int k = column(u);
        if (!live || k >= a.D) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] *= inv;
        if (a.weight) {
            float w[8];
            load8(a.weight + set + k, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] *= w[i] + a.offset;
        }
        if (a.shift) {
            float w[8];
            load8(a.shift + set + k, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] += w[i];
        }
    }
    if constexpr (OUT == kSame) {
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (live && column(u) < a.D) put8(reinterpret_cast<T*>(a.out) + (size_t)m * a.ldo + column(u), v[u]);
    } else if constexpr (OUT == kE4m3) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int k = column(u);
            float top = absmax8(v[u]);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float s = top / kE4m3Max;
            if (live && k < a.D) {
                store8(reinterpret_cast<uint8_t*>(a.out) + (size_t)m * a.D + k, v[u], s);
                if (k % 128 == 0) a.scale[(size_t)(k / 128) * a.M + m] = s;
            }
        }
    } else {
        float top = 0.f;
#pragma unroll
        for (int u = 0; u < V; ++u) top = max_nan(top, absmax8(v[u]));
        const float row = row_scale4(over_row(top, part[2], Max())), six = 6.f * row;
        const int pieces = a.D / kPieceCols4;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int k = column(u);
            uint32_t* codes =
                live && k < a.D ? reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(a.out) + ((size_t)m * a.D + k) / 2) : nullptr;
            uint32_t* word = k < a.D && k % kPieceCols4 == 0 ? a.words + piece_word4(m, k / kPieceCols4, pieces) : nullptr;
            store_fp4(v[u], row, six, codes, word);
            if (!live && word) *word = 0u;
        }
        if (live && threadIdx.x == 0) a.row_scale[m] = row;
    }
}

template <typename T, int OUT>
wdc_status launch(Ctx* c, const AddNormArgs& a, cudaStream_t s) {
    const int eights = a.D / 8;
    const int v = eights <= 32 ? 1 : (eights <= 128 ? 2 : kHeld);
    const int warps = (eights + 32 * v - 1) / (32 * v);
    const int per = warps >= 8 ? 1 : (warps >= 4 ? 2 : (warps >= 2 ? 4 : 8));
    // (e2m1: the rows behind M of the last 128 too, whose scales are zero)
    const long long rows = OUT == kE2m1 ? ((long long)(a.M - 1) / 128 + 1) * 128 : a.M;
    const dim3 block(32 * warps, per), grid((unsigned)((rows + per - 1) / per));
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_NORM, s);
        if (v == 1) launch_kernel(add_norm_kernel<T, OUT, 1>, grid, block, 0, s, 1, a);
        else if (v == 2) launch_kernel(add_norm_kernel<T, OUT, 2>, grid, block, 0, s, 1, a);
        else launch_kernel(add_norm_kernel<T, OUT, kHeld>, grid, block, 0, s, 1, a);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("residual norm: ") + cudaGetErrorString(e));
    return WDC_OK;
}

template <typename T>
wdc_status launch(Ctx* c, const AddNormArgs& a, int out, cudaStream_t s) {
    return out == kSame ? launch<T, kSame>(c, a, s) : (out == kE4m3 ? launch<T, kE4m3>(c, a, s) : launch<T, kE2m1>(c, a, s));
}

}  // namespace

wdc_status op_add_norm(Ctx* c, const wdc_add_norm* n, int M, int D, cudaStream_t s) {
    if (!n) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: no wdc_add_norm");
    if (M < 0 || D <= 0) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: M >= 0 and D > 0 wanted");
    if (D % 16 || D > kMaxD) return fail(c, WDC_ERR_UNSUPPORTED, "residual norm needs D % 16 == 0, at most 16384");
    if (M > kMaxRows4) return fail(c, WDC_ERR_UNSUPPORTED, "residual norm: more than 2^31 - 128 rows");
    if (!(n->eps >= 0.f)) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: eps must be >= 0");
    if (n->rows_per_set < 0) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: rows_per_set must be >= 0");
    const int kinds = (n->out != nullptr) + (n->q8 != nullptr) + (n->q4 != nullptr);
    if (kinds != 1) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: one of out, q8 and q4 is wanted");
    if (n->q4 && D % 64) return fail(c, WDC_ERR_UNSUPPORTED, "residual norm: e2m1 needs D % 64 == 0");
    if (n->gate && !n->delta) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: a gate without a branch");
    if (n->ldx < D || (n->delta && n->ldd < D) || (n->total && n->ldt < D) || (n->out && n->ldo < D))
        return fail(c, WDC_ERR_INVALID_ARG, "residual norm: row stride below D");
    if (n->ldx % 8 || (n->delta && n->ldd % 8) || (n->total && n->ldt % 8) || (n->out && n->ldo % 8))
        return fail(c, WDC_ERR_UNSUPPORTED, "residual norm: row strides must be multiples of 8");
    if (M == 0) return WDC_OK;
    if (!n->x || (n->q8 && !n->scale)) return fail(c, WDC_ERR_INVALID_ARG, "residual norm: null pointer");
    if (((uintptr_t)n->x | (uintptr_t)n->delta | (uintptr_t)n->total | (uintptr_t)n->out | (uintptr_t)n->q8 |
         (uintptr_t)n->scale | (uintptr_t)n->weight | (uintptr_t)n->shift | (uintptr_t)n->gate) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "residual norm: pointers must be 16-byte aligned");
    if (n->q4)
        if (wdc_status st = check_fp4(c, n->q4)) return st;
    AddNormArgs a{};
    a.x = n->x; a.ldx = n->ldx; a.delta = n->delta; a.ldd = n->ldd; a.total = n->total; a.ldt = n->ldt;
    a.weight = n->weight; a.shift = n->shift; a.gate = n->gate;
    a.offset = n->weight_offset; a.eps = n->eps; a.by = 1.0f / (float)D;
    a.M = M; a.D = D; a.rows_per_set = n->rows_per_set; a.center = n->center;
    int out = kSame;
    a.out = n->out;
    a.ldo = n->ldo;
    if (n->q8) {
        out = kE4m3;
        a.out = n->q8;
        a.scale = n->scale;
    } else if (n->q4) {
        out = kE2m1;
        a.out = n->q4->codes;
        a.words = (uint32_t*)n->q4->scale;
        a.row_scale = n->q4->row_scale;
    }
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, a, out, s) : launch<float>(c, a, out, s);
}

}  // namespace wdc
