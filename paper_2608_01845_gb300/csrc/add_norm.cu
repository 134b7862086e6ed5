// The step between a block's halves, one pass over the rows:
//   r = x + gate * delta,   y = (r [- mean r]) / sqrt(mean (.)^2 + eps) * (weight + offset) + shift,
// with y in the model's type, in e4m3 with a scale for 128 columns, or in e2m1 with
// scales for 16 columns and the row.  A row's fp32 values stay in the registers of its
// warps from the sum to the last conversion (a layer norm's variance is that of the
// centred values), so that x and delta are read once.  Bound by memory: for bf16 6
// bytes an element and those of y (2, 1.03 or 0.56).  17776 x 5120 with a gated branch,
// root-mean-square norm, to bf16: 119.5 us (6.1 TB/s); 4050 x 4096 layer norm with gate,
// weight and shift by frame to e4m3: 28 us in L2, 33 from memory (3.5 TB/s), where a row's
// chain (two sums, a root, two conversions) is what a short call waits for: without the
// three vectors 24.  To e2m1, with a second meeting of the warps for the row's maximum, 32 us in L2 and
// 35 from memory; 17776 x 5120 154 us, its conversions' instructions.  Rows pass L1 by, which keeps the vectors: 32 -> 28 us.  Two pieces of 8
// columns a thread: with four, and so fewer rows at a time, 17776 x 5120 took 167 us.
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
constexpr int kMaxThreads = 512;                   // of a row
constexpr int kRowsAtOnce = 8;                     // of a block whose rows have a warp each
constexpr int kMaxD = 8 * kHeld * kMaxThreads;

// A block takes rows a grid apart: one at a time with all its threads, or (blockDim.y ==
// kRowsAtOnce) one a warp; a thread has V pieces of 8 columns, and the next row's loads
// are under way while one is worked on.  The warps of a row meet once for its
// statistics: each brings the mean of its own values and the squares around it, which join
// exactly as those of the whole row would be formed (the squares around the row's mean
// are those plus n (mean - row's mean)^2 a warp).
template <typename T, int OUT, int V>
__global__ void __launch_bounds__(kMaxThreads) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
    __shared__ float2 stat[2][kMaxThreads / 32];
    __shared__ float tops[2][kMaxThreads / 32];
    chain_release();
    chain_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const unsigned step = gridDim.x * blockDim.y, M = a.M; // (unsigned: a row and a step stay below 2^32)
    // (e2m1: the rows behind M of the last 128 too, whose scales are zero)
    const unsigned rows = OUT == kE2m1 ? (M + 127) / 128 * 128 : M;
    int col[V];
#pragma unroll
    for (int u = 0; u < V; ++u) col[u] = (u * (int)blockDim.x + (int)threadIdx.x) * 8;
    auto count = [&](int w) {                              // a warp's columns
        int n = 0;
#pragma unroll
        for (int u = 0; u < V; ++u) n += max(0, min(256, a.D - (u * (int)blockDim.x + w * 32) * 8));
        return (float)n;
    };
    const float n = count(warp), by_n = n > 0.f ? 1.0f / n : 0.f;
    const int other = lane & 15;                           // the warp whose statistics this lane joins
    const float n_other = other < warps ? count(other) : 0.f;
    const bool wide_rows = is_wide(a.x) && is_wide(a.delta) && is_wide(a.total) && is_wide(a.out);
    const bool wide_sets = is_wide(a.gate) && is_wide(a.weight) && is_wide(a.shift);
    Raw8<T> xr[V], dr[V];
    auto load = [&](unsigned m) {
        if (m >= M) return;
        const T* x = reinterpret_cast<const T*>(a.x) + (size_t)m * a.ldx;
        const T* d = reinterpret_cast<const T*>(a.delta) + (size_t)m * a.ldd;
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (col[u] < a.D) {
                load_once(x + col[u], xr[u], wide_rows);
                if (a.delta) load_once(d + col[u], dr[u], wide_rows);
            }
    };
    unsigned m = blockIdx.x * blockDim.y + threadIdx.y;
    int parity = 0;
    load(m);
    for (; m < rows; m += step, parity ^= 1) {
        const bool live = m < M;
        const size_t set = live && a.rows_per_set ? (size_t)(m / (unsigned)a.rows_per_set) * a.D : 0;
        float v[V][8];
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if (live && col[u] < a.D) {
                widen8(xr[u], v[u]);
                if (a.delta) {
                    float d[8], g[8];
                    widen8(dr[u], d);
                    if (a.gate) {
                        load8(a.gate + set + col[u], g, wide_sets);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) g[i] = 1.f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[u][i] = fmaf(g[i], d[i], v[u][i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
            }
        }
        load(m + step);
        if (a.total && live) {
            T* total = reinterpret_cast<T*>(a.total) + (size_t)m * a.ldt;
#pragma unroll
            for (int u = 0; u < V; ++u)
                if (col[u] < a.D) put8(total + col[u], v[u], wide_rows);
        }
        float mean = 0.f, ss = 0.f;
        if (a.center) {
#pragma unroll
            for (int u = 0; u < V; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) mean += v[u][i];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
            mean *= by_n;
        }
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (col[u] < a.D) {
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(v[u][i] - mean, v[u][i] - mean, ss);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (warps > 1) {
            if (lane == 0) stat[parity][warp] = make_float2(mean, ss);
            __syncthreads();
            const float2 s = other < warps ? stat[parity][other] : make_float2(0.f, 0.f);
            ss = s.y;
            if (a.center) {
                mean = s.x * n_other;
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
                mean *= a.by;
                ss = fmaf(n_other * (s.x - mean), s.x - mean, ss);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        }
        const float inv = rsqrtf(ss * a.by + a.eps);
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if (!live || col[u] >= a.D) continue;
            if (a.center) {
                // (the difference first: v inv - mean inv in one step adds mean inv's rounding, so that a row of
                // 100.5s, whose mean is exact, came out as up to 4e-3 instead of 0 with eps 1e-6)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = (v[u][i] - mean) * inv;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] *= inv;
            }
            if (a.weight) {
                float w[8];
                load8(a.weight + set + col[u], w, wide_sets);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] *= w[i] + a.offset;
            }
            if (a.shift) {
                float w[8];
                load8(a.shift + set + col[u], w, wide_sets);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] += w[i];
            }
        }
        if constexpr (OUT == kSame) {
            T* out = reinterpret_cast<T*>(a.out) + (size_t)m * a.ldo;
#pragma unroll
            for (int u = 0; u < V; ++u)
                if (live && col[u] < a.D) put8(out + col[u], v[u], wide_rows);
        } else if constexpr (OUT == kE4m3) {
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const int k = col[u];
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
            float tops8[V], top = 0.f;
#pragma unroll
            for (int u = 0; u < V; ++u) top = max_nan(top, tops8[u] = absmax8(v[u]));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (warps > 1) {
                if (lane == 0) tops[parity][warp] = top;
                __syncthreads();
                top = other < warps ? tops[parity][other] : 0.f;
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            }
            const Row4 row(top);
            uint8_t* codes = reinterpret_cast<uint8_t*>(a.out) + (size_t)m * a.D / 2;
            uint32_t* words = a.words + piece_word4((int)m, 0, a.D / kPieceCols4);
#pragma unroll
            for (int u = 0; u < V; ++u) {
                uint32_t* word = words + (size_t)(col[u] / kPieceCols4) * (kPiece4 / 4);
                store_fp4(v[u], tops8[u], row, live && col[u] < a.D, reinterpret_cast<uint32_t*>(codes + col[u] / 2), word);
                if (!live && col[u] < a.D && col[u] % kPieceCols4 == 0) *word = 0u;
            }
            if (live && threadIdx.x == 0) a.row_scale[m] = row.row;
        }
    }
}

template <typename T, int OUT, int V>
wdc_status launch(Ctx* c, const AddNormArgs& a, int warps, cudaStream_t s) {
    const int per = warps == 1 ? kRowsAtOnce : 1;
    const long long rows = OUT == kE2m1 ? ((long long)(a.M - 1) / 128 + 1) * 128 : a.M;
    const long long blocks = (rows + per - 1) / per;
    static PerDevice<int> held[kMaxThreads / 32 + 1];
    const int most = held[warps].get(c->device, [&](int& n) {
        n = resident_blocks(c, add_norm_kernel<T, OUT, V>, 32 * warps * per);
        return true;
    });
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_NORM, s);
        launch_kernel(add_norm_kernel<T, OUT, V>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(32 * warps, per), 0, s, 1, a);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("residual norm: ") + cudaGetErrorString(e));
    return WDC_OK;
}

template <typename T, int OUT>
wdc_status launch(Ctx* c, const AddNormArgs& a, cudaStream_t s) {
    const int eights = a.D / 8;
    const int v = eights <= 32 ? 1 : (eights <= 2 * kMaxThreads ? 2 : kHeld);
    const int warps = (eights + 32 * v - 1) / (32 * v);
    return v == 1 ? launch<T, OUT, 1>(c, a, warps, s) : (v == 2 ? launch<T, OUT, 2>(c, a, warps, s) : launch<T, OUT, kHeld>(c, a, warps, s));
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
    // Places: an output over an input is its rows, read and written by the same threads; of the others each is
    // one of its own (a block writes a row while others still read theirs).
    const void* few[] = {n->q8, n->q8 ? n->scale : nullptr, n->q4 ? n->q4->codes : nullptr, n->q4 ? n->q4->scale : nullptr,
                         n->q4 ? n->q4->row_scale : nullptr};
    for (const void* p : few)
        if (p && (p == n->x || p == n->delta || p == n->total))
            return fail(c, WDC_ERR_INVALID_ARG, "residual norm: a result in few bits needs a place of its own");
    if (n->total && n->total == n->out)
        return fail(c, WDC_ERR_INVALID_ARG, "residual norm: total and the result must be two places");
    auto shifted = [&](const void* p, long long ld) {
        return M > 1 && p && ((p == n->x && ld != n->ldx) || (p == n->delta && ld != n->ldd));
    };
    if (shifted(n->out, n->ldo) || shifted(n->total, n->ldt))
        return fail(c, WDC_ERR_INVALID_ARG, "residual norm: an output over an input must have its row stride");
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
