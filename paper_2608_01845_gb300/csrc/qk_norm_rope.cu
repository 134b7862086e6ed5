// Norms of the query and key heads and their rotation by position, one pass
// from the rows of a QKV projection to what attention reads:
//   y = x / sqrt(mean(x^2) + eps) * w per head, then on its first rot elements
//   a' = a cos - b sin, b' = b cos + a sin for each pair (a, b).
// Bound by memory: each row is read once and written once, the angles of a
// token are read once for a few of its heads.  A lane holds 16 bytes of a head, so a
// head of 64 bf16 is 8 lanes and a sum over it three shuffles; a warp takes a run
// of one token's heads, kGroups warp-widths at a time, the next ones' loads under way
// while these are worked on (the angles are the token's: loaded once a run).  Sums, weights and angles are fp32; the one rounding is that
// of the result.
#include <type_traits>

#include "dit_kernels.cuh"
#include "paged_index.h"

namespace wdc {

namespace {

constexpr int kGroups = 4;
// Tokens of a V^T tile.  Of a long clip's (RUNS) as many as 32 KB of fp16 hold (17776 x 48 heads of 64: tiles
// of 64 tokens took 65 us beside the norms, of 128 48, of 256 43); of a shorter one's, whose tiles are to be
// on all SMs, 64.  (Tiles of 256 and 128 for every clip: 1350 tokens, 24 heads of 64 6.8 -> 8.4 us, 4 key heads of
// 64 3.9 -> 5.7, 24 of 128 11.0 -> 12.9; 17776 tokens, 24 of 64 69 -> 62, 48 of 64 133 -> 113.)
template <int D, bool RUNS>
constexpr int kVtTokens = RUNS ? 16384 / D : 64;

struct NormArgs {
    const void* qkv;
    long long ld;
    int T, heads, kv;
    int chunks;                        // of kGroups warp-widths, a token
    int per, runs;                     // chunks a warp takes; warps a token
    const float *wq, *wk;
    float eps;
    const float2* rot;                 // null: no rotation
    int rot_positions, rot_dim;
    const int* positions;
    // several axes: the pairs in sections, each with a table of its own
    int axes;
    const float2* axis_rot[4];
    int axis_rows[4], axis_end[4];     // rows of the table; the section's first pair behind it
    const int* coords;                 // [T][axes]
    void *q, *k, *v;
    int ldv;                           // dense: V^T's row stride
    unsigned vt_tiles;                 // dense: blocks that transpose V
    // append
    const int *table, *length, *start;
    int pages, page_log2, sequences, width;
    unsigned* err;
};

// A lane's elements of a head: 16 bytes in two halves, each of E / 2 neighbours.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
        const float4 a = *reinterpret_cast<const float4*>(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
    static __device__ __forceinline__ void load(const float* p, const float* q, float (&v)[4]) {
        const float2 a = *reinterpret_cast<const float2*>(p), b = *reinterpret_cast<const float2*>(q);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    }
    static __device__ __forceinline__ void widen(const uint4& u, float (&v)[4]) {
        v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
    static __device__ __forceinline__ void store(float* p, float* q, const float (&v)[4]) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        *reinterpret_cast<float2*>(q) = make_float2(v[2], v[3]);
    }
};
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void widen(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
// 16 bytes as they lie, in one piece or in two halves.
template <typename T> __device__ __forceinline__ uint4 load_bits(const T* p) { return *reinterpret_cast<const uint4*>(p); }
template <typename T> __device__ __forceinline__ uint4 load_bits(const T* p, const T* q) {
    const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(q);
    return make_uint4(a.x, a.y, b.x, b.y);
}
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&v)[8]) {
        widen(*reinterpret_cast<const uint4*>(p), v);
    }
    static __device__ __forceinline__ void widen(const uint4& u, float (&v)[8]) {
        wdc::widen(u.x, v[0], v[1]); wdc::widen(u.y, v[2], v[3]); wdc::widen(u.z, v[4], v[5]); wdc::widen(u.w, v[6], v[7]);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, __nv_bfloat16* q, const float (&v)[8]) {
        *reinterpret_cast<uint2*>(p) = make_uint2(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]));
        *reinterpret_cast<uint2*>(q) = make_uint2(bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
    }
};

// One tile of V^T: kTokens tokens of one head through shared memory.
template <typename T, int D, bool RUNS>
__device__ void transpose_v(const NormArgs& a, int tile) {
    using V = Vec<T>;
    using Out = typename std::conditional<sizeof(T) == 2, __half, float>::type;
    constexpr int kTokens = kVtTokens<D, RUNS>;
    constexpr int LDS = kTokens + 4 / (int)sizeof(Out);      // (an odd number of words: columns meet different banks)
    __shared__ alignas(16) Out sm[D * LDS];
    const int tiles = (a.T + kTokens - 1) / kTokens;
    const int head = tile / tiles, t0 = (tile - head * tiles) * kTokens;
    const int n = min(kTokens, a.T - t0);
    const T* src = reinterpret_cast<const T*>(a.qkv) + (size_t)(a.heads + a.kv + head) * D;
    bool sat = false;
    constexpr int PER = D / V::E, N = kTokens * PER / 256;   // lanes a token; pieces a thread
    float v[N][V::E];
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int i = u * 256 + threadIdx.x, t = i / PER;
        if (t < n) V::load(src + (size_t)(t0 + t) * a.ld + (i % PER) * V::E, v[u]);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int i = u * 256 + threadIdx.x, t = i / PER, e = (i % PER) * V::E;
        if (t < n) {
#pragma unroll
            for (int j = 0; j < V::E; ++j) {
                if constexpr (sizeof(T) == 2) sm[(e + j) * LDS + t] = to_vt_half(v[u][j], sat);
                else sm[(e + j) * LDS + t] = v[u][j];
            }
        }
    }
    if (sat) atomicOr(a.err, kErrVSaturated);
    __syncthreads();
    Out* dst = reinterpret_cast<Out*>(a.v) + (size_t)head * D * a.ldv + t0;
    if constexpr (sizeof(T) == 2) {
        constexpr int VEC = kTokens / 8;                     // 16-byte pieces a row
        for (int i = threadIdx.x; i < D * VEC; i += 256) {
            const int r = i / VEC, t = (i % VEC) * 8;
            const Out* s = sm + r * LDS + t;
            if (t + 8 <= n) {
                const uint32_t* w = reinterpret_cast<const uint32_t*>(s);
                *reinterpret_cast<uint4*>(dst + (size_t)r * a.ldv + t) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                for (int j = 0; t + j < n; ++j) dst[(size_t)r * a.ldv + t + j] = s[j];
            }
        }
    } else {
        for (int i = threadIdx.x; i < D * kTokens; i += 256) {
            const int r = i / kTokens, t = i % kTokens;
            if (t < n) dst[(size_t)r * a.ldv + t] = sm[r * LDS + t];
        }
    }
}

// What turns the heads: nothing or one table of positions, or a table for each axis.
// RUNS: a warp has several chunks (bf16).
template <typename T, int D, bool APPEND, bool PAIRS, bool AXES, bool RUNS>
__global__ void __launch_bounds__(256, RUNS ? 3 : 4) norm_rope_kernel(const __grid_constant__ NormArgs a) {
    using V = Vec<T>;
    constexpr int E = V::E, LPH = D / E, HPW = 32 / LPH;       // elements a lane, lanes a head, heads a warp-width
    chain_release();
    chain_wait();
    unsigned block = blockIdx.x;
    if (!APPEND && a.vt_tiles > 0) {
        // V^T's tiles among the blocks of norms, evenly: each kind waits for
        // memory at other times (one behind the other 133 us, mixed 124 at 17776 x 72 heads of 128)
        const unsigned v = (unsigned)((unsigned long long)block * a.vt_tiles / gridDim.x);
        if ((unsigned)((unsigned long long)(block + 1) * a.vt_tiles / gridDim.x) > v) {
            transpose_v<T, D, RUNS>(a, (int)v);
            return;
        }
        block -= v;
    }
    const int lane = threadIdx.x & 31;
    const long long w = (long long)block * 8 + (threadIdx.x >> 5);
    const long long tl = w / a.runs;
    if (tl >= a.T) return;
    const int t = (int)tl, chunk0 = (int)(w - tl * a.runs) * (RUNS ? a.per : 1);
    const int chunk1 = RUNS ? min(chunk0 + a.per, a.chunks) : chunk0 + 1;
    const int n_heads = APPEND ? a.heads + 2 * a.kv : a.heads + a.kv;
    const int half = a.rot_dim >> 1, l = lane % LPH;

    // This lane's elements of a head, in two halves whose element i makes a pair
    // (not interleaved), so that a pair is turned within a lane; what is not turned
    // lies behind.  Interleaved, or not turned at all, they are neighbours.
    int ea = l * E, eb = ea + E / 2;
    if (!PAIRS) {
        const int lanes = half / (E / 2);                      // that hold pairs
        ea = l < lanes ? l * (E / 2) : a.rot_dim + (l - lanes) * E;
        eb = l < lanes ? half + ea : ea + E / 2;
    }
    uint4 bits[kGroups];
    const T* row = reinterpret_cast<const T*>(a.qkv) + (size_t)t * a.ld;
    auto load = [&](int chunk) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int h = (chunk * kGroups + u) * HPW + lane / LPH;
            bits[u] = make_uint4(0u, 0u, 0u, 0u);
            if (h < n_heads) {
                if constexpr (PAIRS) bits[u] = load_bits(row + (size_t)h * D + ea);
                else bits[u] = load_bits(row + (size_t)h * D + ea, row + (size_t)h * D + eb);
            }
        }
    };
    // A chunk by itself of the dense form is widened at once (256 tokens of 24 + 24 heads of 128 3.24 us for 3.42,
    // 4050 18.8 for 19.4), other chunks as they are used (64 appended tokens of those 3.66 for 3.76).
    constexpr bool HELD = RUNS || APPEND;
    float wide[HELD ? 1 : kGroups][E];
    if constexpr (HELD) {
        load(chunk0);
    } else {
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int h = (chunk0 * kGroups + u) * HPW + lane / LPH;
            if (h < n_heads) {
                if constexpr (PAIRS) V::widen(load_bits(row + (size_t)h * D + ea), wide[u]);
                else V::widen(load_bits(row + (size_t)h * D + ea, row + (size_t)h * D + eb), wide[u]);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) wide[u][i] = 0.f;
            }
        }
    }

    // this token's place: its row of the cache and its position
    int place = t;
    bool keep = true;                                          // append: the token has a place in the cache
    size_t slot = 0;                                           // its page's first row * kv heads, and the row
    int in_page = 0;
    if constexpr (APPEND) {
        int b = 0;
        for (int i = 0; i < a.sequences; i += 32) {
            const bool mine = i + lane < a.sequences;
            const int end = mine ? a.start[i + lane + 1] : 0;
            const bool past = mine && end <= t;
            // (the first warp: each sequence's numbers, whether it has new tokens or not)
            if (w == 0 && mine && !paged_given(a.start[i + lane], end, a.length[i + lane], a.T, a.width << a.page_log2, a.T))
                atomicOr(a.err, kErrBounds);
            b += __popc(__ballot_sync(0xffffffffu, past));
        }
        if (b >= a.sequences) return;
        const PagedSeq seq = paged_seq(a.start[b], a.start[b + 1], a.length[b], a.T, a.width << a.page_log2);
        if (t < seq.row0 || t >= seq.row0 + seq.n) return;
        place = paged_place(seq, t - seq.row0);
        const int page = place < 0 ? -1 : paged_page(a.table[(size_t)b * a.width + (place >> a.page_log2)], a.pages);
        keep = page >= 0;
        if (!keep && lane == 0) atomicOr(a.err, kErrBounds);
        in_page = place & ((1 << a.page_log2) - 1);
        slot = keep ? (size_t)page * a.kv : 0;
    }

    // its angles, for the pairs of this lane
    float cs[E];                                               // cos, sin of each pair
    const bool turned = (AXES || a.rot) && ea < (PAIRS ? a.rot_dim : half);
    if constexpr (AXES) {
        // (the token, and so its place on each axis, is the same for the whole warp)
        const int first = PAIRS ? ea / 2 : ea;
        int begin = 0;
        for (int x = 0; x < a.axes; ++x) {
            const int end = a.axis_end[x];
            if (end == begin) continue;
            int p = a.coords[(size_t)t * a.axes + x];
            if (p < 0 || p >= a.axis_rows[x]) {
                if (lane == 0) atomicOr(a.err, kErrBounds);
                p = max(0, min(p, a.axis_rows[x] - 1));
            }
            const float2* r = a.axis_rot[x] + (size_t)p * (end - begin) - begin;
            if (turned) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i)
                    if (first + i >= begin && first + i < end) {
                        const float2 c = r[first + i];
                        cs[2 * i] = c.x;
                        cs[2 * i + 1] = c.y;
                    }
            }
            begin = end;
        }
    } else if (a.rot) {
        int p = a.positions ? a.positions[t] : place;
        if (p < 0 || p >= a.rot_positions) {
            if (lane == 0) atomicOr(a.err, kErrBounds);
            p = max(0, min(p, a.rot_positions - 1));
        }
        if (turned) {
            const float4* r = reinterpret_cast<const float4*>(a.rot + (size_t)p * half + (PAIRS ? ea / 2 : ea));
#pragma unroll
            for (int i = 0; i < E / 4; ++i) {
                const float4 c = r[i];
                cs[4 * i] = c.x; cs[4 * i + 1] = c.y; cs[4 * i + 2] = c.z; cs[4 * i + 3] = c.w;
            }
        }
    }

    for (int chunk = chunk0; chunk < chunk1; ++chunk) {
        uint4 now[kGroups];
        if constexpr (HELD) {
#pragma unroll
            for (int u = 0; u < kGroups; ++u) now[u] = bits[u];
            if (RUNS && chunk + 1 < chunk1) load(chunk + 1);
        }
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int h = (chunk * kGroups + u) * HPW + lane / LPH;
            float x[E], ss = 0.f;
            if constexpr (HELD) {
                V::widen(now[u], x);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = wide[u][i];
            }
#pragma unroll
            for (int i = 0; i < E; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
            for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (h >= n_heads) continue;
            auto put = [&](T* head, const float (&v)[E]) {
                if constexpr (PAIRS) V::store(head + ea, v);
                else V::store(head + ea, head + eb, v);
            };
            if (APPEND && h >= a.heads + a.kv) {
                const int g = h - a.heads - a.kv;
                bool sat = false;
                uint32_t p[E / 2];
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const __half2 v = __halves2half2(to_vt_half(x[i], sat), to_vt_half(x[i + 1], sat));
                    p[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
                }
                if (keep) {
                    __half* dst = reinterpret_cast<__half*>(a.v) + (((slot + g) << a.page_log2) + in_page) * D;
                    if constexpr (E == 8) {
                        if constexpr (PAIRS) {
                            *reinterpret_cast<uint4*>(dst + ea) = make_uint4(p[0], p[1], p[2], p[3]);
                        } else {
                            *reinterpret_cast<uint2*>(dst + ea) = make_uint2(p[0], p[1]);
                            *reinterpret_cast<uint2*>(dst + eb) = make_uint2(p[2], p[3]);
                        }
                    }
                    if (sat) atomicOr(a.err, kErrVSaturated);
                }
                continue;
            }
            const float inv = rsqrtf(ss * (1.0f / D) + a.eps);     // (2 ulp; IEEE's root and quotient are 30 instructions)
            float y[E];
            const float* wt = h < a.heads ? a.wq : a.wk;
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] = x[i] * inv;
            if (wt) {
                float f[E];
                if constexpr (E == 8) {
                    Vec<float>::load(wt + ea, *reinterpret_cast<float(*)[4]>(&f[0]));
                    Vec<float>::load(wt + eb, *reinterpret_cast<float(*)[4]>(&f[4]));
                } else {
                    Vec<float>::load(wt + ea, wt + eb, f);
                }
#pragma unroll
                for (int i = 0; i < E; ++i) y[i] *= f[i];
            }
            if (turned) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    float& p = y[PAIRS ? 2 * i : i];
                    float& q = y[PAIRS ? 2 * i + 1 : i + E / 2];
                    const float c = p, d = q;
                    p = c * cs[2 * i] - d * cs[2 * i + 1];
                    q = d * cs[2 * i] + c * cs[2 * i + 1];
                }
            }
            if (h < a.heads) {
                put(reinterpret_cast<T*>(a.q) + (APPEND ? (size_t)t * a.heads + h : (size_t)h * a.T + t) * D, y);
            } else {
                const int g = h - a.heads;
                if constexpr (APPEND) {
                    if (keep) put(reinterpret_cast<T*>(a.k) + (((slot + g) << a.page_log2) + in_page) * D, y);
                } else {
                    put(reinterpret_cast<T*>(a.k) + ((size_t)g * a.T + t) * D, y);
                }
            }
        }
    }
}

template <typename T, int D, bool APPEND>
wdc_status launch(Ctx* c, NormArgs& a, bool pairs, cudaStream_t s) {
    constexpr int HPW = 32 / (D / Vec<T>::E);
    const int n_heads = APPEND ? a.heads + 2 * a.kv : a.heads + a.kv;
    a.chunks = (n_heads + kGroups * HPW - 1) / (kGroups * HPW);
    // Runs of bf16 heads: as few a token as leave 62 runs an SM (which holds 24 at a time), where they come out of
    // equal length; of the dense form, whose tokens are looked up in no table, at most two and of three chunks
    // at least.  us with runs of 1, 2, 3 and all chunks, dense with V^T: 9600 tokens of 24 + 24 heads of
    // 64 40.1, 41.7, 36.4; 5000 of 48 + 48 41.9, 38.8, 37.5, 38.4; 5000 of 24 + 24 of 128 40.1, 41.8, 39.6,
    // 41.7 and 17776 127.9, 131.0, 122.6, 121.2; 9600 of 24 + 2 34.8, 34.5, 36.8 (3 and 1), 30.0, and 4050 12.9,
    // 14.1, 16.4, 14.9.  fp32 heads, twice the loads a chunk, lose: 9600 of 24 + 24 of 64 57.0, 63.3, 61.7, 61.3.
    a.per = 1;
    if constexpr (sizeof(T) == 2) {
        const long long want = 62ll * c->num_sms, fewest = (want + a.T - 1) / a.T;
        if (fewest < a.chunks && fewest <= (APPEND ? a.chunks : 2)) {
            const int per = (a.chunks + (int)fewest - 1) / (int)fewest;
            if (per >= (APPEND ? 2 : 3) && (a.chunks + per - 1) / per == fewest) a.per = per;
        }
    }
    a.runs = (a.chunks + a.per - 1) / a.per;
    const long long blocks = ((long long)a.T * a.runs + 7) / 8;
    const int vt_tokens = a.per > 1 ? kVtTokens<D, true> : kVtTokens<D, false>;
    const long long vt_tiles = !APPEND && a.v ? (long long)((a.T - 1) / vt_tokens + 1) * a.kv : 0;
    if (vt_tiles > 0x3fffffff) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation: more than 2^30 thread blocks");
    if (blocks + vt_tiles > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation: more than 2^31 - 1 thread blocks");
    a.vt_tiles = (unsigned)vt_tiles;
    const dim3 grid((unsigned)(blocks + vt_tiles));
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_NORM, s);
        auto go = [&](auto kernel) { launch_kernel(kernel, grid, 256, 0, s, 1, a); };
        auto of = [&](auto p, auto x) {
            constexpr bool P = decltype(p)::value, X = decltype(x)::value;
            if constexpr (sizeof(T) == 2) {
                if (a.per > 1) return go(norm_rope_kernel<T, D, APPEND, P, X, true>);
            }
            go(norm_rope_kernel<T, D, APPEND, P, X, false>);
        };
        if (a.axes > 0 && pairs) of(std::true_type(), std::true_type());
        else if (a.axes > 0) of(std::false_type(), std::true_type());
        else if (pairs) of(std::true_type(), std::false_type());
        else of(std::false_type(), std::false_type());
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("norm and rotation: ") + cudaGetErrorString(e));
    return WDC_OK;
}

// What both forms check and take over.
wdc_status take(Ctx* c, NormArgs& a, const void* qkv, long long ld, int T, int heads, int kv, int d, const wdc_head_norm* n,
                const wdc_rot_axes* axes) {
    if (!n) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: no wdc_head_norm");
    if (T < 0 || heads < 1 || kv < 1) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: T >= 0, heads and kv_heads >= 1 wanted");
    if (d != 64 && d != 128) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation: head_dim must be 64 or 128");
    if (ld < ((long long)heads + 2ll * kv) * d) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: row stride below (heads + 2 kv_heads) * d");
    if ((long long)heads + 2ll * kv > (1 << 20)) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation: too many heads");
    if (ld % 8) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation needs ld % 8 == 0");
    if (!(n->eps >= 0.f)) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: eps must be >= 0");
    if (n->rot && (n->rot_dim < 0 || n->rot_dim > d || n->rot_dim % 16 || n->rot_positions < 1))
        return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: rot_dim must be a multiple of 16 up to head_dim, rot_positions >= 1");
    if (T > 0 && !qkv) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: null pointer");
    if (((uintptr_t)qkv | (uintptr_t)n->q_weight | (uintptr_t)n->k_weight | (uintptr_t)n->rot) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: pointers must be 16-byte aligned");
    if (!axes && ((uintptr_t)n->positions & 3)) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: positions must be 4-byte aligned");
    a.qkv = qkv; a.ld = ld; a.T = T; a.heads = heads; a.kv = kv;
    a.wq = n->q_weight; a.wk = n->k_weight; a.eps = n->eps;
    a.rot = n->rot_dim > 0 ? reinterpret_cast<const float2*>(n->rot) : nullptr;
    a.rot_positions = n->rot_positions; a.rot_dim = a.rot ? n->rot_dim : 0; a.positions = n->positions;
    a.err = c->err;
    return WDC_OK;
}

// The axes, where there are some (null: the table of wdc_head_norm, or none).
wdc_status take_axes(Ctx* c, NormArgs& a, int d, const wdc_head_norm* n, const wdc_rot_axes* x) {
    if (!x) return WDC_OK;
    if (n->rot) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: a table of positions beside axes");
    if (x->axes < 1 || x->axes > 4) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: 1 to 4 axes wanted");
    long long pairs = 0;
    for (int i = 0; i < x->axes; ++i) {
        if (x->pairs[i] < 0) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: an axis' pairs must be >= 0");
        pairs += x->pairs[i];
        if (pairs > d / 2) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: the axes' pairs exceed head_dim / 2");
        a.axis_end[i] = (int)pairs;
        if (x->pairs[i] == 0) continue;                        // (its table and coordinates are not looked at)
        if (x->rows[i] < 1) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: an axis' table needs rows >= 1");
        if (a.T > 0 && (!x->table[i] || !x->coords)) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: null pointer");
        if ((uintptr_t)x->coords & 3) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: coords must be 4-byte aligned");
        if ((uintptr_t)x->table[i] & 7) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: an axis' table must be 8-byte aligned");
        a.axis_rot[i] = reinterpret_cast<const float2*>(x->table[i]);
        a.axis_rows[i] = x->rows[i];
    }
    if (pairs % 8) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: the axes' pairs must be a multiple of 8 in all");
    if (pairs == 0) return WDC_OK;                             // nothing is turned
    a.axes = x->axes;
    a.coords = x->coords;
    a.rot_dim = 2 * (int)pairs;
    return WDC_OK;
}

}  // namespace

wdc_status op_qk_norm_rope(Ctx* c, const void* qkv, long long ld, int T, int heads, int kv, int d, const wdc_head_norm* n,
                           const wdc_rot_axes* axes, void* q, void* k, void* vt, cudaStream_t s) {
    NormArgs a{};
    if (wdc_status st = take(c, a, qkv, ld, T, heads, kv, d, n, axes)) return st;
    if (wdc_status st = take_axes(c, a, d, n, axes)) return st;
    if (T == 0) return WDC_OK;
    if (!q || !k) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: null pointer");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)vt) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: pointers must be 16-byte aligned");
    const bool bf16 = c->cfg.dtype == WDC_BF16;
    if (bf16 && T > 0x7fffffff - 7) return fail(c, WDC_ERR_UNSUPPORTED, "norm and rotation: T too large");
    a.q = q; a.k = k; a.v = vt;
    a.ldv = bf16 ? (T + 7) / 8 * 8 : T;
    if (bf16)
        return d == 64 ? launch<__nv_bfloat16, 64, false>(c, a, n->interleaved, s)
                       : launch<__nv_bfloat16, 128, false>(c, a, n->interleaved, s);
    return d == 64 ? launch<float, 64, false>(c, a, n->interleaved, s)
                   : launch<float, 128, false>(c, a, n->interleaved, s);
}

wdc_status check_cache(Ctx* c, const wdc_paged_cache* p, int* page_log2) {
    if (c->cfg.dtype != WDC_BF16) return fail(c, WDC_ERR_UNSUPPORTED, "a paged cache needs a bf16 model");
    if (!p) return fail(c, WDC_ERR_INVALID_ARG, "paged cache: null pointer");
    if (p->head_dim != 64 && p->head_dim != 128) return fail(c, WDC_ERR_UNSUPPORTED, "paged cache: head_dim must be 64 or 128");
    int l = 4;
    while (l < 8 && (1 << l) != p->page) ++l;
    if ((1 << l) != p->page) return fail(c, WDC_ERR_UNSUPPORTED, "paged cache: a page must hold 16, 32, 64, 128 or 256 tokens");
    if (p->sequences < 0 || p->table_width < 1 || p->pages < 1 || p->kv_heads < 1)
        return fail(c, WDC_ERR_INVALID_ARG, "paged cache: sizes must be positive");
    if ((long long)p->table_width << l > (1ll << 30) || p->sequences > (1 << 24))
        return fail(c, WDC_ERR_UNSUPPORTED, "paged cache: a sequence may hold 2^30 tokens, a cache 2^24 sequences");
    if (!p->k || !p->v || !p->table || !p->length) {
        if (p->sequences > 0) return fail(c, WDC_ERR_INVALID_ARG, "paged cache: null pointer");
    }
    if (((uintptr_t)p->k | (uintptr_t)p->v) & 15) return fail(c, WDC_ERR_INVALID_ARG, "paged cache: k and v must be 16-byte aligned");
    if (((uintptr_t)p->table | (uintptr_t)p->length) & 3)
        return fail(c, WDC_ERR_INVALID_ARG, "paged cache: table and length must be 4-byte aligned");
    *page_log2 = l;
    return WDC_OK;
}

wdc_status op_qk_norm_rope_append(Ctx* c, const void* qkv, long long ld, int T, int heads, const wdc_head_norm* n,
                                  const wdc_rot_axes* axes, const wdc_paged_cache* p, const int* q_start, void* q,
                                  cudaStream_t s) {
    NormArgs a{};
    if (wdc_status st = check_cache(c, p, &a.page_log2)) return st;
    if (wdc_status st = take(c, a, qkv, ld, T, heads, p->kv_heads, p->head_dim, n, axes)) return st;
    if (wdc_status st = take_axes(c, a, p->head_dim, n, axes)) return st;
    if (T == 0 || p->sequences == 0) return WDC_OK;
    if (!q || !q_start) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: null pointer");
    if ((uintptr_t)q & 15) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: pointers must be 16-byte aligned");
    if ((uintptr_t)q_start & 3) return fail(c, WDC_ERR_INVALID_ARG, "norm and rotation: q_start must be 4-byte aligned");
    a.q = q; a.k = p->k; a.v = p->v;
    a.table = p->table; a.length = p->length; a.start = q_start;
    a.pages = p->pages; a.sequences = p->sequences; a.width = p->table_width;
    return p->head_dim == 64 ? launch<__nv_bfloat16, 64, true>(c, a, n->interleaved, s)
                             : launch<__nv_bfloat16, 128, true>(c, a, n->interleaved, s);
}

}  // namespace wdc
