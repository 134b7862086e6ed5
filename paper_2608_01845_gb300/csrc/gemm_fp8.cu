// Product of e4m3 matrices with block scales on the 5th-generation tensor cores
// (tcgen05 kind::f8f6f4, sm_103a):
//   C[m, n] = epilogue( sum_b sa[b][m] sw[n / 128][b] sum_{k in block b} A[m, k] W[n, k] ),
// blocks of 128 columns of K.  A block is one 128-byte row of the swizzled
// shared-memory tiles and four MMAs (32 of K each) into tensor memory, started
// from zero; the epilogue warps then add that product, times its scales, to sums in
// their registers, while the next blocks' MMAs fill the other buffers.  So a
// sum over K is fp32 beyond a block, whatever the scales.  This file: the entry, the
// choice of the kernel, and the kernel for few rows; gemm_fp8_pair.cu: many rows.
#include "gemm_fp8.cuh"

#include <cmath>

namespace wdc {

namespace {

constexpr int kBlock = kBlock8;
constexpr int kThreads = 192;           // TMA producer, MMA issuer, 4 epilogue warps

__device__ __forceinline__ void epilogue_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// ---------------------------------------------------------------------------
// W's rows as the MMA's M side (128 of them a tile), BN rows of A as its N side:
// a few tokens then cost a narrow MMA instead of a mostly empty one, and a
// warp's lanes are neighbouring columns of C, which it stores without staging.
// A cluster of `split` CTAs shares a tile's K: each sums its blocks, sends the
// others their share of the tile's tokens through distributed shared memory and
// adds what it receives in rank order.
// A round of the issuer (two waits, four MMAs, two commits) takes about 500 cycles
// however narrow the MMAs are, so a stage of the ring, and a TMEM buffer, holds two
// blocks, and one lane runs the issuer's loop (4 x 3072 x 12288 in one piece: 31 us,
// with one lane 26, with both 18).  Ring and buffers are as many as one CTA an SM may
// have where no SM needs two.
constexpr int kMaxStages = 11;
template <int BN>
struct NarrowCfg {
    static constexpr int KB = 2;                           // blocks a stage
    static constexpr uint32_t W_BYTES = 128 * kBlock, A_BYTES = BN * kBlock, BLOCK = W_BYTES + A_BYTES, STAGE = KB * BLOCK;
    static constexpr int BUFS = 256 / (KB * BN);           // (twice as many alone)
    static constexpr uint32_t IDESC = idesc_e4m3(128, BN);
    static constexpr int WINDOW = 16;                      // blocks whose scales are in shared memory at a time
    static constexpr uint32_t WINDOW_BYTES = 2 * WINDOW * BN * 4;
    static constexpr size_t FIXED = WINDOW_BYTES + 1024 + 512;
    static constexpr size_t smem(int stages) { return (size_t)stages * STAGE + FIXED; }
    static constexpr int fit(size_t bytes) {
        return (int)((bytes - FIXED) / STAGE) < kMaxStages ? (int)((bytes - FIXED) / STAGE) : kMaxStages;
    }
    static constexpr int DEEP = fit(227 * 1024), SHARED = fit(113 * 1024);   // one CTA an SM, two
    static_assert(BN * 128 * 4 <= SHARED * STAGE, "partial sums fit the ring");
    static_assert(WINDOW % KB == 0, "whole stages a window");
};

template <typename T, int BN>
__global__ void __launch_bounds__(kThreads, 2)
    gemm8_narrow_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                        const __grid_constant__ Gemm8Args g) {
    using C = NarrowCfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stages = g.stages, bufs = g.bufs;
    float* window = reinterpret_cast<float*>(smem + stages * C::STAGE);     // [2][WINDOW][BN]
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + stages * C::STAGE + C::WINDOW_BYTES);
    uint64_t* empty = full + stages;
    uint64_t* tfull = empty + stages;
    uint64_t* tempty = tfull + bufs;
    uint64_t* mma_done = tempty + bufs;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = g.split, rank = S > 1 ? (int)cluster_ctarank() : 0;
    const int tile = blockIdx.x / S;
    const int m0 = (tile % g.m_tiles) * BN, nb = tile / g.m_tiles;             // neighbouring tiles share W
    const int units = (g.kb + C::KB - 1) / C::KB;          // stages' worth of blocks
    const int kb0 = (int)((long long)rank * units / S) * C::KB;
    const int kb1 = min((int)((long long)(rank + 1) * units / S) * C::KB, g.kb);
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < bufs; ++b) {
            mbar_init(&tfull[b], 1);
            mbar_init(&tempty[b], 4);
        }
        mbar_init(mma_done, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmA);
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, (uint32_t)(bufs * C::KB * BN));
        tmem_relinquish();
    }
    __syncthreads();
    tc_fence_after();
    chain_release();
    chain_wait();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0, armed = 0, parity = 0;         // per stage: a copy was issued; its phase
        for (int kb = kb0; kb < kb1; kb += C::KB) {        // (columns past K are filled with zeros)
            if (!mbar_wait_warp(&empty[stage], phase ^ 1u, abort_flag, g.err)) break;
            if (elect_one()) {
                mbar_arrive_expect_tx(&full[stage], C::STAGE);
#pragma unroll
                for (int i = 0; i < C::KB; ++i) {
                    uint8_t* sw = smem + stage * C::STAGE + i * C::BLOCK;
                    tma_load_2d(sw, &tmW, &full[stage], (kb + i) * kBlock, nb * 128);
                    tma_load_2d(sw + C::W_BYTES, &tmA, &full[stage], (kb + i) * kBlock, m0);
                }
            }
            __syncwarp();
            armed |= 1u << stage;
            parity = (parity & ~(1u << stage)) | (phase << stage);
            if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        // every issued copy has landed before the ring is reused or the CTA exits
        for (int s = 0; s < stages; ++s) {
            if (!((armed >> s) & 1)) continue;
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(&full[s], (parity >> s) & 1) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint64_t dw = sdesc_sw128(smem_u32(smem)), da = sdesc_sw128(smem_u32(smem) + C::W_BYTES);
            int stage = 0, buf = 0;
            uint32_t phase = 0, bphase = 0;
            for (int kb = kb0; kb < kb1; kb += C::KB) {
                if (!mbar_wait(&tempty[buf], bphase ^ 1u, abort_flag, g.err)) break;
                if (!mbar_wait(&full[stage], phase, abort_flag, g.err)) break;
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < C::KB; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma8(tmem + (uint32_t)((buf * C::KB + i) * BN),
                                sdesc_at(dw, stage * C::STAGE + i * C::BLOCK + k * 32),
                                sdesc_at(da, stage * C::STAGE + i * C::BLOCK + k * 32), C::IDESC, k != 0);
                tc_commit(&empty[stage]);
                tc_commit(&tfull[buf]);
                if (++stage == stages) { stage = 0; phase ^= 1u; }
                if (++buf == bufs) { buf = 0; bphase ^= 1u; }
            }
            // all MMAs issued by this lane have completed before TMEM is freed
            tc_commit(mma_done);
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(mma_done, 0) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
        __syncwarp();
    }

    float acc[BN];
    bool ok = true;
    const int lg = warp & 3;                               // TMEM lane quarter this warp may access
    if (warp >= 2) {
        const int tid = threadIdx.x - 64;
        const uint32_t lanes = tmem + ((uint32_t)(lg * 32) << 16);
        // scales sa * sw of the next WINDOW blocks: each thread fetches and
        // multiplies its own, then all meet
        auto fetch = [&](int w) {
            float* dst = window + (w & 1) * C::WINDOW * BN;
            for (int i = tid; i < C::WINDOW * BN; i += 128) {
                const int kb = kb0 + w * C::WINDOW + i / BN, m = m0 + i % BN;
                if (kb < kb1 && m < g.M) cp_async4(dst + i, g.sa + (size_t)kb * g.M + m);
                else dst[i] = 0.f;
            }
        };
        fetch(0);
#pragma unroll
        for (int c = 0; c < BN; ++c) acc[c] = 0.f;
        int buf = 0;
        uint32_t bphase = 0;
        int at = 0, w = 0;                                 // the stage's first block in its window; the window
        for (int kb = kb0; kb < kb1; kb += C::KB) {
            if (at == 0) {
                float* own = window + (w & 1) * C::WINDOW * BN;
                cp_async_wait();
                for (int i = tid; i < C::WINDOW * BN; i += 128) {
                    const int b = kb + i / BN;
                    if (b < kb1) own[i] *= ld_chain(g.sw + (size_t)nb * g.kb + b);
                }
                epilogue_barrier();
                if (kb + C::WINDOW < kb1) fetch(w + 1);
            }
            const float4* s4 = reinterpret_cast<const float4*>(window + ((w & 1) * C::WINDOW + at) * BN);
            ok = ok && mbar_wait_warp(&tfull[buf], bphase, abort_flag, g.err);
            __syncwarp();                                  // (after a wait that gave up nothing else does)
            tc_fence_after();
            constexpr int CH = BN < 32 ? BN : 32, COLS = C::KB * BN;        // columns a load; of the buffer
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += CH) {
                uint32_t p[CH];
                if constexpr (CH == 16) tmem_ld16(lanes + (uint32_t)(buf * COLS + c0), p);
                else tmem_ld32(lanes + (uint32_t)(buf * COLS + c0), p);
                tmem_ld_wait();
                if (c0 + CH == COLS) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&tempty[buf]);
                }
#pragma unroll
                for (int c = 0; c < CH; c += 4) {
                    const float4 s = s4[(c0 + c) / 4];
                    const int a = (c0 + c) % BN;
                    acc[a] = fmaf(__uint_as_float(p[c]), s.x, acc[a]);
                    acc[a + 1] = fmaf(__uint_as_float(p[c + 1]), s.y, acc[a + 1]);
                    acc[a + 2] = fmaf(__uint_as_float(p[c + 2]), s.z, acc[a + 2]);
                    acc[a + 3] = fmaf(__uint_as_float(p[c + 3]), s.w, acc[a + 3]);
                }
            }
            if (++buf == bufs) { buf = 0; bphase ^= 1u; }
            if ((at += C::KB) == C::WINDOW) { at = 0; ++w; }
        }
    }
    // this CTA's copies have landed and its MMAs are done
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, (uint32_t)(bufs * C::KB * BN));
    }
    const int row = lg * 32 + lane, n = nb * 128 + row;
    const bool mine = warp >= 2 && ok && n < g.N;
    float bias = 0.f, gate = 1.f;
    if (mine) {
        if (g.bias) bias = ld_chain(g.bias + n);
        if (g.gate) gate = ld_chain(g.gate + n);
    }
    // residuals are fetched before the first result is stored (C may be where they lie,
    // so the compiler leaves each load behind the store before it)
    const T* res = reinterpret_cast<const T*>(g.res);
    auto fetch_res = [&](int c) {
        const int m = m0 + c;
        return g.res && mine && m < g.M ? ld_act<T>(res + (size_t)m * g.N + n) : 0.f;
    };
    auto put = [&](int c, float v, float r) {
        const int m = m0 + c;
        if (!mine || m >= g.M) return;
        v += bias;
        if (g.gelu) v = gelu_tanh_f(v);
        if (g.res) v = fmaf(gate, v, r);
        reinterpret_cast<T*>(g.out)[(size_t)m * g.N + n] = to_act<T>(v);
    };
    if (S == 1) {
        if (warp >= 2 && g.res) {
            constexpr int CH = BN < 32 ? BN : 32;
#pragma unroll
            for (int c0 = 0; c0 < BN; c0 += CH) {
                float r[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c) r[c] = fetch_res(c0 + c);
#pragma unroll
                for (int c = 0; c < CH; ++c) put(c0 + c, acc[c0 + c], r[c]);
            }
        } else if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < BN; ++c) put(c, acc[c], 0.f);
        }
        return;
    }
    // partial sums lie as [source][4 tokens of the share][row of W]: a warp sends
    // one 512-byte run
    cluster_sync_all();                                    // every ring is free
    const int share = BN / 4 / S;                          // groups of 4 tokens a CTA finishes
    if (warp >= 2) {
#pragma unroll
        for (int c4 = 0; c4 < BN / 4; ++c4) {
            const int to = c4 / share;
            const uint32_t off = (uint32_t)((rank * share + c4 - to * share) * 128 + row) * 16u;
            st_shared_cluster_v4(mapa_shared(smem_u32(smem) + off, to), __float_as_uint(acc[4 * c4]),
                                 __float_as_uint(acc[4 * c4 + 1]), __float_as_uint(acc[4 * c4 + 2]),
                                 __float_as_uint(acc[4 * c4 + 3]));
        }
    }
    cluster_sync_all();
    if (warp >= 2) {
        const float4* part = reinterpret_cast<const float4*>(smem);
        for (int i = 0; i < share; ++i) {
            const int c = 4 * (rank * share + i);
            float r[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] = fetch_res(c + k);
            float4 v = part[i * 128 + row];
            for (int p = 1; p < S; ++p) {
                const float4 x = part[(p * share + i) * 128 + row];
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            put(c, v.x, r[0]);
            put(c + 1, v.y, r[1]);
            put(c + 2, v.z, r[2]);
            put(c + 3, v.w, r[3]);
        }
    }
}

using NarrowKernel = void (*)(const CUtensorMap, const CUtensorMap, const Gemm8Args);
struct Narrow {
    NarrowKernel kernel;
    int deep, shared;                                      // stages of the ring, of one CTA an SM and of two
    int bufs;                                              // TMEM buffers of two
    size_t (*smem)(int stages);
};
template <typename T, int BN>
Narrow narrow_of() {
    using C = NarrowCfg<BN>;
    return {gemm8_narrow_kernel<T, BN>, C::DEEP, C::SHARED, C::BUFS, [](int stages) { return C::smem(stages); }};
}
template <typename T>
Narrow narrow(int bn) {
    switch (bn) {
        case 16: return narrow_of<T, 16>();
        case 32: return narrow_of<T, 32>();
        default: return narrow_of<T, 64>();
    }
}

template <typename T>
wdc_status launch(Ctx* c, const void* A, const void* W, Gemm8Args g, int bn, int split, cudaStream_t s) {
    static PerDevice<bool> attr;
    attr.get(c->device, [](bool& ok) {
        ok = true;
        for (int bn : {16, 32, 64}) ok &= allow_smem(narrow<T>(bn).kernel, narrow<T>(bn).smem(narrow<T>(bn).deep));
        return ok;
    });
    g.m_tiles = (g.M - 1) / bn + 1;
    g.n_tiles = (g.N - 1) / 128 + 1;
    const long long tiles = (long long)g.m_tiles * g.n_tiles;
    g.split = split;
    if (tiles * g.split > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp8 GEMM: more than 2^31 - 1 thread blocks");
    CUtensorMap tw, ta;
    std::string why;
    if (!encode_tmap_2d(&tw, W, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)g.K, kBlock, 128, &why, CU_TENSOR_MAP_DATA_TYPE_UINT8) ||
        !encode_tmap_2d(&ta, A, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)g.K, kBlock, bn, &why, CU_TENSOR_MAP_DATA_TYPE_UINT8))
        return fail(c, WDC_ERR_CUDA, why);
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_GEMM, s);
        const Narrow k = narrow<T>(bn);
        const bool alone = tiles * g.split <= c->num_sms;
        g.stages = alone ? k.deep : k.shared;
        g.bufs = alone ? 2 * k.bufs : k.bufs;
        launch_kernel(k.kernel, dim3((unsigned)(tiles * g.split)), kThreads, k.smem(g.stages), s, g.split, tw, ta, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp8 GEMM launch: ") + cudaGetErrorString(e));
    return WDC_OK;
}

// The kernel for a shape is the one with the least estimated time, by fits to a
// sweep (us, bf16, no residual; narrow kernel n<tokens a tile>,<CTAs a tile>; pair
// kernel p<columns a tile>):
//                          n16,1  n32,1  n64,1  n16,4  n32,4  n64,4   p128   p256
//   4 x 3072 x 3072          7.6                  6.1
//   4 x 3072 x 12288        18.4                  8.9
//   33 x 9216 x 3072        10.5    9.9   14.0   18.3   16.9   13.0
//   64 x 1536 x 6144        11.6   14.0   21.4    8.9    8.3   11.4   17.2
//   100 x 3072 x 12288      26.1   23.2   36.6   28.9   24.0   22.4   29.4
//   226 x 1024 x 1024        5.8    6.8    9.6   11.3    8.1    8.7    7.6    8.6
//   226 x 9216 x 3072       34.8   25.7   21.6   82.1   56.9   44.2   12.5   15.2
//   512 x 3072 x 12288             63.9   59.7          72.8   62.9   29.7   41.7
//   512 x 9216 x 3072              48.2   40.6         110.4   86.1   19.5   16.0
//   1350 x 3072 x 12288                                               66.6   43.1
//   4276 x 9216 x 3072                                                 129    104
// A narrow CTA takes kStage us for two blocks of K; more CTAs than SMs take turns
// (two on an SM are each about half as fast), each turn with its own end, kEnd; a
// cluster's launch, barriers and exchange cost kSplit.  A pair takes 0.25 or 0.37 us
// a block of K and 1 or 1.5 a tile.
struct Choice {
    int bn, split;                     // split 0: the pair kernel
};
Choice choose(const Ctx* c, int M, int N, int kb) {
    constexpr double kStart[3] = {4.2, 4.3, 5.8}, kStage[3] = {0.29, 0.375, 0.56}, kEnd[3] = {0.8, 1.4, 2.3};
    constexpr double kSplit[3] = {1.9, 1.9, 2.2};
    Choice best{16, 1};
    double least = 1e30;
    auto offer = [&](int bn, int split, double est) {
        if (est < least) {
            least = est;
            best = {bn, split};
        }
    };
    for (int i = 0; i < 3; ++i) {
        const int bn = 16 << i;
        const double tiles = (double)((M - 1) / bn + 1) * ((N - 1) / 128 + 1);
        for (int split = 1; split <= bn / 4 && split <= 8 && (split == 1 || 4 * split <= kb); split *= 2) {
            const int stages = (kb + 2 * split - 1) / (2 * split);
            const double again = ceil(tiles * split / c->num_sms) - 1.0;
            offer(bn, split, kStart[i] + stages * kStage[i] + again * (stages * kStage[i] + kEnd[i]) +
                                 (split > 1 ? kSplit[i] : 0.0));
        }
    }
    if (c->num_sms >= 2) {
        const double rows = (M - 1) / 256 + 1, pairs = c->num_sms / 2;
        offer(128, 0, 5.0 + ceil(rows * ((N - 1) / 128 + 1) / pairs) * (kb * 0.25 + 1.0));
        offer(256, 0, 5.0 + ceil(rows * ((N - 1) / 256 + 1) / pairs) * (kb * 0.37 + 1.5));
    }
    return best;
}

}  // namespace

wdc_status op_gemm_fp8(Ctx* c, const void* A, const float* a_scale, const void* W, const float* w_scale,
                       const float* bias, void* C, int M, int N, int K, int gelu, const void* res, const float* gate,
                       cudaStream_t s) {
    if (M < 0 || N <= 0 || K <= 0) return fail(c, WDC_ERR_INVALID_ARG, "fp8 GEMM: M >= 0, N > 0 and K > 0 wanted");
    if (N > kMaxWidth8 || K > kMaxWidth8) return fail(c, WDC_ERR_UNSUPPORTED, "fp8 GEMM: N or K above 2^31 - 512");
    if (N % 8 || K % 16) return fail(c, WDC_ERR_UNSUPPORTED, "fp8 GEMM needs N % 8 == 0 and K % 16 == 0");
    if (M == 0) return WDC_OK;
    if (!A || !a_scale || !W || !w_scale || !C) return fail(c, WDC_ERR_INVALID_ARG, "fp8 GEMM: null pointer");
    if (((uintptr_t)A | (uintptr_t)a_scale | (uintptr_t)W | (uintptr_t)w_scale | (uintptr_t)bias | (uintptr_t)C |
         (uintptr_t)res | (uintptr_t)gate) & 15)
        return fail(c, WDC_ERR_INVALID_ARG, "fp8 GEMM: pointers must be 16-byte aligned");
    Gemm8Args g{};
    g.M = M; g.N = N; g.K = K; g.kb = (K + kBlock - 1) / kBlock; g.sw_rows = (N + 127) / 128;
    g.sa = a_scale; g.sw = w_scale; g.bias = bias; g.gate = res ? gate : nullptr; g.res = res; g.out = C; g.gelu = gelu;
    g.err = c->err;
    const Choice ch = choose(c, M, N, g.kb);
    if (ch.split == 0) return launch_gemm8_pair(c, A, W, g, ch.bn, s);
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, A, W, g, ch.bn, ch.split, s)
                                    : launch<float>(c, A, W, g, ch.bn, ch.split, s);
}

}  // namespace wdc
