// Product of e4m3 matrices with block scales on the 5th-generation tensor cores
// (tcgen05 kind::f8f6f4, sm_103a):
//   C[m, n] = epilogue( sum_b sa[b][m] sw[n / 128][b] sum_{k in block b} A[m, k] W[n, k] ),
// blocks of 128 columns of K.  A block is one 128-byte row of the swizzled
// shared-memory tiles and four MMAs (32 of K each) into a TMEM buffer of its
// own; the epilogue warps then add the buffer, times its scales, to sums in
// their registers, while the next blocks' MMAs fill the other buffers.  So a
// sum over K is fp32 beyond a block, whatever the scales.
#include "gemm_fp8.cuh"

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
template <int BN>
struct NarrowCfg {
    static constexpr uint32_t W_BYTES = 128 * kBlock, A_BYTES = BN * kBlock, STAGE = W_BYTES + A_BYTES;
    static constexpr int STAGES = BN <= 32 ? 5 : (BN == 64 ? 4 : 3);
    static constexpr int BUFS = BN == 128 ? 2 : 4;
    static constexpr uint32_t TMEM_COLS = BUFS * BN;
    static constexpr uint32_t IDESC = idesc_e4m3(128, BN);
    static constexpr int WINDOW = BN == 128 ? 8 : 16;      // blocks whose scales are in shared memory at a time
    static constexpr uint32_t WINDOW_BYTES = 2 * WINDOW * BN * 4;
    static constexpr size_t SMEM = STAGES * STAGE + WINDOW_BYTES + 1024 + 256;
    static_assert(BN * 128 * 4 <= STAGES * STAGE, "partial sums fit the ring");
    static_assert(TMEM_COLS >= 32 && 2 * TMEM_COLS <= 512 && 2 * (SMEM + 1024) <= 227 * 1024, "two CTAs an SM");
};

template <typename T, int BN>
__global__ void __launch_bounds__(kThreads, 2)
    gemm8_narrow_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                        const __grid_constant__ Gemm8Args g) {
    using C = NarrowCfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* window = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE);     // [2][WINDOW][BN]
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::STAGES * C::STAGE + C::WINDOW_BYTES);
    uint64_t* empty = full + C::STAGES;
    uint64_t* tfull = empty + C::STAGES;
    uint64_t* tempty = tfull + C::BUFS;
    uint64_t* mma_done = tempty + C::BUFS;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = g.split, rank = S > 1 ? (int)cluster_ctarank() : 0;
    const int tile = blockIdx.x / S;
    const int m0 = (tile % g.m_tiles) * BN, nb = tile / g.m_tiles;             // neighbouring tiles share W
    const int kb0 = (int)((long long)rank * g.kb / S), kb1 = (int)((long long)(rank + 1) * g.kb / S);
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < C::BUFS; ++b) {
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
        tmem_alloc(tmem_slot, C::TMEM_COLS);
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
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait_warp(&empty[stage], phase ^ 1u, abort_flag, g.err)) break;
            if (elect_one()) {
                mbar_arrive_expect_tx(&full[stage], C::STAGE);
                uint8_t* sw = smem + stage * C::STAGE;
                tma_load_2d(sw, &tmW, &full[stage], kb * kBlock, nb * 128);
                tma_load_2d(sw + C::W_BYTES, &tmA, &full[stage], kb * kBlock, m0);
            }
            __syncwarp();
            armed |= 1u << stage;
            parity = (parity & ~(1u << stage)) | (phase << stage);
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
        // every issued copy has landed before the ring is reused or the CTA exits
        for (int s = 0; s < C::STAGES; ++s) {
            if (!((armed >> s) & 1)) continue;
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(&full[s], (parity >> s) & 1) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
    } else if (warp == 1) {
        const uint64_t dw = sdesc_sw128(smem_u32(smem)), da = sdesc_sw128(smem_u32(smem) + C::W_BYTES);
        int stage = 0, buf = 0;
        uint32_t phase = 0, bphase = 0;
        bool ok = true;                                    // this lane's waits (elect_one)
        for (int kb = kb0; kb < kb1; ++kb) {
            ok = ok && mbar_wait(&tempty[buf], bphase ^ 1u, abort_flag, g.err);
            ok = ok && mbar_wait(&full[stage], phase, abort_flag, g.err);
            tc_fence_after();
            if (elect_one() && ok) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    tc_mma8(tmem + (uint32_t)(buf * BN), sdesc_at(dw, stage * C::STAGE + k * 32),
                            sdesc_at(da, stage * C::STAGE + k * 32), C::IDESC, k != 0);
                tc_commit(&empty[stage]);
                tc_commit(&tfull[buf]);
            }
            __syncwarp();
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
            if (++buf == C::BUFS) { buf = 0; bphase ^= 1u; }
        }
        // all MMAs issued by this warp have completed before TMEM is freed
        if (elect_one()) tc_commit(mma_done);
        __syncwarp();
        const unsigned long long t0 = globaltimer();
        while (!mbar_try_wait(mma_done, 0) && globaltimer() - t0 < kWaitLimitNs) {
        }
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
        for (int kb = kb0; kb < kb1; ++kb) {
            const int at = (kb - kb0) % C::WINDOW, w = (kb - kb0) / C::WINDOW;
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
            tc_fence_after();
            constexpr int CH = BN < 32 ? BN : 32;          // columns a load
#pragma unroll
            for (int c0 = 0; c0 < BN; c0 += CH) {
                uint32_t p[CH];
                if constexpr (CH == 16) tmem_ld16(lanes + (uint32_t)(buf * BN), p);
                else tmem_ld32(lanes + (uint32_t)(buf * BN + c0), p);
                tmem_ld_wait();
                if (c0 + CH == BN) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&tempty[buf]);
                }
#pragma unroll
                for (int c = 0; c < CH; c += 4) {
                    const float4 s = s4[(c0 + c) / 4];
                    acc[c0 + c] = fmaf(__uint_as_float(p[c]), s.x, acc[c0 + c]);
                    acc[c0 + c + 1] = fmaf(__uint_as_float(p[c + 1]), s.y, acc[c0 + c + 1]);
                    acc[c0 + c + 2] = fmaf(__uint_as_float(p[c + 2]), s.z, acc[c0 + c + 2]);
                    acc[c0 + c + 3] = fmaf(__uint_as_float(p[c + 3]), s.w, acc[c0 + c + 3]);
                }
            }
            if (++buf == C::BUFS) { buf = 0; bphase ^= 1u; }
        }
    }
    // this CTA's copies have landed and its MMAs are done
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, C::TMEM_COLS);
    }
    const int row = lg * 32 + lane, n = nb * 128 + row;
    const bool mine = warp >= 2 && ok && n < g.N;
    float bias = 0.f, gate = 1.f;
    if (mine) {
        if (g.bias) bias = ld_chain(g.bias + n);
        if (g.gate) gate = ld_chain(g.gate + n);
    }
    auto put = [&](int c, float v) {
        const int m = m0 + c;
        if (!mine || m >= g.M) return;
        v += bias;
        if (g.gelu) v = gelu_tanh_f(v);
        const size_t at = (size_t)m * g.N + n;
        if (g.res) v = fmaf(gate, v, ld_act<T>(reinterpret_cast<const T*>(g.res) + at));
        reinterpret_cast<T*>(g.out)[at] = to_act<T>(v);
    };
    if (S == 1) {
        if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < BN; ++c) put(c, acc[c]);
        }
        return;
    }
    // partial sums lie as [source][token of the share][row of W]
    cluster_sync_all();                                    // every ring is free
    if (warp >= 2) {
        int to = 0;
#pragma unroll
        for (int c = 0; c < BN; ++c) {
            while (c >= (to + 1) * BN / S) ++to;
            const int first = to * BN / S, width = (to + 1) * BN / S - first;
            const uint32_t off = (uint32_t)((rank * width + c - first) * 128 + row) * 4u;
            st_shared_cluster_f32(mapa_shared(smem_u32(smem) + off, to), acc[c]);
        }
    }
    cluster_sync_all();
    if (warp >= 2) {
        const int first = rank * BN / S, width = (rank + 1) * BN / S - first;
        const float* part = reinterpret_cast<const float*>(smem);
        for (int c = 0; c < width; ++c) {
            float v = part[c * 128 + row];
            for (int p = 1; p < S; ++p) v += part[(p * width + c) * 128 + row];
            put(first + c, v);
        }
    }
}

using NarrowKernel = void (*)(const CUtensorMap, const CUtensorMap, const Gemm8Args);
struct Narrow {
    NarrowKernel kernel;
    size_t smem;
};
template <typename T>
Narrow narrow(int bn) {
    switch (bn) {
        case 16: return {gemm8_narrow_kernel<T, 16>, NarrowCfg<16>::SMEM};
        case 32: return {gemm8_narrow_kernel<T, 32>, NarrowCfg<32>::SMEM};
        case 64: return {gemm8_narrow_kernel<T, 64>, NarrowCfg<64>::SMEM};
        default: return {gemm8_narrow_kernel<T, 128>, NarrowCfg<128>::SMEM};
    }
}

template <typename T>
wdc_status launch(Ctx* c, const void* A, const void* W, Gemm8Args g, cudaStream_t s) {
    static PerDevice<bool> attr;
    attr.get(c->device, [](bool& ok) {
        ok = true;
        for (int bn : {16, 32, 64, 128}) ok &= allow_smem(narrow<T>(bn).kernel, narrow<T>(bn).smem);
        return ok;
    });
    int bn = 16;
    while (bn < 128 && bn < g.M) bn *= 2;
    g.m_tiles = (g.M + bn - 1) / bn;
    g.n_tiles = (g.N + 127) / 128;
    const long long tiles = (long long)g.m_tiles * g.n_tiles;
    g.split = 1;
    while (g.split < 8 && 2 * g.split <= g.kb && tiles * g.split * 2 <= c->num_sms) g.split *= 2;
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
        launch_kernel(k.kernel, dim3((unsigned)(tiles * g.split)), kThreads, k.smem, s, g.split, tw, ta, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp8 GEMM launch: ") + cudaGetErrorString(e));
    return WDC_OK;
}

}  // namespace

wdc_status op_gemm_fp8(Ctx* c, const void* A, const float* a_scale, const void* W, const float* w_scale,
                       const float* bias, void* C, int M, int N, int K, int gelu, const void* res, const float* gate,
                       cudaStream_t s) {
    if (M < 0 || N <= 0 || K <= 0) return fail(c, WDC_ERR_INVALID_ARG, "fp8 GEMM: M >= 0, N > 0 and K > 0 wanted");
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
    if (M >= 512) return launch_gemm8_pair(c, A, W, g, 256, s);
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, A, W, g, s) : launch<float>(c, A, W, g, s);
}

}  // namespace wdc
