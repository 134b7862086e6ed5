// Product of e2m1 matrices with e4m3 scales of 16 columns and fp32 scales of rows:
//   C[m, n] = epilogue( ra[m] rw[n] sum_k (a s_a)[m, k] (w s_w)[n, k] ),
// and of two such products the gated form act(A W^T) * (A U^T), on the 5th-generation
// tensor cores (tcgen05 kind::mxf4nvf4, sm_103a), which multiply the scales of 16 of K in:
// the sums over K are the tensor core's fp32, the rows' scales the epilogue's.  This file:
// the entries, the choice of the kernel, and the kernel for few rows; gemm_fp4_pair.cu: many.
#include "gemm_fp4.cuh"

#include <cmath>
#include <type_traits>

namespace wdc {

namespace {

// ---------------------------------------------------------------------------
// Few rows of A: W's rows are the MMA's M side (128 of them a tile), BN rows of A its N
// side, so that a few tokens cost a narrow MMA instead of a mostly empty one and a warp's
// lanes are neighbouring columns of C.  A tile of BN < 128 is all of A's rows (their scales
// lie 128 rows a piece, which a tile starts on).  A stage of the ring is 256 of K: the
// codes' tiles and, for each of its four MMAs, a piece of scales of either side, which one
// thread copies to the stage's columns of tensor memory before the MMAs.  The sums stay in
// tensor memory over all of K.
// A cluster of `split` CTAs shares a tile's K: each sums its part, sends the others their
// share of the tile's tokens through distributed shared memory and adds what it
// receives in rank order.
// Bound by the weights' bytes: gated 3 x 13824 x 5120 14.7 us (5.4 TB/s), 4 x 15360 x 5120 9.9
// (4.5 TB/s: 120 CTAs, of whose 10 us about 4 are the launch, the ring's first tiles and the
// end); with weights in L2 by the issue of a stage's copies and MMAs, 0.17 us for 16 KB of
// codes (an issuer each for the two was no faster).

template <int BN, bool GATED>
struct Narrow4Cfg {
    static constexpr int WS = GATED ? 2 : 1;                           // weights
    // Epilogue warps for each quarter of the lanes, which take 16 tokens by turns: 128 x 4096 x
    // 4096 with the residual 15.4 us with one, 11.0 with two, 9.2 with four; 64 x 4096 x 16384,
    // whose K is split, 9.8, 9.1 and 9.8.
    static constexpr int TURNS = BN == 16 ? 1 : (BN == 128 ? 4 : 2);
    static constexpr int THREADS = 64 + 128 * TURNS;                   // TMA producer, MMA issuer, epilogue
    static constexpr uint32_t W_BYTES = 128 * 128, A_BYTES = BN * 128, S_BYTES = 4 * kPiece4;
    static constexpr uint32_t STAGE = WS * W_BYTES + A_BYTES + (WS + 1) * S_BYTES;
    static constexpr int SCALE_COLS = 16 * (WS + 1);                   // of a stage, in tensor memory
    static constexpr int ACC_COLS = WS * BN;
    static constexpr size_t FIXED = 1024 + 512 + BN * 4;               // alignment, barriers, the tokens' scales
    static constexpr int BY_SMEM = (int)((227 * 1024 - FIXED) / STAGE), BY_TMEM = (512 - ACC_COLS) / SCALE_COLS;
    static constexpr int STAGES = BY_SMEM < BY_TMEM ? BY_SMEM : BY_TMEM;
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + FIXED;
    static constexpr uint32_t IDESC = idesc_e2m1(128, BN);
    static_assert(ACC_COLS * 128 * 4 <= STAGES * STAGE, "partial sums fit the ring");
    static_assert(STAGE % 1024 == 0 && STAGES * 2 * 8 + 64 <= 512, "tiles are aligned, barriers fit");
};

template <typename T, int BN, bool GATED>
__global__ void __launch_bounds__(Narrow4Cfg<BN, GATED>::THREADS, 1)
    gemm4_narrow_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmU,
                        const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmSW,
                        const __grid_constant__ CUtensorMap tmSU, const __grid_constant__ CUtensorMap tmSA,
                        const __grid_constant__ Gemm4Args g) {
    using C = Narrow4Cfg<BN, GATED>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* token_scale = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE);
    uint64_t* full = reinterpret_cast<uint64_t*>(token_scale + BN);
    uint64_t* empty = full + C::STAGES;
    uint64_t* done = empty + C::STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = g.split, rank = S > 1 ? (int)cluster_ctarank() : 0;
    const int tile = blockIdx.x / S;
    const int mt = tile % g.m_tiles, nb = tile / g.m_tiles;            // neighbouring tiles share W
    const int m0 = mt * BN;
    const int kb0 = (int)((long long)rank * g.kb / S), kb1 = (int)((long long)(rank + 1) * g.kb / S);
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(done, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmSW);
        prefetch_tmap(&tmSA);
        if (GATED) {
            prefetch_tmap(&tmU);
            prefetch_tmap(&tmSU);
        }
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, 512);
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
        for (int kb = kb0; kb < kb1; ++kb) {               // (what lies past K is filled with zeros)
            if (!mbar_wait_warp(&empty[stage], phase ^ 1u, abort_flag, g.err)) break;
            if (elect_one()) {
                mbar_arrive_expect_tx(&full[stage], C::STAGE);
                uint8_t* at = smem + stage * C::STAGE;
                tma_load_2d(at, &tmW, &full[stage], kb * 128, nb * 128);
                if (GATED) tma_load_2d(at + C::W_BYTES, &tmU, &full[stage], kb * 128, nb * 128);
                at += C::WS * C::W_BYTES;
                tma_load_2d(at, &tmA, &full[stage], kb * 128, m0);
                at += C::A_BYTES;
                tma_load_3d(at, &tmSW, &full[stage], 0, kb * 4, nb);
                if (GATED) tma_load_3d(at + C::S_BYTES, &tmSU, &full[stage], 0, kb * 4, nb);
                tma_load_3d(at + C::WS * C::S_BYTES, &tmSA, &full[stage], 0, kb * 4, mt);
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
        if (elect_one()) {
            const uint32_t base = smem_u32(smem);
            const uint64_t dw = sdesc_sw128(base), da = sdesc_sw128(base + C::WS * C::W_BYTES);
            const uint64_t ds = sdesc_rows16(base + C::WS * C::W_BYTES + C::A_BYTES);
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(&full[stage], phase, abort_flag, g.err)) break;
                tc_fence_after();
                // the stage's columns: the MMAs that read them before are done, as its tiles
                // could not have been loaded again otherwise
                const uint32_t sc = tmem + (uint32_t)(C::ACC_COLS + stage * C::SCALE_COLS);
#pragma unroll
                for (int i = 0; i < 4 * (C::WS + 1); ++i)
                    tc_copy_scales(sc + 4 * i, sdesc_at(ds, stage * C::STAGE + i * kPiece4));
#pragma unroll
                for (int h = 0; h < C::WS; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma4(tmem + (uint32_t)(h * BN), sdesc_at(dw, stage * C::STAGE + h * C::W_BYTES + k * 32),
                                sdesc_at(da, stage * C::STAGE + k * 32), C::IDESC, sc + 16 * h + 4 * k,
                                sc + 16 * C::WS + 4 * k, kb != kb0 || k != 0);
                tc_commit(&empty[stage]);
                if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
            }
            // all MMAs issued by this lane have completed before their sums are read and
            // tensor memory is freed
            tc_commit(done);
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(done, 0) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
        __syncwarp();
    }

    const int lg = warp & 3;                               // TMEM lane quarter this warp may access
    const int turn = (warp - 2) >> 2;                      // and which of its warps it is
    const int row = lg * 32 + lane, n = nb * 128 + row;
    bool ok = true;
    float rw = 0.f, ru = 0.f, bias = 0.f, up_bias = 0.f, gate = 1.f;
    if (warp >= 2) {
        // (fetched where they are used, a group of 16 tokens behind the other, they took 1 us each)
        const int c = threadIdx.x - 64;
        if (c < BN) token_scale[c] = m0 + c < g.M ? ld_chain(g.ra + m0 + c) : 0.f;
        asm volatile("bar.sync 1, %0;" ::"n"(128 * C::TURNS) : "memory");      // the epilogue's warps
        if (n < g.N) {
            rw = ld_chain(g.rw + n);
            if (g.bias) bias = ld_chain(g.bias + n);
            if (g.gate) gate = ld_chain(g.gate + n);
            if (GATED) {
                ru = ld_chain(g.ru + n);
                if (g.up_bias) up_bias = ld_chain(g.up_bias + n);
            }
        }
        ok = mbar_wait_warp(done, 0, abort_flag, g.err) && !*abort_flag;
        __syncwarp();                                      // (after a wait that gave up nothing else does)
        tc_fence_after();
    }
    const uint32_t lanes = tmem + ((uint32_t)(lg * 32) << 16);
    // Finishes CH tokens from c on.  All is worked out for all of them, and only what lies in C
    // is loaded and stored: a branch a token leaves the warp, alone on its scheduler, waiting
    // for each instruction in turn.
    const bool mine = ok && n < g.N;
    auto finish = [&](int c, auto& v, auto& u) {
        constexpr int CH = sizeof(v) / sizeof(float);
        const int left = mine ? g.M - m0 - c : 0;          // tokens
        const size_t at = (size_t)(m0 + c) * g.N + n;
        float r[CH];
        if (!GATED && g.res) {
            const T* res = reinterpret_cast<const T*>(g.res) + at;
#pragma unroll
            for (int i = 0; i < CH; ++i) r[i] = i < left ? ld_act<T>(res + (size_t)i * g.N) : 0.f;
        }
        T* out = reinterpret_cast<T*>(g.out) + at;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float ra = token_scale[c + i];
            float x = fmaf(v[i] * ra, rw, bias);
            if constexpr (GATED) {
                x = (g.gelu ? gelu_tanh_f(x) : silu_f(x)) * fmaf(u[i] * ra, ru, up_bias);
            } else {
                if (g.gelu) x = gelu_tanh_f(x);
                if (g.res) x = fmaf(gate, x, r[i]);
            }
            v[i] = x;
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i < left) out[(size_t)i * g.N] = to_act<T>(v[i]);
    };
    auto load16 = [&](int c, float (&v)[16]) {             // 16 columns of sums
        uint32_t p[16];
        tmem_ld16(lanes + (uint32_t)c, p);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(p[i]);
    };
    if (S == 1) {
        if (warp >= 2) {
#pragma unroll 1
            for (int c0 = 16 * turn; c0 < BN && m0 + c0 < g.M; c0 += 16 * C::TURNS) {
                float v[16], u[16] = {};
                load16(c0, v);
                if (GATED) load16(BN + c0, u);
                finish(c0, v, u);
                __syncwarp();
            }
        }
    } else {
        // partial sums lie as [weights][source][4 tokens of the share][row of W]: a warp
        // sends one 512-byte run
        __syncthreads();                                   // this CTA's copies have landed, its MMAs are done
        cluster_sync_all();                                // every ring is free
        const int share = BN / 4 / S;                      // groups of 4 tokens a CTA finishes
        if (warp >= 2) {
#pragma unroll
            for (int h = 0; h < C::WS; ++h)
#pragma unroll 1
                for (int c0 = 16 * turn; c0 < BN && m0 + c0 < g.M; c0 += 16 * C::TURNS) {
                    float v[16];
                    load16(h * BN + c0, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int c4 = c0 / 4 + i, to = c4 / share;
                        const uint32_t off = (uint32_t)(((h * S + rank) * share + c4 - to * share) * 128 + row) * 16u;
                        st_shared_cluster_v4(mapa_shared(smem_u32(smem) + off, to), __float_as_uint(v[4 * i]),
                                             __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                                             __float_as_uint(v[4 * i + 3]));
                    }
                }
        }
        cluster_sync_all();
        if (warp >= 2) {
            const float4* part = reinterpret_cast<const float4*>(smem);
            // G groups from i on, the sources in rank order
            auto join = [&](int i, auto groups) {
                constexpr int G = decltype(groups)::value;
                float v[2][4 * G] = {};
#pragma unroll
                for (int h = 0; h < C::WS; ++h)
                    for (int p = 0; p < S; ++p)
#pragma unroll
                        for (int k = 0; k < G; ++k) {
                            const float4 x = part[((h * S + p) * share + i + k) * 128 + row];
                            v[h][4 * k] += x.x; v[h][4 * k + 1] += x.y; v[h][4 * k + 2] += x.z; v[h][4 * k + 3] += x.w;
                        }
                finish(4 * (rank * share + i), v[0], v[1]);
            };
            if (share % 4 == 0) {
                for (int i = 4 * turn; i < share && m0 + 4 * (rank * share + i) < g.M;
                     i += 4 * C::TURNS) join(i, std::integral_constant<int, 4>());
            } else {
                for (int i = turn; i < share && m0 + 4 * (rank * share + i) < g.M;
                     i += C::TURNS) join(i, std::integral_constant<int, 1>());
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

using NarrowKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                              const CUtensorMap, const Gemm4Args);
struct Narrow {
    NarrowKernel kernel;
    size_t smem;
    int threads;
};
template <typename T, int BN, bool GATED>
Narrow narrow_of() {
    using C = Narrow4Cfg<BN, GATED>;
    return {gemm4_narrow_kernel<T, BN, GATED>, C::SMEM, C::THREADS};
}
template <typename T, bool GATED>
Narrow narrow(int bn) {
    switch (bn) {
        case 16: return narrow_of<T, 16, GATED>();
        case 32: return narrow_of<T, 32, GATED>();
        case 64: return narrow_of<T, 64, GATED>();
        default: return narrow_of<T, 128, GATED>();
    }
}

template <typename T, bool GATED>
wdc_status launch_narrow(Ctx* c, Gemm4Args g, int bn, int split, cudaStream_t s) {
    static PerDevice<bool> attr;
    attr.get(c->device, [](bool& ok) {
        ok = true;
        for (int n : {16, 32, 64, 128}) ok &= allow_smem(narrow<T, GATED>(n).kernel, narrow<T, GATED>(n).smem);
        return ok;
    });
    g.m_tiles = (g.M - 1) / bn + 1;
    g.n_tiles = (g.N - 1) / 128 + 1;
    g.kb = (g.K - 1) / kTileK4 + 1;
    g.split = split;
    const long long ctas = (long long)g.m_tiles * g.n_tiles * split;
    if (ctas > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM: more than 2^31 - 1 thread blocks");
    CUtensorMap tw, tu, ta, tsw, tsu, tsa;
    std::string why;
    if (!encode_codes(&tw, g.W, g.N, g.K, 128, &why) || !encode_codes(&tu, GATED ? g.U : g.W, g.N, g.K, 128, &why) ||
        !encode_codes(&ta, g.A, g.M, g.K, bn, &why) || !encode_scales(&tsw, g.sw, g.N, g.pieces, &why) ||
        !encode_scales(&tsu, GATED ? g.su : g.sw, g.N, g.pieces, &why) || !encode_scales(&tsa, g.sa, g.M, g.pieces, &why))
        return fail(c, WDC_ERR_CUDA, why);
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_GEMM, s);
        const Narrow k = narrow<T, GATED>(bn);
        launch_kernel(k.kernel, dim3((unsigned)ctas), k.threads, k.smem, s, split, tw, tu, ta, tsw, tsu, tsa, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 GEMM launch: ") + cudaGetErrorString(e));
    return WDC_OK;
}

// The kernel for a shape is the one with the least estimated time, by fits to a sweep (us,
// bf16, no residual, operands in L2; narrow kernel n<tokens a tile>,<CTAs a tile>; pair kernel p):
//                          n16,1  n16,4  n32,1  n32,4  n64,1  n64,4  n128,1 n128,4    p
//   4 x 1024 x 1024          3.8                                       4.1           7.2
//   4 x 4096 x 16384        14.0    7.3                               15.2   15.0   22.9
//   4 x 15360 x 5120         6.7                                      13.0          16.3
//   32 x 4096 x 4096                       6.2    5.6                  6.4    8.4   10.4
//   32 x 4096 x 16384                     14.6    7.7                 14.6    9.7   23.0
//   64 x 27648 x 2048                                     9.9         11.9          12.3
//   64 x 4096 x 16384                                    14.9    8.5  14.9   10.0   23.1
//   100 x 1024 x 1024                                                  5.2           8.0
//   200 x 4096 x 4096                                                  7.6   15.0   11.2
//   200 x 15360 x 5120                                                15.6          12.9
//   400 x 4096 x 16384                                                16.1          24.0
//   700 x 4096 x 4096                                                 14.2          11.6
//   gated 64 x 10240 x 4096                               9.0          9.7          16.6
//   gated 200 x 10240 x 4096                                          20.0          17.1
//   gated 100 x 2048 x 2048                                            7.9    9.0    9.3
//   gated 200 x 1024 x 8192                                           15.7   11.2   15.7
// A narrow CTA takes kStage us for 256 of K and a little for each token; more CTAs than
// the device holds (fewer than its SMs in clusters of 8) take turns; a cluster's launch
// and exchange cost what `split` adds.
struct Choice {
    int bn, split;                     // split 0: the pair kernel
};
Choice choose(const Ctx* c, int M, int N, int K, bool gated) {
    constexpr double kStage[2][4] = {{0.17, 0.17, 0.175, 0.175}, {0.26, 0.26, 0.30, 0.34}};
    const int kb = (K - 1) / kTileK4 + 1;
    Choice best{128, 1};
    double least = 1e30;
    auto offer = [&](int bn, int split, double est) {
        if (est < least) {
            least = est;
            best = {bn, split};
        }
    };
    for (int i = 0; i < 4; ++i) {
        const int bn = 16 << i;
        if (bn < 128 && M > bn) continue;
        const double tiles = (double)((M - 1) / bn + 1) * ((N - 1) / 128 + 1), tokens = M < bn ? M : bn;
        for (int split = 1; split <= 8 && split <= bn / 4 && (split == 1 || 2 * split <= kb); split *= 2) {
            const double held = split == 8 ? 0.74 * c->num_sms : c->num_sms;
            const double turn = (kb + split - 1) / split * kStage[gated][i] + 1.6 + (gated ? 0.016 : 0.01) * tokens / split;
            const double join = (gated ? 1.4 : 1.2) + (gated ? 0.02 : 0.01) * tokens + (bn == 128 ? 1.3 : 0.0);
            offer(bn, split, 1.5 + ceil(tiles * split / held) * (turn + (split > 1 ? join : 0.0)));
        }
    }
    if (c->num_sms >= 2) {
        const double tiles = (double)((M - 1) / 256 + 1) * ((N - 1) / (gated ? 128 : 256) + 1);
        offer(256, 0, 5.8 + ceil(tiles / (c->num_sms / 2)) * (kb * 0.265 + 1.4));
    }
    return best;
}

wdc_status launch(Ctx* c, const Gemm4Args& g, cudaStream_t s) {
    const Choice ch = choose(c, g.M, g.N, g.K, g.U != nullptr);
    if (ch.split == 0) return launch_gemm4_pair(c, g, s);
    if (c->cfg.dtype == WDC_BF16)
        return g.U ? launch_narrow<__nv_bfloat16, true>(c, g, ch.bn, ch.split, s)
                   : launch_narrow<__nv_bfloat16, false>(c, g, ch.bn, ch.split, s);
    return g.U ? launch_narrow<float, true>(c, g, ch.bn, ch.split, s) : launch_narrow<float, false>(c, g, ch.bn, ch.split, s);
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

wdc_status fp4_plan(Ctx* c, int M, int N, int K, bool gated, int* plan) {
    if (M <= 0 || N <= 0 || K <= 0 || N > kMaxWidth4 || K > kMaxWidth4 || M > kMaxRows4 || N % 8 || K % 64)
        return fail(c, WDC_ERR_INVALID_ARG, "fp4 plan: not a shape of the products");
    const Choice ch = choose(c, M, N, K, gated);
    plan[0] = ch.bn;
    plan[1] = ch.split;
    plan[2] = plan[3] = 0;
    if (ch.split > 0) return WDC_OK;
    Gemm4Args g{};
    const uint8_t none = 0;
    g.M = M; g.N = N; g.K = K;
    g.U = gated ? &none : nullptr;
    if (!plan_gemm4_pair(c, g)) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 plan: the pair kernel cannot take it");
    plan[2] = g.parts > 1 ? g.tail : 0;
    plan[3] = g.parts > 1 ? g.parts : 0;
    return WDC_OK;
}

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
