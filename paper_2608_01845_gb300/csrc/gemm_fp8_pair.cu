// Product of e4m3 matrices with block scales (see gemm_fp8.cu), CTA-pair kernel:
// products with tiles enough for the pairs.
//
// A pair of CTAs takes a tile of 256 rows of A by BN of W, 256 x BN x 32 MMAs
// issued by the even one; each CTA holds its 128 rows of A and its half of the
// W tile, and the sums of its 128 rows in registers: eight epilogue warps, a
// warpgroup for each half of the columns, one row a lane, so a block's scale is
// one value a lane and a buffer's addition 64 paired multiply-adds (BN = 256).
// A block's MMAs take 512 cycles of the tensor core (BN = 256); a block comes out
// every 700 to 750: tensor memory holds two buffers of 256 columns, and from a
// buffer's last MMA to its next first one pass the commit, the epilogue's reads and
// additions and their arrival at the issuer, about 900 cycles, of which the other
// buffer's MMAs cover 512.  (Buffers of half a tile, four of them, were slower: 63 us
// where these took 50, as each costs a round of its own.)
//
// Bound by that round: 17776 x 9216 x 3072 bf16 380 to 400 us, 2520 to 2650 TFLOP/s, 0.65
// to 0.69 of the fp8 rate; 1350 x 3072 x 12288 43 to 46 us, where 72 tiles of 76 pairs hold
// 12% rows past M; 1576 rows 80 us, as 84 tiles take two rounds.
//
// Once a tile's last block is added, the warps finish it (bias, GELU, gated
// residual), a slab of 32 rows x 128 bytes at a time through swizzled shared
// memory and TMA; the tensor core is then at most two blocks ahead.
#include "gemm_fp8.cuh"

namespace wdc {

namespace {

constexpr int kBlock = kBlock8;
constexpr int kPairThreads = 384;           // three warpgroups: TMA producer and MMA issuer; epilogue (two)
// Registers a thread: 168 at launch (65536 / 384, a multiple of 8), of which the
// first warpgroup hands most to the others.
constexpr uint32_t kRegsLaunch = 168, kRegsControl = 56, kRegsEpilogue = 224;
static_assert(128 * kRegsControl + 256 * kRegsEpilogue <= 384 * kRegsLaunch, "register split exceeds the launch");
constexpr int kChunk = 4, kSlots = 3;       // blocks of a slot of scales, slots
template <int BN>
struct Pair8Cfg {
    static constexpr uint32_t A_BYTES = 128 * kBlock, B_BYTES = BN / 2 * kBlock, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = BN == 256 ? 5 : 6;
    static constexpr uint32_t SLAB = 32 * 128;
    static constexpr uint32_t STAGING = 8 * SLAB;
    // scales sa * sw of kChunk blocks a slot: [block][side][128 rows]
    static constexpr uint32_t SLOT = kChunk * 2 * 128 * 4;
    static constexpr int COLS = BN / 2;                    // columns of a side
    static constexpr uint32_t IDESC = idesc_e4m3(256, BN);
    static constexpr uint32_t VECTORS = 8 * 2 * COLS * 4;  // bias and gate of each epilogue warp's columns
    static constexpr size_t SMEM = STAGES * STAGE + STAGING + kSlots * SLOT + VECTORS + 1024 + 512;
    static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
};

__device__ __forceinline__ uint64_t pack64(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t twice(float v) { return pack64(__float_as_uint(v), __float_as_uint(v)); }
__device__ __forceinline__ float2 unpack64(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}

// gelu_tanh_f of two values with one reciprocal for both: 1 / a = b / (a b).  The
// epilogue's exponentials and reciprocals (16 a clock) are what a GELU costs.  The
// exponent is cut off at 60, so that a b is finite; beyond it (x < -7) the result,
// below 2^-60 |x|, is 0, as gelu_tanh_f's is from 2^-126 on.  PAIRED: the exponents by
// instructions for two values, the same bits (17776 x 12288 x 3072 with bf16 results 595
// -> 570 us; with fp32 results, whose slabs hold half the columns, 1350 rows 62 -> 69).
template <bool PAIRED>
__device__ __forceinline__ void gelu_pair(float& x, float& y) {
    const float k0 = 0.7978845608028654f, k1 = 0.044715f, m2log2e = -2.0f * 1.4426950408889634f;
    float u, v, a, b, r;
    if constexpr (PAIRED) {
        const uint64_t p = pack64(__float_as_uint(x), __float_as_uint(y));
        const float2 e = unpack64(mul2(twice(k0 * m2log2e), fma2(mul2(mul2(twice(k1), p), p), p, p)));
        u = e.x;
        v = e.y;
    } else {
        u = k0 * m2log2e * fmaf(k1 * x * x, x, x);
        v = k0 * m2log2e * fmaf(k1 * y * y, y, y);
    }
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(fminf(u, 60.f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(fminf(v, 60.f)));
    a += 1.0f;
    b += 1.0f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a * b));
    x *= u > 60.f ? 0.f : r * b;
    y *= v > 60.f ? 0.f : r * a;
}

// A 16-byte piece of a slab's row.
__device__ __forceinline__ void load_piece(const float* p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load_piece(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store_piece(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T, int BN, bool GELU, bool RESID>
__global__ void __launch_bounds__(kPairThreads, 1)
    gemm8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                      const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmR,
                      const __grid_constant__ Gemm8Args g) {
    using C = Pair8Cfg<BN>;
    constexpr int COLS = C::COLS;                  // columns of a side, and so of a warp
    constexpr int SC = 128 / (int)sizeof(T);       // columns of a slab
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + C::STAGES * C::STAGE;
    float* scales = reinterpret_cast<float*>(staging + C::STAGING);          // [kSlots][kChunk][2 sides][128 rows]
    float* vectors = scales + kSlots * (C::SLOT / 4);                        // [8 warps][bias, gate][COLS]
    uint64_t* full = reinterpret_cast<uint64_t*>(vectors + C::VECTORS / 4);  // even CTA: both halves landed
    uint64_t* empty = full + C::STAGES;
    uint64_t* tfull = empty + C::STAGES;           // [2]
    uint64_t* tempty = tfull + 2;                  // [2] even CTA: both CTAs' warps have read the buffer
    uint64_t* sfull = tempty + 2;                  // [kSlots]
    uint64_t* sempty = sfull + kSlots;             // [kSlots]
    uint64_t* mma_done = sempty + kSlots;
    uint64_t* rbars = mma_done + 1;                // [8 warps] residual slabs
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(rbars + 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int tiles = g.m_tiles * g.n_tiles;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tfull[b], 1);
            mbar_init(&tempty[b], 16);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(&sfull[i], 1);
            mbar_init(&sempty[i], 8);
        }
        mbar_init(mma_done, 1);
        for (int i = 0; i < 8; ++i) mbar_init(&rbars[i], 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmC);
    }
    if (warp == 1) {
        tmem_alloc2(tmem_slot, 512);
        tmem_relinquish2();
    }
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    chain_release();
    chain_wait();
    const uint32_t own_base = *tmem_slot;
    const uint32_t tmem = rank == 0 ? own_base : ld_shared_cluster_u32(mapa_shared(smem_u32(tmem_slot), 0));
    if (threadIdx.x == 0 && tmem != own_base) atomicOr(g.err, kErrTmem);

    // tile -> 256-row block and column block: columns fastest inside groups of
    // column blocks whose rows of W stay in L2
    auto place = [&](int tile, int& mb, int& nb) {
        const int per = g.m_tiles * g.group_n, grp = tile / per, r = tile - grp * per;
        const int first = grp * g.group_n, width = min(g.group_n, g.n_tiles - first);
        mb = r / width;
        nb = first + (r - mb * width);
    };

    if (warp < 4) {
      setmaxnreg_dec<kRegsControl>();
      if (warp == 0) {
          int stage = 0;
          uint32_t phase = 0, armed = 0, parity = 0;         // per stage: a copy was issued; its phase
          bool ok = true;
          for (int tile = pair; tile < tiles && ok; tile += pairs) {
              int mb, nb;
              place(tile, mb, nb);
              const int m0 = mb * 256 + (int)rank * 128, n0 = nb * BN + (int)rank * COLS;
              for (int kb = 0; kb < g.kb; ++kb) {
                  if (!mbar_wait_warp(&empty[stage], phase ^ 1u, abort_flag, g.err)) { ok = false; break; }
                  if (elect_one()) {
                      if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * C::STAGE);
                      const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
                      uint8_t* sa = smem + stage * C::STAGE;
                      tma_load_2d_pair(sa, &tmA, fb, kb * kBlock, m0);
                      tma_load_2d_pair(sa + C::A_BYTES, &tmW, fb, kb * kBlock, n0);
                  }
                  __syncwarp();
                  armed |= 1u << stage;
                  parity = (parity & ~(1u << stage)) | (phase << stage);
                  if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
              }
          }
          // every copy of the pair has landed (even CTA's full) and the MMAs have
          // released every stage (both CTAs' empty)
          for (int s = 0; s < C::STAGES; ++s) {
              if (!((armed >> s) & 1)) continue;
              if (rank == 0) {
                  const unsigned long long t0 = globaltimer();
                  while (!mbar_try_wait(&full[s], (parity >> s) & 1) && globaltimer() - t0 < kWaitLimitNs) {
                  }
              }
              const unsigned long long t1 = globaltimer();
              while (!mbar_try_wait(&empty[s], (parity >> s) & 1) && globaltimer() - t1 < kWaitLimitNs) {
              }
          }
      } else if (warp == 1) {
          if (rank == 0) {
              const uint64_t da = sdesc_sw128(smem_u32(smem)), db = sdesc_sw128(smem_u32(smem) + C::A_BYTES);
              int stage = 0, buf = 0;
              uint32_t phase = 0, bphase = 0;
              bool ok = true;                                // this lane's waits (elect_one)
              for (int tile = pair; tile < tiles; tile += pairs) {
                  for (int kb = 0; kb < g.kb; ++kb) {
                      ok = ok && mbar_wait(&full[stage], phase, abort_flag, g.err);
                      ok = ok && mbar_wait(&tempty[buf], bphase ^ 1u, abort_flag, g.err);
                      tc_fence_after();
                      if (elect_one() && ok) {
#pragma unroll
                          for (int k = 0; k < 4; ++k)
                              tc_mma8_2(tmem + (uint32_t)(buf * 256), sdesc_at(da, stage * C::STAGE + k * 32),
                                        sdesc_at(db, stage * C::STAGE + k * 32), C::IDESC, k != 0);
                          tc_commit2_mc(&tfull[buf], (uint16_t)0x3);
                          tc_commit2_mc(&empty[stage], (uint16_t)0x3);
                      }
                      __syncwarp();
                      if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                      buf ^= 1;
                      if (buf == 0) bphase ^= 1u;
                  }
              }
              if (elect_one()) tc_commit2_mc(mma_done, (uint16_t)0x1);
              __syncwarp();
              const unsigned long long t0 = globaltimer();
              while (!mbar_try_wait(mma_done, 0) && globaltimer() - t0 < kWaitLimitNs) {
              }
          }
          __syncwarp();
      } else if (warp == 2) {
          // scales of this CTA's rows times those of each side's columns, a
          // chunk of blocks at a time (fetched by the epilogue warps themselves
          // they cost 7 of 50 us at 1350 x 3072 x 12288)
          int slot = 0;
          uint32_t phase = 0;
          bool ok = true;
          for (int tile = pair; tile < tiles && ok; tile += pairs) {
              int mb, nb;
              place(tile, mb, nb);
              const int m0 = mb * 256 + (int)rank * 128 + lane;
              const float* sw0 = g.sw + (size_t)min(nb * BN / kBlock, g.sw_rows - 1) * g.kb;
              const float* sw1 = g.sw + (size_t)min((nb * BN + COLS) / kBlock, g.sw_rows - 1) * g.kb;
              for (int kb = 0; kb < g.kb; kb += kChunk) {
                  if (!mbar_wait_warp(&sempty[slot], phase ^ 1u, abort_flag, g.err)) { ok = false; break; }
                  float* dst = scales + slot * (C::SLOT / 4) + lane;
#pragma unroll
                  for (int i = 0; i < kChunk; i += 2) {
                      float a[2][4], w[2][2];
#pragma unroll
                      for (int k = 0; k < 2; ++k) {
                          const int b = min(kb + i + k, g.kb - 1);
#pragma unroll
                          for (int r = 0; r < 4; ++r)     // (rows past M: any scale, their results are clipped)
                              a[k][r] = ld_chain(g.sa + (size_t)b * g.M + min(m0 + 32 * r, g.M - 1));
                          w[k][0] = ld_chain(sw0 + b);
                          w[k][1] = ld_chain(sw1 + b);
                      }
#pragma unroll
                      for (int k = 0; k < 2; ++k)
#pragma unroll
                          for (int r = 0; r < 4; ++r) {
                              dst[(i + k) * 256 + 32 * r] = a[k][r] * w[k][0];
                              dst[(i + k) * 256 + 128 + 32 * r] = a[k][r] * w[k][1];
                          }
                  }
                  __syncwarp();
                  if (lane == 0) mbar_arrive(&sfull[slot]);
                  if (++slot == kSlots) { slot = 0; phase ^= 1u; }
              }
          }
      }
    } else {
        setmaxnreg_inc<kRegsEpilogue>();
        const int quarter = warp & 3, side = (warp >> 2) - 1;    // TMEM lane quarter; half of the columns
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(side * COLS);
        const uint32_t leader0 = mapa_shared(smem_u32(&tempty[0]), 0);
        uint8_t* slab = staging + (warp - 4) * C::SLAB;
        uint64_t* rbar = rbars + (warp - 4);
        float* bias = vectors + (warp - 4) * 2 * COLS;
        float* gate = bias + COLS;
        uint32_t rphase = 0;
        bool pending = false;                              // a residual slab requested and not awaited
        int buf = 0, slot = 0;
        uint32_t bphase = 0, sphase = 0;
        bool ok = true;
        auto request = [&](int col, int row) {             // the residual of the slab at col
            if (lane == 0) {
                bulk_wait_read<0>();
                mbar_arrive_expect_tx(rbar, C::SLAB);
                tma_load_2d(slab, &tmR, rbar, col, row);
            }
            pending = true;
        };
        for (int tile = pair; tile < tiles && ok; tile += pairs) {
            int mb, nb;
            place(tile, mb, nb);
            int m0 = mb * 256 + (int)rank * 128 + quarter * 32, n0 = nb * BN + side * COLS;
            int end = min(n0 + COLS, g.N);
            const bool rows = m0 < g.M;
            if (RESID && rows && n0 < end) request(n0, m0);
            // bias and gate of the tile's columns, on their way to shared memory meanwhile
            // (not where no row waits for them: the next tile's would be under way too)
            if (rows && 4 * lane < COLS && n0 + 4 * lane < g.N) {
                if (g.bias) cp_async16(bias + 4 * lane, g.bias + n0 + 4 * lane);
                if (RESID && g.gate) cp_async16(gate + 4 * lane, g.gate + n0 + 4 * lane);
            }
            uint64_t acc[COLS / 2];
#pragma unroll
            for (int c = 0; c < COLS / 2; ++c) acc[c] = 0ull;
            for (int kb = 0; kb < g.kb; ++kb) {
                const int in = kb % kChunk;
                if (in == 0 && !mbar_wait_warp(&sfull[slot], sphase, abort_flag, g.err)) { ok = false; break; }
                const float s = scales[slot * (C::SLOT / 4) + in * 256 + side * 128 + quarter * 32 + lane];
                const uint64_t s2 = pack64(__float_as_uint(s), __float_as_uint(s));
                if (!mbar_wait_warp(&tfull[buf], bphase, abort_flag, g.err)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 64) {
                    uint32_t p[64];
                    tmem_ld32(lanes + (uint32_t)(buf * 256 + c0), *reinterpret_cast<uint32_t(*)[32]>(&p[0]));
                    tmem_ld32(lanes + (uint32_t)(buf * 256 + c0 + 32), *reinterpret_cast<uint32_t(*)[32]>(&p[32]));
                    tmem_ld_wait();
                    if (c0 + 64 == COLS) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_remote_relaxed(leader0 + (uint32_t)buf * 8);
                    }
#pragma unroll
                    for (int c = 0; c < 64; c += 2)
                        acc[(c0 + c) / 2] = fma2(pack64(p[c], p[c + 1]), s2, acc[(c0 + c) / 2]);
                }
                buf ^= 1;
                if (buf == 0) bphase ^= 1u;
                if (in + 1 == kChunk || kb + 1 == g.kb) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sempty[slot]);
                    if (++slot == kSlots) { slot = 0; sphase ^= 1u; }
                }
            }
            if (!ok) break;
            if (!rows) continue;
            cp_async_wait();
            __syncwarp();
            // the tile's columns, a slab at a time (addresses from an opaque copy
            // of the lane: worked out before the loop over K they would spill in it)
            int l = lane;
            asm volatile("" : "+r"(l));
            if constexpr (RESID) {                         // (the tile's place anew, for the same reason)
                int again = tile;
                asm volatile("" : "+r"(again));
                place(again, mb, nb);
                m0 = mb * 256 + (int)rank * 128 + quarter * 32;
                n0 = nb * BN + side * COLS;
                end = min(n0 + COLS, g.N);
            }
            const uint32_t piece0 = (uint32_t)(l * 128), swap = (uint32_t)(l & 7);
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += SC) {
                const int col0 = n0 + c0;
                if (col0 >= end) break;
                if constexpr (RESID) {
                    if (pending && ok) ok = mbar_wait_warp(rbar, rphase, abort_flag, g.err);
                    if (ok) {
                        rphase ^= 1u;
                        pending = false;
                    }
                } else {
                    if (lane == 0) bulk_wait_read<0>();
                    __syncwarp();
                }
                constexpr int E = 16 / (int)sizeof(T);     // columns of a 16-byte piece
#pragma unroll
                for (int c = 0; c < SC; c += E) {
                    float v[E];
#pragma unroll
                    for (int j = 0; j < E; j += 2) {
                        const float2 f = unpack64(acc[(c0 + c + j) / 2]);
                        v[j] = f.x;
                        v[j + 1] = f.y;
                    }
                    if (g.bias) {
#pragma unroll
                        for (int j = 0; j < E; j += 4) {
                            const float4 b = *reinterpret_cast<const float4*>(bias + c0 + c + j);
                            v[j] += b.x; v[j + 1] += b.y; v[j + 2] += b.z; v[j + 3] += b.w;
                        }
                    }
                    if constexpr (GELU) {
#pragma unroll
                        for (int j = 0; j < E; j += 2) gelu_pair<sizeof(T) == 2>(v[j], v[j + 1]);
                    }
                    T* at = reinterpret_cast<T*>(slab + piece0 + (((c / E) ^ swap) << 4));
                    if constexpr (RESID) {
                        float r[E];
                        load_piece(at, r);
#pragma unroll
                        for (int j = 0; j < E; j += 4) {
                            float4 t = make_float4(1.f, 1.f, 1.f, 1.f);
                            if (g.gate) t = *reinterpret_cast<const float4*>(gate + c0 + c + j);
                            v[j] = fmaf(t.x, v[j], r[j]);
                            v[j + 1] = fmaf(t.y, v[j + 1], r[j + 1]);
                            v[j + 2] = fmaf(t.z, v[j + 2], r[j + 2]);
                            v[j + 3] = fmaf(t.w, v[j + 3], r[j + 3]);
                        }
                    }
                    store_piece(at, v);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && ok) {
                    tma_store_2d(&tmC, slab, col0, m0);
                    bulk_commit();
                }
                if (RESID && ok && col0 + SC < end) request(col0 + SC, m0);
            }
        }
        if (lane == 0) bulk_wait_read<0>();                // the slabs stay until their stores have read them
        if (pending) {                                     // after a wait has given up: no copy is left in flight
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(rbar, rphase) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
    }
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(own_base, 512);
    }
}

using PairKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const Gemm8Args);
template <typename T, int BN>
PairKernel pair_kernel(bool gelu, bool resid) {
    if (gelu) return resid ? gemm8_pair_kernel<T, BN, true, true> : gemm8_pair_kernel<T, BN, true, false>;
    return resid ? gemm8_pair_kernel<T, BN, false, true> : gemm8_pair_kernel<T, BN, false, false>;
}

// Pairs resident at a time.
int resident_pairs(const Ctx* c, PairKernel k, size_t smem) {
    static PerDevice<int> cap;
    const int n = cap.get(c->device, [&](int& v) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(c->num_sms / 2 * 2, 1, 1);
        cfg.blockDim = dim3(kPairThreads, 1, 1);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&v, (const void*)k, &cfg) == cudaSuccess && v >= 1) return true;
        cudaGetLastError();
        v = c->num_sms / 2 > 0 ? c->num_sms / 2 : 1;
        return false;
    });
    return n < c->num_sms / 2 ? n : c->num_sms / 2;
}

template <typename T, int BN>
wdc_status launch(Ctx* c, const void* A, const void* W, Gemm8Args g, cudaStream_t s) {
    using Cf = Pair8Cfg<BN>;
    static PerDevice<bool> fits;
    const bool regs_ok = fits.get(c->device, [](bool& ok) {
        bool smem = ok = true;
        for (int f = 0; f < 4; ++f) {
            const PairKernel k = pair_kernel<T, BN>(f & 1, f & 2);
            smem &= allow_smem(k, Cf::SMEM);
            // the warpgroups' register requests must fit the launch allocation,
            // or setmaxnreg.inc would wait forever: refuse to launch otherwise
            cudaFuncAttributes fa;
            ok &= cudaFuncGetAttributes(&fa, k) == cudaSuccess && fa.maxThreadsPerBlock >= kPairThreads &&
                  (uint32_t)fa.numRegs * kPairThreads >= 128 * kRegsControl + 256 * kRegsEpilogue;
        }
        cudaGetLastError();
        return smem && ok;
    });
    if (!regs_ok) return fail(c, WDC_ERR_UNSUPPORTED, "fp8 GEMM kernel's register allocation is below its warpgroup split");
    const PairKernel k = pair_kernel<T, BN>(g.gelu != 0, g.res != nullptr);
    g.m_tiles = (g.M - 1) / 256 + 1;
    g.n_tiles = (g.N - 1) / BN + 1;
    const long long tiles = (long long)g.m_tiles * g.n_tiles;
    if (tiles > 0x3fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "fp8 GEMM: more than 2^30 tiles");
    // raster groups whose rows of W (at most about 40 MB) stay in L2 while A
    // streams past them once a group
    int gn = (int)(40.0e6 / ((double)BN * g.K));
    gn = gn < 1 ? 1 : (gn > g.n_tiles ? g.n_tiles : gn);
    const int groups = (g.n_tiles + gn - 1) / gn;
    g.group_n = (g.n_tiles + groups - 1) / groups;
    constexpr CUtensorMapDataType kOut = sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const uint64_t K = g.K, N = g.N, M = g.M, ldc = N * sizeof(T);
    CUtensorMap ta, tw, tc, tr;
    std::string why;
    if (!encode_tmap_2d(&ta, A, K, M, K, kBlock, 128, &why, CU_TENSOR_MAP_DATA_TYPE_UINT8) ||
        !encode_tmap_2d(&tw, W, K, N, K, kBlock, BN / 2, &why, CU_TENSOR_MAP_DATA_TYPE_UINT8) ||
        !encode_tmap_2d(&tc, g.out, N, M, ldc, 128 / sizeof(T), 32, &why, kOut) ||
        !encode_tmap_2d(&tr, g.res ? g.res : g.out, N, M, ldc, 128 / sizeof(T), 32, &why, kOut))
        return fail(c, WDC_ERR_CUDA, why);
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_GEMM, s);
        const int pairs = resident_pairs(c, k, Cf::SMEM);
        launch_kernel(k, dim3(2 * (unsigned)(tiles < pairs ? tiles : pairs)), kPairThreads, Cf::SMEM, s, 2, ta, tw, tc, tr, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp8 GEMM launch: ") + cudaGetErrorString(e));
    return WDC_OK;
}

}  // namespace

wdc_status launch_gemm8_pair(Ctx* c, const void* A, const void* W, Gemm8Args g, int bn, cudaStream_t s) {
    if (c->cfg.dtype == WDC_BF16)
        return bn == 256 ? launch<__nv_bfloat16, 256>(c, A, W, g, s) : launch<__nv_bfloat16, 128>(c, A, W, g, s);
    return bn == 256 ? launch<float, 256>(c, A, W, g, s) : launch<float, 128>(c, A, W, g, s);
}

}  // namespace wdc
