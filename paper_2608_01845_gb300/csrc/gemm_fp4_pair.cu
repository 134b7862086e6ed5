// Product of e2m1 matrices with scales (see gemm_fp4.cu), CTA-pair kernel: many rows.
//
// A pair of CTAs takes a tile of 256 rows of A by 256 of W (gated: by 128 of W_gate and
// the same 128 of W_up), 256 x 256 x 64 block-scaled MMAs issued by the even one.  Each CTA
// holds its 128 rows of A and half of the weights' rows (gated: the even CTA W_gate's, the odd
// one W_up's), and the scales of its rows of A and of all the tile's weights, which the
// issuing thread copies from each CTA's shared memory to its tensor memory.  The sums of all of
// K stay in 256 columns of tensor memory, the scales of a stage in 48 of the others: the
// 240 columns of five stages leave no room for a second tile's sums, so eight epilogue
// warps first take the tile to their registers, a row a lane and 128 columns a warp, and
// hand tensor memory back before they finish it.
//
// Tiles that would make a last round of fewer than the pairs are split over K, and these
// parts come first: each writes its sums to the context's workspace, a warp's 32 x 128
// at a time, and the warp that comes last (a counter a warp's piece) adds all of them in
// the order of K and finishes the tile, while the MMAs of the whole tiles run; nobody
// waits for another.
//
// Bound by the tensor core and its power: 17776 x 16384 x 4096 with GELU 370 us (6.4 PFLOP/s)
// by itself, 425 to 435 in a loop, where the power cap holds the SM clock at 1.63 GHz; 17776
// x 4096 x 16384 330 us (7.2 PFLOP/s, four times the measured bf16 burst is 7.8).  A stage
// takes about 600 cycles, its MMAs 512: the twelve copies of its scales pass through the same
// queue (between MMAs, or from another warp, they cost more: 4864 x 4096 x 16384 85 us, then
// 94 to 97); from a tile's last MMA to the next one's first pass about 1000 (commit, the reads
// into registers 175, the arrival at the issuer; the first copies are under way by then: gated
// 1576 x 10240 x 4096 52.5 -> 51.6).  Tiles of 192 columns with
// room for two left the scales 2.7 stages, and waiting for their columns cost more: 159 us.
// Parts of the last tiles before the whole ones: 1350 x 4096 x 16384 44.6 -> 36 us.  K is split behind a
// whole round only, and where the tiles behind it are at most half the pairs: 1024 x 2560 x 16384 (40
// tiles) 25 us, for 11 of operations.  The 128 sums a thread leave 40 of the launch's registers for the
// rest of the epilogue: nine of the twelve forms spill 20 to 32 bytes.
#include "gemm_fp4.cuh"
#include "pair_epilogue.cuh"

namespace wdc {

namespace {

constexpr int kPairThreads = 384;           // three warpgroups: TMA producer, MMA issuer, vectors; epilogue (two)
// Registers a thread: 168 at launch (65536 / 384, a multiple of 8), of which the
// first warpgroup hands most to the others.
constexpr uint32_t kRegsControl = 56, kRegsEpilogue = 224, kRegsLaunch = 168;
static_assert(128 * kRegsControl + 256 * kRegsEpilogue <= 384 * kRegsLaunch, "register split exceeds the launch");

struct Pair4Cfg {
    static constexpr uint32_t TILE = 128 * 128, S_BYTES = 4 * kPiece4;         // codes of 128 rows; scales of 128 rows
    static constexpr uint32_t STAGE = 2 * TILE + 3 * S_BYTES;
    static constexpr int STAGES = 5;
    static constexpr int SCALE_COLS = 48;                                      // of a stage, in tensor memory
    static constexpr uint32_t SLAB = 32 * 128, STAGING = 8 * SLAB;
    static constexpr uint32_t VECTORS = 2 * 3 * 128 * 4;                       // [half of the columns][rw, bias, gate][128]
    static constexpr uint32_t IDESC = idesc_e2m1(256, 256);
    static constexpr size_t SMEM = STAGES * STAGE + STAGING + VECTORS + 512 + 1024;
    static_assert(STAGE % 1024 == 0 && SMEM <= 227 * 1024, "shared memory per CTA");
    static_assert(256 + STAGES * SCALE_COLS <= 512, "tensor memory");
};

enum Form { kStore = 0, kGelu = 1, kResid = 2, kGeluResid = 3, kSiluGated = 4, kGeluGated = 5 };

template <typename T, int FORM>
__global__ void __launch_bounds__(kPairThreads, 1)
    gemm4_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                      const __grid_constant__ CUtensorMap tmU, const __grid_constant__ CUtensorMap tmSA,
                      const __grid_constant__ CUtensorMap tmSW, const __grid_constant__ CUtensorMap tmSU,
                      const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmR,
                      const __grid_constant__ Gemm4Args g) {
    using C = Pair4Cfg;
    constexpr bool GATED = FORM >= kSiluGated, RESID = FORM == kResid || FORM == kGeluResid;
    constexpr bool GELU = FORM == kGelu || FORM == kGeluResid || FORM == kGeluGated;
    constexpr int BN = GATED ? 128 : 256;          // columns of C in a tile
    constexpr int COLS = BN / 2;                   // and of those a warp finishes
    constexpr int SC = 128 / (int)sizeof(T);       // columns of a slab
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + C::STAGES * C::STAGE;
    float* vectors = reinterpret_cast<float*>(staging + C::STAGING);
    uint64_t* full = reinterpret_cast<uint64_t*>(vectors + C::VECTORS / 4);    // even CTA: both CTAs' tiles landed
    uint64_t* empty = full + C::STAGES;
    uint64_t* tfull = empty + C::STAGES;           // the tile's sums are complete
    uint64_t* tempty = tfull + 1;                  // even CTA: both CTAs' warps have them in registers
    uint64_t* vfull = tempty + 1;                  // the tile's vectors
    uint64_t* vempty = vfull + 1;
    uint64_t* mma_done = vempty + 1;
    uint64_t* rbars = mma_done + 1;                // [8 warps] residual slabs
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(rbars + 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    // this pair's jobs: at most one part of a tile, then a whole tile each
    const int first = pair < g.tail * g.parts ? 1 : 0, jobs = first + (g.whole - pair + pairs - 1) / pairs;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(tfull, 1);
        mbar_init(tempty, 16);
        mbar_init(vfull, 1);
        mbar_init(vempty, 8);
        mbar_init(mma_done, 1);
        for (int i = 0; i < 8; ++i) mbar_init(&rbars[i], 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmW);
        prefetch_tmap(&tmSA);
        prefetch_tmap(&tmSW);
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
    // job j: its tile's place and its part of K; what the part is of (tail tile, -1: none)
    struct Job {
        int mb, nb, kb0, kb1, tail, part;
    };
    auto job = [&](int j) {
        Job t;
        int tile = pair + (j - first) * pairs;
        t.tail = -1;
        t.part = 0;
        t.kb0 = 0;
        t.kb1 = g.kb;
        if (j < first) {
            t.tail = pair / g.parts;
            t.part = pair - t.tail * g.parts;
            tile = g.whole + t.tail;
            t.kb0 = (int)((long long)t.part * g.kb / g.parts);
            t.kb1 = (int)((long long)(t.part + 1) * g.kb / g.parts);
            if (g.parts == 1) t.tail = -1;
        }
        place(tile, t.mb, t.nb);
        return t;
    };

    if (warp < 4) {
      setmaxnreg_dec<kRegsControl>();
      if (warp == 0) {
          int stage = 0;
          uint32_t phase = 0, armed = 0, parity = 0;         // per stage: a copy was issued; its phase
          bool ok = true;
          for (int j = 0; j < jobs && ok; ++j) {
              const Job t = job(j);
              const int nb = t.nb, mblock = t.mb * 2 + (int)rank;    // of 128 rows
              const int w0 = GATED ? nb * 128 : nb * 256 + (int)rank * 128;
              const CUtensorMap* weights = GATED && rank == 1 ? &tmU : &tmW;
              for (int kb = t.kb0; kb < t.kb1; ++kb) {
                  if (!mbar_wait_warp(&empty[stage], phase ^ 1u, abort_flag, g.err)) { ok = false; break; }
                  if (elect_one()) {
                      if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * C::STAGE);
                      const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
                      uint8_t* at = smem + stage * C::STAGE;
                      tma_load_2d_pair(at, &tmA, fb, kb * 128, mblock * 128);
                      tma_load_2d_pair(at + C::TILE, weights, fb, kb * 128, w0);
                      at += 2 * C::TILE;
                      tma_load_3d_pair(at, &tmSA, fb, 0, kb * 4, mblock);
                      tma_load_3d_pair(at + C::S_BYTES, &tmSW, fb, 0, kb * 4, GATED ? nb : nb * 2);
                      tma_load_3d_pair(at + 2 * C::S_BYTES, GATED ? &tmSU : &tmSW, fb, 0, kb * 4, GATED ? nb : nb * 2 + 1);
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
              const uint32_t base = smem_u32(smem);
              const uint64_t da = sdesc_sw128(base), db = sdesc_sw128(base + C::TILE), ds = sdesc_rows16(base + 2 * C::TILE);
              int stage = 0;
              uint32_t phase = 0, tphase = 0;
              bool ok = true;                                // this lane's waits (elect_one)
              // (a stage's columns are free once its tiles have landed: they could not have been
              // loaded again before the MMAs that read the columns were done)
              auto copies = [&]() {
                  const uint32_t sc = tmem + (uint32_t)(256 + stage * C::SCALE_COLS);
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                      const uint32_t at = stage * C::STAGE + k * kPiece4;
                      tc_copy_scales2(sc + 12 * k, sdesc_at(ds, at));
                      tc_copy_scales2(sc + 12 * k + 4, sdesc_at(ds, at + C::S_BYTES));
                      tc_copy_scales2(sc + 12 * k + 8, sdesc_at(ds, at + 2 * C::S_BYTES));
                  }
              };
              auto mmas = [&](bool first, bool last) {
                  const uint32_t sc = tmem + (uint32_t)(256 + stage * C::SCALE_COLS);
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                      tc_mma4_2(tmem, sdesc_at(da, stage * C::STAGE + k * 32), sdesc_at(db, stage * C::STAGE + k * 32), C::IDESC,
                                sc + 12 * k, sc + 12 * k + 4, !first || k != 0);
                  if (last) tc_commit2_mc(tfull, (uint16_t)0x3);
                  tc_commit2_mc(&empty[stage], (uint16_t)0x3);
              };
              auto advance = [&]() {
                  __syncwarp();
                  if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
              };
              for (int j = 0; j < jobs; ++j) {
                  const Job t = job(j);
                  // a tile's first copies are under way while the tile before is taken
                  ok = ok && mbar_wait(&full[stage], phase, abort_flag, g.err);
                  tc_fence_after();
                  if (elect_one() && ok) copies();
                  __syncwarp();
                  ok = ok && mbar_wait(tempty, tphase ^ 1u, abort_flag, g.err);
                  tphase ^= 1u;
                  tc_fence_after();
                  if (elect_one() && ok) mmas(true, t.kb0 + 1 == t.kb1);
                  advance();
                  for (int kb = t.kb0 + 1; kb < t.kb1; ++kb) {
                      ok = ok && mbar_wait(&full[stage], phase, abort_flag, g.err);
                      tc_fence_after();
                      if (elect_one() && ok) {
                          copies();
                          mmas(false, kb + 1 == t.kb1);
                      }
                      advance();
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
          // the tile's vectors: [half h of the 256 sums' columns][rw, bias, gate][128]
          uint32_t phase = 0;
          for (int j = 0; j < jobs; ++j) {
              const int nb = job(j).nb;
              float v[2][3][4];
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                      const int n = (GATED ? nb * 128 : nb * 256 + h * 128) + i * 32 + lane;
                      const bool in = n < g.N;
                      const float* rw = GATED && h ? g.ru : g.rw;
                      const float* b = GATED && h ? g.up_bias : g.bias;
                      v[h][0][i] = in ? ld_chain(rw + n) : 0.f;
                      v[h][1][i] = in && b ? ld_chain(b + n) : 0.f;
                      v[h][2][i] = RESID && in && g.gate ? ld_chain(g.gate + n) : 1.f;
                  }
              if (!mbar_wait_warp(vempty, phase ^ 1u, abort_flag, g.err)) break;
              phase ^= 1u;
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                  for (int k = 0; k < 3; ++k)
#pragma unroll
                      for (int i = 0; i < 4; ++i) vectors[(h * 3 + k) * 128 + i * 32 + lane] = v[h][k][i];
              __syncwarp();
              if (lane == 0) mbar_arrive(vfull);
          }
      }
    } else {
        setmaxnreg_inc<kRegsEpilogue>();
        const int quarter = warp & 3, side = (warp >> 2) - 1;    // TMEM lane quarter; part of the columns
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t leader = mapa_shared(smem_u32(tempty), 0);
        uint8_t* slab = staging + (warp - 4) * C::SLAB;
        uint64_t* rbar = rbars + (warp - 4);
        uint32_t rphase = 0, tphase = 0;
        bool pending = false;                              // a residual slab requested and not awaited
        bool ok = true;
        auto request = [&](int col, int row) {             // the residual of the slab at col
            if (lane == 0) {
                bulk_wait_read<0>();
                mbar_arrive_expect_tx(rbar, C::SLAB);
                tma_load_2d(slab, &tmR, rbar, col, row);
            }
            pending = true;
        };
        // After a wait that gave up, a warp goes on to the end of its tile and stores nothing: what it
        // hands back is handed back, and its part of a split tile is counted all the same (what that
        // tile then holds is wrong, as the error word says), so that the counters are 0 for the next launch.
        for (int j = 0; j < jobs && ok; ++j) {
            const Job t = job(j);
            const int m0 = t.mb * 256 + (int)rank * 128 + quarter * 32, n0 = t.nb * BN + side * COLS;
            const int end = min(n0 + COLS, g.N);
            bool rows = m0 < g.M;                          // the warp has something to finish
            if (RESID && rows && n0 < end && t.tail < 0) request(n0, m0);
            const float ra = m0 + lane < g.M ? ld_chain(g.ra + m0 + lane) : 0.f;
            ok = mbar_wait_warp(tfull, tphase, abort_flag, g.err);
            tc_fence_after();
            // gated: 64 columns of each half; else 128 of one
            float acc[128];
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 32) {
                const int col = GATED ? (c0 / 64) * 128 + side * 64 + c0 % 64 : side * 128 + c0;
                tmem_ld32(lanes + (uint32_t)col, *reinterpret_cast<uint32_t(*)[32]>(&acc[c0]));
            }
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote_relaxed(leader);
            ok = mbar_wait_warp(vfull, tphase, abort_flag, g.err) && ok;
            tphase ^= 1u;
            if (t.tail >= 0 && rows) {
                const size_t piece = (size_t)(t.tail * 2 + (int)rank) * 8 + (warp - 4);
                float4* parts = reinterpret_cast<float4*>(g.work) + piece * g.parts * (32 * 32) + lane;
#pragma unroll
                for (int c = 0; c < 128; c += 4)
                    __stcg(parts + t.part * (32 * 32) + c / 4 * 32, make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]));
                __threadfence();
                __syncwarp();
                unsigned before = 0;
                if (lane == 0) before = atomicAdd(g.counters + piece, 1u);
                rows = __shfl_sync(0xffffffffu, before, 0) + 1 == (unsigned)g.parts;
                if (rows) {                                // the last one: all parts, in order
                    __threadfence();
                    if (lane == 0) g.counters[piece] = 0u;
                    if (RESID && n0 < end) request(n0, m0);
#pragma unroll
                    for (int c = 0; c < 128; ++c) acc[c] = 0.f;
                    for (int q = 0; q < g.parts; ++q)
#pragma unroll
                        for (int c = 0; c < 128; c += 4) {
                            const float4 v = __ldcg(parts + q * (32 * 32) + c / 4 * 32);
                            acc[c] += v.x; acc[c + 1] += v.y; acc[c + 2] += v.z; acc[c + 3] += v.w;
                        }
                }
            }
            if (rows) {
                // rw, bias and gate of the warp's columns; gated: of W_gate's, and behind them W_up's
                const float* vec = GATED ? vectors + side * 64 : vectors + side * 3 * 128;
                const uint32_t piece0 = (uint32_t)(lane * 128), swap = (uint32_t)(lane & 7);
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
                        for (int j = 0; j < E; j += 4) {
                            const float4 s = *reinterpret_cast<const float4*>(vec + c0 + c + j);
                            const float4 b = *reinterpret_cast<const float4*>(vec + 128 + c0 + c + j);
                            v[j] = fmaf(acc[c0 + c + j] * ra, s.x, b.x);
                            v[j + 1] = fmaf(acc[c0 + c + j + 1] * ra, s.y, b.y);
                            v[j + 2] = fmaf(acc[c0 + c + j + 2] * ra, s.z, b.z);
                            v[j + 3] = fmaf(acc[c0 + c + j + 3] * ra, s.w, b.w);
                        }
                        if constexpr (GELU) {
#pragma unroll
                            for (int j = 0; j < E; j += 2) gelu_pair<sizeof(T) == 2>(v[j], v[j + 1]);
                        }
                        if constexpr (GATED) {
                            if constexpr (!GELU) {
#pragma unroll
                                for (int j = 0; j < E; j += 2) silu_pair(v[j], v[j + 1]);
                            }
#pragma unroll
                            for (int j = 0; j < E; j += 4) {
                                const float4 s = *reinterpret_cast<const float4*>(vec + 3 * 128 + c0 + c + j);
                                const float4 b = *reinterpret_cast<const float4*>(vec + 4 * 128 + c0 + c + j);
                                const float* u = &acc[GATED ? 64 + c0 + c + j : 0];
                                v[j] *= fmaf(u[0] * ra, s.x, b.x);
                                v[j + 1] *= fmaf(u[1] * ra, s.y, b.y);
                                v[j + 2] *= fmaf(u[2] * ra, s.z, b.z);
                                v[j + 3] *= fmaf(u[3] * ra, s.w, b.w);
                            }
                        }
                        T* at = reinterpret_cast<T*>(slab + piece0 + (((c / E) ^ swap) << 4));
                        if constexpr (RESID) {
                            float r[E];
                            load_piece(at, r);
#pragma unroll
                            for (int j = 0; j < E; j += 4) {
                                const float4 t = *reinterpret_cast<const float4*>(vec + 2 * 128 + c0 + c + j);
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
            __syncwarp();
            if (lane == 0) mbar_arrive(vempty);
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

using PairKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                            const CUtensorMap, const CUtensorMap, const CUtensorMap, const Gemm4Args);
template <typename T>
PairKernel pair_kernel(int form) {
    switch (form) {
        case kStore: return gemm4_pair_kernel<T, kStore>;
        case kGelu: return gemm4_pair_kernel<T, kGelu>;
        case kResid: return gemm4_pair_kernel<T, kResid>;
        case kGeluResid: return gemm4_pair_kernel<T, kGeluResid>;
        case kSiluGated: return gemm4_pair_kernel<T, kSiluGated>;
        default: return gemm4_pair_kernel<T, kGeluGated>;
    }
}

// A split product on another stream than the last one's waits for that one, as they share the
// context's workspace and counters.  (Not under capture: what a graph is ordered with is the
// caller's.)
struct SplitOrder {
    Ctx* c;
    cudaStream_t s;
    bool on;
    unsigned long long id = 0;
    SplitOrder(Ctx* c_, bool split, cudaStream_t s_) : c(c_), s(s_), on(split) {
        if (!on) return;
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(s, &st) != cudaSuccess) cudaGetLastError();
        on = st == cudaStreamCaptureStatusNone;
    }
    wdc_status begin() {
        if (!on) return WDC_OK;
        WDC_CUDA_TRY(c, cudaStreamGetId(s, &id));
        if (id != c->fp4_stream) WDC_CUDA_TRY(c, cudaStreamWaitEvent(s, c->fp4_done, 0));
        return WDC_OK;
    }
    wdc_status end() {
        if (!on) return WDC_OK;
        WDC_CUDA_TRY(c, cudaEventRecord(c->fp4_done, s));
        c->fp4_stream = id;
        return WDC_OK;
    }
};

// Pairs resident at a time.
int resident_pairs(const Ctx* c, PairKernel k) {
    static PerDevice<int> cap;
    const int n = cap.get(c->device, [&](int& v) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(c->num_sms / 2 * 2, 1, 1);
        cfg.blockDim = dim3(kPairThreads, 1, 1);
        cfg.dynamicSmemBytes = Pair4Cfg::SMEM;
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

// Parts of K that `tail` tiles are split in, before whole tiles of kb stages: the parts'
// stages, and what of their merging the next tile's stages do not hide.
int tail_parts(int tail, int pairs, int kb) {
    constexpr double kStage = 0.30, kMerge = 8.0, kPart = 0.8;     // us
    int best = 1;
    double least = kb * kStage;
    for (int p = 2; p <= 8 && tail > 0 && tail * p <= pairs && 2 * p <= kb; ++p) {
        const double merge = kMerge + p * kPart - kb * kStage;
        const double est = (kb + p - 1) / p * kStage + (merge > 0.0 ? merge : 0.0);
        if (est < least) {
            least = est;
            best = p;
        }
    }
    return best;
}

// Lets the kernels take their shared memory; false: their registers do not allow the warpgroups' split.
template <typename T>
bool ready(const Ctx* c) {
    static PerDevice<bool> fits;
    return fits.get(c->device, [](bool& ok) {
        bool smem = ok = true;
        for (int f = 0; f < 6; ++f) {
            const PairKernel k = pair_kernel<T>(f);
            smem &= allow_smem(k, Pair4Cfg::SMEM);
            // the warpgroups' register requests must fit the launch allocation,
            // or setmaxnreg.inc would wait forever: refuse to launch otherwise
            cudaFuncAttributes fa;
            ok &= cudaFuncGetAttributes(&fa, k) == cudaSuccess && fa.maxThreadsPerBlock >= kPairThreads &&
                  (uint32_t)fa.numRegs * kPairThreads >= 128 * kRegsControl + 256 * kRegsEpilogue;
        }
        cudaGetLastError();
        return smem && ok;
    });
}

// The tiles, and which of them are split over K; false: too many.
bool plan(const Ctx* c, PairKernel k, Gemm4Args& g, int* pairs) {
    g.m_tiles = (g.M - 1) / 256 + 1;
    g.n_tiles = (g.N - 1) / (g.U ? 128 : 256) + 1;
    g.kb = (g.K - 1) / kTileK4 + 1;
    const long long tiles = (long long)g.m_tiles * g.n_tiles;
    if (tiles > 0x3fffffffll) return false;
    *pairs = resident_pairs(c, k);
    g.tail = (int)(tiles % *pairs);
    g.whole = (int)(tiles - g.tail);
    g.parts = g.whole > 0 ? tail_parts(g.tail, *pairs, g.kb) : 1;
    if (g.parts > c->fp4_parts / (g.tail > 0 ? g.tail : 1)) g.parts = 1;
    return true;
}

template <typename T>
wdc_status launch(Ctx* c, Gemm4Args g, cudaStream_t s) {
    if (!ready<T>(c)) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM kernel's register allocation is below its warpgroup split");
    const bool gated = g.U != nullptr;
    const PairKernel k = pair_kernel<T>(gated ? (g.gelu ? kGeluGated : kSiluGated)
                                              : (g.res ? (g.gelu ? kGeluResid : kResid) : (g.gelu ? kGelu : kStore)));
    int pairs;
    if (!plan(c, k, g, &pairs)) return fail(c, WDC_ERR_UNSUPPORTED, "fp4 GEMM: more than 2^30 tiles");
    // raster groups whose rows of W (at most about 40 MB) stay in L2 while A
    // streams past them once a group
    int gn = (int)(40.0e6 / (256.0 * g.K * 0.5625));
    gn = gn < 1 ? 1 : (gn > g.n_tiles ? g.n_tiles : gn);
    const int groups = (g.n_tiles + gn - 1) / gn;
    g.group_n = (g.n_tiles + groups - 1) / groups;
    constexpr CUtensorMapDataType kOut = sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const uint64_t N = g.N, M = g.M, ldc = N * sizeof(T);
    CUtensorMap ta, tw, tu, tsa, tsw, tsu, tc, tr;
    std::string why;
    if (!encode_codes(&ta, g.A, g.M, g.K, 128, &why) || !encode_codes(&tw, g.W, g.N, g.K, 128, &why) ||
        !encode_codes(&tu, gated ? g.U : g.W, g.N, g.K, 128, &why) || !encode_scales(&tsa, g.sa, g.M, g.pieces, &why) ||
        !encode_scales(&tsw, g.sw, g.N, g.pieces, &why) || !encode_scales(&tsu, gated ? g.su : g.sw, g.N, g.pieces, &why) ||
        !encode_tmap_2d(&tc, g.out, N, M, ldc, 128 / sizeof(T), 32, &why, kOut) ||
        !encode_tmap_2d(&tr, g.res ? g.res : g.out, N, M, ldc, 128 / sizeof(T), 32, &why, kOut))
        return fail(c, WDC_ERR_CUDA, why);
    g.work = c->fp4_work;
    g.counters = c->fp4_counters;
    SplitOrder order(c, g.parts > 1, s);
    if (wdc_status st = order.begin()) return st;
    {
        OverlapScope ov(c, s);
        LaunchScope ls(c, WDC_K_GEMM, s);
        launch_kernel(k, dim3(2 * (unsigned)(g.whole > 0 ? pairs : g.tail * g.parts)), kPairThreads, Pair4Cfg::SMEM, s, 2, ta, tw, tu, tsa,
                      tsw, tsu, tc, tr, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("fp4 GEMM launch: ") + cudaGetErrorString(e));
    return order.end();
}

}  // namespace

bool plan_gemm4_pair(const Ctx* c, Gemm4Args& g) {
    int pairs;
    const bool bf16 = c->cfg.dtype == WDC_BF16;
    return (bf16 ? ready<__nv_bfloat16>(c) : ready<float>(c)) &&
           plan(c, bf16 ? pair_kernel<__nv_bfloat16>(kStore) : pair_kernel<float>(kStore), g, &pairs);
}

wdc_status launch_gemm4_pair(Ctx* c, const Gemm4Args& g, cudaStream_t s) {
    return c->cfg.dtype == WDC_BF16 ? launch<__nv_bfloat16>(c, g, s) : launch<float>(c, g, s);
}

}  // namespace wdc
