// Attention of a chunk of new tokens over a paged cache on the tcgen05 tensor
// cores (sm_103a): o = softmax(q K^T / sqrt(d)) V, a token seeing the tokens of
// its sequence up to a limit (include/wdc.h).  Q bf16 [T, heads, d]; K bf16 and
// V fp16 in pages [page][d] of a key head; S = Q K^T in fp32, P in fp16, O and the
// row sums in fp32; d = 64 or 128.
//
// One CTA per (sequence, key head, block of query rows) or a part of its keys, with
// the roles of the dense attention (attn_tc.cu): a TMA producer, an MMA issuer and
// a softmax warpgroup of one thread a row for each tile.  What differs:
//  * Rows are (token, query head of the key head's group), token-major: a tile
//    of 128 rows is 128 / G tokens of all G heads of a group, one TMA box of the
//    packed q.  A single token's group shares one read of the cache.
//  * K and V come page by page: a step of BK keys is BK / page boxes (or a part
//    of one), whose page numbers the producer's lanes look up a step ahead.  A
//    page number out of range becomes a coordinate past the pool, which TMA fills
//    with zeros, like the pages behind a sequence's end.
//  * V lies as the cache holds it, keys along its rows: the MMA takes it as an
//    MN-major operand.
//  * Behind the sequence's last token its last page may hold anything.  Scores
//    there are masked; a probability of 0 times an infinity or NaN of V would not
//    be 0, so the producer zeroes those rows of the last step's V in shared
//    memory before that step's PV products.
//  * Each row has a limit of its own.  A row that has seen nothing yet (masked, or
//    scores of -infinity) takes the next tile's maximum as its exponent base, as at
//    the first step, and nothing over from before it.
//  * P is fp16, as the PV product takes it, and so are the exponents (exp2_pair_f); row sums
//    add these probabilities in fp32 (mixed-precision adds).
//  * A base is a rounded product, off by up to 2^-24 of itself: 8 at scores of 2^27,
//    still within what fp16 holds.
// Measured: one token of 32 heads on 8 of 128 in 16 sequences of 16000 keys 5.9 TB/s,
// 0.87 of a copy (one tile: bound by memory, what is missing are the parts' starts and
// ends); 24 heads of 128, 13568 tokens onto themselves 1640 to 1730 TFLOP/s, 48 of 64, 17776
// 1180 to 1200 (two tiles: bound by the chain S -> softmax -> P -> PV, whose S and P have one
// buffer a tile, 0.77 us a step of 64 keys of 128 or 1.0 of 128 keys of 64).
// Where there are few units, each is split over its keys into parts of equal
// numbers of steps (find_item), which the last of them to be done (one tile) or a second kernel
// (two) merges in order.
#include "attn_softmax.cuh"
#include "dit_kernels.cuh"
#include "paged_index.h"
#include "ptx.cuh"

#include <climits>
#include <type_traits>

namespace wdc {

namespace {

constexpr int BQ = 128;                // rows a tile

// NT tiles a CTA.  Two: chunks, 12 warps, one CTA an SM.  One: chunks whose rows
// fit a tile (single tokens above all), 8 warps, two CTAs an SM, so that one
// streams the cache while the other starts or ends.
template <int D, int NT>
struct PagedCfg {
    static constexpr int BK = (NT == 2 ? 128 : 64) * 64 / D;   // keys a step
    static constexpr int THREADS = 128 * (1 + NT);
    static constexpr int ATOMS = D / 64;                       // 128-byte atoms along d
    static constexpr uint32_t Q_TILE = BQ * D * 2;
    static constexpr uint32_t K_TILE = BK * D * 2;
    static constexpr uint32_t STAGE = 2 * K_TILE;              // 32 KB, or 16 KB for one tile
    static constexpr int STAGES = NT == 2 ? 5 : (D == 64 ? 5 : 4);
    static constexpr uint32_t SMEM = NT * Q_TILE + STAGES * STAGE + 1024 + 256;
    static constexpr uint32_t TMEM_COLS = NT == 2 ? 512 : 256;
    static constexpr int CTAS = 3 - NT;                        // an SM
    static constexpr int MIN_STEPS = NT == 1 ? 6 : 8;          // of a part of a split unit
    // two tiles: registers a thread, 168 at launch (65536 / 384, a multiple of 8),
    // of which the control warpgroup hands most to the softmax warpgroups
    static constexpr uint32_t REGS_CONTROL = D == 64 ? 40 : 88;
    static constexpr uint32_t REGS_SOFTMAX = D == 64 ? 232 : 208;
    static_assert(128 * REGS_CONTROL + 256 * REGS_SOFTMAX <= 384 * 168, "register split exceeds the launch");
    static_assert(NT * (BK + BK / 2 + D) <= (int)TMEM_COLS, "S, P and O exceed tensor memory");
    static_assert(CTAS * (SMEM + 1024) <= 228 * 1024, "shared memory");
    __device__ static constexpr uint32_t s_col(int t) { return (uint32_t)(BK + BK / 2 + D) * t; }
    __device__ static constexpr uint32_t p_col(int t) { return s_col(t) + BK; }
    __device__ static constexpr uint32_t o_col(int t) { return s_col(t) + BK + BK / 2; }
};

struct PagedArgs {
    int T, heads, kv, G, tpt;          // G query heads a key head, tpt tokens a tile
    int sequences, q_blocks, max_new;  // q_blocks: of max_new tokens
    int by_length;                     // whole units go longest sequence first
    int items, wave;                   // most parts of units (0: none is split); parts that run at a time
    int page_log2, pages, width, frame;
    const int *table, *length, *start;
    float scale_log2;
    __nv_bfloat16* o;
    float* part_o;                     // [item][rows_unit][d]
    float2* part_ml;                   // [item][rows_unit] base, row sum
    int rows_unit;                     // rows of a unit (host's bound)
    unsigned* counter;                 // one tile: [item] parts of a split unit that are done; 0 between launches
    int4* record;                      // two tiles: [item] sequence, head, query block; parts of the unit (high half) and which it is
    unsigned* err;
};

__device__ __forceinline__ PagedSeq sequence(const PagedArgs& g, int b) {
    return paged_seq(g.start[b], g.start[b + 1], g.length[b], g.T, g.width << g.page_log2);
}

// A unit is (sequence, key head, block of NT * tpt tokens).  Where there are so
// few that whole units would leave SMs without work, or units of different
// lengths, each is split into parts of `chunk` steps: the fewest for which all
// parts run in k rounds of the SMs, with the k = 1 .. kRounds of the least
// estimated time, if that is less than the whole units'.  Estimates are in steps:
// kStart a unit for its start and end, kPart a part (whose sums go out in fp32), and
// what merging takes.  One tile is bound by memory, whose bandwidth few CTAs fill too (0.55:
// one step's time of a lone CTA); of two tiles, units of like length take whole rounds,
// others fill the gaps that the longest leave, up to a share of the last.  Both sides
// (us, whole, split): 300 tokens onto 3000, 32 heads of 128, 46 and 38; 1024 onto 2048,
// 16 of 64, 35 and 30; four sequences of up to 900 onto 3000, 16 of 128, 54 and 64;
// 4096 onto none, 8 of 128, 56 and 59.
// The lengths are the device's, so the first warp of each CTA works the plan out, two
// sequences a lane, in whole numbers as floats (exact below 2^24).  (A kernel of
// its own for the plan and one for the merging cost 10 of 48 us at one token of 32
// heads over 32000.)
constexpr int kRounds = 3;
constexpr int kPlanned = 2;            // sequences a lane; more than 32 of these are not split

// What a CTA does: part `part` of `parts` of a unit.  The blocks with the most keys
// come first in a sequence.  Where its blocks differ, over all heads, so that what
// begins last is short (head by head: causal over 3000 tokens of 16 heads of 128 58 us,
// 42 so; over 13568 of 24 746 and 705); where they do not, head by head, so that a
// head's keys stay in L2 (17776 tokens of 48 heads of 64 onto themselves 3235 us, over all heads 3416).
struct Item : PagedSeq {
    int b, h, qb, part, parts, chunk;
    int j0, nj;                        // its steps
    int slot;                          // of the unit's first part in the plan: where its workspace rows begin
};

template <int D, int NT>
__device__ bool find_item(const PagedArgs& g, int index, int lane, Item& it) {
    constexpr int BK = PagedCfg<D, NT>::BK, kMin = PagedCfg<D, NT>::MIN_STEPS;
    constexpr float kStart = NT == 2 ? 8.f : 6.f, kPart = NT == 2 ? 11.f : 6.f;
    // merging: one tile's by four warps, eight parts of a row of D / 4 lanes at a time
    const float turns = ceilf((float)(g.rows_unit * D) / 512.f);
    auto merging = [&](float parts) { return NT == 2 ? (D == 64 ? 6.f : 10.f) : 2.f + turns * ceilf(parts / 8.f); };
    constexpr unsigned kAll = 0xffffffffu;
    const int block = NT * g.tpt;
    float with = 0.f;                  // steps a part; 0: whole units
    float units[kPlanned], steps[kPlanned];
    bool by_length = false;
    if (g.items > 0 || g.by_length) {
        float n = 0.f, work = 0.f, bound = 0.f, most = 0.f, least = 3e38f;
#pragma unroll
        for (int i = 0; i < kPlanned; ++i) {
            const int b = 32 * i + lane;
            units[i] = 0.f;
            steps[i] = b < g.sequences ? 0.f : -1.f;
            if (b < g.sequences) {
                const PagedSeq s = sequence(g, b);
                const int rows = min(s.n, g.max_new);
                if (rows > 0) {
                    const float low = (float)((paged_limit(s, g.frame, min(rows, block) - 1) + BK - 1) / BK);
                    units[i] = (float)((rows + block - 1) / block * g.kv);
                    steps[i] = (float)((paged_limit(s, g.frame, s.n - 1) + BK - 1) / BK);
                    least = fminf(least, low);
                    most = fmaxf(most, steps[i]);
                    n += units[i];
                    work += units[i] * 0.5f * (steps[i] + low);
                    bound += units[i] * steps[i];
                }
            }
        }
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) {
            n += __shfl_xor_sync(kAll, n, o);
            work += __shfl_xor_sync(kAll, work, o);
            bound += __shfl_xor_sync(kAll, bound, o);
            most = fmaxf(most, __shfl_xor_sync(kAll, most, o));
            least = fminf(least, __shfl_xor_sync(kAll, least, o));
        }
        // (the order takes a CTA about 5 us: a long sequence that begins last costs more)
        by_length = g.by_length && most - least > 64.f;
        const float wave = (float)g.wave;
        const bool alike = 4.f * least >= 3.f * most;
        auto estimate = [&](float c, float parts, float start, float late) {
            const float rounds = ceilf(parts / wave);
            if (NT == 1) return fmaxf(work / wave, 0.55f * c) + rounds * start;
            return (alike ? rounds * c : fmaxf(c, work / wave + late * c)) + rounds * start;
        };
        float best = g.items > 0 ? estimate(most, n, kStart, 0.3f) : 0.f;
#pragma unroll 1
        for (int k = 1; k <= kRounds && g.items > 0 && most > (float)kMin; ++k) {
            const float items = (float)min(k * g.wave, g.items);
            // (with the places all full, and no part short: no less than that)
            if (n >= items || estimate(bound / items, items, kPart, 0.6f) + merging(2.f) >= best) continue;
            float c, parts;
            if (g.sequences == 1) {    // as many parts a unit as there are places
                c = fmaxf((float)kMin, ceilf(most / floorf(items / n)));
                parts = n * ceilf(most / c);
            } else {
                // sum u ceil(s / c) lies between sum u s / c and that + n
                float lo = fminf(most, fmaxf((float)kMin, floorf(bound / items)));
                float hi = fminf(most, fmaxf(lo, ceilf(bound / (items - n)) + 1.f));
#pragma unroll 1
                do {
                    c = plan_middle(lo, hi);
                    parts = 0.f;
#pragma unroll
                    for (int i = 0; i < kPlanned; ++i) parts += units[i] * fmaxf(1.f, ceilf(steps[i] / c));
                    parts = (float)__reduce_add_sync(kAll, (unsigned)parts);
                    if (lo == hi) break;
                    if (parts <= items) hi = c;
                    else lo = c + 1.f;
                } while (true);
            }
            auto offer = [&](float c, float parts) {
                const float est = estimate(c, parts, kPart, 0.6f) + merging(ceilf(most / c));
                if (c < most && est < best) {
                    best = est;
                    with = c;
                }
            };
            if (parts <= items) {
                offer(c, parts);
                // fewer parts, as many as merge at a time (60 tokens onto 3000, 24 heads
                // of 128: 45 us, 27 so, 59 whole)
                const float eighth = ceilf(most / 8.f);
                if (NT == 1 && eighth > c) offer(eighth, fminf(parts, ceilf(bound / eighth) + n));
            }
        }
    }
    if (with == 0.f) {                 // whole units in order, some of them empty
        const int r = index / g.q_blocks;
        it.b = r / g.kv;
        if (it.b >= g.sequences) return false;
        if (by_length) {               // the sequence of that rank instead, ties in order
            int rank[kPlanned] = {};
#pragma unroll
            for (int k = 0; k < kPlanned; ++k)
#pragma unroll 4
                for (int o = 0; o < min(32, g.sequences - 32 * k); ++o) {
                    const float other = __shfl_sync(kAll, steps[k], o);
#pragma unroll
                    for (int i = 0; i < kPlanned; ++i)
                        rank[i] += other > steps[i] || (other == steps[i] && 32 * k + o < 32 * i + lane);
                }
#pragma unroll
            for (int i = 0; i < kPlanned; ++i) {
                const unsigned at = __ballot_sync(kAll, rank[i] == r / g.kv);
                if (at) it.b = 32 * i + __ffs(at) - 1;
            }
        }
        static_cast<PagedSeq&>(it) = sequence(g, it.b);
        const bool even = 4ll * paged_limit(it, g.frame, min(it.n, block) - 1) >= 3ll * paged_limit(it, g.frame, it.n - 1);
        const int unit = index % (g.kv * g.q_blocks);
        it.h = even ? unit / g.q_blocks : unit % g.kv;
        it.qb = g.q_blocks - 1 - (even ? unit % g.q_blocks : unit / g.kv);
        it.part = it.slot = 0;
        it.parts = 1;
        it.chunk = INT_MAX;
        return it.qb * block < it.n;
    }
    int before = 0;
#pragma unroll
    for (int i = 0; i < kPlanned; ++i) {
        const int mine = (int)fmaxf(1.f, ceilf(steps[i] / with)), n = (int)units[i] * mine;
        int sum = n;                   // inclusive over the lanes
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(kAll, sum, o);
            if (lane >= o) sum += v;
        }
        const unsigned past = __ballot_sync(kAll, before + sum > index);
        if (past) {
            const int at = __ffs(past) - 1;
            const int r = index - before - __shfl_sync(kAll, sum - n, at);
            it.b = 32 * i + at;
            it.parts = __shfl_sync(kAll, mine, at);
            static_cast<PagedSeq&>(it) = sequence(g, it.b);
            const int nq = (min(it.n, g.max_new) + block - 1) / block, unit = r / it.parts;
            it.part = r - unit * it.parts;
            it.h = unit % g.kv;
            it.qb = max(0, nq - 1 - unit / g.kv);
            it.chunk = (int)with;
            it.slot = index - it.part;
            return true;
        }
        before += __shfl_sync(kAll, sum, 31);
    }
    return false;
}

template <int N>
__device__ __forceinline__ void softmax_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory"); }

// Merges the parts of a unit's rows, in the parts' order: o = sum_p 2^(m_p - m) O_p /
// sum_p 2^(m_p - m) l_p with m the largest base so far.  D / 4 lanes a row, rows
// w, w + step, ... of the unit's by this warp; AHEAD parts loaded at a time (past
// L1, which may hold the workspace's earlier contents).
template <int D, int NT>
__device__ __forceinline__ void merge_parts(const PagedArgs& g, const Item& un, int w, int step, int lane) {
    constexpr int LANES = D / 4, ROWS = 32 / LANES, AHEAD = NT == 1 ? 8 : 4;
    const int tok0 = un.qb * NT * g.tpt, rows = min(min(un.n, g.max_new) - tok0, NT * g.tpt) * g.G;
    const int col = (lane % LANES) * 4;
    for (int r = w * ROWS + lane / LANES; r < rows; r += step * ROWS) {
        const size_t p0 = (size_t)un.slot * g.rows_unit + r;
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = 0; p < un.parts; p += AHEAD) {
            float2 ml[AHEAD];
            float4 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const size_t row = p0 + (size_t)min(p + k, un.parts - 1) * g.rows_unit;
                ml[k] = __ldcg(g.part_ml + row);
                v[k] = __ldcg(reinterpret_cast<const float4*>(g.part_o + row * D + col));
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (p + k >= un.parts) ml[k].x = -INFINITY;
                top = fmaxf(top, ml[k].x);
            }
            const float a = m == -INFINITY ? 0.f : ex2(m - top);
            l *= a;
            acc.x *= a; acc.y *= a; acc.z *= a; acc.w *= a;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (ml[k].x == -INFINITY) continue;          // (saw nothing)
                const float b = ex2(ml[k].x - top);
                l = fmaf(ml[k].y, b, l);
                acc.x = fmaf(v[k].x, b, acc.x);
                acc.y = fmaf(v[k].y, b, acc.y);
                acc.z = fmaf(v[k].z, b, acc.z);
                acc.w = fmaf(v[k].w, b, acc.w);
            }
            m = top;
        }
        const float inv = l != 0.f ? 1.0f / l : 0.f;
        const size_t t = (size_t)un.row0 + tok0 + r / g.G;
        *reinterpret_cast<uint2*>(g.o + (t * g.heads + un.h * g.G + r % g.G) * D + col) =
            make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
    }
}

// Two tiles: the merging of a split unit's rows is work for more than one CTA, so
// kMergeCtas for each of its parts.  (300 rows of 8 heads on one over 6000 31.5 -> 26.7
// us against sixteen for each part's place, of which a unit's first did the work; one or
// two for each part are slower where there are few parts, eight where there are many.)
constexpr int kMergeCtas = 4;
template <int D>
__global__ void __launch_bounds__(256) paged_merge_kernel(const __grid_constant__ PagedArgs g) {
    chain_release();
    chain_wait();
    const int4 rec = g.record[blockIdx.x];
    const int parts = rec.w >> 16, part = rec.w & 0xffff;
    if (parts < 2) return;
    Item un;
    static_cast<PagedSeq&>(un) = sequence(g, rec.x);
    un.h = rec.y;
    un.qb = rec.z;
    un.parts = parts;
    un.slot = blockIdx.x - part;
    merge_parts<D, 2>(g, un, (part * kMergeCtas + blockIdx.y) * 8 + (threadIdx.x >> 5), parts * kMergeCtas * 8, threadIdx.x & 31);
}

template <int D, int NT>
__global__ void __launch_bounds__(PagedCfg<D, NT>::THREADS, PagedCfg<D, NT>::CTAS)
    attn_paged_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                      const __grid_constant__ CUtensorMap tv, const __grid_constant__ PagedArgs g) {
    using C = PagedCfg<D, NT>;
    constexpr int BKV = C::BK;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sq = smem;                                       // [NT tiles][ATOMS][128 x 128 B]
    uint8_t* skv = smem + NT * C::Q_TILE;                     // [STAGES][K | V], each [ATOMS][BK x 128 B]
    uint64_t* bars = reinterpret_cast<uint64_t*>(skv + C::STAGES * C::STAGE);
    uint64_t* q_full = bars;
    uint64_t* kv_full = q_full + 1;
    uint64_t* kv_empty = kv_full + C::STAGES;
    uint64_t* s_full = kv_empty + C::STAGES;                  // [2]
    uint64_t* s_free = s_full + 2;                            // [2]
    uint64_t* p_full = s_free + 2;                            // [2]
    uint64_t* p_free = p_full + 2;                            // [2]
    uint64_t* o_final = p_free + 2;                           // [2]
    uint64_t* v_ready = o_final + 2;                          // the last step's V is clear behind the sequence
    uint64_t* stagger = v_ready + 1;                          // tile 0 has stored its first P
    uint64_t* mma_done = stagger + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wg = warp >> 2;
    __shared__ Item s_item;
    __shared__ int s_has, s_last;
    if (threadIdx.x == 64) {
        mbar_init(q_full, 1);
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&kv_full[s], 2);         // K's producer and V's
            mbar_init(&kv_empty[s], NT);       // each MMA issuer's, or the one's and the producer's
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&s_full[w], 1);
            mbar_init(&s_free[w], 4);
            mbar_init(&p_full[w], 4);
            mbar_init(&p_free[w], 1);
            mbar_init(&o_final[w], 1);
        }
        mbar_init(v_ready, 1);
        mbar_init(stagger, 4);
        mbar_init(mma_done, NT);
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tq);
        prefetch_tmap(&tk);
        prefetch_tmap(&tv);
    }
    // (a CTA past the first round may have nothing to do: it asks before it allocates)
    const bool early = blockIdx.x < (unsigned)g.wave;
    if (warp == 1 && early) {
        tmem_alloc(tmem_slot, C::TMEM_COLS);
        tmem_relinquish();
    }
    if (warp >= 4) {                                          // rows of a tile that no box fills
        const int row = threadIdx.x & 127;
        if (row >= g.tpt * g.G) {
            uint4* q = reinterpret_cast<uint4*>(sq + ((warp >> 2) - 1) * C::Q_TILE + row * 128);
            for (int a = 0; a < C::ATOMS; ++a)
                for (int i = 0; i < 8; ++i) q[a * (BQ * 8) + i] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
    }
    chain_wait();
    if (warp == 0) {
        Item it{};
        const bool has = find_item<D, NT>(g, blockIdx.x, lane, it);
        if (has) {
            const int keys = paged_limit(it, g.frame, min((it.qb + 1) * NT * g.tpt, it.n) - 1);
            const int steps = (keys + BKV - 1) / BKV;
            it.j0 = it.parts > 1 ? min(it.part * it.chunk, steps) : 0;
            it.nj = (it.parts > 1 ? min(it.j0 + it.chunk, steps) : steps) - it.j0;
        }
        if (lane == 0) {
            s_item = it;
            s_has = has;
            if (NT == 2 && (int)blockIdx.x < g.items)
                g.record[blockIdx.x] = make_int4(it.b, it.h, it.qb, has ? it.parts << 16 | it.part : 0);
        }
    } else if (warp == 3 && lane == 0 && blockIdx.x < (unsigned)g.sequences) {
        // a sequence's numbers, whether it has new tokens or not (there are as many CTAs, or more)
        const int b = blockIdx.x;
        if (!paged_given(g.start[b], g.start[b + 1], g.length[b], g.T, g.width << g.page_log2, g.max_new))
            atomicOr(g.err, kErrBounds);
    }
    __syncthreads();
    if (!s_has) {
        if (warp == 1 && early) {
            tc_fence_after();
            tmem_dealloc(*tmem_slot, C::TMEM_COLS);
        }
        return;
    }
    if (!early) {
        if (warp == 1) {
            tmem_alloc(tmem_slot, C::TMEM_COLS);
            tmem_relinquish();
        }
        __syncthreads();
    }
    tc_fence_after();
    chain_release();
    const uint32_t tmem = *tmem_slot;
    const Item un = s_item;

    const int tok0 = un.qb * NT * g.tpt;                      // the chunk's first token here
    const int nt = NT == 2 && tok0 + g.tpt < un.n ? 2 : 1;    // tiles with rows
    const int j0 = un.j0, nj = un.nj;
    const int page = 1 << g.page_log2;
    const int used = (un.len + page - 1) >> g.page_log2;      // pages of the sequence
    // rows of the last step's V that lie behind the sequence, in its last page
    const int last0 = (j0 + nj - 1) * BKV;
    const int clear0 = un.len - last0, clear1 = min(BKV, (used << g.page_log2) - last0);
    const bool clear = nj > 0 && clear0 < clear1;

    if (wg == 0) {
        if constexpr (NT == 2) setmaxnreg_dec<C::REGS_CONTROL>();
        if (warp == 0 || warp == 3) {
            // producers: warp 0 of K, warp 3 of Q and V (one for all three is behind
            // with pages of 16: 16 boxes a step at d = 128)
            const bool of_v = warp == 3;
            if (nj > 0) {
                if (of_v && elect_one()) {
                    mbar_arrive_expect_tx(q_full, (uint32_t)(nt * C::ATOMS * g.G * g.tpt) * 128u);
                    for (int t = 0; t < nt; ++t)
                        for (int a = 0; a < C::ATOMS; ++a)
                            tma_load_4d(sq + t * C::Q_TILE + a * (BQ * 128), &tq, q_full, 64 * a, 0, un.h,
                                        un.row0 + tok0 + t * g.tpt);
                }
                __syncwarp();
                const CUtensorMap* map = of_v ? &tv : &tk;
                uint8_t* tile0 = skv + (of_v ? C::K_TILE : 0);
                const int rows = min(page, BKV), boxes = BKV / rows;
                // page of this lane's box of step j
                auto lookup = [&](int j) {
                    int p = g.pages;                          // past the pool: filled with zeros
                    const int i = ((j * BKV) >> g.page_log2) + lane;
                    if (lane < boxes && i < used) {
                        p = paged_page(g.table[(size_t)un.b * g.width + i], g.pages);
                        if (p < 0) {
                            atomicOr(g.err, kErrBounds);
                            p = g.pages;
                        }
                    }
                    return p;
                };
                int stage = 0;
                uint32_t phase = 0;
                uint32_t armed = 0, parity = 0;               // per stage: a copy was issued; its phase
                int next = lookup(j0);
                bool ok = true;
                for (int j = j0; j < j0 + nj; ++j) {
                    const int p = next;
                    if (j + 1 < j0 + nj) next = lookup(j + 1);
                    if (!mbar_wait_warp(&kv_empty[stage], phase ^ 1u, abort_flag, g.err)) { ok = false; break; }
                    if (elect_one()) {
                        mbar_arrive_expect_tx(&kv_full[stage], C::K_TILE);
                        if (NT == 2 && nt == 1 && !of_v) mbar_arrive(&kv_empty[stage]);
                    }
                    __syncwarp();
                    if (lane < boxes) {
                        uint8_t* dst = tile0 + stage * C::STAGE + lane * rows * 128;
                        const int y = boxes > 1 ? 0 : (j * BKV) & (page - 1);
                        for (int a = 0; a < C::ATOMS; ++a)
                            tma_load_4d(dst + a * (BKV * 128), map, &kv_full[stage], 64 * a, y, un.h, p);
                    }
                    __syncwarp();
                    armed |= 1u << stage;
                    parity = (parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                }
                if (ok && clear && of_v) {
                    const int st = (nj - 1) % C::STAGES;
                    if (mbar_wait_warp(&kv_full[st], (parity >> st) & 1, abort_flag, g.err)) {
                        for (int a = 0; a < C::ATOMS; ++a) {
                            uint4* v = reinterpret_cast<uint4*>(skv + st * C::STAGE + C::K_TILE + a * (BKV * 128));
                            for (int i = clear0 * 8 + lane; i < clear1 * 8; i += 32) v[i] = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(v_ready);
                    }
                }
                if (of_v) {
                    const unsigned long long t0 = globaltimer();
                    while (!mbar_try_wait(q_full, 0) && globaltimer() - t0 < kWaitLimitNs) {
                    }
                }
                for (int s = 0; s < C::STAGES; ++s) {
                    if (!((armed >> s) & 1)) continue;
                    const unsigned long long t0 = globaltimer();
                    while (!mbar_try_wait(&kv_full[s], (parity >> s) & 1) && globaltimer() - t0 < kWaitLimitNs) {
                    }
                }
            }
        } else if (((NT == 1 && warp == 1) || (NT == 2 && warp - 1 < nt && warp <= 2)) && nj > 0) {
            constexpr uint32_t idesc_s = idesc_bf16(BQ, BKV);
            constexpr uint32_t idesc_o = idesc_f16_mn(BQ, D);    // P (fp16, TMEM) x V (fp16, MN-major)
            const int t = NT == 1 ? 0 : warp - 1;
            constexpr bool kOneLane = D == 128;                  // (as in the dense attention)
            auto leads = [] { return kOneLane || elect_one(); };
            auto rejoin = [] { if (!kOneLane) __syncwarp(); };
            if (!kOneLane || elect_one()) {
                const uint64_t dq = sdesc_sw128(smem_u32(sq) + t * C::Q_TILE), dk = sdesc_sw128(smem_u32(skv));
                const uint64_t dv = sdesc_sw128_mn(smem_u32(skv) + C::K_TILE, BKV * 128);
                bool ok = mbar_wait(q_full, 0, abort_flag, g.err);        // this lane's waits (elect_one)
                int stage = 0, prev = 0;
                uint32_t phase = 0;
                auto issue_s = [&](int st) {
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const uint32_t off = (ks >> 2) * (BQ * 128) + (ks & 3) * 32;
                        const uint32_t koff = (ks >> 2) * (BKV * 128) + (ks & 3) * 32;
                        tc_mma(tmem + C::s_col(t), sdesc_at(dq, off), sdesc_at(dk, st * C::STAGE + koff), idesc_s, ks != 0);
                    }
                };
                // O(t) (+)= P(t) V: 16 keys (rows of V, 2 KB) = 8 columns of P an MMA
                auto issue_pv = [&](int st, bool acc) {
#pragma unroll
                    for (int ks = 0; ks < BKV / 16; ++ks)
                        tc_mma_ts(tmem + C::o_col(t), tmem + C::p_col(t) + ks * 8, sdesc_at(dv, st * C::STAGE + ks * 2048),
                                  idesc_o, (acc || ks != 0) ? 1u : 0u);
                };
                // tiles half a step apart (as in the dense attention), from two steps on
                if (t == 1 && nj > 1) ok = ok && mbar_wait(stagger, 0, abort_flag, g.err);
                ok = ok && mbar_wait(&kv_full[0], 0, abort_flag, g.err);
                for (int j = 0; j < nj; ++j) {
                    // here K(j) has landed, and S(t, j - 1) is in the softmax's registers
                    tc_fence_after();
                    if (leads() && ok) {
                        issue_s(stage);
                        tc_commit(&s_full[t]);
                    }
                    rejoin();
                    const int cur = stage;
                    if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                    auto next_k = [&]() { if (j + 1 < nj) ok = ok && mbar_wait(&kv_full[stage], phase, abort_flag, g.err); };
                    if (D == 128) next_k();
                    if (j > 0) {
                        ok = ok && mbar_wait(&p_full[t], (j - 1) & 1, abort_flag, g.err);
                        tc_fence_after();
                        if (leads() && ok) {
                            issue_pv(prev, j > 1);
                            tc_commit(&p_free[t]);
                            tc_commit(&kv_empty[prev]);
                        }
                        rejoin();
                    }
                    prev = cur;
                    if (D == 64) next_k();
                    if (j + 1 < nj) ok = ok && mbar_wait(&s_free[t], j & 1, abort_flag, g.err);
                }
                ok = ok && mbar_wait(&p_full[t], (nj - 1) & 1, abort_flag, g.err);
                if (clear) ok = ok && mbar_wait(v_ready, 0, abort_flag, g.err);
                tc_fence_after();
                if (leads() && ok) {
                    issue_pv(prev, nj > 1);
                    tc_commit(&kv_empty[prev]);
                    tc_commit(&o_final[t]);
                }
                rejoin();
                if (leads()) {
                    tc_commit(mma_done);
                    if (NT == 2 && nt == 1) mbar_arrive(mma_done);
                }
            }
            __syncwarp();
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(mma_done, 0) && globaltimer() - t0 < kWaitLimitNs) {
            }
        }
    } else {
        if constexpr (NT == 2) setmaxnreg_inc<C::REGS_SOFTMAX>();
        // softmax warpgroups: t = tile, quarter = TMEM lane quarter
        const int t = wg - 1;
        const int quarter = warp & 3;
        const int row = quarter * 32 + lane;                 // row within the tile = TMEM lane
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t s_addr = tmem + lane_base + C::s_col(t);
        const uint32_t p_addr = tmem + lane_base + C::p_col(t);
        const uint32_t o_addr = tmem + lane_base + C::o_col(t);
        const int i = tok0 + t * g.tpt + row / g.G;          // the chunk's token
        const bool valid = row < g.tpt * g.G && i < min(un.n, g.max_new);
        const int lim = valid ? paged_limit(un, g.frame, i) : INT_MAX;    // (other rows hold what they hold)
        const int min_lim = __reduce_min_sync(0xffffffffu, lim);
        const bool work = __any_sync(0xffffffffu, valid);    // else the warp only keeps step
        float m_run = -INFINITY, l_run = 0.f;
        const uint64_t scale2 = pair(g.scale_log2, g.scale_log2);
        bool ok = true, s_ready = false;
        const int mine = t < nt ? nj : 0;
        auto hand_over = [&](int j) {
            if (lane == 0) {
                mbar_arrive(&p_full[t]);
                if (NT == 2 && j == 0 && t == 0) mbar_arrive(stagger);
            }
        };
        // one step (j counts this CTA's) of a warp with rows; `masked`: some row's
        // limit lies within it.  (The masked steps, the last few, are code of their
        // own: as a branch in every step they cost 5% at d = 128.)
        auto step = [&](int j, auto masked) {
            if (!s_ready && !mbar_wait_warp(&s_full[t], j & 1, abort_flag, g.err)) return false;
            tc_fence_after();
            float s[BKV];
#pragma unroll
            for (int c = 0; c < BKV / 32; ++c) tmem_ld32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
            tmem_ld_wait();
            // S(t) is in registers: the MMA may compute S(t, j+1) now
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_free[t]);
            const int k0 = (j0 + j) * BKV;
            (void)k0;
            if constexpr (decltype(masked)::value) {
                const int left = lim - k0;
#pragma unroll
                for (int c = 0; c < BKV; ++c)
                    if (c >= left) s[c] = -INFINITY;
            }
            auto tile_max = [&]() {
                // 8 independent partial maxima (short dependency chains)
                float m8[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) m8[q] = fmaxf(s[q], s[8 + q]);
#pragma unroll
                for (int c = 16; c < BKV; c += 16)
#pragma unroll
                    for (int q = 0; q < 8; ++q) m8[q] = fmax3(m8[q], s[c + q], s[c + 8 + q]);
                return fmax3(fmax3(m8[0], m8[1], m8[2]), fmax3(m8[3], m8[4], m8[5]), fmaxf(m8[6], m8[7]));
            };
            // numerators 2^(s * scale - base) into p (fp16 pairs); returns their fp32 sum
            uint32_t p[BKV / 2];
            auto numerators = [&](float base) {
                float lo[2] = {0.f, 0.f}, hi[2] = {0.f, 0.f};
                const uint64_t nm2 = pair(-base, -base);
#pragma unroll
                for (int c = 0; c < BKV; c += 2)
                    p[c / 2] = exp2_pair_f(s[c], s[c + 1], scale2, nm2, lo[(c / 2) & 1], hi[(c / 2) & 1]);
                return (lo[0] + lo[1]) + (hi[0] + hi[1]);
            };
            float base = m_run;
            if (__any_sync(0xffffffffu, l_run == 0.f)) {     // a row that has seen nothing yet
                const float top = tile_max() * g.scale_log2;
                if (l_run == 0.f) base = top == -INFINITY ? 0.f : top;
            }
            float sum;
            // A numerator above 2^8 implies a row sum above 2^8 (so does a
            // non-finite one): only then take the tile max, move the base and
            // recompute, as a second pass of the same code.
#pragma unroll 1
            for (int pass = 0;; ++pass) {
                sum = numerators(base);
                const bool redo = pass == 0 && !(sum <= 256.0f);
                if (!__any_sync(0xffffffffu, redo)) break;
                if (redo) base = fmaxf(base, tile_max() * g.scale_log2);
            }
            const bool moved = __any_sync(0xffffffffu, base != m_run);
            // 1 when the base stays; 0 before a row has seen something, when the base it
            // leaves means nothing (and may lie above the new one by more than ex2 holds)
            const float corr = l_run == 0.f ? 0.f : ex2(m_run - base);
            l_run = l_run * corr + sum;
            m_run = base;
            // PV(t, j-1) must be done before P(t) is overwritten and O(t) rescaled
            if (j > 0) {
                if (!mbar_wait_warp(&p_free[t], (j - 1) & 1, abort_flag, g.err)) return false;
                tc_fence_after();
            }
            if (j > 0 && moved) {
                // PV(t, j-1) is complete: rescale O in place
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(o_addr + c, o);
                    tmem_ld_wait();
                    uint32_t lo[16], hi[16];
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        lo[q] = __float_as_uint(__uint_as_float(o[q]) * corr);
                        hi[q] = __float_as_uint(__uint_as_float(o[16 + q]) * corr);
                    }
                    tmem_st16(o_addr + c, lo);
                    tmem_st16(o_addr + c + 16, hi);
                }
            }
            // P (BK / 2 columns of fp16 pairs)
#pragma unroll
            for (int c = 0; c < BKV / 2; c += 16) tmem_st16(p_addr + c, *reinterpret_cast<uint32_t(*)[16]>(&p[c]));
            const bool next = D == 64 && mbar_test(&s_full[t], (j + 1) & 1);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            hand_over(j);
            if (D == 64) s_ready = __all_sync(0xffffffffu, next);
            return true;
        };
        if (work) {
            const int open = max(0, min(mine, (min_lim - j0 * BKV) / BKV));
            int j = 0;
#pragma unroll 1
            for (; ok && j < open; ++j) ok = step(j, std::false_type{});
#pragma unroll 1
            for (; ok && j < mine; ++j) ok = step(j, std::true_type{});
        } else {                                             // a warp without rows only keeps step
            for (int j = 0; ok && j < mine; ++j) {
                ok = mbar_wait_warp(&s_full[t], j & 1, abort_flag, g.err);
                if (ok && lane == 0) mbar_arrive(&s_free[t]);
                if (ok && j > 0) ok = mbar_wait_warp(&p_free[t], (j - 1) & 1, abort_flag, g.err);
                if (ok) hand_over(j);
            }
        }
        if (ok && mine > 0) ok = mbar_wait_warp(&o_final[t], 0, abort_flag, g.err);
        if (ok && work) {
            tc_fence_after();
            const bool seen = l_run != 0.f;                  // (a NaN is seen)
            const bool split = un.parts > 1;
            const float inv = seen ? 1.0f / l_run : 0.f;
            if constexpr (NT == 2) {
                // A row's pieces are a lane's; stored from there a warp would write 16 bytes
                // of 32 rows at a time.  So they pass through the tile's Q, which no MMA reads
                // any more, 16-byte pieces swapped within groups of 8 by the row, and go out
                // whole rows at a time; partial sums half a row at a time.  (Two prompts of
                // 6001, 24 heads of 128, 327 -> 308 us; six ragged sequences 75.6 -> 69.4.)
                constexpr int PIECES = D / 8, ROWS = 32 / PIECES;          // pieces of a staged row, rows a store
                uint8_t* stage = sq + t * C::Q_TILE + quarter * (32 * D * 2);
                const unsigned rows = __ballot_sync(0xffffffffu, valid);
                const size_t prow = (size_t)(un.slot + un.part) * g.rows_unit + t * g.tpt * g.G + row;
                const size_t at = split ? prow * D : ((size_t)(un.row0 + i) * g.heads + un.h * g.G + row % g.G) * D;
                if (split && valid) g.part_ml[prow] = make_float2(seen ? m_run : -INFINITY, l_run);
                __syncwarp();
                auto put = [&](int piece, uint4 w) {
                    *reinterpret_cast<uint4*>(stage + lane * (D * 2) + ((piece ^ (lane & 7)) << 4)) = seen ? w : make_uint4(0, 0, 0, 0);
                };
                auto send = [&](auto* out, int col) {        // staged rows to out + their places + col
                    __syncwarp();
#pragma unroll 4
                    for (int r0 = 0; r0 < 32; r0 += ROWS) {
                        const int r = r0 + lane / PIECES, piece = lane % PIECES;
                        const size_t to = __shfl_sync(0xffffffffu, (unsigned long long)at, r);
                        const uint4 w = *reinterpret_cast<const uint4*>(stage + r * (D * 2) + ((piece ^ (r & 7)) << 4));
                        if ((rows >> r) & 1u) *reinterpret_cast<uint4*>(out + to + col + piece * (16 / sizeof(*out))) = w;
                    }
                    __syncwarp();
                };
                if (split) {
#pragma unroll
                    for (int c0 = 0; c0 < D; c0 += D / 2) {
#pragma unroll
                        for (int c = 0; c < D / 2; c += 32) {
                            uint32_t o[32];
                            if (mine > 0) {
                                tmem_ld32(o_addr + c0 + c, o);
                                tmem_ld_wait();
                            }
#pragma unroll
                            for (int q = 0; q < 8; ++q) put(c / 4 + q, make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]));
                        }
                        send(g.part_o, c0);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        if (mine > 0) {
                            tmem_ld32(o_addr + c, o);
                            tmem_ld_wait();
                        }
                        auto two = [&](int k) { return pack2(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv); };
#pragma unroll
                        for (int q = 0; q < 4; ++q) put(c / 8 + q, make_uint4(two(8 * q), two(8 * q + 2), two(8 * q + 4), two(8 * q + 6)));
                    }
                    send(g.o, 0);
                }
            } else {
                const size_t prow = (size_t)(un.slot + un.part) * g.rows_unit + t * g.tpt * g.G + row;
                __nv_bfloat16* out = g.o + ((size_t)(un.row0 + i) * g.heads + un.h * g.G + row % g.G) * D;
                float* po = g.part_o + prow * D;
                if (split && valid) g.part_ml[prow] = make_float2(seen ? m_run : -INFINITY, l_run);
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    __syncwarp();                            // (lanes with a row come from its stores)
                    if (mine > 0) {
                        tmem_ld32(o_addr + c, o);
                        tmem_ld_wait();
                    }
                    if (!valid) continue;
                    if (split) {
                        float4* dst = reinterpret_cast<float4*>(po + c);
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            dst[q] = seen ? make_float4(__uint_as_float(o[4 * q]), __uint_as_float(o[4 * q + 1]),
                                                        __uint_as_float(o[4 * q + 2]), __uint_as_float(o[4 * q + 3]))
                                          : make_float4(0.f, 0.f, 0.f, 0.f);
                    } else {
                        uint4* dst = reinterpret_cast<uint4*>(out + c);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint4 w = make_uint4(0, 0, 0, 0);
                            if (seen) {
                                w.x = pack2(__uint_as_float(o[8 * q + 0]) * inv, __uint_as_float(o[8 * q + 1]) * inv);
                                w.y = pack2(__uint_as_float(o[8 * q + 2]) * inv, __uint_as_float(o[8 * q + 3]) * inv);
                                w.z = pack2(__uint_as_float(o[8 * q + 4]) * inv, __uint_as_float(o[8 * q + 5]) * inv);
                                w.w = pack2(__uint_as_float(o[8 * q + 6]) * inv, __uint_as_float(o[8 * q + 7]) * inv);
                            }
                            dst[q] = w;
                        }
                    }
                }
            }
        }
        tc_fence_before();
        if (NT == 1 && un.parts > 1) {
            // the last of a unit's parts to be done merges them
            __threadfence();
            softmax_barrier<NT * 128>();
            if (threadIdx.x == 128) {
                unsigned* counter = g.counter + un.slot;
                const bool last = atomicInc(counter, (unsigned)un.parts - 1u) == (unsigned)un.parts - 1u;
                __threadfence();
                s_last = last;
            }
            __syncwarp();
            softmax_barrier<NT * 128>();
            if (s_last) merge_parts<D, NT>(g, un, warp - 4, NT * 4, lane);
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, C::TMEM_COLS);
    }
}

template <int D, int NT>
wdc_status launch(Ctx* c, const void* q, const wdc_paged_cache* p, PagedArgs g, cudaStream_t s) {
    using Cf = PagedCfg<D, NT>;
    static PerDevice<bool> fits;
    const bool regs_ok = fits.get(c->device, [](bool& ok) {
        const bool smem = allow_smem(attn_paged_kernel<D, NT>, Cf::SMEM);
        // the warpgroups' register requests must fit the launch allocation,
        // or setmaxnreg.inc would wait forever: refuse to launch otherwise
        cudaFuncAttributes fa;
        ok = cudaFuncGetAttributes(&fa, attn_paged_kernel<D, NT>) == cudaSuccess && fa.maxThreadsPerBlock >= Cf::THREADS &&
             (NT == 1 || (uint32_t)fa.numRegs * Cf::THREADS >= 128 * Cf::REGS_CONTROL + 256 * Cf::REGS_SOFTMAX);
        cudaGetLastError();
        return smem && ok;
    });
    if (!regs_ok) return fail(c, WDC_ERR_UNSUPPORTED, "paged attention kernel's register allocation is below its warpgroup split");
    CUtensorMap tq, tk, tv;
    std::string why;
    const uint64_t row = (uint64_t)D * 2, pg = (uint64_t)p->page;
    const uint64_t qd[4] = {D, (uint64_t)g.G, (uint64_t)g.kv, (uint64_t)g.T}, qs[3] = {row, row * g.G, row * g.heads};
    const uint32_t qb[4] = {64, (uint32_t)g.G, 1, (uint32_t)g.tpt};
    const uint64_t kd[4] = {D, pg, (uint64_t)g.kv, (uint64_t)g.pages}, ks[3] = {row, row * pg, row * pg * g.kv};
    const uint32_t kb[4] = {64, (uint32_t)(p->page < Cf::BK ? p->page : Cf::BK), 1, 1};
    if (!encode_tmap_4d(&tq, q, qd, qs, qb, false, &why) || !encode_tmap_4d(&tk, p->k, kd, ks, kb, false, &why) ||
        !encode_tmap_4d(&tv, p->v, kd, ks, kb, true, &why))
        return fail(c, WDC_ERR_CUDA, why);
    g.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    const int block = NT * g.tpt;
    g.q_blocks = (g.max_new + block - 1) / block;
    const long long units = (long long)g.sequences * g.kv * g.q_blocks;
    if (units > 0x7fffffffll) return fail(c, WDC_ERR_UNSUPPORTED, "paged attention: more than 2^31 - 1 thread blocks");
    // (the workspace holds the partial rows of a few rounds of CTAs)
    g.rows_unit = (g.max_new < block ? g.max_new : block) * g.G;
    g.wave = Cf::CTAS * c->num_sms;
    const long long room = (long long)c->num_sms * 256 * c->attn_part_rounds / g.rows_unit;
    // rounds of parts: the fewest that like units would fill by nine tenths; two or
    // more where sequences may differ
    long long items = 0;
    for (int k = g.sequences > 1 ? 2 : 1; k <= kRounds; ++k) {
        items = (long long)k * g.wave;
        if (units > 0 && 10 * (items / units * units) >= 9 * items) break;
    }
    if (items > room) items = room / g.wave * g.wave;
    const long long steps = (((long long)g.width << g.page_log2) + Cf::BK - 1) / Cf::BK;
    g.items = c->attn_part && g.sequences <= 32 * kPlanned && steps > Cf::MIN_STEPS && units < items ? (int)items : 0;
    // more units than run at a time: the longest sequences may go first, so that none
    // begins last (64 tokens over up to 4000, 8 key heads of 128: 132 -> 112 us)
    g.by_length = NT == 1 && g.q_blocks == 1 && g.sequences > 1 && g.sequences <= 32 * kPlanned && units > g.wave;
    g.counter = c->attn_counters;
    g.record = reinterpret_cast<int4*>(c->attn_records);
    g.part_o = c->attn_part;
    g.part_ml = reinterpret_cast<float2*>(c->attn_ml);
    const long long grid = g.items > units ? g.items : units;      // (parts, or whole units)
    OverlapScope ov(c, s);
    {
        LaunchScope ls(c, WDC_K_ATTN, s);
        launch_kernel(attn_paged_kernel<D, NT>, dim3((unsigned)grid), Cf::THREADS, Cf::SMEM, s, 1, tq, tk, tv, g);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("paged attention launch: ") + cudaGetErrorString(e));
    if (NT == 2 && g.items > 0) {
        LaunchScope ls(c, WDC_K_OTHER, s);
        launch_kernel(paged_merge_kernel<D>, dim3((unsigned)g.items, kMergeCtas), 256, 0, s, 1, g);
        e = cudaGetLastError();
        if (e != cudaSuccess) return fail(c, WDC_ERR_CUDA, std::string("paged attention merge launch: ") + cudaGetErrorString(e));
    }
    return WDC_OK;
}

}  // namespace

wdc_status op_attention_paged(Ctx* c, const void* q, const wdc_paged_cache* p, const int* q_start, int T, int heads,
                              int max_new, int frame, void* o, cudaStream_t s) {
    PagedArgs g{};
    if (wdc_status st = check_cache(c, p, &g.page_log2)) return st;
    if (T < 0 || heads < 1 || max_new < 0 || frame < 0) return fail(c, WDC_ERR_INVALID_ARG, "paged attention: bad sizes");
    if (heads % p->kv_heads) return fail(c, WDC_ERR_INVALID_ARG, "paged attention: heads must be a multiple of kv_heads");
    if (heads / p->kv_heads > BQ) return fail(c, WDC_ERR_UNSUPPORTED, "paged attention: at most 128 query heads a key head");
    if (T == 0 || p->sequences == 0 || max_new == 0) return WDC_OK;
    if (!q || !o || !q_start) return fail(c, WDC_ERR_INVALID_ARG, "paged attention: null pointer");
    if (((uintptr_t)q | (uintptr_t)o) & 15) return fail(c, WDC_ERR_INVALID_ARG, "paged attention: q and o must be 16-byte aligned");
    if ((uintptr_t)q_start & 3) return fail(c, WDC_ERR_INVALID_ARG, "paged attention: q_start must be 4-byte aligned");
    g.T = T; g.heads = heads; g.kv = p->kv_heads; g.G = heads / p->kv_heads; g.tpt = BQ / g.G;
    g.max_new = max_new < T ? max_new : T;
    g.pages = p->pages; g.width = p->table_width; g.frame = frame;
    g.table = p->table; g.length = p->length; g.start = q_start;
    g.o = reinterpret_cast<__nv_bfloat16*>(o);
    g.err = c->err;
    g.sequences = p->sequences;
    if (g.max_new <= g.tpt) return p->head_dim == 64 ? launch<64, 1>(c, q, p, g, s) : launch<128, 1>(c, q, p, g, s);
    return p->head_dim == 64 ? launch<64, 2>(c, q, p, g, s) : launch<128, 2>(c, q, p, g, s);
}

}  // namespace wdc
