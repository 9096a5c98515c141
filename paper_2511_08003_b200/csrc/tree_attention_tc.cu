// Attention of many query rows over a K/V cache in bf16 (drafted trees, chunks of a prompt) on the fifth-generation
// tensor cores.
//
// A segment is up to 256 query rows of one (sequence, KV head), as two tiles of up to 128 (as many whole nodes as
// fit, so that one TMA box fetches them); a unit is 128 keys of it.  One
// CTA per SM: a warp that loads (TMA ring of K and V tiles, 32 KB each at head_dim 128), a warp that issues
// the products, two warpgroups that turn scores into weights, two warps that clean the value tiles that hold rows
// nobody may see.  Work goes in steps, each one stream's scores, weights and weighted sums:
//   more than 128 rows   stream w owns row tile w; both take every key tile
//   up to 128 rows       both streams own row tile 0 and take the key tiles in turn; joined in tensor memory at the end
// While one stream's warpgroup works on its scores the tensor cores work for the other.  Scores, weights (bf16, in the
// place of the scores they came from) and sums live in tensor memory: 2 x (128 + 128) columns.  A thread owns a
// query row, so the softmax needs no shuffles.  Sums are rescaled only when a row's maximum has grown by more than 2^8
// since they last were (weights then stay below 256, which bf16 and the fp32 sums hold as well as 1).
//
// What bounds it is the hand-over between a stream's scores and its products.  Measured with the join (4 KV heads x 128, 7
// query heads each): a tree of 64 over 50,432 rows 57 us (0.81 PFLOP/s, tensor pipe 48 % active), trees of 5 to 41 over 37,712
// ragged rows 40.5 us, a chunk of 509 over 10,944 rows 91 us (0.9 PFLOP/s of what its rows see).
#include "tcgen05.cuh"
#include "tree_attention.cuh"

#include <cuda_bf16.h>

namespace sharpv {
namespace {

constexpr int kKeys = kTcTileKeys;              // 128
constexpr int kRows = 256;                      // places for query rows: 128 a stream
constexpr int kThreads = 384;
constexpr int kLoadWarp = 8, kMmaWarp = 9, kAuxWarp = 10;       // warps 0-3, 4-7: the streams; 10, 11: aux
constexpr uint32_t kCols = 512, kSumCol = 256;  // tensor memory: scores of stream w at 128 w, sums at 256 + DP w
constexpr float kLazy = 8.f;

template <int DP>
struct Cfg {
    static constexpr int kTileBytes = 128 * DP * 2;             // 128 rows of Q, K or V
    static constexpr int kStages = DP == 64 ? 10 : 5;           // K and V tiles in turn
    static constexpr int kHalf = 128 * 128;                     // bytes of a 64-column box
};

template <int DP>
struct Shared {
    using C = Cfg<DP>;
    uint8_t q[2][C::kTileBytes];
    uint8_t tiles[C::kStages][C::kTileBytes];
    Portion part[2];                            // kt1 < 0: there are no more
    float m[128], l[128];                       // of stream 1, when the streams share their rows
    uint64_t full[C::kStages], empty[C::kStages];
    uint64_t part_full[2], part_empty[2];
    uint64_t clean[C::kStages];                 // value tiles: gone through (or nothing to do)
    uint64_t q_full, q_empty;
    uint64_t scores[2], weights[2], sums[2];    // per stream: scores formed, weights written, a portion's weighted sums added
    uint64_t merge_full, merge_done, drain;
    int poison[2];
    uint32_t tmem;
    PlanScratch<kThreads> plan;
};

// what every role derives from a portion
struct Steps {
    int tiles, n;               // key tiles, steps
    bool pair;                  // two row tiles
    __device__ __forceinline__ Steps(const Portion& p, const Split& sp) {
        tiles = p.kt1 - p.kt0;
        pair = p.s.nodes * sp.group - p.rt * sp.rows > sp.rows / 2;
        n = pair ? 2 * tiles : tiles;
    }
    __device__ __forceinline__ int of_stream(int w) const { return pair ? tiles : (tiles + 1 - w) >> 1; }
};

// Every second item of the ring (key tiles are the even ones, value tiles the odd ones): its stage, and how often the
// ring has gone round.
template <int STAGES>
struct Ring {
    int stage;
    uint32_t round;
    __device__ __forceinline__ void next() {
        stage += 2;
        if (stage >= STAGES) {
            stage -= STAGES;
            ++round;
        }
    }
    // uses of the stage for a tile of the same kind so far: with an odd number of stages every other round is one
    __device__ __forceinline__ uint32_t use() const { return STAGES % 2 ? round >> 1 : round; }
};

// keys of tile kt that are there, and whether it has to be masked
__device__ __forceinline__ int keys_left(const AttnArgs& a, const Portion& p, int kt) {
    return kt < p.kt_cache ? p.s.len - kt * kKeys : (a.split.draft ? p.s.nodes - (kt - p.kt_cache) * kKeys : 0);
}
__device__ __forceinline__ bool tile_masked(const AttnArgs& a, const Portion& p, int kt) {
    return kt >= p.kt_cache || keys_left(a, p, kt) < kKeys;
}

// Sums of two at a time (one instruction each on this architecture).
__device__ __forceinline__ uint64_t pack2(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attn_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnMaps maps) {
    using C = Cfg<DP>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 1);
            mbar_init(&sm.clean[i], 2);             // both aux warps
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.part_full[i], 1);
            mbar_init(&sm.part_empty[i], 11);           // the warps that read it
            mbar_init(&sm.scores[i], 1);
            mbar_init(&sm.weights[i], 4);
            mbar_init(&sm.sums[i], 1);
        }
        mbar_init(&sm.q_full, 1);
        mbar_init(&sm.q_empty, 1);
        mbar_init(&sm.merge_full, 128);
        mbar_init(&sm.merge_done, 128);
        mbar_init(&sm.drain, 1);
        mbar_fence_init();
    }
    if (warp == kMmaWarp) tmem_alloc(&sm.tmem, kCols);
    if (warp == kLoadWarp && lane < 5) tma_prefetch(&maps.cache_k + lane);
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kThreads>(a.seqs, a.split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    bool alive = true;          // a wait that gave up ends the role; the others then give up as well
    auto wait = [&](uint64_t* bar, uint32_t phase) {            // by one thread
        if (alive && !mbar_wait(bar, phase & 1)) alive = false;
        return alive;
    };
    auto wait_warp = [&](uint64_t* bar, uint32_t phase) {       // by a whole warp: its lanes ask together and get one answer
        if (alive) alive = mbar_wait(bar, phase & 1);
        return alive;
    };

    if (warp >= kLoadWarp) {
        fewer_registers<96>();
        if (warp == kLoadWarp) {
            if (lane == 0) {
                Walk walk(plan, first, end);
                Portion p, last;
                uint32_t it = 0, queries = 0;                       // tiles, and portions whose query rows were asked for
                for (uint32_t pn = 0; alive; ++pn) {
                    const int at = pn & 1;
                    last = p;
                    const bool more = walk.next(a.seqs, a.split, p);
                    if (!more) note_shared(a, pn > 0, last, end, plan);
                    if (pn >= 2 && !wait(&sm.part_empty[at], (pn >> 1) - 1)) break;
                    if (!more) p.kt1 = -1;
                    sm.poison[at] = 0;
                    sm.part[at] = p;
                    mbar_arrive(&sm.part_full[at]);
                    if (!more) break;
                    // query rows: whole nodes, the group's heads of each next to each other
                    const Steps st(p, a.split);
                    if (pn > 0 && !wait(&sm.q_empty, pn - 1)) break;
                    const int nodes = a.split.rows / (2 * G);
                    ++queries;
                    mbar_expect(&sm.q_full, (st.pair ? 2 : 1) * (DP / 64) * (a.split.rows / 2) * 128);
                    for (int w = 0; w < (st.pair ? 2 : 1); ++w)
#pragma unroll
                        for (int x = 0; x < DP / 64; ++x)
                            tma_load(sm.q[w] + x * C::kHalf, &maps.query, &sm.q_full, x * 64, p.h * G, p.s.node0 + (p.rt * 2 + w) * nodes);
                    for (int kt = p.kt0; kt < p.kt1 && alive; ++kt) {
                        const bool drafted = kt >= p.kt_cache;
                        const int row = drafted ? p.s.node0 + (kt - p.kt_cache) * kKeys : (int)p.s.begin + kt * kKeys;
                        for (int v = 0; v < 2; ++v, ++it) {
                            const int stage = it % C::kStages;
                            if (it >= C::kStages && !wait(&sm.empty[stage], it / C::kStages - 1)) break;
                            if (drafted && !a.split.draft) {        // the empty tile of rows without keys
                                mbar_arrive(&sm.full[stage]);
                                continue;
                            }
                            mbar_expect(&sm.full[stage], C::kTileBytes);
                            const CUtensorMap* map = drafted ? (v ? &maps.draft_v : &maps.draft_k) : (v ? &maps.cache_v : &maps.cache_k);
#pragma unroll
                            for (int x = 0; x < DP / 64; ++x)
                                tma_load(sm.tiles[stage] + x * C::kHalf, map, &sm.full[stage], x * 64, row, p.h);
                        }
                    }
                }
                if (!alive) note_shared(a, false, p, end, plan);    // nothing to join
                // copies in flight land before the CTA ends, also where the warps that wanted them gave up
                for (uint32_t i = 0; i < (uint32_t)C::kStages && i < it; ++i) {
                    const uint32_t at = it - 1 - i;
                    (void)mbar_wait(&sm.full[at % C::kStages], (at / C::kStages) & 1);
                }
                if (queries > 0) (void)mbar_wait(&sm.q_full, (queries - 1) & 1);
            }
        } else if (warp == kMmaWarp) {
            // The whole warp walks and waits, one thread issues.  The tensor cores queue only a few products, so what
            // happens between two batches is kept short: one wait that is mostly over, one commit.
            constexpr uint32_t k_shape = mma_shape(128, false), v_shape = mma_shape(DP, true);
            const uint64_t q_op = smem_operand(smem_u32(sm.q[0]), 1024, 16), k_op = smem_operand(smem_u32(sm.tiles[0]), 1024, 16);
            const uint64_t v_op = smem_operand(smem_u32(sm.tiles[0]), 1024, C::kHalf);
            Ring<C::kStages> kr{0, 0}, vr{1, 0};                        // where the next key and value tile to wait for are
            uint32_t steps0[2] = {0, 0};                                // steps of the portions before
            for (uint32_t pn = 0;; ++pn) {
                if (!wait_warp(&sm.part_full[pn & 1], pn >> 1)) break;
                const Portion& p = sm.part[pn & 1];
                if (p.kt1 < 0) break;
                const Steps st(p, a.split);
                const bool pair = __shfl_sync(0xffffffffu, (int)st.pair, 0) != 0;
                const int n = __shfl_sync(0xffffffffu, st.n, 0);
                if (!wait_warp(&sm.q_full, pn)) break;
                auto scores = [&](int t) {                              // scores of step t
                    const int w = t & 1;
                    if (!pair || w == 0) {
                        if (!wait_warp(&sm.full[kr.stage], kr.round)) return;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t q = q_op + (pair ? w : 0) * (C::kTileBytes >> 4), k = k_op + kr.stage * (C::kTileBytes >> 4);
#pragma unroll
                        for (int ks = 0; ks < DP / 16; ++ks) {
                            const uint32_t off = ((ks >> 2) * C::kHalf + (ks & 3) * 32) >> 4;
                            mma_ss(tmem + w * 128, q + off, k + off, k_shape, ks > 0);
                        }
                        mma_commit(&sm.scores[w]);
                        if (!pair || w == 1) mma_commit(&sm.empty[kr.stage]);
                        if (t == n - 1) mma_commit(&sm.q_empty);
                    }
                    __syncwarp();
                    if (!pair || w == 1) kr.next();
                };
                scores(0);
                if (n > 1 && alive) scores(1);
                for (int t = 0; t < n && alive; ++t) {
                    const int w = t & 1, mine = t >> 1;
                    if (!pair || w == 0) {
                        if (!wait_warp(&sm.clean[vr.stage], vr.use())) break;
                    }
                    if (!wait_warp(&sm.weights[w], steps0[w] + mine)) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t v = v_op + vr.stage * (C::kTileBytes >> 4);
#pragma unroll
                        for (int kk = 0; kk < kKeys / 16; ++kk)
                            mma_ts(tmem + kSumCol + w * DP, tmem + w * 128 + kk * 8, v + kk * (16 * 128 >> 4), v_shape, mine > 0 || kk > 0);
                        // a step's scores say that the weighted sums of the step before are in; of the last step this does
                        if (t + 2 >= n) mma_commit(&sm.sums[w]);
                    }
                    __syncwarp();
                    const int v_stage = vr.stage;
                    const bool v_done = !pair || w == 1;
                    if (v_done) vr.next();
                    if (t + 2 < n) scores(t + 2);
                    if (v_done && elect_one()) mma_commit(&sm.empty[v_stage]);
                    __syncwarp();
                }
                if (!alive) break;
                steps0[0] += st.of_stream(0);
                steps0[1] += st.of_stream(1);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.part_empty[pn & 1]);
            }
            // the products in flight end before the tensor memory is given back
            __syncwarp();
            if (elect_one()) mma_commit(&sm.drain);
            __syncwarp();
            (void)mbar_wait(&sm.drain, 0);
        } else {
            // value tiles with rows that are not there (or, drafted, that some query rows must not see): 0 times what such
            // rows hold would not be 0 if that is not finite
            const int t64 = threadIdx.x - kAuxWarp * 32;
            uint32_t it0 = 0;
            for (uint32_t pn = 0;; ++pn) {
                if (!wait_warp(&sm.part_full[pn & 1], pn >> 1)) break;
                const Portion p = sm.part[pn & 1];
                if (p.kt1 < 0) break;
                constexpr int CH = DP / 8;
                for (int kt = p.kt0; kt < p.kt1; ++kt) {
                    const uint32_t item = it0 + 2 * (kt - p.kt0) + 1, key_item = item - 1;
                    // the key tile's arrival as well: a phase that is waited for has to be the next one of its barrier
                    if (!wait_warp(&sm.full[key_item % C::kStages], key_item / C::kStages) ||
                        !wait_warp(&sm.full[item % C::kStages], item / C::kStages)) break;
                    if (tile_masked(a, p, kt)) {
                        uint8_t* tile = sm.tiles[item % C::kStages];
                        const int left = keys_left(a, p, kt);
                        const bool drafted = kt >= p.kt_cache;
                        bool odd = false;
#pragma unroll 8
                        for (int x = t64; x < 128 * CH; x += 64) {
                            const int key = (x >> 3) & 127;         // 128 rows of 8 chunks, then the next 64 columns
                            uint4* at = reinterpret_cast<uint4*>(tile + x * 16);
                            if (key >= left) {
                                *at = make_uint4(0, 0, 0, 0);
                            } else if (drafted) {
                                const uint4 v = *at;
                                if (any_nonfinite(v)) {
                                    odd = true;
                                    *at = make_uint4(v.x & ~nonfinite_bf16(v.x), v.y & ~nonfinite_bf16(v.y), v.z & ~nonfinite_bf16(v.z),
                                                     v.w & ~nonfinite_bf16(v.w));
                                }
                            }
                        }
                        if (odd) sm.poison[pn & 1] = 1;
                        async_proxy_fence();
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive(&sm.clean[item % C::kStages]);
                }
                if (!alive) break;
                it0 += 2 * (p.kt1 - p.kt0);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.part_empty[pn & 1]);
            }
        }
    } else {
        more_registers<200>();
        const int w = warp >> 2, r_in = threadIdx.x & 127;          // stream, row of its tile
        const uint32_t lanes = (uint32_t)(warp & 3) * 32 << 16;
        const uint32_t t_scores = tmem + lanes + w * 128, t_sums = tmem + lanes + kSumCol + w * DP;
        const uint64_t c2 = pack2(a.scale_log2, a.scale_log2);
        uint32_t steps = 0, merges = 0, summed = 0;
        for (uint32_t pn = 0;; ++pn) {
            if (!wait_warp(&sm.part_full[pn & 1], pn >> 1)) break;
            const Portion p = sm.part[pn & 1];
            if (p.kt1 < 0) break;
            const Steps st(p, a.split);
            const int tile_rows = a.split.rows / 2;
            const int r_tile = p.rt * a.split.rows + (st.pair ? w * tile_rows : 0);
            const int row = r_tile + r_in;
            const int r_all = r_in < tile_rows ? p.s.nodes * G : 0;                     // the thread has a row if row < r_all
            const bool work = (warp & 3) * 32 < min(tile_rows, p.s.nodes * G - r_tile);     // some thread of the warp has one
            const int mine = st.of_stream(w);
            float m2 = neg_inf(), l = 0.f;                          // maximum in log 2 units, as used; sum
            for (int x = 0; x < mine; ++x) {
                const int kt = p.kt0 + (st.pair ? x : 2 * x + w);
                const bool masked = tile_masked(a, p, kt);
                uint32_t sees[4] = {~0u, ~0u, ~0u, ~0u};            // the keys that the row sees, looked up ahead of the scores
                if (work && masked) {
                    const int left = keys_left(a, p, kt);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (kt < p.kt_cache) {
                            const int n = left - i * 32;
                            sees[i] = n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u);
                        } else {
                            sees[i] = a.split.draft && row < r_all ? draft_sees(a, p.s, row / G, (kt - p.kt_cache) * kKeys + i * 32) : 0u;
                        }
                    }
                }
                if (!wait_warp(&sm.scores[w], steps + x)) break;
                if (work) {
                    tc_fence_after();
                    uint32_t s[4][32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld32(s[i], t_scores + i * 32);
                    tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (__all_sync(0xffffffffu, sees[i] == ~0u)) continue;
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!(sees[i] >> k & 1)) s[i][k] = 0xff800000u;
                        }
                    }
                    float top4[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        top4[i] = __uint_as_float(s[i][0]);
#pragma unroll
                        for (int k = 1; k < 31; k += 2) top4[i] = max3(top4[i], __uint_as_float(s[i][k]), __uint_as_float(s[i][k + 1]));
                        top4[i] = fmaxf(top4[i], __uint_as_float(s[i][31]));
                    }
                    const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * a.scale_log2;
                    const bool grows = top > m2 + kLazy;
                    if (__any_sync(0xffffffffu, grows)) {
                        const float next = grows ? top : m2;
                        const float al = grows ? ex2(m2 - next) : 1.f;      // 0 where nothing was seen yet
                        m2 = next;
                        l *= al;
                        if (x > 0) {            // the sums of step x - 1 are in: its products came before this step's scores
#pragma unroll 1
                            for (int c = 0; c < DP; c += 32) {
                                uint32_t o[32];
                                tmem_ld32(o, t_sums + c);
                                tmem_wait_ld();
#pragma unroll
                                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * al);
                                tmem_st32(t_sums + c, o);
                            }
                        }
                    }
                    const float base = m2 == neg_inf() ? 0.f : m2;
                    const uint64_t nb = pack2(-base, -base);
                    uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const uint64_t y = fma2(pack2(__uint_as_float(s[i][2 * k]), __uint_as_float(s[i][2 * k + 1])), c2, nb);
                            float y0, y1;
                            unpack2(y, y0, y1);
                            y0 = ex2(y0);
                            y1 = ex2(y1);
                            sum2[k & 1] = add2(sum2[k & 1], pack2(y0, y1));
                            // weights are rounded to bf16 for the product with the values; their sum is not
                            pk[k] = pack_bf16(y0, y1);
                        }
                        tmem_st16(t_scores + i * 16, pk);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.weights[w]);
                    float s0, s1;
                    unpack2(add2(sum2[0], sum2[1]), s0, s1);
                    l += s0 + s1;
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.weights[w]);
                }
            }
            if (!alive) break;
            // ---- the portion's result
            if (mine > 0 && !wait_warp(&sm.sums[w], summed++)) break;
            tc_fence_after();
            steps += mine;
            float f0 = 1.f, f1 = 0.f;
            if (!st.pair) {
                if (w == 1) {
                    sm.m[r_in] = m2;
                    sm.l[r_in] = l;
                    mbar_arrive(&sm.merge_full);
                    if (!wait_warp(&sm.merge_done, merges)) break;
                } else {
                    if (!wait_warp(&sm.merge_full, merges)) break;
                    tc_fence_after();
                    const float m1 = sm.m[r_in], l1 = sm.l[r_in], top = fmaxf(m2, m1), base = top == neg_inf() ? 0.f : top;
                    f0 = ex2(m2 - base);
                    f1 = ex2(m1 - base);
                    l = st.of_stream(1) > 0 ? l * f0 + l1 * f1 : l * f0;
                    m2 = top;
                }
                ++merges;
            }
            if (w == 0 || st.pair) {
                const bool both = !st.pair && st.of_stream(1) > 0;
                const bool complete = p.kt0 == 0 && p.kt1 == p.kt_all;
                const int slot = portion_slot(blockIdx.x, p.kt0);
                const int r = (st.pair ? w * 128 : 0) + r_in;
                const float inv = row_scale(l);
                const int64_t at = (int64_t)(p.s.node0 + row / G) * HQ + p.h * G + row % G;
                const bool poison = sm.poison[pn & 1] != 0;
                if (work) {
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        if (c >= D) break;
                        uint32_t o[32];
                        tmem_ld32(o, t_sums + c);
                        tmem_wait_ld();
                        if (both) {
                            uint32_t o1[32];
                            tmem_ld32(o1, t_sums + DP + c);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                o[k] = __float_as_uint(__uint_as_float(o[k]) * f0 + __uint_as_float(o1[k]) * f1);
                        }
                        if (row < r_all) {
                            if (poison) {           // drafted values that were set aside come back to the rows that see them
                                const int j0 = (max(p.kt0, p.kt_cache) - p.kt_cache) * kKeys;
                                const int j1 = min(p.s.nodes, (p.kt1 - p.kt_cache) * kKeys);
#pragma unroll 1
                                for (int j = j0; j < j1; ++j) {
                                    if (!(draft_sees(a, p.s, row / G, j & ~31) >> (j & 31) & 1)) continue;
                                    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                                        a.draft_v + (int64_t)(p.s.node0 + j) * a.dv_node) + p.h * D + c;
#pragma unroll
                                    for (int k = 0; k < 32; ++k) {
                                        if (c + k >= D) break;
                                        const float y = __bfloat162float(v[k]);
                                        if (!finite_f32(y)) o[k] = __float_as_uint(__uint_as_float(o[k]) + y);
                                    }
                                }
                            }
#pragma unroll
                            for (int k = 0; k < 32; k += 8) {
                                if (c + k >= D) break;
                                float y[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(o[k + i]);
                                if (complete) {
                                    *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at * D + c + k) =
                                        make_uint4(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                                                   pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv));
                                } else {            // four columns of all rows next to each other: whole lines a warp
                                    float4* to = reinterpret_cast<float4*>(a.part_o) + ((int64_t)slot * (D / 4) + (c + k) / 4) * kRows + r;
                                    __stcg(to, make_float4(y[0], y[1], y[2], y[3]));
                                    __stcg(to + kRows, make_float4(y[4], y[5], y[6], y[7]));
                                }
                            }
                        }
                    }
                    if (row < r_all) {
                        if (complete) {
                            a.lse[at] = row_lse(m2, l);
                        } else {
                            a.part_ml[(int64_t)slot * 2 * kRows + r] = m2;
                            a.part_ml[((int64_t)slot * 2 + 1) * kRows + r] = l;
                        }
                    }
                }
                if (!st.pair) {
                    tc_fence_before();
                    mbar_arrive(&sm.merge_done);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.part_empty[pn & 1]);
        }
    }
    if (!alive) report(a.status_word, SHARPV_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) tmem_free(tmem, kCols);
}

// Joins the parts of the segments that several CTAs shared: CTA (x, y, z) takes 32 places (lane = place) of the x-th, each
// warp CG groups of four columns.  The parts are added in the order of the CTAs, with a running maximum; 12 loads are
// in flight.  CG = 1 where segments have many parts; with few, one warp takes all its columns at once (CG = 4), and
// all CTAs are resident together (16 ragged trees 40 us a call against 46, a chunk of 509 nodes 91.5 against 99).
template <int CG>
__global__ void __launch_bounds__(256)
attn_tc_join_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kAhead = 12 / CG;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G, tile_rows = a.split.rows / 2;
    const int r = blockIdx.y * 32 + lane, c4 = blockIdx.z * 8 + warp;
    if (c4 * 4 >= D) return;
    cudaGridDependencySynchronize();
    SharedSegment seg;
    if (!find_shared(a, blockIdx.x, seg)) return;
    const int row = seg.rt * a.split.rows + (r >> 7) * tile_rows + (r & 127), c0 = seg.first, c1 = seg.last;
    if ((r & 127) >= tile_rows || row >= seg.rows) return;
    float top = neg_inf(), sum = 0.f;
    float4 acc[CG];
#pragma unroll
    for (int g = 0; g < CG; ++g) acc[g] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = c0; i <= c1; i += kAhead) {
        float4 v[kAhead][CG];
        float m[kAhead], l[kAhead];
#pragma unroll
        for (int x = 0; x < kAhead; ++x) {
            const int c = i + x;
            const int64_t slot = c * 2 + (c == c0);
            m[x] = c <= c1 ? __ldcg(a.part_ml + slot * 2 * kRows + r) : neg_inf();
            l[x] = c <= c1 ? __ldcg(a.part_ml + (slot * 2 + 1) * kRows + r) : 0.f;
#pragma unroll
            for (int g = 0; g < CG; ++g)
                v[x][g] = c <= c1 && (c4 + g * 8) * 4 < D
                              ? __ldcg(reinterpret_cast<const float4*>(a.part_o) + (slot * (D / 4) + c4 + g * 8) * kRows + r)
                              : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float next_top = top;
#pragma unroll
        for (int x = 0; x < kAhead; ++x) next_top = fmaxf(next_top, m[x]);
        const float base = next_top == neg_inf() ? 0.f : next_top, old = ex2(top - base);
        top = next_top;
        sum *= old;
#pragma unroll
        for (int g = 0; g < CG; ++g) acc[g] = make_float4(acc[g].x * old, acc[g].y * old, acc[g].z * old, acc[g].w * old);
#pragma unroll
        for (int x = 0; x < kAhead; ++x) {
            if (i + x > c1) break;
            const float f = ex2(m[x] - base);
            sum = fmaf(f, l[x], sum);
#pragma unroll
            for (int g = 0; g < CG; ++g)
                acc[g] = make_float4(fmaf(f, v[x][g].x, acc[g].x), fmaf(f, v[x][g].y, acc[g].y), fmaf(f, v[x][g].z, acc[g].z),
                                     fmaf(f, v[x][g].w, acc[g].w));
        }
    }
    const float inv = row_scale(sum);
    const int64_t at = (int64_t)(seg.node0 + row / G) * HQ + seg.h * G + row % G;
#pragma unroll
    for (int g = 0; g < CG; ++g)
        if ((c4 + g * 8) * 4 < D)
            *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at * D + (c4 + g * 8) * 4) =
                make_uint2(pack_bf16(acc[g].x * inv, acc[g].y * inv), pack_bf16(acc[g].z * inv, acc[g].w * inv));
    if (c4 == 0) a.lse[at] = row_lse(top, sum);
}

template <int DP>
sharpv_status launch(const AttnArgs& a, cudaStream_t stream) {
    auto kern = attn_tc_kernel<DP>;
    const size_t smem = sizeof(Shared<DP>);
    static_assert(sizeof(Shared<DP>) <= 227 * 1024, "shared memory of one CTA");
    static_assert(kSumCol + 2 * DP <= kCols, "tensor memory");
    AttnMaps maps;
    const sharpv_status ms = encode_attn_maps(a, kKeys, maps);
    if (ms != SHARPV_OK) return ms;
    const int64_t all = a.seqs.total_nodes * a.split.group;
    const unsigned rows = (unsigned)(all <= a.split.rows / 2 ? all : kRows);        // places that any segment can use
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kThreads), smem, stream, a, maps);
    if (e == cudaSuccess) {
        const unsigned x = (unsigned)join_ctas(a), y = (rows + 31) / 32;
        e = many_parts(a) ? launch_dependent(attn_tc_join_kernel<1>, dim3(x, y, (unsigned)(a.head_dim + 31) / 32), dim3(256), 0, stream, a)
                          : launch_dependent(attn_tc_join_kernel<4>, dim3(x, y), dim3(256), 0, stream, a);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

}  // namespace

sharpv_status attn_tc_launch(AttnArgs& a, int sms, cudaStream_t stream) {
    a.ctas = sms < kMaxTcCtas ? sms : kMaxTcCtas;
    return a.head_dim <= 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}

}  // namespace sharpv
