// Attention of few query rows over a K/V cache in 8 bits: every code is read once, and that is what bounds it.
//
// The organisation is that of the bf16 kernel (tree_attention_rows.cu): one CTA per SM, a warp that keeps a ring of TMA tile loads
// in flight, two groups of four warps that take the ring's stages in turn, 16 keys a warp, products on mma.sync.  Tiles are 64 keys as
// well, half the bytes.  What differs is the arithmetic.
//
//   Products are of fp16, because codes of both kinds are halves exactly, at half an instruction a code (e4m3) or one (int8).
//   Query rows are multiplied by a power of two that brings their largest element to [2^14, 2^15): what bf16 holds is then exact in
//   fp16 down to 2^-31 of a row's largest element, and off by 2^-39 of it below.
//   ldmatrix hands a thread four neighbouring codes of a key, so the products take the columns of 16 in the order
//   0 1 4 5 8 9 12 13 | 2 3 6 7 10 11 14 15, and the query rows are laid out in that order.  Of transposed value tiles it
//   hands two keys of two neighbouring columns: even columns are one product, odd ones another.
//   A key's scale multiplies the sum of products first: that is between 2^-33 and 2^32, so neither large queries over small scales
//   nor small codes under large ones pass fp32 before the score itself does (and 0 stays 0).  A value's scale 2^e goes to its
//   weight: the softmax runs over s_j + e_j, with m as its running maximum,
//     out = sum_j 2^(s_j + e_j - m) code_j / l,   l = sum_j 2^(s_j + e_j - m) 2^-e_j,
//   so weights never pass what fp16 holds whatever the scales are.  m is set 8 under the maximum and kept until that has grown by
//   7 more (sums are then rarely rescaled): the largest weight is between 2^8 and 2^15, weights down to 2^-14 are rounded to
//   11 bits, and smaller ones lose 2^-25, 2^-33 of the largest, at most.  That is of the largest with its value's scale on it, whatever
//   the codes there are: a weight p_j itself is off by 2^-33 2^(E - e_j) of the largest p, E being the largest exponent so far.  So a
//   warp takes a tile with e_j < E - 8 (SpanOfScales) by products of bf16, which has fp32's exponents and holds the codes of both
//   kinds: weights have 8 bits there, however far the scales are apart.  Elsewhere p_j is off by 2^-25 of the largest at most.
//
// Drafted tokens are bf16, which may be anything that fp16 does not hold, so they take products of bf16 and their weights are rounded to
// 8 bits (both operands of a product are of one type), in a buffer of their own (there are few of them).
//
// Up to eight query rows have a kernel of their own, below.  Measured (4 KV heads x 128), up to 8 rows and up to 16, us with the join:
// one sequence of 50,432 rows 20.8 / 28 (int8 22.4 / 30.5), the ragged batch of 16 (37,712 rows) 20 / 27, 64 over 2,000 rows each 42 / 58.
// In the first 5.4 us go by until the first tile is there, 8 stream the 52 MB, 2 join the warps and write; the rest joins the CTAs.
// The vote on the scales is in these: 0.2 to 0.9 us of int8 and of up to 16 rows, nothing of e4m3 up to 8.
#include "q8.cuh"
#include "tma.cuh"
#include "tree_attention.cuh"

#include <cuda_bf16.h>

namespace sharpv {
namespace {

constexpr int kKeys = kRowsTileKeys;            // of a tile
// The split with what ending a segment and beginning another costs in these tiles, which take half the time of bf16 ones.  3 against 6:
// the ragged batch of 16 tokens 25.5 against 20.5 us (int8 27.2 / 22.1), of pairs 33.3 / 27.0; where segments are even it decides
// nothing (64 over 2,000 rows each 42.1 / 42.1).
struct CodeSplit : Split {
    static constexpr uint32_t kSwitch = 6;
};

constexpr float kNominal = 8.f, kLazy = 7.f;    // the largest weight is 2^8 when the maximum is set, and stays under 2^15

template <int DP, int ROWS>
struct Cfg {
    static constexpr int kWarps = ROWS == 8 ? 16 : 8;           // that compute, in groups of four
    static constexpr int kGroups = kWarps / 4, kThreads = kWarps * 32 + 32;
    static constexpr int kBox = DP < 128 ? DP : 128;            // bytes of a row in a TMA box
    static constexpr int kTileBytes = kKeys * DP;               // codes of K or V
    static constexpr int kDraftBytes = kKeys * DP * 2;
    static constexpr int kStages = ROWS == 8 ? (DP == 64 ? 12 : 8) : (DP == 64 ? 12 : (DP == 128 ? 6 : 2));
    static_assert(kStages % kGroups == 0, "a stage belongs to one group");
    static constexpr int kQPitch = DP * 2 + 16;                 // bytes; 16 more, so that 8 rows fall on 8 bank groups
    static constexpr int kCols = DP < 128 ? 64 : 128;           // columns that are joined at a time (16 rows)
};

template <int DP, int ROWS>
struct Shared {
    using C = Cfg<DP, ROWS>;
    uint8_t tiles[C::kStages][2][C::kTileBytes];
    // drafted tiles; 8 rows: the second 64 columns of the warps' sums as well, once a portion's tiles are gone through
    uint8_t draft[2][C::kDraftBytes];
    float merge[C::kWarps][ROWS][ROWS == 8 ? 64 : C::kCols + 4];
    float m[C::kWarps][ROWS], l[C::kWarps][ROWS];
    uint8_t q[2][ROWS * C::kQPitch];            // query rows of this portion and the next
    uint8_t qh[ROWS * C::kQPitch];              // this portion's as halves
    float q_unit[ROWS];                         // what a product of them stands for, times the scale of the scores
    Portion part[2];                            // kt1 < 0: there are no more
    uint64_t full[C::kStages], empty[C::kStages], part_full[2], part_empty[2], draft_full, draft_empty;
    int poison[2], dead;
    PlanScratch<C::kThreads> plan;
};

template <int WARPS>
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" :: "n"(WARPS * 32) : "memory"); }

// an 8 x 8 block of 16-bit elements, a row every four lanes, transposed
__device__ __forceinline__ void transpose8(uint32_t& to, uint32_t from) {
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(to) : "r"(from));
}

// The exponents that a warp's values have had so far in a portion, as far as fp16 weights go by them.
struct SpanOfScales {
    static constexpr int kSpan = 8;
    int top = kScaleLeast - 1;
    // Whether values of this tile, whose exponents the lanes that `have` one hold, have weights that fp16 does not hold well.  By a whole
    // warp, with one vote where nothing is new.
    __device__ __forceinline__ bool wide(int exponent, bool have) {
        if (!__any_sync(0xffffffffu, have && (exponent > top || exponent < top - kSpan))) return false;
        top = max(top, __reduce_max_sync(0xffffffffu, have ? exponent : kScaleLeast - 1));
        return __any_sync(0xffffffffu, have && exponent < top - kSpan);
    }
};

// What a tile's products of weights and values take: fp16, or bf16 where the scales are far apart.
struct InHalves {
    __device__ __forceinline__ static uint32_t pack(float lo, float hi) { return pack_f16(lo, hi); }
    template <int CODE> __device__ __forceinline__ static void codes(uint32_t four, uint32_t& lo, uint32_t& hi) { halves_of<CODE>(four, lo, hi); }
    __device__ __forceinline__ static void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) { mma_f16(c, a, b0, b1); }
};
struct InBf16 {
    __device__ __forceinline__ static uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    template <int CODE> __device__ __forceinline__ static void codes(uint32_t four, uint32_t& lo, uint32_t& hi) {
        float x[4];
        floats_of<CODE>(four, x);
        lo = pack_bf16(x[0], x[1]);
        hi = pack_bf16(x[2], x[3]);
    }
    __device__ __forceinline__ static void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) { mma_bf16(c, a, b0, b1); }
};

// byte offset of 16-byte chunk c of a row of codes
template <int DP>
__device__ __forceinline__ uint32_t code_chunk(int row, int c) {
    return DP == 64 ? swizzle64(row, c) : (c >> 3) * (kKeys * 128) + swizzle128(row, c & 7);
}

// The warp that brings portions, query rows and tiles ahead of the warps that compute.
template <int DP, int ROWS>
__device__ __forceinline__ void load_portions(const AttnArgs& a, const AttnMaps& maps, Shared<DP, ROWS>& sm, const PlanStart& plan, int64_t first,
                                              int64_t end) {
    using C = Cfg<DP, ROWS>;
    constexpr int kRows = ROWS, kLanes = 32 / ROWS;     // lanes a query row
    const int lane = threadIdx.x & 31, D = a.head_dim, G = a.split.group;
    bool alive = true;                          // a wait that gave up
    uint32_t ring = 0, drafts = 0, pn = 0;
    Walk walk(plan, first, end);
    Portion p, last;
    for (;; ++pn) {
        const int slot = pn & 1;
        last = p;
        const bool more = walk.next(a.seqs, a.split, p);
        if (pn >= 2) alive = __all_sync(0xffffffffu, mbar_wait(&sm.part_empty[slot], ((pn >> 1) - 1) & 1));
        if (!alive) break;                  // the place may still be read: the others give up on the portion that does not come
        if (more) {
            const int r_base = p.rt * kRows, r_all = p.s.nodes * G;
            const int r = lane / kLanes, row = r_base + r;
            const bool there = row < r_all;
            const int node = there ? row / G : 0, g = there ? row - node * G : 0;
            const char* q = a.q + (int64_t)(p.s.node0 + node) * a.q_node + (int64_t)(p.h * G + g) * D * 2;
            uint8_t* to = sm.q[slot] + r * C::kQPitch;
#pragma unroll
            for (int c = lane % kLanes; c < DP / 8; c += kLanes) cp_async16(to + c * 16, c * 8 < D ? q + c * 16 : q, there && c * 8 < D);
        }
        cp_async_arrive(&sm.part_full[slot]);
        if (lane == 0) {
            if (!more) p.kt1 = -1;
            sm.part[slot] = p;
            mbar_arrive(&sm.part_full[slot]);
        }
        if (!more) break;
        if (lane == 0) {
            for (int kt = p.kt0; kt < p.kt1; ++kt) {
                if (kt >= p.kt_cache && a.split.draft) {
                    if (drafts >= 1) alive = mbar_wait(&sm.draft_empty, (drafts - 1) & 1);
                    // with 8 rows the warps' sums of the portion before are joined in the same place
                    if (ROWS == 8 && pn >= 1 && alive) alive = mbar_wait(&sm.part_empty[slot ^ 1], ((pn - 1) >> 1) & 1);
                    if (!alive) break;
                    mbar_expect(&sm.draft_full, 2 * C::kDraftBytes);
                    const int row = p.s.node0 + (kt - p.kt_cache) * kKeys;
#pragma unroll
                    for (int x = 0; x < DP / 64; ++x) {
                        tma_load(sm.draft[0] + x * kKeys * 128, &maps.draft_k, &sm.draft_full, x * 64, row, p.h);
                        tma_load(sm.draft[1] + x * kKeys * 128, &maps.draft_v, &sm.draft_full, x * 64, row, p.h);
                    }
                    ++drafts;
                    continue;
                }
                const int stage = ring % C::kStages;
                if (ring >= C::kStages) alive = mbar_wait(&sm.empty[stage], (ring / C::kStages - 1) & 1);
                if (!alive) break;
                ++ring;
                if (kt >= p.kt_cache) {                     // the empty tile of rows without keys
                    mbar_arrive(&sm.full[stage]);
                    continue;
                }
                mbar_expect(&sm.full[stage], 2 * C::kTileBytes);
                const int row = (int)p.s.begin + kt * kKeys;
#pragma unroll
                for (int x = 0; x < DP / C::kBox; ++x) {
                    tma_load(sm.tiles[stage][0] + x * kKeys * C::kBox, &maps.cache_k, &sm.full[stage], x * C::kBox, row, p.h);
                    tma_load(sm.tiles[stage][1] + x * kKeys * C::kBox, &maps.cache_v, &sm.full[stage], x * C::kBox, row, p.h);
                }
            }
        }
        alive = __all_sync(0xffffffffu, alive);
        if (!alive) break;
    }
    if (lane == 0) {
        if (!alive) report(a.status_word, SHARPV_ERR_TIMEOUT);
        note_shared(a, alive && pn > 0, last, end, plan);
        // copies in flight land before the CTA ends, also where the warps that wanted them gave up
        for (int i = 0; i < C::kStages && (uint32_t)i < ring; ++i) {
            const uint32_t at = ring - 1 - i;
            (void)mbar_wait(&sm.full[at % C::kStages], (at / C::kStages) & 1);
        }
        if (drafts > 0) (void)mbar_wait(&sm.draft_full, (drafts - 1) & 1);
    }
    cp_async_wait<0>();
}

// Query rows as halves in the order of the products' columns, each by one warp.
template <int DP, int ROWS>
__device__ __forceinline__ void halve_queries(Shared<DP, ROWS>& sm, int at_part, float scale_log2) {
    using C = Cfg<DP, ROWS>;
    const int lane = threadIdx.x & 31;
    for (int r = threadIdx.x >> 5; r < ROWS; r += C::kWarps) {
        const uint8_t* from = sm.q[at_part] + r * C::kQPitch;
        constexpr int N = (DP / 4 + 31) / 32;               // groups of four columns a lane
        float x[N][4], top = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = n * 32 + lane;
            const uint2 w = c < DP / 4 ? *reinterpret_cast<const uint2*>(from + c * 8) : make_uint2(0, 0);
            x[n][0] = __uint_as_float(w.x << 16);
            x[n][1] = __uint_as_float(w.x & 0xffff0000u);
            x[n][2] = __uint_as_float(w.y << 16);
            x[n][3] = __uint_as_float(w.y & 0xffff0000u);
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[n][e]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int up = min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 126);
        const float f = power_of_two(up);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = n * 32 + lane;
            if (c < DP / 4) {
                uint8_t* to = sm.qh + r * C::kQPitch + (c >> 2) * 32 + (c & 3) * 4;
                *reinterpret_cast<uint32_t*>(to) = pack_f16(x[n][0] * f, x[n][1] * f);
                *reinterpret_cast<uint32_t*>(to + 16) = pack_f16(x[n][2] * f, x[n][3] * f);
            }
        }
        if (lane == 0) sm.q_unit[r] = power_of_two(-up) * scale_log2;
    }
}

// Two columns of a joined row, written as the portion's (a partial result, or the row itself) with what was set aside of drafted
// values given back if the row sees it.
template <int ROWS>
__device__ __forceinline__ void write_columns(const AttnArgs& a, const Portion& p, int r, int c, float2 acc, float top, float sum, bool poison) {
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G, row = p.rt * ROWS + r;
    if (poison) {
        const int j0 = (max(p.kt0, p.kt_cache) - p.kt_cache) * kKeys, j1 = min(p.s.nodes, (p.kt1 - p.kt_cache) * kKeys);
        for (int j = j0; j < j1; ++j) {
            if (!(draft_sees(a, p.s, row / G, j & ~31) >> (j & 31) & 1)) continue;
            const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                a.draft_v + (int64_t)(p.s.node0 + j) * a.dv_node) + p.h * D + c;
            const float v0 = __bfloat162float(v[0]), v1 = __bfloat162float(v[1]);
            if (!finite_f32(v0)) acc.x += v0;
            if (!finite_f32(v1)) acc.y += v1;
        }
    }
    if (p.kt0 == 0 && p.kt1 == p.kt_all) {
        const int64_t to = (int64_t)(p.s.node0 + row / G) * HQ + p.h * G + row % G;
        const float inv = row_scale(sum);
        *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(a.out) + to * D + c) = pack_bf16(acc.x * inv, acc.y * inv);
        if (c == 0) a.lse[to] = row_lse(top, sum);
    } else {
        const int64_t slot = portion_slot(blockIdx.x, p.kt0);
        *reinterpret_cast<float2*>(a.part_o + (slot * ROWS + r) * D + c) = acc;
        if (c == 0) {
            a.part_ml[slot * 2 * ROWS + r] = top;
            a.part_ml[(slot * 2 + 1) * ROWS + r] = sum;
        }
    }
}

// What warp `lane` (of up to 16) counts for in row r's joined sums, and the row's maximum and sum: by a whole warp.
template <int DP, int ROWS>
__device__ __forceinline__ float warp_share(const Shared<DP, ROWS>& sm, int r, float& top, float& sum) {
    constexpr int kWarps = Cfg<DP, ROWS>::kWarps;
    const int w = threadIdx.x & 15;
    const float m = w < kWarps ? sm.m[w][r] : neg_inf();
    top = m;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float f = ex2(m - (top == neg_inf() ? 0.f : top));
    sum = w < kWarps ? f * sm.l[w][r] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return f;
}

// 64 columns of a row from c0 on: by a whole warp, two columns a lane.  `at`: where warp w's sums of the lane's columns are.
template <int DP, int ROWS, class At>
__device__ __forceinline__ void join_row(const AttnArgs& a, const Shared<DP, ROWS>& sm, const Portion& p, int r, int c0, bool poison, At at) {
    constexpr int kWarps = Cfg<DP, ROWS>::kWarps;
    const int c = c0 + (threadIdx.x & 31) * 2;
    if (p.rt * ROWS + r >= p.s.nodes * a.split.group) return;
    float top, sum;
    const float share = warp_share<DP, ROWS>(sm, r, top, sum);
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const float f = __shfl_sync(0xffffffffu, share, w);
        const float2 v = *reinterpret_cast<const float2*>(at(w));
        acc.x = fmaf(f, v.x, acc.x);
        acc.y = fmaf(f, v.y, acc.y);
    }
    if (c < a.head_dim) write_columns<ROWS>(a, p, r, c, acc, top, sum, poison);
}

template <int CODE, int DP>
__global__ void __launch_bounds__(Cfg<DP, 16>::kThreads, 1)
attn_rows_q8_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnMaps maps) {
    using C = Cfg<DP, 16>;
    constexpr int kWarps = C::kWarps, kThreads = C::kThreads, kRows = 16;
    constexpr bool kQInRegs = DP <= 128;
    // where a tile's scales are looked at decides how the compiler orders the rest: 256 columns, tree of 64 over 6,272 rows, in front of the
    // products with the keys or behind the weights: e4m3 108 us against 118, int8 132 against 125; 128 columns 29.2 against 28.2
    constexpr bool kScalesFirst = DP > 128 && CODE == SHARPV_E4M3;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP, 16>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 4);
        }
        mbar_init(&sm.draft_full, 1);
        mbar_init(&sm.draft_empty, 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.part_full[i], 33);        // 32 lanes' query rows have landed, and the portion is written
            mbar_init(&sm.part_empty[i], kWarps);
        }
        mbar_fence_init();
        sm.poison[0] = sm.poison[1] = sm.dead = 0;
    }
    if (warp == kWarps && lane < 4) tma_prefetch(&maps.cache_k + lane);
    __syncthreads();
    cudaGridDependencySynchronize();
    // the warps that compute are told their portions: where one warp can, the plan is the loading warp's alone
    int64_t first, end;
    PlanStart plan;
    if (!a.warp_plans) plan = plan_cta<kThreads>(a.seqs, CodeSplit{a.split}, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    else if (warp == kWarps) (void)plan_warp(a.seqs, CodeSplit{a.split}, blockIdx.x, a.ctas, plan, first, end, a.status_word, true);
    bool alive = true;                          // a wait that gave up: nothing is waited for any more, the result is void
    uint32_t ring = 0, drafts = 0, pn = 0;      // tiles in the ring, drafted tiles and portions of this CTA so far
    const int G = a.split.group;

    if (warp == kWarps) {                       // portions, query rows and tiles ahead of the warps that compute
        load_portions<DP, 16>(a, maps, sm, plan, first, end);
        return;
    }

    const int group = warp >> 2, sub = warp & 3;        // stages of this parity, 16 keys from sub * 16 on
    const int qr = lane >> 2, qc = (lane & 3) * 2;      // fragment row (and row + 8), column (and column + 1)
    for (;; ++pn) {
        const int at_part = pn & 1;
        if (alive && !mbar_wait(&sm.part_full[at_part], (pn >> 1) & 1)) {
            alive = false;
            report(a.status_word, SHARPV_ERR_TIMEOUT);
        }
        if (!alive) sm.dead = 1;
        consumer_sync<kWarps>();                        // all eight warps go on or none does
        const Portion p = sm.part[at_part];
        if (p.kt1 < 0 || sm.dead) break;
        const int r_base = p.rt * kRows, r_all = p.s.nodes * G;
        // lanes 0 to 15: what stands at the scales of the warp's keys; 16 to 31: of its values.  Looked up a tile ahead.
        const uint8_t* scales = (lane < 16 ? a.k_scales : a.v_scales) + p.h * a.scale_head;
        auto scale_of = [&](int kt) {
            const int key = kt * kKeys + sub * 16 + (lane & 15);
            return kt < p.kt_cache && key < p.s.len ? (uint32_t)__ldg(scales + ((p.s.begin + key) >> a.scale_shift)) : 127u;
        };
        uint32_t next_scale = scale_of(p.kt0 + (int)((group ^ ring) & 1));
        halve_queries<DP, 16>(sm, at_part, a.scale_log2);
        consumer_sync<kWarps>();
        const uint32_t q_off = (lane & 15) * C::kQPitch + (lane >> 4) * 16;
        const uint32_t qh_base = smem_u32(sm.qh) + q_off, q_base = smem_u32(sm.q[at_part]) + q_off;
        const float unit[2] = {sm.q_unit[qr], sm.q_unit[qr + 8]};
        uint32_t qf[kQInRegs ? DP / 16 : 1][4];
        if constexpr (kQInRegs) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) ldmatrix4(qf[ks], qh_base + ks * 32);
        }
        // of 16 columns from 16 j on: o[j][0] the even ones, o[j][1] the odd ones; a thread has columns 4 (lane & 3) .. + 3
        float o[DP / 16][2][4];
        float m[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};        // of rows qr and qr + 8
        SpanOfScales span;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][0][i] = o[j][1][i] = 0.f;
        bool poison = false;                    // a drafted value that is not finite was set aside

        // scores (with the values' exponents on top) to weights, relative to the running maximum
        auto weigh = [&](float (&s)[2][4]) {
            float top[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float x = fmaxf(fmaxf(s[0][half * 2], s[0][half * 2 + 1]), fmaxf(s[1][half * 2], s[1][half * 2 + 1]));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                top[half] = x - kNominal;
            }
            const bool grows0 = top[0] > m[0] + kLazy, grows1 = top[1] > m[1] + kLazy;
            if (__any_sync(0xffffffffu, grows0 || grows1)) {
                const float a0 = grows0 ? ex2(m[0] - top[0]) : 1.f;         // 0 where nothing was seen yet
                const float a1 = grows1 ? ex2(m[1] - top[1]) : 1.f;
                m[0] = grows0 ? top[0] : m[0];
                m[1] = grows1 ? top[1] : m[1];
                l[0] *= a0;
                l[1] *= a1;
#pragma unroll
                for (int j = 0; j < DP / 16; ++j)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        o[j][y][0] *= a0;
                        o[j][y][1] *= a0;
                        o[j][y][2] *= a1;
                        o[j][y][3] *= a1;
                    }
            }
            const float b0 = m[0] == neg_inf() ? 0.f : m[0], b1 = m[1] == neg_inf() ? 0.f : m[1];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] = ex2(s[n][i] - (i < 2 ? b0 : b1));
        };

        for (int kt = p.kt0; kt < p.kt1; ++kt) {
            const bool drafted = kt >= p.kt_cache && a.split.draft;
            const uint32_t at = drafted ? drafts++ : ring++;
            // a phase that is waited for has to be the next one of its barrier: a stage (their number is even) always has the
            // same group, and so has the buffer of drafted tiles
            if ((drafted ? 0 : (int)(at & 1)) != group) continue;
            uint64_t* full = drafted ? &sm.draft_full : &sm.full[at % C::kStages];
            uint64_t* empty = drafted ? &sm.draft_empty : &sm.empty[at % C::kStages];
            const uint32_t scale_code = next_scale;
            next_scale = scale_of(kt + 2);
            const int left = drafted ? p.s.nodes - (kt - p.kt_cache) * kKeys : (kt < p.kt_cache ? p.s.len - kt * kKeys : 0);     // keys of the tile that are there
            bool wide = false;
            auto look_at_scales = [&] { wide = span.wide(scale_exponent(scale_code), lane >= 16 && sub * 16 + (lane & 15) < left); };
            if (kScalesFirst && !drafted) look_at_scales();
            if (alive && !mbar_wait(full, (drafted ? at : at / C::kStages) & 1)) {
                alive = false;
                report(a.status_word, SHARPV_ERR_TIMEOUT);
            }
            float s[2][4] = {};
            const int krow = sub * 16 + (lane >> 4) * 8 + (lane & 7), vrow = sub * 16 + (lane & 15);
            if (!drafted) {
                const int stage = at % C::kStages;
                const uint32_t ks_base = smem_u32(sm.tiles[stage][0]), vs_base = smem_u32(sm.tiles[stage][1]);
#pragma unroll
                for (int ks = 0; ks < DP / 16; ks += 2) {
                    uint32_t k4[4];
                    ldmatrix4(k4, ks_base + code_chunk<DP>(krow, ks + ((lane >> 3) & 1)));
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        uint32_t q4[4], b0, b1;
                        if constexpr (kQInRegs) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) q4[i] = qf[ks + y][i];
                        } else {
                            ldmatrix4(q4, qh_base + (ks + y) * 32);
                        }
                        halves_of<CODE>(k4[y], b0, b1);
                        mma_f16(s[0], q4, b0, b1);
                        halves_of<CODE>(k4[2 + y], b0, b1);
                        mma_f16(s[1], q4, b0, b1);
                    }
                }
                const int exponent = scale_exponent(scale_code);
                int ve[2][2];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float kx = power_of_two(__shfl_sync(0xffffffffu, exponent, n * 8 + qc + i));
                        ve[n][i] = __shfl_sync(0xffffffffu, exponent, 16 + n * 8 + qc + i);
                        const bool sees = sub * 16 + n * 8 + qc + i < left;
                        s[n][i] = sees ? fmaf(s[n][i] * kx, unit[0], (float)ve[n][i]) : neg_inf();
                        s[n][2 + i] = sees ? fmaf(s[n][2 + i] * kx, unit[1], (float)ve[n][i]) : neg_inf();
                    }
                weigh(s);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float d0 = power_of_two(-ve[n][0]), d1 = power_of_two(-ve[n][1]);
                    l[0] += fmaf(s[n][0], d0, s[n][1] * d1);
                    l[1] += fmaf(s[n][2], d0, s[n][3] * d1);
                }
                auto values = [&](auto in) {
                    using In = decltype(in);
                    // weights are rounded for the product with the values; their sum is not
                    const uint32_t pf[4] = {In::pack(s[0][0], s[0][1]), In::pack(s[0][2], s[0][3]), In::pack(s[1][0], s[1][1]), In::pack(s[1][2], s[1][3])};
#pragma unroll
                    for (int j = 0; j < DP / 16; j += 2) {
                        uint32_t v4[4];
                        ldmatrix4_trans(v4, vs_base + code_chunk<DP>(vrow, j + (lane >> 4)));
                        if (left < kKeys) {
                            // rows that are not there may hold anything: 0 times them would not be 0
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int key = sub * 16 + (i & 1) * 8 + qc;
                                if (key >= left) v4[i] = 0u;
                                else if (key + 1 >= left) v4[i] &= 0xffffu;
                            }
                        }
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            uint32_t even0, odd0, even1, odd1;
                            In::template codes<CODE>(__byte_perm(v4[y * 2], 0u, 0x3120), even0, odd0);
                            In::template codes<CODE>(__byte_perm(v4[y * 2 + 1], 0u, 0x3120), even1, odd1);
                            In::mma(o[j + y][0], pf, even0, even1);
                            In::mma(o[j + y][1], pf, odd0, odd1);
                        }
                    }
                };
                if constexpr (!kScalesFirst) look_at_scales();
                if (!wide) values(InHalves{});
                else values(InBf16{});
            } else {
                const uint32_t ks_base = smem_u32(sm.draft[0]), vs_base = smem_u32(sm.draft[1]);
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) {
                    uint32_t k4[4], q4[4];
                    ldmatrix4(k4, ks_base + (ks >> 2) * (kKeys * 128) + swizzle128(krow, (ks & 3) * 2 + ((lane >> 3) & 1)));
                    ldmatrix4(q4, q_base + ks * 32);
                    mma_bf16(s[0], q4, k4[0], k4[1]);
                    mma_bf16(s[1], q4, k4[2], k4[3]);
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int row = r_base + qr + half * 8;
                    const int key0 = (kt - p.kt_cache) * kKeys + (sub >> 1) * 32;
                    const uint32_t sees = row < r_all ? draft_sees(a, p.s, row / G, key0) >> ((sub & 1) * 16) : 0u;
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            s[n][half * 2 + i] = sees >> (n * 8 + qc + i) & 1 ? s[n][half * 2 + i] * a.scale_log2 : neg_inf();
                }
                weigh(s);
                uint32_t pf[4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    l[0] += s[n][0] + s[n][1];
                    l[1] += s[n][2] + s[n][3];
                    pf[n * 2] = pack_bf16(s[n][0], s[n][1]);
                    pf[n * 2 + 1] = pack_bf16(s[n][2], s[n][3]);
                }
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) {
                    uint32_t v4[4];
                    ldmatrix4_trans(v4, vs_base + (j >> 2) * (kKeys * 128) + swizzle128(vrow, (j & 3) * 2 + (lane >> 4)));
                    // rows that are not there may hold anything, and so may drafted rows that some query rows do not see
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = sub * 16 + (i & 1) * 8 + qc;
                        if (key >= left) v4[i] = 0u;
                        else if (key + 1 >= left) v4[i] &= 0xffffu;
                        const uint32_t off = nonfinite_bf16(v4[i]);
                        v4[i] &= ~off;
                        poison |= off != 0;
                    }
                    // columns in the order of the sums: even ones, then odd ones
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int from = ((2 * qr + y) & 7) * 4 + (lane & 3);
                        uint32_t b[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t low = __shfl_sync(0xffffffffu, v4[i], from), high = __shfl_sync(0xffffffffu, v4[2 + i], from);
                            b[i] = qr < 4 ? low : high;
                        }
                        mma_bf16(o[j][y], pf, b[0], b[1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty);
        }

        // ---- the eight warps' results are joined, up to 128 columns at a time
        if (poison) sm.poison[0] = 1;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
            if ((lane & 3) == 0) { sm.m[warp][qr + half * 8] = m[half]; sm.l[warp][qr + half * 8] = l[half]; }
        }
#pragma unroll
        for (int c0 = 0; c0 < DP; c0 += C::kCols) {
#pragma unroll
            for (int j = c0 / 16; j < (c0 + C::kCols) / 16; ++j) {
                const int col = j * 16 - c0 + (lane & 3) * 4;
                *reinterpret_cast<float4*>(&sm.merge[warp][qr][col]) = make_float4(o[j][0][0], o[j][1][0], o[j][0][1], o[j][1][1]);
                if (r_base + 8 < r_all)         // rows 8 to 15 hold something
                    *reinterpret_cast<float4*>(&sm.merge[warp][qr + 8][col]) = make_float4(o[j][0][2], o[j][1][2], o[j][0][3], o[j][1][3]);
            }
            consumer_sync<kWarps>();
            for (int x = warp; x < 16 * (C::kCols / 64); x += kWarps) {
                const int r = x / (C::kCols / 64), c = x % (C::kCols / 64) * 64;
                join_row<DP, 16>(a, sm, p, r, c0 + c, sm.poison[0], [&](int w) { return &sm.merge[w][r][c + lane * 2]; });
            }
            consumer_sync<kWarps>();
        }
        if (threadIdx.x == 0) sm.poison[0] = 0;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.part_empty[at_part]);
    }
}

// Up to eight query rows a tile: keys, and columns of the values, are the rows of the products, query rows their eight columns, so
// nothing is computed for rows that are not there, and sums take half the registers.  That leaves room for four
// groups of warps, four warps a scheduler instead of two: the chain from codes to weights is what a warp waits for.  The next
// portion's query rows are made halves, and its first scales looked up, while one is joined.
// A thread has the scores of keys lane / 4 and 8 further for query rows 2 (lane % 4) and the next.
template <int CODE, int DP>
__global__ void __launch_bounds__(Cfg<DP, 8>::kThreads, 1)
attn_rows8_q8_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnMaps maps) {
    using C = Cfg<DP, 8>;
    constexpr int kWarps = C::kWarps, kThreads = C::kThreads;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP, 8>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 4);
        }
        mbar_init(&sm.draft_full, 1);
        mbar_init(&sm.draft_empty, 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.part_full[i], 33);        // 32 lanes' query rows have landed, and the portion is written
            mbar_init(&sm.part_empty[i], kWarps);
        }
        mbar_fence_init();
        sm.poison[0] = sm.poison[1] = sm.dead = 0;
    }
    if (warp == kWarps && lane < 4) tma_prefetch(&maps.cache_k + lane);
    __syncthreads();
    cudaGridDependencySynchronize();
    // the warps that compute are told their portions: where one warp can, the plan is the loading warp's alone
    int64_t first, end;
    PlanStart plan;
    if (!a.warp_plans) plan = plan_cta<kThreads>(a.seqs, CodeSplit{a.split}, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    else if (warp == kWarps) (void)plan_warp(a.seqs, CodeSplit{a.split}, blockIdx.x, a.ctas, plan, first, end, a.status_word, true);
    if (warp == kWarps) {
        load_portions<DP, 8>(a, maps, sm, plan, first, end);
        return;
    }
    bool alive = true;                                  // a wait that gave up: nothing is waited for any more, the result is void
    uint32_t ring = 0, drafts = 0;                      // tiles in the ring and drafted tiles so far
    const int G = a.split.group;
    const int group = warp >> 2, sub = warp & 3;        // stages of this remainder, 16 keys from sub * 16 on
    const int kr = lane >> 2, qc = (lane & 3) * 2;      // fragment row (and row + 8), column (and column + 1)
    // A portion's tiles in the ring (its cached ones, or one for rows without any key), which of them is the group's first, and lanes
    // 0 to 15: what stands at the scales of the warp's keys in it, 16 to 31: of its values.  Scales are looked up a tile ahead.
    constexpr int kTurn = C::kGroups * kKeys;           // rows from one of a group's tiles to its next: whole blocks
    static_assert(kTurn % kMaxBlockTokens == 0, "scales of a group's tiles are a whole number of blocks apart");
    struct Tiles { int n, first; };
    auto tiles_of = [&](const Portion& p) {
        return Tiles{a.split.draft ? max(min(p.kt1, p.kt_cache) - p.kt0, 0) : p.kt1 - p.kt0, (int)((group - ring) & (C::kGroups - 1))};
    };
    const uint8_t* scale_at = nullptr;                  // of the lane's key in the tile that is looked up
    int scale_key = 0;                                  // that key
    auto look_up = [&](int len) {
        const uint32_t code = scale_key < len ? (uint32_t)__ldg(scale_at) : 127u;
        scale_key += kTurn;
        scale_at += kTurn >> a.scale_shift;
        return code;
    };
    auto first_scale = [&](const Portion& p) {
        scale_key = (p.kt0 + tiles_of(p).first) * kKeys + sub * 16 + (lane & 15);
        scale_at = (lane < 16 ? a.k_scales : a.v_scales) + p.h * a.scale_head + ((p.s.begin + scale_key) >> a.scale_shift);
        return look_up(p.kt0 < p.kt_cache ? p.s.len : 0);
    };
    auto await_portion = [&](uint32_t n) {
        if (alive && !mbar_wait(&sm.part_full[n & 1], (n >> 1) & 1)) {
            alive = false;
            report(a.status_word, SHARPV_ERR_TIMEOUT);
        }
        if (!alive) sm.dead = 1;
    };
    await_portion(0);
    consumer_sync<kWarps>();                            // all warps go on or none does
    if (sm.dead || sm.part[0].kt1 < 0) return;
    uint32_t next_scale = first_scale(sm.part[0]);
    halve_queries<DP, 8>(sm, 0, a.scale_log2);
    consumer_sync<kWarps>();
    for (uint32_t pn = 0;; ++pn) {
        const int at_part = pn & 1;
        const Portion p = sm.part[at_part];
        const int r_base = p.rt * 8, r_all = p.s.nodes * G;
        const uint32_t q_off = (lane & 7) * C::kQPitch + (lane >> 3) * 16;
        const uint32_t q_base = smem_u32(sm.q[at_part]) + q_off;
        const float unit[2] = {sm.q_unit[qc], sm.q_unit[qc + 1]};
        uint32_t qf[DP / 32][4];                        // of 32 columns
#pragma unroll
        for (int ks = 0; ks < DP / 32; ++ks) ldmatrix4(qf[ks], smem_u32(sm.qh) + q_off + ks * 64);
        // of 16 columns from 16 j on a thread has the columns 2 kr and 2 kr + 1 of its two query rows
        float o[DP / 16][4];
        float m[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};
        SpanOfScales span;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        bool poison = false;                            // a drafted value that is not finite was set aside

        // scores (with the values' exponents on top) to weights, relative to the running maximum
        auto weigh = [&](float (&s)[4]) {
            float top[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float x = fmaxf(s[y], s[2 + y]);
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                top[y] = x - kNominal;
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const bool grows = top[y] > m[y] + kLazy;
                    const float f = grows ? ex2(m[y] - top[y]) : 1.f;       // 0 where nothing was seen yet
                    m[y] = grows ? top[y] : m[y];
                    l[y] *= f;
#pragma unroll
                    for (int j = 0; j < DP / 16; ++j) {
                        o[j][y] *= f;
                        o[j][2 + y] *= f;
                    }
                }
            }
            const float b0 = m[0] == neg_inf() ? 0.f : m[0], b1 = m[1] == neg_inf() ? 0.f : m[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = ex2(s[i] - (i & 1 ? b1 : b0));
        };

        const int vrow = sub * 16 + (lane & 15);
        auto await_tile = [&](uint64_t* full, uint32_t phase) {
            if (alive && !mbar_wait(full, phase & 1)) {
                alive = false;
                report(a.status_word, SHARPV_ERR_TIMEOUT);
            }
        };
        auto give_back = [&](uint64_t* empty) {
            __syncwarp();
            if (lane == 0) mbar_arrive(empty);
        };
        // a phase that is waited for has to be the next one of its barrier: a stage always has the same group, and so has the
        // buffer of drafted tiles
        const Tiles tiles = tiles_of(p);
        int left = (p.kt0 < p.kt_cache ? p.s.len : 0) - (p.kt0 + tiles.first) * kKeys;        // keys of the tile that are there
        for (int i = tiles.first; i < tiles.n; i += C::kGroups, left -= kTurn) {
            const uint32_t at = ring + i;
            const int stage = at % C::kStages;
            const int exponent = scale_exponent(next_scale);
            next_scale = look_up(p.s.len);
            const bool wide = span.wide(exponent, lane >= 16 && sub * 16 + (lane & 15) < left);
            await_tile(&sm.full[stage], at / C::kStages);
            float s[4] = {};
            const uint32_t ks_base = smem_u32(sm.tiles[stage][0]), vs_base = smem_u32(sm.tiles[stage][1]);
            float s1[4] = {};               // odd blocks of 16 columns: two chains of products
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks += 2) {
                uint32_t k4[4], k0[4], k1[4];
                ldmatrix4(k4, ks_base + code_chunk<DP>(vrow, ks + (lane >> 4)));
                halves_of<CODE>(k4[0], k0[0], k0[2]);
                halves_of<CODE>(k4[1], k0[1], k0[3]);
                halves_of<CODE>(k4[2], k1[0], k1[2]);
                halves_of<CODE>(k4[3], k1[1], k1[3]);
                mma_f16(s, k0, qf[ks / 2][0], qf[ks / 2][1]);
                mma_f16(s1, k1, qf[ks / 2][2], qf[ks / 2][3]);
            }
            int ve[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float kx = power_of_two(__shfl_sync(0xffffffffu, exponent, n * 8 + kr));
                ve[n] = __shfl_sync(0xffffffffu, exponent, 16 + n * 8 + kr);
                const bool sees = sub * 16 + n * 8 + kr < left;
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    s[n * 2 + y] = sees ? fmaf((s[n * 2 + y] + s1[n * 2 + y]) * kx, unit[y], (float)ve[n]) : neg_inf();
            }
            weigh(s);
            const float d0 = power_of_two(-ve[0]), d1 = power_of_two(-ve[1]);
            l[0] += fmaf(s[0], d0, s[2] * d1);
            l[1] += fmaf(s[1], d0, s[3] * d1);
            auto values = [&](auto in) {
                using In = decltype(in);
                // weights are rounded for the product with the values; their sum is not
                uint32_t pf[2];
                transpose8(pf[0], In::pack(s[0], s[1]));
                transpose8(pf[1], In::pack(s[2], s[3]));
#pragma unroll
                for (int j = 0; j < DP / 16; j += 2) {
                    uint32_t v4[4];
                    ldmatrix4_trans(v4, vs_base + code_chunk<DP>(vrow, j + (lane >> 4)));
                    if (left < kKeys) {
                        // rows that are not there may hold anything: 0 times them would not be 0
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = sub * 16 + (i & 1) * 8 + qc;
                            if (key >= left) v4[i] = 0u;
                            else if (key + 1 >= left) v4[i] &= 0xffffu;
                        }
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        uint32_t v[4];          // even columns, odd columns of keys 0 to 7, then of keys 8 to 15
                        In::template codes<CODE>(__byte_perm(v4[y * 2], 0u, 0x3120), v[0], v[1]);
                        In::template codes<CODE>(__byte_perm(v4[y * 2 + 1], 0u, 0x3120), v[2], v[3]);
                        In::mma(o[j + y], v, pf[0], pf[1]);
                    }
                }
            };
            if (!wide) values(InHalves{});
            else values(InBf16{});
            give_back(&sm.empty[stage]);
        }
        ring += tiles.n;
        for (int kt = max(p.kt0, p.kt_cache); a.split.draft && kt < p.kt1; ++kt, ++drafts) {
            if (group != 0) continue;
            await_tile(&sm.draft_full, drafts);
            float s[4] = {};
            const uint32_t ks_base = smem_u32(sm.draft[0]), vs_base = smem_u32(sm.draft[1]);
            const int left = p.s.nodes - (kt - p.kt_cache) * kKeys;
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks += 2) {
                uint32_t q4[4];
                ldmatrix4(q4, q_base + ks * 32);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    uint32_t k4[4];
                    ldmatrix4(k4, ks_base + (ks >> 2) * (kKeys * 128) + swizzle128(vrow, ((ks + y) & 3) * 2 + (lane >> 4)));
                    mma_bf16(s, k4, q4[y * 2], q4[y * 2 + 1]);
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int row = r_base + qc + y;
                const int key0 = (kt - p.kt_cache) * kKeys + (sub >> 1) * 32;
                const uint32_t sees = row < r_all ? draft_sees(a, p.s, row / G, key0) >> ((sub & 1) * 16) : 0u;
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    s[n * 2 + y] = sees >> (n * 8 + kr) & 1 ? s[n * 2 + y] * a.scale_log2 : neg_inf();
            }
            weigh(s);
            l[0] += s[0] + s[2];
            l[1] += s[1] + s[3];
            uint32_t pf[2];
            transpose8(pf[0], pack_bf16(s[0], s[1]));
            transpose8(pf[1], pack_bf16(s[2], s[3]));
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
                uint32_t v4[4], v[4];
                ldmatrix4_trans(v4, vs_base + (j >> 2) * (kKeys * 128) + swizzle128(vrow, (j & 3) * 2 + (lane >> 4)));
                // rows that are not there may hold anything, and so may drafted rows that some query rows do not see
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = sub * 16 + (i & 1) * 8 + qc;
                    if (key >= left) v4[i] = 0u;
                    else if (key + 1 >= left) v4[i] &= 0xffffu;
                    const uint32_t off = nonfinite_bf16(v4[i]);
                    v4[i] &= ~off;
                    poison |= off != 0;
                }
                // columns in the order of the sums: even ones, then odd ones
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int from = ((2 * kr + y) & 7) * 4 + (lane & 3);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t low = __shfl_sync(0xffffffffu, v4[i], from), high = __shfl_sync(0xffffffffu, v4[2 + i], from);
                        v[i * 2 + y] = kr < 4 ? low : high;
                    }
                }
                mma_bf16(o[j], v, pf[0], pf[1]);
            }
            give_back(&sm.draft_empty);
        }

        // ---- the warps' results are joined; meanwhile the next portion's query rows and first scales
        if (poison) sm.poison[at_part] = 1;
        await_portion(pn + 1);
        const bool more = sm.part[at_part ^ 1].kt1 >= 0 && alive;
        if (more) next_scale = first_scale(sm.part[at_part ^ 1]);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], w);
        consumer_sync<kWarps>();                        // the portion before is written, and this one's tiles are gone through
        if (sm.dead) break;
        // pairs of columns of every second row lie 64 bytes further round, so that four lanes with the same columns do not meet
        float (*const late)[8][64] = reinterpret_cast<float (*)[8][64]>(&sm.draft[0][0]);
        static_assert(DP == 64 || sizeof(sm.merge) <= sizeof(sm.draft), "");
        auto pair_at = [](int row, int pair) { return (pair ^ (row >> 1 & 3) << 3) * 2; };
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            if (kr == 0) { sm.m[warp][qc + y] = m[y]; sm.l[warp][qc + y] = l[y]; }
#pragma unroll
            for (int j = 0; j < DP / 16; ++j)
                *reinterpret_cast<float2*>(&(j < 4 ? sm.merge : late)[warp][qc + y][pair_at(qc + y, (j & 3) * 8 + kr)]) = make_float2(o[j][y], o[j][2 + y]);
        }
        if (more) halve_queries<DP, 8>(sm, at_part ^ 1, a.scale_log2);
        if (threadIdx.x == 0) sm.poison[at_part ^ 1] = 0;
        consumer_sync<kWarps>();
        for (int x = warp; x < 8 * (DP / 64); x += kWarps) {
            const int r = x / (DP / 64), c = x % (DP / 64);
            join_row<DP, 8>(a, sm, p, r, c * 64, sm.poison[at_part] != 0, [&](int w) { return &(c == 0 ? sm.merge : late)[w][r][pair_at(r, lane)]; });
        }
        async_proxy_fence();                            // drafted tiles come by TMA where `late` was
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.part_empty[at_part]);
        if (!more) break;
    }
}

template <int ROWS, int DP>
sharpv_status launch(void (*kern)(AttnArgs, AttnMaps), const AttnArgs& a, cudaStream_t stream) {
    using C = Cfg<DP, ROWS>;
    const size_t smem = sizeof(Shared<DP, ROWS>);
    static_assert(sizeof(Shared<DP, ROWS>) <= 227 * 1024, "shared memory of one CTA");
    AttnMaps maps;
    const sharpv_status ms = encode_attn_maps(a, kKeys, maps, C::kBox);
    if (ms != SHARPV_OK) return ms;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        launch_dependent(kern, dim3((unsigned)a.ctas), dim3(C::kThreads), smem, stream, a, maps) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int CODE>
sharpv_status by_dim(const AttnArgs& a, cudaStream_t stream) {
    if (a.split.rows == 8)
        return a.head_dim <= 64 ? launch<8, 64>(attn_rows8_q8_kernel<CODE, 64>, a, stream) : launch<8, 128>(attn_rows8_q8_kernel<CODE, 128>, a, stream);
    if (a.head_dim <= 64) return launch<16, 64>(attn_rows_q8_kernel<CODE, 64>, a, stream);
    if (a.head_dim <= 128) return launch<16, 128>(attn_rows_q8_kernel<CODE, 128>, a, stream);
    return launch<16, 256>(attn_rows_q8_kernel<CODE, 256>, a, stream);
}

}  // namespace

sharpv_status attn_rows_q8_launch(AttnArgs& a, sharpv_dtype code, int sms, cudaStream_t stream) {
    a.ctas = sms < kMaxRowsCtas ? sms : kMaxRowsCtas;
    return code == SHARPV_E4M3 ? by_dim<SHARPV_E4M3>(a, stream) : by_dim<SHARPV_I8>(a, stream);
}

}  // namespace sharpv
