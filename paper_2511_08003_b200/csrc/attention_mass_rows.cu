// The attention weight that every cached token collects, bf16 caches: K is read once, and that is what bounds it.
//
// Keys are the rows of the tensor cores' products (mma.sync, 16 keys a warp), query rows their columns: a thread then
// holds scores of two keys, adds the weights of all query rows of all heads to two registers, and four lanes
// are added at the end of a tile.  Every key has one owner, so nothing is joined afterwards and the result is written
// (with what the row had collected before) by the same kernel.  A unit is 32 keys of a sequence for every KV head; one
// warp keeps a ring of TMA tile loads in flight, four pairs of warps take the tiles in turn.  The query rows of
// the nodes that count stay in shared memory for a whole portion; if they do not fit, the portion is gone through
// again for the next ones, as many KV heads of them as fit with eight rows each (8 x 256 columns, 8 query heads each, 6,272
// rows: 64 nodes, in 22 lots, 85 us; 509 nodes, in 170, 642 us).
//
// Measured (4 KV heads x 128, 7 query heads each): 1 node over 50,432 rows 15.6 us, of which 5 us go by until the query
// rows are there; then K streams at 6.2 TB/s.  56 query rows a head: 17.4 us.
#include "attention_mass.cuh"
#include "tma.cuh"

namespace sharpv {
namespace {

constexpr int kKeys = 32;               // of a tile
constexpr int kWarps = 8, kPairs = 4;
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kRingBytes = 96 * 1024;
constexpr int kQueryBytes = 108 * 1024; // query rows, their weights and log-sum-exps
constexpr int kRowsMax = 512;           // query rows of a head in a pass

template <int DP>
struct Cfg {
    static constexpr int kTileBytes = kKeys * DP * 2;
    static constexpr int kStages = kRingBytes / kTileBytes / kPairs;        // of a pair's own ring
    static constexpr int kPitch = DP * 2 + 16;              // of a query row: 8 rows fall on 8 bank groups
};

// What of the query rows is in shared memory at a time: `heads` KV heads, `rows` rows of each (a multiple of 8).
struct Pass {
    int heads, rows;
};

template <int DP>
struct Shared {
    using C = Cfg<DP>;
    uint8_t tiles[kPairs][C::kStages][C::kTileBytes];       // every pair waits for every use of its stages, in order
    uint64_t full[kPairs][C::kStages], empty[kPairs][C::kStages];
    int list[kRowsMax + 1];                                 // nodes of a pass that count
    int64_t row_at[kRowsMax];                               // byte offset of a query row (of head 0 of its group), -1: none
    int scan[kWarps];
    int dead;
    PlanScratch<kThreads> plan;
    __align__(16) uint8_t query[kQueryBytes];               // [heads][rows] pitch, then log-sum-exps [heads][rows], weights [rows]
};

__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" :: "n"(kWarps * 32) : "memory"); }

__device__ __forceinline__ bool counts(const MassArgs& a, int64_t node) {
    return a.weight == nullptr || __ldg(a.weight + node) != 0.f;
}

// The weights of N blocks of eight query rows for the warp's 16 keys, added to the thread's two keys.
template <int N, int DP>
__device__ __forceinline__ void weigh(const uint32_t (&kf)[DP / 16][4], uint32_t qb, const float* lse2, const float* weight, int nb,
                                      float scale_log2, float& sum0, float& sum1) {
    float c[N][4];
#pragma unroll
    for (int j = 0; j < N; ++j) c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ks += 2) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            uint32_t q4[4];
            ldmatrix4(q4, qb + (nb + j) * 8 * Cfg<DP>::kPitch + ks * 32);
            mma_bf16(c[j], kf[ks], q4[0], q4[1]);
            mma_bf16(c[j], kf[ks + 1], q4[2], q4[3]);
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float2 ls = *reinterpret_cast<const float2*>(lse2 + (nb + j) * 8), wt = *reinterpret_cast<const float2*>(weight + (nb + j) * 8);
        sum0 = add_weight(sum0, wt.x, c[j][0], scale_log2, ls.x);
        sum0 = add_weight(sum0, wt.y, c[j][1], scale_log2, ls.y);
        sum1 = add_weight(sum1, wt.x, c[j][2], scale_log2, ls.x);
        sum1 = add_weight(sum1, wt.y, c[j][3], scale_log2, ls.y);
    }
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
mass_rows_kernel(const __grid_constant__ MassArgs a, const __grid_constant__ CUtensorMap map, const Pass ps) {
    using C = Cfg<DP>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int D = a.head_dim, G = a.split.group, H = a.split.heads, HQ = H * G;
    const KeySplit split{kKeys, G, a.weight != nullptr};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairs * C::kStages; ++i) {
            mbar_init(&sm.full[0][i], 1);
            mbar_init(&sm.empty[0][i], 2);
        }
        mbar_fence_init();
        sm.dead = 0;
    }
    if (warp == kWarps && lane == 0) tma_prefetch(&map);
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kThreads>(a.seqs, split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    KeyWalk walk(plan, first, end);
    const int head_passes = (H + ps.heads - 1) / ps.heads;
    bool alive = true;

    if (warp == kWarps) {
        uint32_t it[kPairs] = {};                       // tiles of every pair so far
        while (walk.next(a.seqs, split)) {
            // how often the portion is gone through: by the number of nodes that count
            int active = 0;
            if (a.weight == nullptr) {
                active = walk.s.nodes;
            } else {
                for (int x = 0; x < walk.s.nodes; x += 32)
                    active += __popc(__ballot_sync(0xffffffffu, x + lane < walk.s.nodes && counts(a, walk.s.node0 + x + lane)));
            }
            const int row_passes = (int)(((int64_t)active * G + ps.rows - 1) / ps.rows);
            if (lane == 0) {
                for (int rp = 0; rp < row_passes; ++rp)
                    for (int hp = 0; hp < head_passes; ++hp) {
                        const int h0 = hp * ps.heads, h1 = min(H, h0 + ps.heads);
                        for (int kt = walk.kt0; kt < walk.kt1; kt += kPairs) {
                            const int n = min(kPairs, walk.kt1 - kt);
                            for (int h = h0; h < h1; ++h)
#pragma unroll
                                for (int t = 0; t < kPairs; ++t) {
                                    if (t >= n || !alive) break;
                                    const int stage = it[t] % C::kStages;
                                    if (it[t] >= C::kStages) alive = mbar_wait(&sm.empty[t][stage], (it[t] / C::kStages - 1) & 1);
                                    if (!alive) break;
                                    mbar_expect(&sm.full[t][stage], C::kTileBytes);
#pragma unroll
                                    for (int x = 0; x < DP / 64; ++x)
                                        tma_load(sm.tiles[t][stage] + x * kKeys * 128, &map, &sm.full[t][stage], x * 64,
                                                 (int)walk.s.begin + (kt + t) * kKeys, h);
                                    ++it[t];
                                }
                        }
                    }
            }
            alive = __all_sync(0xffffffffu, alive);
            if (!alive) break;
        }
        if (lane == 0) {
            if (!alive) report(a.status_word, SHARPV_ERR_TIMEOUT);
            // copies in flight land before the CTA ends, also where the warps that wanted them gave up
#pragma unroll
            for (int t = 0; t < kPairs; ++t)
                for (uint32_t i = 0; i < (uint32_t)C::kStages && i < it[t]; ++i) {
                    const uint32_t last = it[t] - 1 - i;
                    (void)mbar_wait(&sm.full[t][last % C::kStages], (last / C::kStages) & 1);
                }
        }
        return;
    }

    const int pair = warp >> 1, sub = warp & 1;
    const int tid = threadIdx.x;
    uint32_t it = 0;                            // the pair's tiles so far
    float* const lse2 = reinterpret_cast<float*>(sm.query + (size_t)ps.heads * ps.rows * C::kPitch);
    float* const weight = lse2 + ps.heads * ps.rows;
    while (walk.next(a.seqs, split)) {
        const SeqInfo& s = walk.s;
        const int p0 = walk.kt0 * kKeys + sub * 16 + (lane >> 2);       // key of this thread in tile kt0 (and 8 further)

        for (int rp = 0;; ++rp) {
            // ---- the nodes of this pass: rows [rp * rows, ...) of the rows of the nodes that count, node by node
            const int row0 = rp * ps.rows;
            const int k0 = row0 / G;                                    // first node of the pass, in order of those that count
            consumer_sync();
            if (sm.dead) return;
            int seen = 0;
            if (a.weight == nullptr) {
                seen = s.nodes;
            } else {
                for (int x0 = 0; x0 < s.nodes; x0 += kWarps * 32) {
                    const int x = x0 + tid;
                    const bool on = x < s.nodes && counts(a, s.node0 + x);
                    const uint32_t mask = __ballot_sync(0xffffffffu, on);
                    if (lane == 0) sm.scan[warp] = __popc(mask);
                    consumer_sync();
                    int at = seen + __popc(mask & ((1u << lane) - 1u));
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        if (w < warp) at += sm.scan[w];
                        seen += sm.scan[w];
                    }
                    if (on && at >= k0 && at - k0 < kRowsMax + 1) sm.list[at - k0] = x;
                    consumer_sync();
                }
            }
            const int all_rows = seen * G;
            const int rows = max(0, min(ps.rows, all_rows - row0));     // of this pass, a head
            const int blocks = (rows + 7) / 8;
            for (int r = tid; r < blocks * 8; r += kWarps * 32) {
                int64_t at = -1;
                float wt = 0.f;
                if (r < rows) {
                    const int k = (row0 + r) / G, g = row0 + r - k * G;
                    const int64_t node = s.node0 + (a.weight == nullptr ? k : sm.list[k - k0]);
                    at = node * a.q_node + (int64_t)g * D * 2;
                    wt = a.weight == nullptr ? 1.f : __ldg(a.weight + node);
                }
                sm.row_at[r] = at;
                weight[r] = wt;
            }
            consumer_sync();
            for (int hp = 0; hp < head_passes; ++hp) {
                const int h0 = hp * ps.heads, hn = min(H - h0, ps.heads);
                if (hp > 0) consumer_sync();
                constexpr int CH = DP / 8;
                for (int h = 0; h < hn; ++h)            // log-sum-exps first, then the query rows, all on their way at the same time
                    for (int r = tid; r < blocks * 8; r += kWarps * 32) {
                        if (r < rows) {
                            const int k = (row0 + r) / G, g = row0 + r - k * G;
                            const int64_t node = s.node0 + (a.weight == nullptr ? k : sm.list[k - k0]);
                            cp_async4(&lse2[h * ps.rows + r], a.lse + node * HQ + (h0 + h) * G + g);
                        } else {
                            lse2[h * ps.rows + r] = kNoRow;
                        }
                    }
                for (int h = 0; h < hn; ++h) {
                    for (int r = tid / CH; r < blocks * 8; r += kWarps * 32 / CH) {
                        const int c = tid % CH;
                        const int64_t at = sm.row_at[r];
                        const bool there = at >= 0 && c * 8 < D;
                        cp_async16(sm.query + (size_t)(h * ps.rows + r) * C::kPitch + c * 16,
                                   there ? a.q + at + (int64_t)(h0 + h) * G * D * 2 + c * 16 : a.q, there);
                    }
                }
                cp_async_wait_all();
                for (int h = 0; h < hn; ++h)
                    for (int r = tid; r < blocks * 8; r += kWarps * 32) {       // the thread's own
                        if (r < rows) lse2[h * ps.rows + r] = lse_log2(lse2[h * ps.rows + r]);
                    }
                consumer_sync();
                const bool fresh = rp == 0 && hp == 0;
                for (int kt = walk.kt0; kt < walk.kt1; kt += kPairs) {
                    const int n = min(kPairs, walk.kt1 - kt);
                    if (pair >= n) continue;
                    const int key = p0 + (kt - walk.kt0 + pair) * kKeys;            // of the sequence
                    const bool writes = (lane & 3) < 2;                             // lane 0 of four: key, lane 1: key + 8
                    const int my_key = key + (lane & 3) * 8;
                    float old = 0.f;
                    if (writes && my_key < s.len) {
                        if (!fresh) old = a.out[s.begin + my_key];
                        else if (a.mass != nullptr && a.decay != 0.f) old = a.decay * a.mass[s.begin + my_key];
                    }
                    float sum0 = 0.f, sum1 = 0.f;
                    if (rows > 0) {
                        for (int h = 0; h < hn; ++h, ++it) {
                            const int stage = it % C::kStages;
                            if (alive && !mbar_wait(&sm.full[pair][stage], (it / C::kStages) & 1)) {
                                alive = false;
                                sm.dead = 1;
                                report(a.status_word, SHARPV_ERR_TIMEOUT);
                            }
                            const uint32_t kb = smem_u32(sm.tiles[pair][stage]);
                            uint32_t kf[DP / 16][4];
#pragma unroll
                            for (int ks = 0; ks < DP / 16; ++ks)
                                ldmatrix4(kf[ks], kb + (ks >> 2) * (kKeys * 128) + swizzle128(sub * 16 + (lane & 15), (ks & 3) * 2 + (lane >> 4)));
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&sm.empty[pair][stage]);
                            const uint32_t qb = smem_u32(sm.query) + (uint32_t)(h * ps.rows + (lane & 7)) * C::kPitch + (lane >> 3) * 16;
                            const float* hl = lse2 + h * ps.rows + (lane & 3) * 2;
                            const float* hw = weight + (lane & 3) * 2;
                            // four blocks of eight query rows at a time: products of one block wait for one another
                            int nb = 0;
                            for (; nb + 4 <= blocks; nb += 4) weigh<4, DP>(kf, qb, hl, hw, nb, a.scale_log2, sum0, sum1);
                            if (nb + 2 <= blocks) {
                                weigh<2, DP>(kf, qb, hl, hw, nb, a.scale_log2, sum0, sum1);
                                nb += 2;
                            }
                            if (nb < blocks) weigh<1, DP>(kf, qb, hl, hw, nb, a.scale_log2, sum0, sum1);
                        }
                    }
                    sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1);
                    sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
                    sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1);
                    sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
                    if (writes && my_key < s.len) a.out[s.begin + my_key] = old + ((lane & 3) == 0 ? sum0 : sum1);
                }
            }
            if (all_rows - row0 <= ps.rows) break;
        }

    }
}

template <int DP>
sharpv_status launch(const MassArgs& a, const Pass& ps, cudaStream_t stream) {
    auto kern = mass_rows_kernel<DP>;
    const size_t smem = sizeof(Shared<DP>);
    static_assert(sizeof(Shared<DP>) <= 227 * 1024, "shared memory of one CTA");
    CUtensorMap map;
    if (!encode_rows_map(&map, a.cache_k, a.head_dim, a.seqs.cache_tokens, a.kv_token, a.split.heads, a.kv_head, kKeys))
        return SHARPV_ERR_CUDA;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kThreads), smem, stream, a, map, ps) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

}  // namespace

sharpv_status mass_rows_launch(MassArgs& a, int sms, cudaStream_t stream) {
    a.ctas = sms;
    const int DP = a.head_dim <= 64 ? 64 : (a.head_dim <= 128 ? 128 : 256);
    const int row_bytes = DP * 2 + 16 + 8;
    // all heads at a time if eight rows of each fit; then as many rows as fit, but no more than there can be
    Pass ps;
    ps.heads = a.split.heads;
    if ((int64_t)ps.heads * 8 * row_bytes > kQueryBytes) ps.heads = kQueryBytes / (8 * row_bytes);
    const int64_t fit = kQueryBytes / ((int64_t)ps.heads * row_bytes) / 8 * 8;
    const int64_t can = (a.seqs.total_nodes * a.split.group + 7) / 8 * 8;
    ps.rows = (int)(can < fit ? (can > 8 ? can : 8) : fit);
    if (ps.rows > kRowsMax) ps.rows = kRowsMax;
    if (DP == 64) return launch<64>(a, ps, stream);
    if (DP == 128) return launch<128>(a, ps, stream);
    return launch<256>(a, ps, stream);
}

}  // namespace sharpv
