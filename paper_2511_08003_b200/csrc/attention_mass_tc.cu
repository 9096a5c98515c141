// The attention weight that every cached token collects from many query rows, bf16 caches, on the fifth-generation
// tensor cores.
//
// The scores of 128 keys with up to 256 query rows are one product of 128 x 256 x head_dim into tensor memory, keys
// as lanes: a thread owns a key and adds the weights of all query rows of all heads to one register, without
// shuffles.  Two such blocks of columns take turns, so the tensor cores work on one while eight warps weigh the
// other (the two warps of a lane quarter take 32 columns in turn and are added once a tile).  A unit is 128 keys of a
// sequence for every KV head; every key has one owner and the result is written by the same kernel, as in
// attention_mass_rows.cu.  The query rows of the nodes that count stay in shared memory for a whole portion, for as many
// heads at a time as fit; K is read once unless one head's rows alone do not fit.
//
// What bounds it are the exponentials, one a (key, query row).  Measured (4 KV heads x 128, 7 query heads each): 64 nodes over
// 50,432 rows 32 us (0.71 PFLOP/s); accepted nodes of 16 ragged sequences 23.5 us; 509 nodes over 10,944 rows, in several
// passes, 144 us (0.28 PFLOP/s).
#include "attention_mass.cuh"
#include "tcgen05.cuh"

namespace sharpv {
namespace {

constexpr int kKeys = 128;
constexpr int kWeighWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kThreads = 320, kWeighThreads = 256;
constexpr int kStages = 5;              // of the ring: 64 columns of a key tile each, 16 KB
constexpr int kRowsMax = 512;           // query rows in shared memory, all heads of a pass together
constexpr int kBlock = 32;              // columns a warp weighs at a time; rows of a head are padded to it

// What of a sequence's query rows is in shared memory at a time: `heads` KV heads, `rows` rows of each (a multiple of
// kBlock).  As many heads as fit with all their rows, in even lots; if not even one does, its rows one lot after the other.
struct Pass {
    int heads, rows;
    __device__ __forceinline__ Pass(int all_rows, int num_heads) {
        const int need = max((all_rows + kBlock - 1) / kBlock, 1) * kBlock;
        heads = need >= kRowsMax ? 1 : min(kRowsMax / need, num_heads);
        const int lots = (num_heads + heads - 1) / heads;
        heads = (num_heads + lots - 1) / lots;
        rows = min(need, kRowsMax / heads / kBlock * kBlock);
    }
};

template <int DP>
struct Shared {
    uint8_t query[kRowsMax * DP * 2];                       // [heads][64-column halves][rows] 128 bytes, swizzled
    uint8_t tiles[kStages][kKeys * 128];
    float lse2[kRowsMax], weight[kRowsMax];                 // [heads][rows], [rows]
    int list[kRowsMax + 1];                                 // nodes of a pass that count
    float half[kKeys];                                      // sums of the second warp of every lane quarter
    uint64_t full[kStages], empty[kStages], scored[2], weighed[2], ready, taken, drain;
    int scan[kWeighWarps];
    int rows, room, heads, last;                            // of the pass that is ready: rows of a head, places for them, heads, whether
                                                            // it is a portion's last
    int dead;
    uint32_t tmem;
    PlanScratch<kThreads> plan;
};

__device__ __forceinline__ void weigh_sync() { asm volatile("bar.sync 1, %0;" :: "n"(kWeighThreads) : "memory"); }

__device__ __forceinline__ bool counts(const MassArgs& a, int64_t node) {
    return a.weight == nullptr || __ldg(a.weight + node) != 0.f;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
mass_tc_kernel(const __grid_constant__ MassArgs a, const __grid_constant__ CUtensorMap map) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    const int D = a.head_dim, G = a.split.group, H = a.split.heads, HQ = H * G;
    const KeySplit split{kKeys, G, a.weight != nullptr};
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.scored[i], 1);
            mbar_init(&sm.weighed[i], kWeighWarps);
        }
        mbar_init(&sm.ready, kWeighThreads);
        mbar_init(&sm.taken, 1);
        mbar_init(&sm.drain, 1);
        mbar_fence_init();
        sm.dead = 0;
    }
    if (warp == kMmaWarp) tmem_alloc(&sm.tmem, 512);
    if (warp == kLoadWarp && lane == 0) tma_prefetch(&map);
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kThreads>(a.seqs, split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    KeyWalk walk(plan, first, end);
    bool alive = true;          // a wait that gave up ends the role; the others then give up as well
    auto wait = [&](uint64_t* bar, uint32_t phase) {
        if (alive && !mbar_wait(bar, phase & 1)) alive = false;
        return alive;
    };

    if (warp == kLoadWarp) {
        uint32_t it = 0;
        while (alive && walk.next(a.seqs, split)) {
            int active = 0;                             // how often the portion is gone through: by the nodes that count
            if (a.weight == nullptr) {
                active = walk.s.nodes;
            } else {
                for (int x = 0; x < walk.s.nodes; x += 32)
                    active += __popc(__ballot_sync(0xffffffffu, x + lane < walk.s.nodes && counts(a, walk.s.node0 + x + lane)));
            }
            const Pass ps(active * G, H);
            const int row_passes = (active * G + ps.rows - 1) / ps.rows, head_passes = (H + ps.heads - 1) / ps.heads;
            if (lane == 0) {
                for (int pass = 0; pass < row_passes * head_passes && alive; ++pass) {
                    const int h0 = pass % head_passes * ps.heads, h1 = min(H, h0 + ps.heads);
                    for (int kt = walk.kt0; kt < walk.kt1 && alive; ++kt)
                        for (int h = h0; h < h1; ++h)
#pragma unroll
                            for (int x = 0; x < DP / 64; ++x, ++it) {
                                const int stage = it % kStages;
                                if (it >= kStages && !wait(&sm.empty[stage], it / kStages - 1)) break;
                                mbar_expect(&sm.full[stage], kKeys * 128);
                                tma_load(sm.tiles[stage], &map, &sm.full[stage], x * 64, (int)walk.s.begin + kt * kKeys, h);
                            }
                }
            }
            alive = __all_sync(0xffffffffu, alive);
        }
        if (lane == 0) {
            // copies in flight land before the CTA ends, also where the warps that wanted them gave up
            for (uint32_t i = 0; i < (uint32_t)kStages && i < it; ++i) {
                const uint32_t last = it - 1 - i;
                (void)mbar_wait(&sm.full[last % kStages], (last / kStages) & 1);
            }
        }
    } else if (warp == kMmaWarp) {
        if (lane == 0) {
            uint32_t it = 0, step = 0, pass = 0;
            bool issued = false;
            while (alive && walk.next(a.seqs, split)) {
                for (bool last = false; !last && alive; ++pass) {
                    if (!wait(&sm.ready, pass)) break;
                    const int rows = sm.rows, room = sm.room, hn = sm.heads;
                    last = sm.last != 0;
                    mbar_arrive(&sm.taken);
                    if (rows == 0) continue;
                    const int cols = (rows + kBlock - 1) / kBlock * kBlock;
                    for (int kt = walk.kt0; kt < walk.kt1 && alive; ++kt)
                        for (int h = 0; h < hn && alive; ++h, it += DP / 64) {
#pragma unroll
                            for (int x = 0; x < DP / 64; ++x) wait(&sm.full[(it + x) % kStages], (it + x) / kStages);
                            for (int c = 0; c < cols && alive; c += 256, ++step) {
                                const int w = step & 1, n = min(256, cols - c);
                                if (step >= 2 && !wait(&sm.weighed[w], (step >> 1) - 1)) break;
                                tc_fence_after();
                                const uint32_t qb = smem_u32(sm.query) + (uint32_t)(h * (DP / 64) * room + c) * 128;
                                const uint32_t shape = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(n / 8) << 17 | 128u / 16 << 24;
#pragma unroll
                                for (int x = 0; x < DP / 64; ++x) {
                                    const uint32_t kb = smem_u32(sm.tiles[(it + x) % kStages]);
#pragma unroll
                                    for (int ks = 0; ks < 4; ++ks)
                                        mma_ss(tmem + w * 256, smem_operand(kb + ks * 32, 1024, 16),
                                               smem_operand(qb + x * room * 128 + ks * 32, 1024, 16), shape, x > 0 || ks > 0);
                                }
                                mma_commit(&sm.scored[w]);
                                issued = true;
                            }
                            if (!alive) break;
#pragma unroll
                            for (int x = 0; x < DP / 64; ++x) mma_commit(&sm.empty[(it + x) % kStages]);
                        }
                }
            }
            if (issued) {
                // the products in flight end before the tensor memory is given back
                mma_commit(&sm.drain);
                (void)mbar_wait(&sm.drain, 0);
            }
        }
    } else {
        const int quarter = warp & 3, second = warp >> 2;           // lanes of tensor memory, which of their two warps
        const uint32_t lanes = (uint32_t)quarter * 32 << 16;
        uint32_t step = 0, pass = 0;
        while (walk.next(a.seqs, split)) {
            const SeqInfo& s = walk.s;
            // the nodes that count: how many, and what that leaves of the rows in shared memory at a time
            int seen = 0;
            if (a.weight == nullptr) {
                seen = s.nodes;
            } else {
                for (int x = lane; x < s.nodes; x += 32) seen += counts(a, s.node0 + x);
                seen = warp_sum_int(seen);
            }
            const int all_rows = seen * G;
            const Pass ps(all_rows, H);
            const int head_passes = (H + ps.heads - 1) / ps.heads;
            bool over = false;
            for (int rp = 0; !over; ++rp) {
                const int row0 = rp * ps.rows, k0 = row0 / G;       // first row, first node of the pass (of those that count)
                weigh_sync();
                if (sm.dead) {
                    alive = false;
                    break;
                }
                if (a.weight != nullptr) {
                    int before = 0;
                    for (int x0 = 0; x0 < s.nodes; x0 += kWeighThreads) {
                        const int x = x0 + tid;
                        const bool on = x < s.nodes && counts(a, s.node0 + x);
                        const uint32_t mask = __ballot_sync(0xffffffffu, on);
                        if (lane == 0) sm.scan[warp] = __popc(mask);
                        weigh_sync();
                        int at = before + __popc(mask & ((1u << lane) - 1u));
#pragma unroll
                        for (int w = 0; w < kWeighWarps; ++w) {
                            if (w < warp) at += sm.scan[w];
                            before += sm.scan[w];
                        }
                        if (on && at >= k0 && at - k0 <= kRowsMax) sm.list[at - k0] = x;
                        weigh_sync();
                    }
                }
                over = all_rows - row0 <= ps.rows;
                const int rows = max(0, min(ps.rows, all_rows - row0)), cols = (rows + kBlock - 1) / kBlock * kBlock;
                for (int hp = 0; hp < head_passes; ++hp) {
                    const int h0 = hp * ps.heads, hn = min(H - h0, ps.heads);
                    if (hp > 0) weigh_sync();
                    constexpr int CH = DP / 8;
                    // log-sum-exps and weights first, then the query rows, all on their way at the same time
                    for (int r = tid; r < cols; r += kWeighThreads) {
                        if (r < rows) {
                            const int k = (row0 + r) / G, g = row0 + r - k * G;
                            const int64_t node = s.node0 + (a.weight == nullptr ? k : sm.list[k - k0]);
                            for (int h = 0; h < hn; ++h) cp_async4(&sm.lse2[h * ps.rows + r], a.lse + node * HQ + (h0 + h) * G + g);
                            if (a.weight != nullptr) cp_async4(&sm.weight[r], a.weight + node);
                            else sm.weight[r] = 1.f;
                        } else {
                            for (int h = 0; h < hn; ++h) sm.lse2[h * ps.rows + r] = kNoRow;
                            sm.weight[r] = 0.f;
                        }
                    }
                    // query rows: CH threads a row, so that a row's place is found once for its chunks
                    for (int r = tid / CH; r < cols; r += kWeighThreads / CH) {
                        const int c = tid % CH;
                        const bool there = r < rows && c * 8 < D;
                        const char* q = a.q;
                        if (there) {
                            const int k = (row0 + r) / G, g = row0 + r - k * G;
                            const int64_t node = s.node0 + (a.weight == nullptr ? k : sm.list[k - k0]);
                            q += node * a.q_node + ((int64_t)(h0 * G + g) * D + c * 8) * 2;
                        }
                        for (int h = 0; h < hn; ++h)
                            cp_async16(sm.query + (size_t)((h * (DP / 64) + (c >> 3)) * ps.rows) * 128 + swizzle128(r, c & 7),
                                       q + (there ? (int64_t)h * G * D * 2 : 0), there);
                    }
                    cp_async_wait_all();
                    for (int r = tid; r < rows; r += kWeighThreads)             // the thread's own
                        for (int h = 0; h < hn; ++h) sm.lse2[h * ps.rows + r] = lse_log2(sm.lse2[h * ps.rows + r]);
                    weigh_sync();
                    if (tid == 0) {
                        if (pass > 0 && !wait(&sm.taken, pass - 1)) sm.dead = 1;
                        sm.rows = rows;
                        sm.room = ps.rows;
                        sm.heads = hn;
                        sm.last = over && hp == head_passes - 1;
                    }
                    async_proxy_fence();
                    mbar_arrive(&sm.ready);
                    ++pass;
                    const bool fresh = rp == 0 && hp == 0;
                    for (int kt = walk.kt0; kt < walk.kt1; ++kt) {
                        const int key = kt * kKeys + quarter * 32 + lane;
                        const bool writes = second == 0 && key < s.len;
                        float old = 0.f;
                        if (writes) {
                            if (!fresh) old = a.out[s.begin + key];
                            else if (a.mass != nullptr && a.decay != 0.f) old = a.decay * a.mass[s.begin + key];
                        }
                        float sum[2] = {0.f, 0.f};
                        if (rows > 0) {
                            for (int h = 0; h < hn; ++h) {
                                for (int c = 0; c < cols; c += 256, ++step) {
                                    const int w = step & 1, n = min(256, cols - c);
                                    if (alive && !__all_sync(0xffffffffu, mbar_wait(&sm.scored[w], (step >> 1) & 1))) {
                                        alive = false;
                                        sm.dead = 1;
                                    }
                                    tc_fence_after();
                                    for (int x = second * kBlock; x < n; x += 2 * kBlock) {
                                        uint32_t v[32];
                                        tmem_ld32(v, tmem + lanes + w * 256 + x);
                                        const float4* ls = reinterpret_cast<const float4*>(sm.lse2 + h * ps.rows + c + x);
                                        const float4* wt = reinterpret_cast<const float4*>(sm.weight + c + x);
                                        tmem_wait_ld();
#pragma unroll
                                        for (int k = 0; k < 8; ++k) {
                                            const float4 l4 = ls[k], w4 = wt[k];
                                            sum[0] = add_weight(sum[0], w4.x, __uint_as_float(v[4 * k]), a.scale_log2, l4.x);
                                            sum[1] = add_weight(sum[1], w4.y, __uint_as_float(v[4 * k + 1]), a.scale_log2, l4.y);
                                            sum[0] = add_weight(sum[0], w4.z, __uint_as_float(v[4 * k + 2]), a.scale_log2, l4.z);
                                            sum[1] = add_weight(sum[1], w4.w, __uint_as_float(v[4 * k + 3]), a.scale_log2, l4.w);
                                        }
                                    }
                                    tc_fence_before();
                                    __syncwarp();
                                    if (lane == 0) mbar_arrive(&sm.weighed[w]);
                                }
                            }
                        }
                        const float mine = sum[0] + sum[1];
                        if (second == 1) sm.half[quarter * 32 + lane] = mine;
                        weigh_sync();
                        if (writes) a.out[s.begin + key] = old + (mine + sm.half[quarter * 32 + lane]);
                        weigh_sync();
                    }
                }
            }
            if (!alive) break;
        }
    }
    if (!alive) report(a.status_word, SHARPV_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

template <int DP>
sharpv_status launch(const MassArgs& a, cudaStream_t stream) {
    auto kern = mass_tc_kernel<DP>;
    const size_t smem = sizeof(Shared<DP>);
    static_assert(sizeof(Shared<DP>) <= 227 * 1024, "shared memory of one CTA");
    CUtensorMap map;
    if (!encode_rows_map(&map, a.cache_k, a.head_dim, a.seqs.cache_tokens, a.kv_token, a.split.heads, a.kv_head, kKeys))
        return SHARPV_ERR_CUDA;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kThreads), smem, stream, a, map) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

}  // namespace

sharpv_status mass_tc_launch(MassArgs& a, int sms, cudaStream_t stream) {
    a.ctas = sms;
    return a.head_dim <= 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}

}  // namespace sharpv
