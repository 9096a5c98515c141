// Attention of few query rows over a K/V cache in bf16: every K and V row is read once, and that is what bounds it.
//
// One CTA per SM takes its share of the key tiles (64 keys, K and V together 32 KB at head_dim 128).  One warp
// keeps a ring of TMA tile loads in flight; two groups of four warps take the tiles in turn, every warp 16 keys of its
// tile for all of the segment's 16 query rows: scores and weighted sums on the tensor cores (mma.sync: 16
// rows fill it, and the time is that of the loads), running maximum, sum and result in registers.  A warp needs nobody
// else until the end of its portion, where the eight results are joined through shared memory.
//
// Measured (4 KV heads x 128, 7 query heads each): one token over 50,432 rows 26.4 us with the join, of which 14 us stream
// the 103 MB; 16 single tokens over 37,712 ragged rows 24.4 us; 64 over 2,000 rows each 51 us (5.2 TB/s).
#include "tma.cuh"
#include "tree_attention.cuh"

#include <cuda_bf16.h>

namespace sharpv {
namespace {

constexpr int kKeys = kRowsTileKeys;            // of a tile
constexpr int kRows = kRowsTileRows;
constexpr int kWarps = 8;                       // that compute, in two groups of four
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kMergeCols = 128;                 // columns that are joined at a time

template <int DP>
struct Cfg {
    static constexpr int kHalves = DP / 64;                     // TMA boxes of 64 columns
    static constexpr int kTileBytes = kKeys * DP * 2;           // K or V
    static constexpr int kStages = DP == 64 ? 8 : (DP == 128 ? 4 : 2);
    static constexpr bool kQInRegs = DP <= 128;
    static constexpr int kQPitch = DP * 2 + 16;                 // bytes; 16 more, so that 8 rows fall on 8 bank groups
    static constexpr int kCols = DP < kMergeCols ? DP : kMergeCols;
};

template <int DP>
struct Shared {
    using C = Cfg<DP>;
    uint8_t tiles[C::kStages][2][C::kTileBytes];
    float merge[kWarps][16][C::kCols + 4];
    float m[kWarps][16], l[kWarps][16];
    float top[16], sum[16];
    uint8_t q[2][kRows * C::kQPitch];         // query rows of this portion and the next
    Portion part[2];                            // kt1 < 0: there are no more
    uint64_t full[C::kStages], empty[C::kStages], part_full[2], part_empty[2];
    int poison, dead;
    PlanScratch<kThreads> plan;
};

__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" :: "n"(kWarps * 32) : "memory"); }

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attn_rows_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnMaps maps) {
    using C = Cfg<DP>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    auto& sm = *reinterpret_cast<Shared<DP>*>(smem_raw);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.part_full[i], 33);        // 32 lanes' query rows have landed, and the portion is written
            mbar_init(&sm.part_empty[i], kWarps);
        }
        mbar_fence_init();
        sm.poison = sm.dead = 0;
    }
    if (warp == kWarps && lane < 4) tma_prefetch(&maps.cache_k + lane);
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kThreads>(a.seqs, a.split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    bool alive = true;                          // a wait that gave up: nothing is waited for any more, the result is void
    uint32_t it = 0, pn = 0;                    // tiles and portions of this CTA so far
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G;

    if (warp == kWarps) {                       // portions, query rows and tiles ahead of the warps that compute
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
                // two lanes a row, every second chunk each
                const int r = lane >> 1, row = r_base + r;
                const bool there = row < r_all;
                const int node = there ? row / G : 0, g = there ? row - node * G : 0;
                const char* q = a.q + (int64_t)(p.s.node0 + node) * a.q_node + (int64_t)(p.h * G + g) * D * 2;
                uint8_t* to = sm.q[slot] + r * C::kQPitch;
#pragma unroll
                for (int c = lane & 1; c < DP / 8; c += 2) cp_async16(to + c * 16, c * 8 < D ? q + c * 16 : q, there && c * 8 < D);
            }
            cp_async_arrive(&sm.part_full[slot]);
            if (lane == 0) {
                if (!more) p.kt1 = -1;
                sm.part[slot] = p;
                mbar_arrive(&sm.part_full[slot]);
            }
            if (!more) break;
            if (lane == 0) {
                for (int kt = p.kt0; kt < p.kt1; ++kt, ++it) {
                    const int stage = it % C::kStages;
                    if (it >= C::kStages) alive = mbar_wait(&sm.empty[stage], (it / C::kStages - 1) & 1);
                    if (!alive) break;
                    const bool drafted = kt >= p.kt_cache;
                    if (drafted && !a.split.draft) {            // the empty tile of rows without keys
                        mbar_arrive(&sm.full[stage]);
                        continue;
                    }
                    mbar_expect(&sm.full[stage], 2 * C::kTileBytes);
                    const CUtensorMap* mk = drafted ? &maps.draft_k : &maps.cache_k;
                    const CUtensorMap* mv = drafted ? &maps.draft_v : &maps.cache_v;
                    const int row = drafted ? p.s.node0 + (kt - p.kt_cache) * kKeys : (int)p.s.begin + kt * kKeys;
#pragma unroll
                    for (int x = 0; x < C::kHalves; ++x)
                        tma_load(sm.tiles[stage][0] + x * kKeys * 128, mk, &sm.full[stage], x * 64, row, p.h);
#pragma unroll
                    for (int x = 0; x < C::kHalves; ++x)
                        tma_load(sm.tiles[stage][1] + x * kKeys * 128, mv, &sm.full[stage], x * 64, row, p.h);
                }
            }
            alive = __all_sync(0xffffffffu, alive);
            if (!alive) break;
        }
        if (lane == 0) {
            if (!alive) report(a.status_word, SHARPV_ERR_TIMEOUT);
            note_shared(a, alive && pn > 0, last, end, plan);
            // copies in flight land before the CTA ends, also where the warps that wanted them gave up
            for (int i = 0; i < C::kStages && (uint32_t)i < it; ++i) {
                const uint32_t at = it - 1 - i;
                (void)mbar_wait(&sm.full[at % C::kStages], (at / C::kStages) & 1);
            }
        }
        cp_async_wait<0>();
        return;
    }

    const int group = warp >> 2, sub = warp & 3;        // tiles of this parity, 16 keys from sub * 16 on
    const int qr = lane >> 2, qc = (lane & 3) * 2;      // fragment row (and row + 8), column (and column + 1)
    for (;; ++pn) {
        const int at_part = pn & 1;
        if (alive && !mbar_wait(&sm.part_full[at_part], (pn >> 1) & 1)) {
            alive = false;
            report(a.status_word, SHARPV_ERR_TIMEOUT);
        }
        if (!alive) sm.dead = 1;
        consumer_sync();                        // all eight warps go on or none does
        const Portion p = sm.part[at_part];
        if (p.kt1 < 0 || sm.dead) break;
        const int r_base = p.rt * kRows, r_all = p.s.nodes * G;
        const uint32_t q_base = smem_u32(sm.q[at_part]) + (lane & 15) * C::kQPitch + (lane >> 4) * 16;
        uint32_t qf[C::kQInRegs ? DP / 16 : 1][4];
        if constexpr (C::kQInRegs) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) ldmatrix4(qf[ks], q_base + ks * 32);
        }
        float o[DP / 8][4];
        float m[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};        // of rows qr and qr + 8
#pragma unroll
        for (int j = 0; j < DP / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        bool poison = false;                    // a drafted value that is not finite was set aside

        for (int kt = p.kt0; kt < p.kt1; ++kt, ++it) {
            if ((int)(it & 1) != group) continue;
            const int stage = it % C::kStages;
            if (alive && !mbar_wait(&sm.full[stage], (it / C::kStages) & 1)) {
                alive = false;
                report(a.status_word, SHARPV_ERR_TIMEOUT);
            }
            const uint32_t ks_base = smem_u32(sm.tiles[stage][0]), vs_base = smem_u32(sm.tiles[stage][1]);
            float s[2][4] = {};
            const int krow = sub * 16 + (lane >> 4) * 8 + (lane & 7);
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) {
                uint32_t k4[4];
                ldmatrix4(k4, ks_base + (ks >> 2) * (kKeys * 128) + swizzle128(krow, (ks & 3) * 2 + ((lane >> 3) & 1)));
                if constexpr (C::kQInRegs) {
                    mma_bf16(s[0], qf[ks], k4[0], k4[1]);
                    mma_bf16(s[1], qf[ks], k4[2], k4[3]);
                } else {
                    uint32_t q4[4];
                    ldmatrix4(q4, q_base + ks * 32);
                    mma_bf16(s[0], q4, k4[0], k4[1]);
                    mma_bf16(s[1], q4, k4[2], k4[3]);
                }
            }
            const bool drafted = kt >= p.kt_cache;
            const int left = drafted ? (a.split.draft ? p.s.nodes - (kt - p.kt_cache) * kKeys : 0)
                                     : p.s.len - kt * kKeys;        // keys of the tile that are there
            const bool masked = drafted || left < kKeys;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] *= a.scale_log2;
            if (masked) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int row = r_base + qr + half * 8;
                    uint32_t sees;                                  // the warp's 16 keys
                    if (!drafted) {
                        const int n = left - sub * 16;
                        sees = n >= 16 ? 0xffffu : (n <= 0 ? 0u : (1u << n) - 1u);
                    } else {
                        const int key0 = (kt - p.kt_cache) * kKeys + (sub >> 1) * 32;
                        sees = a.split.draft && row < r_all ? draft_sees(a, p.s, row / G, key0) >> ((sub & 1) * 16) : 0u;
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (!(sees >> (n * 8 + qc + i) & 1)) s[n][half * 2 + i] = neg_inf();
                }
            }
            float top[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float x = fmaxf(fmaxf(s[0][half * 2], s[0][half * 2 + 1]), fmaxf(s[1][half * 2], s[1][half * 2 + 1]));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                top[half] = fmaxf(x, m[half]);
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
                const float a0 = m[0] == top[0] ? 1.f : ex2(m[0] - top[0]);
                const float a1 = m[1] == top[1] ? 1.f : ex2(m[1] - top[1]);
                m[0] = top[0];
                m[1] = top[1];
                l[0] *= a0;
                l[1] *= a1;
#pragma unroll
                for (int j = 0; j < DP / 8; ++j) {
                    o[j][0] *= a0;
                    o[j][1] *= a0;
                    o[j][2] *= a1;
                    o[j][3] *= a1;
                }
            }
            const float b0 = m[0] == neg_inf() ? 0.f : m[0], b1 = m[1] == neg_inf() ? 0.f : m[1];
            uint32_t pf[4];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float p0 = ex2(s[n][0] - b0), p1 = ex2(s[n][1] - b0);
                const float p2 = ex2(s[n][2] - b1), p3 = ex2(s[n][3] - b1);
                l[0] += p0 + p1;
                l[1] += p2 + p3;
                // weights are rounded to bf16 for the product with the values; their sum is not
                pf[n * 2] = pack_bf16(p0, p1);
                pf[n * 2 + 1] = pack_bf16(p2, p3);
            }
            const int vrow = sub * 16 + (lane & 15);
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
                uint32_t v4[4];
                ldmatrix4_trans(v4, vs_base + (j >> 2) * (kKeys * 128) + swizzle128(vrow, (j & 3) * 2 + (lane >> 4)));
                if (masked) {
                    // rows that are not there may hold anything, and so may drafted rows that some query rows do
                    // not see: 0 times them would not be 0
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = sub * 16 + (i & 1) * 8 + qc;
                        if (key >= left) v4[i] = 0u;
                        else if (key + 1 >= left) v4[i] &= 0xffffu;
                        if (drafted) {
                            const uint32_t off = nonfinite_bf16(v4[i]);
                            v4[i] &= ~off;
                            poison |= off != 0;
                        }
                    }
                }
                mma_bf16(o[j * 2], pf, v4[0], v4[1]);
                mma_bf16(o[j * 2 + 1], pf, v4[2], v4[3]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[stage]);
        }

        // ---- the eight warps' results are joined, up to 128 columns at a time
        const bool complete = p.kt0 == 0 && p.kt1 == p.kt_all;
        const int slot = portion_slot(blockIdx.x, p.kt0);
        if (poison) sm.poison = 1;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
            if ((lane & 3) == 0) { sm.m[warp][qr + half * 8] = m[half]; sm.l[warp][qr + half * 8] = l[half]; }
        }
#pragma unroll
        for (int c0 = 0; c0 < DP; c0 += C::kCols) {
#pragma unroll
            for (int j = c0 / 8; j < (c0 + C::kCols) / 8; ++j) {
                *reinterpret_cast<float2*>(&sm.merge[warp][qr][j * 8 - c0 + qc]) = make_float2(o[j][0], o[j][1]);
                if (r_base + 8 < r_all)         // rows 8 to 15 hold something
                    *reinterpret_cast<float2*>(&sm.merge[warp][qr + 8][j * 8 - c0 + qc]) = make_float2(o[j][2], o[j][3]);
            }
            consumer_sync();
            constexpr int V = C::kCols / 4;
            for (int x = threadIdx.x; x < 16 * V; x += kWarps * 32) {
                const int r = x / V, c = c0 + (x % V) * 4, row = r_base + r;
                if (row >= r_all || c >= D) continue;
                float top = sm.m[0][r];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm.m[w][r]);
                const float base = top == neg_inf() ? 0.f : top;
                float sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float f = ex2(sm.m[w][r] - base);
                    const float4 v = *reinterpret_cast<const float4*>(&sm.merge[w][r][c - c0]);
                    sum = fmaf(f, sm.l[w][r], sum);
                    acc.x = fmaf(f, v.x, acc.x);
                    acc.y = fmaf(f, v.y, acc.y);
                    acc.z = fmaf(f, v.z, acc.z);
                    acc.w = fmaf(f, v.w, acc.w);
                }
                if (sm.poison) {
                    // what was set aside comes back to the rows that see it
                    const int j0 = (max(p.kt0, p.kt_cache) - p.kt_cache) * kKeys, j1 = min(p.s.nodes, (p.kt1 - p.kt_cache) * kKeys);
                    for (int j = j0; j < j1; ++j) {
                        if (!(draft_sees(a, p.s, row / G, j & ~31) >> (j & 31) & 1)) continue;
                        const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(
                            a.draft_v + (int64_t)(p.s.node0 + j) * a.dv_node) + p.h * D + c;
                        const float v0 = __bfloat162float(v[0]), v1 = __bfloat162float(v[1]);
                        const float v2 = __bfloat162float(v[2]), v3 = __bfloat162float(v[3]);
                        if (!finite_f32(v0)) acc.x += v0;
                        if (!finite_f32(v1)) acc.y += v1;
                        if (!finite_f32(v2)) acc.z += v2;
                        if (!finite_f32(v3)) acc.w += v3;
                    }
                }
                const int64_t at = (int64_t)(p.s.node0 + row / G) * HQ + p.h * G + row % G;
                if (complete) {
                    const float inv = row_scale(sum);
                    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at * D + c) =
                        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                    if (c == 0) a.lse[at] = row_lse(top, sum);
                } else {
                    *reinterpret_cast<float4*>(a.part_o + ((int64_t)slot * kRows + r) * D + c) = acc;
                    if (c == 0) {
                        a.part_ml[(int64_t)slot * 2 * kRows + r] = top;
                        a.part_ml[((int64_t)slot * 2 + 1) * kRows + r] = sum;
                    }
                }
            }
            consumer_sync();
        }
        if (threadIdx.x == 0) sm.poison = 0;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.part_empty[at_part]);
    }
}

template <int DP>
sharpv_status launch(const AttnArgs& a, cudaStream_t stream) {
    using C = Cfg<DP>;
    auto kern = attn_rows_kernel<DP>;
    const size_t smem = sizeof(Shared<DP>);
    static_assert(sizeof(Shared<DP>) <= 227 * 1024, "shared memory of one CTA");
    AttnMaps maps;
    const sharpv_status ms = encode_attn_maps(a, kKeys, maps);
    if (ms != SHARPV_OK) return ms;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kThreads), smem, stream, a, maps) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

}  // namespace

sharpv_status encode_attn_maps(const AttnArgs& a, int box_rows, AttnMaps& maps) {
    const int D = a.head_dim, H = a.split.heads;
    const int64_t T = a.seqs.cache_tokens > 0 ? a.seqs.cache_tokens : 1, N = a.seqs.total_nodes;
    const int64_t most = (int64_t)1 << 40;              // what a tensor map's strides can say
    if (a.kv_token >= most || a.kv_head >= most || a.dk_node >= most || a.dv_node >= most || a.q_node >= most) return SHARPV_ERR_UNSUPPORTED;
    bool ok = encode_rows_map(&maps.cache_k, a.cache_k, D, T, a.kv_token, H, a.kv_head, box_rows) &&
              encode_rows_map(&maps.cache_v, a.cache_v, D, T, a.kv_token, H, a.kv_head, box_rows);
    if (a.split.draft)
        ok = ok && encode_rows_map(&maps.draft_k, a.draft_k, D, N, a.dk_node, H, (int64_t)D * 2, box_rows) &&
             encode_rows_map(&maps.draft_v, a.draft_v, D, N, a.dv_node, H, (int64_t)D * 2, box_rows);
    else {
        maps.draft_k = maps.cache_k;
        maps.draft_v = maps.cache_v;
    }
    if (ok && box_rows == kTcTileKeys)
        ok = encode_heads_map(&maps.query, a.q, D, H * a.split.group, N, a.q_node, a.split.group, a.split.rows / (2 * a.split.group));
    return ok ? SHARPV_OK : SHARPV_ERR_CUDA;
}

sharpv_status attn_rows_launch(AttnArgs& a, int sms, cudaStream_t stream) {
    a.ctas = sms < kMaxRowsCtas ? sms : kMaxRowsCtas;
    if (a.head_dim <= 64) return launch<64>(a, stream);
    if (a.head_dim <= 128) return launch<128>(a, stream);
    return launch<256>(a, stream);
}

}  // namespace sharpv
