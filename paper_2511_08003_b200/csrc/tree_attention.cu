// Attention of drafted tokens over a K/V cache (sharpv_tree_attention).
//
//   s_rj = scale q_r . k_j over the cached rows of the row's sequence and the drafted tokens its node sees,
//   out_r = sum_j exp(s_rj - m_r) v_j / l_r,   l_r = sum_j exp(s_rj - m_r),   lse_r = m_r + ln l_r.
//
// Kernels (and those of tree_attention_rows.cu and tree_attention_tc.cu for bf16 caches):
//   attn_simt_kernel      fp32 caches: one pass over the keys with a running maximum and sum per row, on the fp32 units
//   attn_join_kernel      (dependent launch) joins the partial results of segments that several CTAs share
#include "q8.cuh"
#include "tree_attention.cuh"

#include <cuda_bf16.h>

#include <type_traits>

namespace sharpv {
namespace {

constexpr int kSimtThreads = 128;
constexpr int kSimtKeys = 32;           // keys of a tile: one per lane

template <int DT> struct Store;
template <> struct Store<SHARPV_F32> {
    using T = float;
    __device__ __forceinline__ static T from(float x) { return x; }
};
template <> struct Store<SHARPV_BF16> {
    using T = __nv_bfloat16;
    __device__ __forceinline__ static T from(float x) { return __float2bfloat16_rn(x); }
};

constexpr int kSimtRows = 8;            // of a warp

template <int R, int DP>
struct SimtShared {
    static constexpr int kParts = 4 * kSimtRows / R;        // warps that share the rows and split a tile's keys
    float q[R][DP + 4];                 // 4 words of padding: 16 bytes of up to 32 rows are read without bank conflicts
    float k[2][kSimtKeys][DP + 4];      // at a portion's end also the weighted sums of warps that split keys
    float v[2][kSimtKeys][DP];
    float p[R][kSimtKeys];
    float m[kParts][R], l[kParts][R];
    PlanScratch<kSimtThreads> plan;
};

// One tile of up to 32 rows of `src` (byte stride `row_bytes`, `valid` of them, D elements each) into shared memory, the
// rest zero.
template <int DP, int PITCH>
__device__ __forceinline__ void simt_load(float (&dst)[kSimtKeys][PITCH], const char* src, int64_t row_bytes, int valid,
                                          int D) {
    constexpr int VPR = DP / 4;
    for (int x = threadIdx.x; x < kSimtKeys * VPR; x += kSimtThreads) {
        const int j = x / VPR, c = x % VPR * 4;
        const bool there = j < valid && c < D;
        cp_async16(&dst[j][c], there ? src + (int64_t)j * row_bytes + c * 4 : src, there);
    }
}

__device__ __forceinline__ void simt_columns(float (&to)[4], const float* from) {
    const float4 x = *reinterpret_cast<const float4*>(from);
    to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
}
__device__ __forceinline__ void simt_columns(float (&to)[2], const float* from) {
    const float2 x = *reinterpret_cast<const float2*>(from);
    to[0] = x.x; to[1] = x.y;
}

// fp32 caches: the tensor cores would round the operands, so products run on the fp32 units.  A warp owns 8 rows: with R = 32
// each warp others and all of a tile's keys, with R = 8 all warps the same and a quarter of the keys each (K and V then
// leave shared memory once), joined at a portion's end.  For scores a lane forms RS rows x KS keys (so that reads of shared
// memory keep up with the multiply-adds); for the weighted sums it owns DP / 32 columns of the 8 rows.  What bounds it is
// latency with the few warps that shared memory has room for (three CTAs an SM with R = 8: 63 us against 73 with two).
// Measured: one token over 1,600 rows of 2 x 64 9.4 us, over 50,432 of 4 x 128 63 us (3.3 TB/s); a tree of 64 over 6,272 of
// 4 x 128, 7 query heads each, 230 us (25 TFLOP/s of the fp32 units' 72); 19 nodes over 6,249 of 8 x 128, 5 each, 110 us.
template <int R, int DP>
__global__ void __launch_bounds__(kSimtThreads, DP > 128 ? 2 : 3)
attn_simt_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) char smem_raw[];
    auto& sm = *reinterpret_cast<SimtShared<R, DP>*>(smem_raw);
    constexpr int RW = kSimtRows, PARTS = SimtShared<R, DP>::kParts, KW = kSimtKeys / PARTS;   // rows and keys of a warp
    constexpr int LK = PARTS == 1 ? 16 : 8, KS = KW / LK, RS = RW * LK / 32;                    // lanes along keys; keys, rows of a lane
    constexpr int VW = DP < 128 ? 2 : 4, NV = DP / 32 / VW;                                     // columns: NV times VW neighbours
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kl = lane % LK, rl = lane / LK;
    const int row0 = PARTS == 1 ? warp * RW : 0, key0 = PARTS == 1 ? 0 : warp * KW;
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G;
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kSimtThreads>(a.seqs, a.split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    Walk walk(plan, first, end);
    Portion part;
    bool any = false;
    while (walk.next(a.seqs, a.split, part)) {
        const SeqInfo& s = part.s;
        const int kt_all = part.kt_all, kt_cache = part.kt_cache, kt0 = part.kt0, kt1 = part.kt1, h = part.h;
        const int r_base = part.rt * R, r_all = s.nodes * G;
        any = true;

        auto load_tile = [&](int kt, int buf) {
            const char *k, *v;
            int64_t kb, vb;
            int valid;
            if (kt < kt_cache) {
                const int64_t at = (int64_t)h * a.kv_head + (s.begin + (int64_t)kt * kSimtKeys) * a.kv_token;
                k = a.cache_k + at; v = a.cache_v + at; kb = vb = a.kv_token;
                valid = s.len - kt * kSimtKeys;
            } else {
                const int j0 = (kt - kt_cache) * kSimtKeys;
                const int64_t hb = (int64_t)h * D * 4;
                k = a.draft_k + (int64_t)(s.node0 + j0) * a.dk_node + hb; kb = a.dk_node;
                v = a.draft_v + (int64_t)(s.node0 + j0) * a.dv_node + hb; vb = a.dv_node;
                valid = a.split.draft ? s.nodes - j0 : 0;
            }
            simt_load<DP>(sm.k[buf], k, kb, valid, D);
            simt_load<DP>(sm.v[buf], v, vb, valid, D);
            cp_async_commit();
        };

        __syncthreads();                        // the previous portion's buffers are free
        load_tile(kt0, 0);
        constexpr int VPR = DP / 4;
        for (int x = threadIdx.x; x < R * VPR; x += kSimtThreads) {
            const int r = x / VPR, c = x % VPR * 4, row = r_base + r;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (row < r_all && c < D)
                w = ld_cached(a.q + (int64_t)(s.node0 + row / G) * a.q_node + ((int64_t)(h * G + row % G) * D + c) * 4);
            *reinterpret_cast<uint4*>(&sm.q[r][c]) = w;
        }
        float m[RS], l[RS], o[RW][NV][VW];
#pragma unroll
        for (int i = 0; i < RS; ++i) { m[i] = neg_inf(); l[i] = 0.f; }
#pragma unroll
        for (int i = 0; i < RW; ++i)
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int c = 0; c < VW; ++c) o[i][n][c] = 0.f;
        const bool busy = r_base + row0 < r_all;

        for (int kt = kt0; kt < kt1; ++kt) {
            const int buf = (kt - kt0) & 1;
            cp_async_wait<0>();
            __syncthreads();                    // the tile is there, and nobody reads the other buffer any more
            if (kt + 1 < kt1) load_tile(kt + 1, buf ^ 1);
            if (!busy) continue;
            float acc[RS][KS];
#pragma unroll
            for (int i = 0; i < RS; ++i)
#pragma unroll
                for (int y = 0; y < KS; ++y) acc[i][y] = 0.f;
#pragma unroll 4
            for (int c = 0; c < D; c += 4) {
                float4 k4[KS];
#pragma unroll
                for (int y = 0; y < KS; ++y) k4[y] = *reinterpret_cast<const float4*>(&sm.k[buf][key0 + y * LK + kl][c]);
#pragma unroll
                for (int i = 0; i < RS; ++i) {
                    const float4 q4 = *reinterpret_cast<const float4*>(&sm.q[row0 + rl * RS + i][c]);
#pragma unroll
                    for (int y = 0; y < KS; ++y)
                        acc[i][y] = fmaf(q4.x, k4[y].x, fmaf(q4.y, k4[y].y, fmaf(q4.z, k4[y].z, fmaf(q4.w, k4[y].w, acc[i][y]))));
                }
            }
            const bool drafted = kt >= kt_cache;
            const int left = drafted ? 0 : s.len - kt * kSimtKeys;
            float al[RS];
            bool grown = false;
#pragma unroll
            for (int i = 0; i < RS; ++i) {
                const int r = row0 + rl * RS + i, row = r_base + r;
                uint32_t sees = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
                if (drafted) sees = a.split.draft && row < r_all ? draft_sees(a, s, row / G, (kt - kt_cache) * kSimtKeys) : 0u;
                float x[KS], top = m[i];
#pragma unroll
                for (int y = 0; y < KS; ++y) {
                    x[y] = sees >> (key0 + y * LK + kl) & 1 ? acc[i][y] * a.scale_log2 : neg_inf();
                    top = fmaxf(top, x[y]);
                }
#pragma unroll
                for (int w = LK / 2; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                const float base = top == neg_inf() ? 0.f : top;
                al[i] = m[i] == top ? 1.f : exp2f(m[i] - top);
                grown = grown || al[i] != 1.f;
                float sum = 0.f;
#pragma unroll
                for (int y = 0; y < KS; ++y) {
                    const int key = key0 + y * LK + kl;
                    const bool seen = sees >> key & 1;
                    const float p = seen ? exp2f(x[y] - base) : 0.f;
                    sum += p;
                    sm.p[r][key] = seen || !drafted ? p : -1.f;     // -1: its value row is not looked at
                }
                l[i] = l[i] * al[i] + sum;                          // of the lane's keys
                m[i] = top;
            }
            __syncwarp();
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int i = 0; i < RW; ++i) {
                    const float f = __shfl_sync(0xffffffffu, al[i % RS], i / RS * LK);
#pragma unroll
                    for (int n = 0; n < NV; ++n)
#pragma unroll
                        for (int c = 0; c < VW; ++c) o[i][n][c] *= f;
                }
            }
            auto weigh = [&](auto select) {
#pragma unroll 2
                for (int j = key0; j < key0 + KW; j += 4) {
                    float v[4][NV][VW];
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int n = 0; n < NV; ++n) simt_columns(v[y][n], &sm.v[buf][j + y][n * 128 + lane * VW]);
#pragma unroll
                    for (int i = 0; i < RW; ++i) {
                        const float4 p4 = *reinterpret_cast<const float4*>(&sm.p[row0 + i][j]);
                        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                        for (int y = 0; y < 4; ++y)
#pragma unroll
                            for (int n = 0; n < NV; ++n)
#pragma unroll
                                for (int c = 0; c < VW; ++c) {
                                    const float x = fmaf(p[y], v[y][n][c], o[i][n][c]);
                                    o[i][n][c] = (!decltype(select)::value || !(p[y] < 0.f)) ? x : o[i][n][c];
                                }
                    }
                }
            };
            // cached rows behind the sequence's end are zeros in shared memory; drafted ones that a row does not see are
            // others' and may hold anything
            if (drafted) weigh(std::true_type{}); else weigh(std::false_type{});
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < RS; ++i) {
#pragma unroll
            for (int w = LK / 2; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
            if (kl == 0) {
                sm.m[PARTS == 1 ? 0 : warp][row0 + rl * RS + i] = m[i];
                sm.l[PARTS == 1 ? 0 : warp][row0 + rl * RS + i] = l[i];
            }
        }
        const bool complete = kt0 == 0 && kt1 == kt_all;
        const int slot = portion_slot(blockIdx.x, kt0);
        auto write = [&](int r, const float (&x)[NV][VW], float top, float sum) {
            const int row = r_base + r;
            if (row >= r_all) return;
            const int64_t at = (int64_t)(s.node0 + row / G) * HQ + h * G + row % G;
            const float f = complete ? row_scale(sum) : 1.f;
            float* to = complete ? reinterpret_cast<float*>(a.out) + at * D : a.part_o + ((int64_t)slot * R + r) * D;
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int col = n * 128 + lane * VW;
                if (col >= D) continue;
                if constexpr (VW == 4) *reinterpret_cast<float4*>(to + col) = make_float4(x[n][0] * f, x[n][1] * f, x[n][2] * f, x[n][3] * f);
                else *reinterpret_cast<float2*>(to + col) = make_float2(x[n][0] * f, x[n][1] * f);
            }
            if (lane != 0) return;
            if (complete) {
                a.lse[at] = row_lse(top, sum);
            } else {
                a.part_ml[(int64_t)slot * 2 * R + r] = top;
                a.part_ml[((int64_t)slot * 2 + 1) * R + r] = sum;
            }
        };
        if constexpr (PARTS == 1) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < RW; ++i) write(row0 + i, o[i], sm.m[0][row0 + i], sm.l[0][row0 + i]);
        } else {
            float (*sums)[RW][DP] = reinterpret_cast<float (*)[RW][DP]>(&sm.k[0][0][0]);
            static_assert(sizeof(float) * PARTS * RW * DP <= sizeof(sm.k), "");
            __syncthreads();                    // K is no longer read
#pragma unroll
            for (int i = 0; i < RW; ++i)
#pragma unroll
                for (int n = 0; n < NV; ++n)
#pragma unroll
                    for (int c = 0; c < VW; ++c) sums[warp][i][n * 128 + lane * VW + c] = o[i][n][c];
            __syncthreads();
            for (int r = warp; r < RW; r += 4) {
                float top = neg_inf(), sum = 0.f, x[NV][VW] = {};
#pragma unroll
                for (int w = 0; w < PARTS; ++w) top = fmaxf(top, sm.m[w][r]);
                const float base = top == neg_inf() ? 0.f : top;
#pragma unroll
                for (int w = 0; w < PARTS; ++w) {
                    const float f = exp2f(sm.m[w][r] - base);
                    sum = fmaf(sm.l[w][r], f, sum);
#pragma unroll
                    for (int n = 0; n < NV; ++n)
#pragma unroll
                        for (int c = 0; c < VW; ++c) x[n][c] = fmaf(f, sums[w][r][n * 128 + lane * VW + c], x[n][c]);
                }
                write(r, x, top, sum);
            }
        }
    }
    if (threadIdx.x == 0) note_shared(a, any, part, end, plan);
}

// CTA (x, y) joins 8 / W rows of the x-th segment that several CTAs of the kernel before shared, W warps a row (one takes
// every W-th part): the parts' running maxima and sums are brought to the common maximum, the weighted sums
// added in a fixed order (results do not depend on scheduling), divided, rounded once.  What bounds it is the latency
// of dependent reads, hence all loads of 8 W parts in flight together (one token over 50,432 rows 28.6 -> 26.4 us, with
// the notes found by segment), and W = 8 where a segment may have many parts.
// With few parts a segment one warp a row keeps all CTAs resident at once: 16 sequences of one token 36 us a call with eight,
// 27 with one.
constexpr int kJoinAhead = 8;
template <int DT, int W>
__global__ void __launch_bounds__(256)
attn_join_kernel(const __grid_constant__ AttnArgs a) {
    using St = Store<DT>;
    constexpr int KD = kMaxHeadDim / 128;
    __shared__ float4 part[W > 1 ? W : 1][KD][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G, R = a.split.rows;
    const int r = blockIdx.y * (8 / W) + warp / W, w = warp % W;
    cudaGridDependencySynchronize();
    SharedSegment seg;
    if (!find_shared(a, blockIdx.x, seg)) return;
    const int row = seg.rt * R + r;
    if (row >= seg.rows) return;                            // with W = 8 the whole CTA, else a warp of its own
    const int n = seg.last - seg.first + 1;                 // parts
    auto slot = [&](int p) { return (int64_t)((seg.first + p) * 2 + (p == 0)); };
    auto load = [&](int p, int k) {
        const int col = k * 128 + lane * 4;
        return p < n && col < D ? __ldcg(reinterpret_cast<const float4*>(a.part_o + (slot(p) * R + r) * D + col))
                                : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    // everything that is read for up to 64 parts is on its way before any of it is used
    float m[2], l[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int p = k * 32 + lane;
        m[k] = p < n ? __ldcg(a.part_ml + slot(p) * 2 * R + r) : neg_inf();
        l[k] = p < n ? __ldcg(a.part_ml + (slot(p) * 2 + 1) * R + r) : 0.f;
    }
    float4 v[kJoinAhead][KD];
#pragma unroll
    for (int x = 0; x < kJoinAhead; ++x)
#pragma unroll
        for (int k = 0; k < KD; ++k) v[x][k] = k * 128 < D ? load(w + x * W, k) : make_float4(0.f, 0.f, 0.f, 0.f);
    float top = fmaxf(m[0], m[1]);
    for (int p = 64 + lane; p < n; p += 32) top = fmaxf(top, __ldcg(a.part_ml + slot(p) * 2 * R + r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == neg_inf() ? 0.f : top;
    const float f[2] = {exp2f(m[0] - base), exp2f(m[1] - base)};
    float sum = l[0] * f[0] + l[1] * f[1];
    for (int p = 64 + lane; p < n; p += 32)
        sum = fmaf(__ldcg(a.part_ml + (slot(p) * 2 + 1) * R + r), exp2f(__ldcg(a.part_ml + slot(p) * 2 * R + r) - base), sum);
    sum = warp_sum(sum);                        // every warp of a row has all of it
    float4 acc[KD];
#pragma unroll
    for (int k = 0; k < KD; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float fp, const float4& y, float4& to) {
        to = make_float4(fmaf(fp, y.x, to.x), fmaf(fp, y.y, to.y), fmaf(fp, y.z, to.z), fmaf(fp, y.w, to.w));
    };
#pragma unroll
    for (int x = 0; x < kJoinAhead; ++x) {
        const int p = w + x * W;                // under 64
        const float fp = __shfl_sync(0xffffffffu, x * W < 32 ? f[0] : f[1], p & 31);
        if (p < n) {
#pragma unroll
            for (int k = 0; k < KD; ++k) add(fp, v[x][k], acc[k]);
        }
    }
    for (int p = w + kJoinAhead * W; p < n; p += W) {
        const float fp = exp2f(__ldcg(a.part_ml + slot(p) * 2 * R + r) - base);
#pragma unroll
        for (int k = 0; k < KD; ++k) add(fp, load(p, k), acc[k]);
    }
    if constexpr (W > 1) {
#pragma unroll
        for (int k = 0; k < KD; ++k) part[w][k][lane] = acc[k];
        __syncthreads();
        if (w != 0) return;
        for (int y = 1; y < W; ++y) {
#pragma unroll
            for (int k = 0; k < KD; ++k) add(1.f, part[y][k][lane], acc[k]);
        }
    }
    const float inv = row_scale(sum);
    const int64_t at = (int64_t)(seg.node0 + row / G) * HQ + seg.h * G + row % G;
    auto* out = reinterpret_cast<typename St::T*>(a.out) + at * D;
#pragma unroll
    for (int k = 0; k < KD; ++k) {
        const int col = k * 128 + lane * 4;
        if (col < D) {
            out[col] = St::from(acc[k].x * inv);
            out[col + 1] = St::from(acc[k].y * inv);
            out[col + 2] = St::from(acc[k].z * inv);
            out[col + 3] = St::from(acc[k].w * inv);
        }
    }
    if (lane == 0) a.lse[at] = row_lse(top, sum);
}

template <int R, int DP>
sharpv_status simt_launch(AttnArgs& a, int sms, cudaStream_t stream) {
    auto kern = attn_simt_kernel<R, DP>;
    const size_t smem = sizeof(SimtShared<R, DP>);
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    const int per_sm = min(3, max(1, (int)(220 * 1024 / smem)));
    a.ctas = min(sms * per_sm, kMaxAttnCtas);
    if (launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kSimtThreads), smem, stream, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int DT>
sharpv_status join_launch(const AttnArgs& a, cudaStream_t stream) {
    // rows that any segment can have
    const int64_t all = a.seqs.total_nodes * a.split.group;
    const unsigned rows = (unsigned)(all < a.split.rows ? all : a.split.rows);
    const unsigned x = (unsigned)join_ctas(a);
    const cudaError_t e = many_parts(a) ? launch_dependent(attn_join_kernel<DT, 8>, dim3(x, rows), dim3(256), 0, stream, a)
                                             : launch_dependent(attn_join_kernel<DT, 1>, dim3(x, (rows + 7) / 8), dim3(256), 0, stream, a);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int R>
sharpv_status simt_by_dim(AttnArgs& a, int sms, cudaStream_t stream) {
    if (a.head_dim <= 64) return simt_launch<R, 64>(a, sms, stream);
    if (a.head_dim <= 128) return simt_launch<R, 128>(a, sms, stream);
    return simt_launch<R, 256>(a, sms, stream);
}

// Which kernels a call takes, by type, head_dim and the average query rows of a (sequence, KV head).  Up to 16 rows one
// row tile of the row kernel takes them all and K and V are read once; with more it would read them again for every 16,
// and the tensor cores' kernel is ahead at once (21 rows, 4 KV heads x 128, us: 50,432 rows 36 against 55, the ragged
// batch of 16 34 against 54, 6,272 rows 19 against 23; 56 rows: 37 / 77, 36 / 84, 19 / 34).  It holds up to 128 columns and
// groups of up to 128 heads; beyond, the row kernel takes any number of rows, 16 at a time (4 x 256, 7 query heads each, 6,272
// rows: one token 18 us, 64 nodes 120, a chunk of 509 926).
// The host knows the average alone.  One large sequence among many small ones is taken by the kernel of the small ones: 63
// tokens over 2,000 rows each and a tree of 64 over 50,432 (4 x 128) 399 us in one call, 50 + 58 in two; with 15 tokens,
// where the average is over 16, 77 in one and 22 + 58 in two.
// Over an 8-bit cache the bounds are the same, for tiles have to be widened for the tensor cores: 9 to 16 rows, e4m3, us, row kernel against
// tensor cores' kernel: 50,432 rows 27 / 37, the ragged batch 26 / 35, 6,272 rows 13 / 18, 64 over 2,000 rows each 58 / 77; int8 29 / 36,
// 28 / 34, 14 / 18, 63 / 76.  Up to 8 rows there is a kernel with keys as the products' rows (21 against 27 at 50,432 rows).
// 4 x 256 (7 query heads each, 6,272 rows): one token 20, 64 nodes 108, a chunk of 509 888 (int8 125 and 1,024).  63 tokens over
// 2,000 rows each and a tree of 64 over 50,432: 504 in one call, 41 + 61 in two.
constexpr int64_t kMaxRowsPath = 16;
enum class Path { simt, rows, tc };
struct Choice {
    Path path;
    int rows;               // of a tile
    int places;             // for rows in a partial result
    int max_ctas;           // sizes the workspace
};
Choice choose(sharpv_dtype dtype, int head_dim, int group, int64_t avg_rows) {
    if (dtype == SHARPV_F32) return avg_rows <= 8 ? Choice{Path::simt, 8, 8, kMaxAttnCtas} : Choice{Path::simt, 32, 32, kMaxAttnCtas};
    if (head_dim <= 128 && group <= 128 && avg_rows > kMaxRowsPath) return {Path::tc, tc_rows(group), kTcPlaces, kMaxTcCtas};
    if (q8_dtype_ok(dtype) && head_dim <= 128 && avg_rows <= 8) return {Path::rows, 8, 8, kMaxRowsCtas};
    return {Path::rows, kRowsTileRows, kRowsTileRows, kMaxRowsCtas};
}
int64_t average_rows(int32_t num_seqs, int64_t total_nodes, int64_t group) {
    return num_seqs > 0 ? total_nodes * group / num_seqs : 0;
}

// the parts of the workspace
size_t shared_bytes() { return 256 + align_up(kMaxAttnCtas * sizeof(SharedSegment), 256); }
size_t part_ml_bytes(const Choice& c) { return align_up((size_t)c.max_ctas * 2 * 2 * c.places * 4, 256); }
size_t part_o_bytes(const Choice& c, int32_t head_dim) { return align_up((size_t)c.max_ctas * 2 * c.places * head_dim * 4, 256); }

size_t workspace_bytes(int32_t num_seqs, int64_t total_nodes, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                       sharpv_dtype dtype) {
    if (total_nodes < 0) total_nodes = 0;
    if (num_kv_heads < 1) num_kv_heads = 1;
    if (num_q_heads < 0) num_q_heads = 0;
    if (head_dim < 1) head_dim = 1;
    if (head_dim > kMaxHeadDim) head_dim = kMaxHeadDim;
    const int group = num_q_heads / num_kv_heads;
    const Choice c = choose(dtype, head_dim, group > 0 ? group : 1, average_rows(num_seqs, total_nodes, group));
    return shared_bytes() + part_ml_bytes(c) + part_o_bytes(c, head_dim);
}

// Both entry points, behind the checks of the cache.  eb: bytes of an element of q, of drafted rows and of out.
sharpv_status attend(
    const void* q, int64_t ld_q, const void* draft_k, int64_t ld_draft_k, const void* draft_v, int64_t ld_draft_v,
    int32_t num_q_heads, const void* kv, const sharpv_kv_layout* layout, const uint8_t* scales,
    const sharpv_kv_scales* scales_layout, int64_t eb, int32_t layer, int64_t cache_tokens,
    int32_t num_seqs, const int32_t* seq_begin, const int32_t* seq_len, const int32_t* node_offsets,
    int64_t total_nodes, const uint32_t* tree_mask, int32_t mask_words, float scale, void* out, float* out_lse,
    void* workspace, size_t workspace_size, int32_t* status_word, void* cuda_stream) {
    const int D = layout->head_dim, H = layout->num_kv_heads;
    const int64_t kv_eb = elem_bytes(layout->dtype);
    if (layer < 0 || layer >= layout->num_layers || cache_tokens < 0 || num_seqs < 0 || total_nodes < 0 ||
        num_q_heads < 1 || num_q_heads % H != 0 || (draft_k == nullptr) != (draft_v == nullptr) ||
        mask_words < 0 || !(scale > 0.f) || !(scale < __builtin_huge_valf()))
        return SHARPV_ERR_INVALID_ARG;
    if (D > kMaxHeadDim || cache_tokens >= (int64_t)1 << 31 || total_nodes * num_q_heads >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
    if (num_seqs == 0 || total_nodes == 0) return SHARPV_OK;
    if (!q || !seq_begin || !seq_len || !node_offsets || !out || !out_lse || (tree_mask && mask_words < 1) ||
        ld_q < (int64_t)num_q_heads * D || (draft_k && (ld_draft_k < (int64_t)H * D || ld_draft_v < (int64_t)H * D)))
        return SHARPV_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || (ld_q * eb) % 16 ||
        (draft_k && (!aligned16(draft_k) || !aligned16(draft_v) || (ld_draft_k * eb) % 16 || (ld_draft_v * eb) % 16)))
        return SHARPV_ERR_UNSUPPORTED;
    if (workspace_size < workspace_bytes(num_seqs, total_nodes, num_q_heads, H, D, layout->dtype)) return SHARPV_ERR_WORKSPACE;
    if (!workspace) return SHARPV_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return SHARPV_ERR_UNSUPPORTED;

    AttnArgs a = {};
    a.q = (const char*)q;
    a.q_node = ld_q * eb;
    a.cache_k = (const char*)kv + (int64_t)layer * layout->stride_layer * kv_eb;
    a.cache_v = a.cache_k + layout->stride_kv * kv_eb;
    a.kv_head = layout->stride_head * kv_eb;
    a.kv_token = layout->stride_token * kv_eb;
    a.draft_k = (const char*)draft_k;
    a.draft_v = (const char*)draft_v;
    a.dk_node = ld_draft_k * eb;
    a.dv_node = ld_draft_v * eb;
    a.mask = tree_mask;
    a.mask_words = mask_words;
    a.head_dim = D;
    a.scale_log2 = scale * kLog2e;
    a.out = out;
    a.lse = out_lse;
    a.seqs = SeqTables{seq_begin, seq_len, node_offsets, num_seqs, cache_tokens, total_nodes};
    const int group = num_q_heads / H;
    const Choice ch = choose(layout->dtype, D, group, average_rows(num_seqs, total_nodes, group));
    a.split = Split{ch.rows, ch.path == Path::tc ? kTcTileKeys : (ch.path == Path::rows ? kRowsTileKeys : kSimtKeys), group, H,
                    draft_k != nullptr};
    const int64_t segments = (total_nodes * group / ch.rows + num_seqs) * H;     // rounding a sequence's last tile up adds one at most
    a.max_segments = (int)(segments < kMaxAttnCtas ? segments : kMaxAttnCtas);
    char* ws = (char*)workspace;
    a.head = (SharedHead*)ws;
    a.shared = (SharedSegment*)(ws + 256);
    a.part_ml = (float*)(ws + shared_bytes());
    a.part_o = (float*)(ws + shared_bytes() + part_ml_bytes(ch));
    a.status_word = status_word;
    if (scales) {
        a.k_scales = scales + layer * scales_layout->stride_layer;
        a.v_scales = a.k_scales + scales_layout->stride_kv;
        a.scale_head = scales_layout->stride_head;
        a.scale_shift = log2_of(scales_layout->block_tokens);
        // units that a sequence can have: key tiles times row tiles times heads
        const int64_t units = ((cache_tokens + total_nodes) / a.split.keys + 3) * (total_nodes * group / ch.rows + 1) * H;
        a.warp_plans = num_seqs <= 32 && units < 1 << 20;
    }
    int sms = 0;
    const sharpv_status ss = current_sms(sms);
    if (ss != SHARPV_OK) return ss;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (ch.path == Path::tc) return attn_tc_launch(a, layout->dtype, sms, stream);
    if (ch.path == Path::rows) {
        const sharpv_status st = scales ? attn_rows_q8_launch(a, layout->dtype, sms, stream) : attn_rows_launch(a, sms, stream);
        return st == SHARPV_OK ? join_launch<SHARPV_BF16>(a, stream) : st;
    }
    const sharpv_status st = ch.rows == 8 ? simt_by_dim<8>(a, sms, stream) : simt_by_dim<32>(a, sms, stream);
    return st == SHARPV_OK ? join_launch<SHARPV_F32>(a, stream) : st;
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" size_t sharpv_tree_attention_workspace_bytes(int32_t num_seqs, int64_t total_nodes, int32_t num_q_heads,
                                                        int32_t num_kv_heads, int32_t head_dim, sharpv_dtype dtype) {
    return workspace_bytes(num_seqs, total_nodes, num_q_heads, num_kv_heads, head_dim, q8_dtype_ok(dtype) ? SHARPV_BF16 : dtype);
}

extern "C" size_t sharpv_tree_attention_q8_workspace_bytes(int32_t num_seqs, int64_t total_nodes, int32_t num_q_heads,
                                                           int32_t num_kv_heads, int32_t head_dim) {
    return workspace_bytes(num_seqs, total_nodes, num_q_heads, num_kv_heads, head_dim, SHARPV_E4M3);
}

extern "C" sharpv_status sharpv_tree_attention(
    const void* q, int64_t ld_q, const void* draft_k, int64_t ld_draft_k, const void* draft_v, int64_t ld_draft_v,
    int32_t num_q_heads, const void* kv, const sharpv_kv_layout* layout, int32_t layer, int64_t cache_tokens,
    int32_t num_seqs, const int32_t* seq_begin, const int32_t* seq_len, const int32_t* node_offsets,
    int64_t total_nodes, const uint32_t* tree_mask, int32_t mask_words, float scale, void* out, float* out_lse,
    void* workspace, size_t workspace_bytes, int32_t* status_word, void* cuda_stream) {
    const sharpv_status ls = kv_layout_status(kv, layout, true);
    if (ls != SHARPV_OK) return ls;
    return attend(q, ld_q, draft_k, ld_draft_k, draft_v, ld_draft_v, num_q_heads, kv, layout, nullptr, nullptr,
                  elem_bytes(layout->dtype), layer, cache_tokens, num_seqs, seq_begin, seq_len, node_offsets, total_nodes, tree_mask,
                  mask_words, scale, out, out_lse, workspace, workspace_bytes, status_word, cuda_stream);
}

extern "C" sharpv_status sharpv_tree_attention_q8(
    const void* q, int64_t ld_q, const void* draft_k, int64_t ld_draft_k, const void* draft_v, int64_t ld_draft_v,
    int32_t num_q_heads, const void* kv, const sharpv_kv_layout* layout, const uint8_t* scales,
    const sharpv_kv_scales* scales_layout, int32_t layer, int64_t cache_tokens, int32_t num_seqs, const int32_t* seq_begin,
    const int32_t* seq_len, const int32_t* node_offsets, int64_t total_nodes, const uint32_t* tree_mask, int32_t mask_words,
    float scale, void* out, float* out_lse, void* workspace, size_t workspace_bytes, int32_t* status_word, void* cuda_stream) {
    sharpv_status st = kv_layout_status_if(kv, layout, q8_dtype_ok);
    if (st != SHARPV_OK) return st;
    st = kv_scales_status(scales, scales_layout);
    if (st != SHARPV_OK) return st;
    return attend(q, ld_q, draft_k, ld_draft_k, draft_v, ld_draft_v, num_q_heads, kv, layout, scales, scales_layout,
                  elem_bytes(SHARPV_BF16), layer, cache_tokens, num_seqs, seq_begin, seq_len, node_offsets, total_nodes, tree_mask,
                  mask_words, scale, out, out_lse, workspace, workspace_bytes, status_word, cuda_stream);
}
