// The attention weight that every cached token collects (sharpv_attention_mass).
//
//   out[p] = decay mass[p] + sum_r w_r exp(scale q_r . k_p - lse_r)   over the rows r = (node, query head)
//
// The softmax's own sum is known (lse), so one pass over the keys suffices and every key is independent of the
// others: keys are spread over CTAs, a key's sum over the rows of one KV head stays in a register, and the KV heads'
// sums are added in a second, small kernel in the order of the heads (no atomics: the order is fixed).
//
// Kernels (fp32 caches; bf16 ones take those of attention_mass_rows.cu and attention_mass_tc.cu):
//   mass_simt_kernel      (sequence, KV head, 32 keys) a step, lane = key, on the fp32 units
//   mass_join_kernel      (dependent launch) adds the heads' sums and what the rows collected before
#include "attention_mass.cuh"

namespace sharpv {
namespace {

constexpr int kMassThreads = 128;
constexpr int kMassKeys = 32;
constexpr int kNodeWindow = 512;        // nodes whose weights are looked at together
constexpr int kMaxMassHeadDim = 256;
// bf16: average query rows of a (sequence, KV head) up to which the row kernel is taken.  It spreads keys finer (32 a unit
// against 128), the tensor cores' kernel weighs more rows at once; 56 rows, 4 KV heads x 128, us: 50,432 rows 17.1 against
// 17.8, 6,272 rows 7.7 / 9.4, the ragged batch of 16 21.4 / 18.7; 84 rows: 19.3 / 18.1, 8.5 / 9.8, 23.4 / 19.4.  As with the
// attention, an average over unlike sequences finds the kernel of the small ones: 63 single nodes over 2,000 rows each and 64
// nodes over 50,432 121 us in one call, 30 + 32 in two; fp32 (6,272 rows in place of 50,432) 993, 89 + 106 in two.
constexpr int64_t kMaxRowsPath = 64;

// The nodes [w0, w0 + kNodeWindow) of a sequence that count, as a list in ascending order.  Returns their number.
template <int NT>
__device__ __forceinline__ int active_nodes(const MassArgs& a, const SeqInfo& s, int w0, int* list, int* scan) {
    const int n = min(kNodeWindow, s.nodes - w0);
    int count = 0;
    for (int x0 = 0; x0 < n; x0 += NT) {
        const int x = x0 + threadIdx.x;
        const int on = x < n && (a.weight == nullptr || __ldg(a.weight + s.node0 + w0 + x) != 0.f);
        int total;
        const int at = block_exclusive_scan<NT>(on, scan, total);
        if (on) list[count + at] = w0 + x;
        count += total;
    }
    __syncthreads();
    return count;
}

template <int R, int DP>
struct MassShared {
    float k[2][kMassKeys][DP + 4];
    float q[R][DP];
    float lse2[R], weight[R];
    float sum[kMassThreads / 32][kMassKeys];
    int list[kNodeWindow], scan[kMassThreads / 32 + 1];
    PlanScratch<kMassThreads> plan;
};

// What bounds it is the latency of a tile's products (few warps an SM).  Measured: 1 node x 7 heads over 1,600 rows of 2 x 64
// 7.9 us, over 50,432 of 4 x 128 43 us (2.4 TB/s); 64 nodes over 6,272 of 4 x 128 107 us (27 TFLOP/s).
template <int R, int DP>
__global__ void __launch_bounds__(kMassThreads)
mass_simt_kernel(const __grid_constant__ MassArgs a) {
    extern __shared__ __align__(16) char smem_raw[];
    auto& sm = *reinterpret_cast<MassShared<R, DP>*>(smem_raw);
    constexpr int RW = R / 4, VPR = DP / 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int D = a.head_dim, G = a.split.group, HQ = a.split.heads * G;
    cudaGridDependencySynchronize();
    int64_t first, end;
    const PlanStart plan = plan_cta<kMassThreads>(a.seqs, a.split, blockIdx.x, a.ctas, sm.plan, first, end, a.status_word);
    Walk walk(plan, first, end);
    Portion part;
    while (walk.next(a.seqs, a.split, part)) {
        const SeqInfo& s = part.s;
        const int h = part.h, kt0 = part.kt0, kt1 = part.kt1;
        if (s.len == 0) continue;
        auto load_keys = [&](int kt, int buf) {
            const char* src = a.cache_k + (int64_t)h * a.kv_head + (s.begin + (int64_t)kt * kMassKeys) * a.kv_token;
            const int valid = s.len - kt * kMassKeys;
            for (int x = threadIdx.x; x < kMassKeys * VPR; x += kMassThreads) {
                const int j = x / VPR, c = x % VPR * 4;
                const bool there = j < valid && c < D;
                cp_async16(&sm.k[buf][j][c], there ? src + (int64_t)j * a.kv_token + c * 4 : src, there);
            }
            cp_async_commit();
        };
        __syncthreads();
        load_keys(kt0, 0);
        for (int kt = kt0; kt < kt1; ++kt) {
            const int buf = (kt - kt0) & 1;
            if (kt + 1 < kt1) {
                load_keys(kt + 1, buf ^ 1);
                cp_async_wait<1>();
            } else {
                cp_async_wait<0>();
            }
            __syncthreads();
            float sum = 0.f;
            for (int w0 = 0; w0 < s.nodes; w0 += kNodeWindow) {
                const bool one_chunk = s.nodes <= kNodeWindow && s.nodes * G <= R;      // rows stay in place from tile to tile
                int rows = 0;
                if (!one_chunk || kt == kt0) rows = active_nodes<kMassThreads>(a, s, w0, sm.list, sm.scan) * G;
                for (int r0 = 0; r0 < rows || (one_chunk && r0 == 0); r0 += R) {        // rows past the end have weight 0
                    if (!one_chunk || kt == kt0) {
                        __syncthreads();
                        for (int x = threadIdx.x; x < R * VPR; x += kMassThreads) {
                            const int r = x / VPR, c = x % VPR * 4, row = r0 + r;
                            uint4 w = make_uint4(0, 0, 0, 0);
                            if (row < rows && c < D)
                                w = ld_cached(a.q + (int64_t)(s.node0 + sm.list[row / G]) * a.q_node + ((int64_t)(h * G + row % G) * D + c) * 4);
                            *reinterpret_cast<uint4*>(&sm.q[r][c]) = w;
                        }
                        if (threadIdx.x < R) {
                            const int row = r0 + threadIdx.x;
                            float wt = 0.f, ls = 0.f;
                            if (row < rows) {
                                const int64_t node = s.node0 + sm.list[row / G];
                                ls = __ldg(a.lse + node * HQ + h * G + row % G);
                                wt = ls == neg_inf() ? 0.f : (a.weight ? __ldg(a.weight + node) : 1.f);
                            }
                            sm.lse2[threadIdx.x] = ls * kLog2e;
                            sm.weight[threadIdx.x] = wt;
                        }
                        __syncthreads();
                    }
                    float acc[RW];
#pragma unroll
                    for (int i = 0; i < RW; ++i) acc[i] = 0.f;
                    for (int c = 0; c < D; c += 4) {
                        const float4 k4 = *reinterpret_cast<const float4*>(&sm.k[buf][lane][c]);
#pragma unroll
                        for (int i = 0; i < RW; ++i) {
                            const float4 q4 = *reinterpret_cast<const float4*>(&sm.q[warp * RW + i][c]);
                            acc[i] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, acc[i]))));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < RW; ++i) {
                        const float wt = sm.weight[warp * RW + i];
                        const float p = exp2f(fmaf(acc[i], a.scale_log2, -sm.lse2[warp * RW + i]));
                        if (wt != 0.f) sum = fmaf(wt, p, sum);
                    }
                }
            }
            sm.sum[warp][lane] = sum;
            __syncthreads();
            if (warp == 0 && kt * kMassKeys + lane < s.len) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < kMassThreads / 32; ++w) t += sm.sum[w][lane];
                a.part[(int64_t)h * a.seqs.cache_tokens + s.begin + kt * kMassKeys + lane] = t;
            }
            __syncthreads();
        }
    }
}

// blockIdx.y walks the sequences, blockIdx.x the rows of one.  Its time (one launch, a read of the heads' sums) is in the
// figures above.
__global__ void __launch_bounds__(256)
mass_join_kernel(const __grid_constant__ MassArgs a) {
    cudaGridDependencySynchronize();
    bool bad = false;
    for (int b = blockIdx.y; b < a.seqs.num_seqs; b += gridDim.y) {
        const SeqInfo s = load_seq(a.seqs, b, bad);
        for (int i = blockIdx.x * 256 + threadIdx.x; i < s.len; i += gridDim.x * 256) {
            const int64_t p = s.begin + i;
            float t = 0.f;
            if (s.nodes > 0)
                for (int h = 0; h < a.split.heads; ++h) t += __ldcg(a.part + (int64_t)h * a.seqs.cache_tokens + p);
            a.out[p] = a.mass && a.decay != 0.f ? fmaf(a.decay, a.mass[p], t) : t;
        }
    }
}

template <int R, int DP>
sharpv_status mass_simt_launch(MassArgs a, int sms, cudaStream_t stream) {
    auto kern = mass_simt_kernel<R, DP>;
    const size_t smem = sizeof(MassShared<R, DP>);
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    a.ctas = sms * (smem * 4 <= 220 * 1024 ? 4 : 2);
    return launch_dependent(kern, dim3((unsigned)a.ctas), dim3(kMassThreads), smem, stream, a) == cudaSuccess
               ? SHARPV_OK : (cudaGetLastError(), SHARPV_ERR_CUDA);
}

template <int R>
sharpv_status mass_by_dim(const MassArgs& a, int sms, cudaStream_t stream) {
    if (a.head_dim <= 64) return mass_simt_launch<R, 64>(a, sms, stream);
    if (a.head_dim <= 128) return mass_simt_launch<R, 128>(a, sms, stream);
    return mass_simt_launch<R, 256>(a, sms, stream);
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" size_t sharpv_attention_mass_workspace_bytes(int64_t cache_tokens, int32_t num_kv_heads, sharpv_dtype dtype) {
    if (dtype == SHARPV_BF16) return 0;
    if (cache_tokens < 1) cache_tokens = 1;
    if (num_kv_heads < 1) num_kv_heads = 1;
    return align_up((size_t)cache_tokens * num_kv_heads * 4, 256);
}

extern "C" sharpv_status sharpv_attention_mass(
    const void* q, int64_t ld_q, const float* lse, const float* node_weight, int32_t num_q_heads, const void* kv,
    const sharpv_kv_layout* layout, int32_t layer, int64_t cache_tokens, int32_t num_seqs, const int32_t* seq_begin,
    const int32_t* seq_len, const int32_t* node_offsets, int64_t total_nodes, float scale, float decay,
    const float* mass, float* out_mass, void* workspace, size_t workspace_bytes, int32_t* status_word,
    void* cuda_stream) {
    const sharpv_status ls = kv_layout_status(kv, layout, true);
    if (ls != SHARPV_OK) return ls;
    const int D = layout->head_dim, H = layout->num_kv_heads;
    const int64_t eb = elem_bytes(layout->dtype);
    if (layer < 0 || layer >= layout->num_layers || cache_tokens < 0 || num_seqs < 0 || total_nodes < 0 ||
        num_q_heads < 1 || num_q_heads % H != 0 || !(scale > 0.f) || !(scale < __builtin_huge_valf()) ||
        !(decay >= 0.f) || !(decay < __builtin_huge_valf()))
        return SHARPV_ERR_INVALID_ARG;
    if (D > kMaxMassHeadDim || cache_tokens >= (int64_t)1 << 31 || total_nodes * num_q_heads >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
    if (num_seqs == 0 || cache_tokens == 0) return SHARPV_OK;
    if (!seq_begin || !seq_len || !node_offsets || !out_mass || (total_nodes > 0 && (!q || !lse)) ||
        ld_q < (int64_t)num_q_heads * D)
        return SHARPV_ERR_INVALID_ARG;
    if (mass && mass != out_mass && mass < out_mass + cache_tokens && out_mass < mass + cache_tokens) return SHARPV_ERR_INVALID_ARG;
    if (!aligned16(q) || (ld_q * eb) % 16) return SHARPV_ERR_UNSUPPORTED;
    const size_t need = sharpv_attention_mass_workspace_bytes(cache_tokens, H, layout->dtype);
    if (workspace_bytes < need) return SHARPV_ERR_WORKSPACE;
    if (need > 0 && !workspace) return SHARPV_ERR_INVALID_ARG;
    if (need > 0 && reinterpret_cast<uintptr_t>(workspace) % 256) return SHARPV_ERR_UNSUPPORTED;

    MassArgs a = {};
    a.q = (const char*)q;
    a.q_node = ld_q * eb;
    a.lse = lse;
    a.weight = node_weight;
    a.cache_k = (const char*)kv + (int64_t)layer * layout->stride_layer * eb;
    a.kv_head = layout->stride_head * eb;
    a.kv_token = layout->stride_token * eb;
    a.head_dim = D;
    a.scale_log2 = scale * kLog2e;
    a.decay = decay;
    a.mass = mass;
    a.out = out_mass;
    a.part = (float*)workspace;
    const int group = num_q_heads / H;
    a.seqs = SeqTables{seq_begin, seq_len, node_offsets, num_seqs, cache_tokens, total_nodes};
    a.split = Split{1 << 30, kMassKeys, group, H, 0};
    a.status_word = status_word;
    int sms = 0;
    sharpv_status st = current_sms(sms);
    if (st != SHARPV_OK) return st;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int64_t avg = total_nodes * group / num_seqs;     // query rows of a (sequence, KV head)
    if (layout->dtype == SHARPV_BF16) {
        const int64_t most = (int64_t)1 << 40;              // what a tensor map's strides can say
        if (a.kv_token >= most || a.kv_head >= most) return SHARPV_ERR_UNSUPPORTED;
        return avg > kMaxRowsPath && D <= 128 ? mass_tc_launch(a, sms, stream) : mass_rows_launch(a, sms, stream);
    }
    st = avg <= 8 ? mass_by_dim<8>(a, sms, stream)
                                             : mass_by_dim<32>(a, sms, stream);
    if (st != SHARPV_OK) return st;
    const int y = num_seqs < 1024 ? num_seqs : 1024;
    int64_t x = (cache_tokens / num_seqs + 255) / 256;
    const int64_t most = 8 * sms / y > 1 ? 8 * sms / y : 1;
    if (x > most) x = most;
    if (x < 1) x = 1;
    if (launch_dependent(mass_join_kernel, dim3((unsigned)x, (unsigned)y), dim3(256), 0, stream, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}
