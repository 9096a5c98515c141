// Arguments of the kernels that collect attention weight.
#pragma once

#include "decode_common.cuh"
#include "tma.cuh"

namespace sharpv {

struct MassArgs {
    const char* q;
    int64_t q_node;
    const float* lse;           // [nodes, heads * group]
    const float* weight;        // [nodes] or null
    const char* cache_k;
    int64_t kv_head, kv_token;
    int head_dim;
    float scale_log2, decay;
    const float* mass;          // null: nothing collected yet
    float* out;
    float* part;                // [heads][cache_tokens] (fp32 caches)
    SeqTables seqs;
    Split split;                // rows: all of a sequence's in one tile
    int ctas;
    int32_t* status_word;
};

// bf16 kernels: a query row's log-sum-exp in units of log 2.  Places without a row and rows that saw nothing have kNoRow and
// are left out by selection: their product with a key that is not finite need not be 0.
constexpr float kNoRow = 3.402823466e38f;
__device__ __forceinline__ float lse_log2(float lse) { return lse == neg_inf() ? kNoRow : lse * kLog2e; }
__device__ __forceinline__ float add_weight(float sum, float weight, float product, float scale_log2, float lse2) {
    const float x = fmaf(weight, ex2(fmaf(product, scale_log2, -lse2)), sum);
    return lse2 != kNoRow ? x : sum;
}

// units in their order; all of a portion belong to one sequence
struct KeyWalk {
    int64_t u, end, before;
    SeqInfo s;
    int b, kt0, kt1;
    __device__ __forceinline__ KeyWalk(const PlanStart& p, int64_t first, int64_t last)
        : u(first), end(last), before(p.before), s(p.s), b(p.b) {}
    __device__ __forceinline__ bool next(const SeqTables& t, const KeySplit& sp) {
        if (u >= end) return false;
        for (;;) {
            const int64_t mine = sp.units(s);
            if (u - before < mine) break;
            before += mine;
            bool bad = false;
            s = load_seq(t, ++b, bad);
        }
        kt0 = (int)(u - before);
        kt1 = (int)min(sp.units(s), kt0 + (end - u));
        u += kt1 - kt0;
        return true;
    }
};

// bf16 caches: kernels that write a.out.  Few query rows a (sequence, KV head), any head_dim; many of them, head_dim of at
// most 128.
sharpv_status mass_rows_launch(MassArgs& a, int sms, cudaStream_t stream);
sharpv_status mass_tc_launch(MassArgs& a, int sms, cudaStream_t stream);

}  // namespace sharpv
