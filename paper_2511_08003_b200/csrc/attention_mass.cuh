// Arguments of the kernels that collect attention weight.
#pragma once

#include "decode_common.cuh"

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

// bf16 caches: one kernel that writes a.out
sharpv_status mass_rows_launch(MassArgs& a, int sms, cudaStream_t stream);

}  // namespace sharpv
