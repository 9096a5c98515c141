// Arguments that the kernels of the attention over a cache share.
#pragma once

#include <cuda.h>

#include "decode_common.cuh"

namespace sharpv {

constexpr int kMaxAttnCtas = 3 * 160;       // resident CTAs a call may use; sizes the workspace
constexpr int kMaxRowsCtas = 160;           // of them the row kernel's
constexpr int kMaxHeadDim = 256;

struct AttnArgs {
    const char* q;              // [nodes, heads * group, D]; byte strides between nodes
    int64_t q_node;
    const char* cache_k;        // the layer's K and V blocks
    const char* cache_v;
    int64_t kv_head, kv_token;  // bytes
    const char* draft_k;        // [nodes, heads, D], or null
    const char* draft_v;
    int64_t dk_node, dv_node;   // bytes
    const uint32_t* mask;       // [nodes, mask_words]: bit j of a row = the node sees node j of its sequence; null: j <= i
    int mask_words;
    int head_dim;               // elements
    float scale_log2;           // scale * log2(e): scores are kept in units of log 2
    void* out;                  // [nodes, heads * group, D]
    float* lse;                 // [nodes, heads * group]
    SeqTables seqs;
    Split split;
    // workspace
    SharedHead* head;
    SharedSegment* shared;      // [ctas]
    float* part_ml;             // [slots][2][rows]: running maximum and sum of each row
    float* part_o;              // [slots][rows][D]: weighted sums, not yet divided
    int ctas;
    int max_segments;           // that there can be
    int32_t* status_word;
    // caches in 8 bits: the layer's scales of K and V, bytes between heads, log2 of a block's rows
    const uint8_t* k_scales;
    const uint8_t* v_scales;
    int64_t scale_head;
    int scale_shift;
    int warp_plans;             // few enough sequences and units for the loading warp to plan on its own
};

// Tensor maps of a call (bf16): boxes of 64 columns and a key tile's rows.  draft_* repeat cache_* where there are none.
struct AttnMaps {
    CUtensorMap cache_k, cache_v, draft_k, draft_v, query;      // query: boxes of whole nodes' rows of one KV head (tcgen05 kernel)
};
// box_bytes: a cache in 8 bits, boxes of so many bytes of cache_k and cache_v
sharpv_status encode_attn_maps(const AttnArgs& a, int box_rows, AttnMaps& maps, int box_bytes = 0);

// Few query rows, bf16: a.split has kRowsTileRows rows and kRowsTileKeys keys a tile.  Sets a.ctas to what it launches.
constexpr int kRowsTileRows = 16, kRowsTileKeys = 64;
sharpv_status attn_rows_launch(AttnArgs& a, int sms, cudaStream_t stream);
// the same for a cache in 8 bits; also with tiles of 8 rows, head_dim of at most 128
sharpv_status attn_rows_q8_launch(AttnArgs& a, sharpv_dtype code, int sms, cudaStream_t stream);

// Many query rows, bf16 or codes with scales, head_dim and group of at most 128: a.split has tc_rows(group) rows and kTcTileKeys keys a tile.
// A partial result has room for kTcPlaces rows.  Joins the parts as well.
constexpr int kTcPlaces = 256, kTcTileKeys = 128, kMaxTcCtas = 160;
inline int tc_rows(int group) { return 2 * (128 / group * group); }
sharpv_status attn_tc_launch(AttnArgs& a, sharpv_dtype dtype, int sms, cudaStream_t stream);

// Which keys of the 32 from key0 on node `i` of a sequence sees, as bits (drafted tokens).
__device__ __forceinline__ uint32_t draft_sees(const AttnArgs& a, const SeqInfo& s, int i, int key0) {
    const int left = s.nodes - key0;
    if (left <= 0) return 0u;
    const uint32_t there = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
    uint32_t sees;
    if (a.mask == nullptr) {
        const int upto = i - key0;              // keys key0 .. i
        sees = upto < 0 ? 0u : (upto >= 31 ? 0xffffffffu : (2u << upto) - 1u);
    } else {
        sees = key0 / 32 < a.mask_words ? __ldg(a.mask + ((int64_t)s.node0 + i) * a.mask_words + key0 / 32) : 0u;
    }
    return sees & there;
}

// What a CTA says of the segment that it shares with the CTAs behind it, by one thread: `last` is its last portion (the only
// one that can start a segment without ending it), `any` whether it has one.
__device__ __forceinline__ void note_shared(const AttnArgs& a, bool any, const Portion& last, int64_t end, const PlanStart& plan) {
    const bool pieces = plan.segments >= 0;
    if (blockIdx.x == 0) *a.head = SharedHead{pieces, plan.segments};
    SharedSegment seg = {0, 0, 0, 0, 0, -1};
    if (any && last.kt0 == 0 && last.kt1 < last.kt_all)
        seg = SharedSegment{last.s.node0, last.s.nodes * a.split.group, last.h, last.rt, (int)blockIdx.x,
                            pieces ? plan.last : Deal(plan.units, a.ctas).owner(end + (last.kt_all - last.kt1) - 1)};
    if (!pieces) a.shared[blockIdx.x] = seg;
    else if (plan.ordinal >= 0) a.shared[plan.ordinal] = seg;
}

// Whether segments have many parts each.  Then there are few shared segments, and a joining kernel has a CTA row for
// each, found among the CTAs' notes; else one for every CTA of the kernel before, most of which have something to join.
__host__ __device__ inline bool many_parts(const AttnArgs& a) { return a.ctas >= 8 * a.max_segments; }
__host__ __device__ inline int join_ctas(const AttnArgs& a) { return many_parts(a) ? a.max_segments : a.ctas; }

// The x-th shared segment; false if there is none.  By a whole warp.
__device__ __forceinline__ bool find_shared(const AttnArgs& a, int x, SharedSegment& seg) {
    const int2 head = __ldcg(reinterpret_cast<const int2*>(a.head));
    seg = a.shared[x];
    if (head.x) return x < head.y && seg.last >= 0;
    if (!many_parts(a)) return seg.last >= 0;
    const int lane = threadIdx.x & 31;
    constexpr int N = (kMaxAttnCtas + 31) / 32;
    int last[N];
#pragma unroll
    for (int k = 0; k < N; ++k) last[k] = k * 32 + lane < a.ctas ? __ldcg(&a.shared[k * 32 + lane].last) : -1;
    int found = -1, count = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t valid = __ballot_sync(0xffffffffu, last[k] >= 0);
        const uint32_t mine = __ballot_sync(0xffffffffu, last[k] >= 0 && count + __popc(valid & ((1u << lane) - 1u)) == x);
        if (mine) found = k * 32 + __ffs(mine) - 1;
        count += __popc(valid);
    }
    if (found >= 0) seg = a.shared[found];
    return found >= 0;
}

// out and lse of one row element from its weighted sum, running maximum (log 2 units) and sum
__device__ __forceinline__ float row_scale(float l) { return l == 0.f ? 0.f : 1.0f / l; }
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? neg_inf() : (m + log2f(l)) * kLn2; }

}  // namespace sharpv
