// K/V rows into a cache whose sequences have room to grow (sharpv_kv_append): for every plane the rows src_pos[j] of
// sequence b go to dst_begin[b] + (j - src_seq_offsets[b]), bit for bit.
//
// The copy is organised as the out-of-place compaction is: short-lived CTAs at full thread occupancy, one (row
// tile, plane) each, 128-bit loads all issued before the first store.  A tile's source and destination rows are looked
// up once by as many threads as it has rows, so the search in the offset table is not repeated per vector.
//
// HBM bounds it: 37,712 rows of 224 planes x 256 bytes in 650 to 700 us (0.96 to 1.03 of a plain copy's rate); 43 rows 4.1 us.
#include "decode_common.cuh"

namespace sharpv {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendUnroll = 4;
constexpr int kAppendCtasPerSm = 8;

struct AppendArgs {
    const char* src;
    char* dst;
    int64_t src_layer, src_kv, src_head, src_token, dst_layer, dst_kv, dst_head, dst_token;    // bytes
    int64_t src_tokens, dst_tokens;
    int num_kv_heads, layer_begin, row_vecs, tile_rows;
    const int32_t* src_pos;
    const int32_t* offsets;
    const int32_t* dst_begin;
    int num_seqs;
    int64_t capacity;
    int32_t* status_word;
};

__global__ void __launch_bounds__(kAppendThreads, kAppendCtasPerSm)
kv_append_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ int from[kAppendThreads * kAppendUnroll], to[kAppendThreads * kAppendUnroll];
    const int plane = blockIdx.y;
    const int h = plane % a.num_kv_heads, kv = (plane / a.num_kv_heads) & 1, li = plane / (2 * a.num_kv_heads);
    cudaGridDependencySynchronize();
    const int64_t all = __ldg(a.offsets + a.num_seqs);
    const int64_t n = min(max(all, (int64_t)0), a.capacity);
    const bool first = blockIdx.x == 0 && plane == 0 && threadIdx.x == 0;
    if (first && all > a.capacity) report(a.status_word, SHARPV_ERR_CAPACITY);
    const char* s = a.src + (a.layer_begin + li) * a.src_layer + kv * a.src_kv + h * a.src_head;
    char* o = a.dst + (a.layer_begin + li) * a.dst_layer + kv * a.dst_kv + h * a.dst_head;
    for (int64_t row0 = (int64_t)blockIdx.x * a.tile_rows; row0 < n; row0 += (int64_t)gridDim.x * a.tile_rows) {
        __syncthreads();
        for (int r = threadIdx.x; r < a.tile_rows && row0 + r < n; r += kAppendThreads) {
            const int64_t j = row0 + r;
            const int b = upper_segment(a.offsets, a.num_seqs, (int)j);
            const int64_t f = __ldg(a.src_pos + j);
            const int64_t t = (int64_t)__ldg(a.dst_begin + b) + (j - __ldg(a.offsets + b));
            const bool ok = f >= 0 && f < a.src_tokens && t >= 0 && t < a.dst_tokens;
            if (!ok && plane == 0) report(a.status_word, SHARPV_ERR_BOUNDS);
            from[r] = ok ? (int)f : -1;
            to[r] = (int)t;
        }
        __syncthreads();
        uint4 v[kAppendUnroll];
        unsigned moved = 0;
#pragma unroll
        for (int u = 0; u < kAppendUnroll; ++u) {
            const int q = threadIdx.x + u * kAppendThreads;
            const int rr = q / a.row_vecs;
            if (rr < a.tile_rows && row0 + rr < n && from[rr] >= 0) {
                v[u] = ld_stream(s + from[rr] * a.src_token + (int64_t)(q - rr * a.row_vecs) * 16);
                moved |= 1u << u;
            }
        }
#pragma unroll
        for (int u = 0; u < kAppendUnroll; ++u) {
            const int q = threadIdx.x + u * kAppendThreads;
            const int rr = q / a.row_vecs;
            if (moved >> u & 1) st_stream(o + to[rr] * a.dst_token + (int64_t)(q - rr * a.row_vecs) * 16, v[u]);
        }
    }
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" sharpv_status sharpv_kv_append(
    const void* kv_src, const sharpv_kv_layout* src_layout, int64_t src_tokens, void* kv_dst,
    const sharpv_kv_layout* dst_layout, int64_t dst_tokens, int32_t layer_begin, int32_t layer_end,
    const int32_t* src_pos, const int32_t* src_seq_offsets, const int32_t* dst_begin, int32_t num_seqs,
    int64_t capacity, int32_t* status_word, void* cuda_stream) {
    sharpv_status st = kv_layout_status(kv_src, src_layout, false);
    if (st != SHARPV_OK) return st;
    st = kv_layout_status(kv_dst, dst_layout, false);
    if (st != SHARPV_OK) return st;
    if (src_layout->dtype != dst_layout->dtype || src_layout->head_dim != dst_layout->head_dim ||
        src_layout->num_kv_heads != dst_layout->num_kv_heads || src_layout->num_layers != dst_layout->num_layers ||
        layer_begin < 0 || layer_end > src_layout->num_layers || layer_begin > layer_end || capacity < 0 ||
        num_seqs < 0 || src_tokens < 0 || dst_tokens < 0)
        return SHARPV_ERR_INVALID_ARG;
    if (capacity >= (int64_t)1 << 31 || src_tokens >= (int64_t)1 << 31 || dst_tokens >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
    const int planes = (layer_end - layer_begin) * 2 * src_layout->num_kv_heads;
    if (planes == 0 || capacity == 0 || num_seqs == 0) return SHARPV_OK;
    if (!src_pos || !src_seq_offsets || !dst_begin) return SHARPV_ERR_INVALID_ARG;
    const int64_t eb = elem_bytes(src_layout->dtype);
    const int row_vecs = (int)(src_layout->head_dim * eb / 16);
    if (planes > 65535 || row_vecs > kAppendThreads * kAppendUnroll) return SHARPV_ERR_UNSUPPORTED;
    if (src_tokens > 0 && dst_tokens > 0) {
        uintptr_t s_lo, s_hi, d_lo, d_hi;
        kv_extent(kv_src, src_layout, layer_begin, layer_end, src_tokens, s_lo, s_hi);
        kv_extent(kv_dst, dst_layout, layer_begin, layer_end, dst_tokens, d_lo, d_hi);
        if (s_lo < d_hi && d_lo < s_hi) return SHARPV_ERR_INVALID_ARG;
    }
    AppendArgs a = {};
    a.src = (const char*)kv_src;
    a.dst = (char*)kv_dst;
    a.src_layer = src_layout->stride_layer * eb; a.src_kv = src_layout->stride_kv * eb;
    a.src_head = src_layout->stride_head * eb;   a.src_token = src_layout->stride_token * eb;
    a.dst_layer = dst_layout->stride_layer * eb; a.dst_kv = dst_layout->stride_kv * eb;
    a.dst_head = dst_layout->stride_head * eb;   a.dst_token = dst_layout->stride_token * eb;
    a.src_tokens = src_tokens;
    a.dst_tokens = dst_tokens;
    a.num_kv_heads = src_layout->num_kv_heads;
    a.layer_begin = layer_begin;
    a.row_vecs = row_vecs;
    a.tile_rows = kAppendThreads * kAppendUnroll / row_vecs;
    a.src_pos = src_pos;
    a.offsets = src_seq_offsets;
    a.dst_begin = dst_begin;
    a.num_seqs = num_seqs;
    a.capacity = capacity;
    a.status_word = status_word;
    int64_t tiles = (capacity + a.tile_rows - 1) / a.tile_rows;
    if (tiles > 65536) tiles = 65536;
    if (launch_dependent(kv_append_kernel, dim3((unsigned)tiles, (unsigned)planes), dim3(kAppendThreads), 0,
                         (cudaStream_t)cuda_stream, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}
