// K/V rows into a cache in 8 bits (sharpv_kv_append_q8): for every plane the rows src_pos[j] of sequence b go to
// dst_begin[b] + (j - src_seq_offsets[b]), rounded to codes with a power of two as the scale of each block of rows:
//
//   e = least exponent with max |value| <= largest code * 2^e (over the rows that the block receives, and not under the scale
//   that rows in front of them have),  code = nearest(value * 2^-e),  and rows in front again if their scale has grown.
//
// A block needs its largest value before its first code, so a team of threads takes whole blocks: it loads up to kVecs 16-byte
// vectors a thread, keeps them in registers, finds the blocks' largest values (bits of non-negative floats order as
// integers: one warp reduction and one atomic of shared memory a warp), and writes codes from the registers: every
// row is read once.  Blocks that are larger than what a team holds are read twice, the second time out of L2.
// Maxima do not depend on the order of atomics, multiplying by a power of two is exact, and one rounding remains.
//
// A team is a CTA where sequences receive many rows, and a warp where they receive a few (accepted tokens: 224 planes x
// 16 sequences of 1 to 6 rows are 3,584 small pieces, which have to be resident together).
//
// HBM bounds long lists, latency (tables, rows, maximum, codes) short ones.
#include "q8.cuh"

namespace sharpv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTileRows = 256;

struct AppendQ8Args {
    const char* src;
    uint8_t* dst;
    const uint8_t* src_scales;
    uint8_t* dst_scales;
    int64_t src_layer, src_kv, src_head, src_token, dst_layer, dst_kv, dst_head, dst_token;    // bytes
    int64_t ss_layer, ss_kv, ss_head, ds_layer, ds_kv, ds_head;
    int64_t src_tokens, dst_tokens;
    int src_shift, dst_shift;           // log2 of the blocks' rows
    int num_kv_heads, layer_begin, planes, row_vecs, code_vecs;     // 16-byte vectors of a source row, of a row of codes
    int tile_rows;                      // a multiple of the block's rows
    const int32_t* src_pos;
    const int32_t* offsets;
    const int32_t* dst_begin;
    int num_seqs;
    int64_t capacity;
    int32_t* status_word;
};

template <int SRC> struct Source {      // a 16-byte vector as fp32
    static constexpr int kPerVec = Elem<SRC>::kPerVec;
    __device__ __forceinline__ static void widen(const uint4& v, float (&x)[kPerVec]) { Elem<SRC>::widen(v, x); }
};
template <int CODE> struct CodeSource {
    static constexpr int kPerVec = 16;
    __device__ __forceinline__ static void widen(const uint4& v, float (&x)[16]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[4];
            floats_of<CODE>(w[i], y);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = y[j];
        }
    }
};
template <> struct Source<SHARPV_E4M3> : CodeSource<SHARPV_E4M3> {};
template <> struct Source<SHARPV_I8> : CodeSource<SHARPV_I8> {};

template <int CODE, int P>
__device__ __forceinline__ void store_codes(uint8_t* to, const float (&x)[P], float f) {
    uint32_t w[P / 4];
#pragma unroll
    for (int i = 0; i < P / 4; ++i) w[i] = to_codes<CODE>(x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f, x[4 * i + 3] * f);
    if constexpr (P == 4) __stcs(reinterpret_cast<uint32_t*>(to), w[0]);
    else if constexpr (P == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(w[0], w[1]));
    else st_stream(to, make_uint4(w[0], w[1], w[2], w[3]));
}

struct Team {
    int from[kMaxTileRows];             // source row of a row of the tile; -1: none
    float unit[kMaxTileRows];           // scale of that row (sources in 8 bits)
    uint32_t top[kMaxTileRows];         // of the tile's blocks: bits of the largest value, then the exponent
    int old;                            // of the first block, where rows lie in front
};

template <int SRC, int CODE, int TEAM, int VECS>
__global__ void __launch_bounds__(kThreads, VECS > 4 ? 3 : 4)
kv_append_q8_kernel(const __grid_constant__ AppendQ8Args a) {
    using S = Source<SRC>;
    constexpr int P = S::kPerVec, kTeams = kThreads / TEAM;
    constexpr bool kCodes = SRC == SHARPV_E4M3 || SRC == SHARPV_I8;
    __shared__ Team teams[kTeams];
    auto sync = [] { if constexpr (TEAM == 32) __syncwarp(); else __syncthreads(); };
    const int tid = threadIdx.x % TEAM, lane = threadIdx.x & 31;
    Team& sm = teams[threadIdx.x / TEAM];
    const int plane = blockIdx.y * kTeams + threadIdx.x / TEAM;
    cudaGridDependencySynchronize();
    if (plane >= a.planes) return;
    const int h = plane % a.num_kv_heads, kv = (plane / a.num_kv_heads) & 1, l = a.layer_begin + plane / (2 * a.num_kv_heads);
    const int64_t all = __ldg(a.offsets + a.num_seqs);
    const int64_t n = min(max(all, (int64_t)0), a.capacity);
    const bool speaks = plane == 0 && tid == 0;
    if (speaks && blockIdx.x == 0 && all > a.capacity) report(a.status_word, SHARPV_ERR_CAPACITY);
    // sequence b has the CTAs from offsets[b] / tile_rows + b on: enough for its tiles but one, which its last CTA takes as well
    auto offset = [&](int b) { return min(max((int64_t)__ldg(a.offsets + b), (int64_t)0), n); };
    auto first_cta = [&](int b) { return (int64_t)((uint32_t)offset(b) / (uint32_t)a.tile_rows) + b; };
    int b = 0;
    for (int hi = a.num_seqs; hi - b > 1;) {
        const int mid = (b + hi) >> 1;
        if (first_cta(mid) <= blockIdx.x) b = mid; else hi = mid;
    }
    const int64_t j0 = offset(b), j1 = max(offset(b + 1), j0), begin = __ldg(a.dst_begin + b);
    // rows of dst [lo, hi) of this sequence; row t holds list entry j0 + t - begin
    const int64_t lo = min(max(begin, (int64_t)0), a.dst_tokens), hi = min(max(begin + (j1 - j0), lo), a.dst_tokens);
    if (speaks && j1 > j0 && (begin < 0 || begin + (j1 - j0) > a.dst_tokens)) report(a.status_word, SHARPV_ERR_BOUNDS);
    if (lo >= hi) return;
    const int block_rows = 1 << a.dst_shift;
    const int64_t base = lo >> a.dst_shift << a.dst_shift;         // first row of the sequence's first block
    const int64_t tiles = (hi - base + a.tile_rows - 1) / a.tile_rows;
    const int64_t mine = blockIdx.x - first_cta(b), ctas = first_cta(b + 1) - first_cta(b);
    if (mine < 0) return;               // offsets that do not begin at 0
    const char* s = a.src + l * a.src_layer + kv * a.src_kv + h * a.src_head;
    const uint8_t* ss = kCodes ? a.src_scales + l * a.ss_layer + kv * a.ss_kv + h * a.ss_head : nullptr;
    uint8_t* d = a.dst + l * a.dst_layer + kv * a.dst_kv + h * a.dst_head;
    uint8_t* ds = a.dst_scales + l * a.ds_layer + kv * a.ds_kv + h * a.ds_head;

    for (int64_t tile = mine; tile < (mine + 1 == ctas ? tiles : min(tiles, mine + 1)); ++tile) {
        const int64_t row0 = base + tile * a.tile_rows;
        const int rows = (int)min((int64_t)a.tile_rows, hi - row0), blocks = (rows + block_rows - 1) >> a.dst_shift;
        const int lead = (int)max(lo - row0, (int64_t)0);           // rows of the first block that lie in front
        sync();
        for (int r = tid; r < rows; r += TEAM) {
            int from = -1;
            if (r >= lead) {
                const int64_t f = __ldg(a.src_pos + j0 + (row0 + r - begin));
                if (f >= 0 && f < a.src_tokens) from = (int)f;
                else if (plane == 0) report(a.status_word, SHARPV_ERR_BOUNDS);
            }
            sm.from[r] = from;
            if constexpr (kCodes) sm.unit[r] = from >= 0 ? power_of_two(scale_exponent(__ldg(ss + (from >> a.src_shift)))) : 0.f;
        }
        for (int i = tid; i < blocks; i += TEAM) sm.top[i] = 0;
        if (tid == 0 && lead > 0) sm.old = scale_exponent(ds[row0 >> a.dst_shift]);
        sync();
        const int vecs = rows * a.row_vecs, block_vecs = a.row_vecs << a.dst_shift;
        const bool whole_warps = block_vecs % 32 == 0;
        uint4 v[VECS];
        unsigned there = 0;
        auto load = [&](int q0) {
            there = 0;
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                const int q = q0 + u * TEAM + tid, r = q / a.row_vecs;
                if (q < vecs && sm.from[r] >= 0) {
                    v[u] = ld_stream(s + sm.from[r] * a.src_token + (int64_t)(q - r * a.row_vecs) * 16);
                    there |= 1u << u;
                }
            }
        };
        for (int q0 = 0; q0 < vecs; q0 += VECS * TEAM) {
            load(q0);
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                const int q = q0 + u * TEAM + tid;
                uint32_t top = 0;
                if (there >> u & 1) {
                    float x[P];
                    S::widen(v[u], x);
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const uint32_t m = __float_as_uint(x[e]) & 0x7fffffffu;
                        top = max(top, m < 0x7f800000u ? m : 0u);
                    }
                    if constexpr (kCodes) top = __float_as_uint(__uint_as_float(top) * sm.unit[q / a.row_vecs]);
                }
                if (whole_warps) {              // the warp's 32 vectors lie in one block
                    top = __reduce_max_sync(0xffffffffu, top);
                    if (lane == 0 && top) atomicMax(&sm.top[q / block_vecs], top);
                } else if (top) {
                    atomicMax(&sm.top[q / block_vecs], top);
                }
            }
        }
        sync();
        for (int i = tid; i < blocks; i += TEAM) {
            int e = exponent_for<CODE>(sm.top[i]);
            if (i == 0 && lead > 0) e = max(e, sm.old);
            sm.top[i] = (uint32_t)e;
            ds[(row0 >> a.dst_shift) + i] = (uint8_t)(e + 127);
        }
        sync();
        for (int q0 = 0; q0 < vecs; q0 += VECS * TEAM) {
            if (vecs > VECS * TEAM) load(q0);
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                const int q = q0 + u * TEAM + tid;
                if (!(there >> u & 1)) continue;
                const int r = q / a.row_vecs;
                float x[P], f = power_of_two(-(int)sm.top[r >> a.dst_shift]);
                S::widen(v[u], x);
                if constexpr (kCodes) f *= sm.unit[r];
                store_codes<CODE>(d + (row0 + r) * a.dst_token + (int64_t)(q - r * a.row_vecs) * P, x, f);
            }
        }
        if (lead > 0 && (int)sm.top[0] != sm.old) {         // rows in front, by the new scale
            const float f = power_of_two(sm.old - (int)sm.top[0]);
            for (int q = tid; q < lead * a.code_vecs; q += TEAM) {
                const int r = q / a.code_vecs;
                uint4* at = reinterpret_cast<uint4*>(d + (row0 + r) * a.dst_token) + (q - r * a.code_vecs);
                float x[16];
                CodeSource<CODE>::widen(*at, x);
                store_codes<CODE>(reinterpret_cast<uint8_t*>(at), x, f);
            }
        }
    }
}

template <int SRC, int CODE, int TEAM, int VECS>
sharpv_status launch(AppendQ8Args& a, cudaStream_t stream) {
    const int block_rows = 1 << a.dst_shift;
    int rows = VECS * TEAM / a.row_vecs / block_rows * block_rows;      // what a team holds, in whole blocks; one at least
    if (rows < block_rows) rows = block_rows;
    if (rows > kMaxTileRows) rows = kMaxTileRows;
    a.tile_rows = rows;
    const int64_t ctas = a.capacity / rows + a.num_seqs;
    const int y = (a.planes + kThreads / TEAM - 1) / (kThreads / TEAM);
    if (ctas >= (int64_t)1 << 31 || y > 65535) return SHARPV_ERR_UNSUPPORTED;
    if (launch_dependent(kv_append_q8_kernel<SRC, CODE, TEAM, VECS>, dim3((unsigned)ctas, (unsigned)y), dim3(kThreads), 0, stream, a) !=
        cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int SRC, int CODE>
sharpv_status by_size(AppendQ8Args& a, cudaStream_t stream) {
    // a warp a piece where a sequence's rows are no more than a warp takes in two goes; else a CTA, with eight vectors a thread
    // where four do not hold a block
    const int64_t vecs = a.capacity / a.num_seqs * a.row_vecs;
    if (vecs <= 2 * 4 * 32) return launch<SRC, CODE, 32, 4>(a, stream);
    if ((a.row_vecs << a.dst_shift) <= 4 * kThreads) return launch<SRC, CODE, kThreads, 4>(a, stream);
    return launch<SRC, CODE, kThreads, 8>(a, stream);
}

template <int SRC>
sharpv_status by_code(AppendQ8Args& a, sharpv_dtype code, cudaStream_t stream) {
    return code == SHARPV_E4M3 ? by_size<SRC, SHARPV_E4M3>(a, stream) : by_size<SRC, SHARPV_I8>(a, stream);
}

// the bytes that the scales of `rows` rows of the planes of the layers span
void scales_extent(const uint8_t* scales, const sharpv_kv_scales* s, const sharpv_kv_layout* L, int layer_begin, int layer_end,
                   int64_t rows, uintptr_t& lo, uintptr_t& hi) {
    lo = reinterpret_cast<uintptr_t>(scales) + (uintptr_t)(layer_begin * s->stride_layer);
    hi = reinterpret_cast<uintptr_t>(scales) + (uintptr_t)((layer_end - 1) * s->stride_layer + s->stride_kv +
                                                          (L->num_kv_heads - 1) * s->stride_head + (rows - 1) / s->block_tokens + 1);
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" sharpv_status sharpv_kv_append_q8(
    const void* kv_src, const sharpv_kv_layout* src_layout, const uint8_t* src_scales, const sharpv_kv_scales* src_scales_layout,
    int64_t src_tokens, void* kv_dst, const sharpv_kv_layout* dst_layout, uint8_t* dst_scales,
    const sharpv_kv_scales* dst_scales_layout, int64_t dst_tokens, int32_t layer_begin, int32_t layer_end, const int32_t* src_pos,
    const int32_t* src_seq_offsets, const int32_t* dst_begin, int32_t num_seqs, int64_t capacity, int32_t* status_word,
    void* cuda_stream) {
    sharpv_status st = kv_layout_status_if(kv_src, src_layout, [](sharpv_dtype t) { return dtype_ok(t) || q8_dtype_ok(t); });
    if (st != SHARPV_OK) return st;
    st = kv_layout_status_if(kv_dst, dst_layout, q8_dtype_ok);
    if (st != SHARPV_OK) return st;
    const bool codes = q8_dtype_ok(src_layout->dtype);
    if (codes != (src_scales != nullptr) || codes != (src_scales_layout != nullptr)) return SHARPV_ERR_INVALID_ARG;
    st = codes ? kv_scales_status(src_scales, src_scales_layout) : SHARPV_OK;
    if (st != SHARPV_OK) return st;
    st = kv_scales_status(dst_scales, dst_scales_layout);
    if (st != SHARPV_OK) return st;
    if (src_layout->head_dim != dst_layout->head_dim || src_layout->num_kv_heads != dst_layout->num_kv_heads ||
        src_layout->num_layers != dst_layout->num_layers || layer_begin < 0 || layer_end > src_layout->num_layers ||
        layer_begin > layer_end || capacity < 0 || num_seqs < 0 || src_tokens < 0 || dst_tokens < 0)
        return SHARPV_ERR_INVALID_ARG;
    if (capacity >= (int64_t)1 << 31 || src_tokens >= (int64_t)1 << 31 || dst_tokens >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
    const int64_t planes = (int64_t)(layer_end - layer_begin) * 2 * src_layout->num_kv_heads;
    if (planes == 0 || capacity == 0 || num_seqs == 0) return SHARPV_OK;
    if (!src_pos || !src_seq_offsets || !dst_begin) return SHARPV_ERR_INVALID_ARG;
    const int64_t eb = elem_bytes(src_layout->dtype);
    const int row_vecs = (int)(src_layout->head_dim * eb / 16);
    if (planes > 65535 || src_layout->head_dim > 1024 || row_vecs > 128) return SHARPV_ERR_UNSUPPORTED;
    if (src_tokens > 0 && dst_tokens > 0) {
        uintptr_t s_lo, s_hi, d_lo, d_hi;
        kv_extent(kv_src, src_layout, layer_begin, layer_end, src_tokens, s_lo, s_hi);
        kv_extent(kv_dst, dst_layout, layer_begin, layer_end, dst_tokens, d_lo, d_hi);
        if (s_lo < d_hi && d_lo < s_hi) return SHARPV_ERR_INVALID_ARG;
        if (codes) {
            scales_extent(src_scales, src_scales_layout, src_layout, layer_begin, layer_end, src_tokens, s_lo, s_hi);
            scales_extent(dst_scales, dst_scales_layout, dst_layout, layer_begin, layer_end, dst_tokens, d_lo, d_hi);
            if (s_lo < d_hi && d_lo < s_hi) return SHARPV_ERR_INVALID_ARG;
        }
    }
    AppendQ8Args a = {};
    a.src = (const char*)kv_src;
    a.dst = (uint8_t*)kv_dst;
    a.src_layer = src_layout->stride_layer * eb; a.src_kv = src_layout->stride_kv * eb;
    a.src_head = src_layout->stride_head * eb;   a.src_token = src_layout->stride_token * eb;
    a.dst_layer = dst_layout->stride_layer; a.dst_kv = dst_layout->stride_kv;
    a.dst_head = dst_layout->stride_head;   a.dst_token = dst_layout->stride_token;
    a.src_scales = src_scales;
    if (codes) {
        a.ss_layer = src_scales_layout->stride_layer;
        a.ss_kv = src_scales_layout->stride_kv;
        a.ss_head = src_scales_layout->stride_head;
        a.src_shift = log2_of(src_scales_layout->block_tokens);
    }
    a.dst_scales = dst_scales;
    a.ds_layer = dst_scales_layout->stride_layer;
    a.ds_kv = dst_scales_layout->stride_kv;
    a.ds_head = dst_scales_layout->stride_head;
    a.dst_shift = log2_of(dst_scales_layout->block_tokens);
    a.src_tokens = src_tokens;
    a.dst_tokens = dst_tokens;
    a.num_kv_heads = src_layout->num_kv_heads;
    a.layer_begin = layer_begin;
    a.planes = (int)planes;
    a.row_vecs = row_vecs;
    a.code_vecs = src_layout->head_dim / 16;
    a.src_pos = src_pos;
    a.offsets = src_seq_offsets;
    a.dst_begin = dst_begin;
    a.num_seqs = num_seqs;
    a.capacity = capacity;
    a.status_word = status_word;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    switch (src_layout->dtype) {
        case SHARPV_F32: return by_code<SHARPV_F32>(a, dst_layout->dtype, stream);
        case SHARPV_BF16: return by_code<SHARPV_BF16>(a, dst_layout->dtype, stream);
        case SHARPV_E4M3: return by_code<SHARPV_E4M3>(a, dst_layout->dtype, stream);
        default: return by_code<SHARPV_I8>(a, dst_layout->dtype, stream);
    }
}
