// Norm of every query and key head and its position rotation in one pass (sharpv_qk_norm_rope):
//
//   y = x / sqrt(mean(x^2) + eps) * weight            (left out where the call wants the rotation alone)
//   out_i = y_i cos a_i - y_{i+R/2} sin a_i,  out_{i+R/2} = y_{i+R/2} cos a_i + y_i sin a_i,  i < R/2,
//   a_i = positions[axis_i] * base^(-2i/R);  the elements from R on are y.
//
// Every row (a token's head) is read and written once, by LP neighbouring lanes.  A lane holds a vector of the first half
// of the rotated part and its partner of the second half, so the rotation needs no exchange and the norm LP - 1
// shuffles at most.  The angles of a token are the same for all its heads: a CTA takes whole tokens and keeps their cosines and
// sines in shared memory, in the order in which the lanes of a row read them (neighbouring 16 bytes).  Angles are
// formed in turns and reduced in 64 bits (a position of 2^31 is off by 2^-23 of a turn at most); their sine and cosine are
// taken in fp32, as the products are; the one rounding to the storage type is the last.
//
// A CTA takes about eight rounds of rows, the next round's loads in flight while one is worked on; arithmetic goes two elements
// an instruction.  Without either 50,432 tokens of 28 + 4 heads x 128 in bf16 take 164 us, with the first 149, with both 141: 5.9 TB/s,
// 0.91 of a plain copy's rate, and what is left is the issue of about 15 instructions an element.  1,600 tokens of 14 + 2 heads x 64 in
// fp32 4.4 us, 16 tokens 3.1 us (latency: positions, sine, one row).
#include "decode_common.cuh"
#include "overlap.h"

#include <cuda_bf16.h>

#include <cmath>

namespace sharpv {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 2;               // rows of a lane that are loaded before the first is worked on
constexpr int kMaxPairs = 128;          // head_dim of at most 256
constexpr int kMaxAxes = 8;
constexpr int kMaxTileTokens = 16;

struct NormRopeArgs {
    const char* q;
    const char* k;
    char* out_q;
    char* out_k;
    uint32_t q_token, q_head, k_token, k_head, oq_token, oq_head, ok_token, ok_head;    // bytes
    const char* q_weight;               // or null: ones
    const char* k_weight;
    const int32_t* positions;           // [axes][ld_positions]
    int64_t ld_positions, tokens;
    int q_heads, all_heads;             // all_heads: with the key heads
    int row_vecs, half_vecs, units, half;       // 16-byte vectors of a row, of half of the rotated part; lanes at work; pairs
    int tile_tokens;
    int norm;
    float eps, inv_d;
    double freq[kMaxPairs];             // turns a position
    uint8_t axis[kMaxPairs];
};

// Two fp32 at a time (one instruction each on this architecture).
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two() : v(0) {}
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ float2 parts() const {
        float2 r;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
        return r;
    }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

template <int DT>
__device__ __forceinline__ void widen2(const uint4& v, Two (&x)[Elem<DT>::kPerVec / 2]) {
    float y[Elem<DT>::kPerVec];
    Elem<DT>::widen(v, y);
#pragma unroll
    for (int i = 0; i < Elem<DT>::kPerVec / 2; ++i) x[i] = Two(y[2 * i], y[2 * i + 1]);
}
template <int DT>
__device__ __forceinline__ uint4 narrow(const Two (&x)[Elem<DT>::kPerVec / 2]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < Elem<DT>::kPerVec / 2; ++i) {
        const float2 p = x[i].parts();
        if constexpr (DT == SHARPV_F32) {
            w[2 * i] = __float_as_uint(p.x);
            w[2 * i + 1] = __float_as_uint(p.y);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(p.x, p.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 128 bits that are not read again; not by way of the read-only path, since an output may be its own input
__device__ __forceinline__ uint4 ld_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <int DT, int LP>
__global__ void __launch_bounds__(kThreads, 3)
qk_norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
    using E = Elem<DT>;
    constexpr int P = E::kPerVec, kGroups = kThreads / LP, kRound = kGroups * kAhead;
    extern __shared__ float4 table[];   // [tokens][P / 2][half_vecs]: cosines of two pairs, then their sines
    const int u = threadIdx.x % LP, group = threadIdx.x / LP;
    // the lane's two vectors: a pair of the rotated part, or two neighbours behind it
    const bool pair = u < a.half_vecs, busy = u < a.units;
    const int v0 = pair ? u : 2 * u, v1 = pair ? u + a.half_vecs : v0 + 1;
    const bool second = busy && v1 < a.row_vecs;
    cudaGridDependencySynchronize();
    const int64_t token0 = (int64_t)blockIdx.x * a.tile_tokens;
    const int tokens = (int)min((int64_t)a.tile_tokens, a.tokens - token0), rows = tokens * a.all_heads;
    // the group's rows are every kGroups-th from its first on (several CTAs share a token in turns of kRound)
    struct At { int r, t, h; };
    auto next = [&](At p, int by, int dt, int dh) {
        p.r += by;
        p.t += dt;
        p.h += dh;
        if (p.h >= a.all_heads) {
            p.h -= a.all_heads;
            ++p.t;
        }
        return p;
    };
    const int turn = gridDim.y * kRound, dt_turn = turn / a.all_heads, dh_turn = turn % a.all_heads;
    const char* const q = a.q + token0 * a.q_token;
    const char* const k = a.k + token0 * a.k_token;
    char* const out_q = a.out_q + token0 * a.oq_token;
    char* const out_k = a.out_k + token0 * a.ok_token;
    auto at_offset = [](auto* base, int t, uint32_t token, int h, uint32_t head) { return base + (uint64_t)(uint32_t)t * token + (uint64_t)(uint32_t)h * head; };
    auto load = [&](At p, uint4& x0, uint4& x1) {
        x0 = x1 = make_uint4(0, 0, 0, 0);
        if (p.r < rows && busy) {
            const char* row = p.h < a.q_heads ? at_offset(q, p.t, a.q_token, p.h, a.q_head) : at_offset(k, p.t, a.k_token, p.h - a.q_heads, a.k_head);
            x0 = ld_once(row + v0 * 16);
            if (second) x1 = ld_once(row + v1 * 16);
        }
    };
    At at[kAhead];                      // of the rows that are loaded
    uint4 x0[kAhead], x1[kAhead];
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
        const int r = blockIdx.y * kRound + y * kGroups + group;
        at[y] = At{r, r / a.all_heads, r % a.all_heads};
        load(at[y], x0[y], x1[y]);
    }
    if (blockIdx.y * kRound < rows) {   // while the rows are on their way
        const int step = a.half > 0 ? kThreads / a.half : 0;
        if (threadIdx.x < step * a.half) {
            const int i = threadIdx.x % a.half;
            const double freq = a.freq[i];
            const int32_t* positions = a.positions + a.axis[i] * a.ld_positions + token0;
            float* to = reinterpret_cast<float*>(table) + ((i % P >> 1) * a.half_vecs + i / P) * 4 + (i & 1);
            for (int t = threadIdx.x / a.half; t < tokens; t += step) {
                const double turns = __ldg(positions + t) * freq;
                float s, c;
                sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
                to[t * (P / 2) * a.half_vecs * 4] = c;
                to[t * (P / 2) * a.half_vecs * 4 + 2] = s;
            }
        }
    }
    __syncthreads();
    for (int r0 = blockIdx.y * kRound; r0 < rows; r0 += gridDim.y * kRound) {
#pragma unroll
        for (int y = 0; y < kAhead; ++y) {
            const At p = at[y];
            Two lo[P / 2], hi[P / 2];
            widen2<DT>(x0[y], lo);
            widen2<DT>(x1[y], hi);
            at[y] = next(p, turn, dt_turn, dh_turn);
            load(at[y], x0[y], x1[y]);              // as soon as the registers are free
            const bool is_q = p.h < a.q_heads;
            if (a.norm) {
                Two sum2;
#pragma unroll
                for (int e = 0; e < P / 2; ++e) sum2 = fma(lo[e], lo[e], fma(hi[e], hi[e], sum2));
                float sum = sum2.parts().x + sum2.parts().y;
#pragma unroll
                for (int o = LP / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float f = rsqrtf(fmaf(sum, a.inv_d, a.eps));
                const Two f2(f, f);
                const char* weight = is_q ? a.q_weight : a.k_weight;
                if (weight && busy) {
                    Two w[P / 2];
                    widen2<DT>(ld_cached(weight + v0 * 16), w);
#pragma unroll
                    for (int e = 0; e < P / 2; ++e) lo[e] = lo[e] * (f2 * w[e]);
                    if (second) {
                        widen2<DT>(ld_cached(weight + v1 * 16), w);
#pragma unroll
                        for (int e = 0; e < P / 2; ++e) hi[e] = hi[e] * (f2 * w[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < P / 2; ++e) {
                        lo[e] = lo[e] * f2;
                        hi[e] = hi[e] * f2;
                    }
                }
            }
            if (p.r >= rows || !busy) continue;
            if (pair) {
                const float4* cs = table + p.t * (P / 2) * a.half_vecs + u;
                const Two minus(-1.f, -1.f);
#pragma unroll
                for (int e = 0; e < P / 2; ++e) {
                    const float4 w = cs[e * a.half_vecs];
                    const Two c(w.x, w.y), s(w.z, w.w), x = lo[e];
                    lo[e] = fma(hi[e] * s, minus, x * c);
                    hi[e] = fma(hi[e], c, x * s);
                }
            }
            char* row = is_q ? at_offset(out_q, p.t, a.oq_token, p.h, a.oq_head) : at_offset(out_k, p.t, a.ok_token, p.h - a.q_heads, a.ok_head);
            st_stream(row + v0 * 16, narrow<DT>(lo));
            if (second) st_stream(row + v1 * 16, narrow<DT>(hi));
        }
    }
}

template <int DT, int LP>
sharpv_status launch(NormRopeArgs& a, int sms, cudaStream_t stream) {
    constexpr int kRound = kThreads / LP * kAhead;
    // about eight rounds a CTA, so that the angles are formed while others stream; with few tokens a CTA each, and with fewer
    // still several CTAs share a token's heads and form its angles each
    int64_t tile = (8 * kRound + a.all_heads - 1) / a.all_heads;
    const int64_t share = a.tokens / (2 * sms);
    if (tile > share) tile = share;
    if (tile > kMaxTileTokens) tile = kMaxTileTokens;
    if (tile < 1) tile = 1;
    a.tile_tokens = (int)tile;
    const int64_t ctas = (a.tokens + tile - 1) / tile;
    int y = 1;
    if (tile == 1) {
        y = (a.all_heads + kRound - 1) / kRound;
        const int64_t room = 4 * sms / ctas;
        if (y > room) y = room > 1 ? (int)room : 1;
    }
    const size_t smem = (size_t)tile * a.half * sizeof(float2);
    if (launch_dependent(qk_norm_rope_kernel<DT, LP>, dim3((unsigned)ctas, (unsigned)y), dim3(kThreads), smem, stream, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int DT>
sharpv_status by_lanes(NormRopeArgs& a, int sms, cudaStream_t stream) {
    if (a.units <= 2) return launch<DT, 2>(a, sms, stream);
    if (a.units <= 4) return launch<DT, 4>(a, sms, stream);
    if (a.units <= 8) return launch<DT, 8>(a, sms, stream);
    if (a.units <= 16) return launch<DT, 16>(a, sms, stream);
    return launch<DT, 32>(a, sms, stream);
}

// Rows of heads: what an output must not share with what is read, unless it is its own input.
struct HeadRows {
    const void* p;
    int64_t token, head;                // bytes
    int heads;
};
Runs runs_of(const HeadRows& r, int64_t tokens, int64_t row) {
    return Runs{reinterpret_cast<uintptr_t>(r.p), row, 2, {r.token, r.head}, {tokens, r.heads}};
}
bool same_rows(const HeadRows& a, const HeadRows& b, int64_t tokens) {
    return a.p == b.p && a.heads == b.heads && (tokens == 1 || a.token == b.token) && (a.heads == 1 || a.head == b.head);
}
sharpv_status outputs_status(const HeadRows (&in)[2], const HeadRows (&out)[2], int64_t tokens, int64_t row, const Runs (&tables)[3]) {
    Share worst = share_bytes(runs_of(out[0], tokens, row), runs_of(out[1], tokens, row));
    auto add = [&](Share s) { if (worst != Share::yes && s != Share::no) worst = s; };
    for (int i = 0; i < 2; ++i) {
        const Runs mine = runs_of(out[i], tokens, row);
        add(shares_own_bytes(mine));
        add(share_bytes(mine, runs_of(in[1 - i], tokens, row)));
        if (!same_rows(out[i], in[i], tokens)) add(share_bytes(mine, runs_of(in[i], tokens, row)));
        for (const Runs& t : tables) add(share_bytes(mine, t));
    }
    return worst == Share::no ? SHARPV_OK : (worst == Share::yes ? SHARPV_ERR_INVALID_ARG : SHARPV_ERR_UNSUPPORTED);
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" sharpv_status sharpv_qk_norm_rope(
    const void* q, int64_t ld_q, int64_t head_q, const void* k, int64_t ld_k, int64_t head_k, sharpv_dtype dtype,
    int64_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t norm, const void* q_weight,
    const void* k_weight, float eps, const int32_t* positions, int64_t ld_positions, int32_t num_axes,
    const uint8_t* pair_axis, int32_t rotary_dim, double rope_base, void* out_q, int64_t ld_out_q, int64_t head_out_q,
    void* out_k, int64_t ld_out_k, int64_t head_out_k, void* cuda_stream) {
    if (!dtype_ok(dtype)) return SHARPV_ERR_UNSUPPORTED;
    if (num_tokens < 0 || num_q_heads < 1 || num_kv_heads < 1 || head_dim < 1 || rotary_dim < 0 || rotary_dim > head_dim ||
        rotary_dim % 2 || (norm != 0 && norm != 1) || (norm && (!(eps >= 0.f) || !(eps < __builtin_huge_valf()))) ||
        (!norm && (q_weight || k_weight)) || (rotary_dim > 0 && (num_axes < 1 || !pair_axis || !(rope_base > 0.0) || !(rope_base < __builtin_huge_val()))))
        return SHARPV_ERR_INVALID_ARG;
    if (rotary_dim == 0 && !norm) return SHARPV_ERR_INVALID_ARG;
    const int64_t eb = elem_bytes(dtype), row = head_dim * eb;
    if (head_dim > 2 * kMaxPairs || row % 16 || (rotary_dim / 2 * eb) % 16 || num_axes > kMaxAxes ||
        (int64_t)num_q_heads + num_kv_heads > 4096 || num_tokens >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (pair_axis[i] >= num_axes) return SHARPV_ERR_INVALID_ARG;
    if (num_tokens == 0) return SHARPV_OK;
    if (!q || !k || !out_q || !out_k || (rotary_dim > 0 && (!positions || (num_axes > 1 && ld_positions < num_tokens && ld_positions != 0))))
        return SHARPV_ERR_INVALID_ARG;
    const int64_t strides[8] = {ld_q, head_q, ld_k, head_k, ld_out_q, head_out_q, ld_out_k, head_out_k};
    for (int i = 0; i < 8; ++i) {
        if (strides[i] < head_dim) return SHARPV_ERR_INVALID_ARG;
        if ((strides[i] * eb) % 16 || strides[i] * eb >= (int64_t)1 << 31) return SHARPV_ERR_UNSUPPORTED;
    }
    if (!aligned16(q) || !aligned16(k) || !aligned16(out_q) || !aligned16(out_k) || !aligned16(q_weight) || !aligned16(k_weight))
        return SHARPV_ERR_UNSUPPORTED;
    const HeadRows in[2] = {{q, ld_q * eb, head_q * eb, num_q_heads}, {k, ld_k * eb, head_k * eb, num_kv_heads}};
    const HeadRows out[2] = {{out_q, ld_out_q * eb, head_out_q * eb, num_q_heads}, {out_k, ld_out_k * eb, head_out_k * eb, num_kv_heads}};
    const Runs tables[3] = {{reinterpret_cast<uintptr_t>(q_weight), q_weight ? row : 0, 0}, {reinterpret_cast<uintptr_t>(k_weight), k_weight ? row : 0, 0},
                            {reinterpret_cast<uintptr_t>(positions), rotary_dim > 0 ? num_tokens * 4 : 0, 1, {ld_positions * 4}, {num_axes}}};
    const sharpv_status os = outputs_status(in, out, num_tokens, row, tables);
    if (os != SHARPV_OK) return os;
    NormRopeArgs a = {};
    a.q = (const char*)q;
    a.k = (const char*)k;
    a.out_q = (char*)out_q;
    a.out_k = (char*)out_k;
    uint32_t* const bytes[8] = {&a.q_token, &a.q_head, &a.k_token, &a.k_head, &a.oq_token, &a.oq_head, &a.ok_token, &a.ok_head};
    for (int i = 0; i < 8; ++i) *bytes[i] = (uint32_t)(strides[i] * eb);
    a.q_weight = (const char*)q_weight;
    a.k_weight = (const char*)k_weight;
    a.positions = positions;
    a.ld_positions = ld_positions;
    a.tokens = num_tokens;
    a.q_heads = num_q_heads;
    a.all_heads = num_q_heads + num_kv_heads;
    a.half = rotary_dim / 2;
    a.row_vecs = (int)(row / 16);
    a.half_vecs = (int)(a.half * eb / 16);
    a.units = a.half_vecs + (a.row_vecs - 2 * a.half_vecs + 1) / 2;
    a.norm = norm;
    a.eps = eps;
    a.inv_d = 1.0f / (float)head_dim;
    // powers one after the other, in 64 bits of mantissa: the last of 128 is off by 2^-57
    const long double ratio = a.half > 0 ? std::pow((long double)rope_base, -1.0L / a.half) : 0.0L;
    long double freq = 1.0L / 6.283185307179586476925286766559L;
    for (int i = 0; i < a.half; ++i, freq *= ratio) {
        a.axis[i] = pair_axis[i];
        a.freq[i] = (double)freq;
    }
    int sms = 0;
    const sharpv_status st = current_sms(sms);
    if (st != SHARPV_OK) return st;
    return dtype == SHARPV_F32 ? by_lanes<SHARPV_F32>(a, sms, (cudaStream_t)cuda_stream)
                               : by_lanes<SHARPV_BF16>(a, sms, (cudaStream_t)cuda_stream);
}
