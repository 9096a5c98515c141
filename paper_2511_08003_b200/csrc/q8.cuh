// Caches in 8 bits: codes (e4m3 or int8) with a power of two as the scale of each block of rows, head, K or V.
#pragma once

#include <cuda_fp16.h>

#include "decode_common.cuh"

namespace sharpv {

// Exponents of a scale that are used.  Twice their range and the softmax's own stays inside fp32's exponents.
constexpr int kScaleLeast = -48, kScaleMost = 48;
constexpr int kMaxBlockTokens = 256;

inline bool q8_dtype_ok(sharpv_dtype dt) { return dt == SHARPV_E4M3 || dt == SHARPV_I8; }

inline sharpv_status kv_scales_status(const uint8_t* scales, const sharpv_kv_scales* s) {
    if (!scales || !s || s->stride_layer < 0 || s->stride_kv < 0 || s->stride_head < 0) return SHARPV_ERR_INVALID_ARG;
    const int b = s->block_tokens;
    if (b < 1 || b > kMaxBlockTokens || (b & (b - 1))) return SHARPV_ERR_UNSUPPORTED;
    return SHARPV_OK;
}
inline int log2_of(int x) {
    int n = 0;
    while (1 << n < x) ++n;
    return n;
}

// the exponent that a scale's byte stands for
__device__ __forceinline__ int scale_exponent(uint32_t code) { return min(max((int)code - 127, kScaleLeast), kScaleMost); }
// 2^e for e of -126 to 127
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// The least e with x <= largest code * 2^e, within what is used; x by its bits, finite and not negative.  The largest codes are
// 1.75 * 2^8 and 1.984375 * 2^6: a mantissa beyond theirs carries into the exponent.
template <int CODE>
__device__ __forceinline__ int exponent_for(uint32_t bits) {
    const int e = CODE == SHARPV_E4M3 ? (int)((bits + 0x1fffffu) >> 23) - 127 - 8 : (int)((bits + 0x1ffffu) >> 23) - 127 - 6;
    return min(max(e, kScaleLeast), kScaleMost);
}

// Four values to four codes, nearest, ties to even, the largest codes beyond them.
template <int CODE>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    uint32_t r;
    if constexpr (CODE == SHARPV_E4M3) {
        asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
            : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    } else {
        uint32_t hi;
        asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(hi) : "r"(__float2int_rn(d)), "r"(__float2int_rn(c)), "r"(0));
        asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(__float2int_rn(b)), "r"(__float2int_rn(a)), "r"(hi));
    }
    return r;
}

// Two codes (bytes 0, 1 of the low or the high half) as halves, exactly.
__device__ __forceinline__ uint32_t half2_of_e4m3(uint16_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
    return r;
}

// Four codes to four halves: lo holds codes 0 and 1, hi codes 2 and 3.
template <int CODE>
__device__ __forceinline__ void halves_of(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    if constexpr (CODE == SHARPV_E4M3) {
        lo = half2_of_e4m3((uint16_t)codes);
        hi = half2_of_e4m3((uint16_t)(codes >> 16));
    } else {
        // the bytes behind 0x64 are halves of 1024 to 1279
        const uint32_t biased = codes ^ 0x80808080u;
        uint32_t a = __byte_perm(biased, 0x64646464u, 0x4140), b = __byte_perm(biased, 0x64646464u, 0x4342);
        const __half2 off = __half2half2(__ushort_as_half(0x6480));        // 1152
        const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), off), y = __hsub2(*reinterpret_cast<__half2*>(&b), off);
        lo = *reinterpret_cast<const uint32_t*>(&x);
        hi = *reinterpret_cast<const uint32_t*>(&y);
    }
}

// Four codes to fp32.
template <int CODE>
__device__ __forceinline__ void floats_of(uint32_t codes, float (&x)[4]) {
    if constexpr (CODE == SHARPV_E4M3) {
        uint32_t lo, hi;
        halves_of<CODE>(codes, lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(codes >> (8 * i));
    }
}

}  // namespace sharpv
