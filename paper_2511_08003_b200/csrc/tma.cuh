// Tensor maps (host) and the PTX of mbarriers, TMA tile loads, ldmatrix and mma that the attention kernels use.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace sharpv {

// A map over bf16 rows of D elements in two levels (inner count and byte stride, outer count and byte stride) whose box is
// 64 elements of box_inner x box_outer rows, laid out in shared memory with the 128-byte swizzle; elements outside
// read as zero.  box_bytes: for rows of D bytes instead, boxes of so many bytes (128, or 64 with the 64-byte swizzle).
inline bool encode_map(CUtensorMap* map, const void* base, int D, int64_t inner, int64_t inner_bytes, int64_t outer,
                       int64_t outer_bytes, int box_inner, int box_outer, int box_bytes = 0) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<Encode>(fn);
    }();
    if (!encode) return false;
    // a stride that no element needs may be anything the map accepts
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)inner, (cuuint64_t)outer};
    const cuuint64_t strides[2] = {inner > 1 ? (cuuint64_t)inner_bytes : 16u, outer > 1 ? (cuuint64_t)outer_bytes : 16u};
    const cuuint32_t box[3] = {box_bytes ? (cuuint32_t)box_bytes : 64u, (cuuint32_t)box_inner, (cuuint32_t)box_outer}, ones[3] = {1, 1, 1};
    return encode(map, box_bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims,
                  strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [heads][rows][D]: a box is box_rows rows of one head
inline bool encode_rows_map(CUtensorMap* map, const void* base, int D, int64_t rows, int64_t row_bytes, int heads,
                            int64_t head_bytes, int box_rows) {
    return encode_map(map, base, D, rows, row_bytes, heads, head_bytes, box_rows, 1);
}
// the same with rows of D bytes
inline bool encode_codes_map(CUtensorMap* map, const void* base, int D, int64_t rows, int64_t row_bytes, int heads,
                             int64_t head_bytes, int box_rows, int box_bytes) {
    return encode_map(map, base, D, rows, row_bytes, heads, head_bytes, box_rows, 1, box_bytes);
}
// [nodes][heads][D], heads next to each other: a box is box_heads heads of box_nodes nodes
inline bool encode_heads_map(CUtensorMap* map, const void* base, int D, int heads, int64_t nodes, int64_t node_bytes, int box_heads,
                             int box_nodes) {
    return encode_map(map, base, D, heads, (int64_t)D * 2, nodes, node_bytes, box_heads, box_nodes);
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(bar)) : "memory");
}

// one arrival when this thread's cp.async copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" :: "r"(smem_u32(bar)) : "memory");
}

// Waits for the phase of the given parity to complete, for two seconds at most (far beyond any kernel of this library);
// false if it did not.
constexpr unsigned long long kWaitNs = 2000000000ull;
__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool mbar_try(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity) {
    unsigned long long since = 0;
    for (uint32_t i = 1;; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 0) {
            const unsigned long long now = global_ns();
            if (since == 0) since = now;
            else if (now - since > kWaitNs) return false;
        }
    }
}

__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// writes of this thread to shared memory become visible to the tensor cores and to TMA
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// byte offset of 16-byte chunk c (0..7) of a 128-byte row in a swizzled tile that starts on a 1024-byte boundary
__device__ __forceinline__ uint32_t swizzle128(int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); }

// the same in a tile of 64-byte rows with the 64-byte swizzle (c 0..3)
__device__ __forceinline__ uint32_t swizzle64(int row, int c) { return (uint32_t)(row * 64 + ((c ^ (row >> 1 & 3)) << 4)); }

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// two fp32 rounded to fp16, `lo` in the low half
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// two fp32 rounded to bf16, `lo` in the low half
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// the bits of the halves of a bf16 pair that are infinite or NaN
__device__ __forceinline__ uint32_t nonfinite_bf16(uint32_t x) {
    return ((x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// whether one of eight bf16 is infinite or NaN: an exponent of ones carries into the sign's place
__device__ __forceinline__ bool any_nonfinite(const uint4& v) {
    auto carry = [](uint32_t x) { return (x & 0x7f807f80u) + 0x00800080u; };
    return ((carry(v.x) | carry(v.y) | carry(v.z) | carry(v.w)) & 0x80008000u) != 0;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace sharpv
