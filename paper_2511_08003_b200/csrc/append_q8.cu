// K/V rows into a cache in 8 bits (sharpv_kv_append_q8): for every plane the rows src_pos[j] of sequence b go to
// dst_begin[b] + (j - src_seq_offsets[b]), rounded to codes with a power of two as the scale of each block of rows:
//
//   e = least exponent with max |value| <= largest code * 2^e (over the rows that the block receives, and not under the scale
//   that rows in front of them have),  code = nearest(value * 2^-e),  and rows in front again if their scale has grown.
//
// A block needs its largest value before its first code, so a team of threads takes whole blocks: it loads up to kVecs 16-byte
// vectors a thread, keeps them in registers, finds the blocks' largest values (bits of non-negative floats order as
// integers: one warp reduction and one atomic of shared memory a warp), and writes codes from the registers: every
// row is read once, and one barrier a plane is enough.  Blocks that are larger than what a team holds are read twice, the second
// time out of L2.  Maxima do not depend on the order of atomics, multiplying by a power of two is exact, and one rounding remains.
//
// A team is a CTA where sequences receive many rows, and a warp where they receive a few (accepted tokens: 224 planes x
// 16 sequences of 1 to 6 rows are 3,584 small pieces, which have to be resident together).  Where there are many tiles a team
// takes several planes of one: what the tables say of the tile holds for all of them.
//
// The arithmetic is kept to about two instructions an element either way, or it would be what bounds it: largest values are found
// two at a time in the source's own type, products with powers of two are formed two at a time, and rounding to whole
// numbers is the addition of a number whose last place is 1.
//
// HBM bounds long lists: 37,712 rows of 224 planes x 256 bytes 513 to 519 us (6.3 TB/s, 0.97 to 0.98 of a plain copy's rate; 636 without the next
// plane's loads in flight, 1,634 with every index divided out and elements compared one at a time).  From 8 bits to 8 bits there are
// more codes a byte, and instructions bound it: half of these rows, int8 to int8, 211 us (0.79).  43 rows 7.1 us: latency
// (tables, rows, maximum, codes).  The 37,712 rows from bf16 to int8 530 us (0.95), e4m3 to e4m3 434 (0.77), to int8 551 (0.61), int8 to
// e4m3 438 (0.77), to int8 398 (0.84); half of the planes from fp32 440 either way (0.95).
#include "overlap.h"
#include "q8.cuh"

#include <cuda_bf16.h>

namespace sharpv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTileRows = 256;
constexpr int kMaxTeamPlanes = 16;

// Where planes lie, in bytes.
struct Planes {
    int64_t layer, kv, head;
    __device__ __forceinline__ int64_t at(int l, int v, int h) const { return l * layer + v * kv + h * head; }
};

struct AppendQ8Args {
    const char* src;
    uint8_t* dst;
    const uint8_t* src_scales;
    uint8_t* dst_scales;
    Planes src_to, dst_to, ss_to, ds_to;
    uint32_t src_token, dst_token;      // bytes
    int64_t src_tokens, dst_tokens;
    int src_shift, dst_shift;           // log2 of the blocks' rows
    int num_kv_heads, layer_begin, planes, row_vecs, code_vecs;     // 16-byte vectors of a source row, of a row of codes
    int go_rows;                        // rows that a team's threads hold one vector each of
    bool go_in_block;                   // such rows are a whole part of a block's
    int tile_rows;                      // a multiple of the block's rows
    int team_planes;                    // that a team takes of a tile, one after the other
    const int32_t* src_pos;
    const int32_t* offsets;
    const int32_t* dst_begin;
    int num_seqs;
    int64_t capacity;
    int32_t* status_word;
};

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t bits_of(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); }

// Low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// What a source's 16-byte vector gives: a running maximum of its magnitudes in the source's own form (`add`), that as bits of
// fp32 with whether something was not finite (`top`; without the source's scale), the largest finite magnitude the long way
// (`finite`), and its values as fp32.
template <int SRC> struct Source {
    static constexpr int kPerVec = Elem<SRC>::kPerVec;
    static constexpr bool kCodes = false;
    __device__ __forceinline__ static void widen(const uint4& v, float (&x)[kPerVec]) { Elem<SRC>::widen(v, x); }
    __device__ __forceinline__ static uint32_t add(uint32_t m, const uint4& v) {
        if constexpr (SRC == SHARPV_F32)
            return max(max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu)), m);
        else
            return __vmaxu2(__vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)), m);
    }
    __device__ __forceinline__ static uint32_t top(uint32_t m, bool& odd) {
        if constexpr (SRC == SHARPV_BF16) m = max(m & 0xffff0000u, m << 16);
        odd = m >= 0x7f800000u;
        return m;
    }
    __device__ __forceinline__ static uint32_t finite(const uint4& v) {
        float x[kPerVec];
        widen(v, x);
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < kPerVec; ++e) {
            const uint32_t y = __float_as_uint(x[e]) & 0x7fffffffu;
            m = max(m, y < 0x7f800000u ? y : 0u);
        }
        return m;
    }
};
template <int CODE> struct CodeSource {
    static constexpr int kPerVec = 16;
    static constexpr bool kCodes = true;
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
    // the codes of a vector two at a time in the high bytes of halves, where what stands in the low ones decides nothing
    __device__ __forceinline__ static uint32_t add(uint32_t m, const uint4& v) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (CODE == SHARPV_E4M3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = w[i] & 0x7f7f7f7fu;
                m = __vmaxu2(__vmaxu2(x, x << 8), m);
            }
            return m;
        } else {
            uint32_t hi = 0, lo = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi = __vmaxs2(__vmaxs2(w[i], w[i] << 8), hi);
                lo = __vmins2(__vmins2(w[i], w[i] << 8), lo);
            }
            const int most = max((int)hi >> 24, (int)(hi << 16) >> 24), least = min((int)lo >> 24, (int)(lo << 16) >> 24);
            return max(m, (uint32_t)max(most, -least));
        }
    }
    __device__ __forceinline__ static uint32_t top(uint32_t m, bool& odd) {
        if constexpr (CODE == SHARPV_E4M3) {
            m = max(m >> 24, m >> 8 & 0xffu);
            odd = m == 0x7fu;
            return __float_as_uint(__half2float(__low2half(as_half2(half2_of_e4m3((uint16_t)m)))));
        } else {
            odd = false;
            return __float_as_uint((float)m);
        }
    }
    __device__ __forceinline__ static uint32_t finite(const uint4& v) {
        float x[16];
        widen(v, x);
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t y = __float_as_uint(x[e]) & 0x7fffffffu;
            m = max(m, y < 0x7f800000u ? y : 0u);
        }
        return m;
    }
};
template <> struct Source<SHARPV_E4M3> : CodeSource<SHARPV_E4M3> {};
template <> struct Source<SHARPV_I8> : CodeSource<SHARPV_I8> {};

// The codes of a vector's values times 2^k.  `plain`: everything in it is finite and no product is beyond the largest code.
template <int SRC, int CODE>
__device__ __forceinline__ void store_codes(uint8_t* to, const uint4& v, int k, bool plain) {
    using S = Source<SRC>;
    constexpr int P = S::kPerVec;
    uint32_t w[P / 4];
    if constexpr (SRC == CODE) {
        // fp16 holds the codes and the products that round to something; 2^-24 takes what is below to 0 as well, and k > 15 only
        // goes with codes under 2^-7 (e4m3) or none (int8)
        const uint32_t c[4] = {v.x, v.y, v.z, v.w};
        const __half2 f = __float2half2_rn(power_of_two(min(max(k, -24), 15)));
        const bool more = CODE == SHARPV_E4M3 && k > 15;
        const __half2 g = __float2half2_rn(power_of_two(min(max(k - 15, 0), 2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo, hi;
            halves_of<CODE>(c[i], lo, hi);
            if constexpr (CODE == SHARPV_E4M3) {
                __half2 a = __hmul2(as_half2(lo), f), b = __hmul2(as_half2(hi), f);
                if (more) {
                    a = __hmul2(a, g);
                    b = __hmul2(b, g);
                }
                asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f16x2 l, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 h, %2;\n\tmov.b32 %0, {l, h};\n\t}"
                    : "=r"(w[i]) : "r"(bits_of(a)), "r"(bits_of(b)));
            } else {
                const __half2 one = __float2half2_rn(1536.f);       // whole numbers from here to 2048
                const uint32_t a = bits_of(__hfma2(as_half2(lo), f, one)), b = bits_of(__hfma2(as_half2(hi), f, one));
                w[i] = __byte_perm(a, b, 0x6420);
            }
        }
    } else {
        const float f = power_of_two(k);
        float x[P];
        if constexpr (SRC == SHARPV_BF16) {
            const __nv_bfloat162 f2 = __float2bfloat162_rn(f);
            const __nv_bfloat162 y[4] = {__hmul2(as_bf162(v.x), f2), __hmul2(as_bf162(v.y), f2), __hmul2(as_bf162(v.z), f2), __hmul2(as_bf162(v.w), f2)};
            S::widen(*reinterpret_cast<const uint4*>(y), x);
        } else {
            S::widen(v, x);
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] *= f;
        }
        if (CODE == SHARPV_I8 && plain) {
#pragma unroll
            for (int i = 0; i < P; ++i) x[i] += 12582912.f;         // 1.5 * 2^23: its last place is 1
#pragma unroll
            for (int i = 0; i < P / 4; ++i)
                w[i] = low_bytes(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
        } else {
#pragma unroll
            for (int i = 0; i < P / 4; ++i) w[i] = to_codes<CODE>(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        }
    }
    if constexpr (P == 4) __stcs(reinterpret_cast<uint32_t*>(to), w[0]);
    else if constexpr (P == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(w[0], w[1]));
    else st_stream(to, make_uint4(w[0], w[1], w[2], w[3]));
}

struct Team {
    int64_t plane[kMaxTeamPlanes][4];   // where the team's planes lie: source, its scales, destination, its scales
    uint32_t top[3][kMaxTileRows];      // of the tile's blocks: bits of the largest value; a plane after the other
};

constexpr int ctas_an_sm(int team, int vecs) { return team == 32 || vecs == 4 ? 3 : 2; }

// GOES: a tile may hold more rows than the team's threads (VECS vectors each), and is gone through twice a plane.
template <int SRC, int CODE, int TEAM, int VECS, bool GOES>
__global__ void __launch_bounds__(kThreads, ctas_an_sm(TEAM, VECS))
kv_append_q8_kernel(const __grid_constant__ AppendQ8Args a) {
    using S = Source<SRC>;
    constexpr int P = S::kPerVec, kTeams = kThreads / TEAM;
    __shared__ Team teams[kTeams];
    auto sync = [] { if constexpr (TEAM == 32) __syncwarp(); else __syncthreads(); };
    const int tid = threadIdx.x % TEAM, lane = threadIdx.x & 31;
    Team& sm = teams[threadIdx.x / TEAM];
    const int plane0 = (blockIdx.y * kTeams + threadIdx.x / TEAM) * a.team_planes;
    cudaGridDependencySynchronize();
    if (plane0 >= a.planes) return;
    const int64_t all = __ldg(a.offsets + a.num_seqs);
    const int n = (int)min(max(all, (int64_t)0), a.capacity);
    const bool speaks = plane0 == 0 && tid == 0;
    if (speaks && blockIdx.x == 0 && all > a.capacity) report(a.status_word, SHARPV_ERR_CAPACITY);
    // sequence b has the CTAs from offsets[b] / tile_rows + b on: enough for its tiles but one, which its last CTA takes as well
    auto offset = [&](int b) { return min(max(__ldg(a.offsets + b), 0), n); };
    auto first_cta = [&](int b) { return (uint32_t)offset(b) / (uint32_t)a.tile_rows + (uint32_t)b; };
    int b = 0;
    for (int left = a.num_seqs; left > 1;) {                // a warp narrows 32 ways a round
        const int step = (left + 31) / 32, at = lane * step;
        const uint32_t not_behind = __ballot_sync(0xffffffffu, at < left && first_cta(b + at) <= blockIdx.x);
        const int skip = max(__popc(not_behind) - 1, 0) * step;
        b += skip;
        left = min(step, left - skip);
    }
    const int j0 = offset(b), j1 = max(offset(b + 1), j0);
    const int64_t begin = __ldg(a.dst_begin + b);
    // rows of dst [lo, hi) of this sequence; row t holds list entry j0 + t - begin
    const int64_t lo = min(max(begin, (int64_t)0), a.dst_tokens), hi = min(max(begin + (j1 - j0), lo), a.dst_tokens);
    if (speaks && j1 > j0 && (begin < 0 || begin + (j1 - j0) > a.dst_tokens)) report(a.status_word, SHARPV_ERR_BOUNDS);
    const uint32_t cta0 = (uint32_t)j0 / (uint32_t)a.tile_rows + (uint32_t)b, ctas = first_cta(b + 1) - cta0;
    // nothing here, offsets that do not begin at 0, or CTAs behind the last sequence's (there are as many as capacity may need)
    if (lo >= hi || blockIdx.x < cta0 || blockIdx.x - cta0 >= ctas) return;
    const int block_rows = 1 << a.dst_shift;
    const int64_t base = lo >> a.dst_shift << a.dst_shift;  // first row of the sequence's first block
    const uint32_t tiles = ((uint32_t)(hi - base) + a.tile_rows - 1) / (uint32_t)a.tile_rows;
    const uint32_t mine = blockIdx.x - cta0, last_tile = mine + 1 == ctas ? tiles : min(tiles, mine + 1);
    // a thread has one column vector of every go_rows-th row
    const int y0 = tid / a.row_vecs, col = tid - y0 * a.row_vecs;
    const int go = VECS * a.go_rows;                        // rows that the team holds

    for (uint32_t tile = mine; tile < last_tile; ++tile) {
        const int64_t row0 = base + (int64_t)tile * a.tile_rows;
        const int rows = (int)min((int64_t)a.tile_rows, hi - row0), blocks = (rows + block_rows - 1) >> a.dst_shift;
        const int lead = (int)max(lo - row0, (int64_t)0);   // rows of the first block that lie in front
        const int fresh = rows - lead;
        int from[VECS];                                     // source rows of the thread's vectors
        unsigned there = 0;                                 // which of them there are
        auto look_up = [&](int g0, bool tell) {
            there = 0;
#pragma unroll
            for (int u = 0; u < VECS; ++u) {
                const int y = g0 + y0 + u * a.go_rows;
                from[u] = 0;
                if (y0 < a.go_rows && y < fresh) {
                    const int64_t f = __ldg(a.src_pos + j0 + (row0 + lead + y - begin));
                    if (f >= 0 && f < a.src_tokens) {
                        from[u] = (int)f;
                        there |= 1u << u;
                    } else if (tell && plane0 == 0) {
                        report(a.status_word, SHARPV_ERR_BOUNDS);
                    }
                }
            }
        };
        sync();                                             // the lists of the tile before are read
        for (int i = tid; i < blocks; i += TEAM) sm.top[0][i] = sm.top[1][i] = sm.top[2][i] = 0;
        const int planes = min(a.team_planes, a.planes - plane0);
        if (tid < planes) {
            const int p = plane0 + tid, h = p % a.num_kv_heads, kv = (p / a.num_kv_heads) & 1, l = a.layer_begin + p / (2 * a.num_kv_heads);
            sm.plane[tid][0] = a.src_to.at(l, kv, h);
            sm.plane[tid][1] = a.ss_to.at(l, kv, h);
            sm.plane[tid][2] = a.dst_to.at(l, kv, h);
            sm.plane[tid][3] = a.ds_to.at(l, kv, h);
        }
        look_up(0, true);
        sync();
        int turn = 0;                                       // which of the three lists of largest values
        const char* const s0 = a.src + col * 16;
        uint8_t* const d0 = a.dst + (row0 + lead + y0) * a.dst_token + col * P;        // the thread's first vector
        uint8_t* const ds0 = a.dst_scales + (row0 >> a.dst_shift);
        const int64_t d_go = (int64_t)a.go_rows * a.dst_token;
        uint4 v[VECS], next[GOES ? 1 : VECS];
        int unit[S::kCodes ? VECS : 1];             // exponent of the source's scale
        uint32_t next_unit[S::kCodes && !GOES ? VECS : 1];
        auto load = [&](int plane, uint4* to, auto* units) {
            const char* s = s0 + sm.plane[plane][0];
            [[maybe_unused]] const uint8_t* ss = S::kCodes ? a.src_scales + sm.plane[plane][1] : nullptr;
#pragma unroll
            for (int u = 0; u < VECS; ++u)
                if (there >> u & 1) {
                    to[u] = ld_stream(s + (uint64_t)(uint32_t)from[u] * a.src_token);
                    if constexpr (S::kCodes) units[u] = __ldg(ss + (from[u] >> a.src_shift));
                }
        };
        auto exponents = [&] {
            if constexpr (S::kCodes) {
#pragma unroll
                for (int u = 0; u < VECS; ++u) unit[u] = scale_exponent(unit[u]);
            }
        };
        if constexpr (!GOES) load(0, next, next_unit);
        for (int plane = 0; plane < planes; ++plane) {
            uint8_t* const d = d0 + sm.plane[plane][2];
            uint8_t* const ds = ds0 + sm.plane[plane][3];
            uint32_t* tops = sm.top[turn];
            const int old = lead > 0 ? scale_exponent(*ds) : kScaleLeast;       // of the first block's rows in front
            if constexpr (!GOES) {                  // the next plane's are on their way while this one's are worked on
#pragma unroll
                for (int u = 0; u < VECS; ++u) {
                    v[u] = next[u];
                    if constexpr (S::kCodes) unit[u] = next_unit[u];
                }
                if (plane + 1 < planes) load(plane + 1, next, next_unit);
                exponents();
            }
            unsigned odd = 0;                       // vectors with something that is not finite
            auto largest = [&](int g0) {
                if (blocks == 1 && !S::kCodes) {    // all of a thread's vectors together
                    uint32_t m = 0;
#pragma unroll
                    for (int u = 0; u < VECS; ++u)
                        if (there >> u & 1) m = S::add(m, v[u]);
                    bool strange;
                    uint32_t top = S::top(m, strange);
                    if (strange) {
                        odd = ~0u;
                        top = 0;
#pragma unroll
                        for (int u = 0; u < VECS; ++u)
                            if (there >> u & 1) top = max(top, S::finite(v[u]));
                    }
                    top = __reduce_max_sync(0xffffffffu, top);
                    if (lane == 0 && top) atomicMax(&tops[0], top);
                    return;
                }
                uint32_t most = 0;                  // of a tile's only block
#pragma unroll
                for (int u = 0; u < VECS; ++u) {
                    uint32_t top = 0;
                    if (there >> u & 1) {
                        bool strange;
                        top = S::top(S::add(0, v[u]), strange);
                        if (strange) {
                            odd |= 1u << u;
                            top = S::finite(v[u]);
                        }
                        if constexpr (S::kCodes) top = __float_as_uint(__uint_as_float(top) * power_of_two(unit[u]));
                    }
                    if (blocks == 1) {
                        most = max(most, top);
                        continue;
                    }
                    const int block = (lead + g0 + y0 + u * a.go_rows) >> a.dst_shift;
                    // a round's vectors lie in one block, or a warp's do
                    if ((S::kCodes && lead == 0 && a.go_in_block) || __all_sync(0xffffffffu, block == __shfl_sync(0xffffffffu, block, 0) || top == 0)) {
                        top = __reduce_max_sync(0xffffffffu, top);
                        if (lane == 0 && top) atomicMax(&tops[block], top);
                    } else if (top) {
                        atomicMax(&tops[block], top);
                    }
                }
                if (blocks == 1) {
                    most = __reduce_max_sync(0xffffffffu, most);
                    if (lane == 0 && most) atomicMax(&tops[0], most);
                }
            };
            if constexpr (GOES) {
                for (int g0 = 0; g0 < fresh; g0 += go) {
                    if (fresh > go) look_up(g0, g0 > 0 && plane == 0);
                    load(plane, v, unit);
                    exponents();
                    largest(g0);
                }
            } else {
                largest(0);
            }
            sync();
            // the list after the next: nobody reads it any more, and nobody adds to it before the next barrier
            auto each_block = [&](auto f) {
                if constexpr (TEAM >= kMaxTileRows) {
                    if (tid < blocks) f(tid);
                } else {
                    for (int i = tid; i < blocks; i += TEAM) f(i);
                }
            };
            uint32_t* const later = sm.top[turn == 0 ? 2 : turn - 1];
            auto exponent = [&](int block) {
                const int e = exponent_for<CODE>(tops[block]);
                return block == 0 ? max(e, old) : e;
            };
            each_block([&](int i) {
                later[i] = 0;
                ds[i] = (uint8_t)(exponent(i) + 127);
            });
            const int only = exponent(0);
            auto write = [&](int g0) {
                uint8_t* to = d + (GOES ? (int64_t)g0 * a.dst_token : 0);
#pragma unroll
                for (int u = 0; u < VECS; ++u, to += d_go) {
                    if (!(there >> u & 1)) continue;
                    const int e = blocks == 1 ? only : exponent((lead + g0 + y0 + u * a.go_rows) >> a.dst_shift);
                    store_codes<SRC, CODE>(to, v[u], (S::kCodes ? unit[S::kCodes ? u : 0] : 0) - e, !(odd >> u & 1) && e < kScaleMost);
                }
            };
            if constexpr (GOES) {
                for (int g0 = 0; g0 < fresh; g0 += go) {
                    if (fresh > go) {
                        look_up(g0, false);
                        load(plane, v, unit);
                        exponents();
                        odd = ~0u;                  // what was seen in a vector is not kept: each is taken for strange
                    }
                    write(g0);
                }
            } else {
                write(0);
            }
            if (lead > 0 && only != old) {          // rows in front, by the new scale
                uint8_t* front = d - (int64_t)(lead + y0) * a.dst_token - col * P;
                const int k = old - only, all_vecs = lead * a.code_vecs;
                constexpr int kAhead = 4;
                for (int q0 = tid; q0 < all_vecs; q0 += kAhead * TEAM) {
                    uint4 w[kAhead];
                    uint8_t* at[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int q = q0 + u * TEAM, r = q / a.code_vecs;
                        at[u] = front + (uint64_t)(uint32_t)r * a.dst_token + (q - r * a.code_vecs) * 16;
                        if (q < all_vecs) w[u] = *reinterpret_cast<const uint4*>(at[u]);
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (q0 + u * TEAM < all_vecs) store_codes<CODE, CODE>(at[u], w[u], k, false);
                }
            }
            turn = turn == 2 ? 0 : turn + 1;
        }
    }
}

template <int SRC, int CODE, int TEAM, int VECS, bool GOES>
sharpv_status launch(AppendQ8Args& a, int sms, cudaStream_t stream) {
    const int block_rows = 1 << a.dst_shift;
    a.go_rows = TEAM / a.row_vecs;
    a.go_in_block = block_rows % a.go_rows == 0;
    int rows = VECS * a.go_rows / block_rows * block_rows;      // what a team holds, in whole blocks; one at least
    if (rows < block_rows) rows = block_rows;
    if (rows > kMaxTileRows) rows = kMaxTileRows;
    a.tile_rows = rows;
    const int64_t ctas = a.capacity / rows + a.num_seqs;
    // several planes a team as long as there are four times as many teams as SMs hold
    constexpr int kTeams = kThreads / TEAM;
    a.team_planes = 1;
    while (a.team_planes < kMaxTeamPlanes && ctas * a.planes / (2 * a.team_planes) >= (int64_t)sms * kTeams * ctas_an_sm(TEAM, VECS) * 4) a.team_planes *= 2;
    const int y = (a.planes + kTeams * a.team_planes - 1) / (kTeams * a.team_planes);
    if (ctas >= (int64_t)1 << 31 || y > 65535) return SHARPV_ERR_UNSUPPORTED;
    if (launch_dependent(kv_append_q8_kernel<SRC, CODE, TEAM, VECS, GOES>, dim3((unsigned)ctas, (unsigned)y), dim3(kThreads), 0, stream, a) !=
        cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

template <int SRC, int CODE>
sharpv_status by_size(AppendQ8Args& a, int sms, cudaStream_t stream) {
    // a warp a piece where a sequence's rows are no more than a warp takes in two goes; else a CTA, with eight vectors a thread
    // where four do not hold a block, and in several goes where those do not either
    const int64_t vecs = a.capacity / a.num_seqs * a.row_vecs;
    if (vecs <= 2 * 4 * 32 && a.row_vecs <= 32) return launch<SRC, CODE, 32, 4, true>(a, sms, stream);
    const int block_rows = 1 << a.dst_shift, go_rows = kThreads / a.row_vecs;
    if (block_rows <= 4 * go_rows) return launch<SRC, CODE, kThreads, 4, false>(a, sms, stream);
    if (block_rows <= 8 * go_rows) return launch<SRC, CODE, kThreads, 8, false>(a, sms, stream);
    return launch<SRC, CODE, kThreads, 8, true>(a, sms, stream);
}

template <int SRC>
sharpv_status by_code(AppendQ8Args& a, sharpv_dtype code, int sms, cudaStream_t stream) {
    return code == SHARPV_E4M3 ? by_size<SRC, SHARPV_E4M3>(a, sms, stream) : by_size<SRC, SHARPV_I8>(a, sms, stream);
}

// the bytes that the scales of `rows` rows of the planes of the layers span
void scales_extent(const uint8_t* scales, const sharpv_kv_scales* s, const sharpv_kv_layout* L, int layer_begin, int layer_end,
                   int64_t rows, uintptr_t& lo, uintptr_t& hi) {
    lo = reinterpret_cast<uintptr_t>(scales) + (uintptr_t)(layer_begin * s->stride_layer);
    hi = reinterpret_cast<uintptr_t>(scales) + (uintptr_t)((layer_end - 1) * s->stride_layer + s->stride_kv +
                                                          (L->num_kv_heads - 1) * s->stride_head + (rows - 1) / s->block_tokens + 1);
}

Runs runs_of(const void* kv, const sharpv_kv_layout* L, int layer_begin, int layer_end, int64_t rows) {
    const int64_t eb = elem_bytes(L->dtype);
    return Runs{reinterpret_cast<uintptr_t>(kv) + (uintptr_t)(layer_begin * L->stride_layer * eb), L->head_dim * eb, 4,
                {L->stride_layer * eb, L->stride_kv * eb, L->stride_head * eb, L->stride_token * eb},
                {layer_end - layer_begin, 2, L->num_kv_heads, rows}};
}
Runs runs_of(const uint8_t* scales, const sharpv_kv_scales* s, const sharpv_kv_layout* L, int layer_begin, int layer_end, int64_t rows) {
    return Runs{reinterpret_cast<uintptr_t>(scales) + (uintptr_t)(layer_begin * s->stride_layer), rows > 0 ? (rows - 1) / s->block_tokens + 1 : 0, 3,
                {s->stride_layer, s->stride_kv, s->stride_head}, {layer_end - layer_begin, 2, L->num_kv_heads}};
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
    if (planes > 65535 || src_layout->head_dim > 1024 || row_vecs > 128 ||
        src_layout->stride_token * eb >= (int64_t)1 << 31 || dst_layout->stride_token >= (int64_t)1 << 31)
        return SHARPV_ERR_UNSUPPORTED;
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
    // what is written: no byte twice, and none that is read
    const Runs to = runs_of(kv_dst, dst_layout, layer_begin, layer_end, dst_tokens);
    const Runs to_scales = runs_of(dst_scales, dst_scales_layout, dst_layout, layer_begin, layer_end, dst_tokens);
    Share shares[5] = {shares_own_bytes(to), shares_own_bytes(to_scales), share_bytes(to, to_scales),
                       share_bytes(to_scales, runs_of(kv_src, src_layout, layer_begin, layer_end, src_tokens)), Share::no};
    if (codes) shares[4] = share_bytes(to, runs_of(src_scales, src_scales_layout, src_layout, layer_begin, layer_end, src_tokens));
    for (const Share s : shares)
        if (s != Share::no) return s == Share::yes ? SHARPV_ERR_INVALID_ARG : SHARPV_ERR_UNSUPPORTED;
    AppendQ8Args a = {};
    a.src = (const char*)kv_src;
    a.dst = (uint8_t*)kv_dst;
    const int H = src_layout->num_kv_heads;
    a.src_to = {src_layout->stride_layer * eb, src_layout->stride_kv * eb, src_layout->stride_head * eb};
    a.dst_to = {dst_layout->stride_layer, dst_layout->stride_kv, dst_layout->stride_head};
    a.src_token = (uint32_t)(src_layout->stride_token * eb);
    a.dst_token = (uint32_t)dst_layout->stride_token;
    a.src_scales = src_scales;
    if (codes) {
        a.ss_to = {src_scales_layout->stride_layer, src_scales_layout->stride_kv, src_scales_layout->stride_head};
        a.src_shift = log2_of(src_scales_layout->block_tokens);
    }
    a.dst_scales = dst_scales;
    a.ds_to = {dst_scales_layout->stride_layer, dst_scales_layout->stride_kv, dst_scales_layout->stride_head};
    a.dst_shift = log2_of(dst_scales_layout->block_tokens);
    a.src_tokens = src_tokens;
    a.dst_tokens = dst_tokens;
    a.num_kv_heads = H;
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
    int sms = 0;
    st = current_sms(sms);
    if (st != SHARPV_OK) return st;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    switch (src_layout->dtype) {
        case SHARPV_F32: return by_code<SHARPV_F32>(a, dst_layout->dtype, sms, stream);
        case SHARPV_BF16: return by_code<SHARPV_BF16>(a, dst_layout->dtype, sms, stream);
        case SHARPV_E4M3: return by_code<SHARPV_E4M3>(a, dst_layout->dtype, sms, stream);
        default: return by_code<SHARPV_I8>(a, dst_layout->dtype, sms, stream);
    }
}
