// What the operators that decode over a K/V cache share: the sequence tables (where a sequence's rows sit in
// the cache, which query nodes are its own) with their range checks, and the split of an attention call into
// units that the resident CTAs share evenly.
#pragma once

#include "common.cuh"

namespace sharpv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

struct SeqTables {
    const int32_t* begin;       // first cache row of sequence b
    const int32_t* len;         // its rows
    const int32_t* node_off;    // its nodes: [node_off[b], node_off[b + 1])
    int num_seqs;
    int64_t cache_tokens;       // rows a plane of the cache holds
    int64_t total_nodes;
};

struct SeqInfo {
    int64_t begin;
    int len, node0, nodes;
};

// Entry b of the tables, cut to what the cache and the node arrays hold; `bad` is set if something was cut.
__device__ __forceinline__ SeqInfo load_seq(const SeqTables& t, int b, bool& bad) {
    SeqInfo s;
    const int64_t begin = __ldg(t.begin + b), len = __ldg(t.len + b);
    const int64_t n0 = __ldg(t.node_off + b), n1 = __ldg(t.node_off + b + 1);
    s.begin = begin < 0 ? 0 : (begin > t.cache_tokens ? t.cache_tokens : begin);
    int64_t l = begin < 0 || len < 0 ? 0 : len;
    if (l > t.cache_tokens - s.begin) l = t.cache_tokens - s.begin;
    s.len = (int)l;
    const int64_t a = n0 < 0 ? 0 : (n0 > t.total_nodes ? t.total_nodes : n0);
    const int64_t e = n1 < a ? a : (n1 > t.total_nodes ? t.total_nodes : n1);
    s.node0 = (int)a;
    s.nodes = (int)(e - a);
    bad = bad || s.begin != begin || l != len || a != n0 || e != n1;
    return s;
}

// The split of an attention call.  A segment is one (sequence, KV head, tile of `rows` query rows); a query
// row is a (node, query head of the KV head's group) pair, nodes outermost.  A segment's keys are its cached rows
// in tiles of `keys`, then its drafted tokens in tiles of `keys`; a unit is one such key tile of one segment,
// numbered with the key tile innermost.  Units are dealt to the CTAs in one of two ways, and the segments that several
// CTAs share are joined from partial results afterwards:
//   pieces  every segment is cut into even pieces of a cost of at most m, one CTA each, m as small as the CTAs allow;
//   runs    CTA c of G takes the units [c U / G, (c + 1) U / G), whose numbers differ by one at most, but many CTAs
//           end one segment and begin the next, which costs them about kSwitch.
// Pieces are taken where m is no more than a run's cost and that (and there are at most 32 sequences: one a lane).
// Against runs alone, us: tree of 64 nodes over 50,432 rows 58.9 -> 57.0, ragged trees 47.1 -> 46.0, one token over 50,432
// rows 29.3 -> 28.7, weight of ragged trees 26.3 -> 24.4; a chunk of 509 nodes over 10,944 rows keeps runs.  kSwitch was chosen
// on these, which are bf16; the fp32 kernels use it as it is, although a tile of theirs (32 keys) takes another time.
struct Split {
    static constexpr uint32_t kSwitch = 3;      // what ending one segment and beginning another costs, in tiles
    __host__ __device__ uint32_t cost(const SeqInfo&) const { return 1; }
    int rows, keys, group, heads;
    int draft;                  // the drafted tokens' keys take part
    __host__ __device__ int row_tiles(const SeqInfo& s) const {
        return (int)(((uint32_t)s.nodes * (uint32_t)group + (uint32_t)rows - 1) / (uint32_t)rows);     // under 2^31 query rows
    }
    __host__ __device__ int cache_tiles(const SeqInfo& s) const { return (s.len + keys - 1) / keys; }
    // at least one (then empty), so that rows without any key are written as well
    __host__ __device__ int key_tiles(const SeqInfo& s) const {
        const int n = cache_tiles(s) + (draft ? (s.nodes + keys - 1) / keys : 0);
        return n > 0 ? n : 1;
    }
    __host__ __device__ int64_t segments(const SeqInfo& s) const { return (int64_t)row_tiles(s) * heads; }
    __host__ __device__ int tiles(const SeqInfo& s) const { return key_tiles(s); }
    __host__ __device__ int64_t units(const SeqInfo& s) const { return segments(s) * key_tiles(s); }
};

// The split of a call that gives every cached row a value: a unit is `keys` rows of one sequence.  Its cost goes by the
// query rows that weigh them (a KV head's, `share` halvings for nodes that count for nothing), from the 64 on that
// take longer than the keys' loads.
struct KeySplit {
    int keys, group, share;
    static constexpr uint32_t kSwitch = 12;
    __host__ __device__ int64_t segments(const SeqInfo& s) const { return s.len > 0; }
    __host__ __device__ int tiles(const SeqInfo& s) const { return (s.len + keys - 1) / keys; }
    __host__ __device__ int64_t units(const SeqInfo& s) const { return tiles(s); }
    __host__ __device__ uint32_t cost(const SeqInfo& s) const {
        const int64_t rows = ((int64_t)s.nodes * group >> share) / 32;
        return rows < 1 ? 2u : (rows > 62 ? 64u : (uint32_t)rows + 1u);
    }
};

// 64-bit division that takes the 32-bit one where the numbers allow it (nearly always: the 64-bit one is a routine of
// its own, and several of them in a row cost a microsecond at the start of a kernel).
__device__ __forceinline__ int64_t div64(int64_t a, int64_t b) {
    return ((uint64_t)(a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// `units` dealt to `ctas` CTAs in contiguous runs whose lengths differ by one at most.  No more CTAs take part than
// there are units, so each of those has at least one.
struct Deal {
    int64_t each, extra;        // the first `extra` CTAs have one unit more
    int busy;                   // CTAs that take part
    __device__ __forceinline__ Deal(int64_t units, int ctas) {
        busy = units < ctas ? (int)units : ctas;
        each = busy ? div64(units, busy) : 0;
        extra = units - each * busy;
    }
    __device__ __forceinline__ int64_t first(int c) const { return c * each + (c < extra ? c : extra); }
    __device__ __forceinline__ int owner(int64_t u) const {
        const int64_t head = extra * (each + 1);
        return (int)(u < head ? div64(u, each + 1) : extra + div64(u - head, each));
    }
};

struct PlanStart {
    SeqInfo s;                  // sequence of the CTA's first unit
    int b;
    int64_t before;             // units in front of that sequence
    int64_t units;              // of the whole call
    // pieces (segments >= 0): how many segments there are, the number of the CTA's if it begins one (else -1) and the CTA that
    // ends it
    int segments, ordinal, last;
};

template <int NT>
struct PlanScratch {
    int64_t warp[NT / 32 + 1];
    PlanStart start;
};

// The plan of CTA `cta` by one warp, a sequence a lane and all in 32 bits; false where there are more units than that allows.
// At most 32 sequences.  CTA 0 reports tables that do not fit, by the warp that `tells`.
template <class S>
__device__ __forceinline__ bool plan_warp(const SeqTables& t, const S& sp, int cta, int ctas, PlanStart& p, int64_t& first, int64_t& end,
                                          int32_t* status_word, bool tells) {
    const int lane = threadIdx.x & 31;
    bool bad = false;
    SeqInfo s = {};
    if (lane < t.num_seqs) s = load_seq(t, lane, bad);
    const int64_t wide = sp.units(s);
    if (!__all_sync(0xffffffffu, wide < (1 << 20))) return false;
    const uint32_t segments = (uint32_t)sp.segments(s), tiles = (uint32_t)sp.tiles(s), units = (uint32_t)wide, cost = sp.cost(s);
    const uint32_t total = __reduce_add_sync(0xffffffffu, units), costs = __reduce_add_sync(0xffffffffu, units * cost);
    auto pieces = [&](uint32_t m) { return segments * min(tiles, (tiles * cost + m - 1) / m); };
    uint32_t lo = costs > (uint32_t)ctas ? (costs + ctas - 1) / ctas : 1, hi = lo + S::kSwitch;
    const bool cut = __reduce_add_sync(0xffffffffu, pieces(hi)) <= (uint32_t)ctas;
    while (cut && lo < hi) {
        const uint32_t m = (lo + hi) >> 1;
        if (__reduce_add_sync(0xffffffffu, pieces(m)) <= (uint32_t)ctas) hi = m; else lo = m + 1;
    }
    // the lane's sequence has the CTAs (pieces) or the units (runs) [inc - mine, inc)
    const uint32_t mine = cut ? pieces(hi) : units;
    uint32_t inc = mine, units_inc = units, segments_inc = segments;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t n = __shfl_up_sync(0xffffffffu, inc, o), u = __shfl_up_sync(0xffffffffu, units_inc, o);
        const uint32_t g = __shfl_up_sync(0xffffffffu, segments_inc, o);
        if (lane >= o) {
            inc += n;
            units_inc += u;
            segments_inc += g;
        }
    }
    const uint32_t busy = total < (uint32_t)ctas ? total : ctas, each = busy ? total / busy : 0, extra = total - each * busy;
    auto run_first = [&](uint32_t c) { return c * each + (c < extra ? c : extra); };
    const uint32_t at = cut ? (uint32_t)cta : ((uint32_t)cta < busy ? run_first(cta) : total);
    const uint32_t found = __ballot_sync(0xffffffffu, at >= inc - mine && at < inc);
    const int b = found ? __ffs(found) - 1 : 0;
    p.s.begin = __shfl_sync(0xffffffffu, s.begin, b);
    p.s.len = __shfl_sync(0xffffffffu, s.len, b);
    p.s.node0 = __shfl_sync(0xffffffffu, s.node0, b);
    p.s.nodes = __shfl_sync(0xffffffffu, s.nodes, b);
    p.b = b;
    p.before = __shfl_sync(0xffffffffu, units_inc - units, b);
    p.units = total;
    p.segments = cut ? (int)__shfl_sync(0xffffffffu, segments_inc, 31) : -1;
    p.ordinal = p.last = -1;
    first = end = total;
    if (found && !cut) {
        first = at;
        end = run_first(cta + 1);
    }
    const uint32_t cta_first = __shfl_sync(0xffffffffu, inc - mine, b);
    const uint32_t segments_before = __shfl_sync(0xffffffffu, segments_inc - segments, b);
    if (found && cut) {
        const uint32_t n = (uint32_t)sp.tiles(p.s), of = min(n, (n * sp.cost(p.s) + hi - 1) / hi), local = at - cta_first;
        const uint32_t segment = local / of, piece = local - segment * of;
        first = p.before + segment * n + n * piece / of;
        end = p.before + segment * n + n * (piece + 1) / of;
        if (piece == 0) {
            p.ordinal = (int)(segments_before + segment);
            p.last = cta + (int)of - 1;
        }
    }
    if (cta == 0 && tells && bad) report(status_word, SHARPV_ERR_BOUNDS);
    return true;
}

// Every thread of the block (NT threads) gets the plan of this CTA, `first` its first unit and `end` the one behind
// its last.  CTA 0 reports tables that do not fit.
template <int NT, class S>
__device__ __forceinline__ PlanStart plan_cta(const SeqTables& t, const S& sp, int cta, int ctas,
                                              PlanScratch<NT>& sm, int64_t& first, int64_t& end, int32_t* status_word) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (t.num_seqs <= 32) {                     // every warp on its own with the same result
        PlanStart p;
        if (plan_warp(t, sp, cta, ctas, p, first, end, status_word, warp == 0)) {
            __syncthreads();                    // what was set up in front of the plan is seen
            return p;
        }
    }
    const int per = (t.num_seqs + NT - 1) / NT;
    const int lo = min(t.num_seqs, (int)threadIdx.x * per), hi = min(t.num_seqs, lo + per);
    int64_t sum = 0;
    bool bad = false;
    SeqInfo s = {};
    for (int b = lo; b < hi; ++b) {
        s = load_seq(t, b, bad);
        sum += sp.units(s);
    }
    int64_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t n = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += n;
    }
    if (lane == 31) sm.warp[warp] = inc;
    __syncthreads();
    int64_t run = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const int64_t v = sm.warp[w];
        if (w < warp) run += v;
        total += v;
    }
    const Deal deal(total, ctas);
    first = cta < deal.busy ? deal.first(cta) : total;
    end = cta < deal.busy ? deal.first(cta + 1) : total;
    if (first >= run && first < run + sum) {            // the sequence is among this thread's
        int b = lo;
        for (; per > 1; ++b) {
            s = load_seq(t, b, bad);
            const int64_t n = sp.units(s);
            if (first < run + n) break;
            run += n;
        }
        sm.start.s = s;
        sm.start.b = b;
        sm.start.before = run;
    }
    if (threadIdx.x == 0) {
        sm.start.units = total;
        sm.start.segments = sm.start.ordinal = sm.start.last = -1;
    }
    if (cta == 0 && bad) report(status_word, SHARPV_ERR_BOUNDS);
    __syncthreads();
    return sm.start;
}

// A portion: the units of one segment that one CTA works on.
struct Portion {
    SeqInfo s;
    int h, rt;                          // KV head, row tile
    int kt0, kt1;                       // key tiles of the portion
    int kt_all, kt_cache;               // of the segment; of those, tiles of cached rows
};

// Walks the portions of a CTA's units [u, end).
struct Walk {
    int64_t u, end, before;
    SeqInfo s;
    int b;
    __device__ __forceinline__ Walk(const PlanStart& p, int64_t first, int64_t last)
        : u(first), end(last), before(p.before), s(p.s), b(p.b) {}
    __device__ __forceinline__ bool next(const SeqTables& t, const Split& sp, Portion& p) {
        if (u >= end) return false;
        for (;;) {                              // sequences without nodes have no units
            const int64_t mine = sp.units(s);
            if (u - before < mine) break;
            before += mine;
            bool bad = false;
            s = load_seq(t, ++b, bad);
        }
        p.s = s;
        p.kt_all = sp.key_tiles(s);
        p.kt_cache = sp.cache_tiles(s);
        const int64_t seg = div64(u - before, p.kt_all);
        p.kt0 = (int)(u - before - seg * p.kt_all);
        p.kt1 = (int)min((int64_t)p.kt_all, p.kt0 + (end - u));
        const int rts = sp.row_tiles(s);
        p.h = (int)div64(seg, rts);
        p.rt = (int)(seg - (int64_t)p.h * rts);
        u += p.kt1 - p.kt0;
        return true;
    }
};

// Where a portion that is not a whole segment leaves its partial result: slot 1 of the CTA if it starts at the segment's
// first key tile, else slot 0.  A CTA has at most one of each.
__device__ __forceinline__ int portion_slot(int cta, int first_key_tile) { return cta * 2 + (first_key_tile == 0); }

// A segment whose first units CTA `first` has and whose last ones it has not (at most one a CTA): the CTAs first .. last hold
// its parts.  Noted at the segment's number where segments are cut into pieces, else at the CTA's.
struct SharedSegment {
    int node0, rows;                    // first node of the sequence, its query rows
    int h, rt;
    int first, last;                    // last -1: there is none
};
struct SharedHead {
    int pieces, segments;               // whether the notes go by segment, and how many there are
};

// 16 bytes from global to shared memory without passing registers; zeros where `valid` is false
__device__ __forceinline__ void cp_async16(void* smem, const void* gmem, bool valid) {
    const unsigned dst = (unsigned)__cvta_generic_to_shared(smem);
    const int n = valid ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(gmem), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async4(void* smem, const void* gmem) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"((unsigned)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ bool finite_f32(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// The layout checks of the calls that read a cache through its layout struct (the same as the compaction's).
template <class Ok>
inline sharpv_status kv_layout_status_if(const void* kv, const sharpv_kv_layout* L, Ok ok) {
    if (!kv || !L) return SHARPV_ERR_INVALID_ARG;
    if (!ok(L->dtype)) return SHARPV_ERR_UNSUPPORTED;
    if (L->num_layers < 1 || L->num_kv_heads < 1 || L->head_dim < 1 || L->stride_layer < 0 || L->stride_kv < 0 ||
        L->stride_head < 0 || L->stride_token < L->head_dim)
        return SHARPV_ERR_INVALID_ARG;
    const int64_t eb = elem_bytes(L->dtype);
    if ((L->head_dim * eb) % 16 || (L->stride_layer * eb) % 16 || (L->stride_kv * eb) % 16 ||
        (L->stride_head * eb) % 16 || (L->stride_token * eb) % 16 || !aligned16(kv))
        return SHARPV_ERR_UNSUPPORTED;
    return SHARPV_OK;
}

inline sharpv_status kv_layout_status(const void* kv, const sharpv_kv_layout* L, bool computes) {
    return kv_layout_status_if(kv, L, computes ? dtype_ok : copy_dtype_ok);
}

inline sharpv_status current_sms(int& sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}

}  // namespace sharpv
