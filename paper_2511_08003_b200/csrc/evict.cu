// The cached tokens that stay when a sequence is over its budget (sharpv_evict_select).
//
// A sequence's k-th key is found by counting, eight bits at a time from the top (the key is the monotone 32-bit
// image of the mass), by a cluster of CTAs that share the sequence's rows in contiguous slices: every CTA counts
// its slice in shared memory, and all read one another's counts.  The rows above the k-th key stay, and of those equal
// to it the first ones; the warps' and slices' counts give every warp the place where its survivors go.
// What bounds it is latency: a CTA walks its slice seven times (once to read it, a time a round, once to count the survivors,
// once to write them), with a barrier of the cluster a round and two behind the count.  The keys are read from memory
// once and kept in shared memory (slices too long for that are read again every time), and in the first round lanes of a
// warp that count the same digit (weights span few powers of two) count it with one atomic.
#include <cooperative_groups.h>

#include "decode_common.cuh"

namespace sharpv {
namespace {

constexpr int kEvictThreads = 512;
constexpr int kEvictCluster = 8;
constexpr int kBins = 256;
constexpr int kKeyRoom = 24 * 1024;     // keys of a slice in shared memory: 96 KB, two CTAs on an SM

struct EvictArgs {
    const float* mass;
    int64_t cache_tokens;
    int num_seqs;
    const int32_t* begin;
    const int32_t* len;
    const int32_t* budget;
    int sink, recent;
    int32_t* kept_pos;
    int32_t* kept_offsets;
    float* out_mass;
    int64_t capacity;
    int key_room;               // keys of a slice that shared memory holds
    int32_t* status_word;
};

// NaN of either sign ranks above +inf
__device__ __forceinline__ uint32_t mass_key(float x) { return x != x ? 0xffffffffu : order_key(x); }

// rows of sequence b and how many of them stay
__device__ __forceinline__ void seq_rows(const EvictArgs& a, int b, int64_t& begin, int& len, int& keep, bool& bad) {
    const int64_t b0 = __ldg(a.begin + b), l0 = __ldg(a.len + b);
    begin = b0 < 0 ? 0 : (b0 > a.cache_tokens ? a.cache_tokens : b0);
    int64_t l = b0 < 0 || l0 < 0 ? 0 : l0;
    if (l > a.cache_tokens - begin) l = a.cache_tokens - begin;
    bad = bad || begin != b0 || l != l0;
    len = (int)l;
    keep = min(max(__ldg(a.budget + b), 0), len);
}

// One cluster per sequence.  Measured: 16 ragged sequences (37,712 rows) 10.5 us, one of 50,432 rows 21 us.  Of that, by time
// stamps from cold caches (10.9 and 22.3 us): tables and slice read 1.7 and 3.2, four rounds 5.0 and 10.6, survivors counted
// and exchanged 2.3 and 3.3, written 0.5 and 5.1.
__global__ void __cluster_dims__(kEvictCluster, 1, 1) __launch_bounds__(kEvictThreads)
evict_select_kernel(const __grid_constant__ EvictArgs a) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ uint32_t keys[];
    constexpr int kWarps = kEvictThreads / 32;
    __shared__ int hist[2][kBins];
    __shared__ int total[kBins];
    __shared__ int counts[2];                   // rows of the slice above the k-th key, and equal to it
    __shared__ int warp_up[kWarps], warp_eq[kWarps];
    __shared__ int64_t base_part[kEvictThreads / 32];
    __shared__ int pick[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster.block_rank();
    const int b = blockIdx.x / kEvictCluster;
    cudaGridDependencySynchronize();
    bool bad = false;
    int64_t begin;
    int len, keep;
    // survivors of the sequences in front of this one
    int64_t sum = 0;
    for (int i = tid; i < b; i += kEvictThreads) {
        seq_rows(a, i, begin, len, keep, bad);
        sum += keep;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) base_part[warp] = sum;
    for (int i = tid; i < 2 * kBins; i += kEvictThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    int64_t base = 0;
#pragma unroll
    for (int w = 0; w < kEvictThreads / 32; ++w) base += base_part[w];
    bad = false;
    seq_rows(a, b, begin, len, keep, bad);
    if (rank == 0 && tid == 0) {
        if (bad) report(a.status_word, SHARPV_ERR_BOUNDS);
        // a running count past 2^31 - 1 saturates (it is over any capacity then)
        a.kept_offsets[b] = (int32_t)min(base, (int64_t)INT32_MAX);
        if (b == a.num_seqs - 1) {
            a.kept_offsets[b + 1] = (int32_t)min(base + keep, (int64_t)INT32_MAX);
            if (base + keep > a.capacity) report(a.status_word, SHARPV_ERR_CAPACITY);
        }
    }
    // Protected rows: [0, s_end) and [r_begin, len).  If they alone reach the budget the choice is among them, else they
    // all stay and the choice is among the others.
    const int s_end = min(a.sink, len), r_begin = max(s_end, len - min(a.recent, len));
    const int guarded = s_end + (len - r_begin);
    const bool among_guarded = guarded > keep;
    const int want = among_guarded ? keep : keep - guarded;         // rows to choose
    const int choice = among_guarded ? guarded : len - guarded;     // out of so many
    const bool choose = want > 0 && want < choice;
    // contiguous slice of this CTA
    const int lo = (int)((int64_t)len * rank / kEvictCluster), hi = (int)((int64_t)len * (rank + 1) / kEvictCluster);
    const float* mass = a.mass + begin;
    const bool kept_here = hi - lo <= a.key_room;
    if (kept_here) {
#pragma unroll 4
        for (int i = lo + tid; i < hi; i += kEvictThreads) keys[i - lo] = mass_key(__ldg(mass + i));
        __syncthreads();
    }
    auto key_of = [&](int i) { return kept_here ? keys[i - lo] : mass_key(__ldg(mass + i)); };
    uint32_t prefix = 0, need = (uint32_t)want;                      // the k-th key's known bits; rank among those that share them
    if (choose) {                                                    // the same in every CTA of the cluster
#pragma unroll 1
        for (int pass = 0; pass < 4; ++pass) {
            const int shift = 24 - 8 * pass;
            int* h = hist[pass & 1];
            for (int i0 = lo; i0 < hi; i0 += kEvictThreads) {
                const int i = i0 + tid;
                const uint32_t key = i < hi ? key_of(i) : 0u;
                const bool in = i < hi && (i < s_end || i >= r_begin) == among_guarded && (pass == 0 || key >> (shift + 8) == prefix);
                if (pass == 0) {
                    const int digit = in ? (int)(key >> 24) : kBins;
                    const uint32_t same = __match_any_sync(0xffffffffu, digit);
                    if (in && lane == __ffs(same) - 1) atomicAdd(&h[digit], __popc(same));
                } else if (in) {
                    atomicAdd(&h[key >> shift & 255], 1);
                }
            }
            cluster.sync();
            if (tid < kBins) {
                int t = 0;
#pragma unroll
                for (int r = 0; r < kEvictCluster; ++r) t += cluster.map_shared_rank(h, r)[tid];
                total[tid] = t;
            } else if (tid < 2 * kBins) {
                hist[(pass + 1) & 1][tid - kBins] = 0;               // read by nobody since the sync of the pass before
            }
            __syncthreads();
            // bin of the k-th key: the largest d with (rows in bins above d) < need <= (rows in bins d and above)
            if (warp == 0) {
                int mine[8], s = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) { mine[i] = total[255 - (lane * 8 + i)]; s += mine[i]; }
                int inc = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int n = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += n;
                }
                int run = inc - s;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (run < (int)need && (int)need <= run + mine[i]) { pick[0] = 255 - (lane * 8 + i); pick[1] = (int)need - run; }
                    run += mine[i];
                }
            }
            __syncthreads();
            prefix = prefix << 8 | (uint32_t)pick[0];
            need = (uint32_t)pick[1];
        }
    }
    // A row stays if it is protected (and all of those stay), or a candidate above the k-th key, or among the first
    // `need` candidates equal to it.
    auto state = [&](int i) {                   // 2: stays, 1: equal to the k-th key, 0: goes
        const bool guard = i < s_end || i >= r_begin;
        if (guard != among_guarded) return guard ? 2 : 0;
        if (!choose) return want > 0 ? 2 : 0;
        const uint32_t key = key_of(i);
        return key > prefix ? 2 : (key == prefix ? 1 : 0);
    };
    // contiguous piece of this warp, counted first, written then
    const int n = hi - lo;
    const int w_lo = lo + (int)((int64_t)n * warp / kWarps), w_hi = lo + (int)((int64_t)n * (warp + 1) / kWarps);
    int up = 0, eq = 0;
#pragma unroll 4
    for (int x = w_lo; x < w_hi; x += 32) {
        const int st = x + lane < w_hi ? state(x + lane) : 0;
        up += __popc(__ballot_sync(0xffffffffu, st == 2));
        eq += __popc(__ballot_sync(0xffffffffu, st == 1));
    }
    if (lane == 0) { warp_up[warp] = up; warp_eq[warp] = eq; }
    __syncthreads();
    int up_before = 0, eq_before = 0, up_all = 0, eq_all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) { up_before += warp_up[w]; eq_before += warp_eq[w]; }
        up_all += warp_up[w];
        eq_all += warp_eq[w];
    }
    if (tid == 0) { counts[0] = up_all; counts[1] = eq_all; }
    cluster.sync();
#pragma unroll
    for (int r = 0; r < kEvictCluster; ++r) {
        const int* c = cluster.map_shared_rank(counts, r);
        const int c0 = c[0], c1 = c[1];
        if (r < rank) { up_before += c0; eq_before += c1; }
    }
    cluster.sync();                             // nobody leaves while its counts are read
    int64_t at = base + up_before + min(eq_before, (int)need);
    for (int x = w_lo; x < w_hi; x += 32) {
        const int i = x + lane;
        const int st = i < w_hi ? state(i) : 0;
        const uint32_t below = (1u << lane) - 1u;
        const uint32_t equal = __ballot_sync(0xffffffffu, st == 1);
        const bool stays = st == 2 || (st == 1 && eq_before + __popc(equal & below) < (int)need);
        const uint32_t all = __ballot_sync(0xffffffffu, stays);
        const int64_t j = at + __popc(all & below);
        if (stays && j < a.capacity) {
            a.kept_pos[j] = (int32_t)(begin + i);
            if (a.out_mass) a.out_mass[j] = __ldg(mass + i);
        }
        at += __popc(all);
        eq_before += __popc(equal);
    }
}

}  // namespace
}  // namespace sharpv

using namespace sharpv;

extern "C" sharpv_status sharpv_evict_select(
    const float* mass, int64_t cache_tokens, int32_t num_seqs, const int32_t* seq_begin, const int32_t* seq_len,
    const int32_t* budget, int32_t sink, int32_t recent, int32_t* out_kept_pos, int32_t* out_kept_seq_offsets,
    float* out_mass, int64_t capacity, int32_t* status_word, void* cuda_stream) {
    if (cache_tokens < 0 || num_seqs < 0 || sink < 0 || recent < 0 || capacity < 0 || !out_kept_seq_offsets)
        return SHARPV_ERR_INVALID_ARG;
    if (cache_tokens >= (int64_t)1 << 31 || num_seqs > (INT32_MAX / kEvictCluster)) return SHARPV_ERR_UNSUPPORTED;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (num_seqs == 0)
        return cudaMemsetAsync(out_kept_seq_offsets, 0, sizeof(int32_t), stream) == cudaSuccess ? SHARPV_OK
                                                                                                : SHARPV_ERR_CUDA;
    if (!seq_begin || !seq_len || !budget || (cache_tokens > 0 && !mass) || (capacity > 0 && !out_kept_pos))
        return SHARPV_ERR_INVALID_ARG;
    if (out_mass && mass && out_mass < mass + cache_tokens && mass < out_mass + capacity) return SHARPV_ERR_INVALID_ARG;
    // room for a slice of the longest sequence that the cache can hold, up to kKeyRoom
    const int64_t slice = (cache_tokens + kEvictCluster - 1) / kEvictCluster + 1;
    const int room = (int)(slice < kKeyRoom ? slice : kKeyRoom);
    EvictArgs a = {mass, cache_tokens, num_seqs, seq_begin, seq_len, budget, sink, recent,
                   out_kept_pos, out_kept_seq_offsets, out_mass, capacity, room, status_word};
    if (cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeyRoom * 4) != cudaSuccess ||
        launch_dependent(evict_select_kernel, dim3((unsigned)num_seqs * kEvictCluster), dim3(kEvictThreads), (size_t)room * 4, stream, a) !=
        cudaSuccess) {
        (void)cudaGetLastError();
        return SHARPV_ERR_CUDA;
    }
    return SHARPV_OK;
}
