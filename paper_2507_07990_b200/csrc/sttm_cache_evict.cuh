// Eviction from a paged cache by accumulated attention weight (sttm_cache_evict).
//
// k_cache_select: which slots of a (sequence, KV head) row stay.  One cluster per row; its CTAs hold
// the row's scores in shared memory as 32-bit keys whose unsigned order is the order of the scores,
// find the keep-th largest key by radix steps of 11, 11 and 10 bits (a histogram per step, added up in
// the first CTA's shared memory), then every CTA numbers its chosen slots and writes them in order.  A row
// is read once; what it costs beyond that is a few cluster barriers.
// k_cache_move: copies keys and values of the chosen slots to the destination's pages, in order:
// every row of 2 x dim channels is read and written once, HBM bounds it.
#pragma once

#include "sttm_cache.cuh"

namespace sttm {

constexpr int kSelThreads = 512;
constexpr int kSelMaxCluster = 8;
constexpr int kSelBins = 2048;
constexpr int kMoveThreads = 256;

struct EvictArgs {
    CacheView src, dst;
    const int32_t *lengths, *keep;
    int max_len, first, last, kept_width;
    const float* scores;
    long long score_seq, score_head;
    int32_t* new_lengths;
    int32_t* kept;                // [seqs * heads][kept_width]
    float* new_scores;            // [seqs * heads][kept_width]
    int32_t* status;
    int slice_cap;                // keys a CTA can hold in shared memory
};

__device__ __forceinline__ int evict_length(const EvictArgs& a, int b) { return min(max(a.lengths[b], 0), a.max_len); }
// slots that stay: what is asked for, what there is, what fits
__device__ __forceinline__ int evict_keep(const EvictArgs& a, int b, int len) {
    return min(min(max(a.keep[b], 0), len), min(a.kept_width, a.dst.table_width * a.dst.page));
}

// A slot's key.  Protected slots come before all others, NaN after all others, -0 equals +0.
__device__ __forceinline__ uint32_t score_key(float x, bool is_protected) {
    if (is_protected) return 0xffffffffu;
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ void dsmem_add(uint32_t cluster_addr, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t dsmem_load(uint32_t cluster_addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    cluster_arrive();
    cluster_wait();
}

// inclusive prefix sum over the block (kSelThreads threads); total in `total`
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums, uint32_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kSelThreads / 32; w++) {
        if (w < warp) before += warp_sums[w];
        sum += warp_sums[w];
    }
    total = sum;
    return v + before;
}

__global__ void __launch_bounds__(kSelThreads) k_cache_select(const __grid_constant__ EvictArgs a) {
    extern __shared__ uint32_t keys[];                      // [slice_cap], this CTA's slots
    __shared__ uint32_t hist[kSelBins];
    __shared__ uint32_t warp_sums[kSelThreads / 32];
    __shared__ uint32_t found[2];                           // bin, keys above it: the first CTA's answer
    __shared__ uint32_t counts[2];                          // chosen above the threshold / equal to it, in this CTA
    const int rank = (int)cluster_rank();
    int size;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    wait_for_prior_kernel();
    let_next_kernel_start();
    const int row = (int)cluster_id(), b = row / a.src.heads, h = row % a.src.heads;
    const int len = evict_length(a, b), keep = evict_keep(a, b, len);
    if (rank == 0 && threadIdx.x == 0) {
        if (h == 0) a.new_lengths[b] = keep;
        if (a.lengths[b] < 0 || a.lengths[b] > a.max_len) raise_status(a.status, kStatusCapacity);
        if (a.keep[b] > keep && keep < len) raise_status(a.status, kStatusCapacity);
    }
    // contiguous slices, an odd number of slots per thread (its slots are neighbours: no bank conflicts)
    int per_thread = (len + size * kSelThreads - 1) / (size * kSelThreads);
    per_thread |= 1;
    const int slice = per_thread * kSelThreads;
    const int lo = min(len, rank * slice), n = min(len, lo + slice) - lo;
    const float* score = a.scores + b * a.score_seq + h * a.score_head;
    auto fresh_key = [&](int i) { return score_key(score[lo + i], lo + i < a.first || lo + i >= len - a.last); };
    for (int i = threadIdx.x; i < min(n, a.slice_cap); i += kSelThreads) keys[i] = fresh_key(i);
    auto key_at = [&](int i) { return i < a.slice_cap ? keys[i] : fresh_key(i); };

    int32_t* kept = a.kept + (long long)row * a.kept_width;
    float* out = a.new_scores + (long long)row * a.kept_width;
    for (int i = keep + rank * kSelThreads + threadIdx.x; i < a.kept_width; i += size * kSelThreads) {
        kept[i] = -1;
        out[i] = 0.f;
    }

    // the keep-th largest key, 11 + 11 + 10 bits from the top
    uint32_t prefix = 0, want = (uint32_t)keep;             // want: rank of the threshold among the keys under the prefix
    const uint32_t hist0 = map_to_rank(smem_u32(hist), 0);
    if (keep > 0) {
        int shift = 21, bits = 11;
#pragma unroll 1
        for (int pass = 0; pass < 3; pass++) {
            for (int i = threadIdx.x; i < kSelBins; i += kSelThreads) hist[i] = 0;
            cluster_barrier();
            const uint32_t above = pass == 0 ? 0u : 0xffffffffu << (shift + bits);
            for (int i = threadIdx.x; i < n; i += kSelThreads) {
                const uint32_t k = key_at(i);
                if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
            }
            if (size > 1) {
                __syncthreads();
                if (rank != 0)
                    for (int i = threadIdx.x; i < kSelBins; i += kSelThreads)
                        if (hist[i] != 0) dsmem_add(hist0 + 4 * i, hist[i]);
                cluster_barrier();
            } else {
                __syncthreads();
            }
            if (rank == 0) {
                // bins from the top: thread t holds the four bins below kSelBins - 4 t
                uint32_t v[4], sum = 0, total;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    v[e] = hist[kSelBins - 1 - 4 * threadIdx.x - e];
                    sum += v[e];
                }
                uint32_t up = block_scan(sum, warp_sums, total) - sum;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    if (up < want && up + v[e] >= want) {
                        found[0] = kSelBins - 1 - 4 * threadIdx.x - e;
                        found[1] = up;
                    }
                    up += v[e];
                }
            }
            cluster_barrier();
            const uint32_t f0 = map_to_rank(smem_u32(found), 0);
            const uint32_t bin = dsmem_load(f0), over = dsmem_load(f0 + 4);
            prefix |= bin << shift;
            want -= over;
            bits = pass == 1 ? 10 : 11;
            shift = pass == 0 ? 10 : 0;
        }
    }
    static_assert(kSelBins == 4 * kSelThreads, "four bins per thread");

    // all keys above the threshold stay, and of those equal to it the `want` with the lowest slots
    const uint32_t threshold = prefix;
    const int from = min(n, (int)threadIdx.x * per_thread), to = keep > 0 ? min(n, from + per_thread) : from;
    uint32_t more = 0, equal = 0;
    for (int i = from; i < to; i++) {
        const uint32_t k = key_at(i);
        more += k > threshold;
        equal += k == threshold;
    }
    uint32_t more_all, equal_all;
    const uint32_t more_before = block_scan(more, warp_sums, more_all) - more;
    const uint32_t equal_before = block_scan(equal, warp_sums, equal_all) - equal;
    if (threadIdx.x == 0) {
        counts[0] = more_all;
        counts[1] = equal_all;
    }
    cluster_barrier();
    uint32_t m = more_before, e = equal_before;
    for (int r = 0; r < rank; r++) {
        const uint32_t at = map_to_rank(smem_u32(counts), r);
        m += dsmem_load(at);
        e += dsmem_load(at + 4);
    }
    for (int i = from; i < to; i++) {
        const uint32_t k = key_at(i);
        if (k > threshold || (k == threshold && e < want)) {
            const uint32_t at = m + min(e, want);
            kept[at] = lo + i;
            out[at] = score[lo + i];
        }
        m += k > threshold;
        e += k == threshold;
    }
    cluster_barrier();                                      // nobody leaves while its counts may be read
}

template <int DIM>
__global__ void __launch_bounds__(kMoveThreads) k_cache_move(const __grid_constant__ EvictArgs a, int chunks) {
    constexpr int WORDS = DIM / 8;                          // 16-byte words of a slot's keys (and of its values)
    constexpr int SLOTS = kMoveThreads / (2 * WORDS);       // slots in one go: half of the threads copy keys, half values
    constexpr int STEPS = 4;                                // loads in flight per thread
    wait_for_prior_kernel();
    let_next_kernel_start();
    const int row = blockIdx.x / chunks, b = row / a.src.heads, h = row % a.src.heads;
    const int keep = evict_keep(a, b, evict_length(a, b));
    const int word = threadIdx.x % WORDS, values = threadIdx.x / WORDS % 2, sub = threadIdx.x / (2 * WORDS);
    const uint4* from = reinterpret_cast<const uint4*>((values ? a.src.v : a.src.k) + h * a.src.head_stride) + word;
    uint4* to = reinterpret_cast<uint4*>((values ? a.dst.v : a.dst.k) + h * a.dst.head_stride) + word;
    const int32_t* kept = a.kept + (long long)row * a.kept_width;
    const bool speaks = word == 0 && values == 0;
    for (int i0 = (blockIdx.x % chunks) * SLOTS * STEPS; i0 < keep; i0 += chunks * SLOTS * STEPS) {
        long long src[STEPS], dst[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            const int i = i0 + s * SLOTS + sub;
            src[s] = dst[s] = -1;
            if (i < keep) {
                src[s] = slot_at(a.src, b, kept[i], speaks ? a.status : nullptr);
                dst[s] = slot_at(a.dst, b, i, speaks ? a.status : nullptr);
            }
        }
        uint4 x[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; s++)
            if (src[s] >= 0 && dst[s] >= 0) x[s] = from[src[s] / 8];
#pragma unroll
        for (int s = 0; s < STEPS; s++)
            if (src[s] >= 0 && dst[s] >= 0) to[dst[s] / 8] = x[s];
    }
}

}  // namespace sttm
