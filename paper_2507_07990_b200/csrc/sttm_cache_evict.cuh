// Eviction from a paged cache by accumulated attention weight (sttm_cache_evict).
//
// k_cache_select: which slots of a (sequence, KV head) row stay.  One cluster per row.  Scores become
// 32-bit keys whose unsigned order is the order of the scores; a thread holds a stretch of neighbouring keys in
// registers.  The keep-th largest key is found by radix steps of 11, 11 and 10 bits: every CTA counts its
// keys, adds its counts to every CTA's totals, and after one cluster barrier all of them find the same bin.
// Then a prefix sum over threads (and CTAs) says where each thread's chosen slots go; they are put together
// in shared memory and written in one piece.  A row is read once (its chosen scores twice, the second time
// out of L2).  What bounds the kernel is the instructions per key (about 35, against some 150 when every
// stretch of a warp's keys was numbered by votes) and the five cluster barriers.
// k_cache_select_long: the same for rows beyond what a cluster's registers hold; the keys are read again for
// every step.
// k_cache_move: copies keys and values of the chosen slots to the destination's pages, in order:
// every row of 2 x dim channels is read and written once, HBM bounds it.
#pragma once

#include "sttm_cache.cuh"

namespace sttm {

constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelMaxCluster = 8;
constexpr int kSelBins = 2048;
constexpr int kSelMaxKeys = 33;                             // keys per thread at most (k_cache_select)
constexpr int kSelStrides = 32;                             // stretches of kSelThreads keys that k_cache_select_long numbers in one go
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
};

__device__ __forceinline__ int evict_length(const EvictArgs& a, int b) { return min(max(a.lengths[b], 0), a.max_len); }
// slots that stay: what is asked for, what there is, what fits
__device__ __forceinline__ int evict_keep(const EvictArgs& a, int b, int len) {
    return min(min(max(a.keep[b], 0), len), min(a.kept_width, a.dst.table_width * a.dst.page));
}

// A score's key: NaN, 1, before every number; -0 equals +0.  0 stands for no slot at all, all ones for a
// protected slot.
constexpr uint32_t kNoKey = 0u, kNanKey = 1u, kTopKey = 0xffffffffu;
__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? kNanKey : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
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

// Exclusive prefix sum over the block's threads, and the total.  Two counters travel in one number: the lower
// half and the upper half.
template <typename V>
__device__ __forceinline__ V block_scan(V v, V* warp_sums, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V x = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += x;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    V w = warp_sums[lane];                                  // kSelWarps = 32: every warp scans the warps' sums
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V x = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += x;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const V before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return s - v + (warp > 0 ? before : (V)0);
}
template <typename V>
__device__ __forceinline__ uint2 halves(V v) {
    constexpr int kHalf = sizeof(V) * 4;
    return make_uint2((uint32_t)(v & (((V)1 << kHalf) - 1)), (uint32_t)(v >> kHalf));
}

// What the threads of a select kernel share.
struct SelectShared {
    uint32_t hist[kSelBins], totals[3][kSelBins];           // counts of this CTA, and of the cluster per step
    unsigned long long warp_sums[kSelWarps];
    uint32_t found[2];                                      // bin, keys above it
    uint2 counts;                                           // this CTA's keys above the threshold, and equal to it
};

// The row and slice of a CTA; the outputs beyond what is kept.
struct SelectRow {
    int rank, size, len, keep, lo, n;                       // slice: slots lo ... lo + n - 1
    int first, last;
    const float* score;                                     // of the slice
    int32_t* kept;
    float* out;
    __device__ __forceinline__ bool is_protected(int i) const { return lo + i < first || lo + i >= len - last; }
    __device__ __forceinline__ uint32_t key(int i) const { return is_protected(i) ? kTopKey : score_key(score[i]); }
};

// `unit`: slices are multiples of so many slots
__device__ __forceinline__ SelectRow select_begin(const EvictArgs& a, SelectShared& sh, int unit) {
    SelectRow r;
    r.rank = (int)cluster_rank();
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r.size));
    for (int i = threadIdx.x; i < kSelBins; i += kSelThreads) sh.hist[i] = sh.totals[0][i] = sh.totals[1][i] = sh.totals[2][i] = 0;
    cluster_arrive();                                       // waited for before anything is added to another CTA's totals
    wait_for_prior_kernel();
    let_next_kernel_start();
    const int row = (int)cluster_id(), b = row / a.src.heads, h = row % a.src.heads;
    r.len = evict_length(a, b);
    r.keep = evict_keep(a, b, r.len);
    if (r.rank == 0 && threadIdx.x == 0) {
        if (h == 0) a.new_lengths[b] = r.keep;
        if (a.lengths[b] < 0 || a.lengths[b] > a.max_len) raise_status(a.status, kStatusCapacity);
        if (a.keep[b] > r.keep && r.keep < r.len) raise_status(a.status, kStatusCapacity);
    }
    const long long per = ((long long)r.len + (long long)r.size * unit - 1) / ((long long)r.size * unit) * unit;
    r.lo = (int)min((long long)r.len, r.rank * per);
    r.n = (int)min((long long)(r.len - r.lo), per);
    r.first = a.first;
    r.last = a.last;
    r.score = a.scores + b * a.score_seq + h * a.score_head + r.lo;
    r.kept = a.kept + (long long)row * a.kept_width;
    r.out = a.new_scores + (long long)row * a.kept_width;
    for (int i = r.keep + r.rank * kSelThreads + threadIdx.x; i < a.kept_width; i += r.size * kSelThreads) {
        r.kept[i] = -1;
        r.out[i] = 0.f;
    }
    return r;
}

// One radix step, after the CTA's keys under `prefix` were counted: into which bin the want-th largest of
// them falls.  Called by all threads; `prefix` and `want` become those of the next step.
__device__ __forceinline__ void select_step(SelectShared& sh, int size, int pass, int shift, uint32_t& prefix, uint32_t& want) {
    __syncthreads();
    if (size > 1) {
        for (int i = threadIdx.x; i < kSelBins; i += kSelThreads) {
            const uint32_t v = sh.hist[i];
            sh.hist[i] = 0;
            if (v != 0)
                for (int r = 0; r < size; r++) dsmem_add(map_to_rank(smem_u32(&sh.totals[pass][i]), r), v);
        }
        cluster_barrier();
    }
    // bins from the top: thread t holds bins kSelBins - 1 - 2 t and the one below.  The warps' sums say which warp
    // has the bin; that one looks closer.
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, top = kSelBins - 1 - 2 * (int)threadIdx.x;
    const uint32_t v0 = sh.totals[pass][top], v1 = sh.totals[pass][top - 1];
    uint32_t* warp_sums = reinterpret_cast<uint32_t*>(sh.warp_sums);
    const uint32_t mine = __reduce_add_sync(0xffffffffu, v0 + v1);
    if (lane == 0) warp_sums[warp] = mine;
    __syncthreads();
    const uint32_t w = warp_sums[lane];
    uint32_t upto = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    const int owner = __ffs(__ballot_sync(0xffffffffu, upto >= want)) - 1;
    if (warp == owner) {
        uint32_t up = v0 + v1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += x;
        }
        up += __shfl_sync(0xffffffffu, upto - w, owner) - (v0 + v1);     // keys above this thread's bins
        if (up < want && up + v0 >= want) {
            sh.found[0] = top;
            sh.found[1] = up;
        } else if (up + v0 < want && up + v0 + v1 >= want) {
            sh.found[0] = top - 1;
            sh.found[1] = up + v0;
        }
    }
    __syncthreads();
    prefix |= sh.found[0] << shift;
    want -= sh.found[1];
}

// {keys above the threshold, keys equal to it} in the CTAs before this one
__device__ __forceinline__ uint2 select_before(SelectShared& sh, const SelectRow& r, uint2 total) {
    uint2 before = make_uint2(0, 0);
    if (r.size == 1) return before;
    if (threadIdx.x == 0) sh.counts = total;
    cluster_barrier();
    // a lane per CTA before this one
    const int k = threadIdx.x & 31;
    if (k < r.rank) {
        const uint32_t at = map_to_rank(smem_u32(&sh.counts), k);
        before = make_uint2(dsmem_load(at), dsmem_load(at + 4));
    }
    return make_uint2(__reduce_add_sync(0xffffffffu, before.x), __reduce_add_sync(0xffffffffu, before.y));
}

// the radix steps: bits that the steps before have fixed, lowest bit of the step's digit, its mask
__device__ __forceinline__ constexpr uint32_t step_above(int pass) { return pass == 0 ? 0u : (pass == 1 ? 0xffe00000u : 0xfffffc00u); }
__device__ __forceinline__ constexpr int step_shift(int pass) { return pass == 0 ? 21 : (pass == 1 ? 10 : 0); }
__device__ __forceinline__ constexpr uint32_t step_digit(int pass) { return pass == 2 ? 1023u : 2047u; }

// KPT: keys per thread (odd: stretches of an odd number of words meet no bank conflict)
template <int KPT>
__global__ void __launch_bounds__(kSelThreads) k_cache_select(const __grid_constant__ EvictArgs a) {
    static_assert(kSelWarps == 32 && kSelBins == 2 * kSelThreads && KPT % 2 == 1, "");
    extern __shared__ uint32_t keys[];                      // [KPT * kSelThreads]: the slice's keys, later its chosen slots
    __shared__ SelectShared sh;
    const SelectRow r = select_begin(a, sh, 1);
    const int per = ((r.n + kSelThreads - 1) / kSelThreads) | 1;        // <= KPT
    uint32_t* const first_counts = r.size > 1 ? sh.hist : sh.totals[0];
    __syncthreads();
    // (the first step counts the keys while they are made)
    if (r.first > r.lo || r.len - r.last < r.lo + r.n) {
#pragma unroll 4
        for (int i = threadIdx.x; i < r.n; i += kSelThreads) {
            const uint32_t k = r.key(i);
            keys[i] = k;
            atomicAdd(&first_counts[k >> step_shift(0)], 1u);
        }
    } else {
#pragma unroll 8
        for (int i = threadIdx.x; i < r.n; i += kSelThreads) {
            const uint32_t k = score_key(r.score[i]);
            keys[i] = k;
            atomicAdd(&first_counts[k >> step_shift(0)], 1u);
        }
    }
    cluster_wait();
    if (r.keep > 0) {
        uint32_t threshold = 0, want = (uint32_t)r.keep;    // want: rank of the threshold among the keys under the prefix
        select_step(sh, r.size, 0, step_shift(0), threshold, want);
        uint32_t k[KPT];
#pragma unroll
        for (int c = 0; c < KPT; c++) k[c] = c < per && (int)threadIdx.x * per + c < r.n ? keys[threadIdx.x * per + c] : kNoKey;
#pragma unroll
        for (int pass = 1; pass < 3; pass++) {
            uint32_t* counted = r.size > 1 ? sh.hist : sh.totals[pass];
#pragma unroll
            for (int c = 0; c < KPT; c++)
                if ((k[c] & step_above(pass)) == threshold) atomicAdd(&counted[(k[c] >> step_shift(pass)) & step_digit(pass)], 1u);
            select_step(sh, r.size, pass, step_shift(pass), threshold, want);
        }
        // all keys above the threshold stay, and of those equal to it the `want` with the lowest slots
        uint32_t mine = 0, sum;                             // keys above | keys equal << 16
#pragma unroll
        for (int c = 0; c < KPT; c++) mine += (k[c] > threshold ? 1u : 0u) + (k[c] == threshold ? 0x10000u : 0u);
        static_assert(KPT * kSelThreads < 0x10000, "counts of a CTA fit 16 bits");
        const uint2 at = halves(block_scan(mine, reinterpret_cast<uint32_t*>(sh.warp_sums), sum)), total = halves(sum);
        const uint2 before = select_before(sh, r, total);
        const uint32_t base = before.x + min(before.y, want), chosen = before.x + total.x + min(before.y + total.y, want) - base;
        uint32_t to = at.x + before.x - base, e = at.y + before.y;      // place in this CTA's list: to + min(e, want)
#pragma unroll
        for (int c = 0; c < KPT; c++) {
            const bool more = k[c] > threshold, equal = k[c] == threshold;
            if (more || (equal && e < want)) keys[to + min(e, want)] = threadIdx.x * per + c;
            to += more;
            e += equal;
        }
        __syncthreads();
        for (uint32_t i0 = threadIdx.x; i0 < chosen; i0 += 4 * kSelThreads) {       // (four scores on their way at once)
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (i0 + u * kSelThreads < chosen) x[u] = __ldcg(r.score + (int)keys[i0 + u * kSelThreads]);
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const uint32_t i = i0 + u * kSelThreads;
                if (i < chosen) {
                    r.kept[base + i] = r.lo + (int)keys[i];
                    r.out[base + i] = x[u];
                }
            }
        }
    }
    if (r.size > 1) cluster_barrier();                      // nobody leaves while its counts may be read
}

__global__ void __launch_bounds__(kSelThreads) k_cache_select_long(const __grid_constant__ EvictArgs a) {
    __shared__ SelectShared sh;
    __shared__ uint2 numbers[kSelStrides * kSelWarps];      // keys above the threshold and equal to it, per stretch and warp; then prefix sums
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const SelectRow r = select_begin(a, sh, kSelThreads);
    cluster_wait();
    if (r.keep > 0) {
        uint32_t threshold = 0, want = (uint32_t)r.keep;
        __syncthreads();
#pragma unroll 1
        for (int pass = 0; pass < 3; pass++) {
            uint32_t* counted = r.size > 1 ? sh.hist : sh.totals[pass];
#pragma unroll 4
            for (int i = threadIdx.x; i < r.n; i += kSelThreads) {
                const uint32_t k = r.key(i);
                if ((k & step_above(pass)) == threshold) atomicAdd(&counted[(k >> step_shift(pass)) & step_digit(pass)], 1u);
            }
            select_step(sh, r.size, pass, step_shift(pass), threshold, want);
        }
        unsigned long long mine = 0, sum;                   // keys above | keys equal << 32
#pragma unroll 4
        for (int i = threadIdx.x; i < r.n; i += kSelThreads) {
            const uint32_t k = r.key(i);
            mine += (k > threshold ? 1ull : 0ull) + (k == threshold ? 1ull << 32 : 0ull);
        }
        block_scan(mine, sh.warp_sums, sum);
        uint2 before = select_before(sh, r, halves(sum));
        for (int from = 0; from < r.n; from += kSelStrides * kSelThreads) {
            const int strides = min(kSelStrides, (r.n - from + kSelThreads - 1) / kSelThreads);
            for (int c = 0; c < strides; c++) {
                const int i = from + c * kSelThreads + threadIdx.x;
                const uint32_t k = i < r.n ? r.key(i) : 0u;
                const uint32_t m = __ballot_sync(0xffffffffu, i < r.n && k > threshold), e = __ballot_sync(0xffffffffu, i < r.n && k == threshold);
                if (lane == 0) numbers[c * kSelWarps + warp] = make_uint2(__popc(m), __popc(e));
            }
            __syncthreads();
            // prefix sums in the order of the slots: stretches, their warps
            static_assert(kSelStrides * kSelWarps == kSelThreads, "one entry per thread");
            const uint2 own = (int)threadIdx.x < strides * kSelWarps ? numbers[threadIdx.x] : make_uint2(0, 0);
            numbers[threadIdx.x] = halves(block_scan((unsigned long long)own.y << 32 | own.x, sh.warp_sums, sum));
            __syncthreads();
            for (int c = 0; c < strides; c++) {
                const int i = from + c * kSelThreads + threadIdx.x;
                const uint32_t k = i < r.n ? r.key(i) : 0u;
                const uint32_t m = __ballot_sync(0xffffffffu, i < r.n && k > threshold), e = __ballot_sync(0xffffffffu, i < r.n && k == threshold);
                const uint2 base = numbers[c * kSelWarps + warp];
                const uint32_t below = (1u << lane) - 1;
                const uint32_t mb = before.x + base.x + __popc(m & below), eb = before.y + base.y + __popc(e & below);
                if (i < r.n && (k > threshold || (k == threshold && eb < want))) {
                    const uint32_t to = mb + min(eb, want);
                    r.kept[to] = r.lo + i;
                    r.out[to] = r.score[i];
                }
            }
            before.x += halves(sum).x;
            before.y += halves(sum).y;
            __syncthreads();                                // (numbers is written again)
        }
    }
    if (r.size > 1) cluster_barrier();
}

// A block takes stretches of SLOTS kept slots: the first threads look up where each of them lies and
// goes, then all copy, eight 16-byte words per thread in flight.
constexpr int kMoveWords = 8;

template <int DIM>
__global__ void __launch_bounds__(kMoveThreads) k_cache_move(const __grid_constant__ EvictArgs a, int chunks) {
    constexpr int WORDS = DIM / 8;                          // 16-byte words of a slot's keys (and of its values)
    constexpr int SLOTS = kMoveWords * kMoveThreads / (2 * WORDS);
    __shared__ long long from_at[SLOTS], to_at[SLOTS];
    wait_for_prior_kernel();
    let_next_kernel_start();
    const int row = blockIdx.x / chunks, b = row / a.src.heads, h = row % a.src.heads;
    const int keep = evict_keep(a, b, evict_length(a, b));
    // half of the threads copy keys, half values
    const int word = threadIdx.x % WORDS, values = threadIdx.x / WORDS % 2, sub = threadIdx.x / (2 * WORDS);
    const uint4* from = reinterpret_cast<const uint4*>((values ? a.src.v : a.src.k) + h * a.src.head_stride) + word;
    uint4* to = reinterpret_cast<uint4*>((values ? a.dst.v : a.dst.k) + h * a.dst.head_stride) + word;
    const int32_t* kept = a.kept + (long long)row * a.kept_width;
    for (int i0 = (blockIdx.x % chunks) * SLOTS; i0 < keep; i0 += chunks * SLOTS) {
        for (int s = threadIdx.x; s < SLOTS; s += kMoveThreads) {
            long long f = -1, t = -1;
            if (i0 + s < keep) {
                f = slot_at(a.src, b, kept[i0 + s], a.status);
                t = slot_at(a.dst, b, i0 + s, a.status);
            }
            from_at[s] = f < 0 || t < 0 ? -1 : f / 8;
            to_at[s] = t / 8;
        }
        __syncthreads();
        uint4 x[kMoveWords];
#pragma unroll
        for (int w = 0; w < kMoveWords; w++) {
            const long long f = from_at[w * (SLOTS / kMoveWords) + sub];
            if (f >= 0) x[w] = __ldcs(from + f);
        }
#pragma unroll
        for (int w = 0; w < kMoveWords; w++) {
            const int s = w * (SLOTS / kMoveWords) + sub;
            if (from_at[s] >= 0) to[to_at[s]] = x[w];
        }
        __syncthreads();
    }
}

}  // namespace sttm
