// Attention of one new token per sequence over its paged cache (sttm_cache_attend).
//
//   out[b, h] = sum_s p[h, s] v[s],   p[h, s] = exp(scale q[h] . k[s]) / sum of the same over s
//
// over the slots s of sequence b that its length and its mask leave.  Keys and values are read once
// and everything else is small, so HBM bounds the kernel as long as the products keep up: the group of
// query heads that share a KV head forms the rows of one small matrix product per 16 slots.
//
// *Split.*  Two ways, by the rule in plan_attend().  Equal shares: the slots of all (sequence, KV head) rows are cut
// into tiles and laid end to end; CTA i takes the i-th of equal shares, whatever rows they belong to.  So one long
// sequence or many ragged ones keep every SM streaming equally long; a row that lies in several shares leaves a running
// maximum, a sum and an unscaled output per share, joined in share order by k_cache_join (no atomics: the bits of a
// result do not depend on scheduling).  Clusters: a row is cut evenly over the 1 to 16 CTAs of a cluster, which join
// their parts in shared memory, one launch in all.  5338 slots of 4 KV heads, out of HBM: 12.5 us in clusters of 16, 13.4 us in
// shares.
//
// *Pipeline.*  A producer warp brings a tile's keys and values (32 KB) into a ring of shared-memory stages by tensor
// copies, one box of slots that lie in one page per copy, under the 128-byte swizzle; boxes whose slots are all masked
// are not copied.  Four warps take 32 slots at a time and never wait for one another before the end of a row: each keeps
// its own maximum, sum and output.  32 x 32700 slots of 8 KV heads (4.3 GB) stream in 609 us, 7.0 TB/s, as fast as this memory
// reads; with scores (their logits are written and read once more, 0.5 GB) the call takes 747 to 789 us.
//
// *Products.*  S = Q K^T and O += P V on mma.sync m16n8k16 with fp32 sums.  P is not rounded to 16 bits: it enters as
// hi + lo, two 16-bit numbers that hold 16 bits of it (22 in fp16).  With at most 8 heads (ROWS = 8) the remainder travels
// in the idle rows 8 ... 15 of the same product and costs nothing.  In fp16 the running maximum stands for 2^15, so that
// weights down to 2^-29 of the largest stay clear of the subnormals.  A warp needs some 1800 cycles for its 32 slots of
// 128 channels, a quarter of the time that HBM needs for an SM's share of them: the fifth-generation products, whose
// accumulators would have to travel through tensor memory twice per tile, have nothing to win here (the tensor pipe is busy
// 19 % of the streaming time).  That holds up to 16 query heads per KV head.  Beyond, two or four sets of warps load every tile's
// fragments each for itself, and the products bound the kernel: 8 x 32768 slots of 4 KV heads of 128 channels take 92 us with up to 16 heads
// (5.8 TB/s), 127 with 32 (4.2), 219 with 64 (2.4); 64 channels 90, 131 and 228; 256 channels (8 x 8192 slots, 0.27 GB) 54 with 8, 59 with 16,
// 90 with 32, 159 with 64.
//
// *Registers.*  Two CTAs of five warps leave 168 a thread at 128 channels, of which 172 to 220 bytes spill; one CTA at 256 channels has 255 and
// spills 280 to 312 (64 channels: none).
#pragma once

#include <cuda.h>

#include <type_traits>

#include "sttm_cache.cuh"

namespace sttm {

// Slots per tile: 32 KB of keys and values whatever the head's channels.
__host__ __device__ constexpr int attend_tile(int dim) { return 8192 / dim; }
// stages of a CTA's ring: two CTAs to an SM with 96 KB each, or one with 192 KB
__host__ __device__ constexpr int attend_stages(int dim) { return dim == 256 ? 6 : 3; }
constexpr uint32_t kAttStage = 32768;                       // bytes of a stage: a tile's keys, then its values
constexpr int kAttWarps = 4;                                // consumer warps
constexpr int kAttAhead = 1;                                // matrix fragments are loaded so many products ahead
constexpr int kAttStep = 32;                                // slots that a warp takes at once
constexpr int kAttThreads = (kAttWarps + 1) * 32;
constexpr int kAttMaxStages = 6;
constexpr int kAttBatch = 512;                              // slots that the producer looks up at once: 16 a lane
constexpr int kJoinRegs = 16;                               // output registers of a warp that meet in shared memory at once
constexpr int kAttMaxCluster = 16;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kJoinThreads = 256;
constexpr int kScoreSlots = 2 * kJoinThreads;               // slots whose scores a block updates in one go

struct AttendArgs {
    const int32_t* table;
    long long table_stride, pages;
    int heads, page, seqs;        // KV heads
    int group;                    // query heads per KV head
    int box;                      // slots per tensor copy
    int stages, tile;
    int max_len;
    int cluster;                  // CTAs that share one row and join it in shared memory; 0: equal shares of all tiles
    const uint16_t* q;
    long long q_seq, q_head;
    const int32_t* lengths;
    const uint8_t* mask;          // [seqs][mask_stride], zero: slot left out; may be null
    long long mask_stride;
    float scale_log2;             // scale * log2(e): logits are kept in units of log 2
    uint16_t* out;                // [seqs][heads * group][DIM]
    float* lse;                   // may be null
    int32_t* status;
    int4* rows;                   // [seqs * heads] {first tile, first partial, partials, -} (equal shares)
    float2* stats;                // [partials][group] {reference of the exponentials, their sum}
    float* partial;               // [partials][group][DIM]
    float* logits;                // [tiles][group][tile], null without scores
    float* scores;                // may be null
    long long score_seq, score_head;
    float decay;
};

// D (16x8, fp32) += A (16x16, row) * B (16x8, col).  Not volatile: the compiler may move products past the loads of
// later fragments.  (Kept in program order, every product waited for the load just before it, and a step of 32 slots took
// 1000 cycles for the keys and 1000 for the values.)
template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 2^x; results below 2^-126 become zero (a weight that small adds nothing to a sum that holds a one)
__device__ __forceinline__ float exp2_weight(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// `box` slots of one page and KV head, all channels: [64-channel half][slot][64 channels]
__device__ __forceinline__ void tma_load_slots(uint32_t dst, const CUtensorMap* map, int place, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(place), "r"(0), "r"(head), "r"(page), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void sts_f32x2(uint32_t addr, float x, float y) {
    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(x), "f"(y) : "memory");
}
__device__ __forceinline__ float2 dsmem_f32x2(uint32_t cluster_addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_addr) : "memory");
    return v;
}

// tiles after which teams and stages meet in the same pairs again
__device__ __forceinline__ int attend_lap(int stages, int teams) {
    int lap = stages;
    while (lap % teams != 0) lap += stages;
    return lap;
}

__device__ __forceinline__ int attend_length(const AttendArgs& p, int b) { return min(max(p.lengths[b], 0), p.max_len); }

// Position in the sequence of tiles: sequences, their KV heads, their tiles.
struct Cursor {
    int b, h, j, len, tiles;      // tiles: of the row
    // the next row that has a tile (there is one)
    __device__ __forceinline__ void next_row(const AttendArgs& p) {
        j = 0;
        if (++h < p.heads) return;
        h = 0;
        do {
            b++;
            len = b < p.seqs ? attend_length(p, b) : 1;
            tiles = (len + p.tile - 1) / p.tile;
        } while (tiles == 0);
    }
};

// A CTA's tiles [t0, t1) and where they begin.  Every warp works it out.
struct Share {
    int t0, t1, each;             // each: tiles of a share
    int first_cta, parts;         // of the row, when shares end with rows; else parts = 0
    Cursor c;
};
__device__ __forceinline__ int tiles_of(const AttendArgs& p, int len) { return (len + p.tile - 1) / p.tile; }
__device__ __forceinline__ Share attend_share(const AttendArgs& p, int cta, int lane) {
    Share s;
    if (p.cluster > 0) {                                    // (the grid is made of clusters, of one CTA at least)
        const int row = (int)cluster_id(), rank = (int)cluster_rank(), base = row * tiles_of(p, p.max_len);
        s.c.b = row / p.heads;
        s.c.h = row - s.c.b * p.heads;
        s.c.len = attend_length(p, s.c.b);
        s.c.tiles = tiles_of(p, s.c.len);
        s.c.j = (int)((long long)s.c.tiles * rank / p.cluster);
        s.t0 = base + s.c.j;
        s.t1 = base + (int)((long long)s.c.tiles * (rank + 1) / p.cluster);
        s.each = 1;
        s.first_cta = cta;
        s.parts = 1;
        return s;
    }
    // 32 sequences at a time; with at most 32 everything stays in registers
    const int len0 = lane < p.seqs ? attend_length(p, lane) : 0, tiles0 = tiles_of(p, len0);
    auto sum = [&](auto&& f) {
        int total = __reduce_add_sync(0xffffffffu, f(tiles0));
        for (int b0 = 32; b0 < p.seqs; b0 += 32)
            total += __reduce_add_sync(0xffffffffu, f(b0 + lane < p.seqs ? tiles_of(p, attend_length(p, b0 + lane)) : 0));
        return total * p.heads;
    };
    const int grid = (int)gridDim.x, total = sum([](int tiles) { return tiles; });
    s.each = max(1, (total + grid - 1) / grid);
    // Shares that end with their rows, if somewhat longer ones make room for that: a share of parts of two rows pays
    // for a second end and start, during which its copies stall (256 rows of 4096 slots: 89 us instead of 101).  Short
    // shares would grow by too much, and under a mask tiles are not equal (48 ragged masked rows: 30 us instead of 28).
    bool with_rows = false;
    for (int k = 0; k < 4 && s.each >= 6 && p.mask == nullptr && !with_rows; k++) {
        const int e = s.each + k * (s.each / 6) / 3;        // up to a sixth more
        if (sum([e](int tiles) { return (tiles + e - 1) / e; }) <= (int)gridDim.x) {
            with_rows = true;
            s.each = e;
        }
    }
    // the sequence that this CTA's share begins in: a prefix sum of shares (of tiles, where shares run on)
    const int at = with_rows ? cta : (int)min((long long)cta * s.each, (long long)total);
    s.t0 = s.t1 = s.first_cta = s.parts = 0;
    s.c.b = s.c.h = s.c.j = s.c.len = s.c.tiles = 0;
    int base = 0, base_tiles = 0;
    for (int b0 = 0; b0 < p.seqs; b0 += 32) {
        const int len = b0 == 0 ? len0 : (b0 + lane < p.seqs ? attend_length(p, b0 + lane) : 0), tiles = b0 == 0 ? tiles0 : tiles_of(p, len);
        const int per_row = with_rows ? (tiles + s.each - 1) / s.each : tiles;
        int upto = per_row * p.heads, upto_tiles = tiles * p.heads;         // inclusive prefix sums
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o), w = __shfl_up_sync(0xffffffffu, upto_tiles, o);
            if (lane >= o) {
                upto += v;
                upto_tiles += w;
            }
        }
        const unsigned past = __ballot_sync(0xffffffffu, base + upto > at);
        if (past != 0) {
            const int owner = __ffs(past) - 1, n = __shfl_sync(0xffffffffu, per_row, owner);
            const int off = at - base - __shfl_sync(0xffffffffu, upto - per_row * p.heads, owner);
            s.c.b = b0 + owner;
            s.c.len = __shfl_sync(0xffffffffu, len, owner);
            s.c.tiles = __shfl_sync(0xffffffffu, tiles, owner);
            s.c.h = off / n;
            const int k = off - s.c.h * n;                  // share (tile) of the row
            const int row_tile = base_tiles + __shfl_sync(0xffffffffu, upto_tiles - tiles * p.heads, owner) + s.c.h * s.c.tiles;
            s.c.j = with_rows ? k * s.each : k;
            s.t0 = row_tile + s.c.j;
            s.t1 = min(s.t0 + s.each, with_rows ? row_tile + s.c.tiles : total);
            if (with_rows) {
                s.first_cta = cta - k;
                s.parts = n;
            }
            break;
        }
        base += __shfl_sync(0xffffffffu, upto, 31);
        base_tiles += __shfl_sync(0xffffffffu, upto_tiles, 31);
    }
    return s;
}

template <int DIM, int ROWS>
constexpr size_t attend_fixed_bytes() { return kAttWarps * ROWS * ((8 * kJoinRegs / (ROWS == 8 ? 2 : 4) + 8) * 4 + 8) + 1024; }

// outputs of a sequence that has no slot at all: zero, log-sum-exp -inf
template <int DIM>
__device__ __forceinline__ void attend_empty(const AttendArgs& p, int row) {
    uint32_t* out = reinterpret_cast<uint32_t*>(p.out + (long long)row * p.group * DIM);
    for (int i = threadIdx.x; i < p.group * DIM / 2; i += kAttWarps * 32) out[i] = 0;
    if (p.lse != nullptr)
        for (int i = threadIdx.x; i < p.group; i += kAttWarps * 32) p.lse[(long long)row * p.group + i] = -INFINITY;
    if (threadIdx.x == 0 && p.cluster == 0) p.rows[row] = make_int4(0, 0, 0, 0);
}

// A row's weights under its final statistics: 2^(logit - x) * y; a row without any weight adds none.
__device__ __forceinline__ float2 weight_of(float ref, float sum) {
    return make_float2(ref == -INFINITY ? 0.f : ref, sum == 0.f ? 0.f : 1.f / sum);
}
// slots [0, len) of a row: every slot's weights, added up over the query heads, go to its score
__device__ __forceinline__ void add_scores(const AttendArgs& p, int b, int h, int len, int first_tile, const float2* stat, int thread,
                                           int threads) {
    float* score = p.scores + b * p.score_seq + h * p.score_head;
    for (int i = thread; i < len; i += threads) {
        const float* x = p.logits + ((long long)(first_tile + i / p.tile) * p.group) * p.tile + i % p.tile;
        const float before = score[i];
        float w = 0.f;
        for (int g0 = 0; g0 < p.group; g0 += 8) {           // (eight heads' loads at once: their latency is what the loop costs)
            float v[8];
#pragma unroll
            for (int g = 0; g < 8; g++) v[g] = g0 + g < p.group ? __ldcg(x + (g0 + g) * p.tile) : -INFINITY;
#pragma unroll
            for (int g = 0; g < 8; g++) {
                const float2 s = stat[min(g0 + g, p.group - 1)];
                w = fmaf(exp2_weight(v[g] - s.x), s.y, w);
            }
        }
        score[i] = fmaf(p.decay, before, w);
    }
}

// ---- joining the CTAs of a cluster that share a row.  Every CTA leaves its part in its own shared memory:
// [group][DIM] outputs, then {reference, sum} per head; after a cluster barrier each takes its share of the outputs.
// (Calls with scores have no clusters of more than one CTA.)
template <int DIM>
__device__ __forceinline__ void attend_leave_nothing(const AttendArgs& p, uint32_t at) {
    for (int i = threadIdx.x; i < p.group * DIM / 2; i += kAttWarps * 32) sts_f32x2(at + i * 8, 0.f, 0.f);
    for (int i = threadIdx.x; i < p.group; i += kAttWarps * 32) sts_f32x2(at + p.group * DIM * 4 + i * 8, -INFINITY, 0.f);
}
// by all threads of all CTAs of the cluster
template <typename T, int DIM>
__device__ __noinline__ void attend_join_cluster(const AttendArgs& p, char* mine) {
    const uint32_t at = smem_u32(mine);
    const int rank = (int)cluster_rank(), row = (int)cluster_id(), lane = threadIdx.x & 31;
    // behind this CTA's part: what every part's outputs count in the end [cluster][group]
    float* factor = reinterpret_cast<float*>(mine + p.group * (DIM * 4 + 8));
    cluster_arrive();
    cluster_wait();
    // this CTA's share of the channel pairs: the first of them (as a rule all) are asked for with the statistics
    const int pairs = p.group * DIM / 2, each = (pairs + p.cluster - 1) / p.cluster, end = min(pairs, (rank + 1) * each);
    float2 v[kAttMaxCluster];
    auto ask = [&](int i) {
#pragma unroll
        for (int r = 0; r < kAttMaxCluster; r++)
            if (r < p.cluster) v[r] = dsmem_f32x2(map_to_rank(at + i * 8, r));
    };
    int i = rank * each + threadIdx.x;
    if (i < end) ask(i);
    // 16 lanes to a head, one to a part
    for (int h0 = threadIdx.x / 32 * 2; h0 < p.group; h0 += kAttThreads / 16) {
        const int h = h0 + lane / 16, r = lane % 16;
        const bool is = h < p.group && r < p.cluster;
        const float2 st = is ? dsmem_f32x2(map_to_rank(at + p.group * DIM * 4 + h * 8, r)) : make_float2(-INFINITY, 0.f);
        float ref = st.x;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
        const float f = st.x == ref ? 1.f : exp2_weight(st.x - ref);    // (a part with no slot: sum 0, reference -inf)
        float sum = st.y * f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (is) factor[r * p.group + h] = sum == 0.f ? 0.f : f / sum;
        if (is && r == 0 && rank == 0 && p.lse != nullptr) p.lse[(long long)row * p.group + h] = (ref + log2f(sum)) * kLn2;
    }
    __syncthreads();
    for (; i < end; i += kAttThreads) {
        const float* f = factor + i / (DIM / 2);
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int r = 0; r < kAttMaxCluster; r++)
            if (r < p.cluster) {
                const float w = f[r * p.group];
                x = fmaf(v[r].x, w, x);
                y = fmaf(v[r].y, w, y);
            }
        reinterpret_cast<uint32_t*>(p.out)[(long long)row * pairs + i] = Pair<T>::pack(x, y);
        if (i + kAttThreads < end) ask(i + kAttThreads);
    }
    cluster_arrive();
    cluster_wait();                                         // nobody leaves while its part may be read
}

template <typename T, int DIM, int ROWS>
__global__ void __launch_bounds__(kAttThreads, DIM == 256 ? 1 : 2)
k_cache_attend(const __grid_constant__ AttendArgs p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    constexpr int NT = DIM / 8;                             // 8-channel columns of the output
    constexpr int KS = DIM / 16;                            // 16-channel steps of a logit
    constexpr int OR = ROWS == 8 ? 2 : 4;                   // joined output registers per column
    constexpr int TILE = attend_tile(DIM), PIECES = TILE / kAttStep;    // slots of a tile, and what a warp takes at once of them
    constexpr uint32_t kHalfTile = kAttStage / 2;           // bytes of a stage's keys
    constexpr float kOffset = std::is_same<T, __half>::value ? 15.f : 0.f;
    extern __shared__ __align__(1024) char smem_raw[];
    __shared__ __align__(8) uint64_t bars[(kAttWarps + 1) * kAttMaxStages];
    __shared__ __align__(4) uint16_t slots_on[kAttMaxStages][TILE / 16];    // bit i of word w: slot 16 w + i of the stage's tile counts
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    char* const ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
    float* join = reinterpret_cast<float*>(ring_ptr + p.stages * kAttStage);
    // Query heads go 16 to a set of warps (1, 2 or 4 sets).  The warps of a set share a tile's pieces; when they are more
    // than the pieces they form teams that take the tiles in turn.
    const int sets = ROWS == 8 || p.group <= 16 ? 1 : (p.group <= 32 ? 2 : 4), members = kAttWarps / sets;
    const int teams = members > PIECES ? members / PIECES : 1;
    // A stage has a barrier per team that says it is full: every completion of it concerns that team, so that none
    // passes it by (a wait sees no more than a phase's parity).
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kAttWarps * kAttMaxStages;
    const int cta = blockIdx.x;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; s++) {
            for (int t = 0; t < kAttWarps; t++) mbar_init(full0 + 8 * (t * kAttMaxStages + s), 1);
            mbar_init(empty0 + 8 * s, kAttWarps / teams);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    wait_for_prior_kernel();
    let_next_kernel_start();
    __shared__ int share_info[4];                           // what only a row's end needs, out of the loops' registers
    Cursor c;
    int t0, t1;
    {
        const Share sh = attend_share(p, cta, lane);
        c = sh.c;
        t0 = sh.t0;
        t1 = sh.t1;
        if (threadIdx.x == 0) {
            share_info[0] = sh.each;
            share_info[1] = sh.first_cta;
            share_info[2] = sh.parts;
        }
        if (warp < kAttWarps) named_sync(1, kAttWarps * 32);
    }
    bool timed_out = false;

    if (warp == kAttWarps) {
        // ---- producer: lanes 0, 2, 4, ... copy keys, lanes 1, 3, 5, ... values, one box each
        const int nbox = TILE / p.box;
        const int box = lane >> 1;
        const bool values = lane & 1;
        const uint32_t box_bytes = (uint32_t)p.box * DIM * 2;
        constexpr int BATCH = kAttBatch / TILE;             // tiles
        // Pages and masks are looked up for a batch of tiles of a row at once, and asked for a batch ahead: lane i holds
        // boxes i and i + 32 of the batch, and which of its slots 16 i ... 16 i + 15 count.
        int page[2] = {0, 0}, place[2] = {0, 0}, ask_page[2] = {0, 0}, ask_place[2] = {0, 0};
        uint32_t marks = 0, ask_mask[4] = {0, 0, 0, 0}, ask_slots = 0, any_lo = 0, any_hi = 0;
        auto ask = [&](const Cursor& q) {
            const int first = q.j / BATCH * kAttBatch;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int in = (lane + 32 * e) * p.box, slot = first + in;
                if (slot < q.len && in < kAttBatch) {
                    const int stretch = slot / p.page;
                    ask_place[e] = slot - stretch * p.page;
                    ask_page[e] = p.table[q.b * p.table_stride + stretch];
                }
            }
            const int mine = first + 16 * lane, n = min(max(q.len - mine, 0), 16);
            ask_slots = (1u << n) - 1;
            if (p.mask != nullptr && n > 0) {
                const uint8_t* m = p.mask + q.b * p.mask_stride + mine;
                if (n == 16 && ((uintptr_t)m & 15) == 0) {
                    const uint4 v = *reinterpret_cast<const uint4*>(m);
                    ask_mask[0] = v.x; ask_mask[1] = v.y; ask_mask[2] = v.z; ask_mask[3] = v.w;
                } else {
                    // (two steps, so that all bytes are on their way before the first is needed)
                    uint32_t byte[16];
#pragma unroll
                    for (int i = 0; i < 16; i++) byte[i] = i < n ? m[i] : 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) ask_mask[i] = byte[4 * i] | byte[4 * i + 1] << 8 | byte[4 * i + 2] << 16 | byte[4 * i + 3] << 24;
                }
            }
        };
        auto take = [&]() {
            marks = ask_slots;
            if (p.mask != nullptr) {
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t x = __vsetne4(ask_mask[i], 0u);      // 1 in every byte that is not zero
                    bits |= ((x & 1u) | (x >> 7 & 2u) | (x >> 14 & 4u) | (x >> 21 & 8u)) << (4 * i);
                }
                marks &= bits;
            }
            any_lo = __ballot_sync(0xffffffffu, (marks & 0xffu) != 0);
            any_hi = __ballot_sync(0xffffffffu, (marks >> 8) != 0);
#pragma unroll
            for (int e = 0; e < 2; e++) {
                page[e] = ask_page[e];
                place[e] = ask_place[e];
            }
        };
        int use = 0, s = 0, team = 0;
        if (t0 < t1) ask(c);
        for (int t = t0; t < t1; t++) {
            const int k = c.j % BATCH;                      // tile in the batch
            if (t == t0 || k == 0) {
                take();
                const int left = min(c.tiles - c.j, BATCH - k);     // tiles of this batch from here on
                if (t + left < t1) {
                    Cursor q = c;
                    if (c.j + left < c.tiles) q.j = c.j + left;
                    else q.next_row(p);
                    ask(q);
                }
            }
            const uint32_t full = full0 + 8 * (team * kAttMaxStages + s);
            const int entry = k * nbox + box;
            const int from0 = __shfl_sync(0xffffffffu, page[0], entry & 31), from1 = __shfl_sync(0xffffffffu, page[1], entry & 31);
            const int place0 = __shfl_sync(0xffffffffu, place[0], entry & 31), place1 = __shfl_sync(0xffffffffu, place[1], entry & 31);
            int from = entry < 32 ? from0 : from1;
            // a box is copied if any of its slots counts
            bool mine = box < nbox;
            if (p.box >= 16) mine = mine && ((any_lo | any_hi) >> (entry * (p.box / 16) & 31) & ((1u << (p.box / 16)) - 1)) != 0;
            else mine = mine && ((entry & 1 ? any_hi : any_lo) >> (entry / 2 & 31) & 1u) != 0;
            const unsigned copies = __ballot_sync(0xffffffffu, mine);
            if (mine && (from < 0 || from >= p.pages)) {
                raise_status(p.status, kStatusArg);
                from = (int)p.pages;                        // beyond the tensor: the copy brings zeros
            }
            if (use > 0 && !mbar_wait_warp(empty0 + 8 * s, use - 1, timed_out)) break;
            if (lane / (TILE / 16) == k) slots_on[s][lane % (TILE / 16)] = (uint16_t)marks;
            __syncwarp();
            if (lane == 0) {
                if (copies != 0) mbar_expect_tx(full, __popc(copies) * box_bytes);
                else mbar_arrive(full);
            }
            __syncwarp();
            if (mine)
                tma_load_slots(ring + s * kAttStage + (values ? kHalfTile : 0) + box * box_bytes, values ? &map_v : &map_k,
                               entry < 32 ? place0 : place1, c.h, from, full);
            if (++c.j == c.tiles && t + 1 < t1) c.next_row(p);
            if (++team == teams) team = 0;
            if (++s == p.stages) { s = 0; use++; }
        }
        // No copy may be in flight when the CTA ends: every stage that was filled has been emptied (after a timeout
        // that may not come: then what was started has to arrive).
        const int filled = use * p.stages + s;
        for (int k = max(0, filled - p.stages); k < filled; k++) {
            bool late = timed_out;
            if (!mbar_wait_warp(empty0 + 8 * (k % p.stages), k / p.stages, late)) {
                late = false;
                mbar_wait_warp(full0 + 8 * (k % teams * kAttMaxStages + k % p.stages), k / attend_lap(p.stages, teams), late);
                timed_out = true;
            }
        }
        if (timed_out && lane == 0) raise_status(p.status, kStatusWaitTimeout);
        if (p.cluster > 1) attend_join_cluster<T, DIM>(p, ring_ptr);
        return;
    }

    // ---- consumers
    // warp = member * sets + set; the members of a team are neighbours
    const int set = warp & (sets - 1), member = warp / sets, team = teams == 1 ? 0 : member / PIECES;
    const int pieces = PIECES / (members / teams), piece0 = member % (members / teams) * pieces;     // this warp's of a tile
    const int g = lane >> 2, tq = lane & 3;
    const int head0 = set * 16 + g, head1 = head0 + 8;      // this lane's rows of the products
    const bool has0 = head0 < p.group, has1 = ROWS == 16 && head1 < p.group;
    // ldmatrix: keys as [slots 0-7 | 8-15][channels 0-7 | 8-15], values the other way round
    const int k_slot = ((lane >> 4) << 3) + (lane & 7), k_word = (lane >> 3) & 1;
    const int v_slot = (((lane >> 3) & 1) << 3) + (lane & 7), v_word = lane >> 4;
    const uint32_t half_bytes = (uint32_t)p.box * 128;      // one 64-channel half of a box
    const int box_log = __ffs(p.box) - 1;
    // where a slot of a tile begins in a stage's keys (or values)
    auto slot_row = [&](uint32_t base, int slot) {
        return base + (slot >> box_log) * p.box * (DIM * 2) + (slot & (p.box - 1)) * 128;
    };

    float o[NT][4], ref0 = -INFINITY, ref1 = -INFINITY, sum0 = 0.f, sum1 = 0.f;
    uint32_t qf[KS][ROWS == 8 ? 2 : 4];
    // this warp's next tile: its number in the share, its stage, how often its team has used that stage
    const int lap = attend_lap(p.stages, teams);
    int next = team, s = team % p.stages, use = 0, round = team;
    for (int part = t0; part < t1;) {                       // rows of the share
        const int part_end = min(t1, part + c.tiles - c.j);
        {
            const uint16_t* q0 = p.q + c.b * p.q_seq + (c.h * p.group + head0) * p.q_head + 2 * tq;
            const uint16_t* q1 = q0 + 8 * p.q_head;
#pragma unroll
            for (int k = 0; k < KS; k++) {
                qf[k][0] = has0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * k) : 0u;
                qf[k][1] = has0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * k + 8) : 0u;
                if constexpr (ROWS == 16) {
                    qf[k][2] = has1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * k) : 0u;
                    qf[k][3] = has1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * k + 8) : 0u;
                }
            }
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) o[n][e] = 0.f;
            ref0 = ref1 = -INFINITY;
            sum0 = sum1 = 0.f;
        }
        for (; t0 + next < part_end; next += teams) {
            const int t = t0 + next;
            mbar_wait_warp(full0 + 8 * (team * kAttMaxStages + s), use, timed_out);     // (after a timeout: garbage in, and the status says so)
            const uint32_t kbase = ring + s * kAttStage, vbase = kbase + kHalfTile;
#pragma unroll 1
            for (int i = 0; i < pieces; i++) {
                const int step = (piece0 + i) * kAttStep;       // first slot of the piece in the tile
                const uint32_t step_on = *reinterpret_cast<const uint32_t*>(&slots_on[s][step / 16]);
                float* logits = p.logits == nullptr ? nullptr : p.logits + (long long)t * p.group * TILE + step + 2 * tq;
                if (step_on == 0) {
                    if (logits != nullptr)
#pragma unroll
                        for (int e = 0; e < kAttStep / 8; e++) {
                            const float2 none = make_float2(-INFINITY, -INFINITY);
                            if (has0) *reinterpret_cast<float2*>(logits + head0 * TILE + 8 * e) = none;
                            if (has1) *reinterpret_cast<float2*>(logits + head1 * TILE + 8 * e) = none;
                        }
                    continue;
                }
                // logits: x[n] are the scores of slots 8 n + 2 tq and + 1 for head0, then for head1
                // (two sums each, over even and odd channel steps: eight independent products hide the latency of one)
                float x[kAttStep / 8][4] = {}, x2[kAttStep / 8][4] = {};
                {
                    uint32_t row[kAttStep / 16];
#pragma unroll
                    for (int u = 0; u < kAttStep / 16; u++) row[u] = slot_row(kbase, step + 16 * u + k_slot);
                    // fragments are loaded kAttAhead channel steps before their products
                    uint32_t b[kAttAhead + 1][kAttStep / 16][4];
                    auto load = [&](int k) {
#pragma unroll
                        for (int u = 0; u < kAttStep / 16; u++)
                            ldmatrix_x4(row[u] + (k / 4) * half_bytes + ((((2 * k) & 7) + k_word) ^ (k_slot & 7)) * 16, b[k % (kAttAhead + 1)][u]);
                    };
#pragma unroll
                    for (int k = 0; k < kAttAhead; k++) load(k);
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        if (k + kAttAhead < KS) load(k + kAttAhead);
                        uint32_t a[4];
                        a[0] = qf[k][0];
                        a[2] = qf[k][1];
                        a[1] = ROWS == 16 ? qf[k][ROWS == 16 ? 2 : 0] : 0u;
                        a[3] = ROWS == 16 ? qf[k][ROWS == 16 ? 3 : 0] : 0u;
#pragma unroll
                        for (int u = 0; u < kAttStep / 16; u++) {
                            const uint32_t (&f)[4] = b[k % (kAttAhead + 1)][u];
                            mma_16816<T>(k & 1 ? x2[2 * u] : x[2 * u], a, f[0], f[1]);
                            mma_16816<T>(k & 1 ? x2[2 * u + 1] : x[2 * u + 1], a, f[2], f[3]);
                        }
                    }
                }
                // in units of log 2; slots that do not count: -inf (selected, never computed with)
                const uint32_t on = step_on >> (2 * tq);        // bits 8 n and 8 n + 1: this lane's slots
                float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
                for (int n = 0; n < kAttStep / 8; n++)
#pragma unroll
                    for (int e = 0; e < (ROWS == 16 ? 4 : 2); e++) {
                        x[n][e] = (on >> (8 * n + (e & 1))) & 1u ? (x[n][e] + x2[n][e]) * p.scale_log2 : -INFINITY;
                        float& top = e < 2 ? top0 : top1;
                        top = fmaxf(top, x[n][e]);
                    }
                if (logits != nullptr) {
#pragma unroll
                    for (int n = 0; n < kAttStep / 8; n++) {
                        if (has0) *reinterpret_cast<float2*>(logits + head0 * TILE + 8 * n) = make_float2(x[n][0], x[n][1]);
                        if (has1) *reinterpret_cast<float2*>(logits + head1 * TILE + 8 * n) = make_float2(x[n][2], x[n][3]);
                    }
                }
#pragma unroll
                for (int d = 1; d <= 2; d <<= 1) {
                    top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, d));
                    if constexpr (ROWS == 16) top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, d));
                }
                // a new maximum rescales what was summed under the old one (rare after the first tiles)
                const float new0 = fmaxf(ref0, top0 - kOffset), new1 = ROWS == 16 ? fmaxf(ref1, top1 - kOffset) : ref1;
                if (__any_sync(0xffffffffu, new0 > ref0 || new1 > ref1)) {
                    const float f0 = new0 > ref0 ? exp2_weight(ref0 - new0) : 1.f, f1 = ROWS == 16 ? (new1 > ref1 ? exp2_weight(ref1 - new1) : 1.f) : f0;
                    sum0 *= f0;
                    sum1 *= f1;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        o[n][0] *= f0;
                        o[n][1] *= f0;
                        o[n][2] *= f1;
                        o[n][3] *= f1;
                    }
                    ref0 = new0;
                    ref1 = new1;
                }
                // (a row without any finite logit so far keeps the reference 0: its weights are 2^-inf = 0)
                const float base0 = ref0 == -INFINITY ? 0.f : ref0, base1 = ref1 == -INFINITY ? 0.f : ref1;
                uint32_t hi[kAttStep / 16][4], lo[kAttStep / 16][4];
#pragma unroll
                for (int n = 0; n < kAttStep / 8; n++) {
                    const int u = n / 2, e = 2 * (n & 1);
                    const float a0 = exp2_weight(x[n][0] - base0), a1 = exp2_weight(x[n][1] - base0);
                    sum0 += a0 + a1;
                    hi[u][e] = Pair<T>::pack(a0, a1);
                    const float2 h = Pair<T>::split(hi[u][e]);
                    lo[u][e] = Pair<T>::pack(a0 - h.x, a1 - h.y);
                    if constexpr (ROWS == 16) {
                        const float c0 = exp2_weight(x[n][2] - base1), c1 = exp2_weight(x[n][3] - base1);
                        sum1 += c0 + c1;
                        hi[u][e + 1] = Pair<T>::pack(c0, c1);
                        const float2 h1 = Pair<T>::split(hi[u][e + 1]);
                        lo[u][e + 1] = Pair<T>::pack(c0 - h1.x, c1 - h1.y);
                    } else {
                        hi[u][e + 1] = lo[u][e];                // rows 8 ... 15: the remainders
                    }
                }
                // values of slots that do not count are cleared: 0 x NaN would be NaN
                const bool all_on = step_on == 0xffffffffu;
                uint32_t row[kAttStep / 16];
#pragma unroll
                for (int u = 0; u < kAttStep / 16; u++) row[u] = slot_row(vbase, step + 16 * u + v_slot);
                // eight columns at a time, first with one half of the step's slots, then with the other: eight independent
                // products again; the next fragments are loaded before them
                uint32_t b[2][4][4];
                auto load = [&](int i) {                    // i-th group of fragments: columns 8 (i / 2) ..., slots 16 (i % 2) ...
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const int n = i / 2 * 8 + 2 * q;
                        ldmatrix_x4_trans(row[i & 1] + (n / 8) * half_bytes + (((n & 7) + v_word) ^ (v_slot & 7)) * 16, b[i & 1][q]);
                    }
                };
                load(0);
#pragma unroll
                for (int i = 0; i < NT / 4; i++) {
                    if (i + 1 < NT / 4) load(i + 1);
                    const int u = i & 1;
                    const uint32_t w = on >> (16 * u);
                    const uint32_t and0 = ((w & 1u) ? 0xffffu : 0u) | ((w & 2u) ? 0xffff0000u : 0u);
                    const uint32_t and1 = ((w & 0x100u) ? 0xffffu : 0u) | ((w & 0x200u) ? 0xffff0000u : 0u);
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const int n = i / 2 * 8 + 2 * q;
                        uint32_t (&f)[4] = b[u][q];
                        if (!all_on) {
                            f[0] &= and0; f[1] &= and1;
                            f[2] &= and0; f[3] &= and1;
                        }
                        mma_16816<T>(o[n], hi[u], f[0], f[1]);
                        mma_16816<T>(o[n + 1], hi[u], f[2], f[3]);
                    }
                    if constexpr (ROWS == 16) {
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            const int n = i / 2 * 8 + 2 * q;
                            mma_16816<T>(o[n], lo[u], b[u][q][0], b[u][q][1]);
                            mma_16816<T>(o[n + 1], lo[u], b[u][q][2], b[u][q][3]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty0 + 8 * s);
            s = (s + teams) % p.stages;
            round += teams;
            if (round >= lap) { round -= lap; use++; }
        }

        {
            // ---- the row's part in this share ends.  The warps' outputs meet in shared memory, kJoinRegs registers of
            // each at a time; then every thread adds up the warps' shares of some channel pairs.
#pragma unroll
            for (int d = 1; d <= 2; d <<= 1) {
                sum0 += __shfl_xor_sync(0xffffffffu, sum0, d);
                if constexpr (ROWS == 16) sum1 += __shfl_xor_sync(0xffffffffu, sum1, d);
            }
            const int row = c.b * p.heads + c.h;
            const int first = part - c.j;                   // the row's first tile
            const int each = share_info[0], first_cta = share_info[2] ? share_info[1] : first / each;
            const int parts = share_info[2] ? share_info[2] : (first + c.tiles - 1) / each - first_cta + 1;
            const long long at = (long long)(cta + (p.cluster ? 0 : row));      // grows along the staircase of (CTA, row) pairs: unique
            constexpr int COLS = 8 * kJoinRegs / OR, STRIDE = COLS + 8;         // channels per round; padded: no bank conflict
            // every warp brings its outputs to the row's common reference first
            float2* const warp_stat = reinterpret_cast<float2*>(join + kAttWarps * ROWS * STRIDE);
            named_sync(1, kAttWarps * 32);                  // the buffer is free (and every tile of the part done with)
            if (tq == 0) {
                warp_stat[warp * ROWS + g] = make_float2(ref0, sum0);
                if constexpr (ROWS == 16) warp_stat[warp * ROWS + 8 + g] = make_float2(ref1, sum1);
            }
            named_sync(1, kAttWarps * 32);
            auto common = [&](int of_set, int r) {          // {reference, sum} of row r of a set
                float ref = -INFINITY, sum = 0.f;
                float2 st[kAttWarps];
#pragma unroll
                for (int m = 0; m < kAttWarps; m++) {
                    st[m] = m < members ? warp_stat[(m * sets + of_set) * ROWS + r] : make_float2(-INFINITY, 0.f);
                    ref = fmaxf(ref, st[m].x);
                }
#pragma unroll
                for (int m = 0; m < kAttWarps; m++) sum = fmaf(st[m].y, st[m].x == ref ? 1.f : exp2_weight(st[m].x - ref), sum);
                return make_float2(ref, sum);               // (a warp that saw nothing: sum 0, reference -inf)
            };
            const float2 c0 = common(set, g), c1 = ROWS == 16 ? common(set, 8 + g) : c0;
            // in the end outputs are wanted themselves, not their sums
            const float w0 = parts == 1 && p.cluster <= 1 ? (c0.y == 0.f ? 0.f : 1.f / c0.y) : 1.f;
            const float w1 = ROWS == 16 ? (parts == 1 && p.cluster <= 1 ? (c1.y == 0.f ? 0.f : 1.f / c1.y) : 1.f) : w0;
            const float f0 = (ref0 == c0.x ? 1.f : exp2_weight(ref0 - c0.x)) * w0;
            const float f1 = ROWS == 16 ? (ref1 == c1.x ? 1.f : exp2_weight(ref1 - c1.x)) * w1 : f0;
            if (tq == 0 && warp == set) {                   // (one warp of each set)
                auto say = [&](int head, float2 st) {
                    if (p.cluster > 1) sts_f32x2(ring + p.group * DIM * 4 + head * 8, st.x, st.y);
                    else if (parts > 1 || p.logits != nullptr) p.stats[at * p.group + head] = st;
                    if (parts == 1 && p.cluster <= 1 && p.lse != nullptr)
                        p.lse[(long long)row * p.group + head] = (st.x + log2f(st.y)) * kLn2;
                };
                if (has0) say(head0, c0);
                if (has1) say(head1, c1);
            }
#pragma unroll
            for (int n0 = 0; n0 < NT; n0 += COLS / 8) {
                if (n0 > 0) named_sync(1, kAttWarps * 32);
                float* mine = join + (warp * ROWS + g) * STRIDE + 2 * tq;
#pragma unroll
                for (int n = 0; n < COLS / 8; n++) {
                    const float (&v)[4] = o[n0 + n];
                    *reinterpret_cast<float2*>(mine + 8 * n) =
                        ROWS == 8 ? make_float2((v[0] + v[2]) * f0, (v[1] + v[3]) * f0) : make_float2(v[0] * f0, v[1] * f0);
                    if constexpr (ROWS == 16) *reinterpret_cast<float2*>(mine + 8 * STRIDE + 8 * n) = make_float2(v[2] * f1, v[3] * f1);
                }
                named_sync(1, kAttWarps * 32);
                for (int i = threadIdx.x; i < sets * ROWS * COLS / 2; i += kAttWarps * 32) {
                    const int r = i / (COLS / 2), col = 2 * (i % (COLS / 2)), of_set = r / ROWS;    // row of all sets' rows, channel pair
                    const int head = of_set * 16 + r % ROWS, ch = 8 * n0 + col;
                    if (head >= p.group) continue;
                    float x = 0.f, y = 0.f;
#pragma unroll
                    for (int m = 0; m < kAttWarps; m++)
                        if (m < members) {
                            const float2 v = *reinterpret_cast<const float2*>(join + ((m * sets + of_set) * ROWS + r % ROWS) * STRIDE + col);
                            x += v.x;
                            y += v.y;
                        }
                    if (p.cluster > 1) sts_f32x2(ring + (head * DIM + ch) * 4, x, y);
                    else if (parts == 1) *reinterpret_cast<uint32_t*>(p.out + ((long long)row * p.group + head) * DIM + ch) = Pair<T>::pack(x, y);
                    else *reinterpret_cast<float2*>(p.partial + (at * p.group + head) * DIM + ch) = make_float2(x, y);
                }
            }
            if (p.cluster <= 1) {
                if (threadIdx.x == 0 && cta == first_cta && p.cluster == 0) p.rows[row] = make_int4(first, first_cta + row, parts, 0);
                if (p.cluster == 1 && p.logits != nullptr) {
                    // the only CTA of the row: its warps update the scores
                    named_sync(1, kAttWarps * 32);          // (logits and statistics are in memory; the buffer is free)
                    float2* final_stat = reinterpret_cast<float2*>(join);
                    for (int h = threadIdx.x; h < p.group; h += kAttWarps * 32) {
                        const float2 v = p.stats[at * p.group + h];
                        final_stat[h] = weight_of(v.x, v.y);
                    }
                    named_sync(1, kAttWarps * 32);
                    add_scores(p, c.b, c.h, c.len, first, final_stat, threadIdx.x, kAttWarps * 32);
                }
            }
        }
        part = part_end;
        if (part < t1) c.next_row(p);
    }
    if (timed_out && lane == 0) raise_status(p.status, kStatusWaitTimeout);
    // sequences without a slot, and lengths that cannot be
    if (p.cluster == 1) {
        if (t0 == t1) attend_empty<DIM>(p, cta);
    } else if (p.cluster == 0) {
        for (int b = cta; b < p.seqs; b += gridDim.x)
            if (attend_length(p, b) == 0)
                for (int h = 0; h < p.heads; h++) attend_empty<DIM>(p, b * p.heads + h);
    }
    if (cta == 0)
        for (int b = threadIdx.x; b < p.seqs; b += kAttWarps * 32)
            if (p.lengths[b] < 0 || p.lengths[b] > p.max_len) raise_status(p.status, kStatusCapacity);
    if (p.cluster > 1) {
        if (t0 >= t1) attend_leave_nothing<DIM>(p, ring);
        attend_join_cluster<T, DIM>(p, ring_ptr);
    }
}

// {reference of a head's weights, their sum}: joined over the row's partials by one warp, in one pass
__device__ __forceinline__ float2 join_stats(const AttendArgs& p, const int4& r, int head, int lane) {
    float ref = -INFINITY, sum = 0.f;
    auto add = [&](float2 v) {                              // (a part with no slot: sum 0, reference -inf)
        const float m = fmaxf(ref, v.x);
        sum = sum * (ref == m ? 1.f : exp2_weight(ref - m)) + v.y * (v.x == m ? 1.f : exp2_weight(v.x - m));
        ref = m;
    };
    for (int i0 = 0; i0 < r.z; i0 += 128) {
        float2 v[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int i = i0 + 32 * u + lane;
            v[u] = i < r.z ? __ldcg(p.stats + (long long)(r.y + i) * p.group + head) : make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int u = 0; u < 4; u++) add(v[u]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        add(make_float2(__shfl_xor_sync(0xffffffffu, ref, o), __shfl_xor_sync(0xffffffffu, sum, o)));
    return make_float2(ref, sum);
}

// The end of a call: rows that were split are joined (a block per row and query head), and with scores
// every slot's weight is added to its score (`chunks` blocks per row).
template <typename T, int DIM>
__global__ void __launch_bounds__(kJoinThreads, 4) k_cache_join(const __grid_constant__ AttendArgs p, int join_blocks, int chunks) {
    constexpr int LANES = DIM / 4;                          // threads that hold one head's channels, four each
    constexpr int PARTS = kJoinThreads / LANES;
    __shared__ float4 acc[kJoinThreads];
    __shared__ float2 stat[64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_prior_kernel();
    let_next_kernel_start();
    if ((int)blockIdx.x < join_blocks) {
        const int row = blockIdx.x / p.group, head = blockIdx.x % p.group;
        const int4 r = p.rows[row];
        if (r.z <= 1) return;                               // written by k_cache_attend
        const float2 st = join_stats(p, r, head, lane);
        const int part = threadIdx.x / LANES, ch = threadIdx.x % LANES;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = part; i < r.z; i += PARTS) {
            const long long at = (long long)(r.y + i) * p.group + head;
            const float m = __ldcg(p.stats + at).x;
            const float w = m == st.x ? 1.f : exp2_weight(m - st.x);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p.partial + at * DIM + 4 * ch));
            sum.x = fmaf(v.x, w, sum.x);
            sum.y = fmaf(v.y, w, sum.y);
            sum.z = fmaf(v.z, w, sum.z);
            sum.w = fmaf(v.w, w, sum.w);
        }
        acc[threadIdx.x] = sum;
        __syncthreads();
        if (part == 0) {
#pragma unroll
            for (int k = 1; k < PARTS; k++) {
                const float4 v = acc[k * LANES + ch];
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
            const float inv = st.y == 0.f ? 0.f : 1.f / st.y;
            const long long at = (long long)row * p.group + head;
            *reinterpret_cast<uint2*>(p.out + at * DIM + 4 * ch) =
                make_uint2(Pair<T>::pack(sum.x * inv, sum.y * inv), Pair<T>::pack(sum.z * inv, sum.w * inv));
            if (ch == 0 && p.lse != nullptr) p.lse[at] = (st.x + log2f(st.y)) * kLn2;
        }
        return;
    }
    // two slots to a thread at a time; their logits (the first eight heads') are on their way while the statistics
    // are joined
    const int k = blockIdx.x - join_blocks, row = k / chunks;
    int slot0 = (k % chunks) * kScoreSlots;
    const int b = row / p.heads;
    const int4 r = p.rows[row];
    const int len = attend_length(p, b);
    if (slot0 >= len) return;
    float* score = p.scores + b * p.score_seq + (row % p.heads) * p.score_head;
    float v[2][8], before[2] = {0.f, 0.f};
    auto ask = [&](int g0) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int slot = slot0 + u * kJoinThreads + threadIdx.x;
            const float* x = p.logits + ((long long)(r.x + slot / p.tile) * p.group + g0) * p.tile + slot % p.tile;
#pragma unroll
            for (int g = 0; g < 8; g++) v[u][g] = slot < len && g0 + g < p.group ? __ldcg(x + g * p.tile) : -INFINITY;
            if (g0 == 0 && slot < len) before[u] = score[slot];
        }
    };
    ask(0);
    for (int h = warp; h < p.group; h += kJoinThreads / 32) {
        const float2 st = join_stats(p, r, h, lane);
        if (lane == 0) stat[h] = weight_of(st.x, st.y);
    }
    __syncthreads();
    for (bool first = true; slot0 < len; slot0 += chunks * kScoreSlots, first = false) {
        if (!first) ask(0);
        float w[2] = {0.f, 0.f};
        for (int g0 = 0; g0 < p.group; g0 += 8) {
#pragma unroll
            for (int g = 0; g < 8; g++) {
                const float2 st = stat[min(g0 + g, p.group - 1)];
#pragma unroll
                for (int u = 0; u < 2; u++) w[u] = fmaf(exp2_weight(v[u][g] - st.x), st.y, w[u]);
            }
            if (g0 + 8 < p.group) ask(g0 + 8);
        }
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int slot = slot0 + u * kJoinThreads + threadIdx.x;
            if (slot < len) score[slot] = fmaf(p.decay, before[u], w[u]);
        }
    }
}

}  // namespace sttm
