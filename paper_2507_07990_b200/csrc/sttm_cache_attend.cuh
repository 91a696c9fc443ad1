// Attention of one new token per sequence over its paged cache (sttm_cache_attend).
//
//   out[b, h] = sum_s p[h, s] v[s],   p[h, s] = exp(scale q[h] . k[s]) / sum of the same over s
//
// over the slots s of sequence b that its length and its mask leave.  Keys and values are read once
// and everything else is small, so HBM bounds the kernel as long as the products keep up: the group of
// query heads that share a KV head forms the rows of one small matrix product per 16 slots.
//
// *Split.*  The slots of all (sequence, KV head) rows are cut into tiles of 64 and laid end to end; CTA
// i takes the i-th of equal shares, whatever rows they belong to.  So one long sequence or many ragged
// ones keep every SM streaming equally long; a row that lies in several shares leaves a running
// maximum, a sum and an unscaled output per share, joined in share order by k_cache_join (no
// atomics: the bits of a result do not depend on scheduling).
//
// *Pipeline.*  A producer warp brings a tile's keys and values into a ring of shared-memory stages by
// tensor copies, one box of at most 64 slots that lie in one page per copy, under the 128-byte swizzle.  Four warps
// take 16 slots of a tile each (with more than 16 query heads per KV head: 32 or 64, and share the
// heads), and never wait for one another before the end of a row: each keeps its own maximum, sum and
// output.
//
// *Products.*  S = Q K^T and O += P V on mma.sync m16n8k16 with fp32 sums.  P is not rounded to 16
// bits: it enters as hi + lo, two 16-bit numbers that hold 16 bits of it (22 in fp16).  With
// at most 8 heads (ROWS = 8) the remainder travels in the idle rows 8 ... 15 of the same product and costs
// nothing.  In fp16 the running maximum stands for 2^15, so that weights down to 2^-29 of the largest stay clear
// of the subnormals.
// The fifth-generation product (tcgen05.mma) needs 64 rows: with 7 heads nine tenths of it would be
// padding, and at 8 KB of cache per 32 products the legacy pipe is busy a fifth of the streaming time.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "sttm_cache.cuh"

namespace sttm {

constexpr int kAttTile = 64;                                // slots per tile
constexpr int kAttWarps = 4;                                // consumer warps
constexpr int kAttThreads = (kAttWarps + 1) * 32;
constexpr int kAttMaxStages = 8;
constexpr int kJoinThreads = 128;
constexpr int kScoreChunk = 512;                            // slots per block of the score update

struct AttendArgs {
    const int32_t* table;
    long long table_stride, pages;
    int heads, page, seqs;        // KV heads
    int group;                    // query heads per KV head
    int box;                      // slots per tensor copy
    int stages;
    int max_len;
    int whole;                    // nonzero: one CTA per row, no splitting
    const uint16_t* q;
    long long q_seq, q_head;
    const int32_t* lengths;
    const uint8_t* mask;          // [seqs][mask_stride], zero: slot left out; may be null
    long long mask_stride;
    float scale_log2;             // scale * log2(e): logits are kept in units of log 2
    uint16_t* out;                // [seqs][heads * group][DIM]
    float* lse;                   // may be null
    int32_t* status;
    int4* rows;                   // [seqs * heads] {first tile, first partial, partials, -}
    float2* stats;                // [partials][group] {reference of the exponentials, their sum}
    float* partial;               // [partials][group][DIM]
    float* logits;                // [tiles][group][64], null without scores
    float* scores;                // may be null
    long long score_seq, score_head;
    float decay;
};

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_16816<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    mma_bf16(d, a, b0, b1);
}
template <>
__device__ __forceinline__ void mma_16816<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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

__device__ __forceinline__ int attend_length(const AttendArgs& p, int b) { return min(max(p.lengths[b], 0), p.max_len); }

// Position in the sequence of tiles: sequences, their KV heads, their tiles.
struct Cursor {
    int b, h, j, tiles, len;      // tiles: of the row
    __device__ __forceinline__ void load(const AttendArgs& p) {
        len = attend_length(p, b);
        tiles = (len + kAttTile - 1) / kAttTile;
    }
    __device__ __forceinline__ void next(const AttendArgs& p) {
        if (++j < tiles) return;
        j = 0;
        if (++h < p.heads) return;
        h = 0;
        do {
            if (++b >= p.seqs) { tiles = 0; return; }
            load(p);
        } while (tiles == 0);
    }
};

template <int DIM>
__host__ __device__ constexpr size_t attend_stage_bytes() { return 2u * kAttTile * DIM * 2; }
template <int DIM, int ROWS>
constexpr size_t attend_fixed_bytes() { return 2u * 32 * (DIM / 8) * 2 * 4 + 2u * 32 * 4 * 4 + 1024; }

// outputs of a sequence that has no slot at all: zero, log-sum-exp -inf
template <int DIM>
__device__ __forceinline__ void attend_empty(const AttendArgs& p, int row) {
    uint32_t* out = reinterpret_cast<uint32_t*>(p.out + (long long)row * p.group * DIM);
    for (int i = threadIdx.x; i < p.group * DIM / 2; i += blockDim.x) out[i] = 0;
    if (p.lse != nullptr)
        for (int i = threadIdx.x; i < p.group; i += blockDim.x) p.lse[(long long)row * p.group + i] = -INFINITY;
    if (threadIdx.x == 0) p.rows[row] = make_int4(0, 0, 0, 0);
}

template <typename T, int DIM, int ROWS>
__global__ void __launch_bounds__(kAttThreads, DIM == 256 ? 1 : 2)
k_cache_attend(const __grid_constant__ AttendArgs p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    constexpr int NT = DIM / 8;                             // 8-channel columns of the output
    constexpr int KS = DIM / 16;                            // 16-channel steps of a logit
    constexpr int OR = ROWS == 8 ? 2 : 4;                   // joined output registers per column
    constexpr uint32_t kHalfTile = kAttTile * DIM * 2;      // bytes of a stage's keys
    constexpr float kOffset = std::is_same<T, __half>::value ? 15.f : 0.f;
    extern __shared__ __align__(1024) char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kAttMaxStages];
    __shared__ int sched[6];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    float* join = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)) + (size_t)p.stages * attend_stage_bytes<DIM>());
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kAttMaxStages;
    const int cta = blockIdx.x;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; s++) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, kAttWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_for_prior_kernel();
    let_next_kernel_start();

    // this CTA's share of the tiles
    if (p.whole) {
        if (threadIdx.x == 0) {
            Cursor c;
            c.b = cta / p.heads;
            c.load(p);
            sched[0] = cta * ((p.max_len + kAttTile - 1) / kAttTile); sched[1] = sched[0] + c.tiles; sched[2] = c.b; sched[3] = cta % p.heads; sched[4] = 0; sched[5] = 1;
        }
    } else if (warp == 0) {
        long long total = 0;
        for (int b0 = 0; b0 < p.seqs; b0 += 32) {
            int n = b0 + lane < p.seqs ? (attend_length(p, b0 + lane) + kAttTile - 1) / kAttTile * p.heads : 0;
            n = __reduce_add_sync(0xffffffffu, n);
            total += n;
        }
        const int share = max(1, (int)((total + gridDim.x - 1) / gridDim.x));
        const int t0 = (int)min((long long)cta * share, total), t1 = (int)min((long long)t0 + share, total);
        if (lane == 0) { sched[0] = t0; sched[1] = t1; sched[5] = share; }
        int base = 0;
        for (int b0 = 0; b0 < p.seqs && t0 < t1; b0 += 32) {
            const int n = b0 + lane < p.seqs ? (attend_length(p, b0 + lane) + kAttTile - 1) / kAttTile * p.heads : 0;
            int upto = n;                                   // inclusive prefix sum
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned past = __ballot_sync(0xffffffffu, base + upto > t0);
            if (past != 0) {
                if (lane == __ffs(past) - 1) {
                    const int off = t0 - (base + upto - n), tiles = n / p.heads;
                    sched[2] = b0 + lane;
                    sched[3] = off / tiles;
                    sched[4] = off % tiles;
                }
                break;
            }
            base += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
    __syncthreads();
    const int t0 = sched[0], t1 = sched[1], share = sched[5];
    // sequences without a slot, and lengths that cannot be
    if (p.whole) {
        if (t0 == t1) attend_empty<DIM>(p, cta);
    } else {
        for (int b = cta; b < p.seqs; b += gridDim.x)
            if (attend_length(p, b) == 0)
                for (int h = 0; h < p.heads; h++) attend_empty<DIM>(p, b * p.heads + h);
    }
    if (cta == 0)
        for (int b = threadIdx.x; b < p.seqs; b += blockDim.x)
            if (p.lengths[b] < 0 || p.lengths[b] > p.max_len) raise_status(p.status, kStatusCapacity);
    if (t0 >= t1) return;
    Cursor c;
    c.b = sched[2]; c.h = sched[3]; c.j = sched[4];
    c.load(p);
    bool timed_out = false;

    if (warp == kAttWarps) {
        // ---- producer: lanes 0, 2, 4, ... copy keys, lanes 1, 3, 5, ... values, one box each
        const int nbox = kAttTile / p.box;
        const int box = lane >> 1;
        const bool values = lane & 1;
        const uint32_t box_bytes = (uint32_t)p.box * DIM * 2;
        auto page_of = [&](const Cursor& q) {
            const int slot = q.j * kAttTile + box * p.box;
            if (box >= nbox || q.tiles == 0 || slot >= q.len) return 0;
            return p.table[q.b * p.table_stride + slot / p.page];
        };
        int page = page_of(c), use = 0, s = 0, issued = 0;
        for (int t = t0; t < t1; t++) {
            const int slot = c.j * kAttTile + box * p.box;
            const bool mine = box < nbox && slot < c.len;
            const int nb = min(nbox, (c.len - c.j * kAttTile + p.box - 1) / p.box);
            if (mine && (page < 0 || page >= p.pages)) {
                raise_status(p.status, kStatusArg);
                page = (int)p.pages;                        // beyond the tensor: the copy brings zeros
            }
            Cursor n = c;
            if (t + 1 < t1) n.next(p);
            const int page_next = page_of(n);
            if (use > 0 && !mbar_wait_warp(empty0 + 8 * s, use - 1, timed_out)) break;
            if (lane == 0) mbar_expect_tx(full0 + 8 * s, 2u * nb * box_bytes);
            __syncwarp();
            if (mine)
                tma_load_slots(ring + s * (uint32_t)attend_stage_bytes<DIM>() + (values ? kHalfTile : 0) + box * box_bytes,
                               values ? &map_v : &map_k, slot % p.page, c.h, page, full0 + 8 * s);
            issued++;
            page = page_next;
            c = n;
            if (++s == p.stages) { s = 0; use++; }
        }
        // no copy may be in flight when the CTA ends
        for (int k = max(0, issued - p.stages); k < issued; k++) {
            bool late = false;
            if (!mbar_wait_warp(full0 + 8 * (k % p.stages), k / p.stages, late)) timed_out = true;
        }
        if (timed_out && lane == 0) raise_status(p.status, kStatusWaitTimeout);
        return;
    }

    // ---- consumers.  `sets` groups of warps take 16 heads each; a warp takes `sets` steps of 16 slots of a tile.
    const int sets = ROWS == 8 || p.group <= 16 ? 1 : (p.group <= 32 ? 2 : 4);
    const int members = kAttWarps / sets, set = warp / members, member = warp % members;
    const int g = lane >> 2, tq = lane & 3;
    const int head0 = set * 16 + g, head1 = head0 + 8;      // this lane's rows of the products
    const bool has0 = head0 < p.group, has1 = ROWS == 16 && head1 < p.group;
    // ldmatrix: keys as [slots 0-7 | 8-15][channels 0-7 | 8-15], values the other way round
    const int k_slot = ((lane >> 4) << 3) + (lane & 7), k_word = (lane >> 3) & 1;
    const int v_slot = (((lane >> 3) & 1) << 3) + (lane & 7), v_word = lane >> 4;
    const uint32_t half_bytes = (uint32_t)p.box * 128;      // one 64-channel half of a box
    const int box_log = __ffs(p.box) - 1;

    float o[NT][4], ref0 = -INFINITY, ref1 = -INFINITY, sum0 = 0.f, sum1 = 0.f;
    uint32_t qf[KS][ROWS == 8 ? 2 : 4];
    bool fresh = true;
    int use = 0, s = 0;
    for (int t = t0; t < t1; t++) {
        if (fresh) {
            fresh = false;
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
        // a tile's mask bytes are asked for before the wait for its keys
        uint32_t keep = 0;                                  // bit 4 i + e: slot e of this lane in step i counts
        const int tile0 = c.j * kAttTile;
        for (int i = 0; i < sets; i++) {
            const int first = tile0 + (member * sets + i) * 16 + 2 * tq;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int slot = first + (e >> 1) * 8 + (e & 1);
                bool on = slot < c.len;
                if (on && p.mask != nullptr) on = p.mask[c.b * p.mask_stride + slot] != 0;
                keep |= (on ? 1u : 0u) << (4 * i + e);
            }
        }
        mbar_wait_warp(full0 + 8 * s, use, timed_out);      // (after a timeout: garbage in, and the status says so)
        const uint32_t kbase = ring + s * (uint32_t)attend_stage_bytes<DIM>(), vbase = kbase + kHalfTile;
        for (int i = 0; i < sets; i++) {
            const int step = (member * sets + i) * 16;      // first slot of the step in the tile
            const uint32_t on = (keep >> (4 * i)) & 15u;
            if (__any_sync(0xffffffffu, on != 0)) {
                float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
                {
                    const int r = step + k_slot, bx = r >> box_log, in = r & (p.box - 1);
                    const uint32_t row = kbase + bx * p.box * (DIM * 2) + in * 128;
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        uint32_t b[4];
                        ldmatrix_x4(row + (k / 4) * half_bytes + ((((2 * k) & 7) + k_word) ^ (in & 7)) * 16, b);
                        uint32_t a[4];
                        a[0] = qf[k][0];
                        a[2] = qf[k][1];
                        a[1] = ROWS == 16 ? qf[k][ROWS == 16 ? 2 : 0] : 0u;
                        a[3] = ROWS == 16 ? qf[k][ROWS == 16 ? 3 : 0] : 0u;
                        mma_16816<T>(s0, a, b[0], b[1]);
                        mma_16816<T>(s1, a, b[2], b[3]);
                    }
                }
                // logits in units of log 2; slots that do not count: -inf (selected, never computed with)
                float x[4] = {s0[0], s0[1], s1[0], s1[1]}, y[4] = {s0[2], s0[3], s1[2], s1[3]};
                float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const bool yes = (on >> e) & 1u;
                    x[e] = yes ? x[e] * p.scale_log2 : -INFINITY;
                    top0 = fmaxf(top0, x[e]);
                    if constexpr (ROWS == 16) {
                        y[e] = yes ? y[e] * p.scale_log2 : -INFINITY;
                        top1 = fmaxf(top1, y[e]);
                    }
                }
                if (p.logits != nullptr) {
                    float* dst = p.logits + ((long long)t * p.group) * kAttTile + step + 2 * tq;
                    if (has0) {
                        *reinterpret_cast<float2*>(dst + head0 * kAttTile) = make_float2(x[0], x[1]);
                        *reinterpret_cast<float2*>(dst + head0 * kAttTile + 8) = make_float2(x[2], x[3]);
                    }
                    if (has1) {
                        *reinterpret_cast<float2*>(dst + head1 * kAttTile) = make_float2(y[0], y[1]);
                        *reinterpret_cast<float2*>(dst + head1 * kAttTile + 8) = make_float2(y[2], y[3]);
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
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const float a0 = exp2_weight(x[2 * e] - base0), a1 = exp2_weight(x[2 * e + 1] - base0);
                    sum0 += a0 + a1;
                    hi[2 * e] = Pair<T>::pack(a0, a1);
                    const float2 h = Pair<T>::split(hi[2 * e]);
                    lo[2 * e] = Pair<T>::pack(a0 - h.x, a1 - h.y);
                    if constexpr (ROWS == 16) {
                        const float c0 = exp2_weight(y[2 * e] - base1), c1 = exp2_weight(y[2 * e + 1] - base1);
                        sum1 += c0 + c1;
                        hi[2 * e + 1] = Pair<T>::pack(c0, c1);
                        const float2 h1 = Pair<T>::split(hi[2 * e + 1]);
                        lo[2 * e + 1] = Pair<T>::pack(c0 - h1.x, c1 - h1.y);
                    } else {
                        hi[2 * e + 1] = lo[2 * e];          // rows 8 ... 15: the remainders
                    }
                }
                // values of slots that do not count are cleared: 0 x NaN would be NaN
                const bool all_on = __all_sync(0xffffffffu, on == 15u);
                const uint32_t and0 = ((on & 1u) ? 0xffffu : 0u) | ((on & 2u) ? 0xffff0000u : 0u);
                const uint32_t and1 = ((on & 4u) ? 0xffffu : 0u) | ((on & 8u) ? 0xffff0000u : 0u);
                const int r = step + v_slot, bx = r >> box_log, in = r & (p.box - 1);
                const uint32_t row = vbase + bx * p.box * (DIM * 2) + in * 128;
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    uint32_t b[4];
                    ldmatrix_x4_trans(row + (n / 8) * half_bytes + (((n & 7) + v_word) ^ (in & 7)) * 16, b);
                    if (!all_on) {
                        b[0] &= and0; b[1] &= and1;
                        b[2] &= and0; b[3] &= and1;
                    }
                    mma_16816<T>(o[n], hi, b[0], b[1]);
                    mma_16816<T>(o[n + 1], hi, b[2], b[3]);
                    if constexpr (ROWS == 16) {
                        mma_16816<T>(o[n], lo, b[0], b[1]);
                        mma_16816<T>(o[n + 1], lo, b[2], b[3]);
                    }
                }
            } else if (p.logits != nullptr) {
                float* dst = p.logits + ((long long)t * p.group) * kAttTile + step + 2 * tq;
                const float2 none = make_float2(-INFINITY, -INFINITY);
                if (has0) {
                    *reinterpret_cast<float2*>(dst + head0 * kAttTile) = none;
                    *reinterpret_cast<float2*>(dst + head0 * kAttTile + 8) = none;
                }
                if (has1) {
                    *reinterpret_cast<float2*>(dst + head1 * kAttTile) = none;
                    *reinterpret_cast<float2*>(dst + head1 * kAttTile + 8) = none;
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * s);
        if (++s == p.stages) { s = 0; use++; }

        if (c.j == c.tiles - 1 || t == t1 - 1) {
            // ---- the row's part in this share ends: join the warps of a set (the upper half hands over to
            // the lower, then again), the set's first warp writes
            fresh = true;
#pragma unroll
            for (int d = 1; d <= 2; d <<= 1) {
                sum0 += __shfl_xor_sync(0xffffffffu, sum0, d);
                if constexpr (ROWS == 16) sum1 += __shfl_xor_sync(0xffffffffu, sum1, d);
            }
            if constexpr (ROWS == 8) {
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    o[n][0] += o[n][2];
                    o[n][1] += o[n][3];
                }
            }
            for (int width = members / 2; width >= 1; width >>= 1) {
                // at most two pairs of warps at a time, two registers of a column in one go
                const int pair = set * width + member % width;
                float* xo = join + pair * 32 * NT * 2;
                float* xs = join + 2 * 32 * NT * 2 + pair * 32 * 4;
#pragma unroll
                for (int r = 0; r < OR; r += 2) {           // rows g, then rows g + 8
                    float& ref = r == 0 ? ref0 : ref1;
                    float& sum = r == 0 ? sum0 : sum1;
                    named_sync(1, kAttWarps * 32);          // the buffer is free
                    if (member >= width && member < 2 * width) {
#pragma unroll
                        for (int n = 0; n < NT; n++) {
                            xo[2 * n * 32 + lane] = o[n][r];
                            xo[(2 * n + 1) * 32 + lane] = o[n][r + 1];
                        }
                        xs[lane] = ref;
                        xs[32 + lane] = sum;
                    }
                    named_sync(1, kAttWarps * 32);
                    if (member < width) {
                        const float other = xs[lane], m = fmaxf(ref, other);
                        const float f = ref == m ? 1.f : exp2_weight(ref - m), e = other == m ? 1.f : exp2_weight(other - m);
                        sum = sum * f + xs[32 + lane] * e;
                        ref = m;
#pragma unroll
                        for (int n = 0; n < NT; n++) {
                            o[n][r] = o[n][r] * f + xo[2 * n * 32 + lane] * e;
                            o[n][r + 1] = o[n][r + 1] * f + xo[(2 * n + 1) * 32 + lane] * e;
                        }
                    }
                }
            }
            const int row = c.b * p.heads + c.h;
            const int first = t - c.j;                      // the row's first tile
            const int first_cta = p.whole ? cta : first / share, last_cta = p.whole ? cta : (first + c.tiles - 1) / share;
            const int parts = last_cta - first_cta + 1;
            if (member == 0) {
                const long long at = (long long)(cta + (p.whole ? 0 : row));        // grows along the staircase of (CTA, row) pairs: unique
                if (parts == 1) {
                    const float i0 = sum0 == 0.f ? 0.f : 1.f / sum0, i1 = sum1 == 0.f ? 0.f : 1.f / sum1;
                    uint16_t* dst = p.out + ((long long)row * p.group + head0) * DIM + 2 * tq;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        if (has0) *reinterpret_cast<uint32_t*>(dst + 8 * n) = Pair<T>::pack(o[n][0] * i0, o[n][1] * i0);
                        if (has1) *reinterpret_cast<uint32_t*>(dst + 8 * DIM + 8 * n) = Pair<T>::pack(o[n][2] * i1, o[n][3] * i1);
                    }
                    if (p.lse != nullptr && tq == 0) {
                        constexpr float kLn2 = 0.69314718055994531f;
                        if (has0) p.lse[(long long)row * p.group + head0] = (ref0 + log2f(sum0)) * kLn2;
                        if (has1) p.lse[(long long)row * p.group + head1] = (ref1 + log2f(sum1)) * kLn2;
                    }
                } else {
                    float* dst = p.partial + (at * p.group + head0) * DIM + 2 * tq;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        if (has0) *reinterpret_cast<float2*>(dst + 8 * n) = make_float2(o[n][0], o[n][1]);
                        if (has1) *reinterpret_cast<float2*>(dst + 8 * DIM + 8 * n) = make_float2(o[n][2], o[n][3]);
                    }
                }
                if ((parts > 1 || p.logits != nullptr) && tq == 0) {
                    if (has0) p.stats[at * p.group + head0] = make_float2(ref0, sum0);
                    if (has1) p.stats[at * p.group + head1] = make_float2(ref1, sum1);
                }
                if (set == 0 && lane == 0 && cta == first_cta)
                    p.rows[row] = make_int4(first, first_cta + (p.whole ? 0 : row), parts, 0);
            }
        }
        c.next(p);
    }
    if (timed_out && lane == 0) raise_status(p.status, kStatusWaitTimeout);
}

// {log2 of the sum of a head's weights, its reference}: joined over the row's partials by one warp
__device__ __forceinline__ float2 join_stats(const AttendArgs& p, const int4& r, int head, int lane) {
    float ref = -INFINITY;
    for (int i = lane; i < r.z; i += 32) ref = fmaxf(ref, p.stats[(long long)(r.y + i) * p.group + head].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
    float sum = 0.f;
    for (int i = lane; i < r.z; i += 32) {
        const float2 v = p.stats[(long long)(r.y + i) * p.group + head];
        sum += v.x == ref ? v.y : v.y * exp2f(v.x - ref);   // (a part with no slot: sum 0, reference -inf)
    }
    return make_float2(ref, warp_sum(sum));
}

// The end of a call: rows that were split are joined (a block per row and query head), and with scores
// every slot's weight is added to its score (a block per row and kScoreChunk slots).
template <typename T, int DIM>
__global__ void __launch_bounds__(kJoinThreads) k_cache_join(const __grid_constant__ AttendArgs p, int join_blocks, int chunks) {
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
        for (int i = part; i < r.z; i += PARTS) {
            const long long at = (long long)(r.y + i) * p.group + head;
            const float m = p.stats[at].x;
            const float w = m == st.x ? 1.f : exp2f(m - st.x);
            const float4 v = *reinterpret_cast<const float4*>(p.partial + at * DIM + 4 * ch);
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
            if (ch == 0 && p.lse != nullptr) p.lse[at] = (st.x + log2f(st.y)) * 0.69314718055994531f;
        }
        return;
    }
    const int k = blockIdx.x - join_blocks, row = k / chunks, slot0 = (k % chunks) * kScoreChunk;
    const int b = row / p.heads, len = attend_length(p, b);
    if (slot0 >= len) return;
    const int4 r = p.rows[row];
    for (int h = warp; h < p.group; h += kJoinThreads / 32) {
        const float2 st = join_stats(p, r, h, lane);
        // weight = 2^(logit - reference) / sum; a row without any weight adds none
        if (lane == 0) stat[h] = make_float2(st.x == -INFINITY ? 0.f : st.x, st.y == 0.f ? 0.f : 1.f / st.y);
    }
    __syncthreads();
    float* score = p.scores + b * p.score_seq + (row % p.heads) * p.score_head;
    for (int i = slot0 + threadIdx.x; i < min(len, slot0 + kScoreChunk); i += kJoinThreads) {
        const float* x = p.logits + ((long long)(r.x + i / kAttTile) * p.group) * kAttTile + i % kAttTile;
        float w = 0.f;
        for (int h = 0; h < p.group; h++) w += exp2f(x[h * kAttTile] - stat[h].x) * stat[h].y;
        score[i] = fmaf(p.decay, score[i], w);
    }
}

}  // namespace sttm
