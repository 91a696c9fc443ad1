// Matrix product in 8-bit integers (sttm_quant_matmul):
//
//     out[t][n] = x_scale[t] * w_scale[n] * sum over k of x[t][k] w[n][k]  + bias[n]
//
// on the tensor cores (tcgen05.mma kind::i8, sums of 32 bits in tensor memory: exact, so nothing depends on how the inner
// axis is cut).  Both operands have their inner axis contiguous; a tensor copy brings 128 bytes of it for the 128 rows of one and
// the NT rows of the other into a ring slot under the 128-byte swizzle, which is the K-major operand layout.  What lies
// behind the inner axis or the last row is filled with zeros by the copy.
//
// Few tokens (SWAP): weights are the 128-row operand, tokens the NT columns; the weights' bytes bound it, and a cluster
// shares the inner axis so that their stream is spread over all SMs.  Its CTAs put their sums into shared memory and each adds
// up and writes every size-th token.  Many tokens (k_quant_matmul_pair): the tensor cores bound it; two CTAs of a cluster take 256 tokens
// by 256 output channels together, tile after tile, one accumulator being written out while the other fills.
//
// Measured: 5278 x 3584 x 28672 360 us at full clocks (3.0 POP/s, the tensor cores busy 85 % of the time); 16 x 14336 x 3584
// 12.6 us (the weights at 4.1 TB/s), 1 x 3584 x 28672 22.2 (4.6 TB/s).
#pragma once

#include "sttm_cache.cuh"

namespace sttm {

struct MatmulArgs {
    const float *x_scale, *w_scale, *bias;
    void* out;
    long long out_row;            // elements
    long long rows;               // tokens
    int outer;                    // output channels
    int blocks;                   // steps of 128 along the inner axis
    int a_tiles, b_tiles;         // tiles of 128 rows, of NT rows
    int cluster;                  // CTAs that share the inner axis (SWAP), or 1
    uint32_t stages;
    int32_t* status;
    bool wide;                    // rows of out can be written in 16-byte pieces
};

constexpr int kMatK = 128;                            // inner elements (bytes) per step
constexpr int kMatThreads = 6 * 32;                   // producer, products, four warps that read out
constexpr size_t kMatSmem = 112 * 1024;               // two CTAs to an SM
constexpr int kMatMaxStages = 8, kMatGroup = 12;      // tiles of tokens in a row before the next tile of channels (see tile_at)

__host__ __device__ constexpr int matmul_slot(int nt) { return (128 + nt) * kMatK; }
__host__ __device__ constexpr size_t matmul_fixed_bytes() { return 1024 + (2 * kMatMaxStages + 4) * 8 + 16; }

// tcgen05.mma kind::i8: 32-bit integer accumulator (bits 4-5 = 2), signed A and B (bits 7-9, 10-12 = 1), both K-major
__host__ __device__ constexpr uint32_t matmul_idesc(int nt) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(nt / 8) << 17) | (8u << 24);
}

__device__ __forceinline__ void mma_i8(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %4, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void copy_tile_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ int4 ld_remote_s32x4(uint32_t cluster_addr) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(cluster_addr));
    return v;
}

// Tiles run through kMatGroup tiles of A for every tile of B: the 148 tiles in work share 12 + 13 tiles of rows instead of 1 + 148.
__device__ __forceinline__ void tile_at(const MatmulArgs& a, int tile, int& ta, int& tb) {
    const int per = kMatGroup * a.b_tiles, group = tile / per, first = group * kMatGroup;
    const int size = min(kMatGroup, a.a_tiles - first), in = tile - group * per;
    tb = in / size;
    ta = first + in - tb * size;
}

// A sum as an output.  (The fused form by name: left to the compiler, one of the places below had two roundings where the others have one, and a token's
// last bits in 32-bit outputs depended on how many others came with it.)
template <typename T>
__device__ __forceinline__ T output(int sum, float xs, float ws, float bias) { return (T)fmaf((float)sum * xs, ws, bias); }

template <typename T, int NT>
__global__ void __launch_bounds__(kMatThreads) k_quant_matmul(const __grid_constant__ MatmulArgs a, const __grid_constant__ CUtensorMap map_a,
                                                              const __grid_constant__ CUtensorMap map_b) {
    constexpr int SLOT = matmul_slot(NT);
    constexpr uint32_t COLS = 2 * NT;                           // two accumulators
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t ring = smem_u32(smem);
    const uint32_t bars = ring + a.stages * SLOT;
    const uint32_t full = bars, empty = full + 8 * kMatMaxStages, acc_full = empty + 8 * kMatMaxStages, acc_empty = acc_full + 16;
    uint32_t* tmem_word = reinterpret_cast<uint32_t*>(smem + a.stages * SLOT + (2 * kMatMaxStages + 4) * 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; s++) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(acc_full + 8 * b, 1);
            mbar_init(acc_empty + 8 * b, 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // this CTA's tiles, and its part of the inner axis
    const int size = a.cluster, rank = size > 1 ? (int)cluster_rank() : 0;
    const int tiles = a.a_tiles * a.b_tiles, first = blockIdx.x / size, step = gridDim.x / size;
    const int k0 = (int)((long long)a.blocks * rank / size), k1 = (int)((long long)a.blocks * (rank + 1) / size);
    if (warp == 0) {
        // The weights are called into L2 while the kernel before still runs (whatever that writes, L2 has it too).
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane ? &map_b : &map_a)) : "memory");
        int ta, tb;
        tile_at(a, first, ta, tb);
        if (lane < min(k1 - k0, 32))
            asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(&map_a)), "r"((k0 + lane) * kMatK), "r"(ta * 128) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_word)), "r"(COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_word);
    wait_for_prior_kernel();
    let_next_kernel_start();

    bool timed_out = false;
    int n = 0;                                                  // accumulators taken up so far

    if (warp == 0) {
        uint32_t slot = 0, turn = 1, taken = 0;                 // (the first wait for every slot returns at once: the phase before the first)
        for (int tile = first; tile < tiles && !timed_out; tile += step) {
            int ta, tb;
            tile_at(a, tile, ta, tb);
#pragma unroll 1
            for (int k = k0; k < k1; k++) {
                if (!mbar_wait_near(empty + 8 * slot, turn, timed_out)) break;
                if (lane == 0) {
                    mbar_expect_tx(full + 8 * slot, SLOT);
                    copy_tile_2d(ring + slot * SLOT, &map_a, k * kMatK, ta * 128, full + 8 * slot);
                    copy_tile_2d(ring + slot * SLOT + 128 * kMatK, &map_b, k * kMatK, tb * NT, full + 8 * slot);
                }
                __syncwarp();
                taken++;
                if (++slot == a.stages) {
                    slot = 0;
                    turn ^= 1;
                }
            }
        }
        // the CTA must not end with copies in flight
        for (uint32_t p = taken > a.stages ? taken - a.stages : 0; p < taken; p++) {
            bool late = false;
            mbar_wait_sleep(full + 8 * (p % a.stages), (int)(p / a.stages), late);
            timed_out |= late;
        }
    } else if (warp == 1) {
        const uint32_t ring_lo = one_value((uint32_t)tc_operand(ring)), tm = one_value(tmem), bar = one_value(bars);
        uint32_t slot = 0, turn = 0;
        for (int tile = first; tile < tiles && !timed_out; tile += step, n++) {
            const uint32_t b = one_value(n & 1);
            if (n >= 2 && !mbar_wait_near(acc_empty + 8 * b, (n >> 1) - 1, timed_out)) break;
            tc_fence_after();
#pragma unroll 1
            for (int k = k0; k < k1; k++) {
                const uint32_t at = one_value(slot), lo = ring_lo + at * (SLOT / 16), more = one_value(k > k0), last = one_value(k + 1 == k1);
                if (!mbar_wait_near(full + 8 * slot, turn, timed_out)) break;
                if (elected()) {
#pragma unroll
                    for (int i = 0; i < 4; i++) mma_i8(tm + b * NT, lo + 2 * i, lo + 128 * kMatK / 16 + 2 * i, kOperandHigh, matmul_idesc(NT), i > 0 ? 1 : more);
                    tc_commit(bar + 8 * kMatMaxStages + 8 * at);
                    if (last) tc_commit(bar + 16 * kMatMaxStages + 8 * b);
                }
                __syncwarp();
                if (++slot == a.stages) {
                    slot = 0;
                    turn ^= 1;
                }
            }
        }
        // the last products have completed before the tensor memory is given back
        for (int p = max(0, n - 2); p < n; p++) {
            bool late = false;
            mbar_wait_sleep(acc_full + 8 * (p & 1), p >> 1, late);
            timed_out |= late;
        }
    } else {
        const int row = 32 * (warp & 3) + lane;                 // the accumulator's row of this thread
        const uint32_t mine = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        for (int tile = first; tile < tiles && !timed_out; tile += step, n++) {
            const int b = n & 1;
            int ta, tb;
            tile_at(a, tile, ta, tb);
            if (!mbar_wait_warp(acc_full + 8 * b, n >> 1, timed_out)) break;
            tc_fence_after();
            {
                const int ch = ta * 128 + row;
                const float ws = ch < a.outer ? a.w_scale[ch] : 0.0f, bias = a.bias && ch < a.outer ? a.bias[ch] : 0.0f;
                auto write = [&](int col, int sum) {
                    const long long token = (long long)tb * NT + col;
                    if (ch < a.outer && token < a.rows) ((T*)a.out)[token * a.out_row + ch] = output<T>(sum, a.x_scale[token], ws, bias);
                };
                constexpr int CH = NT < 32 ? NT : 32;
#pragma unroll 1
                for (int c = 0; c < NT; c += CH) {
                    uint32_t v[32];
                    if constexpr (NT < 32) tc_load16(mine + b * NT + c, v);
                    else tc_load32(mine + b * NT + c, v);
                    if (size > 1) {
#pragma unroll
                        for (int i = 0; i < CH; i++) reinterpret_cast<int*>(smem)[(c + i) * 128 + row] = (int)v[i];
                    } else {
#pragma unroll
                        for (int i = 0; i < CH; i++) write(c + i, (int)v[i]);
                    }
                    __syncwarp();                               // (the next load is one for the whole warp)
                }
                if (size > 1) {                                 // (one tile per cluster then, and the ring has been read)
                    cluster_arrive();
                    cluster_wait();
                    // every size-th token, a warp each, four channels a lane
                    const int last = (int)min((long long)NT, a.rows - (long long)tb * NT), ch0 = ta * 128 + 4 * lane;
                    float scale[4], add[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        scale[i] = ch0 + i < a.outer ? a.w_scale[ch0 + i] : 0.0f;
                        add[i] = a.bias != nullptr && ch0 + i < a.outer ? a.bias[ch0 + i] : 0.0f;
                    }
                    for (int col = rank + size * (warp & 3); col < last; col += 4 * size) {
                        const uint32_t at = ring + col * 512 + lane * 16;
                        int4 part[8];
#pragma unroll
                        for (int r = 0; r < 8; r++) part[r] = r < size ? ld_remote_s32x4(map_to_rank(at, r)) : make_int4(0, 0, 0, 0);
                        int sum[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int r = 0; r < 8; r++) {
                            sum[0] += part[r].x; sum[1] += part[r].y; sum[2] += part[r].z; sum[3] += part[r].w;
                        }
                        const long long token = (long long)tb * NT + col;
                        const float xs = a.x_scale[token];
                        T* const out = (T*)a.out + token * a.out_row + ch0;
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (ch0 + i < a.outer) out[i] = output<T>(sum[i], xs, scale[i], add[i]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * b);
        }
    }
    if (size > 1) {
        // warps that have met at the first barrier meet at the second; every other warp, and those whose wait ran out, at both
        if (warp < 2 || n == 0) {
            cluster_arrive();
            cluster_wait();
        }
        cluster_arrive();                                       // no CTA ends while another reads its sums
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
    }
    if (timed_out) raise_status(a.status, kStatusWaitTimeout);
}

// ---- many tokens ----

// Two CTAs of a cluster on one tile (cta_group::2): each brings 128 of the 256 tokens and 128 of the 256 channels into its own
// ring, the first one's issuing thread starts products that read both rings, and each CTA's tensor memory holds the sums of its own
// 128 tokens.  Per step of 128 inner elements a CTA reads 32 KB for 512 cycles of products; a CTA alone would read 48.
constexpr int kPairStages = 6, kPairSlot = 256 * kMatK;         // 128 rows of either operand
constexpr size_t kPairSmem = (size_t)kPairStages * kPairSlot + (2 * kPairStages + 4) * 8 + 16 + 1024;
constexpr int kPairGroup = 8;                                   // tiles of tokens in a row before the next tile of channels

__device__ __forceinline__ void mma_i8_pair(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t accumulate) {
    constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (32u << 17) | (16u << 24);      // as matmul_idesc: N = 256, M = 256
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %4, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(kOperandHigh), "r"(idesc), "r"(accumulate)
        : "memory");
}
// both CTAs' mbarriers at this place get an arrival when every product issued so far has completed
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// a tile into this CTA's memory, its bytes counted by an mbarrier of the pair's first CTA
__device__ __forceinline__ void copy_tile_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar_cluster) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar_cluster)
                 : "memory");
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMatThreads, 1)
k_quant_matmul_pair(const __grid_constant__ MatmulArgs a, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t ring = smem_u32(smem), bars = ring + kPairStages * kPairSlot;
    const uint32_t full = bars, empty = full + 8 * kPairStages, acc_full = empty + 8 * kPairStages, acc_empty = acc_full + 16;
    uint32_t* tmem_word = reinterpret_cast<uint32_t*>(smem + kPairStages * kPairSlot + (2 * kPairStages + 4) * 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = (int)cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; s++) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(acc_full + 8 * b, 1);
            mbar_init(acc_empty + 8 * b, 8);                    // four reading warps of either CTA
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane ? &map_w : &map_x)) : "memory");
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_word)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_word);
    wait_for_prior_kernel();
    let_next_kernel_start();

    const int tiles = a.a_tiles * a.b_tiles, first = blockIdx.x / 2, step = gridDim.x / 2;
    auto place = [&](int tile, int& ta, int& tb) {
        const int per = kPairGroup * a.b_tiles, group = tile / per, at = group * kPairGroup;
        const int size = min(kPairGroup, a.a_tiles - at), in = tile - group * per;
        tb = in / size;
        ta = at + in - tb * size;
    };
    bool timed_out = false;
    if (warp == 0) {
        const uint32_t full0 = map_to_rank(full, 0);
        uint32_t slot = 0, turn = 1, taken = 0;                 // (the first wait for every slot returns at once: the phase before the first)
        for (int tile = first; tile < tiles && !timed_out; tile += step) {
            int ta, tb;
            place(tile, ta, tb);
#pragma unroll 1
            for (int k = 0; k < a.blocks; k++) {
                if (!mbar_wait_near(empty + 8 * slot, turn, timed_out)) break;
                if (lane == 0) {
                    if (rank == 0) mbar_expect_tx(full + 8 * slot, 2 * kPairSlot);
                    const uint32_t to = ring + slot * kPairSlot;
                    copy_tile_pair(to, &map_x, k * kMatK, ta * 256 + rank * 128, full0 + 8 * slot);
                    copy_tile_pair(to + 128 * kMatK, &map_w, k * kMatK, tb * 256 + rank * 128, full0 + 8 * slot);
                }
                __syncwarp();
                taken++;
                if (++slot == kPairStages) {
                    slot = 0;
                    turn ^= 1;
                }
            }
        }
        // The pair must not end with copies in flight: the last products that read them have completed (each CTA sees that on its own
        // `empty`), or, where a wait ran out, the copies themselves (which the first CTA counts).
        for (uint32_t i = taken > kPairStages ? taken - kPairStages : 0; i < taken; i++) {
            bool late = false;
            mbar_wait_sleep((timed_out && rank == 0 ? full : empty) + 8 * (i % kPairStages), (int)(i / kPairStages), late);
            timed_out |= late;
        }
    } else if (warp == 1 && rank == 0) {
        const uint32_t ring_lo = one_value((uint32_t)tc_operand(ring)), tm = one_value(tmem), bar = one_value(bars);
        uint32_t slot = 0, turn = 0;
        int n = 0;
        for (int tile = first; tile < tiles && !timed_out; tile += step, n++) {
            const uint32_t b = one_value(n & 1);
            if (n >= 2 && !mbar_wait(acc_empty + 8 * b, (n >> 1) - 1, timed_out)) break;
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < a.blocks; k++) {
                const uint32_t at = one_value(slot), lo = ring_lo + at * (kPairSlot / 16), more = one_value(k > 0), last = one_value(k + 1 == a.blocks);
                if (!mbar_wait(full + 8 * slot, turn, timed_out)) break;
                if (elected()) {
#pragma unroll
                    for (int i = 0; i < 4; i++) mma_i8_pair(tm + b * 256, lo + 2 * i, lo + 128 * kMatK / 16 + 2 * i, i > 0 ? 1 : more);
                    commit_pair(bar + 8 * kPairStages + 8 * at);
                    if (last) commit_pair(bar + 16 * kPairStages + 8 * b);
                }
                __syncwarp();
                if (++slot == kPairStages) {
                    slot = 0;
                    turn ^= 1;
                }
            }
        }
    } else if (warp >= 2) {
        const int row = 32 * (warp & 3) + lane;
        const uint32_t mine = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const bool weights_wide = (((uintptr_t)a.w_scale | (uintptr_t)a.bias) & 15) == 0;
        int n = 0;
        for (int tile = first; tile < tiles && !timed_out; tile += step, n++) {
            const int b = n & 1;
            int ta, tb;
            place(tile, ta, tb);
            const long long token = (long long)ta * 256 + rank * 128 + row;
            const float xs = token < a.rows ? a.x_scale[token] : 0.0f;
            T* out = (T*)a.out + token * a.out_row;
            if (!mbar_wait_warp(acc_full + 8 * b, n >> 1, timed_out)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 256; c += 32) {
                uint32_t v[32];
                tc_load32(mine + b * 256 + c, v);
                const int ch0 = tb * 256 + c;
                if (token >= a.rows) {
                    // nothing to write
                } else if (a.wide && weights_wide && ch0 + 32 <= a.outer) {
                    constexpr int PER = 16 / sizeof(T);
#pragma unroll
                    for (int i = 0; i < 32; i += PER) {
                        __align__(16) T piece[PER];
#pragma unroll
                        for (int j = 0; j < PER; j += 4) {
                            const float4 w = __ldg(reinterpret_cast<const float4*>(a.w_scale + ch0 + i + j));
                            const float4 o = a.bias ? __ldg(reinterpret_cast<const float4*>(a.bias + ch0 + i + j)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                            piece[j] = output<T>((int)v[i + j], xs, w.x, o.x);
                            piece[j + 1] = output<T>((int)v[i + j + 1], xs, w.y, o.y);
                            piece[j + 2] = output<T>((int)v[i + j + 2], xs, w.z, o.z);
                            piece[j + 3] = output<T>((int)v[i + j + 3], xs, w.w, o.w);
                        }
                        *reinterpret_cast<uint4*>(out + ch0 + i) = *reinterpret_cast<const uint4*>(piece);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i++) {
                        const int ch = ch0 + i;
                        if (ch < a.outer) out[ch] = output<T>((int)v[i], xs, a.w_scale[ch], a.bias ? a.bias[ch] : 0.0f);
                    }
                }
                __syncwarp();                                   // (the next load is one for the whole warp, and some lanes may have no token)
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(map_to_rank(acc_empty + 8 * b, 0));
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();                                           // neither CTA ends while products may read its ring
    cluster_wait();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    if (timed_out) raise_status(a.status, kStatusWaitTimeout);
}

}  // namespace sttm
