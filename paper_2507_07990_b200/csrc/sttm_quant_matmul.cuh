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
// up and writes every size-th token.  Many tokens: tokens are the 128 rows, NT = 256 output channels the columns, the tensor
// cores bound it; one CTA per SM takes tile after tile, one accumulator being written out while the other fills.
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
    int stages;
    int32_t* status;
    bool wide;                    // rows of out can be written in 16-byte pieces
};

constexpr int kMatK = 128;                            // inner elements (bytes) per step
constexpr int kMatThreads = 6 * 32;                   // producer, products, four warps that read out
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
__device__ __forceinline__ int ld_remote_s32(uint32_t cluster_addr) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}

// Tiles run through kMatGroup tiles of A for every tile of B: the 148 tiles in work share 12 + 13 tiles of rows instead of 1 + 148.
__device__ __forceinline__ void tile_at(const MatmulArgs& a, int tile, int& ta, int& tb) {
    const int per = kMatGroup * a.b_tiles, group = tile / per, first = group * kMatGroup;
    const int size = min(kMatGroup, a.a_tiles - first), in = tile - group * per;
    tb = in / size;
    ta = first + in - tb * size;
}

template <typename T>
__device__ __forceinline__ T narrow(float v) { return (T)v; }

template <typename T, int NT, bool SWAP>
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

    // this CTA's tiles, and its part of the inner axis
    const int size = a.cluster, rank = size > 1 ? (int)cluster_rank() : 0;
    const int tiles = a.a_tiles * a.b_tiles, first = blockIdx.x / size, step = gridDim.x / size;
    const int k0 = (int)((long long)a.blocks * rank / size), k1 = (int)((long long)a.blocks * (rank + 1) / size);
    bool timed_out = false;
    int q = 0, n = 0;                                           // slots and accumulators taken up so far

    if (warp == 0) {
        for (int tile = first; tile < tiles && !timed_out; tile += step) {
            int ta, tb;
            tile_at(a, tile, ta, tb);
            for (int k = k0; k < k1; k++, q++) {
                const int s = q % a.stages;
                if (q >= a.stages && !mbar_wait(empty + 8 * s, q / a.stages - 1, timed_out)) break;
                if (lane == 0) {
                    mbar_expect_tx(full + 8 * s, SLOT);
                    copy_tile_2d(ring + s * SLOT, &map_a, k * kMatK, ta * 128, full + 8 * s);
                    copy_tile_2d(ring + s * SLOT + 128 * kMatK, &map_b, k * kMatK, tb * NT, full + 8 * s);
                }
                __syncwarp();
            }
        }
        // the CTA must not end with copies in flight
        for (int p = max(0, q - a.stages); p < q; p++) {
            bool late = false;
            mbar_wait_sleep(full + 8 * (p % a.stages), p / a.stages, late);
            timed_out |= late;
        }
    } else if (warp == 1) {
        for (int tile = first; tile < tiles && !timed_out; tile += step, n++) {
            const int b = n & 1;
            if (n >= 2 && !mbar_wait(acc_empty + 8 * b, (n >> 1) - 1, timed_out)) break;
            tc_fence_after();
            for (int k = k0; k < k1; k++, q++) {
                const int s = q % a.stages;
                if (!mbar_wait(full + 8 * s, q / a.stages, timed_out)) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint64_t da = tc_operand(ring + s * SLOT), db = tc_operand(ring + s * SLOT + 128 * kMatK);
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        mma_i8(tmem + b * NT, (uint32_t)da + 2 * i, (uint32_t)db + 2 * i, (uint32_t)(da >> 32), matmul_idesc(NT), k > k0 || i > 0);
                    tc_commit(empty + 8 * s);
                    if (k + 1 == k1) tc_commit(acc_full + 8 * b);
                }
                __syncwarp();
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
            if constexpr (SWAP) {
                const int ch = ta * 128 + row;
                const float ws = ch < a.outer ? a.w_scale[ch] : 0.0f, bias = a.bias && ch < a.outer ? a.bias[ch] : 0.0f;
                auto write = [&](int col, int sum) {
                    const long long token = (long long)tb * NT + col;
                    if (ch < a.outer && token < a.rows) ((T*)a.out)[token * a.out_row + ch] = narrow<T>((float)sum * a.x_scale[token] * ws + bias);
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
                }
                if (size > 1) {                                 // (one tile per cluster then, and the ring has been read)
                    cluster_arrive();
                    cluster_wait();
                    const int last = (int)min((long long)NT, a.rows - (long long)tb * NT);
                    for (int col = rank; col < last; col += size) {
                        int sum = 0;
                        for (int r = 0; r < size; r++) sum += ld_remote_s32(map_to_rank(ring + (col * 128 + row) * 4, r));
                        write(col, sum);
                    }
                }
            } else {
                const long long token = (long long)ta * 128 + row;
                const float xs = token < a.rows ? a.x_scale[token] : 0.0f;
                T* out = (T*)a.out + token * a.out_row;
#pragma unroll 1
                for (int c = 0; c < NT; c += 32) {
                    uint32_t v[32];
                    tc_load32(mine + b * NT + c, v);
                    const int ch0 = tb * NT + c;
                    if (token >= a.rows) continue;
                    if (a.wide && ch0 + 32 <= a.outer) {
                        constexpr int PER = 16 / sizeof(T);
#pragma unroll
                        for (int i = 0; i < 32; i += PER) {
                            __align__(16) T piece[PER];
#pragma unroll
                            for (int j = 0; j < PER; j++) {
                                const int ch = ch0 + i + j;
                                piece[j] = narrow<T>((float)(int)v[i + j] * xs * __ldg(a.w_scale + ch) + (a.bias ? __ldg(a.bias + ch) : 0.0f));
                            }
                            *reinterpret_cast<uint4*>(out + ch0 + i) = *reinterpret_cast<const uint4*>(piece);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i++) {
                            const int ch = ch0 + i;
                            if (ch < a.outer) out[ch] = narrow<T>((float)(int)v[i] * xs * a.w_scale[ch] + (a.bias ? a.bias[ch] : 0.0f));
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * b);
        }
    }
    if (SWAP && size > 1) {
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

}  // namespace sttm
