// Norm, rotation and cache entry of new tokens (sttm_cache_append).
//
// Every channel is read once and written once; the arithmetic in between (a sum of squares, a
// product, a turn) is a few operations per channel, so HBM bounds the kernel.  A head is taken by
// DIM / 16 lanes, two 16-byte words each, chosen so that both channels of every rotated pair lie in
// one lane: words c and c + rot / 16 for pairs (i, i + rot / 2), words 2 c and 2 c + 1 for pairs
// (2 i, 2 i + 1).  Either way lane c needs the angles 8 c ... 8 c + 7, the same for every head: the
// warp forms the row's rot / 2 angles once, two or so per lane, and passes them round through shared
// memory.
//
// A warp takes a row (few rows: a part of one) in steps of 1 KB and has two steps on their way into
// shared memory while it works on one (asynchronous copies; a lane reads back what it copied itself): 159 us, 6.5 TB/s, on
// 55724 rows of 36 heads of 128 channels in the first calls at 1965 MHz; call after call the power limit has the clock at 1.7 GHz,
// where the instructions bound it: 175 to 183 us, 5.7 TB/s.  In first calls loads into registers, one step ahead, took 191 us (the
// registers cost warps); seven steps on their way, 189 us (so does the shared memory, and L1 with it).
#pragma once

#include "sttm_cache.cuh"

namespace sttm {

struct AppendArgs {
    CacheView c;
    const uint16_t *q, *k, *v;
    long long q_row, q_head, k_row, k_head, v_row, v_head;
    uint16_t* q_out;
    long long rows;
    int q_heads;
    const long long* row_offsets;
    const int32_t* lengths;
    int32_t* new_lengths;
    const void* positions;
    int positions_f32;
    long long axis_stride;
    int sec0, sec1;               // pairs below sec0 turn by axis 0, below sec1 by axis 1, the others by axis 2
    const float* inv_freq;
    int rot;
    const float *q_norm, *k_norm;
    float eps;
    int32_t* status;
    int parts;                    // warps that share one row's heads
};

constexpr int kAppendWarps = 4;
constexpr int kAppendRing = 3;          // steps: two on their way, one being read

__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <typename T, int DIM, bool INTERLEAVED>
__global__ void __launch_bounds__(kAppendWarps * 32) k_cache_append(const __grid_constant__ AppendArgs a) {
    constexpr int LPH = DIM / 16;                           // lanes per head
    constexpr int HPW = 32 / LPH;                           // heads per warp and step
    __shared__ uint4 ring[kAppendWarps][kAppendRing][2][32];
    __shared__ float4 turns[kAppendWarps][DIM / 4];         // {cos, sin} of angles 2 i and 2 i + 1
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_prior_kernel();
    let_next_kernel_start();
    const int seqs = a.c.seqs;
    const long long first = a.row_offsets[0], total = a.row_offsets[seqs];      // rows [first, total) are tokens
    // Offsets may name more rows than there are (those of a merge whose output buffer was too small do): a sequence gets
    // the slots of the rows that are there, no others.
    if (a.new_lengths != nullptr && blockIdx.x == 0)
        for (int b = threadIdx.x; b < seqs; b += blockDim.x) {
            const long long begin = a.row_offsets[b], end = min(a.row_offsets[b + 1], a.rows);
            a.new_lengths[b] = (a.lengths ? a.lengths[b] : 0) + (int)max(end - begin, 0ll);
        }
    if (total > a.rows && blockIdx.x == 0 && threadIdx.x == 0) raise_status(a.status, kStatusCapacity);
    const long long w = (long long)blockIdx.x * kAppendWarps + warp;
    const long long row = w / a.parts;
    const int part = (int)(w - row * a.parts);
    if (row >= a.rows || row < first || row >= total) return;

    const int c = lane % LPH, sub = lane / LPH;
    const int rw = a.rot / 16;                              // rotated words per half = lanes that turn
    int w0, w1;                                             // this lane's 16-byte words of a head
    if (INTERLEAVED) { w0 = 2 * c; w1 = 2 * c + 1; }
    else if (c < rw) { w0 = c; w1 = c + rw; }
    else { w0 = 2 * c; w1 = 2 * c + 1; }                    // (channels from rot on: words 2 rw + 2 (c - rw), and the next)
    const bool turn = c < rw;
    // Steps of HPW heads: queries, keys, values; a step is of one kind for the whole warp.
    const int sq = (a.q_heads + HPW - 1) / HPW, sk = (a.c.heads + HPW - 1) / HPW, steps = sq + 2 * sk;
    auto source = [&](int s, int& h) -> const uint4* {
        const uint16_t* src;
        if (s < sq) {
            h = s * HPW + sub;
            src = h < a.q_heads ? a.q + row * a.q_row + h * a.q_head : nullptr;
        } else if (s < sq + sk) {
            h = (s - sq) * HPW + sub;
            src = h < a.c.heads ? a.k + row * a.k_row + h * a.k_head : nullptr;
        } else {
            h = (s - sq - sk) * HPW + sub;
            src = h < a.c.heads ? a.v + row * a.v_row + h * a.v_head : nullptr;
        }
        return reinterpret_cast<const uint4*>(src);
    };
    const uint32_t mine0 = smem_u32(&ring[warp][0][0][lane]);
    auto copy = [&](int s, int slot) {
        if (s < steps) {
            int h;
            const uint4* src = source(s, h);
            if (src != nullptr) {
                copy_async_16(mine0 + slot * 1024, src + w0);
                copy_async_16(mine0 + slot * 1024 + 512, src + w1);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int d = 0; d < kAppendRing - 1; d++) copy(part + d * a.parts, d);

    // while they are on their way: the row's place, and its turns.  The angle in turns is formed in 64 bits and
    // brought into [-1/2, 1/2] there.
    const int seq = sequence_of(a.row_offsets, seqs, row, lane);
    const long long slot = (a.lengths ? a.lengths[seq] : 0) + (row - a.row_offsets[seq]);
    const long long at = slot_at(a.c, seq, slot, lane == 0 && part == 0 ? a.status : nullptr);
    for (int i = lane; i < a.rot / 2; i += 32) {
        const long long pi = row + (i < a.sec0 ? 0 : (i < a.sec1 ? a.axis_stride : 2 * a.axis_stride));
        const double pos = a.positions_f32 ? (double)((const float*)a.positions)[pi] : (double)((const int32_t*)a.positions)[pi];
        const double t = pos * (double)a.inv_freq[i] * 0.15915494309189533577;     // 1 / (2 pi)
        float sn, cn;
        sincospif(2.f * (float)(t - rint(t)), &sn, &cn);
        reinterpret_cast<float2*>(turns[warp])[i] = make_float2(cn, sn);
    }
    __syncwarp();
    float4 cs[4];                                           // this lane's eight angles (it turns heads of every step by them)
#pragma unroll
    for (int e = 0; e < 4; e++) cs[e] = turn ? turns[warp][4 * c + e] : make_float4(1.f, 0.f, 1.f, 0.f);

    int at_slot = 0;
    for (int s = part; s < steps; s += a.parts) {
        copy(s + (kAppendRing - 1) * a.parts, at_slot == 0 ? kAppendRing - 1 : at_slot - 1);    // into the slot read a step ago
        asm volatile("cp.async.wait_group %0;" ::"n"(kAppendRing - 1) : "memory");
        uint4 x0 = ring[warp][at_slot][0][lane], x1 = ring[warp][at_slot][1][lane];
        if (++at_slot == kAppendRing) at_slot = 0;
        int h;
        const bool mine = source(s, h) != nullptr;
        uint16_t* dst = s < sq ? a.q_out + (row * a.q_heads + h) * DIM
                               : (at < 0 ? nullptr : (s < sq + sk ? a.c.k : a.c.v) + at + h * a.c.head_stride);
        if (s < sq + sk) {
            float f[16];
            const uint32_t u[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float2 p = Pair<T>::split(u[e]);
                f[2 * e] = p.x;
                f[2 * e + 1] = p.y;
            }
            const float* wt = s < sq ? a.q_norm : a.k_norm;
            if (wt != nullptr) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e++) ss = fmaf(f[e], f[e], ss);
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                const float r = rsqrtf(ss * (1.f / DIM) + a.eps);
                const float4* w4 = reinterpret_cast<const float4*>(wt);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float4 g = __ldg(w4 + (e < 2 ? 2 * w0 + e : 2 * w1 + e - 2));
                    f[4 * e] *= r * g.x;
                    f[4 * e + 1] *= r * g.y;
                    f[4 * e + 2] *= r * g.z;
                    f[4 * e + 3] *= r * g.w;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {                   // (lanes that do not turn: by (1, 0))
                float &p = INTERLEAVED ? f[2 * e] : f[e], &t = INTERLEAVED ? f[2 * e + 1] : f[e + 8];
                const float cn = e & 1 ? cs[e / 2].z : cs[e / 2].x, sn = e & 1 ? cs[e / 2].w : cs[e / 2].y;
                const float y = turn ? p * cn - t * sn : p;
                t = turn ? t * cn + p * sn : t;
                p = y;
            }
            x0 = make_uint4(Pair<T>::pack(f[0], f[1]), Pair<T>::pack(f[2], f[3]), Pair<T>::pack(f[4], f[5]), Pair<T>::pack(f[6], f[7]));
            x1 = make_uint4(Pair<T>::pack(f[8], f[9]), Pair<T>::pack(f[10], f[11]), Pair<T>::pack(f[12], f[13]), Pair<T>::pack(f[14], f[15]));
        }
        if (mine && dst != nullptr) {
            reinterpret_cast<uint4*>(dst)[w0] = x0;
            reinterpret_cast<uint4*>(dst)[w1] = x1;
        }
    }
}

}  // namespace sttm
