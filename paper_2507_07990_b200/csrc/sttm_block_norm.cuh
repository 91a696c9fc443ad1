// Between two blocks of a decoder layer (sttm_block_norm): the block's output normed, gated and added to the scaled residual
// stream, and the norm before the next block, its output in the rows' type or in 8 bits; and rows quantized as they come or out
// of a gated activation (sttm_quantize_rows).
//
//     r = a * residual + g * x / sqrt(mean x^2 + eps) * w_post          t = r * w_pre
//     out = t / sqrt(mean r^2 + eps)                                    q = rint(t * 127 / max|t|)
//
// The second norm's factor is the same for a whole row, so it drops out of q and only enters the row's
// scale max|t| / 127 / sqrt(...): the largest |t| and the sum of squares of r are one reduction.
//
// Every element is read once and written once, with some ten operations between: HBM bounds it.  A row is held in registers
// (32 elements a thread at most) by 32 to 1024 threads; sums of squares run in 32 bits.
#pragma once

#include "sttm_cache.cuh"

namespace sttm {

struct NormArgs {
    const void *x, *residual, *gate_rows;
    long long x_row, residual_row, gate_row;            // elements
    const float *post_norm, *gate, *pre_norm;
    float residual_scale, eps;
    void *sum, *out;
    long long sum_row, out_row;
    int8_t* q;
    long long q_row;
    float* q_scale;
    long long rows;
    int dim;
    bool gated;                                         // quantize: x is [rows][2 dim], silu(first half) * second half
};

constexpr int kNormMaxDim = 16384;

// VEC elements in 16 bytes, or one.  A row's words are all on their way before the first is used, and before anything is stored: an
// output may take the place of an input, so the compiler moves no load over a store (plain loads, for the same reason).
template <typename T, int VEC>
struct Elements;
template <typename T>
struct Elements<T, 8> {
    typedef uint4 Raw;
    static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const uint4*>(p); }
    static __device__ __forceinline__ void split(const Raw& w, float (&f)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 v = Pair<T>::split(u[i]);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
    static __device__ __forceinline__ void store(T* p, const float (&f)[8]) {
        *reinterpret_cast<uint4*>(p) = make_uint4(Pair<T>::pack(f[0], f[1]), Pair<T>::pack(f[2], f[3]), Pair<T>::pack(f[4], f[5]), Pair<T>::pack(f[6], f[7]));
    }
};
template <>
struct Elements<float, 4> {
    typedef float4 Raw;
    static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const float4*>(p); }
    static __device__ __forceinline__ void split(const Raw& w, float (&f)[4]) { f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w; }
    static __device__ __forceinline__ void store(float* p, const float (&f)[4]) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T>
struct Elements<T, 1> {
    typedef T Raw;
    static __device__ __forceinline__ Raw load(const T* p) { return *p; }
    static __device__ __forceinline__ void split(const Raw& w, float (&f)[1]) { f[0] = (float)w; }
    static __device__ __forceinline__ void store(T* p, const float (&f)[1]) { *p = (T)f[0]; }
};

template <int VEC>
__device__ __forceinline__ void load_weights(const float* p, float (&f)[VEC]) {
    if constexpr (VEC == 1) {
        f[0] = __ldg(p);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 w = __ldg(reinterpret_cast<const float4*>(p + i));
            f[i] = w.x; f[i + 1] = w.y; f[i + 2] = w.z; f[i + 3] = w.w;
        }
    }
}

// Sum of v over the row's threads, and the largest of the bit patterns m (absolute values: their patterns compare as they do,
// infinities and NaN above all numbers).  `slots`: one per warp, not used by the reduction before.
template <int TPR, bool MAX>
__device__ __forceinline__ void reduce_row(float& v, uint32_t& m, float2* slots) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (MAX) m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (TPR > 32) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0) slots[warp] = make_float2(v, __uint_as_float(m));
        __syncthreads();
        const float2 s = lane < TPR / 32 ? slots[lane] : make_float2(0.0f, 0.0f);
        v = s.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (MAX) m = __reduce_max_sync(0xffffffffu, __float_as_uint(s.y));
    }
}

// Factor that takes a row whose largest |t| has this bit pattern to 8 bits, and the step.  A row that holds an infinity or a
// NaN gives zeros with the step NaN; one below 2^-100 zeros with the step 0.
__device__ __forceinline__ void quant_step(uint32_t largest, float& factor, float& step) {
    const float m = __uint_as_float(largest);
    factor = m < 7.9e-31f || largest >= 0x7f800000u ? 0.0f : 127.0f / m;
    step = largest >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : m < 7.9e-31f ? 0.0f : m * (1.0f / 127.0f);
}

template <int VEC>
__device__ __forceinline__ void store_bytes(int8_t* p, const float (&t)[VEC], float factor) {
    int b[VEC];
#pragma unroll
    for (int i = 0; i < VEC; i++) b[i] = factor == 0.0f ? 0 : __float2int_rn(t[i] * factor);      // (0 * inf)
    if constexpr (VEC == 1) {
        *p = (int8_t)b[0];
    } else {
        uint32_t w[VEC / 4];
#pragma unroll
        for (int i = 0; i < VEC / 4; i++)
            w[i] = (b[4 * i] & 255) | (b[4 * i + 1] & 255) << 8 | (b[4 * i + 2] & 255) << 16 | (uint32_t)b[4 * i + 3] << 24;
        if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
}

// TPR threads per row, each with chunks of VEC elements TPR * VEC apart.  TPR = 32: a warp takes a row, four rows to a block.
template <typename T, int VEC, int TPR>
constexpr int kNormBlock = TPR == 32 ? 128 : TPR;

template <typename T, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(kNormBlock<T, VEC, TPR>) k_block_norm(const __grid_constant__ NormArgs a) {
    using E = Elements<T, VEC>;
    constexpr int PER_BLOCK = kNormBlock<T, VEC, TPR> / TPR;
    __shared__ float2 slots[2][32];
    wait_for_prior_kernel();
    let_next_kernel_start();
    const long long row = (long long)blockIdx.x * PER_BLOCK + threadIdx.x / TPR;
    if (row >= a.rows) return;                                              // (whole warps: TPR is a multiple of 32)
    const int t = threadIdx.x % TPR;
    typename E::Raw x[NCH], residual[NCH], gate[NCH];
    {
        const T *const xs = (const T*)a.x + row * a.x_row, *const rs = (const T*)a.residual + row * a.residual_row, *const gs = (const T*)a.gate_rows + row * a.gate_row;
#pragma unroll
        for (int c = 0; c < NCH; c++) {
            const int at = (c * TPR + t) * VEC;
            if (at < a.dim) x[c] = E::load(xs + at);
        }
        if (a.residual != nullptr)
#pragma unroll
            for (int c = 0; c < NCH; c++) {
                const int at = (c * TPR + t) * VEC;
                if (at < a.dim) residual[c] = E::load(rs + at);
            }
        if (a.gate_rows != nullptr)
#pragma unroll
            for (int c = 0; c < NCH; c++) {
                const int at = (c * TPR + t) * VEC;
                if (at < a.dim) gate[c] = E::load(gs + at);
            }
    }
    float r[NCH][VEC];
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at < a.dim) E::split(x[c], r[c]);
        else
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] = 0.0f;
    }
    uint32_t largest = 0;
    float squares = 0.0f;
    if (a.post_norm != nullptr) {
#pragma unroll
        for (int c = 0; c < NCH; c++)
#pragma unroll
            for (int i = 0; i < VEC; i++) squares += r[c][i] * r[c][i];
        reduce_row<TPR, false>(squares, largest, slots[0]);
        const float f = rsqrtf(squares / (float)a.dim + a.eps);
#pragma unroll
        for (int c = 0; c < NCH; c++) {
            const int at = (c * TPR + t) * VEC;
            if (at < a.dim) {
                float w[VEC];
                load_weights<VEC>(a.post_norm + at, w);
#pragma unroll
                for (int i = 0; i < VEC; i++) r[c][i] = r[c][i] * f * w[i];
            }
        }
    }
    squares = 0.0f;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at >= a.dim) continue;
        float w[VEC];
        if (a.gate != nullptr) {
            load_weights<VEC>(a.gate + at, w);
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] *= w[i];
        }
        if (a.gate_rows != nullptr) {
            E::split(gate[c], w);
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] *= w[i];
        }
        if (a.residual != nullptr) {
            E::split(residual[c], w);
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] = fmaf(a.residual_scale, w[i], r[c][i]);
        }
        if (a.sum != nullptr) E::store((T*)a.sum + row * a.sum_row + at, r[c]);
#pragma unroll
        for (int i = 0; i < VEC; i++) squares += r[c][i] * r[c][i];
        if (a.pre_norm != nullptr) {
            load_weights<VEC>(a.pre_norm + at, w);
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] *= w[i];
        }
        if (a.q != nullptr)
#pragma unroll
            for (int i = 0; i < VEC; i++) largest = max(largest, __float_as_uint(r[c][i]) & 0x7fffffffu);
    }
    if (a.out == nullptr && a.q == nullptr) return;
    float f = 1.0f;
    if (a.pre_norm != nullptr || a.q != nullptr) {
        reduce_row<TPR, true>(squares, largest, slots[1]);
        if (a.pre_norm != nullptr) f = rsqrtf(squares / (float)a.dim + a.eps);
    }
    float factor = 0.0f, step = 0.0f;
    if (a.q != nullptr) {
        quant_step(largest, factor, step);
        if (t == 0) a.q_scale[row] = step * f;
    }
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at >= a.dim) continue;
        if (a.q != nullptr) store_bytes<VEC>(a.q + row * a.q_row + at, r[c], factor);
        if (a.out != nullptr) {
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] *= f;
            E::store((T*)a.out + row * a.out_row + at, r[c]);
        }
    }
}

// Rows to 8 bits, as they are or silu(a) * b of a row [a | b].
template <typename T, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(kNormBlock<T, VEC, TPR>) k_quantize_rows(const __grid_constant__ NormArgs a) {
    using E = Elements<T, VEC>;
    constexpr int PER_BLOCK = kNormBlock<T, VEC, TPR> / TPR;
    __shared__ float2 slots[32];
    wait_for_prior_kernel();
    let_next_kernel_start();
    const long long row = (long long)blockIdx.x * PER_BLOCK + threadIdx.x / TPR;
    if (row >= a.rows) return;
    const int t = threadIdx.x % TPR;
    typename E::Raw x[NCH], b[NCH];
    const T* xs = (const T*)a.x + row * a.x_row;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at < a.dim) x[c] = E::load(xs + at);
    }
    if (a.gated)
#pragma unroll
        for (int c = 0; c < NCH; c++) {
            const int at = (c * TPR + t) * VEC;
            if (at < a.dim) b[c] = E::load(xs + a.dim + at);
        }
    float r[NCH][VEC];
    uint32_t largest = 0;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at >= a.dim) continue;
        E::split(x[c], r[c]);
        if (a.gated) {
            float g[VEC];
            E::split(b[c], g);
#pragma unroll
            for (int i = 0; i < VEC; i++) r[c][i] = r[c][i] / (1.0f + expf(-r[c][i])) * g[i];
        }
#pragma unroll
        for (int i = 0; i < VEC; i++) largest = max(largest, __float_as_uint(r[c][i]) & 0x7fffffffu);
    }
    float none = 0.0f, factor, step;
    reduce_row<TPR, true>(none, largest, slots);
    quant_step(largest, factor, step);
    if (t == 0) a.q_scale[row] = step;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        const int at = (c * TPR + t) * VEC;
        if (at < a.dim) store_bytes<VEC>(a.q + row * a.q_row + at, r[c], factor);
    }
}

}  // namespace sttm
