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
// Every element is read once and written once, with some ten operations between: HBM bounds it.  A row is held in registers by
// 32 to 1024 threads, or goes through a warp out of shared memory.  Sums of squares run in 32 bits, in two chains a thread of at most 16 terms or, for a warp
// to a row (9600 channels at most), 150, and a tree: off by less than 2^-16.7.  Measured: 55724 bf16 rows of 3584, both norms and a gate, 280 us at full
// clocks (5.7 TB/s, 87 % of the copy rate); quantized 106 us (86 %); 15630 fp16 rows of 1157 with gates of their own 48.8 us
// (two elements at a time: instructions bound it).
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
    int32_t* status;
};

constexpr int kNormMaxDim = 16384, kQuantizeMaxDim = 32768;     // (beyond the first: rows of whole 16-byte words only)

// VEC elements in 16 bytes, or one.  A row's words are all on their way before the first is used, and before anything is stored: an
// output may take the place of an input, so the compiler moves no load over a store (plain loads, for the same reason).
template <typename T, int VEC>
struct Elements;
template <typename T>
struct Elements<T, 8> {
    typedef uint4 Raw;
    static __device__ __forceinline__ void split(const Raw& w, uint64_t (&f)[4]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 v = Pair<T>::split(u[i]);
            f[i] = both(v.x, v.y);
        }
    }
    static __device__ __forceinline__ void store(T* p, const uint64_t (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float x, y;
            apart(f[i], x, y);
            w[i] = Pair<T>::pack(x, y);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Elements<float, 4> {
    typedef float4 Raw;
    static __device__ __forceinline__ void split(const Raw& w, uint64_t (&f)[2]) {
        f[0] = both(w.x, w.y);
        f[1] = both(w.z, w.w);
    }
    static __device__ __forceinline__ void store(float* p, const uint64_t (&f)[2]) {
        float4 w;
        apart(f[0], w.x, w.y);
        apart(f[1], w.z, w.w);
        *reinterpret_cast<float4*>(p) = w;
    }
};

template <typename T>
struct Elements<T, 2> {
    typedef uint32_t Raw;
    static __device__ __forceinline__ void split(const Raw& w, uint64_t (&f)[1]) {
        const float2 v = Pair<T>::split(w);
        f[0] = both(v.x, v.y);
    }
    static __device__ __forceinline__ void store(T* p, const uint64_t (&f)[1]) {
        float x, y;
        apart(f[0], x, y);
        *reinterpret_cast<uint32_t*>(p) = Pair<T>::pack(x, y);
    }
};

// A thread's VEC values of a chunk, two to a register pair, and what is done with them.
template <typename T, int VEC>
struct Chunk {
    typedef typename Elements<T, VEC>::Raw Raw;
    uint64_t v[VEC / 2];
    __device__ __forceinline__ void split(const Raw& w) { Elements<T, VEC>::split(w, v); }
    __device__ __forceinline__ void store(T* p) const { Elements<T, VEC>::store(p, v); }
    __device__ __forceinline__ void weights(const float* p) {
        if (VEC == 8 && ((uintptr_t)p & 31) == 0) {             // (two loads of 16 bytes would take twice the L1 cycles)
            asm volatile("ld.global.nc.v4.b64 {%0, %1, %2, %3}, [%4];" : "=l"(v[0]), "=l"(v[1]), "=l"(v[VEC / 2 - 2]), "=l"(v[VEC / 2 - 1]) : "l"(p));
        } else {
#pragma unroll
            for (int i = 0; i < VEC / 2; i += 2) {
                const ulonglong2 w = __ldg(reinterpret_cast<const ulonglong2*>(p + 2 * i));
                v[i] = w.x;
                v[i + 1] = w.y;
            }
        }
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) v[i] = mul2(v[i], both(f, f));
    }
    __device__ __forceinline__ void times(const Chunk& o) {
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) v[i] = mul2(v[i], o.v[i]);
    }
    __device__ __forceinline__ void add(float f, const Chunk& o) {
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) v[i] = fma2(both(f, f), o.v[i], v[i]);
    }
    __device__ __forceinline__ void square(uint64_t& sum) const {
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) sum = fma2(v[i], v[i], sum);
    }
    // weights i, i + 1, ... of `dim` as k_norm_rows keeps them
    __device__ __forceinline__ void kept(const float* p, int i, int dim) {
        const ulonglong2 lo = *reinterpret_cast<const ulonglong2*>(p + (VEC == 8 ? i / 2 : i));
        v[0] = lo.x;
        v[1] = lo.y;
        if constexpr (VEC == 8) {
            const ulonglong2 hi = *reinterpret_cast<const ulonglong2*>(p + dim / 2 + i / 2);
            v[VEC / 2 - 2] = hi.x;
            v[VEC / 2 - 1] = hi.y;
        }
    }
    // the values in 32 bits in the place of two chunks of 16-bit rows, or of one of 32-bit rows
    __device__ __forceinline__ void park(T* x, T* y) const {
        *reinterpret_cast<ulonglong2*>(x) = make_ulonglong2(v[0], v[1]);
        if constexpr (VEC == 8) *reinterpret_cast<ulonglong2*>(y) = make_ulonglong2(v[VEC / 2 - 2], v[VEC / 2 - 1]);
    }
    __device__ __forceinline__ void unpark(const T* x, const T* y) {
        const ulonglong2 lo = *reinterpret_cast<const ulonglong2*>(x);
        v[0] = lo.x;
        v[1] = lo.y;
        if constexpr (VEC == 8) {
            const ulonglong2 hi = *reinterpret_cast<const ulonglong2*>(y);
            v[VEC / 2 - 2] = hi.x;
            v[VEC / 2 - 1] = hi.y;
        }
    }
    __device__ __forceinline__ void largest(float& m) const {   // NaN if one is
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) {
            float x, y;
            apart(v[i], x, y);
            m = max3(m, fabsf(x), fabsf(y));
        }
    }
    __device__ __forceinline__ void gated(const Chunk& g) {     // silu(v) * g
#pragma unroll
        for (int i = 0; i < VEC / 2; i++) {
            float x, y;
            apart(v[i], x, y);
            v[i] = mul2(both(x / (1.0f + expf(-x)), y / (1.0f + expf(-y))), g.v[i]);
        }
    }
    __device__ __forceinline__ void bytes(int8_t* p, float factor) const {
        uint32_t w[VEC / 4];
#pragma unroll
        for (int i = 0; i < VEC / 4; i++) {
            float x[4];
            apart(v[2 * i], x[0], x[1]);
            apart(v[2 * i + 1], x[2], x[3]);
            int b[4];
#pragma unroll
            for (int k = 0; k < 4; k++) b[k] = __float2int_rn(x[k] * factor);
            w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        }
        if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
};
template <typename T>
struct Chunk<T, 1> {
    typedef T Raw;
    float v;
    __device__ __forceinline__ void split(const Raw& w) { v = (float)w; }
    __device__ __forceinline__ void store(T* p) const { *p = (T)v; }
    __device__ __forceinline__ void weights(const float* p) { v = __ldg(p); }
    __device__ __forceinline__ void scale(float f) { v *= f; }
    __device__ __forceinline__ void times(const Chunk& o) { v *= o.v; }
    __device__ __forceinline__ void add(float f, const Chunk& o) { v = fmaf(f, o.v, v); }
    __device__ __forceinline__ void square(uint64_t& sum) const {  // (to either half by turns: chains as short as those of two elements at a time)
        float x, y;
        apart(sum, x, y);
        sum = both(y, fmaf(v, v, x));
    }
    __device__ __forceinline__ void kept(const float* p, int i, int) { v = p[i]; }
    __device__ __forceinline__ void park(T* x, T* y) const {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float*>(x) = v;
        } else {
            *reinterpret_cast<uint16_t*>(x) = (uint16_t)__float_as_uint(v);
            *reinterpret_cast<uint16_t*>(y) = (uint16_t)(__float_as_uint(v) >> 16);
        }
    }
    __device__ __forceinline__ void unpark(const T* x, const T* y) {
        if constexpr (sizeof(T) == 4) v = *reinterpret_cast<const float*>(x);
        else v = __uint_as_float(*reinterpret_cast<const uint16_t*>(x) | (uint32_t)*reinterpret_cast<const uint16_t*>(y) << 16);
    }
    __device__ __forceinline__ void largest(float& m) const { m = max3(m, fabsf(v), 0.0f); }
    __device__ __forceinline__ void gated(const Chunk& g) { v = v / (1.0f + expf(-v)) * g.v; }
    __device__ __forceinline__ void bytes(int8_t* p, float factor) const { *p = (int8_t)__float2int_rn(v * factor); }
};

// Two elements of a 16-bit row that share a 32-bit word, parked as Chunk<T, 1> does it.
template <typename T>
struct Two : Chunk<T, 2> {
    __device__ __forceinline__ void kept(const float* p, int i, int) { this->v[0] = both(p[i], p[i + 1]); }
    __device__ __forceinline__ void park(T* x, T* y) const {
        float e, f;
        apart(this->v[0], e, f);
        *reinterpret_cast<uint32_t*>(x) = __byte_perm(__float_as_uint(e), __float_as_uint(f), 0x5410);
        *reinterpret_cast<uint32_t*>(y) = __byte_perm(__float_as_uint(e), __float_as_uint(f), 0x7632);
    }
    __device__ __forceinline__ void unpark(const T* x, const T* y) {
        const uint32_t lo = *reinterpret_cast<const uint32_t*>(x), hi = *reinterpret_cast<const uint32_t*>(y);
        this->v[0] = both(__uint_as_float(__byte_perm(lo, hi, 0x5410)), __uint_as_float(__byte_perm(lo, hi, 0x7632)));
    }
    __device__ __forceinline__ void bytes(int8_t* p, float factor) const {
        float e, f;
        apart(this->v[0], e, f);
        p[0] = (int8_t)__float2int_rn(e * factor);
        p[1] = (int8_t)__float2int_rn(f * factor);
    }
};

// Sum of v over the row's threads, and the largest of the bit patterns m (absolute values: their patterns compare as they do,
// infinities and NaN above all numbers).  `slots`: one per warp, not used by the reduction before.
template <int TPR>
__device__ __forceinline__ void reduce_row(float& v, uint32_t& m, bool max_too, float2* slots) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (max_too) m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (TPR > 32) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0) slots[warp] = make_float2(v, __uint_as_float(m));
        __syncthreads();
        constexpr int WARPS = TPR / 32;
        const float2 s = slots[lane % WARPS];
        v = s.x;
#pragma unroll
        for (int o = WARPS / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (max_too) m = __reduce_max_sync(0xffffffffu, __float_as_uint(s.y));
    }
}

// Factor that takes a row whose largest |t| has this bit pattern to 8 bits, and the step.  A row that holds an infinity or a
// NaN gives zeros with the step NaN; one below 2^-100 zeros with the step 0.
// (inf * 0 is NaN, and NaN converts to 0.)
__device__ __forceinline__ void quant_step(uint32_t largest, float& factor, float& step) {
    const float m = __uint_as_float(largest);
    factor = m < 7.9e-31f || largest >= 0x7f800000u ? 0.0f : 127.0f / m;
    step = largest >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : m < 7.9e-31f ? 0.0f : m * (1.0f / 127.0f);
}

// ---- few rows: a block each ----

// TPR threads per row with NCH chunks of VEC elements each, TPR * VEC apart.  TPR = 32: each of a block's four warps takes a row.
__host__ __device__ constexpr int norm_block(int tpr) { return tpr == 32 ? 128 : tpr; }

template <typename T, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(norm_block(TPR)) k_block_norm(const __grid_constant__ NormArgs a) {
    typedef Chunk<T, VEC> C;
    constexpr int PER_BLOCK = norm_block(TPR) / TPR, STEP = TPR * VEC;
    __shared__ float2 slots[2][32];
    wait_for_prior_kernel();
    let_next_kernel_start();
    const long long row = (long long)blockIdx.x * PER_BLOCK + threadIdx.x / TPR;
    if (row >= a.rows) return;                                              // (whole warps)
    const int at = threadIdx.x % TPR * VEC;
    bool in[NCH];
#pragma unroll
    for (int c = 0; c < NCH; c++) in[c] = at + c * STEP < a.dim;
    auto fetch = [&](typename C::Raw (&to)[NCH], const void* base, long long stride) {
        if (base == nullptr) return;
        const T* from = (const T*)base + row * stride + at;
#pragma unroll
        for (int c = 0; c < NCH; c++)
            if (in[c]) to[c] = *reinterpret_cast<const typename C::Raw*>(from + c * STEP);
    };
    typename C::Raw x[NCH], residual[NCH], gate[NCH];
    fetch(x, a.x, a.x_row);
    fetch(residual, a.residual, a.residual_row);
    fetch(gate, a.gate_rows, a.gate_row);
    const float per = 1.0f / (float)a.dim;
    C r[NCH], w;
    uint32_t bits = 0;
    float s0, s1, f = 1.0f;
#pragma unroll
    for (int c = 0; c < NCH; c++)
        if (in[c]) r[c].split(x[c]);
    if (a.post_norm != nullptr) {
        uint64_t squares = 0;
#pragma unroll
        for (int c = 0; c < NCH; c++)
            if (in[c]) r[c].square(squares);
        apart(squares, s0, s1);
        s0 += s1;
        reduce_row<TPR>(s0, bits, false, slots[0]);
        f = rsqrtf(s0 * per + a.eps);
    }
    uint64_t squares = 0;
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        if (!in[c]) continue;
        if (a.post_norm != nullptr) {
            r[c].scale(f);
            w.weights(a.post_norm + at + c * STEP);
            r[c].times(w);
        }
        if (a.gate != nullptr) {
            w.weights(a.gate + at + c * STEP);
            r[c].times(w);
        }
        if (a.gate_rows != nullptr) {
            w.split(gate[c]);
            r[c].times(w);
        }
        if (a.residual != nullptr) {
            w.split(residual[c]);
            r[c].add(a.residual_scale, w);
        }
        r[c].square(squares);
        if (a.sum != nullptr) r[c].store((T*)a.sum + row * a.sum_row + at + c * STEP);
        if (a.pre_norm != nullptr) {
            w.weights(a.pre_norm + at + c * STEP);
            r[c].times(w);
        }
        if (a.q != nullptr) r[c].largest(m);
    }
    if (a.out == nullptr && a.q == nullptr) return;
    apart(squares, s0, s1);
    s0 += s1;
    bits = __float_as_uint(m);
    reduce_row<TPR>(s0, bits, a.q != nullptr, slots[1]);
    f = a.pre_norm != nullptr ? rsqrtf(s0 * per + a.eps) : 1.0f;
    float factor = 0.0f, quantum = 0.0f;
    if (a.q != nullptr) {
        quant_step(bits, factor, quantum);
        if (at == 0) a.q_scale[row] = quantum * f;
    }
#pragma unroll
    for (int c = 0; c < NCH; c++) {
        if (!in[c]) continue;
        if (a.q != nullptr) r[c].bytes(a.q + row * a.q_row + at + c * STEP, factor);
        if (a.out != nullptr) {
            r[c].scale(f);
            r[c].store((T*)a.out + row * a.out_row + at + c * STEP);
        }
    }
}

// Rows to 8 bits, as they are or silu(a) * b of a row [a | b].
template <typename T, int VEC, int TPR, int NCH>
__global__ void __launch_bounds__(norm_block(TPR)) k_quantize_rows(const __grid_constant__ NormArgs a) {
    typedef Chunk<T, VEC> C;
    constexpr int PER_BLOCK = norm_block(TPR) / TPR, STEP = TPR * VEC;
    __shared__ float2 slots[32];
    wait_for_prior_kernel();
    let_next_kernel_start();
    const long long row = (long long)blockIdx.x * PER_BLOCK + threadIdx.x / TPR;
    if (row >= a.rows) return;
    const int at = threadIdx.x % TPR * VEC;
    const T* from = (const T*)a.x + row * a.x_row + at;
    typename C::Raw x[NCH], b[NCH];
#pragma unroll
    for (int c = 0; c < NCH; c++)
        if (at + c * STEP < a.dim) {
            x[c] = *reinterpret_cast<const typename C::Raw*>(from + c * STEP);
            if (a.gated) b[c] = *reinterpret_cast<const typename C::Raw*>(from + a.dim + c * STEP);
        }
    C r[NCH];
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < NCH; c++)
        if (at + c * STEP < a.dim) {
            r[c].split(x[c]);
            if (a.gated) {
                C g;
                g.split(b[c]);
                r[c].gated(g);
            }
            r[c].largest(m);
        }
    uint32_t bits = __float_as_uint(m);
    float none = 0.0f, factor, quantum;
    reduce_row<TPR>(none, bits, true, slots);
    quant_step(bits, factor, quantum);
    if (at == 0) a.q_scale[row] = quantum;
#pragma unroll
    for (int c = 0; c < NCH; c++)
        if (at + c * STEP < a.dim) r[c].bytes(a.q + row * a.q_row + at + c * STEP, factor);
}

// ---- many rows: a warp each, out of shared memory ----

// A block's way through a row is latency: its loads, two barriers, the threads that they wait for.  Here a warp brings whole rows into shared
// memory (a bulk copy per array, the next as soon as its last pass over a row is done), so that an SM has a dozen rows or more on
// their way or in work and none waits for another.  The passes: sum of squares of x; r, its sum of squares and t, which takes the place
// of x and the residual (32 bits an element: as much as both); out or the bytes from t.  The weights lie in shared memory too.
// A copy takes whole 16-byte words, those that a row shares with its neighbours included, except before the first row and behind the
// last: there single elements are loaded.
constexpr int kRowsWarps = 24;
constexpr size_t kRowsSmem = 226 * 1024;

struct RowsShape {
    int warps, slots;             // per block; rows that a warp has on their way or in work
    uint32_t pitch, weights;      // bytes of one array's row in shared memory, of one array of weights
};

template <typename T, int VEC, bool QUANTIZE>
__global__ void __launch_bounds__(kRowsWarps * 32) k_norm_rows(const __grid_constant__ NormArgs a, const RowsShape shape) {
    typedef Chunk<T, VEC> C;
    constexpr bool TWOS = VEC == 1 && sizeof(T) == 2 && !QUANTIZE;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool second = QUANTIZE ? a.gated : a.residual != nullptr, third = !QUANTIZE && a.gate_rows != nullptr;
    const int arrays = third ? 3 : 2;                           // (the second's place is wanted for t)
    const uint32_t slot_bytes = arrays * shape.pitch;
    unsigned char* const mine = smem + (size_t)warp * shape.slots * slot_bytes;
    unsigned char* rest = smem + (size_t)shape.warps * shape.slots * slot_bytes;
    const uint32_t bars = smem_u32(rest) + warp * shape.slots * 8;
    rest += (shape.warps * shape.slots * 8 + 127) / 128 * 128;
    if (lane == 0) {
        for (int s = 0; s < shape.slots; s++) mbar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    wait_for_prior_kernel();
    let_next_kernel_start();
    auto source = [&](int k, long long row) -> const T* {
        if (k == 0) return (const T*)a.x + row * a.x_row;
        if (k == 2) return (const T*)a.gate_rows + row * a.gate_row;
        return QUANTIZE ? (const T*)a.x + row * a.x_row + a.dim : (const T*)a.residual + row * a.residual_row;
    };
    auto load = [&](long long row, int slot) {
        if (row >= a.rows) return;
        // a lane looks after an array
        const bool there = lane < arrays && (lane != 1 || second);
        const uintptr_t from = there ? (uintptr_t)source(lane, row) : 0, to = from + (uintptr_t)a.dim * sizeof(T);
        const uint32_t head = (uint32_t)from & 15;
        uintptr_t lo = from - head, hi = (to + 15) & ~(uintptr_t)15;
        unsigned char* const at = mine + slot * slot_bytes + lane * shape.pitch;
        if (VEC == 1 && (row == 0 || row == a.rows - 1)) {
            if (row == 0) lo = (from + 15) & ~(uintptr_t)15;
            if (row == a.rows - 1) hi = to & ~(uintptr_t)15;
            if (there) {                                        // (dim >= 64: there is something between)
                T* const here = reinterpret_cast<T*>(at + head);
                const T* const there_from = reinterpret_cast<const T*>(from);
                for (int i = 0; (uintptr_t)(there_from + i) < lo; i++) here[i] = there_from[i];
                for (int i = a.dim - 1; (uintptr_t)(there_from + i) >= hi; i--) here[i] = there_from[i];
            }
        }
        const uint32_t bytes = there ? (uint32_t)(hi - lo) : 0, total = __reduce_add_sync(0xffffffffu, bytes);
        fence_async_smem();                                     // (the slot's last reads and writes were this warp's own)
        __syncwarp();
        if (lane == 0) mbar_expect_tx(bars + 8 * slot, total);
        __syncwarp();
        if (there) bulk_g2s(smem_u32(at) + (uint32_t)(lo - (from - head)), (const void*)lo, bytes, bars + 8 * slot);
    };
    const long long step = (long long)gridDim.x * shape.warps, first = (long long)blockIdx.x * shape.warps + warp;
    for (int s = 0; s < shape.slots; s++) load(first + s * step, s);
    // Weights: the first and the last four of every eight channels apart, so that a warp's reads of 16 bytes a lane meet no bank twice.
    const float *post = nullptr, *channel = nullptr, *pre = nullptr;
    if constexpr (!QUANTIZE) {
        auto keep = [&](const float* w) -> const float* {
            if (w == nullptr) return nullptr;
            float* const to = reinterpret_cast<float*>(rest);
            rest += shape.weights;
            for (int i = threadIdx.x; i < a.dim; i += blockDim.x) to[VEC == 8 ? (i / 8) * 4 + (i % 4) + (i % 8 / 4) * (a.dim / 2) : i] = __ldg(w + i);
            return to;
        };
        post = keep(a.post_norm);
        channel = keep(a.gate);
        pre = keep(a.pre_norm);
        __syncthreads();
    }
    bool timed_out = false;
    const float per = 1.0f / (float)a.dim;
    int slot = 0, use = 0;
    for (long long row = first; row < a.rows; row += step) {
        if (!mbar_wait_near(bars + 8 * slot, use, timed_out)) break;
        unsigned char* const at = mine + slot * slot_bytes;
        auto row_of = [&](int k) { return reinterpret_cast<T*>(at + k * shape.pitch + (VEC == 1 ? (uint32_t)((uintptr_t)source(k == 1 && !second ? 0 : k, row) & 15) : 0)); };
        T *const xs = row_of(0), *const rs = row_of(1), *const gs = third ? row_of(2) : nullptr;
        float f = 1.0f, s0, s1, m = 0.0f;
        uint64_t squares = 0;
        T *const sums = (T*)a.sum + row * a.sum_row, *const outs = (T*)a.out + row * a.out_row;
        // 16-bit rows of any width go two elements at a time where all arrays' rows begin in the same half of a 32-bit word (15630 rows of
        // 1157 fp16, gates of their own: 48.8 us, one at a time 53.5)
        bool twos = false;
        if constexpr (TWOS) {
            const uintptr_t x = (uintptr_t)source(0, row);
            twos = (((second ? x ^ (uintptr_t)source(1, row) : 0) | (third ? x ^ (uintptr_t)source(2, row) : 0) | (a.sum != nullptr ? x ^ (uintptr_t)sums : 0) |
                     (a.out != nullptr ? x ^ (uintptr_t)outs : 0)) & 2) == 0;
        }
        const int begin = TWOS && twos ? (int)((uintptr_t)source(0, row) >> 1 & 1) : 0;
        auto all = [&](auto&& of) {
            if constexpr (TWOS) {
                if (twos) {
                    const int end = begin + (a.dim - begin) / 2 * 2;
                    if (lane == 0 && begin > 0) of(C(), 0);
                    if (lane == 31 && end < a.dim) of(C(), end);
#pragma unroll 4
                    for (int i = begin + lane * 2; i < end; i += 64) of(Two<T>(), i);
                    return;
                }
            }
#pragma unroll 4
            for (int i = lane * VEC; i < a.dim; i += 32 * VEC) of(C(), i);
        };
        if (!QUANTIZE && post != nullptr) {
            all([&](auto r, int i) {
                r.split(*reinterpret_cast<const typename decltype(r)::Raw*>(xs + i));
                r.square(squares);
            });
            apart(squares, s0, s1);
            s0 += s1;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
            f = rsqrtf(s0 * per + a.eps);
            squares = 0;
        }
        all([&](auto r, int i) {
            typedef typename decltype(r)::Raw Raw;
            decltype(r) w;
            r.split(*reinterpret_cast<const Raw*>(xs + i));
            if constexpr (QUANTIZE) {
                if (second) {
                    w.split(*reinterpret_cast<const Raw*>(rs + i));
                    r.gated(w);
                }
            } else {
                if (post != nullptr) {
                    r.scale(f);
                    w.kept(post, i, a.dim);
                    r.times(w);
                }
                if (channel != nullptr) {
                    w.kept(channel, i, a.dim);
                    r.times(w);
                }
                if (third) {
                    w.split(*reinterpret_cast<const Raw*>(gs + i));
                    r.times(w);
                }
                if (second) {
                    w.split(*reinterpret_cast<const Raw*>(rs + i));
                    r.add(a.residual_scale, w);
                }
                r.square(squares);
                if (a.sum != nullptr) r.store(sums + i);
                if (pre != nullptr) {
                    w.kept(pre, i, a.dim);
                    r.times(w);
                }
            }
            if (a.q != nullptr) r.largest(m);
            r.park(xs + i, rs + i);
        });
        if (a.out != nullptr || a.q != nullptr) {
            apart(squares, s0, s1);
            s0 += s1;
            f = 1.0f;
            if (!QUANTIZE && pre != nullptr) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
                f = rsqrtf(s0 * per + a.eps);
            }
            float factor = 0.0f, quantum = 0.0f;
            if (a.q != nullptr) {
                quant_step(__reduce_max_sync(0xffffffffu, __float_as_uint(m)), factor, quantum);
                if (lane == 0) a.q_scale[row] = quantum * f;
            }
            int8_t* const bytes = a.q + row * a.q_row;
            all([&](auto r, int i) {
                r.unpark(xs + i, rs + i);
                if (a.q != nullptr) r.bytes(bytes + i, factor);
                if (!QUANTIZE && a.out != nullptr) {
                    r.scale(f);
                    r.store(outs + i);
                }
            });
        }
        __syncwarp();
        load(row + shape.slots * step, slot);
        if (++slot == shape.slots) {
            slot = 0;
            use++;
        }
    }
    if (timed_out) {                                            // (the block must not end with copies in flight)
        for (int s = 0; s < shape.slots; s++) {
            bool late = false;
            mbar_wait_sleep(bars + 8 * s, s < slot ? use + 1 : use, late);
        }
        raise_status(a.status, kStatusWaitTimeout);
    }
}

}  // namespace sttm
