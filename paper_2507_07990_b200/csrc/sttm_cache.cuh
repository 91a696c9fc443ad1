// What the kernels on the paged key-value cache share (sm_100a): the cache as a kernel sees it and the
// two 16-bit types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sttm_device.cuh"
#include "sttm_ptx.cuh"

namespace sttm {

enum : int { kStatusArg = 1 << 1, kStatusCapacity = 1 << 4 };   // 1 << STTM_ERR_ARG, 1 << STTM_ERR_CAPACITY

struct CacheView {
    uint16_t *k, *v;              // 16-bit elements of either type
    long long pages, page_stride, head_stride, slot_stride;
    const int32_t* table;
    long long table_stride;
    int table_width, heads, page, seqs;
};

__device__ __forceinline__ void raise_status(int32_t* status, int bit) {
    if (status != nullptr) atomicOr(status, bit);
}

// first element of a slot's head 0, or -1 (and the status bit) when the slot or its page is not there
__device__ __forceinline__ long long slot_at(const CacheView& c, int seq, long long slot, int32_t* status) {
    if (slot < 0 || slot >= (long long)c.table_width * c.page) {
        raise_status(status, kStatusCapacity);
        return -1;
    }
    const int stretch = (int)slot / c.page, place = (int)slot - stretch * c.page;       // (table_width * page < 2^31)
    const int pg = c.table[seq * c.table_stride + stretch];
    if (pg < 0 || pg >= c.pages) {
        raise_status(status, kStatusArg);
        return -1;
    }
    return pg * c.page_stride + place * c.slot_stride;
}

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 split(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) { return pack_bf16x2(x, y); }
};
template <>
struct Pair<__half> {
    static __device__ __forceinline__ float2 split(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

}  // namespace sttm
