// Host helpers of the calls on the paged key-value cache and of a decoder layer: launches, attributes, argument checks.
#pragma once

#include <climits>
#include <type_traits>
#include <utility>

#include "sttm_cache.cuh"
#include "sttm_host.cuh"

namespace sttm {

// Launch with programmatic stream serialization (see launch_after in sttm_api.cu); `cluster` > 1: that many
// blocks to a cluster.
template <typename... KArgs, typename... Args>
sttm_status launch(void (*kernel)(KArgs...), long long grid, unsigned block, size_t smem, unsigned cluster, void* stream,
                   Args&&... args) {
    if (grid < 1 || grid > INT_MAX) return STTM_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...) == cudaSuccess ? STTM_OK : STTM_ERR_CUDA;
}

// raises a kernel's limit on dynamic shared memory once per device
inline sttm_status allow_smem(const void* kernel, size_t bytes, size_t (&allowed)[kMaxDevices]) {
    const int dev = device_slot();
    if (dev < 0) return STTM_ERR_UNSUPPORTED;
    if (allowed[dev] >= bytes) return STTM_OK;
    STTM_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    allowed[dev] = bytes;
    return STTM_OK;
}

// Slots of a row at most: the kernels count them in 32 bits and step up to sm_count() * 4096 beyond the last
// (148 multiprocessors: 606208).
constexpr int kMaxSlots = INT_MAX - (1 << 20);

inline bool multiple_of_8(long long v) { return v % 8 == 0; }
// is any of these arrays of 4-byte numbers (or NULL) at an address that is no multiple of 4?
template <typename... P>
inline bool odd_address(const P*... p) { return (((uintptr_t)p | ...) & 3) != 0; }

struct Span {
    const void* at;               // or NULL: nothing
    long long bytes;
};
inline bool overlap(const Span& a, const Span& b) {
    return a.at != nullptr && b.at != nullptr && (uintptr_t)a.at < (uintptr_t)b.at + (uintptr_t)b.bytes && (uintptr_t)b.at < (uintptr_t)a.at + (uintptr_t)a.bytes;
}
// does `a` share memory with any of these?
template <typename... S>
bool overlaps_any(const Span& a, const S&... others) { return (overlap(a, others) || ...); }

inline sttm_status check_cache(const sttm_cache* c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->table == nullptr) return STTM_ERR_ARG;
    if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->seqs < 1 || c->table_width < 1 || c->dim < 1) return STTM_ERR_ARG;
    if (c->dtype != STTM_BF16 && c->dtype != STTM_F16) return STTM_ERR_UNSUPPORTED;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return STTM_ERR_UNSUPPORTED;
    if (c->page % 8 != 0 || c->pages > INT_MAX - 1) return STTM_ERR_UNSUPPORTED;
    if ((long long)c->table_width * c->page > INT_MAX || (long long)c->seqs * c->heads > INT_MAX / 64) return STTM_ERR_UNSUPPORTED;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || odd_address(c->table)) return STTM_ERR_ARG;
    // (the stride of an axis of length one is never used)
    if ((c->pages > 1 && !multiple_of_8(c->page_stride)) || (c->heads > 1 && !multiple_of_8(c->head_stride)) || !multiple_of_8(c->slot_stride))
        return STTM_ERR_ARG;
    if (c->slot_stride < c->dim || (c->heads > 1 && c->head_stride < c->dim) || (c->pages > 1 && c->page_stride < c->dim)) return STTM_ERR_ARG;
    if (c->seqs > 1 && c->table_stride < c->table_width) return STTM_ERR_ARG;
    return STTM_OK;
}

inline CacheView view_of(const sttm_cache* c) {
    CacheView v;
    v.k = (uint16_t*)c->k;
    v.v = (uint16_t*)c->v;
    v.pages = c->pages;
    v.page_stride = c->pages > 1 ? c->page_stride : 0;
    v.head_stride = c->heads > 1 ? c->head_stride : 0;
    v.slot_stride = c->slot_stride;
    v.table = c->table;
    v.table_stride = c->table_stride;
    v.table_width = c->table_width;
    v.heads = c->heads;
    v.page = c->page;
    v.seqs = c->seqs;
    return v;
}

// a call of `f` with the element type as a value and the channels as a constant
template <typename F>
sttm_status by_type(const sttm_cache* c, F&& f) {
    auto dims = [&](auto tag) -> sttm_status {
        if (c->dim == 64) return f(tag, std::integral_constant<int, 64>());
        if (c->dim == 128) return f(tag, std::integral_constant<int, 128>());
        return f(tag, std::integral_constant<int, 256>());
    };
    return c->dtype == STTM_BF16 ? dims(__nv_bfloat16()) : dims(__half());
}

}  // namespace sttm
