// Host helpers shared by the library's source files.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sttm.h"

namespace sttm {

#define STTM_CUDA_TRY(expr)                          \
    do {                                             \
        cudaError_t e_ = (expr);                     \
        if (e_ != cudaSuccess) return STTM_ERR_CUDA; \
    } while (0)

constexpr int kSmCount = 148;   // B200 (grid sizes of the older kernels; the streaming kernels ask the device)

// multiprocessors of the current device
inline int sm_count() {
    static int cached[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return kSmCount;
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = kSmCount;
        cached[dev] = n;
    }
    return cached[dev];
}

inline size_t align_up(size_t v, size_t a = 256) { return (v + a - 1) / a * a; }

// index of the current device for the per-device tables below (function attributes and occupancy
// answers belong to a device); -1 when it cannot be had or is beyond the tables
constexpr int kMaxDevices = 64;
inline int device_slot() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return -1;
    return dev;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's tensor-map encoder, through the runtime (no link against libcuda); null when it is not there
inline EncodeTiledFn tensor_map_encoder() {
    static EncodeTiledFn encode = nullptr;
    if (encode == nullptr) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            encode = (EncodeTiledFn)fn;
    }
    return encode;
}

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }
inline unsigned blocks_for(long long items, int per_block) { return (unsigned)((items + per_block - 1) / per_block); }

}  // namespace sttm
