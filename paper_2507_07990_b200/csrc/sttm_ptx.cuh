// PTX wrappers shared by the kernels (sm_100a): mbarriers and bounded waits, bulk copies, clusters,
// matrix fragments.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace sttm {

constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // a wait gives up after two seconds

enum : int { kStatusWaitTimeout = 1 << 7 };         // 1 << STTM_ERR_TIMEOUT

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// arrive on an mbarrier of another CTA of the cluster (address from map_to_rank)
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// has the phase with this parity completed?  (no waiting: the callers spin on it, which hands a
// frame from warp to warp faster than a suspending wait does; measured 1.5 % of the kernel's time)
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long global_timer_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Bounded wait for the `use`-th completion (0-based) of an mbarrier: false when it has not
// come within kWaitLimitNs (or an earlier wait of this thread ran out).  The caller then
// leaves its loops without touching the data it waited for; the warps that depend on it
// run out in turn, every CTA still reaches the end of the kernel, and the host sees
// kStatusWaitTimeout in the status word.
__device__ __forceinline__ bool mbar_wait_lane(uint32_t bar, int use, bool& timed_out) {
    if (timed_out) return false;
    const uint32_t parity = (uint32_t)(use & 1);
    if (mbar_test(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    int tries = 0;
    while (!mbar_test(bar, parity)) {
        if ((++tries & 63) == 0 && global_timer_ns() - t0 > kWaitLimitNs) {
            timed_out = true;
            return false;
        }
    }
    return true;
}
// The same for a whole warp (every caller is one): the lanes agree on the outcome, so that a warp
// never splits at the time limit with some lanes leaving and the others entering a warp-wide
// primitive.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, int use, bool& timed_out) {
    const bool ok = mbar_wait_lane(bar, use, timed_out);
    const bool all = __all_sync(0xffffffffu, ok);
    if (!all) timed_out = true;
    return all;
}
// waits until a progress counter in shared memory (written by another warp of the CTA; only
// a timing hint, no data hangs on it) has reached `target`; time-bounded like mbar_wait
__device__ __forceinline__ bool hint_wait(const int* counter, int target, bool& timed_out) {
    bool ok = !timed_out;
    const volatile int* c = counter;
    if (ok && *c < target) {
        const unsigned long long t0 = global_timer_ns();
        while (*c < target) {
            __nanosleep(64);
            if (global_timer_ns() - t0 > kWaitLimitNs) { ok = false; break; }
        }
    }
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) timed_out = true;
    return ok;
}
// this CTA's shared memory -> shared memory of a CTA of the cluster, completion counted in
// bytes on that CTA's mbarrier (both given as cluster addresses)
__device__ __forceinline__ void bulk_s2s(uint32_t dst_cluster, uint32_t src, uint32_t bytes, uint32_t bar_cluster) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst_cluster), "r"(src), "r"(bytes), "r"(bar_cluster)
                 : "memory");
}
// orders this thread's earlier writes to shared memory before later reads of the async proxy
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// asks for a piece of global memory to be brought into L2 (no completion, nothing to wait for)
__device__ __forceinline__ void bulk_prefetch_l2(const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
// global -> this CTA's shared memory, completion counted in bytes on an mbarrier
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_id() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_count() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%nclusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t out;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(addr), "r"(rank));
    return out;
}
__device__ __forceinline__ void named_sync(int id, int count) {
    asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(count) : "memory");
}
// named barrier that also returns the OR of a flag over its `count` threads
__device__ __forceinline__ bool named_sync_or(int id, int count, bool flag) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.red.or.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)flag), "r"(id), "r"(count)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
// D (16x8, fp32) += A (16x16 bf16, row) * B (16x8 bf16, col)
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float lds_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ float4 lds_f32x4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint4 lds_u32x4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint2 lds_u64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}

__device__ __forceinline__ uint32_t pack_bf16x2(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// has the phase with this parity completed?  Suspends the thread for a while (the hardware's own
// limit) instead of returning at once: a waiting warp of these kernels must not take issue slots
// from the warps that have work.
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// bounded wait (see mbar_wait) on the suspending form
__device__ __forceinline__ bool mbar_wait_sleep(uint32_t bar, int use, bool& timed_out) {
    if (timed_out) return false;
    const uint32_t parity = (uint32_t)(use & 1);
    if (mbar_try(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    while (!mbar_try(bar, parity)) {
        if (global_timer_ns() - t0 > kWaitLimitNs) {
            timed_out = true;
            return false;
        }
    }
    return true;
}
// bounded wait whose outcome is the same in every lane of the warp
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, int use, bool& timed_out) {
    const bool ok = mbar_wait_sleep(bar, use, timed_out);
    const bool all = __all_sync(0xffffffffu, ok);
    if (!all) timed_out = true;
    return all;
}

}  // namespace sttm
