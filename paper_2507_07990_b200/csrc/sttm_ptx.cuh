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

// shared-memory operand descriptor, K-major, 128-byte swizzle: start address / 16 in bits 0-13,
// leading offset (unused for this layout) 1 in bits 16-29, 1024 bytes between groups of eight rows
// (/ 16) in bits 32-45, descriptor version 1 in bits 46-47, swizzle mode 2 in bits 61-63
__device__ __forceinline__ uint64_t tc_operand(uint32_t smem_addr) {
    return (uint64_t)((smem_addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// the mbarrier gets one arrival when every product issued so far by this thread has completed
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16 consecutive columns (see tc_load32) into the first 16 registers
__device__ __forceinline__ void tc_load16(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// 32 consecutive columns of this warp's 32 lanes: lane i receives row i
__device__ __forceinline__ void tc_load32(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// the high word of the operand descriptors with 128-byte swizzle and 1024 bytes between groups of eight rows, K-major or not
constexpr uint32_t kOperandHigh = (1024 >> 4) | (1u << 14) | (2u << 29);
// one lane of the warp
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r != 0;
}
// a value that is the same in every lane, told to the compiler
__device__ __forceinline__ uint32_t one_value(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
// Bounded wait of a warp for the `use`-th completion of an mbarrier of this CTA (see mbar_wait).  It polls; its acquire reaches no further than
// the CTA: the one over a cluster costs some 200 cycles more, several times per tile.
__device__ __forceinline__ bool mbar_wait_near(uint32_t bar, int use, bool& timed_out) {
    const uint32_t parity = (uint32_t)(use & 1);
    bool ok = !timed_out;
    if (ok && !mbar_try(bar, parity)) {
        const unsigned long long t0 = global_timer_ns();
        while (ok && !mbar_try(bar, parity)) ok = global_timer_ns() - t0 <= kWaitLimitNs;
    }
    ok = __all_sync(0xffffffffu, ok);
    timed_out = !ok;
    return ok;
}

// two numbers at a time
__device__ __forceinline__ uint64_t both(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void apart(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// the largest of three; NaN if one is
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}

}  // namespace sttm
