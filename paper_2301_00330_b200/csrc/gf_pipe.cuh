// Asynchronous-copy and mbarrier primitives (inline PTX for sm_100a).
// Every wait is bounded: after kWaitCycles it gives up and reports failure, so a
// kernel can set its error word and leave instead of spinning forever.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace gf {

constexpr long long kWaitCycles = 2000000000LL;   // about one second of SM clocks

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}

// Makes freshly initialised barriers visible to the asynchronous proxy.
__device__ __forceinline__ void mbar_fence_init() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

// true once the phase with the given parity has completed; false after `limit` clocks.
__device__ __forceinline__ bool mbar_wait_bounded(uint64_t* bar, uint32_t parity, long long limit = kWaitCycles) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity)) {
        if (clock64() - t0 > limit) return false;
    }
    return true;
}

// The same for a whole converged warp, whose lanes give up together: what follows a wait is often an instruction of
// the whole warp, at which lanes that went on would wait for those that did not.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, long long limit = kWaitCycles) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, limit));
}

// After a wait that ran out: copies or products that were started may still be under way in this block's shared and
// tensor memory.  About a millisecond, after which the block may end.
__device__ __forceinline__ void let_settle() {
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) {}
}

// One contiguous global -> shared copy by the copy engine; both addresses 16-byte
// aligned, bytes a multiple of 16.  Completion is signalled on `bar` as tx bytes.
__device__ __forceinline__ void bulk_g2s(void* dst_smem, const void* src_gmem, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_u32(dst_smem)),
                 "l"(src_gmem), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// One contiguous shared -> global copy by the copy engine (same alignment rules), as part
// of the issuing thread's current bulk group.  bulk_commit() closes the group;
// bulk_wait_read<N>() returns once all but the N most recent groups of this thread have
// finished READING shared memory (the source may be reused); bulk_wait_all() once every
// group has completed.
__device__ __forceinline__ void bulk_s2g(void* dst_gmem, const void* src_smem, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst_gmem), "r"(smem_u32(src_smem)),
                 "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Orders generic-proxy writes to shared memory before later asynchronous-proxy
// accesses (copy engine, tensor core) to the same locations.
__device__ __forceinline__ void fence_proxy_async_smem() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// What a role of a kernel that works in turns, between which all blocks meet, goes on with: `ok` false says that one of
// its waits has run out.  After the last turn nobody meets, and a failure of that turn is still to be reported.
#pragma nv_exec_check_disable
template <typename Meet> __host__ __device__ __forceinline__ bool end_of_turn(int turn, int turns, bool ok, Meet&& meet) {
    return turn + 1 == turns ? ok : meet(ok);
}

// Named barrier `id` over `nthreads` threads that also tells every one of them whether ANY
// of them passed a true predicate: a failed (timed-out) wait of one thread ends the loop of all,
// so that no thread is left alone at a later barrier.
__device__ __forceinline__ bool bar_any(int id, int nthreads, bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %1, 0;\n\t"
        "bar.red.or.pred p, %2, %3, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)pred), "r"(id), "r"(nthreads)
        : "memory");
    return r != 0;
}

}  // namespace gf
