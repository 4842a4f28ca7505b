// Asynchronous copies and the barriers in shared memory that they complete on; work that a running block takes over from one that has
// not begun.  sm_100a only.
#pragma once

#include "common.cuh"

namespace fsg {

// ---- mbarrier / bulk-copy primitives (sm_90+ PTX) -------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(unsigned long long* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned long long* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait: the hardware suspends the thread for up to about the hinted time per try, so a
// wait costs a handful of instructions; false when every try ran out.
constexpr uint32_t kTryHintNs = 10000u;
constexpr uint32_t kTryLimit  = 1u << 18;
__device__ __forceinline__ bool mbar_wait(unsigned long long* bar, uint32_t parity, uint32_t tries = kTryLimit) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t t = 0; t < tries; ++t) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(addr), "r"(parity), "r"(kTryHintNs) : "memory");
        if (ok) return true;
    }
    return false;
}
// One more arrival on a barrier of another block of the cluster; what this thread has written before is visible to whoever waits there.
__device__ __forceinline__ void mbar_arrive_at(unsigned long long* bar, uint32_t block) {
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, %1;\n mbarrier.arrive.release.cluster.shared::cluster.b64 _, [r];\n}" ::"r"(smem_u32(bar)), "r"(block) : "memory");
}
// The same for a barrier that another block of the cluster arrives on, whose writes before are then visible.
__device__ __forceinline__ bool mbar_wait_cluster(unsigned long long* bar, uint32_t parity, uint32_t tries = kTryLimit) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t t = 0; t < tries; ++t) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(addr), "r"(parity), "r"(kTryHintNs) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void bulk_load(void* dst_smem, const void* src_global, uint32_t bytes, unsigned long long* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst_smem)), "l"(__cvta_generic_to_global(src_global)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// ---- clusters ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_block() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
// Every thread of the cluster's blocks; what they wrote before, to shared or global memory, is visible behind it.
// (The instructions want each warp as one: its lanes come together first, wherever they have been.)
__device__ __forceinline__ void cluster_meet() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared memory of the cluster's other blocks.
__device__ __forceinline__ uint32_t address_in(const void* p, uint32_t block) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(block));
    return r;
}
__device__ __forceinline__ uint32_t address_in_cluster(uint32_t at, uint32_t block) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(block));
    return r;
}
__device__ __forceinline__ float4 load_four_from(uint32_t at) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void store_word_to(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t load_from(uint32_t at) { uint32_t v; asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory"); return v; }

// ---- dynamic rows -----------------------------------------------------------------------------
// A grid has a block (or cluster) per piece of work.  One that is running asks for the launch of another to be cancelled and, when that
// is granted, does its work: blocks that have a larger share of their SM take more, and what they set up they set up once.
struct __align__(16) Claim {
    uint4 answer;
    unsigned long long bar;
    unsigned long long pad;
};
__device__ __forceinline__ void claim_init(Claim& c) { mbar_init(&c.bar, 1u); }
// One thread; not again after an answer of -1.
__device__ __forceinline__ void claim_ask(Claim& c) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (the last answer has been read)
    mbar_expect_tx(&c.bar, 16u);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(smem_u32(&c.answer)), "r"(smem_u32(&c.bar)) : "memory");
}
// The answer to the n-th question (n counts from 0): the first block of the work that is now ours, or -1; kNoAnswer where the wait has
// run out.  What was granted then is ours all the same, and the answer still comes: a block asks for it once more before it leaves.
constexpr int kNoAnswer = -2;
__device__ __forceinline__ int claim_answer(Claim& c, uint32_t n, uint32_t tries = kTryLimit) {
    if (!mbar_wait(&c.bar, n & 1u, tries)) return kNoAnswer;
    uint32_t granted, x;
    asm volatile("{\n .reg .pred p;\n .reg .b128 r;\n ld.shared.b128 r, [%2];\n clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
                 " selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
                 : "=r"(granted), "=r"(x) : "r"(smem_u32(&c.answer)) : "memory");
    return granted ? (int)x : -1;
}

}  // namespace fsg
