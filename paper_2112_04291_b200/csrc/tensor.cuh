// Matrix instructions of the fifth-generation tensor cores (tcgen05) with their accumulators in tensor memory, and tiled copies that
// feed them.  sm_100a only.
#pragma once

#include <cuda.h>

#include "async.cuh"

namespace fsg {

// One thread of the warp, the same each time.  Copies and matrix instructions take their operands from registers that a warp has in
// common: where the compiler knows that a single thread issues them, one costs a few cycles, after a comparison of lanes some 150.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0u;
}

// ---- tiled copies -----------------------------------------------------------------------------
// To this block's shared memory; the barrier (an address of the cluster's shared memory) may be this block's or the other's of the pair.
__device__ __forceinline__ void tile_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tile_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// One arrival on a barrier of the pair's, at an address of the cluster's shared memory, and the bytes that copies will bring: the thread itself
// has written nothing that whoever waits would read, and the copies' own completion orders what they write.
__device__ __forceinline__ void mbar_expect_tx_at(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// A box of shared memory to a map's place; what of it lies outside the map is not written.  Boxes of a thread complete in groups.
__device__ __forceinline__ void tile_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void stores_end_group() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void wait_stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// what this thread has written to shared memory is seen by copies and matrix instructions that are issued later
__device__ __forceinline__ void fence_async_reads() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One more arrival on a barrier of another block of the pair, about accumulators alone: what was read of them is ordered by the fences of tensor
// memory on both sides (tmem_before_barrier here, tmem_after_barrier behind the wait, which is one of the cluster's scope), not by the arrival,
// which would otherwise wait for this thread's stores to global memory.
__device__ __forceinline__ void mbar_tell(unsigned long long* bar, uint32_t block) {
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, %1;\n mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [r];\n}" ::"r"(smem_u32(bar)), "r"(block) : "memory");
}

// ---- tensor memory, of a pair of blocks ---------------------------------------------------------
// (one warp of each block; columns: a power of two from 32 on)
__device__ __forceinline__ void tmem_alloc(uint32_t* address, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(address)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t address, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
// columns of this warp's 32 lanes: r[i] is column `at` + i of the thread's own lane, once the wait for it is over
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_before_barrier() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_barrier() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- products -----------------------------------------------------------------------------------
// Operands lie in shared memory in rows of 128 bytes, swizzled in 1024 bytes (eight such rows), as tiled copies leave them.
//   contraction along the row (64 values of it): eight rows of the matrix follow one another every 1024 bytes; 16 values of the
//     contraction further are 32 bytes further in the row.
//   matrix rows along the row (64 of them; the contraction from row to row): eight values of the contraction every 1024 bytes, the
//     next 64 matrix rows `strip` bytes on; 16 values of the contraction further are 2048 bytes further.
// The words of an operand's description: the first holds its place, 16 bytes a unit, and `strip`; the second is the same for all.
__device__ __forceinline__ uint32_t operand_at(uint32_t address, uint32_t strip) { return (address & 0x3FFFFu) >> 4 | strip >> 4 << 16; }
constexpr uint32_t kOperandWord = 1024u >> 4 | 1u << 14 | 2u << 29;
// 32-bit accumulators; bf16 or fp16 operands; `along`: matrix rows lie along the row
__host__ __device__ inline uint32_t product_kind(bool bf16, bool a_along, bool b_along) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_along ? 1u : 0u) << 15 | (b_along ? 1u : 0u) << 16;
}
__device__ __forceinline__ uint32_t product_shape(uint32_t kind, uint32_t m, uint32_t n) { return kind | (n >> 3) << 17 | (m >> 4) << 24; }
// acc (+)= A B^T over 16 values of the contraction, by the tensor cores of a pair of blocks: each has half of A's rows (and of the accumulator's)
// and half of B's, at the same places of its shared memory.  One thread of the pair's first block.
__device__ __forceinline__ void multiply(uint32_t acc, uint32_t a, uint32_t b, uint32_t shape, bool add) {
    asm volatile("{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n}"
                 ::"r"(acc), "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add), "r"(kOperandWord) : "memory");
}
// arrives on the barrier, in both blocks of the pair (`pair`: their bits among the cluster's), once the products that this thread has issued are done
__device__ __forceinline__ void products_arrive(unsigned long long* bar, uint32_t pair) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)pair) : "memory");
}

}  // namespace fsg
