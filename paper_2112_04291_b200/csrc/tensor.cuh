// Matrix instructions of the fifth-generation tensor cores (tcgen05) with their accumulators in tensor memory, and tiled copies that
// feed them.  sm_100a only.
#pragma once

#include <cuda.h>

#include "async.cuh"

namespace fsg {

// ---- tiled copies -----------------------------------------------------------------------------
__device__ __forceinline__ void tile_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tile_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// four rows of a map whose box is one row high
__device__ __forceinline__ void rows_load(uint32_t dst, const CUtensorMap* map, int x, int4 rows, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w), "r"(bar) : "memory");
}
// what this thread has written to shared memory is seen by copies and matrix instructions that are issued later
__device__ __forceinline__ void fence_async_reads() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory ------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t* address, uint32_t columns) {      // one warp; columns: a power of two from 32 on
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(address)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t address, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
// 32 columns of this warp's 32 lanes: r[i] is column `at` + i of the thread's own lane
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_before_barrier() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_barrier() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- products -----------------------------------------------------------------------------------
// Operands lie in shared memory in rows of 128 bytes, swizzled in 1024 bytes (eight such rows), as tiled copies leave them.
//   contraction along the row (64 values of it): eight rows of the matrix follow one another every 1024 bytes; 16 values of the
//     contraction further are 32 bytes further in the row.
//   matrix rows along the row (64 of them; the contraction from row to row): eight values of the contraction every 1024 bytes, the
//     next 64 matrix rows `strip` bytes on; 16 values of the contraction further are 2048 bytes further.
__device__ __forceinline__ uint64_t operand_at(uint32_t address, uint32_t strip) {
    return (uint64_t)((address & 0x3FFFFu) >> 4) | (uint64_t)((strip & 0x3FFFFu) >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 32-bit accumulators; bf16 or fp16 operands; `along`: matrix rows lie along the row
__host__ __device__ inline uint32_t product_kind(bool bf16, bool a_along, bool b_along) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_along ? 1u : 0u) << 15 | (b_along ? 1u : 0u) << 16;
}
__device__ __forceinline__ uint32_t product_shape(uint32_t kind, uint32_t m, uint32_t n) { return kind | (n >> 3) << 17 | (m >> 4) << 24; }
// acc (+)= A B^T over 16 values of the contraction; one thread
__device__ __forceinline__ void multiply(uint32_t acc, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(acc), "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
// arrives on the barrier once the products that this thread has issued are done
__device__ __forceinline__ void products_arrive(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace fsg
