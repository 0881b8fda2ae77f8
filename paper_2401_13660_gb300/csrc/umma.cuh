// Thin wrappers over the sm_100 tensor-core instructions (tcgen05): matrix
// products of operands in shared memory into tensor memory, with block scales
// in tensor memory, and what moves scales and sums there and back. A tensor
// memory address holds the lane in its upper 16 bits and the 32-bit column in
// the lower ones.
#pragma once

#include "tma.cuh"

namespace mbscan {

// kCtas: 1, or 2 for a pair of CTAs (a cluster of two) that work on one product, each with half of both operands in its
// shared memory and its half of the lanes of the sum in its tensor memory. Copies and products of a pair are issued by the
// first of them. A kernel uses one of the two throughout.

// Columns are allocated by one warp (of each CTA), 32 to 512 at a time (a power of two), and freed by it.
template <int kCtas> __device__ __forceinline__ void tmem_alloc(uint32_t *address, uint32_t columns) {
    if constexpr (kCtas == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(address)), "r"(columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(address)), "r"(columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int kCtas> __device__ __forceinline__ void tmem_free(uint32_t address, uint32_t columns) {
    if constexpr (kCtas == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns));
}

// One lane of a whole warp, always the same. What it guards is known to run in one thread: under `lane == 0` the operands of
// products, which live in registers of the warp, cost several times as much.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(one));
    return one != 0;
}

// Order of this thread's tcgen05 operations against those of threads it synchronises with (before, after that).
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Arrive on `bar` (of both CTAs of a pair) once every product and copy that this thread has issued is done.
template <int kCtas> __device__ __forceinline__ void umma_commit(uint64_t *bar) {
    if constexpr (kCtas == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                         smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
}

// Descriptor of an operand in shared memory whose rows are 128 bytes of the sum's dimension, swizzled as a
// CU_TENSOR_MAP_SWIZZLE_128B copy leaves them (1024-byte aligned; groups of 8 rows 1024 bytes apart). The 32-byte column
// block k of it starts 2 k further.
__device__ __forceinline__ uint64_t umma_desc_128(uint32_t smem) {
    return (uint64_t)((smem & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// The same of 32 rows of 16 bytes, one after the other.
__device__ __forceinline__ uint64_t umma_desc_rows16(uint32_t smem) {
    return (uint64_t)((smem & 0x3ffffu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// Copy 32 rows of 16 bytes to four columns of tensor memory, row l to lane l of each of the four quarters of the lanes (in
// each CTA of a pair, from its own shared memory). In order with this thread's products.
template <int kCtas> __device__ __forceinline__ void tmem_copy_scales(uint32_t column, uint64_t desc) {
    if constexpr (kCtas == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
}

// Instruction word of a product of e4m3 operands, both with the sum's dimension innermost, m x n, with e8m0 scales. The
// scales of a row of an operand are the four bytes of a 32-bit word; `scale` of them is taken for both operands.
__device__ __forceinline__ uint32_t umma_word_q8(uint32_t m, uint32_t n, uint32_t scale) {
    return scale << 4 | (n >> 3) << 17 | 1u << 23 | (m >> 4) << 24 | scale << 29;
}

// d (+)= (A sA)(B sB)^T over 32 columns of the sum: row i of A is lane i (of a pair: 128 of 256 rows to a CTA), row j of B
// column j of d (a pair: half of the rows of B in each CTA, all columns in both). Scales of row r are in lane r % 32 (of every
// quarter) of column r / 32 (a pair: those of a CTA's own rows of A, of all rows of B). Issued by one thread.
template <int kCtas>
__device__ __forceinline__ void umma_q8(uint32_t d, uint64_t a, uint64_t b, uint32_t word, uint32_t a_scales, uint32_t b_scales,
                                        bool add) {
    if constexpr (kCtas == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(word), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(word), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
            : "memory");
}

// A 2-D tile to this CTA's shared memory, completing on a barrier of either CTA of a pair (cluster_address).
__device__ __forceinline__ void tma_load_2d_pair(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
// Arrive on a barrier of another CTA of the cluster, and wait for such arrivals: what was written before is visible after.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The same where nothing was written: what this warp has read from tensor memory is in its registers.
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t *bar, uint32_t parity) {
    const long long t0 = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > kWaitCycles) return false;
    }
}

// 16 columns of this warp's quarter of the lanes (the address's lane: 32 * (warp % 4)); wait before they are used.
__device__ __forceinline__ void tmem_load16(uint32_t address, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(address)
        : "memory");
}
// 16 lanes (the address's lane and 15 more, within this warp's quarter) by 32 columns, as fragments of 8 x 8: registers
// 4 c + 2 u and 4 c + 2 u + 1 are lane 8 u + l / 4, columns 8 c + 2 (l % 4) and the next.
__device__ __forceinline__ void tmem_load_fragments(uint32_t address, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(address)
        : "memory");
}
// Four 8 x 8 matrices of 16-bit elements to shared memory, transposed: lane l gives the address of row l % 8 (a column of the
// fragments) of matrix l / 8 and holds two elements of each, row l / 4, columns 2 (l % 4) and the next.
__device__ __forceinline__ void stsm_x4_trans(uint32_t address, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(address), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
// Names the registers it waits for, so that no use of them moves in front.
__device__ __forceinline__ void tmem_load_wait(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                   "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

}  // namespace mbscan
