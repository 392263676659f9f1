// Tensor-core products with accumulators in TMEM (tcgen05.mma), fed by tensor
// copies (cp.async.bulk.tensor): the instructions, as the product kernels use
// them, for one CTA or a pair of CTAs that share a tile.
#pragma once

#include <cuda.h>

#include <cstdint>

#include "aloco_bulk.cuh"

namespace aloco {

// Shared-memory matrix descriptor of fp16 operands in 128-byte swizzled tiles
// whose 8-row groups lie 1024 bytes apart: 16-byte units, bits 0-13 the start
// address, 16-29 the leading and 32-45 the stride offset, 46 the version, 61-63
// the swizzle (2: 128 bytes).
//   K-major (rows of 64 k-elements): the stride offset is from 8 rows to the next.
//   MN-major (rows of 64 m- or n-elements): the stride offset is from 8 k to the
//   next, the leading one from 64 rows or columns to the next.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t leading_bytes) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(leading_bytes >> 4) << 16 |
           (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// Instruction descriptor: fp16 operands, fp32 accumulators, an M x N tile of
// K-major operands; what makes one of them MN-major.
constexpr uint32_t product_desc(int m, int n) {
    return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
constexpr uint32_t kAMnMajor = 1u << 15, kBMnMajor = 1u << 16;

template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {
    if constexpr (kCtas == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                     "r"(columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
                     "r"(columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int kCtas>
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
    if constexpr (kCtas == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "r"(columns));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "r"(columns));
}

// d (+)= a b on the tile: one thread of the (leading) CTA.
template <int kCtas>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t desc,
                                        bool add) {
    if constexpr (kCtas == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
            : "memory");
}

// One arrival on `bar` (of both CTAs of a pair) when the products issued so far
// are done.
template <int kCtas>
__device__ __forceinline__ void product_commit(uint32_t bar) {
    if constexpr (kCtas == 1)
        asm volatile(
            "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
            : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster"
            ".b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
}

__device__ __forceinline__ void tc_fence_before() {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// 32 accumulator columns of this warp's 32 lanes (25 cycles beside running products).
__device__ __forceinline__ void tmem_read32(uint32_t tmem, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
          "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
          "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
          "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]),
          "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(tmem)
        : "memory");
}

// A box of a 3-d tensor to shared memory of this CTA, its bytes counted on `bar`
// (of a pair: an address in the cluster's shared memory, of either CTA).
template <int kCtas>
__device__ __forceinline__ void tensor_load(uint32_t dst, const CUtensorMap *map, int x, int y,
                                            int z, uint32_t bar) {
    if constexpr (kCtas == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global"
            ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

// The address, in the cluster's shared memory, of what lies at `addr` in CTA `rank`.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// (relaxed: what it orders are reads of TMEM, by tc_fence_before(); a release
// would wait for this thread's stores to global memory)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
}
// A tensor map, which is a kernel's parameter, ahead of its first use.
__device__ __forceinline__ void fetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void fetch_l2(const void *p) {
    asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                     : "memory");
}
// What this grid writes before it ends is seen by one that was launched behind
// it and has passed grid_wait().
__device__ __forceinline__ void grid_wait() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void grid_go() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

}  // namespace aloco
