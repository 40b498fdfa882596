// PTX of kernels in which a pair of thread blocks may share a tile (CG = 2), and reads of their accumulators.  Everything is in an
// anonymous namespace.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
#include "tc_ptx.cuh"

namespace {

template <int CG> __device__ __forceinline__ uint32_t pair_rank() {
    uint32_t r = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
template <int CG> __device__ __forceinline__ void pair_sync() {       // every thread of both blocks
    if constexpr (CG == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
// Address of the leading block's copy of a barrier (the two blocks lay out their shared memory alike).
template <int CG> __device__ __forceinline__ uint32_t leader_addr(const void *p) {
    uint32_t a = smem_u32(p);
    if constexpr (CG == 2) asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
    return a;
}
// (Without a cluster-scope release, which waits some 1400 cycles for unrelated stores: what the arrival hands over is ordered
// by tcgen05 fences for tensor memory and by the proxy fence for shared memory.)
template <int CG> __device__ __forceinline__ void arrive_leader(uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(leader_addr<2>(bar)) : "memory");
}
// 2-D box into this block's shared memory, its bytes counted on the leading block's barrier.
template <int CG>
__device__ __forceinline__ void pair_load_2d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y) {
    if constexpr (CG == 1)
        tma_load_2d(dst, map, bar, x, y);
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
            ::"r"(smem_u32(dst)), "l"(map), "r"(leader_addr<2>(bar)), "r"(x), "r"(y) : "memory");
}
template <int CG> __device__ __forceinline__ void pair_tmem_alloc(uint32_t *slot, uint32_t ncols) {   // one whole warp per block
    if constexpr (CG == 1) {
        tmem_alloc(slot, ncols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG> __device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    if constexpr (CG == 1) tmem_dealloc(taddr, ncols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// Arrives on the barrier (of both blocks) when the instructions issued so far have completed.
template <int CG> __device__ __forceinline__ void pair_commit(uint64_t *bar) {
    if constexpr (CG == 1)
        tc_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_load_lane_16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// 16 lanes x 32 columns: register 4i + {0, 1} of lane l holds row l/4, columns 8i + 2(l%4) + {0, 1}; + {2, 3} row l/4 + 8.
__device__ __forceinline__ void tmem_load_16x32(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
template <class T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
}

}  // namespace
