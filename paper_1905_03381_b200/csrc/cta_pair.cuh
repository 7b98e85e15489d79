// Clusters of CTAs: rank, barrier, another CTA's shared memory; and the matrix unit's instructions for one CTA or a pair of CTAs (CG), whose first one issues.
#pragma once

#include "tensor_core.cuh"

namespace aa {

#ifdef __CUDACC__

// One lane of a converged warp.  The matrix unit's instructions take their operands from uniform registers; in a branch on the lane number each of them would be
// moved there first (a slice of four products: 740 cycles instead of 530).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same place in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t of_rank(const void* shared, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(shared)), "r"(rank));
    return a;
}
__device__ __forceinline__ void store_remote(uint32_t at, float4 x) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w) : "memory");
}

// Orders the reads of TMEM and shared memory by tcgen05 only, which the barriers of a pair do at their default scope.
__device__ __forceinline__ void mbar_arrive_at(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Orders ordinary writes before it too, over the pair (dear: not for every slice).
__device__ __forceinline__ void mbar_release_at(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
// A box into this CTA's shared memory whose bytes count on a barrier of either CTA.
template <int CG>
__device__ __forceinline__ void load_box(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar, uint32_t first_bar) {
    if (CG == 1) tma_load_2d(dst, map, x, y, bar);
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)), "l"(map),
                     "r"(first_bar), "r"(x), "r"(y)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (CG == 1) umma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if (CG == 1) umma_bf16(d, a, b, idesc, accumulate);
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                     "r"((uint32_t)accumulate)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void alloc(uint32_t* dst, uint32_t cols) {
    if (CG == 1) {
        tmem_alloc(dst, cols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void dealloc(uint32_t addr, uint32_t cols) {
    if (CG == 1) tmem_dealloc(addr, cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// The same from a stack of planes (three dimensions).
__device__ __forceinline__ void load_plane_box_pair(void* dst, const CUtensorMap* map, int x, int y, int plane, uint32_t first_bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)), "l"(map),
                 "r"(first_bar), "r"(x), "r"(y), "r"(plane)
                 : "memory");
}

#endif  // __CUDACC__

}  // namespace aa
