// PTX helpers of the 4-bit products: fifth-generation tensor core instructions (operands in shared memory, accumulators and block
// scales in tensor memory), tile copies that signal the leading CTA of a pair, and cluster barriers.  CG is the number of
// CTAs that work on one instruction (cta_group).
#pragma once
#include "mor_ptx.cuh"

namespace mor {
namespace {

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's shared window, that `addr` of this CTA has in CTA `rank`.
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ float lds_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// Warp number and choice of a thread in forms that the compiler knows to be the same for the whole warp: tensor-core and copy
// instructions take their operands from uniform registers, and moving each one there from per-thread registers costs more than the
// instruction.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0); }
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(p));
    return p != 0;
}

// Tile copies; `bar` is a shared-window address, with CG = 2 that of the pair's leading CTA.
template <int CG> __device__ __forceinline__ void load_tile_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <int CG> __device__ __forceinline__ void load_tile_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Tensor memory: whole warps of every CTA of the group allocate and free.
template <int CG> __device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t columns)
{
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int CG> __device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns)
{
    if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Arrives on `bar` (of this CTA; with CG = 2 of both CTAs, at the same offset) when everything issued so far has finished.
template <int CG> __device__ __forceinline__ void tc_commit(uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// One scale tile (32 rows of 16 bytes in shared memory) to four columns of tensor memory, repeated for the four groups of 32 lanes;
// with CG = 2 in both CTAs, each from its own shared memory.
template <int CG> __device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    if constexpr (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// Accumulators += (A x block scales) (B x block scales)^T over 64 elements of the reduction axis.
template <int CG, bool E4M3_16>
__device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, bool accumulate)
{
    const uint32_t acc = accumulate;
#define MOR_MMA(CGS, KIND, VEC)                                                                                                   \
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0;\n"                                                                          \
                 "tcgen05.mma.cta_group::" CGS ".kind::" KIND ".block_scale.scale_vec::" VEC " [%0], %1, %2, %3, [%5], [%6], p; }" \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(sfa), "r"(sfb) : "memory")
    if constexpr (CG == 2) {
        if constexpr (E4M3_16) MOR_MMA("2", "mxf4nvf4", "4X");
        else MOR_MMA("2", "mxf4", "2X");
    } else {
        if constexpr (E4M3_16) MOR_MMA("1", "mxf4nvf4", "4X");
        else MOR_MMA("1", "mxf4", "2X");
    }
#undef MOR_MMA
}

// 32 columns of the accumulators, one lane per thread.
__device__ __forceinline__ void tmem_load32(uint32_t* r, uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_load16(uint32_t* r, uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}

// Shared-memory descriptors.  Codes: rows of 128 bytes, 128-byte swizzle, 1024 bytes between groups of eight rows; a step
// of 64 elements along the row adds 32 bytes to the start.  Scales: no swizzle, 128 bytes between groups of eight rows.
__device__ __forceinline__ uint64_t codes_desc(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
// Instruction descriptor of a block-scaled 4-bit product of M x N (M over the whole group): both operands E2M1 and K-major; scale
// type E4M3 or E8M0; `sf` the first of the column's four scale bytes to use.
__host__ __device__ constexpr uint32_t fp4_idesc(int m, int n, bool e4m3_16, int sf)
{
    return ((uint32_t)sf << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (e4m3_16 ? 0u : 1u << 23) | ((uint32_t)(m >> 7) << 27) | ((uint32_t)sf << 29);
}

}  // namespace
}  // namespace mor
