// What the expert products need of the fifth-generation tensor cores: tensor maps, TMA loads, mbarriers with bounded
// waits, tcgen05 products with their accumulators in tensor memory, and the descriptors they take.
//
// Operand tiles lie in shared memory as the 128-byte swizzle leaves them. A K-major tile holds one 128-byte line (64 bf16
// of the contracted axis) per row; eight rows are one 1024-byte pattern. An MN-major tile holds one 128-byte line (64 bf16
// of the outer axis) per step of the contracted axis; eight steps are one pattern and the next 64 of the outer axis lie a
// whole 64-step chunk (8 KB) further on.
#pragma once

#include <cuda.h>

#include "ep_common.cuh"

namespace ep {

// The driver's tensor-map encoder, looked up once (the library does not link against libcuda).
using TensorMapEncode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                     const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                     CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int tensor_map_encoder(TensorMapEncode *fn);

// A bf16 array [outer2][outer1][inner] (row-major), read in boxes of 64 x box_rows x 1; reads past an axis's end give 0.
inline int make_map(TensorMapEncode encode, CUtensorMap *map, const void *base, uint64_t inner, uint64_t outer1, uint64_t outer2,
                    uint32_t box_rows)
{
    const cuuint64_t dim[3] = {inner, outer1, outer2};
    const cuuint64_t stride[2] = {inner * 2, inner * outer1 * 2};
    const cuuint32_t box[3] = {64, box_rows, 1}, step[3] = {1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dim, stride, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        note_cuda_error(cudaErrorInvalidValue);
        return EP_ERR_CUDA;
    }
    return EP_OK;
}

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// --- mbarriers --------------------------------------------------------------------------------------------------

constexpr long long kWaitCycles = 4000000000ll;   // about two seconds: a wait that runs out is an error, not a slow copy

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// CLUSTER: what another CTA of the cluster released with its arrival is seen afterwards.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    if (CLUSTER)
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(bar), "r"(parity)
                     : "memory");
    return ok != 0;
}

// Waits for the phase of the given parity to end. False if it did not within the limit, or if another warp of the block
// gave up before (*gave_up, shared memory): the caller then leaves its loop.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    if (bar_try<CLUSTER>(bar, parity)) return true;
    const long long start = clock64();
    for (;;) {
        if (bar_try<CLUSTER>(bar, parity)) return true;
        if (*gave_up) return false;
        if (clock64() - start > kWaitCycles) {
            *gave_up = 1;
            return false;
        }
    }
}

// The same by a whole warp, with one answer for all its lanes: a lane that sees the phase end while another gives up must not go on alone,
// since what follows are instructions of the whole warp.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    return __all_sync(kFullMask, bar_wait<CLUSTER>(bar, parity, gave_up));
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// The address of the same shared-memory word in the given CTA of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// Arrives on a barrier of any CTA of the cluster. Relaxed: what it hands over is tensor memory, ordered by tmem_fence_before();
// a release at cluster scope would wait for the acknowledgement of every global store in front of it.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// The same with release semantics: what this thread (and, after a __syncwarp, its warp) read and wrote before is done for who waits.
__device__ __forceinline__ void bar_arrive_cluster_release(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ float4 load_cluster(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// --- TMA --------------------------------------------------------------------------------------------------------

// One box at (x, y, z); its bytes are counted on `bar` (CG == 2: a barrier of either CTA of the pair).
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                         dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

// --- tcgen05 ----------------------------------------------------------------------------------------------------

constexpr uint64_t kDescCommon = (uint64_t(1) << 46) | (uint64_t(2) << 61);   // descriptor version, 128-byte swizzle

// K-major: 1024 bytes from one group of eight rows to the next. 16 steps of the contracted axis are 32 bytes.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr)
{
    return kDescCommon | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 16) | ((addr >> 4) & 0x3fff);
}
// MN-major: 8 KB from 64 of the outer axis to the next 64, 1024 bytes from eight contracted steps to the next eight.
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr)
{
    return kDescCommon | (uint64_t(1024 >> 4) << 32) | (uint64_t(8192 >> 4) << 16) | ((addr >> 4) & 0x3fff);
}

// bf16 x bf16 -> fp32
__device__ __forceinline__ uint32_t instr_desc(int m, int n, bool a_mn_major, bool b_mn_major)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(a_mn_major) << 15) | (uint32_t(b_mn_major) << 16) | (uint32_t(n >> 3) << 17) |
           (uint32_t(m >> 4) << 24);
}

template <int CG>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    if (CG == 1)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
                     : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(accumulate))
                     : "memory");
}

// Arrives on `bar` (of both CTAs of a pair) once every product issued so far by this thread has been done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((uint16_t)3)
                     : "memory");
}

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns)
{
    if (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}

template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns)
{
    if (CG == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}

__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 accumulator columns of this warp's 32 lanes: v[c] is the lane's value of column c. The wait is part of the same
// statement, so that no use of v can be moved in front of it.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr)
        : "memory");
}

// True in one lane of a converged warp.
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

#endif  // __CUDACC__

}  // namespace ep
