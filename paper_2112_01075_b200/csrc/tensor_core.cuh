// The tensor cores from a kernel's point of view: barriers and tensor maps' boxes in shared memory, tcgen05 products by one
// SM (CG = 1) or a pair (CG = 2), tensor memory.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace redist {

constexpr int kBK = 64;                 // elements of the sum per slice: 128 bytes, one swizzle row

// ---- shared memory, barriers, tensor memory -----------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// True when the phase is over, false when this lane's `polls` polls have not seen it end.  (The roles that act through one
// lane ask that lane; the storing warps ask all.)  The loop is hidden from the compiler: the loading and the multiplying
// warp stay convergent in its eyes, and the descriptors of what they issue in uniform registers (a k-step took 400 cycles to
// issue when they did not, more than the tensor cores need for it).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t polls)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, %3;\n"
        "POLL:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\t"
        "setp.ne.u32 q, n, 0;\n\t"
        "@q bra POLL;\n"
        "DONE:\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(polls) : "memory");
    return done != 0;
}

// The same where threads of either block of a pair arrive and nothing but tensor memory is handed over: an order of execution, of
// no other memory.  By PTX's description of tcgen05.fence, ::before_thread_sync and ::after_thread_sync need no more than that
// between them: they compose with instructions that order the execution of threads, and then order the tcgen05 instructions on
// either side.  (Its canonical patterns for different threads have mbarrier.arrive.relaxed.cluster behind the one and
// mbarrier.try_wait.relaxed.cluster before the other.)
__device__ __forceinline__ bool bar_wait_order(uint32_t bar, uint32_t parity, uint32_t polls)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, %3;\n"
        "POLL:\n\t"
        "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\t"
        "setp.ne.u32 q, n, 0;\n\t"
        "@q bra POLL;\n"
        "DONE:\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(polls) : "memory");
    return done != 0;
}

// One lane of a convergent warp, always the same.
__device__ __forceinline__ bool elected()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// The address, in the cluster's shared-memory window, of what lies at `addr` in the block of rank 0.
__device__ __forceinline__ uint32_t in_first(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

// ... in the block of rank 1.
__device__ __forceinline__ uint32_t in_second(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(r) : "r"(addr));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One box of an operand; `bar` is this block's own barrier (CG = 1) or the first block's (CG = 2).
template <int CG>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// Shared-memory descriptor of a 128-byte-swizzled operand slice.  Contiguous along the sum: eight rows of 128 bytes
// form a group, groups follow each other every 1024 bytes.  Contiguous along the rows: 64 rows x 8 sum steps form a
// group of 1024 bytes, the next eight steps follow at 1024 bytes, the next 64 rows after the whole box of 64 steps.
__device__ __forceinline__ uint64_t slice_desc(uint32_t addr, int along_rows)
{
    const uint64_t lead = along_rows ? (kBK * 128) >> 4 : 1, stride = 1024 >> 4;
    return uint64_t((addr & 0x3ffff) >> 4) | (lead << 16) | (stride << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}

template <int CG>
__device__ __forceinline__ void mma(uint32_t acc, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}

// Arrive on `bar` (of both blocks, at the same place, for CG = 2) when all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
            ::"r"(bar), "h"(uint16_t(3)) : "memory");
}

template <int CG> __device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns)
{
    if constexpr (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}

template <int CG> __device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this warp's 32 lanes of tensor memory: register j = column j of lane `lane`.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

}  // namespace redist
