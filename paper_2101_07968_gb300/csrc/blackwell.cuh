// Thin wrappers of the sm_103a instructions that the expert products use: mbarriers,
// tensor copies (TMA), the fifth-generation tensor cores (tcgen05) and their memory (TMEM).
#pragma once

#include <cstdint>

namespace dc {
namespace bw {

__device__ __forceinline__ uint32_t smem_addr(const void *p)
{
    return uint32_t(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// One thread of a converged warp. The compiler knows that a branch on this is taken by one
// thread, and so feeds copies and products from uniform registers directly: under a branch
// on the lane number each such instruction took some 200 cycles.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p != 0;
}
// the address of this CTA's shared variable in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_to(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ------------------------------------------------------------------------ mbarriers
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
// Arrivals on this CTA's barriers; with the bytes that copies will bring.
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrivals on a barrier of any CTA of the cluster (address from map_to). A release at
// cluster scope waits for every earlier access of the thread, so the plain form is relaxed:
// it orders nothing but is enough after reads that have already returned.
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster_release(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void fence_cluster() { asm volatile("fence.acq_rel.cluster;" ::: "memory"); }

// A wait that ends: after kWaitTries tries or kWaitNs nanoseconds (a try may sleep a while), or
// once another thread of the CTA has given up, it gives up (false). A wait of this library's
// kernels lasts microseconds; one that may outlast many copies passes a word that changes as the
// CTA's work goes on, `progress`, and gives up once that has stood still for as long.
constexpr uint32_t kWaitTries = 1u << 23;
constexpr uint64_t kWaitNs = 2000000000ull;
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
static __device__ __noinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up,
                                                  volatile uint32_t *progress)
{
    uint64_t start = now_ns();
    uint32_t seen = progress ? *progress : 0;
    for (uint32_t i = 0; i < kWaitTries; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63u) != 63u) continue;
        if (progress && *progress != seen) {
            seen = *progress;
            start = now_ns();
            i = 0;
        }
        if (*gave_up || now_ns() - start > kWaitNs) break;
    }
    *gave_up = 1u;
    return false;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up,
                                         volatile uint32_t *progress = nullptr)
{
    for (int i = 0; i < 16; ++i)
        if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, gave_up, progress);
}

// --------------------------------------------------------------------------- copies
// Boxes of a tensor map into this CTA's shared memory; the bytes are counted on `bar`, a
// barrier of either CTA of the pair.
__device__ __forceinline__ void copy_2d(uint32_t dst, const void *map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
        "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void copy_3d(uint32_t dst, const void *map, int x, int y, int z,
                                        uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
// n bytes (a multiple of 16, both addresses on 16-byte boundaries)
__device__ __forceinline__ void copy_bytes(uint32_t dst, const void *src, uint32_t n, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
        "l"(src), "r"(n), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void prefetch_map(const void *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// this thread's writes to shared memory, made visible to copies and the tensor cores
__device__ __forceinline__ void fence_async()
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// -------------------------------------------------------------------- tensor memory
// of both CTAs of a pair, by a warp of each
__device__ __forceinline__ void tmem_alloc(uint32_t out, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(out), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this warp's 32 lanes: register j is column j of the thread's lane (the wait
// is part of the same statement, so that nothing reads the registers before it)
__device__ __forceinline__ void tmem_load(uint32_t at, float (&v)[32])
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// The same of 64 columns.
__device__ __forceinline__ void tmem_load(uint32_t at, float (&v)[64])
{
    uint32_t r[64];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int j = 0; j < 64; ++j) v[j] = __uint_as_float(r[j]);
}

// --------------------------------------------------------------------- tensor cores
// Shared-memory operand descriptor, 128-byte swizzle. K-major: rows of 64 elements, groups
// of eight rows 1,024 bytes apart. MN-major: lines of 64 elements along M or N, one line per
// k; eight lines are 1,024 bytes (the stride offset), and the next 64 elements lie
// `chunk` bytes on (the leading offset).
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t chunk)
{
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(chunk >> 4) << 16 | uint64_t(1024 >> 4) << 32 |
           uint64_t(1) << 46 | uint64_t(2) << 61;
}
// Instruction descriptor of kind::f16: float accumulators, both operands bfloat16 or both
// half, M and N, and whether A and B are MN-major.
__device__ __forceinline__ uint32_t f16_shape(bool bf16, bool a_mn, bool b_mn, uint32_t m, uint32_t n)
{
    const uint32_t f = bf16 ? 1u : 0u;
    return 1u << 4 | f << 7 | f << 10 | uint32_t(a_mn) << 15 | uint32_t(b_mn) << 16 | (n >> 3) << 17 |
           (m >> 4) << 24;
}
// kind::tf32: floats whose low 13 bits are not read, both operands K-major
__device__ __forceinline__ uint32_t tf32_shape(uint32_t m, uint32_t n)
{
    return 1u << 4 | 2u << 7 | 2u << 10 | (n >> 3) << 17 | (m >> 4) << 24;
}
// Products of a pair of CTAs, by a thread of its first.
__device__ __forceinline__ void mma_tf32(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::tf32 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"(uint32_t(add))
        : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"(uint32_t(add))
        : "memory");
}
// An arrival on `bar` of both CTAs once this thread's products are done.
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            bar),
        "h"(uint16_t(3))
        : "memory");
}

}  // namespace bw
}  // namespace dc
