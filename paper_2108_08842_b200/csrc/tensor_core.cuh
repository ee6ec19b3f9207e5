// Thin wrappers over the sm_100a instructions that the linear kernels use: mbarriers with
// bounded waits, tensor copies, tcgen05 products and tensor memory.
#pragma once

#include <cstdint>

#include <cuda.h>

namespace eden {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// address of the same shared variable in another block of the cluster
__device__ __forceinline__ uint32_t address_in(uint32_t address, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(address), "r"(rank));
    return r;
}

// The whole warp executes the aligned forms as one, so lanes that took different branches meet first.
__device__ __forceinline__ void cluster_arrive_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One lane of a converged warp.  Copies and products are issued under this predicate, not under
// lane == 0: the compiler then knows that one thread runs them and keeps their operands in
// uniform registers (under lane == 0 a step of four products took 580 cycles of issue, which
// bound every tile shape).
__device__ __forceinline__ bool elected()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// ---- mbarriers ----------------------------------------------------------------------
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void barrier_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// bar is an address in the cluster's window (address_in).  Relaxed: what it says is that sums were
// read from tensor memory, which tmem_fence_before orders; a release would also wait for the
// stores of the epilogue.
__device__ __forceinline__ void barrier_arrive_remote(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Every wait ends: after kWaitTries tries (seconds; a tile takes a millisecond at most) it
// gives up and the caller leaves its loop.
constexpr uint32_t kWaitTries = 1u << 22;

// All lanes of the warp wait together; the vote tells the compiler that they leave together.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity)
{
    for (uint32_t i = 0; i < kWaitTries; ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (__all_sync(0xFFFFFFFFu, done)) return true;
    }
    return false;
}

// ---- registers: 4 warps x 56 + 8 x 224 = 12 x 168, or 4 x 40 + 16 x 104 < 20 x 96: no more than
// the block was launched with, which the host checks before the first launch of a kernel
constexpr int kLaunchRegisters[2] = {168, 96};           // a thread's at launch, for SIDES 2 and 4
template <int SIDES>
__device__ __forceinline__ void registers_down()
{
    if constexpr (SIDES == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
}

template <int SIDES>
__device__ __forceinline__ void registers_up()
{
    if constexpr (SIDES == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
}

// ---- tensor copies ------------------------------------------------------------------
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// box of a 2-D map at element (x, y) -> this block's shared memory; the bytes are counted by
// `bar`, an address in the cluster's window: with CG = 2 it may lie in the pair's other block
template <int CG>
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// ---- tensor memory ------------------------------------------------------------------
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns)       // one whole warp
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n\t"
                     "tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(slot), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n\t"
                     "tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(slot), "r"(columns) : "memory");
}

template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t address, uint32_t columns)     // the same warp
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}

__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: lane i gets row i
__device__ __forceinline__ void tmem_load(uint32_t address, float (&v)[32])
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(address)
        : "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}

// the way back, waited for
__device__ __forceinline__ void tmem_store(uint32_t address, const float (&v)[32])
{
    uint32_t r[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(v[j]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n\t"
        "tcgen05.wait::st.sync.aligned;"
        ::"r"(address), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
        "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
        "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// ---- products -----------------------------------------------------------------------
// Shared-memory matrix descriptor, 128-byte swizzle: address, byte strides over 16, version 1
// (bit 46), swizzle code 2 (bits 61..63).  K-major tiles (rows of 64 values along the sum):
// `stride` separates groups of 8 rows, `lead` is unused.  MN-major tiles (rows of 64 values
// along the matrix, one row per step of the sum): `stride` separates groups of 8 steps,
// `lead` blocks of 64 values.  Only the low word changes from tile to tile: the address over
// 16 lies in its low 14 bits (a block's shared memory ends below 2^18; the bits above name the
// block within its cluster and are cut off), so an offset over 16 adds on.
constexpr uint32_t kTileLead = 8192, kTileStride = 1024;
constexpr uint32_t kDescriptorHigh = kTileStride >> 4 | 1u << 14 | 2u << 29;

__device__ __forceinline__ uint32_t descriptor_low(uint32_t address) { return (address >> 4 & 0x3FFFu) | (kTileLead >> 4) << 16; }

__device__ __forceinline__ uint64_t tile_descriptor(uint32_t low) { return (uint64_t)kDescriptorHigh << 32 | low; }

// Instruction descriptor of kind::f16: fp32 sums, both operands bf16 or both fp16.
__host__ __device__ constexpr uint32_t product_descriptor(bool bf16, bool a_mn_major, bool b_mn_major, int m, int n)
{
    return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn_major ? 1u << 15 : 0u) | (b_mn_major ? 1u << 16 : 0u) |
           (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}

template <int CG>
__device__ __forceinline__ void tile_product(uint32_t d, uint64_t a, uint64_t b, uint32_t descriptor, bool add)
{
    if constexpr (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(descriptor), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(descriptor), "r"((uint32_t)add) : "memory");
}

// an arrival on `bar` (with CG = 2 on the barrier at that address in both blocks of the pair
// that starts at rank `leader`) when the products issued so far are done
template <int CG>
__device__ __forceinline__ void tile_commit(uint32_t bar, uint32_t leader)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)(3u << leader)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- shared memory by address -------------------------------------------------------
__device__ __forceinline__ void shared_store(uint32_t address, float v)
{
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(address), "f"(v) : "memory");
}

// address in the cluster's window (address_in)
__device__ __forceinline__ float cluster_load(uint32_t address)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(address));
    return v;
}

}  // namespace eden
