// PTX wrappers and the operand layout of the product kernels (perq_mm_few.cuh, perq_mm_many.cuh).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace perq_mm {

constexpr uint32_t WAIT_POLLS = 1u << 22;

// Set (never cleared by kernels) when a bounded wait ran out: bit 4 in the product for few tokens, bit 5 in the one for many,
// bit 6 in the kernel of 8-bit codes.
static __device__ unsigned int g_error = 0u;
enum : unsigned int { ERROR_FEW = 1u << 4, ERROR_MANY = 1u << 5, ERROR_ROWS = 1u << 6 };

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// (by every thread that initialises one, before the CTA's barrier)
__device__ __forceinline__ void mbar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// At the same offset in the shared memory of another CTA of the cluster.
__device__ __forceinline__ void mbar_arrive_at(uint32_t bar, uint32_t rank)
{
    asm volatile("{ .reg .b32 a; mapa.shared::cluster.u32 a, %0, %1; mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a]; }"
                 ::"r"(bar), "r"(rank) : "memory");
}
__device__ __forceinline__ bool mbar_poll(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0u;
}
// Bounded wait: false if the phase did not complete within WAIT_POLLS polls.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity)
{
    if (mbar_poll(bar, parity)) return true;
    for (uint32_t i = 0; i < WAIT_POLLS; ++i)
        if (mbar_poll(bar, parity)) return true;
    return false;
}
// The same by all lanes of a warp, which go on together and agree: the tensor memory's loads and stores that follow want a converged warp,
// and nothing says that all lanes see a phase complete in the same poll.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

// As in the kernels of the online path: nothing touches global memory before griddep_wait.
__device__ __forceinline__ void griddep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void griddep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// ---------------------------------------------------------------------------------------------- tensor cores
// Operands are K-major rows of 128 bytes (128 8-bit codes) with 128-byte swizzle: the 16-byte chunk c of row r lies at
// r * 128 + ((c ^ r) & 7) * 16 of a tile that starts on a 1024-byte boundary.  A step of the tensor core takes 32 codes.
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | (1u << 16); }
constexpr uint32_t OPERAND_HI = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t operand_at(uint32_t r, uint32_t c) { return r * 128u + ((c ^ r) & 7u) * 16u; }
// 8-bit integers to 32-bit ones: the type of either operand (signed or not), rows m of the first, rows n of the second.
__host__ __device__ constexpr uint32_t product_desc(bool a_signed, bool b_signed, int m, int n)
{
    return (2u << 4) | ((uint32_t)a_signed << 7) | ((uint32_t)b_signed << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CTAS>
__device__ __forceinline__ void product(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    if (CTAS == 1)
        asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.b32 p, %4, 0; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5}; "
                     "tcgen05.mma.cta_group::1.kind::i8 [%0], a, b, %3, p; }"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(OPERAND_HI) : "memory");
    else
        asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.b32 p, %4, 0; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5}; "
                     "tcgen05.mma.cta_group::2.kind::i8 [%0], a, b, %3, p; }"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(OPERAND_HI) : "memory");
}
// The first operand in tensor memory: a row to a lane, four codes to a column.
__device__ __forceinline__ void product_from_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{ .reg .pred p; .reg .b64 b; setp.ne.b32 p, %4, 0; mov.b64 b, {%2, %5}; "
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], [%1], b, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(OPERAND_HI) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16 columns of this warp's 32 lanes; they are there after tmem_wait.
__device__ __forceinline__ void tmem_load16(uint32_t addr, int32_t (&u)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
                   "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait(int32_t (&u)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]),
                   "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15])
                 :: "memory");
}
// 16 columns of this warp's 32 lanes are written; they are there after tmem_store_wait.
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&u)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
                    "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------------ codes
// Packed codes keep their place in a byte, 16 times their value, which saves the shift and the sign: lo(w) are the even codes
// of eight, hi(w) the odd ones.  Products come out 16 (one operand packed) or 256 times too large, which the epilogue
// shifts away: |sum| <= 128 * 240 * 32768 < 2^31.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return (w << 4) & 0xf0f0f0f0u; }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return w & 0xf0f0f0f0u; }

// ----------------------------------------------------------------------------------------------------- results
enum OutType { OUT_BF16 = 0, OUT_F16 = 1, OUT_F32 = 2 };

// s_t s_n (sum + z_t c_n) in fp32: the sum is a whole number below 2^31 and rounded to fp32 once (2^-24), like the
// corrected sum, the two products and the result.
__device__ __forceinline__ float scaled(int32_t acc, int shift, float token, float channel, float zero, float sums)
{
    return fmaf(zero, sums, (float)(acc >> shift)) * token * channel;
}

}  // namespace perq_mm
