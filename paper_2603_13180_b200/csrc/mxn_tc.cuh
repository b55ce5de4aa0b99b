// 5th-generation tensor cores: descriptors, products, tensor memory; bounded waits; maxima that keep a NaN.
#pragma once

#include "mxn_async.cuh"

namespace mxn {

// ---- tensor core plumbing ------------------------------------------------------------------------------------
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// shared-memory operand descriptor: address, stride between groups of 8 rows (`group`), between repeats along the other
// axis (`repeat`), and the swizzle (2: 128 bytes, 4: 64 bytes)
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t group, uint32_t repeat, uint32_t swizzle)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(repeat >> 4) << 16) | ((uint64_t)(group >> 4) << 32) | (1ull << 46) |
           ((uint64_t)swizzle << 61);
}
// instruction descriptors: binary32 sums, M = 128
__host__ __device__ constexpr uint32_t idesc_e4m3(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__host__ __device__ constexpr uint32_t idesc_bf16(int n) { return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__host__ __device__ constexpr uint32_t idesc_f16_bt(int n) { return (1u << 4) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }

__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
#define MXN_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define MXN_U8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define MXN_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of this warp's 32 lanes, a lane's row in its thread
__device__ __forceinline__ void tm_load(uint32_t (&r)[32], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : MXN_R8(r, 0), MXN_R8(r, 8), MXN_R8(r, 16), MXN_R8(r, 24) : "r"(addr) : "memory");
}
// the same in two steps: the values are there after tm_arrived of the same registers
__device__ __forceinline__ void tm_request(uint32_t (&r)[32], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : MXN_R8(r, 0), MXN_R8(r, 8), MXN_R8(r, 16), MXN_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_arrived(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : MXN_U8(r, 0), MXN_U8(r, 8), MXN_U8(r, 16), MXN_U8(r, 24) :: "memory");
}
__device__ __forceinline__ void tm_store32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(addr), MXN_I8(r, 0), MXN_I8(r, 8), MXN_I8(r, 16), MXN_I8(r, 24) : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(addr), MXN_I8(r, 0), MXN_I8(r, 8) : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t (&r)[16], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : MXN_R8(r, 0), MXN_R8(r, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// waits with a limit; a wait that runs out, or one that sees another's, ends the CTA's work
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* dead)
{
    if (mbar_test(bar, parity)) return true;
    for (uint32_t spin = 0; spin < (1u << 20); ++spin) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((spin & 255u) == 255u && *dead) return false;
    }
    *dead = 1;
    return false;
}

__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 f2(float a) { return make_float2(a, a); }

}  // namespace mxn
