// Barriers in shared memory, tensor memory and its matrix instructions, as the prompt kernels use them.
#pragma once

#include "remp_internal.h"

namespace remp {

#ifdef __CUDACC__

constexpr int kRowsM = 128;               // rows of a matrix
constexpr int32_t kWaitTries = 1 << 18;   // polls of a barrier before a wait is given up

// ---- barriers and tensor memory ----

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ void bar_arrive_expecting(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// Bounded: a wait that runs out marks the block, and nothing in it waits any more.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile int* dead, int32_t tries = kWaitTries) {
    for (int32_t i = 0; i < tries; ++i) {
        if (bar_try(bar, parity)) return;
        if (*dead) return;
    }
    *dead = 1;
}
// The last of `times` commits to a barrier has arrived. Always with the full limit.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t times, volatile int* dead) {
    if (times == 0) return;
    for (int32_t i = 0; i < kWaitTries; ++i)
        if (bar_try(bar, (times - 1) & 1)) return;
    *dead = 1;
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t leads) {
    asm volatile("{ .reg .pred q; setp.ne.b32 q, %1, 0; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar),
                 "r"(leads)
                 : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// Loads of 32 columns: asked for, and there (nothing that uses them can be moved before that).
__device__ __forceinline__ void tmem_ask32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_there32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                   "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                   "+r"(r[28]), "+r"(r[29])
                 :
                 : "memory");
    asm volatile("" : "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptors of operands in rows of 128 bytes (64 halves) along K, 16-byte pieces exchanged within 8 rows: the low word goes
// by the address, in units of 16 bytes, the high word is the same for all. Halves times halves into 32 bits, 128 rows.
__device__ __forceinline__ uint32_t operand_low(uint32_t at) { return (at >> 4 & 0x3fff) | 1u << 16; }
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__host__ __device__ constexpr uint32_t shape_of(int n) { return 1u << 4 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRowsM >> 4) << 24; }
template <int N>
constexpr uint32_t kShape = shape_of(N);
constexpr uint32_t kShapeBfloat = 1u << 7 | 1u << 10;  // added to it: bfloat16 times bfloat16
constexpr uint32_t kShapeBAcross = 1u << 16;           // added to it: B lies in rows along N, not along K

// The whole warp gets here with the same operands (so they stay in uniform registers); the lane with `leads` issues.
template <int N>
__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t add, uint32_t leads) {
    asm volatile(
        "{ .reg .pred p, q; .reg .b64 a, b; setp.ne.b32 p, %4, 0; setp.ne.b32 q, %6, 0; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5};"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p; }" ::"r"(d), "r"(a_low), "r"(b_low), "r"(kShape<N>), "r"(add), "r"(kOperandHigh),
        "r"(leads)
        : "memory");
}
template <int N>
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b_low, uint32_t add, uint32_t leads) {
    asm volatile(
        "{ .reg .pred p, q; .reg .b64 b; setp.ne.b32 p, %4, 0; setp.ne.b32 q, %6, 0; mov.b64 b, {%2, %5};"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p; }" ::"r"(d), "r"(a), "r"(b_low), "r"(kShape<N>), "r"(add), "r"(kOperandHigh),
        "r"(leads)
        : "memory");
}

// Two numbers at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{ .reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// The same from one thread (that which elect_one names), with whole descriptors.
__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(is));
    return is;
}
__device__ __forceinline__ uint64_t operand_at(uint32_t at) { return (uint64_t)kOperandHigh << 32 | operand_low(at); }
__device__ __forceinline__ void mma_smem_one(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b),
                 "r"(shape), "r"(add)
                 : "memory");
}
template <int N, uint32_t kMore = 0>
__device__ __forceinline__ void mma_tmem_one(uint32_t d, uint32_t a, uint64_t b, uint32_t add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b),
                 "r"(kShape<N> | kMore), "r"(add)
                 : "memory");
}
__device__ __forceinline__ void commit_one(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void for_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

#endif

}  // namespace remp
