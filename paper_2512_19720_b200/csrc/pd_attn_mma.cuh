// What the attention kernels on the 5th-generation tensor cores share: packed arithmetic of the softmax, issue of products from
// shared memory, matrix descriptors.
#pragma once

#include "pd_tcgen05.cuh"

namespace pd {

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\nfma.rn.f32x2 x, x, y, z;\nmov.b64 {%0, %1}, x;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n.reg .b64 x, y;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// The products of a group are issued inside one `if (elect_one())` by a warp whose other threads keep to the same path.  Timed
// with stamps around the issue, products inside `if (lane == 0)` took 105 clocks each, more than the 64 that they run for;
// with an election for each product the 7 packed prompts take 261 us where one for the group gives 258.
__device__ __forceinline__ void mma_smem_a(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t x;
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\nselp.b32 %0, 1, 0, q;\n}\n" : "=r"(x));
    return x != 0;
}
__device__ __forceinline__ void commit_elected(uint64_t *bar) {
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "elect.sync _|q, 0xffffffff;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
        "}\n" ::"r"(smem_u32(bar))
        : "memory");
}
// Matrix descriptors of operands in rows of 128 bytes with the 128-byte swizzle, groups of 8 rows 1024 bytes apart.  Upper
// half: that distance, the descriptor's version, the swizzle.  Lower half: address; for a B operand whose contraction
// runs over the rows also the distance between its pieces of 64 columns (unused otherwise).
__device__ __forceinline__ uint64_t make_desc(uint32_t lower) {
    constexpr uint32_t upper = (1024u >> 4) | (1u << 14) | (2u << 29);
    return (static_cast<uint64_t>(upper) << 32) | lower;
}
__device__ __forceinline__ uint32_t desc_lower(const void *p, uint32_t piece_bytes) { return (smem_u32(p) >> 4) | ((piece_bytes >> 4) << 16); }

}  // namespace pd
