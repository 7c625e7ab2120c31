// Scales, codes and checks that the calls which write the 8-bit paged cache share.
#pragma once

#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {

// max that hands a NaN on, so that a page with a NaN among its values reads as NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Rounding to a whole number (to nearest even) by adding 1.5 * 2^23: the sum's low byte is the code.  A conversion
// instruction runs at an eighth of the rate.
constexpr float kShift = 12582912.f;
__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
    return prmt(prmt(__float_as_uint(a), __float_as_uint(b), 0x0040), prmt(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

struct Scale {
    float s, inv;    // 1 / s; 0 where s is too small for it, infinite or NaN
    uint32_t keep;   // bits of the codes: none where inv is 0, so that an infinite scale times any code of the page is NaN too
};
__device__ __forceinline__ Scale scale_of(float s_old, float amax) {
    const float s = max_nan(s_old, __fdiv_rn(amax, 127.f)), inv = s >= 0x1p-120f ? __frcp_rn(s) : 0.f;
    return {s, inv, inv > 0.f ? 0xffffffffu : 0u};
}

// sixteen held codes of the smaller scale s_old to those of the larger one
__device__ __forceinline__ void scale_again16(uint4 *p, float s_old, const Scale &sc) {
    const float ratio = s_old * sc.inv;
    const uint4 c = *p;
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float f[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = __fadd_rn(__fmul_rn(static_cast<float>(static_cast<int8_t>(w[j] >> (8 * k))), ratio), kShift);
        r[j] = low_bytes(f[0], f[1], f[2], f[3]) & sc.keep;
    }
    *p = make_uint4(r[0], r[1], r[2], r[3]);
}

__device__ __forceinline__ bool bad_lengths(const AppendArgs &a, int first, int last, int len) {
    return first < 0 || last < first || last > a.n_tokens || len < last - first;
}

}  // namespace pd
