// Rotary positions: angles and the rotation of 16 values, shared by the calls that rotate.
//
// The pair (x, y) of a head turns by t = position * frequency to (x cos t - y sin t, x sin t + y cos t).  The product and its reduction to
// [-1/2, 1/2] turns are done in 64 bits: in 32 bits the angle of position 131071 at a frequency next to 1 would be off by up to 2^-8 of a
// radian.  Three roundings to 53 bits (the product, which has up to 55, the factor 1 / 2 pi and the product with it) leave an error below |t| 2^-51,
// 2^-20 of a radian at the far end of the positions, and the rounding of the reduced angle to 32 bits one below 2^-23.
#pragma once

#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {

// (cos, sin) of position * frequency, turned back for a direction of -1
__device__ __forceinline__ float2 angle(int position, float frequency, float direction) {
    const double turns = static_cast<double>(position) * static_cast<double>(frequency) * 0.15915494309189533577;
    const float half_turns = static_cast<float>(2.0 * (turns - rint(turns)));
    float2 cs;
    sincospif(half_turns, &cs.y, &cs.x);
    cs.y *= direction;
    return cs;
}

// A head's values are taken 16 at a time, as two pieces of 16 bytes: item j holds the pairs 8 j .. 8 j + 7 (those that pairs = head_dim / 2
// would have; behind the last pair its values stay as they are).
template <bool INTERLEAVED>
struct Item {
    int at0, at1;  // first values of the two pieces
    bool turns;
    __device__ __forceinline__ Item(int j, int pairs) {
        turns = 8 * j < pairs;
        const bool apart = !INTERLEAVED && turns;
        at0 = apart ? 8 * j : 16 * j;
        at1 = apart ? pairs + 8 * j : 16 * j + 8;
    }
};

struct Raw16 {
    uint4 v[2];
};
__device__ __forceinline__ Raw16 load16(const uint16_t *head, int at0, int at1) {
    return {{*reinterpret_cast<const uint4 *>(head + at0), *reinterpret_cast<const uint4 *>(head + at1)}};
}

// The 16 values, piece after piece, in binary32.
template <bool BF16>
__device__ __forceinline__ void unpack16(const Raw16 &raw, float (&f)[16]) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint32_t w[4] = {raw.v[p].x, raw.v[p].y, raw.v[p].z, raw.v[p].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 t = Elem<BF16>::to_float2(w[k]);
            f[8 * p + 2 * k] = t.x, f[8 * p + 2 * k + 1] = t.y;
        }
    }
}
template <bool INTERLEAVED>
__device__ __forceinline__ void turn16(float (&f)[16], const float2 (&cs)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float &x = f[INTERLEAVED ? 2 * k : k], &y = f[INTERLEAVED ? 2 * k + 1 : 8 + k];
        const float a = x, b = y;
        x = fmaf(a, cs[k].x, -b * cs[k].y);
        y = fmaf(a, cs[k].y, b * cs[k].x);
    }
}
template <bool BF16>
__device__ __forceinline__ void store16(uint16_t *head, int at0, int at1, const float (&f)[16]) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = Elem<BF16>::from_float2(f[8 * p + 2 * k], f[8 * p + 2 * k + 1]);
        *reinterpret_cast<uint4 *>(head + (p ? at1 : at0)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// The position that pair i of a token turns with; an axis outside the table is reported and counts as the first.  `place` is the
// token's place in its sequence.
__device__ __forceinline__ int position_of(const Rotation &r, int i, int64_t token, int place, uint32_t *status) {
    if (!r.positions) return place;
    int axis = r.axes ? __ldg(r.axes + i) : 0;
    if (axis < 0 || axis >= r.n_axes) {
        latch_error(status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(i));
        axis = 0;
    }
    return __ldg(r.positions + axis * r.axis_stride + token);
}

// A block turns one token of `heads[0] + heads[1]` heads.  cs: the token's angles, shared by all heads.  `ready` says (the same
// in all threads) whether the token is to be turned, and where it is; it runs while the first values are on their way.
constexpr int kAhead = 3;  // items that a thread has under way before it knows the angles
template <int D, bool BF16, bool INTERLEAVED, typename Ready>
__device__ __forceinline__ void turn_token(const HeadsView (&x)[2], const HeadsView (&out)[2], const int (&heads)[2], int token, const Rotation &r,
                                           float2 *cs, uint32_t *status, Ready ready) {
    constexpr int kItems = D / 16;
    const int j = threadIdx.x % kItems, lane_head = threadIdx.x / kItems, step = blockDim.x / kItems, all = heads[0] + heads[1];
    const Item<INTERLEAVED> item(j, r.pairs);
    auto from = [&](const HeadsView (&t)[2], int h) {
        const int which = h < heads[0] ? 0 : 1;
        return static_cast<uint16_t *>(const_cast<void *>(t[which].ptr)) + token * t[which].token_stride + (h - which * heads[0]) * t[which].head_stride;
    };
    Raw16 raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (lane_head + i * step < all) raw[i] = load16(from(x, lane_head + i * step), item.at0, item.at1);
    int place = 0;
    if (!ready(place)) return;
    for (int i = threadIdx.x; i < r.pairs; i += blockDim.x)
        cs[i] = angle(position_of(r, i, token, place, status), __ldg(r.inv_freq + i), r.direction);
    __syncthreads();
    float2 mine[8];
    if (item.turns) {
#pragma unroll
        for (int k = 0; k < 8; ++k) mine[k] = cs[8 * j + k];
    }
    auto finish = [&](int h, const Raw16 &t) {
        float f[16];
        unpack16<BF16>(t, f);
        if (item.turns) turn16<INTERLEAVED>(f, mine);
        store16<BF16>(from(out, h), item.at0, item.at1, f);
    };
    int h = lane_head;
#pragma unroll
    for (int i = 0; i < kAhead; ++i, h += step)
        if (h < all) finish(h, raw[i]);
    for (; h < all; h += step) finish(h, load16(from(x, h), item.at0, item.at1));
}

// Threads of such a block: rounds over the heads that are all full, if that is possible.
inline int turn_threads(int heads, int head_dim, int most) {
    const int items = head_dim / 16, rounds = (heads * items + most - 1) / most;
    return ((heads + rounds - 1) / rounds * items + 31) / 32 * 32;
}

}  // namespace pd
