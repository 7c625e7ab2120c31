// Causal attention over packed prompts: out[i, h] = sum_{j <= i} softmax_j(scale q[i, h] . k[j, g]) v[j, g] inside each sequence.
//
// One pass over the keys with a running maximum m and sum l of each query row (32 bits): with s the scores of a tile,
//     m' = max(m, max s),  l' = l e^(m - m') + sum e^(s - m'),  O' = O e^(m - m') + e^(s - m') V,  out = O / l at the end.
// P = e^(s - m') is rounded to the type of v for its product; l sums the unrounded values.
//
// A thread block takes 64 queries of one head, a warp 16 of them, against tiles of 64 keys.
#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

constexpr int kQ = 64, kK = 64;  // queries of a block, keys of a tile
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], const void *p) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_u32(p)) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], const void *p) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_u32(p)) : "memory");
}
// one of the two 16-bit values is an infinity or a NaN
template <bool BF16>
__device__ __forceinline__ bool non_finite2(uint32_t w) {
    constexpr uint32_t e = BF16 ? 0x7F80u : 0x7C00u;
    return (w & e) == e || ((w >> 16) & e) == e;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(128) attn_prompt_kernel(const PromptArgs a) {
    using E = Elem<BF16>;
    constexpr int P = D + 8;  // row pitch in shared memory
    extern __shared__ __align__(16) uint16_t sm[];
    uint16_t *sq = sm, *sk = sm + kQ * P, *sv = sk + kK * P;
    __shared__ int found, tainted;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // sequence b's blocks are the ids from cu[b] / 64 + b on: never more than the ids before the next sequence's
    if (threadIdx.x == 0) found = 0, tainted = 0;
    __syncthreads();
    int mine = 0;
    for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
        if (min(max(__ldg(a.cu_seqlens + b), 0), a.n_tokens) / kQ + b <= static_cast<int>(blockIdx.x)) mine = b;
    if (mine) atomicMax(&found, mine);
    __syncthreads();
    const int b = found;
    const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1);
    if (first < 0 || last < first || last > a.n_tokens) {
        if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return;
    }
    const int len = last - first, q0 = (static_cast<int>(blockIdx.x) - first / kQ - b) * kQ;
    if (q0 >= len) return;
    const int head = blockIdx.y, kvh = head / (a.q_heads / a.kv_heads);
    const uint16_t *qp = static_cast<const uint16_t *>(a.q.ptr) + first * a.q.token_stride + head * a.q.head_stride;
    const uint16_t *kp = static_cast<const uint16_t *>(a.k.ptr) + first * a.k.token_stride + kvh * a.k.head_stride;
    const uint16_t *vp = static_cast<const uint16_t *>(a.v.ptr) + first * a.v.token_stride + kvh * a.v.head_stride;
    auto load = [&](uint16_t *dst, const uint16_t *src, int64_t stride, int row0) {
        for (int i = threadIdx.x; i < 64 * (D / 8); i += blockDim.x) {
            const int r = i / (D / 8), c = i % (D / 8);
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row0 + r < len) x = __ldg(reinterpret_cast<const uint4 *>(src + (row0 + r) * stride) + c);
            *reinterpret_cast<uint4 *>(dst + r * P + 8 * c) = x;
        }
    };
    load(sq, qp, a.q.token_stride, q0);
    __syncthreads();
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) ldmatrix_x4(qf[k], sq + (warp * 16 + (lane & 15)) * P + 16 * k + 8 * (lane >> 4));
    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    const float f = a.scale * kLog2e;
    const int row0 = q0 + warp * 16 + g;  // and row0 + 8

    for (int k0 = 0; k0 <= q0; k0 += kK) {
        __syncthreads();
        load(sk, kp, a.k.token_stride, k0);
        load(sv, vp, a.v.token_stride, k0);
        __syncthreads();
        if (k0 == q0) {  // some queries do not attend to some of these keys: 0 * infinity must not reach them
            for (int i = threadIdx.x; i < kK * (D / 2); i += blockDim.x) {
                uint32_t *w = reinterpret_cast<uint32_t *>(sv + i / (D / 2) * P) + i % (D / 2);
                if (non_finite2<BF16>(*w)) {
                    tainted = 1;
                    if (non_finite2<BF16>(*w & 0xffffu)) *w &= 0xffff0000u;
                    if (non_finite2<BF16>(*w & 0xffff0000u)) *w &= 0xffffu;
                }
            }
            __syncthreads();
        }
        float s[kK / 8][4];
#pragma unroll
        for (int j = 0; j < kK / 8; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int j = 0; j < kK / 16; ++j) {
                uint32_t kf[4];
                ldmatrix_x4(kf, sk + (j * 16 + (lane & 7) + 8 * (lane >> 4)) * P + 16 * k + 8 * ((lane >> 3) & 1));
                E::mma16816(s[2 * j], qf[k][0], qf[k][1], qf[k][2], qf[k][3], kf[0], kf[1]);
                E::mma16816(s[2 * j + 1], qf[k][0], qf[k][1], qf[k][2], qf[k][3], kf[2], kf[3]);
            }
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int j = 0; j < kK / 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int key = k0 + 8 * j + 2 * t + (k & 1);
                s[j][k] = key <= row0 + 8 * (k >> 1) ? s[j][k] * f : -INFINITY;
                top[k >> 1] = fmaxf(top[k >> 1], s[j][k]);
            }
        float mu[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
            mu[r] = top[r] == -INFINITY ? 0.f : top[r];
            const float shrink = exp2_approx(m[r] - mu[r]);
            m[r] = top[r], l[r] *= shrink;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) o[i][2 * r] *= shrink, o[i][2 * r + 1] *= shrink;
        }
#pragma unroll
        for (int j = 0; j < kK / 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s[j][k] = exp2_approx(s[j][k] - mu[k >> 1]);
                l[k >> 1] += s[j][k];
            }
#pragma unroll
        for (int j = 0; j < kK / 16; ++j) {
            const uint32_t p0 = E::from_float2(s[2 * j][0], s[2 * j][1]), p1 = E::from_float2(s[2 * j][2], s[2 * j][3]);
            const uint32_t p2 = E::from_float2(s[2 * j + 1][0], s[2 * j + 1][1]), p3 = E::from_float2(s[2 * j + 1][2], s[2 * j + 1][3]);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint32_t vf[4];
                ldmatrix_x4_trans(vf, sv + (j * 16 + (lane & 15)) * P + 16 * i + 8 * (lane >> 4));
                E::mma16816(o[2 * i], p0, p1, p2, p3, vf[0], vf[1]);
                E::mma16816(o[2 * i + 1], p0, p1, p2, p3, vf[2], vf[3]);
            }
        }
    }
    const bool taint = tainted != 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        const int row = row0 + 8 * r;
        if (row >= len) continue;
        const float inv = 1.f / l[r];
        uint16_t *y = static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + (first + row) * a.out.token_stride + head * a.out.head_stride;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            float x[2] = {o[i][2 * r] * inv, o[i][2 * r + 1] * inv};
            if (taint) {  // infinities and NaN among the values of the last tile, for the queries that attend to them
                for (int j = q0; j <= row; ++j)
                    for (int k = 0; k < 2; ++k) {
                        const float v = E::to_float(vp[j * a.v.token_stride + 8 * i + 2 * t + k]);
                        if (!(fabsf(v) <= 3.402823466e38f)) x[k] += v;
                    }
            }
            *reinterpret_cast<uint32_t *>(y + 8 * i + 2 * t) = E::from_float2(x[0], x[1]);
        }
    }
}

template <int D, bool BF16>
pd_status launch(const PromptArgs &a, cudaStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    constexpr int bytes = 3 * 64 * (D + 8) * 2;
    if (!ensure_dynamic_smem(attn_prompt_kernel<D, BF16>, bytes, done)) return PD_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>(a.n_tokens / kQ + a.n_seqs), static_cast<unsigned>(a.q_heads));
    attn_prompt_kernel<D, BF16><<<grid, 128, bytes, stream>>>(a);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

}  // namespace

pd_status launch_attn_prompt(const PromptArgs &a, bool bf16, cudaStream_t stream) {
    if (a.head_dim == 128) return bf16 ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
    return bf16 ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
}

}  // namespace pd
