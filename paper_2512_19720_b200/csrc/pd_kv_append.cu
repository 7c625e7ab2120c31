// Writing keys and values into the 8-bit paged cache.
//
// A page holds `page` consecutive tokens of one sequence; for each of its key/value heads it has one scale s and the codes
// c = round(x / s) of its values, so that it stands for c * s.  When tokens are added, the scale only grows:
//     s' = max(s_held, max |x_new| / 127),   held codes c' = round(c * (s_held / s')),   new codes = round(x / s')
// with s_held = 0 for a page whose first token is among the new ones.  Both divisions by s' are products with 1 / s'
// (binary32); a page whose s' is below 2^-120 holds zeros, since 1 / s' would overflow.
//
// One thread block takes one (page, head) of the keys or of the values: 16-bit values are read once, kept in registers
// while the block finds their largest magnitude, and written as codes.  The held codes are read and written again only
// where the scale grew.  Bound by memory: per value 2 bytes in and 1 byte out (3 with the values handed back).
#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

constexpr int kVecs = 8;  // 16-byte pieces (8 values) that a thread keeps in registers

// max that hands a NaN on, so that a page with a NaN among its values reads as NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const int x = __float2int_rn(a), y = __float2int_rn(b), z = __float2int_rn(c), w = __float2int_rn(d);
    return prmt(prmt(static_cast<uint32_t>(x), static_cast<uint32_t>(y), 0x0040), prmt(static_cast<uint32_t>(z), static_cast<uint32_t>(w), 0x0040), 0x5410);
}

template <int D, bool BF16>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendArgs a) {
    using E = Elem<BF16>;
    __shared__ float red[8];
    __shared__ int found;
    const int id = blockIdx.x, head = blockIdx.y, which = blockIdx.z;
    const int page = 1 << a.page_log2;
    // Sequence b's pages are the ids from cu[b] / page + 2 b on: there are never more of them than ids before the next
    // sequence's, so that the page of a block is found from the offsets alone.
    if (threadIdx.x == 0) found = 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the previous kernel drains
    int mine = 0;
    for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
        if ((min(max(__ldg(a.cu_seqlens + b), 0), a.n_tokens) >> a.page_log2) + 2 * b <= id) mine = b;  // ascending in b
    if (mine) atomicMax(&found, mine);
    __syncthreads();
    const int b = found;
    const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1), len = __ldg(a.seq_lens + b);
    if (first < 0 || last < first || last > a.n_tokens || len < last - first) {
        if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return;
    }
    const int pos0 = len - (last - first);  // position of the first new token
    const int pi = (pos0 >> a.page_log2) + id - ((first >> a.page_log2) + 2 * b);
    const int64_t page_start = static_cast<int64_t>(pi) << a.page_log2;
    const int lo = static_cast<int>(max(static_cast<int64_t>(pos0), page_start));
    const int hi = static_cast<int>(min(static_cast<int64_t>(len), page_start + page));
    if (lo >= hi) return;
    const int64_t pid = pi < a.table_width ? __ldg(a.block_table + b * a.table_stride + pi) : -1;
    if (pid < 0 || pid >= a.n_pages) {
        if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return;
    }
    const int held = lo & (page - 1);
    int8_t *codes = a.pages[which].codes + ((pid * a.kv_heads + head) << a.page_log2) * D;
    float *scale = a.pages[which].scale + pid * a.kv_heads + head;
    const float s_old = held ? *scale : 0.f;

    constexpr int kPer = D / 8;  // pieces of a token
    const int n_vec = (hi - lo) * kPer;
    const int64_t tok0 = first + (lo - pos0);
    const uint16_t *x = static_cast<const uint16_t *>(a.x[which].ptr) + head * a.x[which].head_stride;
    uint4 raw[kVecs];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int at = threadIdx.x + i * blockDim.x;
        raw[i] = make_uint4(0, 0, 0, 0);
        if (at < n_vec) raw[i] = __ldg(reinterpret_cast<const uint4 *>(x + (tok0 + at / kPer) * a.x[which].token_stride) + at % kPer);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = E::to_float2(w[j]);
            amax = max_nan(amax, max_nan(fabsf(f.x), fabsf(f.y)));
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, d));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = red[0];
    for (int w = 1; w < static_cast<int>(blockDim.x >> 5); ++w) amax = max_nan(amax, red[w]);
    const float s_new = max_nan(s_old, __fdiv_rn(amax, 127.f));
    const float inv = s_new >= 0x1p-120f ? __frcp_rn(s_new) : 0.f;  // 0 for an infinite scale too; a NaN scale gives codes of 0

    if (held && s_new != s_old) {
        const float ratio = s_old * inv;
        for (int at = threadIdx.x; at < held * (D / 16); at += blockDim.x) {
            uint4 *p = reinterpret_cast<uint4 *>(codes) + at;
            const uint4 c = *p;
            const uint32_t w[4] = {c.x, c.y, c.z, c.w};
            uint32_t r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float f[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = static_cast<float>(static_cast<int8_t>(w[j] >> (8 * k))) * ratio;
                r[j] = pack4(f[0], f[1], f[2], f[3]);
            }
            *p = make_uint4(r[0], r[1], r[2], r[3]);
        }
    }
    uint16_t *values = static_cast<uint16_t *>(a.values[which]);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int at = threadIdx.x + i * blockDim.x;
        if (at < n_vec) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 t = E::to_float2(w[j]);
                f[2 * j] = rintf(t.x * inv), f[2 * j + 1] = rintf(t.y * inv);
            }
            const uint2 c = make_uint2(pack4(f[0], f[1], f[2], f[3]), pack4(f[4], f[5], f[6], f[7]));
            *(reinterpret_cast<uint2 *>(codes + static_cast<int64_t>(held + at / kPer) * D) + at % kPer) = c;
            if (values) {
                const uint4 o = make_uint4(E::from_float2(f[0] * s_new, f[1] * s_new), E::from_float2(f[2] * s_new, f[3] * s_new),
                                           E::from_float2(f[4] * s_new, f[5] * s_new), E::from_float2(f[6] * s_new, f[7] * s_new));
                *(reinterpret_cast<uint4 *>(values + ((tok0 + at / kPer) * a.kv_heads + head) * D) + at % kPer) = o;
            }
        }
    }
    if (threadIdx.x == 0) *scale = s_new;
}

}  // namespace

pd_status launch_kv_append(const AppendArgs &a, bool bf16, cudaStream_t stream) {
    const int page = 1 << a.page_log2;
    const unsigned ids = static_cast<unsigned>(a.n_tokens / page + 2 * a.n_seqs + 1);
    const dim3 grid(ids, static_cast<unsigned>(a.kv_heads), 2);
    const int threads = max(32, min(256, page * a.head_dim / (8 * kVecs)));
    auto kernel = a.head_dim == 128 ? (bf16 ? kv_append_kernel<128, true> : kv_append_kernel<128, false>)
                                    : (bf16 ? kv_append_kernel<64, true> : kv_append_kernel<64, false>);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, a));
}

}  // namespace pd
