// Writing keys and values into the 8-bit paged cache.
//
// A page holds `page` consecutive tokens of one sequence; for each of its key/value heads it has one scale s and the codes
// c = round(x / s) of its values, so that it stands for c * s.  When tokens are added, the scale only grows:
//     s' = max(s_held, max |x_new| / 127),   held codes c' = round(c * (s_held / s')),   new codes = round(x / s')
// with s_held = 0 for a page whose first token is among the new ones.  Both divisions by s' are products with 1 / s'
// (binary32); a page whose s' is below 2^-120 holds zeros, since 1 / s' would overflow.
//
// Bound by memory: per value 2 bytes in and 1 byte out (3 with the values handed back).  Two kernels:
//   pages : a thread block takes one (page, head) of the keys or of the values; the 16-bit values are read once and stay in
//           registers while the block finds their largest magnitude.  What a block has to know before it can load anything (its
//           sequence) is one round of loads, the page's number comes with the values.
//   tokens: a warp takes one (sequence, head) of the keys or of the values and walks over its pages, a token at a time
//           per half warp.  For decode steps: a block per page would mostly wait for four rounds of loads, and half of the
//           blocks would find nothing to do.
// The held codes are read and written again only where the scale grew.
#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

// pages: 16-byte pieces (8 values) that a thread keeps in registers; 8523 tokens, 8 heads of 128, pages of 64: 18.0 us with 4,
// 16.9 with 8, of which the bytes (88 MB) take 13.5
constexpr int kVecs = 8;
constexpr int kMaxThreads = 256;
constexpr int kTokenWarps = 8;   // tokens: warps of a block
// tokens: up to so many new tokens a sequence on average, which is all that the host knows.  Back to back in a graph, heads of
// 128, pages of 64, us with tokens / with pages:
//   8 heads, 64 sequences of 1, 4, 8 tokens: 2.2 / 4.7, 3.0 / 4.8, 4.4 / 5.0;  512 of 1, 4: 3.7 / 23.3, 5.2 / 24.3
//   32 heads, 64 sequences of 1, 4, 8 tokens: 3.1 / 12.4, 4.0 / 12.9, 5.6 / 13.7
// An average does not show a long piece among single tokens, over which one warp then walks (8 heads, 63 sequences of 1 and one of
// 190: 40 / 5.0;  511 of 1 and one of 1500: 336 / 24.8): a program that mixes them does better with a call for each kind, until
// the choice is made for each sequence on the device.
constexpr int kFewTokens = 4;

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

// The largest magnitude, two at a time: without their signs the 16-bit values order like whole numbers, a NaN above all.
__device__ __forceinline__ uint32_t magnitude2(const uint4 &raw, uint32_t most) {
    return __vmaxu2(__vmaxu2(__vmaxu2(raw.x & 0x7fff7fffu, raw.y & 0x7fff7fffu), __vmaxu2(raw.z & 0x7fff7fffu, raw.w & 0x7fff7fffu)), most);
}
template <bool BF16>
__device__ __forceinline__ float warp_magnitude(uint32_t most) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, d));
    return Elem<BF16>::to_float(static_cast<unsigned short>(max(most & 0xffffu, most >> 16)));
}

struct Scale {
    float s, inv;    // 1 / s; 0 where s is too small for it, infinite or NaN
    uint32_t keep;   // bits of the codes: none where inv is 0, so that an infinite scale times any code of the page is NaN too
};
__device__ __forceinline__ Scale scale_of(float s_old, float amax) {
    const float s = max_nan(s_old, __fdiv_rn(amax, 127.f)), inv = s >= 0x1p-120f ? __frcp_rn(s) : 0.f;
    return {s, inv, inv > 0.f ? 0xffffffffu : 0u};
}

// eight values to their codes and, unless nullptr, to the values that those stand for
template <bool BF16>
__device__ __forceinline__ void store8(const uint4 &raw, const Scale &sc, int8_t *codes, uint16_t *values) {
    using E = Elem<BF16>;
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 t = E::to_float2(w[j]);
        f[2 * j] = __fadd_rn(__fmul_rn(t.x, sc.inv), kShift), f[2 * j + 1] = __fadd_rn(__fmul_rn(t.y, sc.inv), kShift);
    }
    *reinterpret_cast<uint2 *>(codes) = make_uint2(low_bytes(f[0], f[1], f[2], f[3]) & sc.keep, low_bytes(f[4], f[5], f[6], f[7]) & sc.keep);
    if (values) {
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = E::from_float2((f[2 * j] - kShift) * sc.s, (f[2 * j + 1] - kShift) * sc.s);
        *reinterpret_cast<uint4 *>(values) = make_uint4(o[0], o[1], o[2], o[3]);
    }
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

template <int D, bool BF16>
__global__ void __launch_bounds__(kMaxThreads, 4) append_pages_kernel(const AppendArgs a) {
    __shared__ float red[kMaxThreads / 32];
    const int id = blockIdx.x, head = blockIdx.y, which = blockIdx.z, lane = threadIdx.x & 31;
    const int page = 1 << a.page_log2;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the previous kernel drains
    if (head == 0 && which == 0) {  // offsets that decrease may keep the search below from ever seeing a sequence: the first blocks look at all
        const int64_t b = static_cast<int64_t>(id) * blockDim.x + threadIdx.x;
        if (b < a.n_seqs && bad_lengths(a, __ldg(a.cu_seqlens + b), __ldg(a.cu_seqlens + b + 1), __ldg(a.seq_lens + b)))
            latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
    }
    // Sequence b's pages are the ids from cu[b] / page + 2 b on: there are never more of them than ids before the next
    // sequence's.  Every warp finds the last sequence that starts at or before the block's id, 32 candidates a round.
    int b = 0, left = a.n_seqs, first, last, len;
    while (true) {
        const int step = (left + 31) / 32, mine = min(b + lane * step, a.n_seqs - 1);
        first = __ldg(a.cu_seqlens + mine), last = __ldg(a.cu_seqlens + mine + 1), len = __ldg(a.seq_lens + mine);
        const unsigned m = __ballot_sync(0xffffffffu, lane * step < left && (min(max(first, 0), a.n_tokens) >> a.page_log2) + 2 * mine <= id);
        const int src = m ? 31 - __clz(m) : 0;
        b += src * step;
        left = min(step, left - src * step);
        if (left <= 1) {
            first = __shfl_sync(0xffffffffu, first, src), last = __shfl_sync(0xffffffffu, last, src), len = __shfl_sync(0xffffffffu, len, src);
            break;
        }
    }
    if (bad_lengths(a, first, last, len)) return;
    const int pos0 = len - (last - first);  // position of the first new token
    const int pi = (pos0 >> a.page_log2) + id - ((first >> a.page_log2) + 2 * b);
    const int64_t page_start = static_cast<int64_t>(pi) << a.page_log2;
    const int lo = static_cast<int>(max(static_cast<int64_t>(pos0), page_start));
    const int hi = static_cast<int>(min(static_cast<int64_t>(len), page_start + page));
    if (lo >= hi) return;
    const int64_t pid = pi < a.table_width ? __ldg(a.block_table + b * a.table_stride + pi) : -1;
    constexpr int kPer = D / 8;  // pieces of a token
    const int n = hi - lo, tok = threadIdx.x / kPer, piece = threadIdx.x % kPer, stride = blockDim.x / kPer;  // a thread takes every stride-th token's piece
    const int64_t tok0 = first + (lo - pos0) + tok;
    const uint16_t *x = static_cast<const uint16_t *>(a.x[which].ptr) + head * a.x[which].head_stride + tok0 * a.x[which].token_stride + 8 * piece;
    uint4 raw[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        raw[i] = make_uint4(0, 0, 0, 0);
        if (tok + i * stride < n) raw[i] = __ldg(reinterpret_cast<const uint4 *>(x));
        x += stride * a.x[which].token_stride;
    }
    if (pid < 0 || pid >= a.n_pages) {
        if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return;
    }
    const int held = lo & (page - 1);
    int8_t *codes = a.pages[which].codes + ((pid * a.kv_heads + head) << a.page_log2) * D;
    float *scale = a.pages[which].scale + pid * a.kv_heads + head;
    const float s_old = held ? *scale : 0.f;
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) most = magnitude2(raw[i], most);
    float amax = warp_magnitude<BF16>(most);
    if (lane == 0) red[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = red[0];
    for (int w = 1; w < static_cast<int>(blockDim.x >> 5); ++w) amax = max_nan(amax, red[w]);
    const Scale sc = scale_of(s_old, amax);
    if (held && sc.s != s_old)
        for (int at = threadIdx.x; at < held * (D / 16); at += blockDim.x) scale_again16(reinterpret_cast<uint4 *>(codes) + at, s_old, sc);
    int8_t *to = codes + (held + tok) * D + 8 * piece;
    uint16_t *values = static_cast<uint16_t *>(a.values[which]);
    if (values) values += (tok0 * a.kv_heads + head) * D + 8 * piece;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
        if (tok + i * stride < n)
            store8<BF16>(raw[i], sc, to + i * stride * D, values ? values + static_cast<int64_t>(i * stride) * a.kv_heads * D : nullptr);
    if (threadIdx.x == 0) *scale = sc.s;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kTokenWarps * 32) append_tokens_kernel(const AppendArgs a) {
    const int lane = threadIdx.x & 31, b = blockIdx.x, item = blockIdx.y * kTokenWarps + (threadIdx.x >> 5);
    const int which = item & 1, head = item >> 1;
    const int page = 1 << a.page_log2;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (head >= a.kv_heads) return;
    const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1), len = __ldg(a.seq_lens + b);
    if (bad_lengths(a, first, last, len)) {
        if (lane == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return;
    }
    constexpr int kPer = D / 8;       // lanes of a token
    constexpr int kSide = 32 / kPer;  // tokens side by side
    const int piece = lane % kPer;
    const uint16_t *x = static_cast<const uint16_t *>(a.x[which].ptr) + head * a.x[which].head_stride + 8 * piece;
    uint16_t *values = static_cast<uint16_t *>(a.values[which]);
    for (int lo = len - (last - first); lo < len;) {
        const int pi = lo >> a.page_log2, held = lo & (page - 1), n = min(len - lo, page - held);
        const int64_t tok0 = first + (lo - (len - (last - first)));
        const int64_t pid = pi < a.table_width ? __ldg(a.block_table + b * a.table_stride + pi) : -1;
        auto load = [&](int tok) { return __ldg(reinterpret_cast<const uint4 *>(x + (tok0 + tok) * a.x[which].token_stride)); };
        const int mine = lane / kPer;
        uint4 raw = make_uint4(0, 0, 0, 0);  // the lane's first token; the others are read twice
        if (mine < n) raw = load(mine);
        if (pid < 0 || pid >= a.n_pages) {
            if (lane == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
            return;
        }
        int8_t *codes = a.pages[which].codes + ((pid * a.kv_heads + head) << a.page_log2) * D;
        float *scale = a.pages[which].scale + pid * a.kv_heads + head;
        const float s_old = held ? *scale : 0.f;
        uint32_t most = magnitude2(raw, 0u);
        for (int tok = mine + kSide; tok < n; tok += kSide) most = magnitude2(load(tok), most);
        const Scale sc = scale_of(s_old, warp_magnitude<BF16>(most));
        if (held && sc.s != s_old)
            for (int at = lane; at < held * (D / 16); at += 32) scale_again16(reinterpret_cast<uint4 *>(codes) + at, s_old, sc);
        for (int tok = mine; tok < n; tok += kSide) {
            // in-place values: a token is read for the last time by the lane that then writes it
            const uint4 v = tok == mine ? raw : *reinterpret_cast<const uint4 *>(x + (tok0 + tok) * a.x[which].token_stride);
            store8<BF16>(v, sc, codes + static_cast<int64_t>(held + tok) * D + 8 * piece,
                         values ? values + ((tok0 + tok) * a.kv_heads + head) * D + 8 * piece : nullptr);
        }
        if (lane == 0) *scale = sc.s;
        lo += n;
    }
}

using Kernel = void (*)(AppendArgs);

}  // namespace

pd_status launch_kv_append(const AppendArgs &a, bool bf16, cudaStream_t stream) {
    const int page = 1 << a.page_log2;
    const bool few = a.n_tokens <= static_cast<int64_t>(kFewTokens) * a.n_seqs;
    cudaLaunchConfig_t cfg = {};
    Kernel kernel;
    if (few) {
        kernel = a.head_dim == 128 ? (bf16 ? append_tokens_kernel<128, true> : append_tokens_kernel<128, false>)
                                   : (bf16 ? append_tokens_kernel<64, true> : append_tokens_kernel<64, false>);
        cfg.gridDim = dim3(static_cast<unsigned>(a.n_seqs), static_cast<unsigned>((2 * a.kv_heads + kTokenWarps - 1) / kTokenWarps));
        cfg.blockDim = dim3(kTokenWarps * 32);
    } else {
        kernel = a.head_dim == 128 ? (bf16 ? append_pages_kernel<128, true> : append_pages_kernel<128, false>)
                                   : (bf16 ? append_pages_kernel<64, true> : append_pages_kernel<64, false>);
        cfg.gridDim = dim3(static_cast<unsigned>(a.n_tokens / page + 2 * a.n_seqs), static_cast<unsigned>(a.kv_heads), 2);
        cfg.blockDim = dim3(static_cast<unsigned>(max(32, page * a.head_dim / (8 * kVecs))));
    }
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
