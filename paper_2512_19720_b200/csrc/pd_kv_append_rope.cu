// Rotating queries and keys and writing keys and values into the 8-bit paged cache.
//
// Rotation as in pd_rotate.cuh, codes and scales as in pd_kv_append; a rotated key is quantised from binary32, without a rounding to 16
// bits between.  Bound by memory: a query 2 bytes in and out, a key or value 2 bytes in and 1 out (3 with the values handed back).
//
// Measured: 64 sequences of one token, 64 and 8 heads 4.4 us; 2048 tokens of 4 prompts, 32 and 32 heads of 128 35 us (117 MB: 18); 9009 tokens,
// 64 and 8 heads 88 us (389 MB: 59).  What bounds the pages is instruction issue beside latency: a value takes 18 instructions, angles
// among them, and the registers (angles, values under way and at hand) leave room for 16 warps an SM; half of the registers spill (52 us).
//
// Three kinds of blocks in one grid:
//   few    : sequences with at most kFew new tokens, a warp for the keys or values of a head with all of its tokens in registers; the
//            block computes the angles of the tokens together
//   pages  : longer pieces, a page (two items of 16 values a thread) walks over several heads, so that the angles, which
//            stay in registers, are computed once for all of them; the next head's values are on their way while this one's largest
//            magnitude is found
//   queries: a token of all query heads each, where they are few; many of them have a launch of their own
// A sequence is in the hands of the first or the second kind by its own length, whatever the others of the call are.
#include <type_traits>

#include "pd_kv_quant.cuh"
#include "pd_rotate.cuh"

namespace pd {
namespace {

// Values of queries from which on they get a launch of their own, where more of them are under way; below, the second launch's start costs more.
// In a graph, 4 prompts, heads of 128, us with a launch of their own / without, at 0.5, 0.7, 1.0, 1.5 and 3.0 times the bound: 64 heads on 8
// 23.2 / 22.1, 33.6 / 31.8, 43.2 / 43.8, 60.7 / 64.1, 107 / 119; 32 on 32 at 0.5, 0.75, 1.0 and 1.5: 59.9 / 56.1, 82.4 / 81.6, 105.6 / 105.5, 151 / 153; 32 on 8,
// where the pages take less of the time, even at 0.5: 33.5 / 34.4, at 1.0 64.1 / 69.2.
constexpr int64_t kManyQueries = 1 << 25;
constexpr int kFew = 8;  // tokens: as many as two items a lane hold at head_dim 128

// 16 values to their codes and, unless nullptr, to the values that those stand for; at0 and at1 as in Item
template <bool BF16>
__device__ __forceinline__ void quantise16(const float (&x)[16], const Scale &sc, int8_t *codes, uint16_t *values, int at0, int at1) {
    float f[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) f[k] = __fadd_rn(__fmul_rn(x[k], sc.inv), kShift);
#pragma unroll
    for (int p = 0; p < 2; ++p)
        *reinterpret_cast<uint2 *>(codes + (p ? at1 : at0)) = make_uint2(low_bytes(f[8 * p], f[8 * p + 1], f[8 * p + 2], f[8 * p + 3]) & sc.keep,
                                                                         low_bytes(f[8 * p + 4], f[8 * p + 5], f[8 * p + 6], f[8 * p + 7]) & sc.keep);
    if (values) {
#pragma unroll
        for (int k = 0; k < 16; ++k) f[k] = (f[k] - kShift) * sc.s;
        store16<BF16>(values, at0, at1, f);
    }
}
__device__ __forceinline__ float magnitude16(const float (&x)[16]) {
    float m[4] = {fabsf(x[0]), fabsf(x[1]), fabsf(x[2]), fabsf(x[3])};
#pragma unroll
    for (int k = 4; k < 16; ++k) m[k & 3] = max_nan(m[k & 3], fabsf(x[k]));
    return max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3]));
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}

// The last sequence whose key(b) is not above `id`, by every warp for itself, 32 candidates a round.
template <typename Key>
__device__ __forceinline__ int last_at_or_before(int n, int id, Key key) {
    const int lane = threadIdx.x & 31;
    int b = 0, left = n;
    while (left > 1) {
        const int step = (left + 31) / 32;
        const unsigned m = __ballot_sync(0xffffffffu, lane * step < left && key(min(b + lane * step, n - 1)) <= id);
        const int src = m ? 31 - __clz(m) : 0;
        b += src * step;
        left = min(step, left - src * step);
    }
    return b;
}

// A token's queries; rows that no sequence claims stay as they are.
template <int D, bool BF16, bool INTERLEAVED>
__device__ __forceinline__ void turn_queries(const AppendRopeArgs &args, int token, float2 *cs) {
    const AppendArgs &a = args.a;
    const HeadsView x[2] = {args.q, {}}, out[2] = {args.q_out, {}};
    const int heads[2] = {args.q_heads, 0};
    turn_token<D, BF16, INTERLEAVED>(x, out, heads, token, args.r, cs, a.status, [&](int &place) {
        const int b = last_at_or_before(a.n_seqs, token, [&](int i) { return __ldg(a.cu_seqlens + i); });
        const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1);
        place = __ldg(a.seq_lens + b) - last + token;
        return token >= first && token < last;
    });
}

struct Grid {
    int few, queries, head_chunks, chunk_heads;  // blocks of the first two kinds; heads that a page block walks over
    bool by_tokens;                              // how sequences are told from a page block's number
    int pages_first;                             // so many page blocks stand before the queries': all where long pieces are likely, or none
};

// page 64 with heads of 64 and 128: 128 and 256 threads; a block has as many heads' worth of them as fit
__host__ __device__ constexpr int sub_threads(int D, int page) { return page * D / 32; }

template <int D, bool BF16, bool INTERLEAVED, int THREADS, bool QUERIES>
__global__ void __launch_bounds__(THREADS, 512 / THREADS) append_rope_kernel(const AppendRopeArgs args, const Grid grid) {
    constexpr int kItems = D / 16;  // of a head
    const AppendArgs &a = args.a;
    const Rotation &r = args.r;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ float2 cs[kFew * (D / 2)];
    __shared__ float red[2][16];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the previous kernel drains
    int id = blockIdx.x;

    if (id < grid.few) {
        // ------------------------------------------------------------ a sequence with few new tokens: a warp for the keys or values of a head
        const int warps = blockDim.x >> 5, per_seq = (2 * a.kv_heads + warps - 1) / warps;
        const int b = id / per_seq, unit = (id - b * per_seq) * warps + warp, which = unit & 1, head = unit >> 1;
        const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1), len = __ldg(a.seq_lens + b), n = last - first;
        if (bad_lengths(a, first, last, len)) {
            if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
            return;
        }
        if (n == 0 || n > kFew) return;
        const int pos0 = len - n, page = 1 << a.page_log2;
        constexpr int kSide = 32 / kItems, kRounds = kFew / kSide;  // tokens side by side
        const int j = lane % kItems, mine = lane / kItems;
        const bool there = head < a.kv_heads;
        const Item<INTERLEAVED> item(j, which == 0 ? r.pairs : 0);
        Raw16 raw[kRounds];
        const uint16_t *x = static_cast<const uint16_t *>(a.x[which].ptr) + head * a.x[which].head_stride;
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            if (there && mine + i * kSide < n) raw[i] = load16(x + static_cast<int64_t>(first + mine + i * kSide) * a.x[which].token_stride, item.at0, item.at1);
        for (int i = threadIdx.x; i < n * r.pairs; i += blockDim.x) {
            const int t = i / r.pairs, p = i - t * r.pairs;
            cs[t * (D / 2) + p] = angle(position_of(r, p, first + t, pos0 + t, a.status), __ldg(r.inv_freq + p), r.direction);
        }
        __syncthreads();
        if (!there) return;
        float f[kRounds][16], most[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            most[i] = 0.f;
            if (mine + i * kSide < n) {
                unpack16<BF16>(raw[i], f[i]);
                if (item.turns) {
                    float2 t[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] = cs[(mine + i * kSide) * (D / 2) + 8 * j + k];
                    turn16<INTERLEAVED>(f[i], t);
                }
                most[i] = magnitude16(f[i]);
            }
        }
        uint16_t *values = static_cast<uint16_t *>(a.values[which]);
        for (int t0 = 0; t0 < n;) {  // page after page
            const int lo = pos0 + t0, pi = lo >> a.page_log2, held = lo & (page - 1), t1 = min(n, t0 + page - held);
            const int64_t pid = pi < a.table_width ? __ldg(a.block_table + b * a.table_stride + pi) : -1;
            if (pid < 0 || pid >= a.n_pages) {
                if (lane == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
                return;
            }
            int8_t *codes = a.pages[which].codes + ((pid * a.kv_heads + head) << a.page_log2) * D;
            float *scale = a.pages[which].scale + pid * a.kv_heads + head;
            const float s_old = held ? *scale : 0.f;
            float amax = 0.f;
#pragma unroll
            for (int i = 0; i < kRounds; ++i)
                if (mine + i * kSide >= t0 && mine + i * kSide < t1) amax = max_nan(amax, most[i]);
            const Scale sc = scale_of(s_old, warp_max(amax));
            if (held && sc.s != s_old)
                for (int at = lane; at < held * (D / 16); at += 32) scale_again16(reinterpret_cast<uint4 *>(codes) + at, s_old, sc);
#pragma unroll
            for (int i = 0; i < kRounds; ++i) {
                const int t = mine + i * kSide;
                if (t >= t0 && t < t1)
                    quantise16<BF16>(f[i], sc, codes + (held + t - t0) * D, values ? values + (static_cast<int64_t>(first + t) * a.kv_heads + head) * D : nullptr, item.at0, item.at1);
            }
            if (lane == 0) *scale = sc.s;
            t0 = t1;
        }
        return;
    }
    id -= grid.few;
    if (QUERIES && id >= grid.pages_first) {
        id -= grid.pages_first;
        if (id < grid.queries) {
            turn_queries<D, BF16, INTERLEAVED>(args, id, cs);
            return;
        }
        id -= grid.queries;
    }
    {
        // ------------------------------------------------------------ a page of a longer piece: keys or values of several heads
        const int page = 1 << a.page_log2, sub_size = sub_threads(D, page), subs = blockDim.x / sub_size;
        const int sub = threadIdx.x / sub_size, t = threadIdx.x - sub * sub_size;
        const int chunk = id % grid.head_chunks, which = (id / grid.head_chunks) & 1, slot = id / grid.head_chunks >> 1;
        // Sequence b's pages are the ids from cu[b] / page + 2 b on, or, where there are more sequences than could have a long piece, from
        // cu[b] (1 / page + 2 / 9) on: n tokens, 9 at least, touch (n - 1) / page + 2 pages at most, never more than ids before the next sequence's.
        auto first_id = [&](int i) {
            const int64_t at = min(max(__ldg(a.cu_seqlens + i), 0), a.n_tokens);
            return static_cast<int>(grid.by_tokens ? (at * (2 * page + kFew + 1) >> a.page_log2) / (kFew + 1) : (at >> a.page_log2) + 2 * static_cast<int64_t>(i));
        };
        const int b = last_at_or_before(a.n_seqs, slot, first_id);
        const int first = __ldg(a.cu_seqlens + b), last = __ldg(a.cu_seqlens + b + 1), len = __ldg(a.seq_lens + b);
        if (bad_lengths(a, first, last, len) || last - first <= kFew) return;  // reported, and taken, by the first kind
        const int pos0 = len - (last - first);
        const int pi = (pos0 >> a.page_log2) + slot - first_id(b);
        const int64_t page_start = static_cast<int64_t>(pi) << a.page_log2;
        const int lo = static_cast<int>(max(static_cast<int64_t>(pos0), page_start));
        const int hi = static_cast<int>(min(static_cast<int64_t>(len), page_start + page));
        if (pi < 0 || lo >= hi) return;
        const int64_t pid = pi < a.table_width ? __ldg(a.block_table + b * a.table_stride + pi) : -1;
        if (pid < 0 || pid >= a.n_pages) {
            if (threadIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
            return;
        }
        const int n = hi - lo, held = lo & (page - 1), j = t % kItems, tok = t / kItems, far = page / 2;  // the thread's tokens: tok and tok + far
        const int64_t tok0 = first + (lo - pos0);
        const Item<INTERLEAVED> item(j, which == 0 ? r.pairs : 0);
        const int head_end = min(a.kv_heads, (chunk + 1) * grid.chunk_heads);
        int head = chunk * grid.chunk_heads + sub;
        const bool has[2] = {tok < n, tok + far < n};
        const uint16_t *x = static_cast<const uint16_t *>(a.x[which].ptr) + (tok0 + tok) * a.x[which].token_stride;
        const int64_t x_far = far * a.x[which].token_stride;
        Raw16 raw[2];
        auto load = [&](int h) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (has[i] && h < head_end) raw[i] = load16(x + h * a.x[which].head_stride + i * x_far, item.at0, item.at1);
        };
        load(head);
        float2 turn[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (has[i] && item.turns) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    turn[i][k] = angle(position_of(r, 8 * j + k, tok0 + tok + i * far, lo + tok + i * far, a.status), __ldg(r.inv_freq + 8 * j + k), r.direction);
            }
        uint16_t *values = static_cast<uint16_t *>(a.values[which]);
        for (int round = 0; chunk * grid.chunk_heads + round * subs < head_end; ++round, head += subs) {  // all threads of the block go through it
            const bool there = head < head_end;
            int8_t *codes = a.pages[which].codes + ((pid * a.kv_heads + head) << a.page_log2) * D;
            float *scale = a.pages[which].scale + pid * a.kv_heads + head;
            const float s_old = there && held ? *scale : 0.f;
            float f[2][16], amax = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (has[i] && there) {
                    unpack16<BF16>(raw[i], f[i]);
                    if (item.turns) turn16<INTERLEAVED>(f[i], turn[i]);
                    amax = max_nan(amax, magnitude16(f[i]));
                }
            load(head + subs);
            amax = warp_max(amax);
            if (lane == 0) red[round & 1][warp] = amax;
            __syncthreads();
            if (!there) continue;
            const int w0 = sub * sub_size / 32;
            amax = red[round & 1][w0];
            for (int w = 1; w < sub_size / 32; ++w) amax = max_nan(amax, red[round & 1][w0 + w]);
            const Scale sc = scale_of(s_old, amax);
            if (held && sc.s != s_old)
                for (int at = t; at < held * (D / 16); at += sub_size) scale_again16(reinterpret_cast<uint4 *>(codes) + at, s_old, sc);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (has[i])
                    quantise16<BF16>(f[i], sc, codes + (held + tok + i * far) * D,
                                     values ? values + ((tok0 + tok + i * far) * a.kv_heads + head) * D : nullptr, item.at0, item.at1);
            if (t == 0) *scale = sc.s;
        }
    }
}

// The same for many tokens, in a kernel of its own: with the registers of the one above too few values would be on their way.
constexpr int kQueryThreads = 256;
template <int D, bool BF16, bool INTERLEAVED>
__global__ void __launch_bounds__(kQueryThreads) queries_rope_kernel(const AppendRopeArgs args) {
    __shared__ float2 cs[D / 2];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    turn_queries<D, BF16, INTERLEAVED>(args, blockIdx.x, cs);
}

template <int D, bool BF16>
pd_status launch(const AppendRopeArgs &args, bool interleaved, cudaStream_t stream) {
    const AppendArgs &a = args.a;
    const int page = 1 << a.page_log2, threads = max(256, sub_threads(D, page)), subs = threads / sub_threads(D, page);
    const int warps = threads / 32;
    const int64_t few = static_cast<int64_t>(a.n_seqs) * ((2 * a.kv_heads + warps - 1) / warps);
    const bool apart = static_cast<int64_t>(a.n_tokens) * args.q_heads * D >= kManyQueries;
    Grid grid = {static_cast<int>(few), args.q_heads && !apart ? a.n_tokens : 0, 1, a.kv_heads, false, 0};
    int64_t page_blocks = 0;
    if (a.n_tokens > kFew) {
        // Longer walks compute fewer angles, more blocks fill the GPU: as long a walk as leaves four blocks for each SM
        // (2048 tokens, 32 heads of 128, us with 2, 4, 8, 16: 40, 38, 41, 50;  9009 tokens, 8 heads: 84, 88, 90, 103).
        grid.by_tokens = 2 * a.n_tokens < (kFew + 1) * 2 * static_cast<int64_t>(a.n_seqs);
        const int64_t used = a.n_tokens / page + 1;
        const int64_t slots = grid.by_tokens ? static_cast<int64_t>(a.n_tokens) * (2 * page + kFew + 1) / ((kFew + 1) * page) + 1 : used + 2 * static_cast<int64_t>(a.n_seqs);
        int64_t chunks = (4 * static_cast<int64_t>(sm_count()) + 2 * used - 1) / (2 * used);
        const int64_t most = (a.kv_heads + subs - 1) / subs;
        chunks = chunks < most ? chunks : most;
        grid.chunk_heads = static_cast<int>((most + chunks - 1) / chunks) * subs;
        grid.head_chunks = (a.kv_heads + grid.chunk_heads - 1) / grid.chunk_heads;
        if (slots * 2 * grid.head_chunks + few + a.n_tokens > INT32_MAX / 2) return PD_ERR_UNSUPPORTED_SHAPE;
        page_blocks = slots * 2 * grid.head_chunks;
        grid.pages_first = grid.by_tokens ? 0 : static_cast<int>(page_blocks);
    }
    if (few > INT32_MAX / 4) return PD_ERR_UNSUPPORTED_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid.few + grid.queries + page_blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    auto pick = [&](auto queries) {
        constexpr bool Q = decltype(queries)::value;
        return threads == 256 ? (interleaved ? append_rope_kernel<D, BF16, true, 256, Q> : append_rope_kernel<D, BF16, false, 256, Q>)
                              : (interleaved ? append_rope_kernel<D, BF16, true, 512, Q> : append_rope_kernel<D, BF16, false, 512, Q>);
    };
    const auto kernel = apart ? pick(std::false_type()) : pick(std::true_type());
    if (cudaLaunchKernelEx(&cfg, kernel, args, grid) != cudaSuccess)
        return PD_ERR_CUDA;
    if (!apart) return PD_OK;
    cfg.gridDim = dim3(static_cast<unsigned>(a.n_tokens));
    cfg.blockDim = dim3(static_cast<unsigned>(turn_threads(args.q_heads, D, kQueryThreads)));
    count_launch();
    return cuda_ok(interleaved ? cudaLaunchKernelEx(&cfg, queries_rope_kernel<D, BF16, true>, args)
                               : cudaLaunchKernelEx(&cfg, queries_rope_kernel<D, BF16, false>, args));
}

}  // namespace

pd_status launch_kv_append_rope(const AppendRopeArgs &a, bool interleaved, bool bf16, cudaStream_t stream) {
    if (a.a.head_dim == 128) return bf16 ? launch<128, true>(a, interleaved, stream) : launch<128, false>(a, interleaved, stream);
    return bf16 ? launch<64, true>(a, interleaved, stream) : launch<64, false>(a, interleaved, stream);
}

}  // namespace pd
