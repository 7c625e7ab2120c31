// Attention of single tokens over the 8-bit paged cache: out[b, h] = sum_j softmax_j(scale q[b, h] . K[j, g]) V[j, g] over the
// tokens j < seq_lens[b], K and V being codes (signed 8 bits) times the scale of their page and head.
//
// Bound by memory: every code is read once, 2 * head_dim bytes per token and key/value head, against 4 * group * head_dim
// operations.  Measured: 64 sequences, 256085 cached tokens, 64 query and 8 key/value heads of 128 (528 MB) 105 us in bursts
// (6.8 TB/s between segment changes) and 113 sustained, where the power limit takes the SM clock down to 1.74 GHz.
//
// Work.  A *segment* is the heads of one sequence that share a key/value head (up to 8 * NT of them); its tokens are cut
// into tiles of 32.  The tiles of all segments, one after another and with what a segment costs beside them, are dealt to
// the warps of the grid in equal contiguous ranges, whatever the lengths are: a long sequence is spread over many warps, a warp
// may take many short ones.  The parts of a segment that was cut are joined in two steps, the warps of a block in shared
// memory and the blocks through the workspace by the last one to arrive (nobody waits), in the order of the tiles: results
// do not depend on the schedule.
//
// Inside a warp.  Tiles are fetched with cp.async into a ring that belongs to the warp alone, so that no barrier is needed.
// In both products tokens (head dimensions) are M and the heads N.  The order of the contracted index and of the output
// rows is free, so that a thread takes 16 contiguous codes of a token per load.
// S^T = K Q^T in whole numbers: the codes go into m16n8k32 products as they are, and a query is three signed bytes a value
// (23 bits).  That is three products for 512 codes where binary16 would be two and five conversions for four codes.
// O^T = V^T P^T in binary16, m16n8k16, 256 codes a product: byte c ^ 0x80 under the upper byte 0x64 is 1024 + (c + 128),
// less 1152, exactly c.  P^T is S^T's accumulator layout transposed in 8 x 8 pieces (movmatrix).
//
// Softmax in base 2 with 32-bit statistics.  The reference maximum m of a head and the reference scale r of V move only
// when a score passes m by more than 8 or a page's scale leaves [r / 8, 8 r]: P is rounded to binary16 as
// 2^(s - m) * (page scale / r) <= 2^11, so that its relative precision does not depend on how stale m and r are, and O
// needs no multiplication at most tiles.  r falls with the page scales as far as O, which is kept in units of r, stays in range.
#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

constexpr int kTile = 32;    // tokens of a tile: a multiple of 16, so that a 16-token product lies in one page
constexpr int kMaxGrid = 1024;
constexpr int kMaxRows = 16;    // heads of a segment
constexpr size_t kCounterBytes = kMaxGrid * kMaxRows * 4;  // for each block and row: parts of the segment that goes on behind the block
constexpr float kLog2e = 1.4426950408889634f;
// A sum that starts from the bits of 1.5 * 2^2 is, read as binary32, that number and 2^-21 of the sum (below 2^22 in magnitude).
constexpr float kShift = 6.f;
constexpr int kShiftBits = 0x40C00000;
constexpr float kMaxLead = 8.f;         // how far (base-2 exponent) a score may pass the reference maximum
constexpr float kSmallestScale = 0x1p-120f;  // a page of V whose scale is below it counts as zeros; so 1 / r is finite
constexpr float kPart = 0x1p-20f;            // parts of a row are kept times this until they are joined, so that sums of large values stay in range
constexpr float kMostOutput = 0x1p100f;      // O, in units of r, stays below about this where r falls; what r does not follow is 2^-100 of O

template <int D, int NT>
struct CacheShape {
    static constexpr int kRows = 8 * NT;                        // heads of a segment
    static constexpr int kWarps = NT == 1 ? 8 : 6;              // what shared memory has room for
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kStage = 2 * kTile * D;                // K, then V
    static constexpr int kRing = kStages * kStage;
    static constexpr int kMeta = kStages * 16;                  // per stage: scales of K and V for the two 16-token halves
    static constexpr int kWarp = kRing + kMeta;
    static constexpr int kPiece = (kRows * D + 2 * kRows) * 4;  // a partial result: O, then m, then l
    // A warp's range starts and ends inside a segment.  The first partial result has a place of its own (the ring goes on
    // being used), the last one takes the ring's.
    static constexpr int kTotal = kWarps * (kWarp + kPiece);
    static_assert(kPiece <= kRing && kWarp % 16 == 0 && kPiece % 16 == 0, "layout");
    static_assert(2 * kThreads * 4 <= kWarps * kPiece && kTotal <= 226 * 1024, "shared memory");
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void cp_async16(void *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// 16 tokens x 32 dimensions of codes against 32 dimensions x 8 heads of signed bytes
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// bytes (0, 1) or (2, 3) of w (each a code ^ 0x80) as two binary16 codes
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return hadd2_u32(prmt(w, 0x64646464u, 0x4140), 0xE480E480u); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return hadd2_u32(prmt(w, 0x64646464u, 0x4342), 0xE480E480u); }

// Work is dealt in units: a segment's tiles and, before them, what its beginning and end cost (measured in tiles).
// In us with 1 / 2 / 4, in short bursts: 64 long sequences with 32 heads on 32 111 / 104 / 106, with 64 on 8 106 / 103 / 102; 96 sequences of
// 20 to 300 tokens with 64 on 8 23.8 / 23.8 / 25.3.
constexpr int kSegmentCost = 2;
// A warp gets so many units at least: with fewer, more parts are to be joined than the shorter ranges save (one token, 64 query
// and 8 key/value heads, 4000 cached tokens: 12.6 us with 1, 13.7 with 2, 15.3 with 3; 16 heads on one, 3 x 16197 tokens: 25.7, 24.1, 20.5).
constexpr int kMinUnits = 2;
__device__ __forceinline__ int tiles_of(int len) { return len > 0 ? (len + kTile - 1) / kTile : 1; }

// A partial result of a segment in a warp's shared memory: which one, and where it starts in the order of all tiles.
struct Piece {
    int first;  // the unit of the segment's first tile; -1: none
    int tiles, b, head0, rows;
};

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(CacheShape<D, NT>::kThreads, 1) attn_cache_kernel(const CacheAttnArgs a) {
    using E = Elem<BF16>;
    using L = CacheShape<D, NT>;
    constexpr int kWarps = L::kWarps, kThreads = L::kThreads, kStages = L::kStages;
    constexpr int MT = D / 16;      // 16-row products of O^T
    constexpr int KS = D / 32;      // contraction steps of S
    constexpr int KC = D / 64;      // 16-byte pieces of a key that a thread takes
    constexpr int VB = D / 8;       // bytes of a value that a thread takes
    extern __shared__ __align__(16) unsigned char smem[];
    static_assert(L::kRows <= kMaxRows && kThreads % 32 == 0, "layout");
    // until every warp has found its first tile: where the first partial results go later
    int *scan = reinterpret_cast<int *>(smem + kWarps * L::kWarp), *scan_len = scan + kThreads;
    __shared__ int warp_sum[kWarps];
    __shared__ Piece pieces[kWarps][2];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int group = a.q_heads / a.kv_heads;
    const int chunks = (group + L::kRows - 1) / L::kRows;
    const int per_seq = a.kv_heads * chunks;  // segments of a sequence
    const int page = 1 << a.page_log2;
    const int64_t room = static_cast<int64_t>(a.table_width) << a.page_log2;

    auto length = [&](int b) {
        const int n = __ldg(a.seq_lens + b);
        return n < 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(n), room));
    };

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the previous kernel drains
    // ---------------------------------------------------------------- tiles before each thread's share of the sequences
    const int share = (a.n_seqs + kThreads - 1) / kThreads;
    int sum = 0, first_len = 0;
    for (int b = threadIdx.x * share; b < min(a.n_seqs, static_cast<int>(threadIdx.x + 1) * share); ++b) {
        const int raw = __ldg(a.seq_lens + b), n = length(b);
        if (blockIdx.x == 0 && raw != n) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        if (b == static_cast<int>(threadIdx.x) * share) first_len = n;
        sum += tiles_of(n) + kSegmentCost;
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    if (lane == 31) warp_sum[warp] = incl;
    if (threadIdx.x < 2 * kWarps) (&pieces[0][0])[threadIdx.x].first = -1;
    __syncthreads();
    int before = 0, total_seq = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += warp_sum[w];
        total_seq += warp_sum[w];
    }
    scan[threadIdx.x] = before + incl - sum;
    scan_len[threadIdx.x] = first_len;
    __syncthreads();
    const int total = total_seq * per_seq;  // the host has seen to it that 32 bits are enough
    const int n_ctas = max(1, min(static_cast<int>(gridDim.x), total / (kWarps * kMinUnits)));
    if (static_cast<int>(blockIdx.x) >= n_ctas) return;
    const int quota = total / n_ctas, more = total - quota * n_ctas;  // the first `more` blocks take a tile more
    auto cta_first = [&](int c) { return c * quota + min(c, more); };
    auto cta_of = [&](int tile) { return tile < more * (quota + 1) ? tile / (quota + 1) : more + (tile - more * (quota + 1)) / quota; };
    const int cta0 = cta_first(blockIdx.x), cta1 = cta_first(blockIdx.x + 1);
    const int warp_quota = (cta1 - cta0) / kWarps, warp_more = (cta1 - cta0) % kWarps;
    const int range0 = cta0 + warp * warp_quota + min(warp, warp_more), range1 = range0 + warp_quota + (warp < warp_more ? 1 : 0);

    // Finds the segment of a unit: sequence b, segment s of it, tile i of the segment (negative: what the segment costs beside its tiles).
    auto locate = [&](int at, int &b, int &s, int &i, int &len) {
        const int seq_tile = at / per_seq;  // a share starts at or before the tile where it starts at or before this
        constexpr int kStep = kThreads / 32;
        int lo = (31 - __clz(__ballot_sync(0xffffffffu, scan[lane * kStep] <= seq_tile))) * kStep;
        lo += 31 - __clz(__ballot_sync(0xffffffffu, lane < kStep && scan[lo + min(lane, kStep - 1)] <= seq_tile));
        b = lo * share;
        len = scan_len[lo];
        int rest = at - scan[lo] * per_seq;
        while (rest >= (tiles_of(len) + kSegmentCost) * per_seq && b + 1 < a.n_seqs) {
            rest -= (tiles_of(len) + kSegmentCost) * per_seq;
            len = length(++b);
        }
        s = rest / (tiles_of(len) + kSegmentCost);
        i = rest - s * (tiles_of(len) + kSegmentCost) - kSegmentCost;
    };

    unsigned char *ring = smem + warp * L::kWarp;
    auto piece_at = [&](int w, int slot) { return reinterpret_cast<float *>(slot == 0 ? smem + kWarps * L::kWarp + w * L::kPiece : smem + w * L::kWarp); };
    float4 *meta = reinterpret_cast<float4 *>(ring + L::kRing);

    // ---------------------------------------------------------------- the warp's tiles
    const float lscale = a.scale * kLog2e;
    int b = 0, s = 0, i0 = 0, len = 0;
    int at = range0;
    if (at < range1) locate(at, b, s, i0, len);
    __syncthreads();
    while (at < range1) {
        const int n_tiles = tiles_of(len), first_unit = at - i0;
        const int kvh = s / chunks, chunk = s - kvh * chunks;
        const int head0 = kvh * group + chunk * L::kRows;
        const int rows = min(L::kRows, group - chunk * L::kRows);
        const int i1 = min(n_tiles, range1 - first_unit);
        i0 = max(i0, 0);
        if (i1 <= i0) break;  // of this segment only the units before its tiles

        // lane j holds page and scales of tile base + j (two pages where a page is half a tile)
        int base = i0 - 32;
        int64_t pid[2] = {0, 0};
        float sk[2] = {0.f, 0.f}, sv[2] = {0.f, 0.f};
        auto issue = [&](int i) {
            if (i < i1) {
                if (i - base >= 32) {
                    base = i;
                    const int mine = i + lane;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int64_t tok = static_cast<int64_t>(mine) * kTile + 16 * k;
                        pid[k] = 0, sk[k] = 0.f, sv[k] = 0.f;
                        if (mine < i1 && tok < len) {
                            if (k == 1 && page > 16) {
                                pid[k] = pid[0], sk[k] = sk[0], sv[k] = sv[0];
                            } else {
                                const int64_t p = __ldg(a.block_table + b * a.table_stride + (tok >> a.page_log2));
                                if (p < 0 || p >= a.n_pages) {
                                    latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
                                } else {
                                    pid[k] = p;
                                    sk[k] = a.pages[0].scale[p * a.kv_heads + kvh];
                                    sv[k] = a.pages[1].scale[p * a.kv_heads + kvh];
                                }
                            }
                        }
                    }
                }
                const int st = (i - i0) % kStages;
                const int src = i - base;
                unsigned char *kdst = ring + st * L::kStage, *vdst = kdst + kTile * D;
                constexpr int kPieces = D / 16, kRowsPer = 32 / kPieces;
                const int c = lane % kPieces;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int64_t p = __shfl_sync(0xffffffffu, pid[half], src);
                    const int64_t tok = static_cast<int64_t>(i) * kTile + 16 * half;
                    const int64_t off = (((p * a.kv_heads + kvh) << a.page_log2) + (tok & (page - 1))) * D;
#pragma unroll
                    for (int k = 0; k < 16 / kRowsPer; ++k) {
                        const int r = k * kRowsPer + lane / kPieces, row = 16 * half + r;
                        if (tok + r < len) {
                            const int ck = D == 128 ? c ^ ((row & 1) * 4) : c;
                            const int cv = D == 128 ? c ^ (row & 6) : c;
                            cp_async16(kdst + row * D + ck * 16, a.pages[0].codes + off + r * D + c * 16);
                            cp_async16(vdst + row * D + cv * 16, a.pages[1].codes + off + r * D + c * 16);
                        }
                    }
                }
                if (lane == src)  // after the copies: the scales may still be on their way
                    meta[st] = make_float4(sk[0], sk[1], sv[0] < kSmallestScale ? 0.f : sv[0], sv[1] < kSmallestScale ? 0.f : sv[1]);
            }
            cp_async_commit();
        };
        __syncwarp();
        if (len > 0) {
#pragma unroll
            for (int k = 0; k < kStages - 1; ++k) issue(i0 + k);
        }
        float o[MT][NT][4];
        float m[NT][2], mu[NT][2], l[NT][2], qs[NT][2];
        uint32_t qf[KS][NT][3][2];
        float ref = 0.f, inv_ref = 0.f, ref_top = 0.f;  // the reference scale of V, its reciprocal, and the largest that O was summed with
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][n][k] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // The head's query as whole numbers of 23 bits, in three signed bytes: multiples of 2^-21 of the power of two 2^e
            // below its largest magnitude.  That is exact for values down to 2^-11 of the largest (2^-14 in bfloat16); smaller ones
            // are off by up to 2^-22 of the largest, four times what binary32 loses of a sum that the largest takes part in.
            const int r = n * 8 + g;
            float x[KC][16], amax = 0.f;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                uint4 w[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (r < rows) {
                    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q.ptr) + b * a.q.token_stride +
                                                                     (head0 + r) * a.q.head_stride + 16 * (t + 4 * c));
                    w[0] = p[0], w[1] = p[1];
                }
                const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 f = E::to_float2(u[k]);
                    x[c][2 * k] = f.x, x[c][2 * k + 1] = f.y;
                    amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            // 2^(21 - e) for every e that binary32 has, in two factors
            const int e = min(max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -126), 127), half = (21 - e) >> 1;
            const float down0 = __uint_as_float(static_cast<uint32_t>(127 + half) << 23);
            const float down1 = __uint_as_float(static_cast<uint32_t>(127 + 21 - e - half) << 23), up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
            float bad = 0.f;  // NaN where the query has an infinity or a NaN
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t byte[3] = {0u, 0u, 0u};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        bad = fmaf(x[c][4 * k + i], 0.f, bad);
                        int rest = __float2int_rn(x[c][4 * k + i] * down0 * down1);
#pragma unroll
                        for (int j = 0; j < 3; ++j) {
                            byte[j] |= (static_cast<uint32_t>(rest) & 0xffu) << (8 * i);
                            rest = (rest >> 8) + ((rest >> 7) & 1);  // less the signed byte
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 3; ++j) qf[c * 2 + k / 2][n][j][k & 1] = byte[j];
                }
            bad += __shfl_xor_sync(0xffffffffu, bad, 1);
            bad += __shfl_xor_sync(0xffffffffu, bad, 2);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                qs[n][k] = lscale * __shfl_sync(0xffffffffu, up + bad, (2 * t + k) * 4);
                m[n][k] = -INFINITY, mu[n][k] = 0.f, l[n][k] = 0.f;
            }
        }

        if (len > 0) {
            // The two 16-token halves of a tile share r: where they are pages whose scales are more than 8 apart, the tile is gone
            // through twice, once for each half.
            int half = 0;  // 0: both at once, 1 and 2: one of them
            for (int i = i0; i < i1; half == 1 ? ++half : (half = 0, ++i)) {
                if (half < 2) {
                    cp_async_wait<kStages - 2>();
                    __syncwarp();
                    issue(i + kStages - 1);
                }
                const int st = (i - i0) % kStages;
                const unsigned char *ks = ring + st * L::kStage, *vs = ks + kTile * D;
                const float4 sc = meta[st];
                if (half == 0 && fmaxf(sc.z, sc.w) > 8.f * fminf(sc.z, sc.w) && fminf(sc.z, sc.w) > 0.f) half = 1;
                const int rest = static_cast<int>(min(len - static_cast<int64_t>(i) * kTile, static_cast<int64_t>(kTile)));  // tokens of the tile
                const int end[2] = {half == 2 ? 0 : rest, half == 1 ? 0 : rest};

                // S^T = K Q^T
                float acc[2][NT][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    int part[NT][3][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 3; ++j)
#pragma unroll
                            for (int k = 0; k < 4; ++k) part[n][j][k] = kShiftBits;
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        const int row = 16 * h + g, piece = D == 128 ? (t + 4 * c) ^ ((row & 1) * 4) : t;
                        const uint4 lo = *reinterpret_cast<const uint4 *>(ks + row * D + piece * 16);
                        const uint4 hi = *reinterpret_cast<const uint4 *>(ks + (row + 8) * D + piece * 16);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < 3; ++j) {
                                mma_s8(part[n][j], lo.x, hi.x, lo.y, hi.y, qf[c * 2][n][j][0], qf[c * 2][n][j][1]);
                                mma_s8(part[n][j], lo.z, hi.z, lo.w, hi.w, qf[c * 2 + 1][n][j][0], qf[c * 2 + 1][n][j][1]);
                            }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float f[3];
#pragma unroll
                            for (int j = 0; j < 3; ++j) f[j] = __int_as_float(part[n][j][k]) - kShift;
                            acc[h][n][k] = fmaf(f[2], 65536.f, fmaf(f[1], 256.f, f[0]));
                        }
                }
                // scores in base 2; places past the end of the sequence or of the other half are chosen away, whatever they hold
                bool lead = false;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float f = (h == 0 ? sc.x : sc.y) * qs[n][k & 1];
                            acc[h][n][k] = 16 * h + g + 8 * (k >> 1) < end[h] ? acc[h][n][k] * f : -INFINITY;
                            lead |= acc[h][n][k] > __fadd_rd(m[n][k & 1], kMaxLead);  // rounded down: P's range is bounded for large scores too
                        }
                const float sv[2] = {half == 2 ? 0.f : sc.z, half == 1 ? 0.f : sc.w}, sv_hi = fmaxf(sv[0], sv[1]);
                const bool move_ref = sv_hi > 8.f * ref || (sv_hi < 0.125f * ref && sv_hi > 0.f);
                if (__any_sync(0xffffffffu, lead) || move_ref) {
                    float factor[NT][2];  // for O
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float top = fmaxf(fmaxf(acc[0][n][k], acc[0][n][k + 2]), fmaxf(acc[1][n][k], acc[1][n][k + 2]));
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            top = fmaxf(top, m[n][k]);
                            const float mu_new = top == -INFINITY ? 0.f : top;
                            factor[n][k] = exp2_approx(m[n][k] - mu_new);  // 0 from -infinity on
                            l[n][k] *= factor[n][k];
                            m[n][k] = top, mu[n][k] = mu_new;
                        }
                    if (move_ref) {
                        float step = ref / sv_hi;
                        if (sv_hi < ref_top * 0x1p-60f) {
                            // far below the largest r that O was summed with: r follows as long as O stays in range
                            float most = 0.f;
#pragma unroll
                            for (int j = 0; j < MT; ++j)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int k = 0; k < 4; ++k)
                                        if (n * 8 + 2 * t + (k & 1) < rows) most = fmaxf(most, fabsf(o[j][n][k] * factor[n][k & 1]));
#pragma unroll
                            for (int d = 1; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
                            step = most > 0.f ? fmaxf(fminf(fminf(step, kMostOutput / most), 0x1p120f), 1.f) : 1.f;  // finite, however little is left of O
                            ref = most > 0.f ? fmaxf(sv_hi, ref / step) : sv_hi;
                            if (most == 0.f) ref_top = 0.f;
                        } else {
                            ref = sv_hi;
                        }
                        ref_top = fmaxf(ref_top, ref);
                        inv_ref = __frcp_rn(ref);
#pragma unroll
                        for (int n = 0; n < NT; ++n) factor[n][0] *= step, factor[n][1] *= step;
                    }
#pragma unroll
                    for (int j = 0; j < MT; ++j)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[j][n][k] *= factor[n][k & 1];
                }
                const float rv[2] = {sv[0] * inv_ref, sv[1] * inv_ref};
                uint32_t pf[2][NT][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float p[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            p[k] = exp2_approx(acc[h][n][k] - mu[n][k & 1]);
                            l[n][k & 1] += p[k];
                            p[k] *= rv[h];
                        }
                        pf[h][n][0] = movmatrix_trans(Elem<false>::from_float2(p[0], p[1]));
                        pf[h][n][1] = movmatrix_trans(Elem<false>::from_float2(p[2], p[3]));
                    }
                // O^T += V^T P^T
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t w[4][VB / 4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = 16 * h + 2 * t + (k & 1) + 8 * (k >> 1);
                        if (D == 128) {
                            const uint4 x = *reinterpret_cast<const uint4 *>(vs + row * D + (g ^ (row & 6)) * 16);
                            w[k][0] = x.x ^ 0x80808080u, w[k][1] = x.y ^ 0x80808080u;
                            w[k][VB / 4 - 2] = x.z ^ 0x80808080u, w[k][VB / 4 - 1] = x.w ^ 0x80808080u;
                        } else {
                            const uint2 x = *reinterpret_cast<const uint2 *>(vs + row * D + g * 8);
                            w[k][0] = x.x ^ 0x80808080u, w[k][1] = x.y ^ 0x80808080u;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < VB / 4; ++j) {
                        const uint32_t ab0 = prmt(w[0][j], w[1][j], 0x5140), ab1 = prmt(w[0][j], w[1][j], 0x7362);
                        const uint32_t cd0 = prmt(w[2][j], w[3][j], 0x5140), cd1 = prmt(w[2][j], w[3][j], 0x7362);
                        const uint32_t x0 = codes_lo(ab0), x1 = codes_hi(ab0), x2 = codes_lo(cd0), x3 = codes_hi(cd0);
                        const uint32_t y0 = codes_lo(ab1), y1 = codes_hi(ab1), y2 = codes_lo(cd1), y3 = codes_hi(cd1);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            Elem<false>::mma16816(o[2 * j][n], x0, x1, x2, x3, pf[h][n][0], pf[h][n][1]);
                            Elem<false>::mma16816(o[2 * j + 1][n], y0, y1, y2, y3, pf[h][n][0], pf[h][n][1]);
                        }
                    }
                }
            }
            cp_async_wait<0>();
            __syncwarp();
        }

        // ------------------------------------------------ the segment's end in this warp: thread (g, t) holds dimensions VB * g .. of heads 2t, 2t + 1
        const bool whole = i0 == 0 && i1 == n_tiles;
        const int slot = i0 > 0 ? 0 : 1;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][k] += __shfl_xor_sync(0xffffffffu, l[n][k], d);
                const int r = n * 8 + 2 * t + k;
                if (r < rows) {
                    if (whole) {
                        const float f = l[n][k] == 0.f ? 0.f : ref / l[n][k];
                        uint32_t w[VB / 2];
#pragma unroll
                        for (int j = 0; j < VB / 2; ++j) w[j] = E::from_float2(o[j][n][k] * f, o[j][n][k + 2] * f);
                        uint4 *p = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + b * a.out.token_stride +
                                                             (head0 + r) * a.out.head_stride + VB * g);
#pragma unroll
                        for (int j = 0; j < VB / 8; ++j) p[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                    }
                }
            }
        if (!whole) {
            float *po = piece_at(warp, slot), *pm = po + L::kRows * D, *pl = pm + L::kRows;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int r = n * 8 + 2 * t + k;
                    if (r < rows) {
                        if (g == 0) pm[r] = m[n][k], pl[r] = l[n][k];
#pragma unroll
                        for (int j = 0; j < VB / 2; ++j)
                            *reinterpret_cast<float2 *>(po + r * D + VB * g + 2 * j) = make_float2(o[j][n][k] * kPart * ref, o[j][n][k + 2] * kPart * ref);
                    }
                }
            if (lane == 0) pieces[warp][slot] = {first_unit, n_tiles, b, head0, rows};
        }
        if (i1 < n_tiles) break;
        at = first_unit + n_tiles;
        i0 = -kSegmentCost;
        if (at < range1 && ++s == per_seq) {
            s = 0;
            len = length(++b);
        }
    }
    __syncthreads();

    // ---------------------------------------------------------------- the block's parts of each segment, in the order of the tiles
    // A warp takes a row at a time, a lane D / 32 of its outputs.  Rows of a segment that other blocks hold parts of are joined
    // by the last block that has written its own.
    constexpr int kPartial = L::kPiece / 4;
    constexpr int V = D / 32;
    struct Sum {
        float top, l, o[V];
    };
    auto weight = [](float m, float top) { return m == -INFINITY ? 0.f : exp2_approx(m - top); };
    auto load_o = [](const float *p, float (&o)[V], bool global) {
        if (V == 4) {
            const float4 x = global ? __ldcg(reinterpret_cast<const float4 *>(p)) : *reinterpret_cast<const float4 *>(p);
            o[0] = x.x, o[1] = x.y, o[V - 2] = x.z, o[V - 1] = x.w;
        } else {
            const float2 x = global ? __ldcg(reinterpret_cast<const float2 *>(p)) : *reinterpret_cast<const float2 *>(p);
            o[0] = x.x, o[1] = x.y;
        }
    };
    auto store_out = [&](const Piece &p, int r, const Sum &x) {
        const float f = x.l == 0.f ? 0.f : 1.f / kPart / x.l;
        uint32_t *y = reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + p.b * a.out.token_stride +
                                                   (p.head0 + r) * a.out.head_stride + V * lane);
        if (V == 4) *reinterpret_cast<uint2 *>(y) = make_uint2(E::from_float2(x.o[0] * f, x.o[1] * f), E::from_float2(x.o[V - 2] * f, x.o[V - 1] * f));
        else *y = E::from_float2(x.o[0] * f, x.o[1] * f);
    };
    auto part_of = [&](int cta, int slot) { return a.partial + (static_cast<size_t>(cta) * 2 + slot) * kPartial; };
    // where each segment's parts begin among the warps' pieces: entry 2 w + slot
    const int my_first = lane < 2 * kWarps ? pieces[lane >> 1][lane & 1].first : -1;
    const unsigned valid = __ballot_sync(0xffffffffu, my_first >= 0);
    const unsigned below = valid & ((1u << lane) - 1u);
    const int first_before = __shfl_sync(0xffffffffu, my_first, below ? 31 - __clz(below) : lane);
    unsigned heads = __ballot_sync(0xffffffffu, my_first >= 0 && (!below || first_before != my_first));
    int open[2] = {-1, -1}, open_item[2] = {0, 0};  // entries of the segments that other blocks hold parts of: started before this one, goes on behind it
    int item = 0;                                   // rows of the segments so far; row r of a segment falls to warp (item + r) % kWarps
    while (heads) {
        const int w0 = __ffs(heads) - 1;
        heads &= heads - 1;
        const unsigned own = valid & (heads ? (1u << (__ffs(heads) - 1)) - 1u : 0xffffffffu) & ~((1u << w0) - 1u);
        const Piece p = pieces[w0 >> 1][w0 & 1];
        const bool mine = p.first >= cta0 && p.first + p.tiles <= cta1;
        const int slot = p.first < cta0 ? 0 : 1;
        if (!mine) open[slot] = w0, open_item[slot] = item;
        for (int r = (warp + kWarps - item % kWarps) % kWarps; r < p.rows; r += kWarps) {
            Sum x = {-INFINITY, 0.f, {}};
            for (unsigned m = own; m; m &= m - 1) {
                const int w = __ffs(m) - 1;
                x.top = fmaxf(x.top, piece_at(w >> 1, w & 1)[L::kRows * D + r]);
            }
            for (unsigned m = own; m; m &= m - 1) {
                const int w = __ffs(m) - 1;
                const float *po = piece_at(w >> 1, w & 1);
                const float f = weight(po[L::kRows * D + r], x.top);
                float o[V];
                load_o(po + r * D + V * lane, o, false);
#pragma unroll
                for (int k = 0; k < V; ++k) x.o[k] = fmaf(o[k], f, x.o[k]);
                x.l = fmaf(po[L::kRows * D + L::kRows + r], f, x.l);
            }
            if (mine) {
                store_out(p, r, x);
                continue;
            }
            float *part = part_of(blockIdx.x, slot);
            if (V == 4) *reinterpret_cast<float4 *>(part + r * D + V * lane) = make_float4(x.o[0], x.o[1], x.o[V - 2], x.o[V - 1]);
            else *reinterpret_cast<float2 *>(part + r * D + V * lane) = make_float2(x.o[0], x.o[1]);
            if (lane == 0) part[L::kRows * D + r] = x.top, part[L::kRows * D + L::kRows + r] = x.l;
        }
        item += p.rows;
    }
    if (open[0] < 0 && open[1] < 0) return;
    // One fence for all rows that the warp has written, then a lane for each row of the two open segments.
    __threadfence();
    __syncwarp();
    const int my_slot = lane >> 4, my_row = lane & 15;
    bool last = false;
    if (open[my_slot] >= 0) {
        const Piece p = pieces[open[my_slot] >> 1][open[my_slot] & 1];
        if (my_row < p.rows && (open_item[my_slot] + my_row) % kWarps == warp) {
            const int c0 = cta_of(p.first), c1 = cta_of(p.first + p.tiles - 1);
            unsigned int *counter = a.counters + c0 * kMaxRows + my_row;
            last = atomicAdd(counter, 1u) == static_cast<unsigned int>(c1 - c0);
            if (last) *counter = 0u;
        }
    }
    unsigned todo = __ballot_sync(0xffffffffu, last);
    if (todo) __threadfence();
    for (; todo; todo &= todo - 1) {
        const int which = __ffs(todo) - 1, r = which & 15;
        const int entry = open[which >> 4];
        const Piece p = pieces[entry >> 1][entry & 1];
        const int c0 = cta_of(p.first), c1 = cta_of(p.first + p.tiles - 1);
        // A lane looks at the statistics of one part, 32 parts at a time; then all lanes add the parts' outputs, sixteen loads in flight.
        Sum x = {-INFINITY, 0.f, {}};
        for (int base = c0; base <= c1; base += 32) {
            const int mine = min(base + lane, c1);
            const float *stats = part_of(mine, p.first < cta_first(mine) ? 0 : 1) + L::kRows * D + r;  // only the first block has it as its last segment
            const float pm = base + lane <= c1 ? __ldcg(stats) : -INFINITY, pl = __ldcg(stats + L::kRows);
            float now = fmaxf(x.top, pm);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, d));
            const float f0 = weight(x.top, now), f = weight(pm, now);
            float sum_l = base + lane <= c1 ? pl * f : 0.f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum_l += __shfl_xor_sync(0xffffffffu, sum_l, d);
            x.l = fmaf(x.l, f0, sum_l);
#pragma unroll
            for (int i = 0; i < V; ++i) x.o[i] *= f0;
            x.top = now;
            const int n = min(32, c1 - base + 1);
            constexpr int kBatch = 16;
            for (int k0 = 0; k0 < n; k0 += kBatch) {
                float po[kBatch][V];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int c = min(base + k0 + k, c1);
                    load_o(part_of(c, p.first < cta_first(c) ? 0 : 1) + r * D + V * lane, po[k], true);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const float fk = __shfl_sync(0xffffffffu, f, k0 + k);  // 0 behind the last part, which is loaded again there
#pragma unroll
                    for (int i = 0; i < V; ++i) x.o[i] = fmaf(po[k][i], fk, x.o[i]);
                }
            }
        }
        store_out(p, r, x);
    }
}

template <int D, int NT, bool BF16>
pd_status launch(const CacheAttnArgs &a, int grid, cudaStream_t stream) {
    using L = CacheShape<D, NT>;
    static std::atomic<bool> done[kMaxDevices];
    if (!ensure_dynamic_smem(attn_cache_kernel<D, NT, BF16>, L::kTotal, done)) return PD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(L::kThreads);
    cfg.dynamicSmemBytes = L::kTotal;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    return cuda_ok(cudaLaunchKernelEx(&cfg, attn_cache_kernel<D, NT, BF16>, a));
}

}  // namespace

size_t attn_cache_scratch_bytes() {
    return kCounterBytes + static_cast<size_t>(min(sm_count(), kMaxGrid)) * 2 * max(CacheShape<128, 1>::kPiece, CacheShape<128, 2>::kPiece);
}

pd_status launch_attn_cache(CacheAttnArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream) {
    a.counters = reinterpret_cast<unsigned int *>(scratch);
    a.partial = reinterpret_cast<float *>(scratch + kCounterBytes);
    const int grid = min(sm_count(), kMaxGrid);
    const bool wide = a.q_heads / a.kv_heads > 8;  // more than 8 heads share a key/value head: two products of 8 heads per load of the codes
    if (a.head_dim == 128) {
        if (wide) return bf16 ? launch<128, 2, true>(a, grid, stream) : launch<128, 2, false>(a, grid, stream);
        return bf16 ? launch<128, 1, true>(a, grid, stream) : launch<128, 1, false>(a, grid, stream);
    }
    if (wide) return bf16 ? launch<64, 2, true>(a, grid, stream) : launch<64, 2, false>(a, grid, stream);
    return bf16 ? launch<64, 1, true>(a, grid, stream) : launch<64, 1, false>(a, grid, stream);
}

}  // namespace pd
