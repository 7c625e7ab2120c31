// Attention of single tokens over the 8-bit paged cache: out[b, h] = sum_j softmax_j(scale q[b, h] . K[j, g]) V[j, g] over the
// tokens j < seq_lens[b], K and V being codes (signed 8 bits) times the scale of their page and head.
//
// Bound by memory: every code is read once, 2 * head_dim bytes per token and key/value head, against 4 * group * head_dim
// operations.
//
// Work.  A *segment* is the heads of one sequence that share a key/value head (up to 8 * NT of them); its tokens are cut
// into tiles of 32.  The tiles of all segments, one after another, are dealt to the warps of the grid in equal contiguous
// ranges, whatever the lengths are: a long sequence is spread over many warps, a warp may take many short ones.  The
// parts of a segment that was cut are joined in two steps, the warps of a block in shared memory and the blocks through the
// workspace by the last one to arrive (nobody waits), in the order of the tiles: results do not depend on the schedule.
//
// Inside a warp.  Tiles are fetched with cp.async into a ring that belongs to the warp alone, so that no barrier is needed.
// S^T = K Q^T and O^T = V^T P^T are m16n8k16 products with tokens (head dimensions) as M and the heads as N: for up to 8
// heads one product covers 256 codes.  The order of the contracted index and of the output rows is free, so that a thread
// takes 16 contiguous codes of a token per load.  A code c becomes binary16 exactly: byte c ^ 0x80 under the upper byte 0x64
// is 1024 + (c + 128), less 1152.  P^T is S^T's accumulator layout transposed in 8 x 8 pieces (movmatrix).
//
// Softmax in base 2 with 32-bit statistics.  The reference maximum m of a head and the reference scale r of V move only
// when a score passes m by more than 8 or a page's scale leaves [r / 8, 8 r]: P is rounded to binary16 as
// 2^(s - m) * (page scale / r) <= 2^11, so that its relative precision does not depend on how stale m and r are, and O
// needs no multiplication at most tiles.
#include "pd_attn.cuh"
#include "pd_ptx.cuh"

namespace pd {
namespace {

constexpr int kTile = 32;    // tokens of a tile: a multiple of 16, so that a 16-token product lies in one page
constexpr int kMaxGrid = 1024;  // counters in the workspace
constexpr size_t kCounterBytes = kMaxGrid * 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMaxLead = 8.f;         // how far (base-2 exponent) a score may pass the reference maximum

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
    static_assert(kTotal <= 225 * 1024, "shared memory");
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
// bytes (0, 1) or (2, 3) of w (each a code ^ 0x80) as two binary16 codes
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return hadd2_u32(prmt(w, 0x64646464u, 0x4140), 0xE480E480u); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return hadd2_u32(prmt(w, 0x64646464u, 0x4342), 0xE480E480u); }

__device__ __forceinline__ int tiles_of(int len) { return len > 0 ? (len + kTile - 1) / kTile : 1; }

// A partial result of a segment in a warp's shared memory: which one, and where it starts in the order of all tiles.
struct Piece {
    int64_t first;  // the segment's first tile; -1: none
    int tiles, b, head0, rows;
};

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(CacheShape<D, NT>::kThreads, 1) attn_cache_kernel(const CacheAttnArgs a) {
    using E = Elem<BF16>;
    using L = CacheShape<D, NT>;
    constexpr int kWarps = L::kWarps, kThreads = L::kThreads, kStages = L::kStages;
    constexpr int MT = D / 16;      // 16-row products of O^T
    constexpr int KS = D / 16;      // contraction steps of S
    constexpr int KC = D / 64;      // 16-byte pieces of a key that a thread takes
    constexpr int VB = D / 8;       // bytes of a value that a thread takes
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int scan[kThreads];
    __shared__ int warp_sum[kWarps];
    __shared__ Piece pieces[kWarps][2];
    __shared__ unsigned int arrived;

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

    // ---------------------------------------------------------------- tiles before each thread's share of the sequences
    const int share = (a.n_seqs + kThreads - 1) / kThreads;
    int sum = 0;
    for (int b = threadIdx.x * share; b < min(a.n_seqs, static_cast<int>(threadIdx.x + 1) * share); ++b) {
        const int n = __ldg(a.seq_lens + b);
        if (blockIdx.x == 0 && (n < 0 || n > room)) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        sum += tiles_of(length(b));
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
    __syncthreads();
    const int64_t total = static_cast<int64_t>(total_seq) * per_seq;
    // At least a tile for each warp of a block: with fewer, a segment would be joined from more parts than it has tiles.
    const int n_ctas = static_cast<int>(max(static_cast<int64_t>(1), min(static_cast<int64_t>(gridDim.x), total / kWarps)));
    if (static_cast<int>(blockIdx.x) >= n_ctas) return;
    auto cta_first = [&](int64_t c) { return total * c / n_ctas; };  // first tile of a block's range
    const int64_t cta0 = cta_first(blockIdx.x), cta1 = cta_first(blockIdx.x + 1);
    const int64_t range0 = cta0 + (cta1 - cta0) * warp / kWarps, range1 = cta0 + (cta1 - cta0) * (warp + 1) / kWarps;

    // Finds the segment of a tile: sequence b, segment s of it, tile i of the segment.
    auto locate = [&](int64_t at, int &b, int &s, int &i, int &len) {
        int lo = 0, hi = kThreads - 1;  // the last share that starts at or before the tile
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (static_cast<int64_t>(scan[mid]) * per_seq <= at) lo = mid;
            else hi = mid - 1;
        }
        b = lo * share;
        int64_t rest = at - static_cast<int64_t>(scan[lo]) * per_seq;
        len = length(b);
        while (rest >= static_cast<int64_t>(tiles_of(len)) * per_seq && b + 1 < a.n_seqs) {
            rest -= static_cast<int64_t>(tiles_of(len)) * per_seq;
            len = length(++b);
        }
        s = static_cast<int>(rest / tiles_of(len));
        i = static_cast<int>(rest - static_cast<int64_t>(s) * tiles_of(len));
    };

    unsigned char *ring = smem + warp * L::kWarp;
    auto piece_at = [&](int w, int slot) { return reinterpret_cast<float *>(slot == 0 ? smem + kWarps * L::kWarp + w * L::kPiece : smem + w * L::kWarp); };
    float4 *meta = reinterpret_cast<float4 *>(ring + L::kRing);

    // ---------------------------------------------------------------- the warp's tiles
    const float lscale = a.scale * kLog2e;
    int b = 0, s = 0, i0 = 0, len = 0;
    int64_t at = range0;
    if (at < range1) locate(at, b, s, i0, len);
    while (at < range1) {
        const int n_tiles = tiles_of(len);
        const int kvh = s / chunks, chunk = s - kvh * chunks;
        const int head0 = kvh * group + chunk * L::kRows;
        const int rows = min(L::kRows, group - chunk * L::kRows);
        const int i1 = static_cast<int>(min(static_cast<int64_t>(n_tiles), i0 + (range1 - at)));

        float o[MT][NT][4];
        float m[NT][2], mu[NT][2], l[NT][2], qs[NT][2];
        uint32_t qf[KS][NT][2];
        float ref = 0.f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][n][k] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // the head's query, scaled by a power of two to a largest magnitude of 1..2: exact in binary16 for both types
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
            // 2^-e with e the exponent of amax, held to what binary32 and its reciprocal can say
            const int e = min(max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100), 100);
            const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23), up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    qf[c * 4 + k][n][0] = Elem<false>::from_float2(x[c][4 * k] * down, x[c][4 * k + 1] * down);
                    qf[c * 4 + k][n][1] = Elem<false>::from_float2(x[c][4 * k + 2] * down, x[c][4 * k + 3] * down);
                }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                qs[n][k] = lscale * __shfl_sync(0xffffffffu, up, (2 * t + k) * 4);
                m[n][k] = -INFINITY, mu[n][k] = 0.f, l[n][k] = 0.f;
            }
        }

        if (len > 0) {
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
                    if (lane == src) meta[st] = make_float4(sk[0], sk[1], sv[0], sv[1]);
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
                }
                cp_async_commit();
            };
            __syncwarp();
#pragma unroll
            for (int k = 0; k < kStages - 1; ++k) issue(i0 + k);
            for (int i = i0; i < i1; ++i) {
                cp_async_wait<kStages - 2>();
                __syncwarp();
                issue(i + kStages - 1);
                const int st = (i - i0) % kStages;
                const unsigned char *ks = ring + st * L::kStage, *vs = ks + kTile * D;
                const float4 sc = meta[st];

                // S^T = K Q^T
                float acc[2][NT][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[h][n][k] = 0.f;
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        const int row = 16 * h + g, piece = D == 128 ? (t + 4 * c) ^ ((row & 1) * 4) : t;
                        const uint4 lo = *reinterpret_cast<const uint4 *>(ks + row * D + piece * 16);
                        const uint4 hi = *reinterpret_cast<const uint4 *>(ks + (row + 8) * D + piece * 16);
                        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t ul = wl[k] ^ 0x80808080u, uh = wh[k] ^ 0x80808080u;
                            const uint32_t a0 = codes_lo(ul), a1 = codes_lo(uh), a2 = codes_hi(ul), a3 = codes_hi(uh);
#pragma unroll
                            for (int n = 0; n < NT; ++n) Elem<false>::mma16816(acc[h][n], a0, a1, a2, a3, qf[c * 4 + k][n][0], qf[c * 4 + k][n][1]);
                        }
                    }
                }
                // scores in base 2; places past the end of the sequence are chosen away, whatever they hold
                bool lead = false;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float f = (h == 0 ? sc.x : sc.y) * qs[n][k & 1];
                            const int64_t tok = static_cast<int64_t>(i) * kTile + 16 * h + g + 8 * (k >> 1);
                            acc[h][n][k] = tok < len ? acc[h][n][k] * f : -INFINITY;
                            lead |= acc[h][n][k] > m[n][k & 1] + kMaxLead;
                        }
                const float sv_hi = fmaxf(sc.z, sc.w);
                const bool move_ref = sv_hi > 8.f * ref || (sv_hi < 0.125f * ref && sv_hi > 0.f);
                if (__any_sync(0xffffffffu, lead) || move_ref) {
                    const float step = move_ref ? ref / sv_hi : 1.f;
                    if (move_ref) ref = sv_hi;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float top = fmaxf(fmaxf(acc[0][n][k], acc[0][n][k + 2]), fmaxf(acc[1][n][k], acc[1][n][k + 2]));
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            top = fmaxf(top, m[n][k]);
                            const float mu_new = top == -INFINITY ? 0.f : top;
                            const float shrink = exp2_approx(m[n][k] - mu_new);  // 0 from -infinity on
                            l[n][k] *= shrink;
                            m[n][k] = top, mu[n][k] = mu_new;
                            const float f = shrink * step;
#pragma unroll
                            for (int j = 0; j < MT; ++j) o[j][n][k] *= f, o[j][n][k + 2] *= f;
                        }
                }
                const float inv_ref = ref > 0.f ? __frcp_rn(ref) : 0.f;
                const float rv[2] = {sc.z == 0.f ? 0.f : sc.z * inv_ref, sc.w == 0.f ? 0.f : sc.w * inv_ref};
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
                            *reinterpret_cast<float2 *>(po + r * D + VB * g + 2 * j) = make_float2(o[j][n][k] * ref, o[j][n][k + 2] * ref);
                    }
                }
            if (lane == 0) pieces[warp][slot] = {at - i0, n_tiles, b, head0, rows};
        }
        at += i1 - i0;
        i0 = 0;
        if (at < range1 && ++s == per_seq) {
            s = 0;
            len = length(++b);
        }
    }
    __syncthreads();

    // ---------------------------------------------------------------- the block's parts of each segment, in the order of the tiles
    auto store_out = [&](const Piece &p, int r, int d, float4 v, float f) {
        uint16_t *y = static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + p.b * a.out.token_stride + (p.head0 + r) * a.out.head_stride + d;
        *reinterpret_cast<uint2 *>(y) = make_uint2(E::from_float2(v.x * f, v.y * f), E::from_float2(v.z * f, v.w * f));
    };
    auto weight = [](float m, float top) { return m == -INFINITY ? 0.f : exp2_approx(m - top); };
    constexpr int kPartial = L::kPiece / 4;
    Piece open[2];  // segments that other blocks hold parts of: the one that started before this block's range, the one that goes on behind it
    open[0].first = open[1].first = -1;
    for (int w0 = 0; w0 < 2 * kWarps;) {
        const Piece p = pieces[w0 >> 1][w0 & 1];
        int w1 = w0 + 1;
        if (p.first < 0) {
            w0 = w1;
            continue;
        }
        while (w1 < 2 * kWarps && (pieces[w1 >> 1][w1 & 1].first < 0 || pieces[w1 >> 1][w1 & 1].first == p.first)) ++w1;
        const bool mine = p.first >= cta0 && p.first + p.tiles <= cta1;
        const int slot = p.first < cta0 ? 0 : 1;
        float *out_part = a.partial + (static_cast<size_t>(blockIdx.x) * 2 + slot) * kPartial;
        for (int idx = threadIdx.x; idx < p.rows * (D / 4); idx += kThreads) {
            const int r = idx / (D / 4), d = idx % (D / 4) * 4;
            float top = -INFINITY;
            for (int w = w0; w < w1; ++w)
                if (pieces[w >> 1][w & 1].first >= 0) top = fmaxf(top, piece_at(w >> 1, w & 1)[L::kRows * D + r]);
            float4 sum4 = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum_l = 0.f;
            for (int w = w0; w < w1; ++w) {
                if (pieces[w >> 1][w & 1].first < 0) continue;
                const float *po = piece_at(w >> 1, w & 1);
                const float f = weight(po[L::kRows * D + r], top);
                const float4 v = *reinterpret_cast<const float4 *>(po + r * D + d);
                sum4.x = fmaf(v.x, f, sum4.x), sum4.y = fmaf(v.y, f, sum4.y), sum4.z = fmaf(v.z, f, sum4.z), sum4.w = fmaf(v.w, f, sum4.w);
                sum_l = fmaf(po[L::kRows * D + L::kRows + r], f, sum_l);
            }
            if (mine) {
                store_out(p, r, d, sum4, sum_l == 0.f ? 0.f : 1.f / sum_l);
            } else {
                *reinterpret_cast<float4 *>(out_part + r * D + d) = sum4;
                if (d == 0) out_part[L::kRows * D + r] = top, out_part[L::kRows * D + L::kRows + r] = sum_l;
            }
        }
        if (!mine) open[slot] = p;
        w0 = w1;
    }

    // ---------------------------------------------------------------- segments that several blocks worked on: the last block to arrive joins them
    for (int slot = 0; slot < 2; ++slot) {
        const Piece p = open[slot];
        if (p.first < 0) continue;  // the same in all threads
        const int c0 = static_cast<int>(((p.first + 1) * n_ctas - 1) / total), c1 = static_cast<int>(((p.first + p.tiles) * n_ctas - 1) / total);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) arrived = atomicAdd(a.counters + c0, 1u);
        __syncthreads();
        if (arrived != static_cast<unsigned int>(c1 - c0)) continue;
        __threadfence();
        if (threadIdx.x == 0) a.counters[c0] = 0u;
        for (int idx = threadIdx.x; idx < p.rows * (D / 4); idx += kThreads) {
            const int r = idx / (D / 4), d = idx % (D / 4) * 4;
            float4 sum4 = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum_l = 0.f, top = -INFINITY;
            for (int c = c0; c <= c1; c += 4) {
                float pm[4], pl[4];
                float4 pv[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int cc = min(c + k, c1);
                    // only the segment's first block may hold it as its last one
                    const float *po = a.partial + (static_cast<size_t>(cc) * 2 + (p.first < cta_first(cc) ? 0 : 1)) * kPartial;
                    pm[k] = c + k <= c1 ? __ldcg(po + L::kRows * D + r) : -INFINITY;
                    pl[k] = __ldcg(po + L::kRows * D + L::kRows + r);
                    pv[k] = __ldcg(reinterpret_cast<const float4 *>(po + r * D + d));
                }
                const float now = fmaxf(top, fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])));
                const float f0 = weight(top, now);
                sum4.x *= f0, sum4.y *= f0, sum4.z *= f0, sum4.w *= f0, sum_l *= f0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (c + k > c1) break;
                    const float f = weight(pm[k], now);
                    sum4.x = fmaf(pv[k].x, f, sum4.x), sum4.y = fmaf(pv[k].y, f, sum4.y), sum4.z = fmaf(pv[k].z, f, sum4.z), sum4.w = fmaf(pv[k].w, f, sum4.w);
                    sum_l = fmaf(pl[k], f, sum_l);
                }
                top = now;
            }
            store_out(p, r, d, sum4, sum_l == 0.f ? 0.f : 1.f / sum_l);
        }
    }
}

template <int D, int NT, bool BF16>
pd_status launch(const CacheAttnArgs &a, int grid, cudaStream_t stream) {
    using L = CacheShape<D, NT>;
    static std::atomic<bool> done[kMaxDevices];
    if (!ensure_dynamic_smem(attn_cache_kernel<D, NT, BF16>, L::kTotal, done)) return PD_ERR_CUDA;
    attn_cache_kernel<D, NT, BF16><<<grid, L::kThreads, L::kTotal, stream>>>(a);
    count_launch();
    return cuda_ok(cudaGetLastError());
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
