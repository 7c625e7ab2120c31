// Causal attention over packed prompts: out[i, h] = sum_{j <= i} softmax_j(scale q[i, h] . k[j, g]) v[j, g] inside each sequence.
//
// One pass over the keys with a running maximum m and sum l of each query row (32 bits, base 2): with s the scores of a tile,
//     m' = max(m, max s),  l' = l 2^(m - m') + sum 2^(s - m'),  O' = O 2^(m - m') + 2^(s - m') V,  out = O / l at the end.
// P = 2^(s - m') is rounded to the type of v for its product; l sums the unrounded values.  m only moves when a score passes
// it by more than 8, so that O is hardly ever rescaled: P is then at most 2^8 and its relative rounding is the same.  In
// binary16 P and l are 2^7 times that, which is what its range has room for: weights down to 2^-21 of the largest keep their
// precision, those below lose up to 2^-32 of it.  In bfloat16 they are 2^-24 times that, so that O, which is divided by l at the
// end, stays in range beside values of any size.
//
// Bound by the tensor cores (4 * head_dim operations per query, key and head) and, as nearly, by the exponentials: a tile of
// 128 x 128 scores is 1024 clocks of products at head_dim 128 and 1024 clocks of the 16 exponentials a clock that an SM has (both
// pipes are busy 59 % of the time; a polynomial for some of the exponentials changed nothing).
// Measured, sustained: 64 query and 8 key/value heads of 128, one prompt of 8192 tokens 985 us (1.11 PFLOP/s at the power limit; 850
// us in short bursts); 7 prompts of 7919 tokens together 257 us (220); 32 heads, 4 prompts of 512 tokens 23.2 us, where what
// surrounds the products counts: first loads, the last units of the blocks, instructions not in the cache.
//
// A block works on units of two *slots* of 128 queries each that read the same keys: two heads that share their key/value
// head where their number is even, else two consecutive pieces of one head's queries.  Tiles of 128 keys: S = Q K^T (both
// operands in shared memory) into tensor memory, softmax by one thread per row, P into tensor memory, O += P V with P from
// tensor memory.  P is handed over in two halves, so that the second product starts while the other half's exponentials
// are computed.
// Tensor memory: one buffer of 128 columns for S that both slots use in turn (a row of S is taken into registers at once, and
// the buffer is free again long before its softmax is done), 64 columns of P and 128 of O for each slot.  So the scores of a
// slot's next tile wait for its softmax, not the softmax for them.  (A buffer of S for each slot with P in its place, where a
// slot's softmax stands still during its own two products: 1110 us where this gave 900, 8192 tokens in short bursts.)
//
// Roles: warps 0-3 and 4-7 the softmax of slot 0 and 1; warp 8 units and TMA; warps 9 and 10 issue the products with the
// keys and with the values (one warp for both, scores first: 20 % slower); warp 11 looks for infinities and NaN among the
// values of a tile on the diagonal, where 0 * v must not reach the queries that do not attend to v: they are set to zero
// there, and the output adds them for the queries that do (a tile on the diagonal is full for the products when warp 11 has
// been through it); warps 12-15 write the output while the softmax is at the next unit.  Every wait is bounded.
// The code is kept short on purpose (rolled loops, one wait routine, one election for a group of products): before that the
// counters had 2.5 warps per issue that waited for their next instruction, now 0.5.
#include "pd_attn.cuh"
#include "pd_tcgen05.cuh"

namespace pd {
namespace {

constexpr int kTile = 128;  // queries of a slot, keys of a tile
constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kUnits = 4;  // units that the producer may be ahead
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMaxLead = 8.f;  // how far (base-2 exponent) a score may pass the reference maximum
constexpr float kFar = 1024.f;   // reference maxima (base-2 exponent) from which on scores are taken from them before they are scaled
constexpr float kRoom = 7.f, kRoomBf16 = -24.f;  // the exponent by which P is larger than the weights in binary16 and bfloat16
constexpr uint32_t kColS = 0, kColP = 128, kColO = 256;  // tensor-memory columns; slot 1: P + 64, O + 128

struct Unit {
    int first, len;  // the sequence's first token and its length; len 0: no more units
    int q0, head;    // first query (in the sequence) and head of slot 0
};

struct Slots {
    bool by_head;  // slots are two heads (else two consecutive tiles of queries)
    __device__ __forceinline__ int q0(const Unit &u, int s) const { return by_head ? u.q0 : u.q0 + s * kTile; }
    __device__ __forceinline__ int head(const Unit &u, int s) const { return by_head ? u.head + s : u.head; }
    // key tiles of a slot; 0: the slot has no queries
    __device__ __forceinline__ int tiles(const Unit &u, int s) const { return q0(u, s) < u.len ? q0(u, s) / kTile + 1 : 0; }
    __device__ __forceinline__ int max_tiles(const Unit &u) const { return max(tiles(u, 0), tiles(u, 1)); }
};

template <int D>
struct PromptSmem {
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kStages = D == 128 ? 4 : 8;  // of keys or values
    static constexpr int kQ = 0;
    static constexpr int kRing = 2 * kTileBytes;
    static constexpr int kOut = kRing + kStages * kTileBytes;  // for each output warp 32 rows of outputs
    static constexpr int kSums = kOut + 4 * 32 * D * 2;          // l of the two slots' rows, for two units
    static constexpr int kBars = kSums + 2 * 2 * kTile * 4;
    static constexpr int kTotal = kBars + 512;
    static_assert(kTotal <= 227 * 1024, "shared memory");
};

struct Bars {
    uint64_t kv_full[8], kv_empty[8];
    uint64_t v_landed[4];  // tiles on a diagonal, in turn: no more of them are in the ring
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], s_free, p_half[2][2], o_done[2], o_last[2], o_empty[2];
    uint64_t unit_full[kUnits], unit_empty[kUnits];
    Unit units[kUnits];
    int taint[kUnits];
    uint32_t tmem;
    int abort_flag;
};
static_assert(sizeof(Bars) <= 512, "barriers");

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
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
// one of the two 16-bit values is an infinity or a NaN
template <bool BF16>
__device__ __forceinline__ bool non_finite2(uint32_t w) {
    constexpr uint32_t e = BF16 ? 0x7F80u : 0x7C00u;
    return (w & e) == e || ((w >> 16) & e) == e;
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

// acc stays zero unless one of the 16-bit values is an infinity or a NaN
template <bool BF16>
__device__ __forceinline__ uint32_t times_zero(uint32_t w, uint32_t acc) {
    uint32_t d;
    if (BF16) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(w), "r"(0u), "r"(acc));
    else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(w), "r"(0u), "r"(acc));
    return d;
}

// Adds to `n` outputs of a row the infinities and NaN among the values of `keys` tokens.
template <bool BF16>
__device__ __noinline__ void add_non_finite(uint16_t *y, int n, const uint16_t *v, int64_t token_stride, int keys) {
    using E = Elem<BF16>;
    for (int c = 0; c < n; c += 8) {
        const uint4 x = *reinterpret_cast<const uint4 *>(y + c);
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        for (int key = 0; key < keys; ++key) {
            const uint4 t = __ldg(reinterpret_cast<const uint4 *>(v + key * token_stride + c));
            const uint32_t b[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 p = E::to_float2(b[i]), o = E::to_float2(w[i]);
                w[i] = E::from_float2(fabsf(p.x) <= 3.402823466e38f ? o.x : o.x + p.x, fabsf(p.y) <= 3.402823466e38f ? o.y : o.y + p.y);
            }
        }
        *reinterpret_cast<uint4 *>(y + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const PromptArgs a) {
    using E = Elem<BF16>;
    using L = PromptSmem<D>;
    constexpr int kStages = L::kStages;
    static_assert(kStages % 2 == 0, "keys and values keep to their own stages");
    constexpr int kPieces = D / 64;                    // sub-tiles of 64 columns
    constexpr int kPieceBytes = kTile * 64 * 2;
    extern __shared__ __align__(1024) unsigned char smem[];  // the swizzle counts from 1024-byte boundaries
    Bars &bar = *reinterpret_cast<Bars *>(smem + L::kBars);
    volatile int *abort_flag = &bar.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.q_heads / a.kv_heads;
    const Slots slots = {group % 2 == 0};
    // Bounded; the first one to give up says where, and the block's last act is to report it.  Short, because it is in the code
    // of every role many times over.
    auto wait = [&](uint64_t *b, uint32_t parity, int where) {
        if (mbar_try_wait(b, parity & 1u)) return true;
        const long long since = clock64();
        while (!mbar_try_wait(b, parity & 1u))
            if (clock64() - since > kWaitCycles) {
                *abort_flag = where;
                return false;
            }
        return true;
    };
    auto wait_warp = [&](uint64_t *b, uint32_t parity, int where) { return __all_sync(0xffffffffu, wait(b, parity, where)) != 0; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(bar.kv_full + i, 1), mbar_init(bar.kv_empty + i, 1);
        for (int i = 0; i < 4; ++i) mbar_init(bar.v_landed + i, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar.q_full + s, 1), mbar_init(bar.q_empty + s, 1), mbar_init(bar.s_full + s, 1);
            mbar_init(bar.p_half[s], 4), mbar_init(bar.p_half[s] + 1, 4), mbar_init(bar.o_done + s, 1);
            mbar_init(bar.o_last + s, 1), mbar_init(bar.o_empty + s, 4);
        }
        mbar_init(&bar.s_free, 4);
        for (int i = 0; i < kUnits; ++i) mbar_init(bar.unit_full + i, 1), mbar_init(bar.unit_empty + i, 15);
        bar.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 9) tcgen05_alloc(&bar.tmem, 512);
    if (warp == 8 && lane < 3) prefetch_tensormap(lane == 0 ? &map_q : (lane == 1 ? &map_k : &map_v));
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    asm volatile("griddepcontrol.wait;" ::: "memory");  // everything before touches no memory of the caller's
    const uint32_t tmem = bar.tmem;

    // The next unit, in the producer's order: every other role reads what the producer wrote.
    uint32_t n_unit = 0;
    auto next_unit = [&](Unit &u) {
        if (!wait_warp(bar.unit_full + n_unit % kUnits, n_unit / kUnits, 50)) return false;
        u = bar.units[n_unit % kUnits];
        return u.len > 0;
    };
    auto done_unit = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar.unit_empty + n_unit % kUnits);
        ++n_unit;
    };

    if (warp >= 8 && warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 8) {
            // -------------------------------------------------------- units and TMA
            // Units in the order of their work, most first, so that the blocks end together: the last queries of every sequence
            // that has as many tiles as the longest, then the tile before those, and so on; all heads of a tile in a row.
            // More than 32 sequences are taken 32 at a time.  A lane knows one sequence; ids only grow, so that the walk over
            // groups and tiles goes forward only.  Behind offsets that decrease no sequence is taken: those before have no token
            // in common, so that the work and its ids stay within what the host has counted for n_tokens.
            const int span = slots.by_head ? kTile : 2 * kTile;                     // queries of a unit
            const int per_tile = slots.by_head ? a.q_heads / 2 : a.q_heads;         // units of a tile
            int g0 = -32, first = 0, len = 0, tiles = 0, level = 0, level_base = 0, group_end = 0;
            uint32_t it = 0, n_diag = 0, phase_q = 3;  // bit s: slot s; the places are free at first
            bool ok = true, in_order = true;
            int id = blockIdx.x;
            while (ok) {
                id = __shfl_sync(0xffffffffu, id, 0);
                while (id >= group_end && g0 < a.n_seqs) {
                    g0 += 32;
                    tiles = 0;
                    int end = first = 0;
                    if (g0 + lane < a.n_seqs) {
                        first = __ldg(a.cu_seqlens + g0 + lane), end = __ldg(a.cu_seqlens + g0 + lane + 1);
                        if (first < 0 || end < first || end > a.n_tokens) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(g0 + lane));
                    }
                    const unsigned down = __ballot_sync(0xffffffffu, end < first);
                    if (in_order && !(down & ((2u << lane) - 1u)) && first >= 0 && end <= a.n_tokens) {
                        len = end - first;
                        tiles = (len + span - 1) / span;
                    }
                    in_order = in_order && !down;
                    level_base = group_end;
                    group_end += __reduce_add_sync(0xffffffffu, tiles) * per_tile;
                    level = __reduce_max_sync(0xffffffffu, tiles) - 1;
                }
                Unit u = {0, 0, 0, 0};
                if (id < group_end) {
                    unsigned m;
                    int n;
                    while (m = __ballot_sync(0xffffffffu, tiles > level), n = __popc(m) * per_tile, id >= level_base + n) level_base += n, --level;
                    const int rank = (id - level_base) / per_tile;
                    const int src = __ffs(__ballot_sync(0xffffffffu, ((m >> lane) & 1u) && __popc(m & ((1u << lane) - 1u)) == rank)) - 1;
                    u = {__shfl_sync(0xffffffffu, first, src), __shfl_sync(0xffffffffu, len, src), level * span,
                         ((id - level_base) % per_tile) * (slots.by_head ? 2 : 1)};
                }
                const bool end_mark = u.len == 0;
                if (lane == 0 && !end_mark) id = static_cast<int>(gridDim.x + atomicAdd(a.counters, 1u));  // known by the time it is needed
                const uint32_t us = n_unit % kUnits, ur = n_unit / kUnits;
                if (ur > 0 && !(ok = wait_warp(bar.unit_empty + us, ur - 1, 51))) break;
                if (lane == 0) {
                    bar.units[us] = u;
                    mbar_arrive(bar.unit_full + us);
                }
                ++n_unit;
                if (end_mark) break;
                if (lane == 0) {
                    const int n0 = slots.tiles(u, 0), n = slots.max_tiles(u), kvh = u.head / group;
                    auto load = [&](const CUtensorMap *map, unsigned char *dst, uint64_t *full, int head, int row) {
                        mbar_arrive_expect_tx(full, L::kTileBytes);
#pragma unroll
                        for (int p = 0; p < kPieces; ++p) tma_load_3d(map, full, dst + p * kPieceBytes, p * 64, head, row);
                    };
#pragma unroll 1
                    for (int j = 0; j < n && ok; ++j) {
#pragma unroll 1
                        for (int kv = 0; kv < 2 && ok; ++kv, ++it) {
                            const uint32_t st = it % kStages, round = it / kStages;
                            if (round > 0 && !(ok = wait(bar.kv_empty + st, round - 1, 53))) break;
                            uint64_t *full = bar.kv_full + st;
                            if (kv == 1 && j >= n0 - 1) full = bar.v_landed + n_diag++ % 4;  // on a diagonal: warp 11 first
                            load(kv == 0 ? &map_k : &map_v, smem + L::kRing + st * L::kTileBytes, full, kvh, u.first + j * kTile);
                            if (j == 0 && kv == 0) {
#pragma unroll 1
                                for (int s = 0; s < 2 && ok; ++s) {
                                    if (slots.tiles(u, s) == 0) continue;
                                    if (!(ok = wait(bar.q_empty + s, phase_q >> s, 52))) break;
                                    phase_q ^= 1u << s;
                                    load(&map_q, smem + L::kQ + s * L::kTileBytes, bar.q_full + s, slots.head(u, s), u.first + slots.q0(u, s));
                                }
                            }
                        }
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
            }
        } else if (warp == 9) {
            // -------------------------------------------------------- S = Q K^T of the units' steps: their slots' tiles in turn
            const uint32_t idesc = kIdescBase<BF16> | (a.scale < 0.f ? 1u << 13 : 0u) | (static_cast<uint32_t>(kTile >> 3) << 17) | (static_cast<uint32_t>(kTile >> 4) << 24);  // bit 13: A negated
            const uint32_t q_desc = desc_lower(smem + L::kQ, 16), k_desc = desc_lower(smem + L::kRing, 16);
            uint32_t it = 0, n_step = 0, phase_q = 0;  // bit s of a phase: the parity of slot s
            bool ok = true;
            Unit u;
            while (ok && next_unit(u)) {
                // the same in all lanes, which the compiler then knows
                u.len = __shfl_sync(0xffffffffu, u.len, 0), u.q0 = __shfl_sync(0xffffffffu, u.q0, 0);
                const int n0 = slots.tiles(u, 0), n1 = slots.tiles(u, 1), n = max(n0, n1);
                for (int j = 0; j < n && ok; ++j, it += 2) {
                    const uint32_t st = it % kStages;
                    if (!(ok = wait_warp(bar.kv_full + st, it / kStages, 54))) break;
                    const uint32_t k = k_desc + st * (L::kTileBytes >> 4);
#pragma unroll 1  // the instructions of the roles that run together have to fit into the caches for them
                    for (int s = 0; s < 2; ++s) {
                        const int ns = s ? n1 : n0;
                        if (j >= ns) continue;
                        if (j == 0) {
                            if (!(ok = wait_warp(bar.q_full + s, phase_q >> s, 55))) break;
                            phase_q ^= 1u << s;
                        }
                        if (n_step > 0 && !(ok = wait_warp(&bar.s_free, n_step - 1, 56))) break;
                        ++n_step;
                        tcgen05_fence_after();
                        if (elect_one())
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = ((kk / 4) * kPieceBytes + (kk % 4) * 32) >> 4;
                            mma_smem_a(tmem + kColS, make_desc(q_desc + s * (L::kTileBytes >> 4) + off), make_desc(k + off), idesc, kk > 0);
                        }
                        commit_elected(bar.s_full + s);
                        if (j + 1 == ns) commit_elected(bar.q_empty + s);
                    }
                    if (ok) commit_elected(bar.kv_empty + st);
                }
                ok = __all_sync(0xffffffffu, ok);
                done_unit();
            }
        } else if (warp == 10) {
            // -------------------------------------------------------- O += P V of the same steps
            constexpr uint32_t kIdesc = kIdescBase<BF16> | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (static_cast<uint32_t>(kTile >> 4) << 24);
            const uint32_t v_desc = desc_lower(smem + L::kRing, kPieceBytes);
            uint32_t it = 0, phase_o = 3, phase_p = 0;  // O of each slot is free at first
            bool ok = true;
            Unit u;
            while (ok && next_unit(u)) {
                u.len = __shfl_sync(0xffffffffu, u.len, 0), u.q0 = __shfl_sync(0xffffffffu, u.q0, 0);
                const int n0 = slots.tiles(u, 0), n1 = slots.tiles(u, 1), n = max(n0, n1);
                for (int j = 0; j < n && ok; ++j, it += 2) {
                    const uint32_t st = (it + 1) % kStages;
                    if (!(ok = wait_warp(bar.kv_full + st, (it + 1) / kStages, 57))) break;
                    const uint32_t v = v_desc + st * (L::kTileBytes >> 4);
#pragma unroll 1
                    for (int s = 0; s < 2; ++s) {
                        if (j >= (s ? n1 : n0)) continue;
                        if (j == 0) {
                            if (!(ok = wait_warp(bar.o_empty + s, phase_o >> s, 58))) break;
                            phase_o ^= 1u << s;
                        }
#pragma unroll 1
                        for (int half = 0; half < 2 && ok; ++half) {
                            if (!(ok = wait_warp(bar.p_half[s] + half, phase_p >> s, 60))) break;
                            tcgen05_fence_after();
                            const uint32_t v_half = v + half * (4 * 2048 >> 4), p_half = tmem + kColP + s * 64 + half * 32;
                            if (elect_one())
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                tcgen05_mma_f16_tmem_a(tmem + kColO + s * 128, p_half + kk * 8, make_desc(v_half + kk * (2048 >> 4)), kIdesc, (j + half + kk > 0) ? 1u : 0u);
                        }
                        if (!ok) break;
                        phase_p ^= 1u << s;
                        commit_elected(bar.o_done + s);
                        if (j + 1 == (s ? n1 : n0)) commit_elected(bar.o_last + s);
                    }
                    if (ok) commit_elected(bar.kv_empty + st);
                }
                ok = __all_sync(0xffffffffu, ok);
                done_unit();
            }
        } else {
            // -------------------------------------------------------- values on the diagonal: no infinities and NaN in shared memory
            uint32_t it = 0, n_diag = 0;
            bool ok = true;
            Unit u;
            while (ok && next_unit(u)) {
                const int n0 = slots.tiles(u, 0), n1 = slots.tiles(u, 1), n = max(n0, n1);
                bool found = false;
                for (int j = n0 - 1; j < n; ++j, ++n_diag) {
                    const uint32_t st = (it + 2 * j + 1) % kStages;
                    if (!(ok = wait_warp(bar.v_landed + n_diag % 4, n_diag / 4, 59))) break;
                    uint4 *p = reinterpret_cast<uint4 *>(smem + L::kRing + st * L::kTileBytes) + lane;
                    uint32_t acc[4] = {0u, 0u, 0u, 0u};
#pragma unroll 8
                    for (int k = 0; k < L::kTileBytes / 16 / 32; ++k) {
                        const uint4 x = p[k * 32];
                        acc[0] = times_zero<BF16>(x.x, acc[0]), acc[1] = times_zero<BF16>(x.y, acc[1]);
                        acc[2] = times_zero<BF16>(x.z, acc[2]), acc[3] = times_zero<BF16>(x.w, acc[3]);
                    }
                    if (__any_sync(0xffffffffu, ((acc[0] | acc[1] | acc[2] | acc[3]) & 0x7fff7fffu) != 0u)) {
                        found = true;
                        for (int k = 0; k < L::kTileBytes / 16 / 32; ++k) {
                            const uint4 x = p[k * 32];
                            uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                if (non_finite2<BF16>(w[c] & 0xffffu)) w[c] &= 0xffff0000u;
                                if (non_finite2<BF16>(w[c] & 0xffff0000u)) w[c] &= 0xffffu;
                            }
                            p[k * 32] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        fence_proxy_async_smem();
                    }
                    if (lane == 0) bar.taint[n_unit % kUnits] = found;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.kv_full + st);
                }
                it += 2 * n;
                done_unit();
            }
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ------------------------------------------------------------ output: O / l of both slots, while the softmax is at the next unit
        const int w = warp & 3;
        uint32_t n_sum[2] = {0, 0};
        bool ok = true;
        Unit u;
        while (ok && next_unit(u)) {
#pragma unroll 1
            for (int s = 0; s < 2; ++s) {
                if (slots.tiles(u, s) == 0) continue;
                const uint32_t k_u = s ? n_sum[1]++ : n_sum[0]++;
                if (!(ok = wait_warp(bar.o_last + s, k_u, 62))) break;
                tcgen05_fence_after();
                const float inv = 1.f / reinterpret_cast<const float *>(smem + L::kSums)[((k_u & 1) * 2 + s) * kTile + w * 32 + lane];
                const uint32_t to = tmem + (static_cast<uint32_t>(w * 32) << 16) + kColO + s * 128;
                // Rows go through shared memory, so that O is free as soon as it has been read, and they leave in whole lines:
                // written by the threads that own them they were 32 pieces of 16 bytes an instruction.
                constexpr int kRow = D * 2, kPer = D / 8;  // bytes and 16-byte pieces of a row
                unsigned char *out = smem + L::kOut + w * (32 * kRow);
#pragma unroll
                for (int c = 0; c < D; c += 16) {
                    uint32_t o[16];
                    tcgen05_ld_32x32b_x16(to + c, o);
                    tcgen05_wait_ld();
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = E::from_float2(__uint_as_float(o[8 * k + 2 * i]) * inv, __uint_as_float(o[8 * k + 2 * i + 1]) * inv);
                        *reinterpret_cast<uint4 *>(out + lane * kRow + (((c / 8 + k) ^ (lane & 7)) * 16)) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                }
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.o_empty + s);
                const int head = slots.head(u, s), row0 = slots.q0(u, s) + w * 32;  // the warp's first row
                const int piece = lane % kPer, rows = min(32, u.len - row0);
                uint16_t *y = static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + static_cast<int64_t>(u.first + row0 + lane / kPer) * a.out.token_stride +
                              head * a.out.head_stride + 8 * piece;
#pragma unroll 4
                for (int i = lane / kPer; i < rows; i += 32 / kPer, y += (32 / kPer) * a.out.token_stride)
                    *reinterpret_cast<uint4 *>(y) = *reinterpret_cast<const uint4 *>(out + i * kRow + ((piece ^ (i & 7)) * 16));
                __syncwarp();
                if (bar.taint[n_unit % kUnits] && lane < rows)
                    add_non_finite<BF16>(static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + static_cast<int64_t>(u.first + row0 + lane) * a.out.token_stride +
                                             head * a.out.head_stride, D,
                                         static_cast<const uint16_t *>(a.v.ptr) + static_cast<int64_t>(u.first + u.q0) * a.v.token_stride +
                                             (head / group) * a.v.head_stride, a.v.token_stride, row0 + lane - u.q0 + 1);
            }
            if (!ok) break;
            done_unit();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        // ------------------------------------------------------------ softmax and output: a thread owns one row of a slot
        const int s = warp >> 2;
        const int r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t ts = lanes + kColS, tp = lanes + kColP + s * 64, to = lanes + kColO + s * 128;
        // The maximum is taken before the scores are scaled, so that the factor is positive: the products give -Q K^T for a
        // negative scale, and a scale of zero is one that makes nothing of any finite score (minus infinity stays what it is):
        // 2^128 * 2^-149 is the most that is left of one.
        const float f = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 0x1p-149f;
        uint32_t n_s = 0, n_sum = 0;  // tiles and units of the slot so far
        bool ok = true;
        Unit u;
        while (ok && next_unit(u)) {
            const int n = slots.tiles(u, s);
            if (n == 0) {
                done_unit();
                continue;
            }
            float m = -INFINITY;  // of the scores before they are scaled
            float sub1 = 0.f;     // what the exponents get added: -m f, and the room of P
            bool far = false;     // the same in all lanes
            float2 l = make_float2(0.f, 0.f);
            for (int j = 0; j < n; ++j, ++n_s) {
                if (!(ok = wait_warp(bar.s_full + s, n_s, 60))) break;
                tcgen05_fence_after();
                if (j == n - 1) {  // on the diagonal: keys 0 .. r of the tile; in place and in a loop, which keeps the code short
#pragma unroll 1
                    for (int c = r & ~31; c < kTile; c += 32) {
                        uint32_t y[32];
                        tcgen05_ld_32x32b_x32(ts + c, y);
                        tcgen05_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c + k > r) y[k] = 0xff800000u;
                        tcgen05_st_32x32b_x32(ts + c, y);
                    }
                    tcgen05_wait_st();
                }
                uint32_t x[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tcgen05_ld_32x32b_x32(ts + 32 * c, x[c]);
                tcgen05_wait_ld();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.s_free);
                float top[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    top[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][31]));
#pragma unroll
                    for (int k = 1; k < 31; k += 2) top[c] = max3(top[c], __uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1]));
                }
                const float best = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                // Before O is rescaled or P written the product with the tile before has to be done.
                bool may_write = n_s == 0;
                auto until_done = [&]() {
                    if (!may_write) {
                        may_write = wait_warp(bar.o_done + s, n_s - 1, 61);
                        tcgen05_fence_after();
                    }
                    return may_write;
                };
                if (__any_sync(0xffffffffu, (best - m) * f > kMaxLead)) {
                    if (!(ok = until_done())) break;
                    const float now = fmaxf(m, best), base = now == -INFINITY ? 0.f : now;
                    const float shrink = exp2_approx((m - base) * f);  // 0 from -infinity on
                    m = now;
                    // x f - m f in one step keeps the rounding of m f: half a unit in its last place, which would be most of P's
                    // range, and more, for large scores.
                    far = __any_sync(0xffffffffu, fabsf(base * f) >= kFar) != 0;
                    sub1 = (far ? 0.f : -base * f) + (BF16 ? kRoomBf16 : kRoom);
                    l.x *= shrink, l.y *= shrink;
                    if (j > 0) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            tcgen05_ld_32x32b_x32(to + c, o);
                            tcgen05_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * shrink);
                            tcgen05_st_32x32b_x32(to + c, o);
                        }
                        tcgen05_wait_st();
                    }
                }
                if (far) {
                    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[c][k] = __float_as_uint(__uint_as_float(x[c][k]) - base);
                }
                const float2 ff = make_float2(f, f), sub = make_float2(sub1, sub1);
                auto quarter = [&](const uint32_t (&w)[32], uint32_t *p) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 t = fma2(make_float2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1])), ff, sub);
                        const float2 e = make_float2(exp2_approx(t.x), exp2_approx(t.y));
                        l = add2(l, e);
                        p[k] = E::from_float2(e.x, e.y);
                    }
                };
                auto hand_over = [&](int half) {
                    tcgen05_wait_st();
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.p_half[s] + half);
                };
                uint32_t p0[32], p1[32];
                quarter(x[0], p0);
                quarter(x[1], p0 + 16);
                if (!(ok = until_done())) break;
                tcgen05_st_32x32b_x32(tp, p0);
                quarter(x[2], p1);  // while the first half is stored
                hand_over(0);
                quarter(x[3], p1 + 16);
                // l goes to the warps that write the output.  They have read what is there from the unit before the last: P of this
                // unit could only be written after a product that waited for them.
                if (j == n - 1) reinterpret_cast<float *>(smem + L::kSums)[((n_sum & 1) * 2 + s) * kTile + r] = l.x + l.y;
                tcgen05_st_32x32b_x32(tp + 32, p1);
                hand_over(1);
            }
            if (!ok) break;
            ++n_sum;
            done_unit();
        }
    }

    // ---------------------------------------------------------------- teardown
    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) latch_error(a.status, PD_ERR_DEVICE_TIMEOUT, static_cast<uint32_t>(*abort_flag));
        for (int i = 0; i < 64; ++i) __nanosleep(10000);  // copies that may still be in flight
        __syncthreads();
    }
    if (warp == 9) {
        tcgen05_fence_after();
        tcgen05_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0) {  // the last block puts the counters back to zero for the next call
        __threadfence();
        if (atomicAdd(a.counters + 1, 1u) == gridDim.x - 1) {
            a.counters[0] = 0u;
            a.counters[1] = 0u;
        }
    }
}

bool make_heads_map(CUtensorMap *map, const HeadsView &x, int tokens, int heads, int head_dim, bool bf16) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(x.head_stride) * 2, static_cast<cuuint64_t>(x.token_stride) * 2};
    const cuuint32_t box[3] = {64, 1, kTile};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(x.ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool BF16>
pd_status launch(const PromptArgs &a, cudaStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    if (!ensure_dynamic_smem(attn_prompt_kernel<D, BF16>, PromptSmem<D>::kTotal, done)) return PD_ERR_CUDA;
    CUtensorMap mq, mk, mv;
    if (!make_heads_map(&mq, a.q, a.n_tokens, a.q_heads, D, BF16) || !make_heads_map(&mk, a.k, a.n_tokens, a.kv_heads, D, BF16) ||
        !make_heads_map(&mv, a.v, a.n_tokens, a.kv_heads, D, BF16))
        return PD_ERR_CUDA;
    const bool by_head = (a.q_heads / a.kv_heads) % 2 == 0;
    const int64_t tiles = a.n_tokens / (by_head ? kTile : 2 * kTile) + a.n_seqs;
    const int64_t ids = tiles * (by_head ? a.q_heads / 2 : a.q_heads);
    if (ids > INT32_MAX / 2) return PD_ERR_UNSUPPORTED_SHAPE;
    const int grid = static_cast<int>(ids < sm_count() ? ids : sm_count());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = PromptSmem<D>::kTotal;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the set-up may run while the previous kernel drains
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, attn_prompt_kernel<D, BF16>, mq, mk, mv, a);
    if (e != cudaSuccess) return PD_ERR_CUDA;
    count_launch();
    return cuda_ok(cudaGetLastError());
}

}  // namespace

pd_status launch_attn_prompt(const PromptArgs &a, bool bf16, cudaStream_t stream) {
    if (a.head_dim == 128) return bf16 ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
    return bf16 ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
}

}  // namespace pd
