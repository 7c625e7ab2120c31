// Attention of several new tokens a sequence over the 8-bit paged cache: out[i, h] = sum_{j <= l - n + i} softmax_j(scale q[i, h] . K[j, g]) V[j, g]
// for the n new tokens of a sequence that has l tokens with them, K and V being codes (signed 8 bits) times the scale of their page and head.
//
// Softmax in one pass over the keys, base 2, 32-bit statistics, as in pd_attn_prompt: the reference maximum m of a row moves only when a score
// passes it by more than 8.  Codes are exact in both 16-bit types, so that the products take them as they are: S = q C_k^T in the queries'
// type, O = P C_v in binary16.  The scales go into the exponents.  With s_k, s_v the scales of a key's page and r a power of two,
//     P = 2^(f s_k S - m + log2(s_v / r) + 7),   l = sum P r / s_v,   out = r O / l.
// P is rounded to binary16, 2^-11 of a weight at most, what a binary16 output loses by its own rounding: the tensor cores take 16-bit weights, and a
// second product with what is left of them would add 1024 of a tile's 2048 clocks of products.
// r is a reference for the pages' scales of V: s_v / r is in [2^-7, 1], so that P stays normal in binary16 where the weight is above 2^-14.
// Where a tile's pages differ by more than that it is gone through again for the others, the smallest first, which happens to hardly any cache.
// Each row has an r of its own, which follows only where the row attends to a page that is taken: pages of later tokens, however large or
// small, do nothing to its O.  What a row attends to of its last tile is taken before or with larger pages of that tile.
//
// A *unit* is 256 or fewer rows of a sequence and key/value head; a row is a token and one of the query heads that share the head,
// heads first.  Two slots of 128 rows (the rows that one product of the tensor cores takes) read the same keys:
//   by rows : 129 to 256 rows, 128 to each slot
//   by keys : up to 128 rows, which both slots hold; the tiles of 128 keys go to the slots in turn, and the two results are joined in
//             tensor memory at the end.  With few rows the kernel is bound by the codes that it reads, and one slot's chain of
//             product, softmax, product would be longer than its tile's loads.
// The keys of all units, one unit after another, are dealt to the blocks in ranges of equal cost whatever the lengths are; where a
// range ends inside a unit the parts are joined by a second kernel, in the order of the keys: results do not depend on the schedule.
//
// Bound.  By rows a tile of 128 keys is 2048 clocks of products and 2048 of the 16 exponentials a clock that an SM has, by keys the 32 KB of its
// codes, 1370 clocks of the SM's share of the memory.  Measured: 2048 tokens behind 16384, 64 heads on 8: 1.24 ms, 0.94 PFLOP/s, 4550 clocks a
// tile; 64 sequences of 4 tokens, 288 thousand keys (600 MB): 262 us, 3950 clocks a tile.  By rows the softmax's warps are busy all the time: half
// with the exponentials of both slots, half with the latencies of waits, loads and scales between them.  By keys it is the conversion: 16 KB
// of codes take 900 to 1200 clocks, two of them a tile, with 300 clocks of waits each; its 64 KB of stores alone keep the shared memory busy
// for 600.  Both suffer when the code of the 16 warps' roles does not fit into the SM's cache for instructions: the waits, loops and rings
// are written for that (counters: warps that wait for instructions 1.2 -> 0.3 an issue, 1.33 -> 1.27 ms;
// one search for the reference of V's scales in the place of two: 1.29 -> 1.24 ms).
// Tried and dropped: P in the place of the scores with both passes over them from tensor memory in loops (1.46 ms), two threads a row (2.5 ms: 24
// warps), 8 warps for the conversion (no change), codes through registers instead of a ring in shared memory (1.75 ms, code too long).
//
// Roles: warps 0-3 and 4-7 the softmax of slot 0 and 1, and the outputs; warp 8 units and pages; warp 11 copies; warps 9 and 10 the products with the keys
// and with the values; warps 12-15 turn codes into 16-bit operands.  Every wait on another role is bounded.
#include "pd_attn.cuh"
#include "pd_attn_mma.cuh"

namespace pd {
namespace {

constexpr int kTile = 128;  // rows of a slot, keys of a tile
constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kSteps = 4;       // steps that the producer may be ahead
constexpr int kReaders = 15;   // warps that read a step
constexpr int kMaxGrid = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMaxLead = 8.f;  // how far (base-2 exponent) a score may pass the reference maximum
constexpr float kFar = 1024.f;   // reference maxima from which on scores are rounded before it is taken off
constexpr float kRoom = 7.f;     // P is 2^7 times the weight, and at most 2^15
constexpr float kSmallestScale = 0x1p-120f;  // a page whose scale is below it counts as zeros
constexpr int kSpread = 7;       // pages of V whose scale is below 2^-7 of the reference are taken in another step
// Shares of the reference that are smaller count as so much: P, 2^(8 + 7) times it at most, is zero in binary16 either way, and the reciprocal, which
// the weights' sum takes it times, stays finite.
constexpr float kLeastShare = 0x1p-60f;
constexpr int kNoRef = -1000;    // of a row that has seen no values but zeros
constexpr int kMostFall = 60;    // how far the reference may fall: O, in its units, grows by as much
constexpr uint32_t kColS = 0, kColP = 128, kColO = 256;  // tensor-memory columns; slot 1: P + 64, O + 128

// What a step costs, in the same units for all: a tile of keys by rows keeps the tensor cores and the exponentials busy for 2048 clocks, by
// keys its copies take about two thirds of that.
constexpr int kCostRows = 3, kCostKeys = 2;  // per key
constexpr int kCostUnit = 3 * kTile;         // what a unit costs beside its keys, in keys
constexpr int kMinKeys = 3 * kTile;          // a block gets so many keys (by keys) at least

enum : int { kSlot0 = 1, kSlot1 = 2, kEnd = 4, kExit = 8, kByKeys = 16 };

struct Step {
    int flags, key0;       // first key of the tile
    int limit;             // last key that the unit's first token attends to
    int ref;               // r = 2^ref for the rows that attend to a key from `first_taken` on
    int token, n_tokens;   // the unit's first token (row of q) and tokens
    int head, done_heads;  // first query head of the rows, and heads from it on that are another unit's
    int part;              // where a part of a unit goes; -1: the whole unit, written to out
    int tainted;           // first key of a page whose scale is not finite
    int first_taken;       // first key, counted from the tile's, whose page's values are not zeros and are taken in this step
    int pad;
    // for keys 16 g .. 16 g + 15 of the tile
    float4 factor[8];      // of the scores, twice, and log2(s_v / r), twice: pairs as the packed arithmetic takes them
    float weight[8];       // r / s_v
    uint32_t place[8];     // of their codes, in blocks of 16 keys from the cache's first; kNoKeys; kZeroValues: the values are zero whatever their codes are
};
static_assert(sizeof(Step) == 240, "layout");
constexpr uint32_t kNoKeys = 0xffffffffu, kZeroValues = 0x80000000u;

struct Bars {
    uint64_t step_full[kSteps], step_empty[kSteps];
    uint64_t raw_full[8], raw_empty[8];
    uint64_t kv_full[8], kv_empty[8];
    uint64_t q_full, q_empty, s_full[2], s_free, p_half[2][2], o_done[2], o_last, o_empty[2], joined;
    uint32_t tmem;
    int abort_flag;
};

template <int D>
struct ChunkSmem {
    static constexpr int kTileBytes = kTile * D * 2, kRawBytes = kTile * D;
    static constexpr int kStages = D == 128 ? 3 : 6, kRaw = D == 128 ? 4 : 8;
    static constexpr int kQ = 0;
    static constexpr int kRing = 2 * kTileBytes;
    static constexpr int kRawRing = kRing + kStages * kTileBytes;
    static constexpr int kStepRing = kRawRing + kRaw * kRawBytes;
    static constexpr int kSums = kStepRing + kSteps * static_cast<int>(sizeof(Step));  // m, l and reference of slot 1's rows, by keys
    static constexpr int kBars = kSums + kTile * 12;
    static constexpr int kTotal = kBars + 512;
    static constexpr int kScan = kRawRing;  // costs before each thread's share of the sequences, until the first unit is found
    static_assert(sizeof(Bars) <= 512 && kTotal <= 227 * 1024 && (kThreads + kWarps) * 8 <= kRaw * kRawBytes, "shared memory");
};

// A part of a unit: rows of O (binary32, in units of r) as [head_dim / 4][256 rows][4], then {m, l, ref, -} of each row.
template <int D>
constexpr int kPartFloats = 256 * D + 256 * 4;

__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 x;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ void sts128(uint32_t at, const uint4 &x) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}

__device__ __forceinline__ bool mbar_sleep_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000) : "memory");
    return ok != 0;
}

// A place in a ring of N stages, and the parity of its round.
template <uint32_t N>
struct Ring {
    uint32_t stage = 0, parity = 0;
    __device__ __forceinline__ void forward(uint32_t n) {
        stage += n;
        if (stage >= N) stage -= N, parity ^= 1u;
    }
};

// Units of a sequence's rows that read one key/value head (a *stream*), and what they cost.
struct Stream {
    int64_t held;   // tokens before the new ones
    int n, span;    // new tokens, tokens of a unit by rows
    __device__ __forceinline__ int whole() const { return n / span; }
    __device__ __forceinline__ int rest() const { return n % span; }
    __device__ __forceinline__ int units() const { return whole() + (rest() ? 1 : 0); }
    __device__ __forceinline__ bool by_keys(int i) const { return i == whole() && 2 * rest() <= span; }
    __device__ __forceinline__ int64_t keys(int i) const { return held + min(n, (i + 1) * span); }
    __device__ __forceinline__ int per_key(int i) const { return by_keys(i) ? kCostKeys : kCostRows; }
    __device__ __forceinline__ int64_t cost(int i) const { return per_key(i) * (keys(i) + kCostUnit); }
    __device__ __forceinline__ int64_t before(int64_t i) const {  // the first i units, all by rows
        return kCostRows * (i * (held + kCostUnit) + span * (i * (i + 1) / 2));
    }
    __device__ __forceinline__ int64_t total() const { return before(whole()) + (rest() ? cost(whole()) : 0); }
};

struct Place {  // a tile of a unit
    int b, stream, unit, tile;
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) attn_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const ChunkArgs a) {
    using E = Elem<BF16>;
    using L = ChunkSmem<D>;
    constexpr int kStages = L::kStages, kRaw = L::kRaw;
    constexpr int kPieces = D / 64;  // sub-tiles of 64 columns
    constexpr int kPieceBytes = kTile * 64 * 2;
    extern __shared__ __align__(1024) unsigned char smem[];  // the swizzle counts from 1024-byte boundaries
    Bars &bar = *reinterpret_cast<Bars *>(smem + L::kBars);
    Step *steps = reinterpret_cast<Step *>(smem + L::kStepRing);
    volatile int *abort_flag = &bar.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.q_heads / a.kv_heads, chunks = (group + kTile - 1) / kTile, heads = (group + chunks - 1) / chunks;  // heads of a row's token
    const int slot_tokens = kTile / heads;
    const int per_seq = a.kv_heads * chunks;  // streams
    const int page = 1 << a.page_log2;
    const int64_t room = static_cast<int64_t>(a.table_width) << a.page_log2;
    // Bounded: a question sleeps for up to 20 us, and there are 2^16 of them.  The first one to give up says where, and the block's last act
    // is to report it.  Short, because it is in the code of every role many times over.  On a barrier that has not been used yet the
    // phase before the first one counts as over, so that who waits for "the use before mine" need not know whether there was one.
    auto wait_warp = [&](uint64_t *b, uint32_t parity, int where) {
        int left = 1 << 16;
#pragma unroll 1
        while (!__all_sync(0xffffffffu, mbar_sleep_wait(smem_u32(b), parity & 1u)) && --left) {}
        if (!left) *abort_flag = where;
        return left != 0;
    };

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSteps; ++i) mbar_init(bar.step_full + i, 1), mbar_init(bar.step_empty + i, kReaders);
        for (int i = 0; i < kRaw; ++i) mbar_init(bar.raw_full + i, 1), mbar_init(bar.raw_empty + i, 4);
        for (int i = 0; i < kStages; ++i) mbar_init(bar.kv_full + i, 4), mbar_init(bar.kv_empty + i, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar.s_full + s, 1), mbar_init(bar.p_half[s], 4), mbar_init(bar.p_half[s] + 1, 4);
            mbar_init(bar.o_done + s, 1), mbar_init(bar.o_empty + s, s == 0 ? 4 : 8);
        }
        mbar_init(&bar.q_full, 1), mbar_init(&bar.q_empty, 1), mbar_init(&bar.s_free, 4), mbar_init(&bar.o_last, 1), mbar_init(&bar.joined, 4);
        bar.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 9) tcgen05_alloc(&bar.tmem, 512);
    if (warp == 8 && lane == 0) prefetch_tensormap(&map_q);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // everything before touches no memory of the caller's

    // ---------------------------------------------------------------- costs before each thread's share of the sequences
    auto stream_of = [&](int b, int &first) {  // sequences with lengths out of range have no new tokens
        first = __ldg(a.cu_seqlens + b);
        const int last = __ldg(a.cu_seqlens + b + 1), len = __ldg(a.seq_lens + b);
        Stream s = {0, 0, 2 * slot_tokens};
        if (first >= 0 && last >= first && last <= a.n_tokens && last - first <= a.max_new && len >= last - first && len <= room)
            s.n = last - first, s.held = len - s.n;
        else if (blockIdx.x == 0) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(b));
        return s;
    };
    int64_t *scan = reinterpret_cast<int64_t *>(smem + L::kScan), *warp_sum = scan + kThreads;
    const int share = (a.n_seqs + kThreads - 1) / kThreads;
    int64_t sum = 0;
    for (int b = threadIdx.x * share; b < min(a.n_seqs, static_cast<int>(threadIdx.x + 1) * share); ++b) {
        int first;
        sum += stream_of(b, first).total();
    }
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    if (lane == 31) warp_sum[warp] = incl;
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    int64_t before = 0, total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += warp_sum[w];
        total += warp_sum[w];
    }
    scan[threadIdx.x] = before + incl - sum;
    __syncthreads();
    total *= per_seq;
    const uint32_t tmem = bar.tmem;
    const int64_t least = static_cast<int64_t>(kCostKeys) * kMinKeys;
    const int n_blocks = static_cast<int>(max(static_cast<int64_t>(1), min(static_cast<int64_t>(gridDim.x), total / least)));

    // The next step, in the producer's order: every other role reads what the producer wrote.
    uint32_t n_step = 0;
    auto next_step = [&]() { return wait_warp(bar.step_full + n_step % kSteps, n_step / kSteps, 50); };
    auto done_step = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar.step_empty + n_step % kSteps);
        ++n_step;
    };

    if (warp >= 8 && warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 8) {
        // ------------------------------------------------------------ units, pages and copies
        // Block c's range starts at c / n_blocks of the total cost; a cut within a sixteenth of a range of a unit's end moves there.
        const int snap = static_cast<int>(total / n_blocks / (16 * kCostRows * kTile)) + 1;
        auto place_of = [&](int c) {
            Place p = {a.n_seqs, 0, 0, 0};
            if (c >= n_blocks) return p;
            const int64_t x = total / n_blocks * c + total % n_blocks * c / n_blocks;
            constexpr int kStep = kThreads / 32;
            int at = (31 - __clz(__ballot_sync(0xffffffffu, scan[lane * kStep] * per_seq <= x))) * kStep;
            at += 31 - __clz(__ballot_sync(0xffffffffu, lane < kStep && scan[at + min(lane, kStep - 1)] * per_seq <= x));
            int64_t rest = x - scan[at] * per_seq;
            int b = at * share, first;
            Stream s = stream_of(min(b, a.n_seqs - 1), first);
            while (b < a.n_seqs && rest >= s.total() * per_seq) {
                rest -= s.total() * per_seq;
                if (++b < a.n_seqs) s = stream_of(b, first);
            }
            if (b >= a.n_seqs) return p;
            p.b = b;
            p.stream = static_cast<int>(rest / s.total());
            rest -= p.stream * s.total();
            int lo = 0, hi = s.units() - 1;  // the last unit that starts at or before rest
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s.before(mid) <= rest) lo = mid;
                else hi = mid - 1;
            }
            p.unit = lo;
            rest = (rest - s.before(lo)) / s.per_key(lo) - kCostUnit;
            const int tiles = static_cast<int>((s.keys(lo) + kTile - 1) / kTile);
            p.tile = rest <= 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(tiles), (rest + kTile / 2) / kTile));
            if (p.tile < snap) p.tile = 0;
            else if (tiles - p.tile < snap) p.tile = tiles;
            return p;
        };
        Place at = {}, end = {};
#pragma unroll 1
        for (int i = 0; i < 2; ++i) at = end, end = place_of(blockIdx.x + i);
        __syncwarp();  // the scan's place is the copies' from here on
        bool ok = true;
        int header[2] = {0, 0};  // of the block's two parts: 1 there, 2 the unit's last
        int4 header_unit = make_int4(0, 0, 0, 0);
        int first = 0;
        Stream s = {0, 0, 1};
        int known = -1;  // the sequence that s is of
        while (ok && at.b < a.n_seqs) {
            if (known != at.b) s = stream_of(at.b, first), known = at.b;
            const bool last_unit = at.b == end.b && at.stream == end.stream && at.unit == end.unit;
            if (at.b > end.b || (at.b == end.b && (at.stream > end.stream || (at.stream == end.stream && at.unit > end.unit)))) break;
            if (at.unit < s.units()) {
                const int keys = static_cast<int>(s.keys(at.unit)), tiles = (keys + kTile - 1) / kTile;
                const int t0 = at.tile, t1 = last_unit ? end.tile : tiles;
                if (t0 < t1) {
                    const bool by_keys = s.by_keys(at.unit);
                    // Shares that do not divide the group evenly overlap: every row has a query of this key/value head, or none of the unit's tokens.
                    const int kvh = at.stream / chunks, done_heads = max((at.stream - kvh * chunks + 1) * heads - group, 0);
                    const int head = kvh * group + (at.stream - kvh * chunks) * heads - done_heads;
                    const int token = first + at.unit * s.span, n_tok = min(s.span, s.n - at.unit * s.span);
                    const int limit = static_cast<int>(s.held) + at.unit * s.span;
                    const int last0 = by_keys ? keys - 1 : limit + slot_tokens - 1;  // last key of slot 0's last token
                    int part = -1;
                    if (t0 > 0 || t1 < tiles) {
                        const int slot = t0 > 0 ? 0 : 1;
                        part = blockIdx.x * 2 + slot;
                        header[slot] = t1 == tiles ? 2 : 1;
                        if (slot == 1) header_unit = make_int4(token, n_tok, head, done_heads);
                    }
                    // A lane knows 16 keys of four tiles, and the page of 16 keys of the next four.
                    const int key_end = min(keys, t1 * kTile);
                    const int32_t *table = a.block_table + at.b * a.table_stride;
                    auto page_of = [&](int quad) {
                        const int key = quad * (4 * kTile) + lane * 16;
                        return key < key_end ? __ldg(table + (key >> a.page_log2)) : 0;
                    };
                    int quad = t0 >> 2;
                    int64_t pid = 0;
                    float sk = 0.f, sv = 0.f, sk_next = 0.f, sv_next = 0.f;
                    int pid_next = page_of(quad);
                    bool good = false, look = false;
                    auto scales_of = [&](int q, int64_t p, float &k, float &v) {
                        const bool there = q * (4 * kTile) + lane * 16 < key_end;
                        k = v = 0.f;
                        if (there && (p < 0 || p >= a.n_pages)) latch_error(a.status, PD_ERR_BAD_INDEX, static_cast<uint32_t>(at.b));
                        else if (there) k = a.pages[0].scale[p * a.kv_heads + kvh], v = a.pages[1].scale[p * a.kv_heads + kvh];
                    };
                    scales_of(quad, pid_next, sk_next, sv_next);
                    int tainted = INT32_MAX, ref = kNoRef, top = kNoRef, said = kNoRef, turn = 0;  // said: the reference of what was last taken
                    const float f0 = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 0.f;
                    float inverse = 0.f;  // 2^-ref
                    float4 entry = make_float4(0.f, 0.f, 0.f, 0.f);  // of the lane's 16 keys: factor, log2(s_v / r), r / s_v, place
                    bool even = false;                               // the four tiles have one reference
                    unsigned counts = 0;                             // lanes whose keys' values are not zeros and are taken
                    uint32_t place = kNoKeys;
                    --quad;
                    for (int j = t0; j < t1 && ok; ++j) {
                        if ((j >> 2) != quad) {
                            quad = j >> 2;
                            pid = pid_next, sk = sk_next, sv = sv_next;
                            const int key = quad * (4 * kTile) + lane * 16;
                            good = key < key_end && pid >= 0 && pid < a.n_pages;
                            // what reads as NaN makes the rows that see it NaN, and nothing else
                            const bool bad = good && !(fabsf(sk) <= 3.402823466e38f && fabsf(sv) <= 3.402823466e38f);
                            if (__any_sync(0xffffffffu, bad)) tainted = min(tainted, __reduce_min_sync(0xffffffffu, bad ? key & ~(page - 1) : INT32_MAX));
                            if (bad) sk = sv = 0.f;
                            if (!(sk >= kSmallestScale)) sk = 0.f;
                            if (!(sv >= kSmallestScale)) sv = 0.f;
                            place = good ? static_cast<uint32_t>((pid * a.kv_heads + kvh) << (a.page_log2 - 4)) + ((lane * 16 & (page - 1)) >> 4) : kNoKeys;
                            if (good && sv == 0.f) place |= kZeroValues;
                            even = false, look = true;
                            pid_next = page_of(quad + 1);
                        }
                        const int key0 = j * kTile;
                        unsigned todo = 0xffu << (8 * (j & 3));  // lanes whose keys are still to be taken
                        while (todo && ok) {
                            if (!even) {
                                // One reference for all four tiles, or for what one tile has left.  The smallest scales first: what a row attends to of a tile
                                // is done before or with the larger pages behind it, so that those move no reference that it still needs.
                                bool now = look || (todo >> lane) & 1u;
                                // positive numbers order like their bits
                                const float least = __uint_as_float(__reduce_min_sync(0xffffffffu, now && sv > 0.f ? __float_as_uint(sv) : 0x7f800000u));
                                const float most = __uint_as_float(__reduce_max_sync(0xffffffffu, now && sv <= least * (1 << (kSpread - 1)) ? __float_as_uint(sv) : 0u));
                                bool all = false;  // whatever is below the reference, down to nothing, is taken with it
                                if (most > 0.f && (most * inverse > 1.f || least * inverse < 1.f / (1 << kSpread))) {
                                    const int e = static_cast<int>(__float_as_uint(most) >> 23) - 126;  // most <= 2^e <= 2^128
                                    ref = max(e, top - kMostFall), top = max(top, ref), all = ref > e;
                                    inverse = __uint_as_float(ref < 127 ? static_cast<uint32_t>(127 - ref) << 23 : 1u << (149 - ref));
                                }
                                const float rel = sv * inverse, held = fmaxf(rel, kLeastShare);
                                now = now && (sv == 0.f || (rel <= 1.f && (all || rel >= 1.f / (1 << kSpread))));
                                const unsigned taken = __ballot_sync(0xffffffffu, now);
                                counts = __ballot_sync(0xffffffffu, now && sv > 0.f);
                                if (look) {
                                    look = false, even = taken == 0xffffffffu;
                                    if (!even) continue;
                                }
                                entry = make_float4(fmaxf(f0 * sk, 0x1p-149f), !now ? -INFINITY : (sv == 0.f ? 0.f : __log2f(held)),
                                                    !now ? 0.f : (sv == 0.f ? 1.f : __frcp_rn(held)), __uint_as_float(place));
                                todo &= ~taken;
                            } else {
                                todo = 0;
                            }
                            const bool holds = (lane >> 3) == (j & 3);  // the lane knows a group of the tile
                            const unsigned mine = (counts >> (8 * (j & 3))) & 0xffu;
                            if (mine) said = ref;
                            int flags = by_keys ? kByKeys | (turn & 1 ? kSlot1 : kSlot0) : kSlot1 | (key0 <= last0 ? kSlot0 : 0);
                            ++turn;
                            const uint32_t ss = n_step % kSteps, sr = n_step / kSteps;
                            if (!(ok = wait_warp(bar.step_empty + ss, sr - 1, 51))) break;
                            Step &st = steps[ss];
                            if (holds) {
                                st.factor[lane & 7] = make_float4(entry.x, entry.x, entry.y, entry.y);
                                st.weight[lane & 7] = entry.z, st.place[lane & 7] = __float_as_uint(entry.w);
                            }
                            if (lane == 0) {
                                *reinterpret_cast<int4 *>(&st.flags) = make_int4(flags, key0, limit, said);
                                *reinterpret_cast<int4 *>(&st.token) = make_int4(token, n_tok, head, done_heads);
                                st.first_taken = 16 * (__ffs(mine | 0x100u) - 1);
                            }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar.step_full + ss);
                            ++n_step;
                        }
                        if ((j & 3) == 2 || (j == t0 && (j & 3) == 3)) scales_of(quad + 1, pid_next, sk_next, sv_next);
                    }
                    if (!ok) break;
                    const uint32_t ss = n_step % kSteps, sr = n_step / kSteps;
                    if (!(ok = wait_warp(bar.step_empty + ss, sr - 1, 51))) break;
                    if (lane == 0) {
                        Step &st = steps[ss];
                        st.flags = kEnd | (by_keys ? kByKeys : 0), st.limit = limit, st.token = token, st.n_tokens = n_tok, st.head = head, st.done_heads = done_heads;
                        st.part = part, st.tainted = tainted;
                        mbar_arrive(bar.step_full + ss);
                    }
                    ++n_step;
                }
            }
            if (last_unit) break;
            at.tile = 0;
            if (++at.unit >= s.units()) {
                at.unit = 0;
                if (++at.stream == per_seq || s.units() == 0) at.stream = 0, ++at.b;
            }
        }
        if (ok) {
            const uint32_t ss = n_step % kSteps, sr = n_step / kSteps;
            if (wait_warp(bar.step_empty + ss, sr - 1, 51)) {
                if (lane == 0) {
                    steps[ss].flags = kExit;
                    mbar_arrive(bar.step_full + ss);
                }
            }
        }
        if (lane == 0) {
            a.headers[blockIdx.x * 4] = make_int4(header[0], header[1], slot_tokens, heads);
            a.headers[blockIdx.x * 4 + 1] = header_unit;
        }
        } else if (warp == 11) {
        // ------------------------------------------------------------ copies: keys of a step, values of the one before, queries of a unit
        uint32_t n_unit = 0, n_raw = 0, place_v = kNoKeys;
        bool ok = true, fresh = true, first = true;
        const uint32_t bytes = static_cast<uint32_t>(page) * D;
        const bool starts = lane < 8 && ((lane * 16) & (page - 1)) == 0;  // the lane's 16 keys are the first ones of a page
        auto copy = [&](int kv, uint32_t place) {
            const uint32_t rs = n_raw % kRaw, rr = n_raw / kRaw;
            if (!(ok = wait_warp(bar.raw_empty + rs, rr - 1, 52))) return;
            ++n_raw;
            const bool there = place != kNoKeys, zeros = there && kv == 1 && (place & kZeroValues);  // a page of V that stands for zeros, whatever its codes are
            unsigned char *to = smem + L::kRawRing + rs * L::kRawBytes + lane * 16 * D;
            const bool copies = there && starts && !zeros;
            const unsigned who = __ballot_sync(0xffffffffu, copies);
            if (__any_sync(0xffffffffu, zeros)) {
                if (zeros)
                    for (int i = 0; i < D; ++i) reinterpret_cast<uint4 *>(to)[i] = make_uint4(0, 0, 0, 0);
                fence_proxy_async_smem();
                __syncwarp();
            }
            if (lane == 0) mbar_arrive_expect_tx(bar.raw_full + rs, __popc(who) * bytes);
            __syncwarp();
            if (copies) bulk_load_1d(to, a.pages[kv].codes + static_cast<int64_t>(place & ~kZeroValues) * (16 * D), bytes, bar.raw_full + rs);
        };
        while (ok && next_step()) {
            const Step &st = steps[n_step % kSteps];
            const int flags = __shfl_sync(0xffffffffu, st.flags, 0), token = st.token, head = st.head;
            const uint32_t place = lane < 8 ? st.place[lane] : kNoKeys;
            done_step();
            if (flags & kEnd) {
                fresh = true;
                continue;
            }
            // one loop for both, so that the code for a copy is there once
#pragma unroll 1
            for (int kv = flags & kExit ? 1 : 0; kv < (first ? 1 : 2) && ok; ++kv) copy(kv, kv == 0 ? place : place_v);
            if (flags & kExit) break;
            first = false, place_v = place;
            if (ok && fresh) {
                fresh = false;
                if (!(ok = wait_warp(&bar.q_empty, n_unit - 1, 53))) break;
                ++n_unit;
                if (lane == 0) {
                    const int slots = flags & kByKeys ? 1 : 2;
                    mbar_arrive_expect_tx(&bar.q_full, slots * kPieces * slot_tokens * heads * 128);
#pragma unroll 1
                    for (int i = 0; i < slots; ++i)
#pragma unroll
                        for (int p = 0; p < kPieces; ++p)
                            tma_load_3d(&map_q, &bar.q_full, smem + L::kQ + i * L::kTileBytes + p * kPieceBytes, p * 64, head, token + i * slot_tokens);
                }
                __syncwarp();
            }
        }
        } else if (warp == 9) {
        // ------------------------------------------------------------ S = Q K^T
        const uint32_t idesc = kIdescBase<BF16> | (a.scale < 0.f ? 1u << 13 : 0u) | (static_cast<uint32_t>(kTile >> 3) << 17) | (static_cast<uint32_t>(kTile >> 4) << 24);  // bit 13: A negated
        const uint32_t q_desc = desc_lower(smem + L::kQ, 16), k_desc = desc_lower(smem + L::kRing, 16);
        uint32_t n_s = 0, n_unit = 0;
        Ring<kStages> at;  // keys of step j are item 2 j - 1, the first ones item 0
        bool ok = true, fresh = true, begun = false;
        while (ok && next_step()) {
            const int flags = __shfl_sync(0xffffffffu, steps[n_step % kSteps].flags, 0);
            done_step();
            if (flags & kExit) break;
            if (flags & kEnd) {
                commit_elected(&bar.q_empty);
                fresh = true, ++n_unit;
                continue;
            }
            if (fresh && !(ok = wait_warp(&bar.q_full, n_unit, 55))) break;
            fresh = false;
            const uint32_t st = at.stage;
            if (!(ok = wait_warp(bar.kv_full + st, at.parity, 54))) break;
            const uint32_t k = k_desc + st * (L::kTileBytes >> 4);
#pragma unroll 1  // the instructions of the roles that run together have to fit into the caches for them
            for (int s = 0; s < 2; ++s) {
                if (!(flags & (kSlot0 << s))) continue;
                if (!(ok = wait_warp(&bar.s_free, n_s - 1, 56))) break;
                ++n_s;
                tcgen05_fence_after();
                const uint32_t q = q_desc + (flags & kByKeys ? 0 : s) * (L::kTileBytes >> 4);
                if (elect_one()) {
                    uint32_t off = 0;
#pragma unroll 1
                    for (int kk = 0; kk < D / 16; ++kk) {
                        mma_smem_a(tmem + kColS, make_desc(q + off), make_desc(k + off), idesc, kk > 0);
                        off += kk == 3 ? (kPieceBytes - 96) >> 4 : 32 >> 4;
                    }
                }
                commit_elected(bar.s_full + s);
            }
            if (ok) commit_elected(bar.kv_empty + st);
            at.forward(begun ? 2 : 1), begun = true;
        }
        } else if (warp == 10) {
        // ------------------------------------------------------------ O += P V, in binary16
        constexpr uint32_t kIdesc = kIdescBase<false> | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (static_cast<uint32_t>(kTile >> 4) << 24);
        const uint32_t v_desc = desc_lower(smem + L::kRing, kPieceBytes);
        uint32_t n_unit = 0, phase_p = 0, fresh = 3;  // bit s: slot s
        Ring<kStages> at;  // values of step j are item 2 j + 2
        at.forward(2);
        bool ok = true;
        while (ok && next_step()) {
            const int flags = __shfl_sync(0xffffffffu, steps[n_step % kSteps].flags, 0);
            done_step();
            if (flags & kExit) break;
            if (flags & kEnd) {
                commit_elected(&bar.o_last);
                fresh = 3, ++n_unit;
                continue;
            }
            const uint32_t st = at.stage;
            if (!(ok = wait_warp(bar.kv_full + st, at.parity, 57))) break;
            const uint32_t v = v_desc + st * (L::kTileBytes >> 4);
            // The softmax's warps read one phase of o_last a unit and arrive on o_empty behind it: the next one must not end before all have,
            // those of a slot that no tile of the unit belongs to among them.
            if (fresh == 3) {
#pragma unroll 1
                for (int s = 0; s < 2 && ok; ++s) ok = wait_warp(bar.o_empty + s, n_unit - 1, 58);
                if (!ok) break;
            }
#pragma unroll 1
            for (int s = 0; s < 2; ++s) {
                if (!(flags & (kSlot0 << s))) continue;
                const uint32_t first = (fresh >> s) & 1u;
                fresh &= ~(1u << s);
#pragma unroll 1
                for (int half = 0; half < 2 && ok; ++half) {
                    if (!(ok = wait_warp(bar.p_half[s] + half, phase_p >> s, 60))) break;
                    tcgen05_fence_after();
                    const uint32_t v_half = v + half * (4 * 2048 >> 4), p_half = tmem + kColP + s * 64 + half * 32;
                    if (elect_one())
#pragma unroll 1
                    for (int kk = 0; kk < 4; ++kk)
                        tcgen05_mma_f16_tmem_a(tmem + kColO + s * 128, p_half + kk * 8, make_desc(v_half + kk * (2048 >> 4)), kIdesc, first && half + kk == 0 ? 0u : 1u);
                }
                if (!ok) break;
                phase_p ^= 1u << s;
                commit_elected(bar.o_done + s);
            }
            if (ok) commit_elected(bar.kv_empty + st);
            at.forward(2);
        }
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // ------------------------------------------------------------ codes to 16-bit operands in rows of 128 bytes with the 128-byte swizzle
        // Keys of a step, then values of the one before: K0 K1 V0 K2 V1 ..  So a step's keys are there before the values of the step
        // before have been asked for, and their place in the ring is that of values three steps back.
        const int t = threadIdx.x - 12 * 32;
        constexpr int kPer = D / 8, kRows = 128 / kPer;  // threads of a token, tokens side by side
        const int row0 = t / kPer, c = t % kPer;
        const uint32_t to0 = smem_u32(smem + L::kRing + (c / 8) * kPieceBytes + row0 * 128 + (((c & 7) ^ (row0 & 7)) << 4));
        uint32_t n_raw = 0;
        Ring<kStages> at;
        bool ok = true, begun = false;
        while (ok && next_step()) {
            const int flags = steps[n_step % kSteps].flags;
            done_step();
            if (flags & kEnd) continue;
            if ((flags & kExit) && !begun) break;
#pragma unroll 1
            for (int kv = flags & kExit ? 1 : 0; kv < (begun ? 2 : 1); ++kv, ++n_raw) {
                if (flags & kExit) at.forward(1);  // the last values' item is behind that of keys that there are none of
                const uint32_t rs = n_raw % kRaw, st = at.stage;
                if (!(ok = wait_warp(bar.raw_full + rs, n_raw / kRaw, 59))) break;
                if (!(ok = wait_warp(bar.kv_empty + st, at.parity ^ 1u, 65))) break;
                uint32_t from = smem_u32(smem + L::kRawRing + rs * L::kRawBytes + t * 8);
                uint32_t to = to0 + st * L::kTileBytes;  // a thread's rows are a multiple of 8 apart: the swizzle is the same for all
                // A short loop: eight loads and conversions written out take 500 clocks for 16 KB instead of 735 where nothing else runs, but
                // here the other roles' instructions then have to be fetched again and again (64 sequences of 4 tokens: 300 us beside 267).
                // Loads are ahead of the stores, which they must not pass.
                auto convert = [&](auto codes4) {
                    uint2 x = lds64(from), y = lds64(from + kRows * D);
#pragma unroll 1
                    for (int i = 0; i < kTile / kRows; i += 2) {
                        from += 2 * kRows * D;
                        const uint2 w0 = x, w1 = y;
                        if (i + 2 < kTile / kRows) x = lds64(from), y = lds64(from + kRows * D);
                        uint2 lo = codes4(w0.x), hi = codes4(w0.y);
                        sts128(to, make_uint4(lo.x, lo.y, hi.x, hi.y));
                        lo = codes4(w1.x), hi = codes4(w1.y);
                        sts128(to + kRows * 128, make_uint4(lo.x, lo.y, hi.x, hi.y));
                        to += 2 * kRows * 128;
                    }
                };
                if (!BF16 || kv == 1) {
                    // byte c ^ 0x80 under the upper byte 0x64 is 1024 + (c + 128), less 1152, exactly c
                    convert([](uint32_t w) {
                        w ^= 0x80808080u;
                        return make_uint2(hadd2_u32(prmt(w, 0x64646464u, 0x4140), 0xE480E480u), hadd2_u32(prmt(w, 0x64646464u, 0x4342), 0xE480E480u));
                    });
                } else {
                    // under the upper byte 0x43 the lower seven bits are 128 + those bits, and the sign bit alone is 128 or 256: their difference is c
                    convert([](uint32_t w) {
                        auto code2 = [](uint32_t v) {
                            uint32_t d;
                            asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(v & 0xff80ff80u), "r"(0xBF80BF80u), "r"(v & 0xff7fff7fu));
                            return d;
                        };
                        return make_uint2(code2(prmt(w, 0x43434343u, 0x4140)), code2(prmt(w, 0x43434343u, 0x4342)));
                    });
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.raw_empty + rs), mbar_arrive(bar.kv_full + st);
                at.forward(1);
            }
            begun = true;
            if (flags & kExit) break;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        // ------------------------------------------------------------ softmax and output: a thread owns one row of a slot
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const int my_token = row / heads, my_head = row - my_token * heads;
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t ts = lanes + kColS, tp = lanes + kColP + s * 64, to = lanes + kColO + s * 128;
        float2 *sums = reinterpret_cast<float2 *>(smem + L::kSums);
        int *sums_ref = reinterpret_cast<int *>(smem + L::kSums + kTile * 8);
        uint32_t n_s = 0, n_unit = 0, n_joined = 0;  // steps of the slot, units, units by keys so far
        int taken = 0, ref = kNoRef;                 // steps of the slot in the unit, the row's reference
        float m = -INFINITY, sub1 = 0.f;
        bool far = false, ok = true;
        float2 l = make_float2(0.f, 0.f);
        while (ok && next_step()) {
            const Step &st = steps[n_step % kSteps];
            const int flags = st.flags;
            if (flags & kExit) {
                done_step();
                break;
            }
            const bool by_keys = (flags & kByKeys) != 0;
            if (flags & kEnd) {
                const int token = st.token + (by_keys ? 0 : s * slot_tokens) + my_token, left = st.n_tokens - (by_keys ? 0 : s * slot_tokens);
                const int head = st.head + my_head, part = st.part;
                const bool valid = my_token < slot_tokens && my_token < left && my_head >= st.done_heads;
                const bool tainted = st.limit + (by_keys ? 0 : s * slot_tokens) + my_token >= st.tainted;
                done_step();
                float sum = l.x + l.y;
                if (tainted) sum = __int_as_float(0x7fc00000);
                if (by_keys && s == 1) {
                    // slot 0 has read what is there from the unit before
                    if (!(ok = wait_warp(bar.o_empty + 1, n_unit - 1, 66))) break;
                    sums[row] = make_float2(m, sum);
                    sums_ref[row] = ref;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar.joined);
                    // Slot 0 writes the output.  This one waits too, and says that it has: a barrier tells two phases apart, so that nobody may
                    // leave one out or come late.
                    if (!(ok = wait_warp(&bar.o_last, n_unit, 69))) break;
                    if (lane == 0) mbar_arrive(bar.o_empty + 1);
                } else {
                    float w0 = taken ? 1.f : 0.f, w1 = 0.f;  // weights of the slots' sums
                    int at = ref;
                    if (by_keys) {
                        if (!(ok = wait_warp(&bar.joined, n_joined, 63))) break;
                        const float2 other = sums[row];
                        if (other.x != -INFINITY || other.y != 0.f) {  // the same in most rows; a row without anything has nothing to add
                            const float top = fmaxf(m, other.x);
                            const float e0 = m == -INFINITY ? 0.f : exp2_approx(m - top), e1 = other.x == -INFINITY ? 0.f : exp2_approx(other.x - top);
                            const int other_ref = sums_ref[row];
                            at = max(ref, other_ref);
                            w0 = e0 * exp2_approx(static_cast<float>(ref - at)), w1 = e1 * exp2_approx(static_cast<float>(other_ref - at));
                            sum = sum * e0 + other.y * e1;
                            m = top;
                        }
                    }
                    const bool use0 = __any_sync(0xffffffffu, w0 != 0.f), use1 = __any_sync(0xffffffffu, w1 != 0.f);
                    if (!(ok = wait_warp(&bar.o_last, n_unit, 62))) break;
                    tcgen05_fence_after();
                    const float scale = __uint_as_float(static_cast<uint32_t>(126 + max(at, -125)) << 23), inv = 2.f / sum;  // r / 2, which is finite
                    uint16_t *y = static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + static_cast<int64_t>(token) * a.out.token_stride + head * a.out.head_stride;
                    float *po = a.partial + static_cast<int64_t>(max(part, 0)) * kPartFloats<D> + ((by_keys ? 0 : s * kTile) + row) * 4;
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        uint32_t o[16];
                        float x[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) x[k] = 0.f;
                        if (use0) {
                            tcgen05_ld_32x32b_x16(to + c, o);
                            tcgen05_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) x[k] = w0 != 0.f ? __uint_as_float(o[k]) * w0 : 0.f;
                        }
                        if (use1) {
                            tcgen05_ld_32x32b_x16(to + 128 + c, o);
                            tcgen05_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) x[k] = w1 != 0.f ? fmaf(__uint_as_float(o[k]), w1, x[k]) : x[k];
                        }
                        if (!valid) continue;
                        if (part < 0) {
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint32_t w[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) w[i] = E::from_float2(x[8 * k + 2 * i] * inv * scale, x[8 * k + 2 * i + 1] * inv * scale);
                                *reinterpret_cast<uint4 *>(y + c + 8 * k) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k) *reinterpret_cast<float4 *>(po + (c / 4 + k) * (256 * 4)) = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                        }
                    }
                    // m and the sum count where nothing is left of O in this part's reference, too
                    if (part >= 0 && valid) *reinterpret_cast<float4 *>(po + 256 * D) = make_float4(m, sum, static_cast<float>(at), 0.f);
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) {  // slot 1's barrier counts the warps of both slots, or its own ones twice
                        mbar_arrive(bar.o_empty + s);
                        if (by_keys || s == 1) mbar_arrive(bar.o_empty + 1);
                    }
                }
                if (by_keys) ++n_joined;
                ++n_unit;
                taken = 0, ref = kNoRef, m = -INFINITY, l = make_float2(0.f, 0.f);
                continue;
            }
            if (!(flags & (kSlot0 << s))) {
                done_step();
                continue;
            }
            if (!(ok = wait_warp(bar.s_full + s, n_s, 64))) break;
            tcgen05_fence_after();
            const int shift = by_keys ? 0 : s * slot_tokens;
            // Before O is rescaled or P written the product with the tile before has to be done.
            bool may_write = false;
            auto until_done = [&]() {
                if (!may_write) {
                    may_write = wait_warp(bar.o_done + s, n_s - 1, 61);
                    tcgen05_fence_after();
                }
                return may_write;
            };
            if ((warp & 3) * 32 >= (st.n_tokens - shift) * heads) {  // rows that stand for nothing: O's are not looked at
                done_step();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.s_free);
                if (!(ok = until_done())) break;
                if (lane == 0) mbar_arrive(bar.p_half[s]), mbar_arrive(bar.p_half[s] + 1);
                ++n_s, ++taken;
                continue;
            }
            int new_ref = st.ref;
            {
                const int limit = st.limit + shift + my_token - st.key0;  // last key of the tile that the row attends to
                const int lowest = __shfl_sync(0xffffffffu, limit, 0);
                if (lowest < kTile - 1) {  // in place and in a loop, which keeps the code short
#pragma unroll 1
                    for (int c = max(lowest + 1, 0) & ~31; c < kTile; c += 32) {
                        uint32_t y[32];
                        tcgen05_ld_32x32b_x32(ts + c, y);
                        tcgen05_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c + k > limit) y[k] = 0xff800000u;
                        tcgen05_st_32x32b_x32(ts + c, y);
                    }
                    tcgen05_wait_st();
                    // A reference that moves for pages behind the row's last key is none of its own: O might leave that one's range.
                    if (limit < st.first_taken || my_token >= min(slot_tokens, st.n_tokens - shift)) new_ref = ref;
                }
            }
            uint32_t x[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tcgen05_ld_32x32b_x32(ts + 32 * c, x[c]);
            tcgen05_wait_ld();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.s_free);
            float best = -INFINITY;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                const uint32_t *w = x[g / 2] + 16 * (g % 2);
                float top = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[15]));
#pragma unroll
                for (int k = 1; k < 15; k += 2) top = max3(top, __uint_as_float(w[k]), __uint_as_float(w[k + 1]));
                best = fmaxf(best, top * st.factor[g].x);
            }
            // Rows that stand for nothing, which hold anything, have no say in when the others' maxima move: their bits would depend on it.
            if (my_token >= min(slot_tokens, st.n_tokens - shift)) best = -INFINITY;
            if (__any_sync(0xffffffffu, best - m > kMaxLead || new_ref != ref)) {
                if (!(ok = until_done())) break;
                const float now = fmaxf(m, best), base = now == -INFINITY ? 0.f : now;
                const float shrink = exp2_approx(m - base);  // 0 from -infinity on
                m = now;
                far = __any_sync(0xffffffffu, fabsf(base) >= kFar) != 0;
                sub1 = (far ? 0.f : -base) + kRoom;
                l.x *= shrink, l.y *= shrink;
                if (taken > 0) {
                    const float f = shrink * exp2_approx(static_cast<float>(ref - new_ref));
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tcgen05_ld_32x32b_x32(to + c, o);
                        tcgen05_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                        tcgen05_st_32x32b_x32(to + c, o);
                    }
                    tcgen05_wait_st();
                }
                ref = new_ref;
            }
            if (far) {  // x f - m in one step would leave the rounding of m in P, more than its range where scores are large
                const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[c][k] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(x[c][k]), st.factor[2 * c + k / 16].x), base));
            }
            auto quarter = [&](int c, uint32_t *p) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 g = st.factor[2 * c + h];
                    const float weight = st.weight[2 * c + h];
                    const float2 ff = far ? make_float2(1.f, 1.f) : make_float2(g.x, g.y), sub = add2(make_float2(sub1, sub1), make_float2(g.z, g.w));
                    float2 part = make_float2(0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 t = fma2(make_float2(__uint_as_float(x[c][16 * h + 2 * k]), __uint_as_float(x[c][16 * h + 2 * k + 1])), ff, sub);
                        const float2 e = make_float2(exp2_approx(t.x), exp2_approx(t.y));
                        part = add2(part, e);
                        p[8 * h + k] = Elem<false>::from_float2(e.x, e.y);
                    }
                    l = fma2(part, make_float2(weight, weight), l);
                }
            };
            auto hand_over = [&](int half) {
                tcgen05_wait_st();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.p_half[s] + half);
            };
            uint32_t p0[32], p1[32];
            quarter(0, p0);
            quarter(1, p0 + 16);
            if (!(ok = until_done())) break;
            tcgen05_st_32x32b_x32(tp, p0);
            quarter(2, p1);  // while the first half is stored
            hand_over(0);
            quarter(3, p1 + 16);
            done_step();
            tcgen05_st_32x32b_x32(tp + 32, p1);
            hand_over(1);
            ++n_s, ++taken;
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
}

// Joins the parts of units that several blocks worked on: block (c, y) the rows 32 y .. of the unit that block c began and did not
// end.  A lane is a row, a warp takes every eighth group of four outputs.
constexpr int kJoinWarps = 8;
template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinWarps * 32) attn_chunk_join_kernel(const ChunkArgs a, int grid) {
    using E = Elem<BF16>;
    __shared__ float top_of[kJoinWarps][32], sum_of[kJoinWarps][32], ref_of[kJoinWarps][32];
    __shared__ int parts;
    const int c0 = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 h = __ldcg(a.headers + c0 * 4), unit = __ldcg(a.headers + c0 * 4 + 1);
    if (h.y != 1) return;
    const int slot_tokens = h.z, heads = h.w;
    const bool by_keys = unit.y <= slot_tokens;
    const int row = blockIdx.y * 32 + lane, s = row / kTile, r = row - s * kTile;
    const int my_token = r / heads, my_head = r - my_token * heads, t = s * slot_tokens + my_token;
    const bool valid = (s == 0 || !by_keys) && my_token < slot_tokens && t < unit.y && my_head >= unit.w;
    if (!__syncthreads_or(valid)) return;
    if (warp == 0) {  // parts: block c0's second, then the first ones of the blocks behind it up to the one that ended the unit
        int n = 1;
        while (c0 + n < grid) {
            const int c = c0 + n + lane;
            const int state = c < grid ? __ldcg(a.headers + c * 4).x : 0;
            const unsigned last = __ballot_sync(0xffffffffu, state != 1);
            if (last) {
                const int at = __ffs(last) - 1;
                n += at + (__shfl_sync(0xffffffffu, state, at) == 2 ? 1 : 0);
                break;
            }
            n += 32;
        }
        if (lane == 0) parts = n;
    }
    __syncthreads();
    const int n = parts;
    auto base_of = [&](int p) { return a.partial + static_cast<int64_t>(p == 0 ? c0 * 2 + 1 : (c0 + p) * 2) * kPartFloats<D> + row * 4; };
    float top = -INFINITY, ref = -1000.f, sum = 0.f;
    for (int p = warp; p < n; p += kJoinWarps) {
        const float4 st = valid ? __ldcg(reinterpret_cast<const float4 *>(base_of(p) + 256 * D)) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        if (st.x == -INFINITY && st.y == 0.f) continue;
        top = fmaxf(top, st.x), ref = fmaxf(ref, st.z);
    }
    top_of[warp][lane] = top, ref_of[warp][lane] = ref;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, top_of[w][lane]), ref = fmaxf(ref, ref_of[w][lane]);
    auto weight = [&](const float4 &st) { return st.x == -INFINITY ? 0.f : exp2_approx(st.x - top); };
    for (int p = warp; p < n; p += kJoinWarps) {
        const float4 st = valid ? __ldcg(reinterpret_cast<const float4 *>(base_of(p) + 256 * D)) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        if (st.x == -INFINITY && st.y == 0.f) continue;
        sum += st.y * (st.y == st.y ? weight(st) : 1.f);
    }
    sum_of[warp][lane] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += sum_of[w][lane];
    if (!valid) return;
    const float inv = 2.f / sum, scale = __uint_as_float(static_cast<uint32_t>(126 + max(static_cast<int>(ref), -125)) << 23);
    uint16_t *y = static_cast<uint16_t *>(const_cast<void *>(a.out.ptr)) + static_cast<int64_t>(unit.x + t) * a.out.token_stride + (unit.z + my_head) * a.out.head_stride;
    constexpr int kMine = D / 4 / kJoinWarps;
    float4 o[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < n; ++p) {
        const float *from = base_of(p);
        const float4 st = __ldcg(reinterpret_cast<const float4 *>(from + 256 * D));
        const float f = st.x == -INFINITY ? 0.f : weight(st) * exp2_approx(st.z - ref);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const float4 x = __ldcg(reinterpret_cast<const float4 *>(from + (warp + i * kJoinWarps) * (256 * 4)));
            if (f != 0.f) o[i].x = fmaf(x.x, f, o[i].x), o[i].y = fmaf(x.y, f, o[i].y), o[i].z = fmaf(x.z, f, o[i].z), o[i].w = fmaf(x.w, f, o[i].w);
        }
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        *reinterpret_cast<uint2 *>(y + 4 * (warp + i * kJoinWarps)) =
            make_uint2(E::from_float2(o[i].x * inv * scale, o[i].y * inv * scale), E::from_float2(o[i].z * inv * scale, o[i].w * inv * scale));
}

template <int D, bool BF16>
pd_status launch(const ChunkArgs &a, cudaStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    if (!ensure_dynamic_smem(attn_chunk_kernel<D, BF16>, ChunkSmem<D>::kTotal, done)) return PD_ERR_CUDA;
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return PD_ERR_CUDA;
    const int group = a.q_heads / a.kv_heads, chunks = (group + kTile - 1) / kTile, heads = (group + chunks - 1) / chunks;
    CUtensorMap map;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(a.q_heads), static_cast<cuuint64_t>(a.n_tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.q.head_stride) * 2, static_cast<cuuint64_t>(a.q.token_stride) * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(heads), static_cast<cuuint32_t>(kTile / heads)};
    const cuuint32_t estr[3] = {1, 1, 1};
    if (fn(&map, BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(a.q.ptr), dims, strides, box, estr,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return PD_ERR_CUDA;
    const int grid = min(sm_count(), kMaxGrid);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = ChunkSmem<D>::kTotal;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch(2);
    if (cudaLaunchKernelEx(&cfg, attn_chunk_kernel<D, BF16>, map, a) != cudaSuccess) return PD_ERR_CUDA;
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 256 / 32);
    cfg.blockDim = dim3(kJoinWarps * 32);
    cfg.dynamicSmemBytes = 0;
    return cuda_ok(cudaLaunchKernelEx(&cfg, attn_chunk_join_kernel<D, BF16>, a, grid));
}

constexpr size_t kHeaderBytes = static_cast<size_t>(kMaxGrid) * 4 * sizeof(int4);

}  // namespace

size_t attn_chunk_scratch_bytes() { return kHeaderBytes + static_cast<size_t>(min(sm_count(), kMaxGrid)) * 2 * kPartFloats<128> * sizeof(float); }

pd_status launch_attn_chunk(ChunkArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream) {
    a.headers = reinterpret_cast<int4 *>(scratch);
    a.partial = reinterpret_cast<float *>(scratch + kHeaderBytes);
    if (a.head_dim == 128) return bf16 ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
    return bf16 ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
}

}  // namespace pd
