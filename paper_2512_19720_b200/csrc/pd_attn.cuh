// What the attention operators (pd_attn_prompt, pd_kv_append, pd_attn_cache, pd_rope, pd_kv_append_rope, pd_attn_chunk) share: their
// arguments and launchers.
#pragma once

#include "pd_common.cuh"

namespace pd {

// A tensor [tokens, heads, head_dim] with contiguous heads: strides in elements.
struct HeadsView {
    const void *ptr;
    int64_t token_stride, head_stride;
};

struct PromptArgs {
    HeadsView q, k, v, out;
    const int32_t *cu_seqlens;  // [n_seqs + 1]
    int n_seqs, n_tokens, q_heads, kv_heads, head_dim;
    float scale;
    uint32_t *status;
    unsigned int *counters;  // two, zero on entry, zero again on return
};

// The 8-bit paged cache: codes [n_pages, kv_heads, page, head_dim], scales [n_pages, kv_heads].
struct KvPages {
    int8_t *codes;
    float *scale;
};

struct AppendArgs {
    HeadsView x[2];      // keys, values
    KvPages pages[2];
    void *values[2];     // [n_tokens, kv_heads, head_dim] or nullptr
    const int32_t *cu_seqlens, *seq_lens, *block_table;
    int64_t table_stride;
    int n_seqs, n_tokens, kv_heads, head_dim, page_log2, table_width;
    int64_t n_pages;
    uint32_t *status;
};

struct CacheAttnArgs {
    HeadsView q, out;
    KvPages pages[2];
    const int32_t *seq_lens, *block_table;
    int64_t table_stride;
    int n_seqs, q_heads, kv_heads, head_dim, page_log2, table_width;
    int64_t n_pages;
    float scale;
    uint32_t *status;
    unsigned int *counters;  // zero on entry, zero again on return
    float *partial;
    // several new tokens a sequence
    const int32_t *cu_seqlens;
    int n_tokens, max_new;
};

// Rotary positions: pair i of a head turns by positions[axes[i]][token] * inv_freq[i].
struct Rotation {
    const int32_t *positions;  // [n_axes, tokens]; nullptr: a token's place in its sequence
    int64_t axis_stride;
    const int32_t *axes;       // [pairs]; nullptr: all of the first axis
    const float *inv_freq;     // [pairs]
    int n_axes, pairs;
    float direction;           // 1, or -1 to turn back
};

struct RopeArgs {
    HeadsView x[2], out[2];  // queries, keys
    int heads[2], n_tokens, head_dim;
    Rotation r;
    uint32_t *status;
};

struct AppendRopeArgs {
    AppendArgs a;
    HeadsView q, q_out;
    int q_heads;  // 0: no queries
    Rotation r;
};

// Attention of several new tokens a sequence over the cache.
struct ChunkArgs {
    HeadsView q, out;
    KvPages pages[2];
    const int32_t *cu_seqlens, *seq_lens, *block_table;
    int64_t table_stride;
    int n_seqs, n_tokens, max_new, q_heads, kv_heads, head_dim, page_log2, table_width;
    int64_t n_pages;
    float scale;
    uint32_t *status;
    float *partial;  // parts of units that several blocks work on
    int4 *headers;
};

size_t attn_chunk_scratch_bytes();  // headers and parts; need not be zero
size_t attn_cache_scratch_bytes();  // counters and partial results

pd_status launch_attn_prompt(const PromptArgs &a, bool bf16, cudaStream_t stream);
pd_status launch_kv_append(const AppendArgs &a, bool bf16, cudaStream_t stream);
pd_status launch_rope(const RopeArgs &a, bool interleaved, bool bf16, cudaStream_t stream);
pd_status launch_kv_append_rope(const AppendRopeArgs &a, bool interleaved, bool bf16, cudaStream_t stream);
pd_status launch_attn_chunk(ChunkArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream);
pd_status launch_attn_cache(CacheAttnArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream);
// The same for max_new tokens a sequence; max_new * (q_heads / kv_heads) is at most kCacheRows.
constexpr int kCacheRows = 16;
pd_status launch_attn_cache_rows(CacheAttnArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream);

}  // namespace pd
