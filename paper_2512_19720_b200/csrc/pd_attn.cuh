// What the attention operators (pd_attn_prompt, pd_kv_append, pd_attn_cache) share: their arguments and launchers.
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
};

size_t attn_cache_scratch_bytes();  // counters and partial results

pd_status launch_attn_prompt(const PromptArgs &a, bool bf16, cudaStream_t stream);
pd_status launch_kv_append(const AppendArgs &a, bool bf16, cudaStream_t stream);
pd_status launch_attn_cache(CacheAttnArgs a, unsigned char *scratch, bool bf16, cudaStream_t stream);

}  // namespace pd
