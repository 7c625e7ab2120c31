// C ABI of the attention operators: argument checks, workspace layout.  Rules and formulas are in include/pd.h.
#include <climits>
#include <cmath>

#include "pd_attn.cuh"

namespace pd {
namespace {

pd_status check_heads(int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale) {
    if (q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads != 0 || !std::isfinite(scale)) return PD_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return PD_ERR_UNSUPPORTED_SHAPE;
    if (q_heads > 65535) return PD_ERR_UNSUPPORTED_SHAPE;  // a dimension of the grid
    return PD_OK;
}

// Strides along dimensions of size 1 say nothing and are set to what a dense tensor would have.
pd_status check_view(HeadsView &x, int64_t tokens, int heads, int head_dim) {
    if (!x.ptr) return PD_ERR_INVALID_ARG;
    if (heads == 1) x.head_stride = head_dim;
    if (tokens == 1) x.token_stride = static_cast<int64_t>(heads) * head_dim;
    if (x.head_stride < head_dim || x.token_stride < head_dim) return PD_ERR_INVALID_ARG;  // overlapping or broadcast
    if (x.head_stride % 8 || x.token_stride % 8 || !aligned16(x.ptr)) return PD_ERR_ALIGNMENT;
    if (x.head_stride >= (int64_t(1) << 38) || x.token_stride >= (int64_t(1) << 38)) return PD_ERR_UNSUPPORTED_SHAPE;
    return PD_OK;
}

pd_status check_workspace(void *workspace, size_t bytes) {
    return !workspace || !aligned256(workspace) || bytes < pd_workspace_bytes(PD_OP_ATTN, 0, 0, 0, 0) ? PD_ERR_WORKSPACE : PD_OK;
}

pd_status check_cache(const void *k_codes, const void *v_codes, const float *k_scale, const float *v_scale, int64_t n_pages, int32_t page,
                      const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width) {
    if (!k_codes || !v_codes || !k_scale || !v_scale || n_pages <= 0 || !seq_lens || !block_table || table_width <= 0 || table_stride < table_width)
        return PD_ERR_INVALID_ARG;
    if ((page != 16 && page != 32 && page != 64 && page != 128) || static_cast<int64_t>(table_width) * page > INT_MAX / 2) return PD_ERR_UNSUPPORTED_SHAPE;
    if (!aligned16(k_codes) || !aligned16(v_codes)) return PD_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale) | reinterpret_cast<uintptr_t>(seq_lens) |
         reinterpret_cast<uintptr_t>(block_table)) & 3u)
        return PD_ERR_ALIGNMENT;
    return PD_OK;
}

int log2_of(int32_t page) { return page == 16 ? 4 : (page == 32 ? 5 : (page == 64 ? 6 : 7)); }

#define PD_TRY(x)                            \
    do {                                     \
        const pd_status st_ = (x);           \
        if (st_ != PD_OK) return st_;        \
    } while (0)

pd_status prompt_impl(HeadsView q, HeadsView k, HeadsView v, const int32_t *cu_seqlens, int32_t n_seqs, int64_t n_tokens, int32_t q_heads,
                      int32_t kv_heads, int32_t head_dim, float scale, HeadsView out, void *workspace, size_t workspace_bytes,
                      void *cuda_stream, bool bf16) {
    if (!cu_seqlens || n_seqs <= 0 || n_tokens < 0) return PD_ERR_INVALID_ARG;
    PD_TRY(check_heads(q_heads, kv_heads, head_dim, scale));
    if (n_tokens > INT_MAX / 2 || n_seqs > INT_MAX / 4) return PD_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return check_workspace(workspace, workspace_bytes);  // nothing to do; empty tensors may have no address
    PD_TRY(check_view(q, n_tokens, q_heads, head_dim));
    PD_TRY(check_view(k, n_tokens, kv_heads, head_dim));
    PD_TRY(check_view(v, n_tokens, kv_heads, head_dim));
    PD_TRY(check_view(out, n_tokens, q_heads, head_dim));
    if (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u) return PD_ERR_ALIGNMENT;
    PD_TRY(check_workspace(workspace, workspace_bytes));
    const PromptArgs a = {q, k, v, out, cu_seqlens, n_seqs, static_cast<int>(n_tokens), q_heads, kv_heads, head_dim, scale,
                          static_cast<uint32_t *>(workspace), reinterpret_cast<unsigned int *>(static_cast<unsigned char *>(workspace) + kStatusBytes)};
    return launch_attn_prompt(a, bf16, static_cast<cudaStream_t>(cuda_stream));
}

pd_status append_impl(HeadsView k, HeadsView v, const int32_t *cu_seqlens, int32_t n_seqs, int64_t n_tokens, int32_t kv_heads,
                      int32_t head_dim, int8_t *k_codes, int8_t *v_codes, float *k_scale, float *v_scale, int64_t n_pages, int32_t page,
                      const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width, void *k_values,
                      void *v_values, void *workspace, size_t workspace_bytes, void *cuda_stream, bool bf16) {
    if (!cu_seqlens || n_seqs <= 0 || n_tokens < 0) return PD_ERR_INVALID_ARG;
    PD_TRY(check_heads(kv_heads, kv_heads, head_dim, 1.f));
    if (n_tokens > INT_MAX / 2 || n_seqs > INT_MAX / 4) return PD_ERR_UNSUPPORTED_SHAPE;
    PD_TRY(check_cache(k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width));
    if (n_tokens == 0) return check_workspace(workspace, workspace_bytes);
    PD_TRY(check_view(k, n_tokens, kv_heads, head_dim));
    PD_TRY(check_view(v, n_tokens, kv_heads, head_dim));
    if (!aligned16(k_values) || !aligned16(v_values) || (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u)) return PD_ERR_ALIGNMENT;
    PD_TRY(check_workspace(workspace, workspace_bytes));
    const AppendArgs a = {{k, v}, {{k_codes, k_scale}, {v_codes, v_scale}}, {k_values, v_values}, cu_seqlens, seq_lens, block_table, table_stride,
                          n_seqs, static_cast<int>(n_tokens), kv_heads, head_dim, log2_of(page), table_width, n_pages,
                          static_cast<uint32_t *>(workspace)};
    return launch_kv_append(a, bf16, static_cast<cudaStream_t>(cuda_stream));
}

pd_status cache_impl(HeadsView q, int32_t n_seqs, int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale, const int8_t *k_codes,
                     const int8_t *v_codes, const float *k_scale, const float *v_scale, int64_t n_pages, int32_t page, const int32_t *seq_lens,
                     const int32_t *block_table, int64_t table_stride, int32_t table_width, HeadsView out, void *workspace,
                     size_t workspace_bytes, void *cuda_stream, bool bf16) {
    if (n_seqs <= 0) return PD_ERR_INVALID_ARG;
    PD_TRY(check_heads(q_heads, kv_heads, head_dim, scale));
    PD_TRY(check_cache(k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width));
    // tiles of at least 16 tokens are counted in 32 bits, for all sequences and heads together
    const int64_t tiles = static_cast<int64_t>(table_width) * (page / 16) + 1;
    if (tiles > INT_MAX / 2 || tiles * n_seqs > INT_MAX / 2 || tiles * n_seqs * q_heads > INT_MAX / 2) return PD_ERR_UNSUPPORTED_SHAPE;
    PD_TRY(check_view(q, n_seqs, q_heads, head_dim));
    PD_TRY(check_view(out, n_seqs, q_heads, head_dim));
    PD_TRY(check_workspace(workspace, workspace_bytes));
    const CacheAttnArgs a = {q, out, {{const_cast<int8_t *>(k_codes), const_cast<float *>(k_scale)}, {const_cast<int8_t *>(v_codes), const_cast<float *>(v_scale)}},
                             seq_lens, block_table, table_stride, n_seqs, q_heads, kv_heads, head_dim, log2_of(page), table_width, n_pages, scale,
                             static_cast<uint32_t *>(workspace), nullptr, nullptr, nullptr, 0, 0};
    return launch_attn_cache(a, static_cast<unsigned char *>(workspace) + kStatusBytes, bf16, static_cast<cudaStream_t>(cuda_stream));
}

pd_status check_rotation(Rotation &r, int64_t n_tokens, int head_dim, int32_t interleaved) {
    if (!r.inv_freq || r.pairs <= 0 || (interleaved != 0 && interleaved != 1)) return PD_ERR_INVALID_ARG;
    if (r.positions && (r.n_axes <= 0 || (r.n_axes > 1 && (!r.axes || r.axis_stride < n_tokens)))) return PD_ERR_INVALID_ARG;
    if (!r.positions && r.axes) return PD_ERR_INVALID_ARG;  // a place in a sequence has one axis
    if (r.pairs % 8 || 2 * r.pairs > head_dim) return PD_ERR_UNSUPPORTED_SHAPE;
    if ((reinterpret_cast<uintptr_t>(r.positions) | reinterpret_cast<uintptr_t>(r.axes) | reinterpret_cast<uintptr_t>(r.inv_freq)) & 3u) return PD_ERR_ALIGNMENT;
    return PD_OK;
}

pd_status rope_impl(HeadsView q, HeadsView k, Rotation r, int32_t interleaved, int64_t n_tokens, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                    HeadsView q_out, HeadsView k_out, void *workspace, size_t workspace_bytes, void *cuda_stream, bool bf16) {
    if (n_tokens < 0 || q_heads <= 0 || k_heads < 0) return PD_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return PD_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens > INT_MAX / 2 || q_heads > 65535 || k_heads > 65535) return PD_ERR_UNSUPPORTED_SHAPE;
    if (n_tokens == 0) return check_workspace(workspace, workspace_bytes);  // nothing to do; empty tensors may have no address
    if (!r.positions) return PD_ERR_INVALID_ARG;
    PD_TRY(check_rotation(r, n_tokens, head_dim, interleaved));
    PD_TRY(check_view(q, n_tokens, q_heads, head_dim));
    PD_TRY(check_view(q_out, n_tokens, q_heads, head_dim));
    if (k_heads) {
        PD_TRY(check_view(k, n_tokens, k_heads, head_dim));
        PD_TRY(check_view(k_out, n_tokens, k_heads, head_dim));
    }
    PD_TRY(check_workspace(workspace, workspace_bytes));
    const RopeArgs a = {{q, k}, {q_out, k_out}, {q_heads, k_heads}, static_cast<int>(n_tokens), head_dim, r, static_cast<uint32_t *>(workspace)};
    return launch_rope(a, interleaved != 0, bf16, static_cast<cudaStream_t>(cuda_stream));
}

pd_status append_rope_impl(HeadsView q, HeadsView k, HeadsView v, const int32_t *cu_seqlens, int32_t n_seqs, int64_t n_tokens, int32_t q_heads, int32_t kv_heads,
                           int32_t head_dim, Rotation r, int32_t interleaved, int8_t *k_codes, int8_t *v_codes, float *k_scale, float *v_scale, int64_t n_pages,
                           int32_t page, const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width, HeadsView q_out,
                           void *k_values, void *v_values, void *workspace, size_t workspace_bytes, void *cuda_stream, bool bf16) {
    if (!cu_seqlens || n_seqs <= 0 || n_tokens < 0 || q_heads < 0) return PD_ERR_INVALID_ARG;
    PD_TRY(check_heads(kv_heads, kv_heads, head_dim, 1.f));
    if (n_tokens > INT_MAX / 2 || n_seqs > INT_MAX / 4 || q_heads > 65535) return PD_ERR_UNSUPPORTED_SHAPE;
    PD_TRY(check_cache(k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width));
    if (n_tokens == 0) return check_workspace(workspace, workspace_bytes);
    PD_TRY(check_rotation(r, n_tokens, head_dim, interleaved));
    PD_TRY(check_view(k, n_tokens, kv_heads, head_dim));
    PD_TRY(check_view(v, n_tokens, kv_heads, head_dim));
    if (q_heads) {
        PD_TRY(check_view(q, n_tokens, q_heads, head_dim));
        PD_TRY(check_view(q_out, n_tokens, q_heads, head_dim));
    }
    if (!aligned16(k_values) || !aligned16(v_values) || (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u)) return PD_ERR_ALIGNMENT;
    PD_TRY(check_workspace(workspace, workspace_bytes));
    const AppendArgs a = {{k, v}, {{k_codes, k_scale}, {v_codes, v_scale}}, {k_values, v_values}, cu_seqlens, seq_lens, block_table, table_stride,
                          n_seqs, static_cast<int>(n_tokens), kv_heads, head_dim, log2_of(page), table_width, n_pages,
                          static_cast<uint32_t *>(workspace)};
    return launch_kv_append_rope({a, q, q_out, q_heads, r}, interleaved != 0, bf16, static_cast<cudaStream_t>(cuda_stream));
}

pd_status chunk_impl(HeadsView q, const int32_t *cu_seqlens, int32_t n_seqs, int64_t n_tokens, int64_t max_new, int32_t q_heads, int32_t kv_heads,
                     int32_t head_dim, float scale, const int8_t *k_codes, const int8_t *v_codes, const float *k_scale, const float *v_scale, int64_t n_pages,
                     int32_t page, const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width, HeadsView out,
                     void *workspace, size_t workspace_bytes, void *cuda_stream, bool bf16) {
    if (!cu_seqlens || n_seqs <= 0 || n_tokens < 0 || max_new < 0) return PD_ERR_INVALID_ARG;
    PD_TRY(check_heads(q_heads, kv_heads, head_dim, scale));
    if (n_tokens > INT_MAX / 2 || n_seqs > INT_MAX / 4) return PD_ERR_UNSUPPORTED_SHAPE;
    PD_TRY(check_cache(k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width));
    // blocks of 16 keys of the cache are counted in 31 bits
    if (n_pages >= INT_MAX || n_pages * (page / 16) >= INT_MAX / kv_heads) return PD_ERR_UNSUPPORTED_SHAPE;
    const bool room = workspace && aligned256(workspace) && workspace_bytes >= pd_workspace_bytes(PD_OP_ATTN_CHUNK, 0, 0, 0, 0);
    if (n_tokens == 0) return room ? PD_OK : PD_ERR_WORKSPACE;
    PD_TRY(check_view(q, n_tokens, q_heads, head_dim));
    PD_TRY(check_view(out, n_tokens, q_heads, head_dim));
    if (reinterpret_cast<uintptr_t>(cu_seqlens) & 3u) return PD_ERR_ALIGNMENT;
    if (!room) return PD_ERR_WORKSPACE;
    const int most = static_cast<int>(max_new == 0 || max_new > n_tokens ? n_tokens : max_new);
    // Few rows that share a key/value head: the products of the kernel for single tokens, which takes codes as they are, instead of 128-row
    // products of converted codes.  64 sequences of 1 to 8 tokens, 32 heads, 20 to 1000 held, with the append: 92 us beside 207.
    const int64_t tiles = static_cast<int64_t>(table_width) * (page / 16) + 1;
    if (most <= kCacheRows && most * (q_heads / kv_heads) <= kCacheRows && tiles < INT_MAX / 2 && tiles * n_seqs < INT_MAX / 2 && tiles * n_seqs * q_heads < INT_MAX / 2) {
        const CacheAttnArgs a = {q, out, {{const_cast<int8_t *>(k_codes), const_cast<float *>(k_scale)}, {const_cast<int8_t *>(v_codes), const_cast<float *>(v_scale)}},
                                 seq_lens, block_table, table_stride, n_seqs, q_heads, kv_heads, head_dim, log2_of(page), table_width, n_pages, scale,
                                 static_cast<uint32_t *>(workspace), nullptr, nullptr, cu_seqlens, static_cast<int>(n_tokens), most};
        return launch_attn_cache_rows(a, static_cast<unsigned char *>(workspace) + kStatusBytes, bf16, static_cast<cudaStream_t>(cuda_stream));
    }
    const ChunkArgs a = {q, out, {{const_cast<int8_t *>(k_codes), const_cast<float *>(k_scale)}, {const_cast<int8_t *>(v_codes), const_cast<float *>(v_scale)}},
                         cu_seqlens, seq_lens, block_table, table_stride, n_seqs, static_cast<int>(n_tokens),
                         most, q_heads, kv_heads, head_dim, log2_of(page), table_width,
                         n_pages, scale, static_cast<uint32_t *>(workspace), nullptr, nullptr};
    return launch_attn_chunk(a, static_cast<unsigned char *>(workspace) + kStatusBytes + attn_cache_scratch_bytes(), bf16, static_cast<cudaStream_t>(cuda_stream));
}

}  // namespace
}  // namespace pd

extern "C" {

#define PD_ATTN_PROMPT(NAME, BF16)                                                                                                         \
    pd_status NAME(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,                    \
                   int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, const int32_t *cu_seqlens,         \
                   int32_t n_seqs, int64_t n_tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale, void *out,          \
                   int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes, void *cuda_stream) {        \
        return pd::prompt_impl({q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, \
                               cu_seqlens, n_seqs, n_tokens, q_heads, kv_heads, head_dim, scale, {out, out_token_stride, out_head_stride}, \
                               workspace, workspace_bytes, cuda_stream, BF16);                                                             \
    }
PD_ATTN_PROMPT(pd_attn_prompt, false)
PD_ATTN_PROMPT(pd_attn_prompt_bf16, true)

#define PD_KV_APPEND(NAME, BF16)                                                                                                         \
    pd_status NAME(const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride,                  \
                   int64_t v_head_stride, const int32_t *cu_seqlens, int32_t n_seqs, int64_t n_tokens, int32_t kv_heads,                 \
                   int32_t head_dim, int8_t *k_codes, int8_t *v_codes, float *k_scale, float *v_scale, int64_t n_pages, int32_t page,    \
                   const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width, void *k_values,       \
                   void *v_values, void *workspace, size_t workspace_bytes, void *cuda_stream) {                                         \
        return pd::append_impl({k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, cu_seqlens, n_seqs, n_tokens,     \
                               kv_heads, head_dim, k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table,             \
                               table_stride, table_width, k_values, v_values, workspace, workspace_bytes, cuda_stream, BF16);            \
    }
PD_KV_APPEND(pd_kv_append, false)
PD_KV_APPEND(pd_kv_append_bf16, true)

#define PD_ATTN_CACHE(NAME, BF16)                                                                                                       \
    pd_status NAME(const void *q, int64_t q_token_stride, int64_t q_head_stride, int32_t n_seqs, int32_t q_heads, int32_t kv_heads,     \
                   int32_t head_dim, float scale, const int8_t *k_codes, const int8_t *v_codes, const float *k_scale,                   \
                   const float *v_scale, int64_t n_pages, int32_t page, const int32_t *seq_lens, const int32_t *block_table,            \
                   int64_t table_stride, int32_t table_width, void *out, int64_t out_token_stride, int64_t out_head_stride,             \
                   void *workspace, size_t workspace_bytes, void *cuda_stream) {                                                        \
        return pd::cache_impl({q, q_token_stride, q_head_stride}, n_seqs, q_heads, kv_heads, head_dim, scale, k_codes, v_codes,         \
                              k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width,                        \
                              {out, out_token_stride, out_head_stride}, workspace, workspace_bytes, cuda_stream, BF16);                 \
    }
PD_ATTN_CACHE(pd_attn_cache, false)
PD_ATTN_CACHE(pd_attn_cache_bf16, true)

#define PD_ROPE(NAME, BF16)                                                                                                                 \
    pd_status NAME(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,                      \
                   int64_t k_head_stride, const int32_t *positions, int64_t axis_stride, int32_t n_axes, const int32_t *axes,                \
                   const float *inv_freq, int32_t pairs, int32_t interleaved, int32_t inverse, int64_t n_tokens, int32_t q_heads,            \
                   int32_t k_heads, int32_t head_dim, void *q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void *k_out,       \
                   int64_t k_out_token_stride, int64_t k_out_head_stride, void *workspace, size_t workspace_bytes, void *cuda_stream) {      \
        return pd::rope_impl({q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride},                                         \
                             {positions, axis_stride, axes, inv_freq, n_axes, pairs, inverse ? -1.f : 1.f}, interleaved, n_tokens, q_heads,  \
                             k_heads, head_dim, {q_out, q_out_token_stride, q_out_head_stride},                                              \
                             {k_out, k_out_token_stride, k_out_head_stride}, workspace, workspace_bytes, cuda_stream, BF16);                 \
    }
PD_ROPE(pd_rope, false)
PD_ROPE(pd_rope_bf16, true)

#define PD_KV_APPEND_ROPE(NAME, BF16)                                                                                                       \
    pd_status NAME(const void *q, int64_t q_token_stride, int64_t q_head_stride, const void *k, int64_t k_token_stride,                      \
                   int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, const int32_t *cu_seqlens,           \
                   int32_t n_seqs, int64_t n_tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim, const int32_t *positions,          \
                   int64_t axis_stride, int32_t n_axes, const int32_t *axes, const float *inv_freq, int32_t pairs, int32_t interleaved,      \
                   int8_t *k_codes, int8_t *v_codes, float *k_scale, float *v_scale, int64_t n_pages, int32_t page, const int32_t *seq_lens, \
                   const int32_t *block_table, int64_t table_stride, int32_t table_width, void *q_out, int64_t q_out_token_stride,           \
                   int64_t q_out_head_stride, void *k_values, void *v_values, void *workspace, size_t workspace_bytes, void *cuda_stream) {  \
        return pd::append_rope_impl({q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride},                                  \
                                    {v, v_token_stride, v_head_stride}, cu_seqlens, n_seqs, n_tokens, q_heads, kv_heads, head_dim,           \
                                    {positions, axis_stride, axes, inv_freq, n_axes, pairs, 1.f}, interleaved, k_codes, v_codes, k_scale,    \
                                    v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width,                                \
                                    {q_out, q_out_token_stride, q_out_head_stride}, k_values, v_values, workspace, workspace_bytes,          \
                                    cuda_stream, BF16);                                                                                      \
    }
PD_KV_APPEND_ROPE(pd_kv_append_rope, false)
PD_KV_APPEND_ROPE(pd_kv_append_rope_bf16, true)

#define PD_ATTN_CHUNK(NAME, BF16)                                                                                                           \
    pd_status NAME(const void *q, int64_t q_token_stride, int64_t q_head_stride, const int32_t *cu_seqlens, int32_t n_seqs,                  \
                   int64_t n_tokens, int64_t max_new, int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale,                      \
                   const int8_t *k_codes, const int8_t *v_codes, const float *k_scale, const float *v_scale, int64_t n_pages, int32_t page,  \
                   const int32_t *seq_lens, const int32_t *block_table, int64_t table_stride, int32_t table_width, void *out,                \
                   int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes, void *cuda_stream) {          \
        return pd::chunk_impl({q, q_token_stride, q_head_stride}, cu_seqlens, n_seqs, n_tokens, max_new, q_heads, kv_heads, head_dim, scale, \
                              k_codes, v_codes, k_scale, v_scale, n_pages, page, seq_lens, block_table, table_stride, table_width,           \
                              {out, out_token_stride, out_head_stride}, workspace, workspace_bytes, cuda_stream, BF16);                      \
    }
PD_ATTN_CHUNK(pd_attn_chunk, false)
PD_ATTN_CHUNK(pd_attn_chunk_bf16, true)

}  // extern "C"
