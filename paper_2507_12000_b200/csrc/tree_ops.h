// Host-side interface of the kernels of a round on a drafted tree (internal to the library).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace dssd {

struct AdjustParams {
    const void *logits;
    void *out;
    int64_t row_stride, out_stride;
    const int32_t *draft_tokens, *parents;
    const int32_t *history;
    int64_t history_stride;
    const int32_t *prompt_len, *history_len;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_tokens;
    const float *bias_values;
    const uint32_t *mask;
    const int32_t *mask_row;
    uint32_t *flags;
    int B, N, V, L, K, mask_rows;
    // geometry
    int pieces;  // of a row, each a turn of a CTA of the copy
    int turns;   // CTAs of the copy per row
    int slots;   // of the table of tokens, a power of two
    int shares;  // CTAs of the list per sequence
    // workspace
    uint4 *list;         // [B, list_size] entries, by buckets
    int2 *buckets;       // [B, n_buckets] first entry and the one behind the last
    long long list_size;
    int n_buckets;
    int gaps;            // buckets may not follow one another
};
int adjust_copy_entries(int dtype);  // of a row, by a CTA of the copy
size_t adjust_workspace(int B, int N, int V, int L, int K);
cudaError_t adjust_launch(AdjustParams &P, int dtype, void *workspace, cudaStream_t stream);

struct TreeVerifyParams {
    const void *logits;
    int64_t row_stride;
    const float *draft_q;
    const int32_t *draft_tokens, *parents;
    const float *uniforms, *uniforms_rs;
    double c1;         // log2(e) / T
    double sum_error;  // of a float32 pass
    int replacement, B, N, V;
    int32_t *accept_len, *path, *token;
    uint32_t *edge_flags, *rs_flags;
    int slice;  // entries of the vocabulary per CTA of the sequence's cluster
    int chunk;  // entries of a warp at a time
};
cudaError_t tree_verify_launch(TreeVerifyParams &P, int dtype, cudaStream_t stream);

struct AppendParams {
    const void *k_new, *v_new;
    void *k_cache, *v_cache;
    int64_t new_l, new_b, new_n, new_h;          // strides in elements
    int64_t cache_l, cache_p, cache_t, cache_h;
    const int32_t *block_table;
    int64_t table_stride;
    int max_pages, num_pages, page_size;
    const int32_t *ctx_len, *accept_len, *path;
    int layers, B, N, Hkv, D;
    int32_t *new_len;
    uint32_t *flags;
};
cudaError_t append_launch(AppendParams &P, cudaStream_t stream);

struct TreeAttentionParams {
    const void *q, *k_new, *v_new, *k_cache, *v_cache;
    int64_t q_b, q_n, q_h;                        // strides in elements
    int64_t new_b, new_n, new_h;
    int64_t cache_p, cache_t, cache_h;
    int64_t o_b, o_n, o_h;
    const int32_t *block_table;
    int64_t table_stride;
    int max_pages, num_pages, page_size;
    const int32_t *ctx_len, *parents;
    int B, N, Hq, Hkv, D;
    float scale;
    void *o;
    float *lse;
    uint32_t *flags;
    // for the library's own test of its waits
    int withhold;           // sequence whose nodes' keys are never copied, -1: none
    long long wait_cycles;  // limit of a wait, 0: the usual one
};
size_t tree_attention_workspace(int B, int N, int Hq, int Hkv, int D);
cudaError_t tree_attention_launch(TreeAttentionParams &P, int dtype, void *workspace, cudaStream_t stream);

}  // namespace dssd
