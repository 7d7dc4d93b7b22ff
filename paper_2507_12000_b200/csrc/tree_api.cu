// C ABI of the round on a drafted tree: argument checks and launches.  See include/dssd.h.
#include <cuda_runtime.h>
#include <math.h>

#include "dssd.h"
#include "dssd_test_hooks.h"
#include "tree_ops.h"

namespace dssd {
void set_last_cuda_error(int e);
}

namespace {

dssd_status done(cudaError_t e)
{
    if (e == cudaSuccess) return DSSD_OK;
    dssd::set_last_cuda_error((int)e);
    return DSSD_ERR_CUDA;
}

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// whether two arrays of 4-byte values share a place
bool overlap(const void *a, long long a_count, const void *b, long long b_count)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && a_count > 0 && b_count > 0 && x < y + 4 * (uintptr_t)b_count && y < x + 4 * (uintptr_t)a_count;
}

dssd_status check_tree(int B, int N, int V)
{
    if (B < 1 || N < 1 || V < 1) return DSSD_ERR_INVALID_ARG;
    if (N > DSSD_TREE_MAX_NODES || V > DSSD_MAX_V || (long long)B * N > (long long)DSSD_MAX_ROWS) return DSSD_ERR_UNSUPPORTED;
    return DSSD_OK;
}

// the cache's and the table's shape
dssd_status check_pages(const int32_t *table, int64_t table_stride, int max_pages, int num_pages, int page_size)
{
    if (max_pages < 0 || num_pages < 0 || page_size < 1 || table_stride < max_pages || (max_pages > 0 && !table)) return DSSD_ERR_INVALID_ARG;
    if ((long long)max_pages * page_size > 0x7fffffff - 65536) return DSSD_ERR_UNSUPPORTED;  // a position is an int
    return DSSD_OK;
}

dssd_status attend(const void *q, const int64_t *q_strides, const void *k_new, const void *v_new,
                   const int64_t *new_strides, const void *k_cache, const void *v_cache,
                   const int64_t *cache_strides, dssd_dtype dtype, const int32_t *block_table,
                   int64_t table_stride, int max_pages, int num_pages, int page_size,
                   const int32_t *ctx_len, const int32_t *parents, int B, int N, int Hq, int Hkv, int D,
                   float scale, void *o, const int64_t *o_strides, float *lse, uint32_t *flags,
                   void *workspace, size_t workspace_bytes, void *cuda_stream, int withhold, long long wait_cycles)
{
    dssd::set_last_cuda_error(0);
    if (B < 1 || N < 1 || Hq < 1 || Hkv < 1 || D < 1 || Hq % Hkv) return DSSD_ERR_INVALID_ARG;
    if (N > DSSD_TREE_MAX_NODES || Hq / Hkv > 128 || D > 128 || D % 8) return DSSD_ERR_UNSUPPORTED;
    if (dtype != DSSD_BF16 && dtype != DSSD_F16) return DSSD_ERR_UNSUPPORTED;
    if ((long long)B * N * Hq > 0x7fffffff) return DSSD_ERR_UNSUPPORTED;
    if (!q || !q_strides || !k_new || !v_new || !new_strides || !cache_strides || !ctx_len || !o || !o_strides) return DSSD_ERR_INVALID_ARG;
    dssd_status st = check_pages(block_table, table_stride, max_pages, num_pages, page_size);
    if (st != DSSD_OK) return st;
    if (num_pages > 0 && (!k_cache || !v_cache)) return DSSD_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !isfinite(scale)) return DSSD_ERR_INVALID_ARG;
    for (const void *p : {q, k_new, v_new, k_cache, v_cache, static_cast<const void *>(o)})
        if (!aligned(p, 16)) return DSSD_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
        if (q_strides[i] < 0 || new_strides[i] < 0 || cache_strides[i] < 0 || o_strides[i] < 0) return DSSD_ERR_INVALID_ARG;
        if ((q_strides[i] | new_strides[i] | cache_strides[i] | o_strides[i]) % 8) return DSSD_ERR_UNSUPPORTED;
    }
    // (a tiled copy takes no stride of nothing)
    if ((B > 1 && (!q_strides[0] || !new_strides[0])) || (N > 1 && (!q_strides[1] || !new_strides[1])) || (Hq > 1 && !q_strides[2]) ||
        (Hkv > 1 && (!new_strides[2] || (num_pages > 0 && !cache_strides[2]))) || (num_pages > 1 && !cache_strides[0]) ||
        (num_pages > 0 && page_size > 1 && !cache_strides[1]))
        return DSSD_ERR_UNSUPPORTED;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < dssd_tree_attention_workspace_bytes(B, N, Hq, Hkv, D)) return DSSD_ERR_WORKSPACE;

    dssd::TreeAttentionParams P{};
    P.q = q, P.k_new = k_new, P.v_new = v_new, P.k_cache = k_cache, P.v_cache = v_cache;
    P.q_b = q_strides[0], P.q_n = q_strides[1], P.q_h = q_strides[2];
    P.new_b = new_strides[0], P.new_n = new_strides[1], P.new_h = new_strides[2];
    P.cache_p = cache_strides[0], P.cache_t = cache_strides[1], P.cache_h = cache_strides[2];
    P.o_b = o_strides[0], P.o_n = o_strides[1], P.o_h = o_strides[2];
    P.block_table = block_table;
    P.table_stride = table_stride;
    P.max_pages = max_pages, P.num_pages = num_pages, P.page_size = page_size;
    P.ctx_len = ctx_len;
    P.parents = parents;
    P.B = B, P.N = N, P.Hq = Hq, P.Hkv = Hkv, P.D = D;
    P.scale = scale;
    P.o = o;
    P.lse = lse;
    P.flags = flags;
    P.withhold = withhold, P.wait_cycles = wait_cycles;
    return done(dssd::tree_attention_launch(P, (int)dtype, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

}  // namespace

extern "C" {

size_t dssd_adjust_logits_workspace_bytes(int B, int N, int V, int L, int K)
{
    if (check_tree(B, N, V) != DSSD_OK || V > DSSD_ADJUST_MAX_V || L < 0 || L >= 1 << 29 || K < 0 || K > 65535) return 0;
    return dssd::adjust_workspace(B, N, V, L, K);
}

dssd_status dssd_adjust_logits(const void *logits, dssd_dtype dtype, int64_t row_stride, int B, int N, int V,
                               const int32_t *draft_tokens, const int32_t *parents, const int32_t *history,
                               int64_t history_stride, int L, const int32_t *prompt_len, const int32_t *history_len,
                               const float *repetition, const float *presence, const float *frequency,
                               const int32_t *bias_tokens, const float *bias_values, int K, const uint32_t *mask,
                               int mask_rows, const int32_t *mask_row, void *out, int64_t out_stride, uint32_t *flags,
                               void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    dssd::set_last_cuda_error(0);
    const dssd_status st = check_tree(B, N, V);
    if (st != DSSD_OK) return st;
    if (dtype != DSSD_F32 && dtype != DSSD_BF16) return DSSD_ERR_UNSUPPORTED;
    const size_t esz = dtype == DSSD_BF16 ? 2 : 4;
    if (!logits || !out || row_stride < V || out_stride < V || !aligned(logits, esz) || !aligned(out, esz)) return DSSD_ERR_INVALID_ARG;
    if (out == logits && out_stride != row_stride) return DSSD_ERR_INVALID_ARG;
    if (N > 1 && !draft_tokens) return DSSD_ERR_INVALID_ARG;
    if (L < 0 || K < 0 || mask_rows < 0) return DSSD_ERR_INVALID_ARG;
    if (L > 0 && (!history || !prompt_len || !history_len || history_stride < L)) return DSSD_ERR_INVALID_ARG;
    if (K > 0 && (!bias_tokens || !bias_values)) return DSSD_ERR_INVALID_ARG;
    if (mask_row && !mask && mask_rows > 0) return DSSD_ERR_INVALID_ARG;
    if (mask && !mask_row && (long long)mask_rows < (long long)B * N) return DSSD_ERR_INVALID_ARG;
    if (K > 65535 || L >= 1 << 29 || V > DSSD_ADJUST_MAX_V) return DSSD_ERR_UNSUPPORTED;
    // CTAs of the copy
    const long long per = dssd::adjust_copy_entries((int)dtype);
    if ((long long)B * N * ((V + per + 7) / per) > 0x7fffffff || (long long)B * 16 > 0x7fffffff) return DSSD_ERR_UNSUPPORTED;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < dssd_adjust_logits_workspace_bytes(B, N, V, L, K)) return DSSD_ERR_WORKSPACE;

    dssd::AdjustParams P{};
    P.logits = logits;
    P.out = out;
    P.row_stride = row_stride;
    P.out_stride = out_stride;
    P.draft_tokens = draft_tokens;
    P.parents = parents;
    P.history = history;
    P.history_stride = history_stride;
    P.prompt_len = prompt_len;
    P.history_len = history_len;
    P.repetition = repetition;
    P.presence = presence;
    P.frequency = frequency;
    P.bias_tokens = bias_tokens;
    P.bias_values = bias_values;
    P.mask = mask;
    P.mask_row = mask ? mask_row : nullptr;
    P.flags = flags;
    P.B = B, P.N = N, P.V = V, P.L = L, P.K = K, P.mask_rows = mask_rows;
    return done(dssd::adjust_launch(P, (int)dtype, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

size_t dssd_tree_attention_workspace_bytes(int B, int N, int Hq, int Hkv, int D)
{
    if (B < 1 || N < 1 || N > DSSD_TREE_MAX_NODES || Hq < 1 || Hkv < 1 || Hq % Hkv || Hq / Hkv > 128 || D < 8 || D > 128 || D % 8) return 0;
    return dssd::tree_attention_workspace(B, N, Hq, Hkv, D);
}

dssd_status dssd_tree_attention(const void *q, const int64_t *q_strides, const void *k_new, const void *v_new,
                                const int64_t *new_strides, const void *k_cache, const void *v_cache,
                                const int64_t *cache_strides, dssd_dtype dtype, const int32_t *block_table,
                                int64_t table_stride, int max_pages, int num_pages, int page_size,
                                const int32_t *ctx_len, const int32_t *parents, int B, int N, int Hq, int Hkv, int D,
                                float scale, void *o, const int64_t *o_strides, float *lse, uint32_t *flags,
                                void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    return attend(q, q_strides, k_new, v_new, new_strides, k_cache, v_cache, cache_strides, dtype, block_table, table_stride, max_pages, num_pages, page_size,
                  ctx_len, parents, B, N, Hq, Hkv, D, scale, o, o_strides, lse, flags, workspace, workspace_bytes, cuda_stream, -1, 0);
}

dssd_status dssd_test_tree_attention_wait_runs_out(const void *q, const int64_t *q_strides, const void *k_new, const void *v_new,
                                                   const int64_t *new_strides, const void *k_cache, const void *v_cache,
                                                   const int64_t *cache_strides, dssd_dtype dtype, const int32_t *block_table,
                                                   int64_t table_stride, int max_pages, int num_pages, int page_size,
                                                   const int32_t *ctx_len, const int32_t *parents, int B, int N, int Hq, int Hkv, int D,
                                                   float scale, void *o, const int64_t *o_strides, float *lse, uint32_t *flags,
                                                   void *workspace, size_t workspace_bytes, int withhold_seq, long long wait_cycles, void *cuda_stream)
{
    if (withhold_seq < 0 || withhold_seq >= B || wait_cycles < 1) return DSSD_ERR_INVALID_ARG;
    return attend(q, q_strides, k_new, v_new, new_strides, k_cache, v_cache, cache_strides, dtype, block_table, table_stride, max_pages, num_pages, page_size,
                  ctx_len, parents, B, N, Hq, Hkv, D, scale, o, o_strides, lse, flags, workspace, workspace_bytes, cuda_stream, withhold_seq, wait_cycles);
}

size_t dssd_tree_verify_workspace_bytes(int B, int N, int V)
{
    if (check_tree(B, N, V) != DSSD_OK) return 0;
    return 256;
}

dssd_status dssd_tree_verify(const void *target_logits, dssd_dtype dtype, int64_t row_stride, const float *draft_q,
                             const int32_t *draft_tokens, const int32_t *parents, const float *uniforms,
                             const float *uniforms_rs, double temperature, int replacement, int B, int N, int V,
                             int32_t *accept_len, int32_t *path, int32_t *token, uint32_t *edge_flags,
                             uint32_t *rs_flags, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    dssd::set_last_cuda_error(0);
    const dssd_status st = check_tree(B, N, V);
    if (st != DSSD_OK) return st;
    if (dtype != DSSD_F32 && dtype != DSSD_BF16) return DSSD_ERR_UNSUPPORTED;
    if (!target_logits || !uniforms_rs || !accept_len || !path || !token || row_stride < V) return DSSD_ERR_INVALID_ARG;
    if (N > 1 && (!draft_q || !draft_tokens || !uniforms)) return DSSD_ERR_INVALID_ARG;
    if (!(temperature > 0.0) || !isfinite(temperature)) return DSSD_ERR_INVALID_ARG;
    if (!aligned(target_logits, dtype == DSSD_BF16 ? 2 : 4) || !aligned(draft_q, 4)) return DSSD_ERR_INVALID_ARG;
    // (beyond these log2(e) / T is no number of float32, or masked entries come near the others)
    if ((long long)B * 16 > 0x7fffffff || temperature > 1e30 || temperature < 1e-30) return DSSD_ERR_UNSUPPORTED;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < dssd_tree_verify_workspace_bytes(B, N, V)) return DSSD_ERR_WORKSPACE;

    dssd::TreeVerifyParams P{};
    P.logits = target_logits;
    P.row_stride = row_stride;
    P.draft_q = draft_q;
    P.draft_tokens = draft_tokens;
    P.parents = parents;
    P.uniforms = uniforms;
    P.uniforms_rs = uniforms_rs;
    P.c1 = 1.4426950408889634074 / temperature;
    P.replacement = replacement != 0;
    P.B = B, P.N = N, P.V = V;
    P.accept_len = accept_len;
    P.path = path;
    P.token = token;
    P.edge_flags = edge_flags;
    P.rs_flags = rs_flags;
    return done(dssd::tree_verify_launch(P, (int)dtype, static_cast<cudaStream_t>(cuda_stream)));
}

dssd_status dssd_cache_append(const void *k_new, const void *v_new, const int64_t *new_strides, void *k_cache,
                              void *v_cache, const int64_t *cache_strides, dssd_dtype dtype, const int32_t *block_table,
                              int64_t table_stride, int max_pages, int num_pages, int page_size, const int32_t *ctx_len,
                              const int32_t *accept_len, const int32_t *path, int layers, int B, int N, int Hkv, int D,
                              int32_t *new_len, uint32_t *flags, void *cuda_stream)
{
    dssd::set_last_cuda_error(0);
    if (layers < 1 || B < 1 || N < 1 || Hkv < 1 || D < 1) return DSSD_ERR_INVALID_ARG;
    if (dtype != DSSD_BF16 && dtype != DSSD_F16) return DSSD_ERR_UNSUPPORTED;
    if (!k_new || !v_new || !new_strides || !cache_strides || !ctx_len || !accept_len) return DSSD_ERR_INVALID_ARG;
    const dssd_status st = check_pages(block_table, table_stride, max_pages, num_pages, page_size);
    if (st != DSSD_OK) return st;
    if (num_pages > 0 && (!k_cache || !v_cache)) return DSSD_ERR_INVALID_ARG;
    if (new_len == ctx_len) return DSSD_ERR_INVALID_ARG;
    for (const void *p : {k_new, v_new, static_cast<const void *>(k_cache), static_cast<const void *>(v_cache)})
        if (!aligned(p, 2)) return DSSD_ERR_INVALID_ARG;
    for (int i = 0; i < 4; ++i)
        if (new_strides[i] < 0 || cache_strides[i] < 0) return DSSD_ERR_INVALID_ARG;
    if ((long long)Hkv * D > 1 << 24 || (double)layers * B * N > 1e9) return DSSD_ERR_UNSUPPORTED;
    // (the CTA that reports for a sequence does not wait for those that read its lengths, path and pages)
    for (const void *r : {static_cast<const void *>(new_len), static_cast<const void *>(flags)})
        if (overlap(r, B, ctx_len, B) || overlap(r, B, accept_len, B) || overlap(r, B, path, (long long)B * N) ||
            overlap(r, B, block_table, (B - 1) * table_stride + max_pages))
            return DSSD_ERR_INVALID_ARG;
    if (overlap(new_len, B, flags, B)) return DSSD_ERR_INVALID_ARG;

    dssd::AppendParams P{};
    P.k_new = k_new, P.v_new = v_new, P.k_cache = k_cache, P.v_cache = v_cache;
    P.new_l = new_strides[0], P.new_b = new_strides[1], P.new_n = new_strides[2], P.new_h = new_strides[3];
    P.cache_l = cache_strides[0], P.cache_p = cache_strides[1], P.cache_t = cache_strides[2], P.cache_h = cache_strides[3];
    P.block_table = block_table;
    P.table_stride = table_stride;
    P.max_pages = max_pages, P.num_pages = num_pages, P.page_size = page_size;
    P.ctx_len = ctx_len;
    P.accept_len = accept_len;
    P.path = path;
    P.layers = layers, P.B = B, P.N = N, P.Hkv = Hkv, P.D = D;
    P.new_len = new_len;
    P.flags = flags;
    return done(dssd::append_launch(P, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
