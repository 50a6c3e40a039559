// C-ABI entry points of the operators around the linear layers (norm, 4-bit
// paged cache, attention): argument checks, always before any HIP call, and
// dispatch to the kernel launchers.
#include "tf_kv4.h"

namespace tf {
int launch_add_rms_norm(bool bf, const void* x, const void* residual, const void* post, const void* gate,
                        int64_t gate_stride, float scale, const void* weight, float offset, float eps, int64_t M,
                        int64_t N, void* r_out, void* y, hipStream_t s);
int launch_kv4_append(const tf_kv4_cache& c, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                      const void* v, int64_t v_stride, const float* cos, const float* sin, int64_t positions,
                      const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens, int q_heads,
                      void* q_out, void* k_out, hipStream_t s);
int launch_kv4_read(const tf_kv4_cache& c, const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens,
                    void* k, void* v, hipStream_t s);
int64_t kv4_attention_workspace_bytes(int64_t batch, int q_len, int q_heads, int kv_heads, int D);
int launch_kv4_attention(const tf_kv4_cache& c, const void* q, int64_t q_stride, const int32_t* lens, int64_t batch,
                         int q_len, int q_heads, float scale, void* out, void* ws, hipStream_t s);
int launch_prompt_attention(bool bf, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int64_t batch,
                            int64_t tokens_q, int64_t tokens_k, int q_heads, int kv_heads, int D, float scale,
                            bool causal, void* out, void* ws, hipStream_t s);
int64_t prompt_attention_workspace_bytes(int64_t batch, int64_t tokens_q, int64_t tokens_k, int q_heads, int D);
}  // namespace tf

namespace {

bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool bad_dtype(int dtype) { return dtype != TF_F16 && dtype != TF_BF16; }
bool bad_head_dim(int d) { return d != 64 && d != 128 && d != 256; }
bool bad_heads(int64_t h) { return h < 1 || h > TF_MAX_HEADS; }
bool bad_stride(int64_t stride, int heads, int d) {
    // a kernel's 32-bit offsets span 64 tokens
    return stride % 8 != 0 || stride < (int64_t)heads * d || stride > (int64_t(1) << 24);
}
// A launch has fewer than 2^32 threads.
bool too_many(int64_t threads) { return threads > (int64_t)UINT32_MAX; }
bool bad_scale(float s) { return !(s > 0.f) || s > 1e30f; }

int check_cache_shape(int64_t pages, int page_size, int kv_heads, int head_dim) {
    if (bad_head_dim(head_dim) || bad_heads(kv_heads)) return TF_ERR_SHAPE;
    if (page_size <= 0 || page_size % tf::kKvTile != 0 || page_size > TF_MAX_DIM) return TF_ERR_SHAPE;
    if (pages < 1 || pages > INT32_MAX) return TF_ERR_SHAPE;
    // offsets are 64-bit
    const int64_t page = (int64_t)kv_heads * (page_size / tf::kKvTile) * tf::kv4_tile_bytes(head_dim);
    if (pages > INT64_MAX / page) return TF_ERR_SHAPE;
    return TF_OK;
}

int check_cache(const tf_kv4_cache* c, int64_t batch) {
    if (!c || !c->data || !c->table) return TF_ERR_NULL;
    if (bad_dtype(c->dtype)) return TF_ERR_ARG;
    const int rc = check_cache_shape(c->pages, c->page_size, c->kv_heads, c->head_dim);
    if (rc) return rc;
    if (batch < 1 || batch > TF_MAX_BATCH) return TF_ERR_SHAPE;
    // positions are 32-bit
    if (c->max_pages < 1 || c->max_pages > INT32_MAX / c->page_size || c->table_stride < c->max_pages ||
        c->table_stride > (int64_t(1) << 40))
        return TF_ERR_SHAPE;
    if (misaligned(c->data, 256) || misaligned(c->table, 4)) return TF_ERR_ALIGN;
    return TF_OK;
}

// Query rows of one key/value head, 16 or 32 a workgroup.
int64_t attention_items(int64_t batch, int q_len, int q_heads, int kv_heads) {
    return batch * kv_heads * (((int64_t)q_len * (q_heads / kv_heads) + 15) / 16);
}

}  // namespace

extern "C" {

int tf_add_rms_norm(int dtype, const void* X, const void* residual, const void* post_weight, const void* gate,
                    int64_t gate_stride, float scale, const void* weight, float weight_offset, float eps, int64_t M,
                    int64_t N, void* residual_out, void* Y, void* stream) {
    if (!X || (!residual_out && !Y) || (Y && !weight)) return TF_ERR_NULL;
    if (bad_dtype(dtype) || !(eps >= 0.f)) return TF_ERR_ARG;
    if (M < 1 || M > TF_MAX_M || N <= 0 || N > TF_MAX_DIM || N % 8 != 0) return TF_ERR_SHAPE;
    if (gate && gate_stride != 0 && (gate_stride < N || gate_stride % 8 != 0 || gate_stride > (int64_t(1) << 40)))
        return TF_ERR_SHAPE;
    for (const void* p : {X, residual, post_weight, gate, weight, (const void*)residual_out, (const void*)Y})
        if (misaligned(p)) return TF_ERR_ALIGN;
    return tf::launch_add_rms_norm(dtype == TF_BF16, X, residual, post_weight, gate, gate_stride, scale, weight,
                                   weight_offset, eps, M, N, residual_out, Y, static_cast<hipStream_t>(stream));
}

int64_t tf_kv4_cache_bytes(int64_t pages, int page_size, int kv_heads, int head_dim) {
    const int rc = check_cache_shape(pages, page_size, kv_heads, head_dim);
    if (rc) return rc;
    return pages * kv_heads * (page_size / tf::kKvTile) * tf::kv4_tile_bytes(head_dim);
}

int tf_kv4_append(const tf_kv4_cache* cache, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                  const void* V, int64_t v_stride, const float* cos, const float* sin, int64_t positions,
                  const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens, int q_heads, void* Q_out,
                  void* K_out, void* stream) {
    int rc = check_cache(cache, batch);
    if (rc) return rc;
    if (!K || !V || !cu || !starts || (!cos) != (!sin) || (!Q) != (!Q_out)) return TF_ERR_NULL;
    if (tokens < 1 || tokens > TF_MAX_M) return TF_ERR_SHAPE;
    if (Q ? bad_heads(q_heads) || bad_stride(q_stride, q_heads, cache->head_dim) : q_heads != 0) return TF_ERR_SHAPE;
    if (bad_stride(k_stride, cache->kv_heads, cache->head_dim) ||
        bad_stride(v_stride, cache->kv_heads, cache->head_dim))
        return TF_ERR_SHAPE;
    if (cos && positions < 1) return TF_ERR_SHAPE;
    if (too_many(tokens * (q_heads + 2 * cache->kv_heads) * (cache->head_dim / 16))) return TF_ERR_SHAPE;
    for (const void* p : {Q, K, V, (const void*)cos, (const void*)sin, (const void*)Q_out, (const void*)K_out})
        if (misaligned(p)) return TF_ERR_ALIGN;
    if (misaligned(cu, 4) || misaligned(starts, 4)) return TF_ERR_ALIGN;
    return tf::launch_kv4_append(*cache, Q, q_stride, K, k_stride, V, v_stride, cos, sin, positions, cu, starts,
                                 batch, tokens, q_heads, Q_out, K_out, static_cast<hipStream_t>(stream));
}

int tf_kv4_read(const tf_kv4_cache* cache, const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens,
                void* K_out, void* V_out, void* stream) {
    int rc = check_cache(cache, batch);
    if (rc) return rc;
    if (!cu || !starts || !K_out || !V_out) return TF_ERR_NULL;
    if (tokens < 1 || tokens > TF_MAX_M) return TF_ERR_SHAPE;
    if (too_many(tokens * 2 * cache->kv_heads * (cache->head_dim / 16))) return TF_ERR_SHAPE;
    if (misaligned(K_out) || misaligned(V_out) || misaligned(cu, 4) || misaligned(starts, 4)) return TF_ERR_ALIGN;
    return tf::launch_kv4_read(*cache, cu, starts, batch, tokens, K_out, V_out, static_cast<hipStream_t>(stream));
}

int64_t tf_kv4_attention_workspace_bytes(int64_t batch, int q_len, int q_heads, int kv_heads, int head_dim) {
    if (q_len < 1 || q_len > TF_KV4_MAX_Q) return TF_ERR_ARG;
    if (batch < 1 || batch > TF_MAX_BATCH || bad_heads(q_heads) || bad_heads(kv_heads) || q_heads % kv_heads != 0 ||
        bad_head_dim(head_dim))
        return TF_ERR_SHAPE;
    return tf::kv4_attention_workspace_bytes(batch, q_len, q_heads, kv_heads, head_dim);
}

int tf_kv4_attention(const tf_kv4_cache* cache, const void* Q, int64_t q_stride, const int32_t* lens, int64_t batch,
                     int q_len, int q_heads, float scale, void* O, void* workspace, size_t workspace_bytes,
                     void* stream) {
    int rc = check_cache(cache, batch);
    if (rc) return rc;
    if (!Q || !lens || !O || !workspace) return TF_ERR_NULL;
    const int64_t need =
        tf_kv4_attention_workspace_bytes(batch, q_len, q_heads, cache->kv_heads, cache->head_dim);
    if (need < 0) return (int)need;
    if (bad_stride(q_stride, q_heads, cache->head_dim)) return TF_ERR_SHAPE;
    // the kernel counts pieces of all sequences and heads in 32 bits
    const int64_t pieces = cache->max_pages * cache->page_size / 128 + 4;
    if (attention_items(batch, q_len, q_heads, cache->kv_heads) > INT32_MAX / pieces) return TF_ERR_SHAPE;
    if (bad_scale(scale) || (int64_t)workspace_bytes < need) return TF_ERR_ARG;
    if (misaligned(Q) || misaligned(O) || misaligned(workspace) || misaligned(lens, 4)) return TF_ERR_ALIGN;
    const auto turn = tf::workspace_turn(workspace);
    return tf::launch_kv4_attention(*cache, Q, q_stride, lens, batch, q_len, q_heads, scale, O, workspace,
                                    static_cast<hipStream_t>(stream));
}

int64_t tf_prompt_attention_workspace_bytes(int64_t batch, int64_t tokens_q, int64_t tokens_k, int q_heads,
                                            int kv_heads, int head_dim) {
    if (bad_head_dim(head_dim) || bad_heads(q_heads) || bad_heads(kv_heads) || q_heads % kv_heads != 0)
        return TF_ERR_SHAPE;
    if (batch < 1 || batch > TF_MAX_BATCH || tokens_q < 1 || tokens_q > TF_MAX_M || tokens_k < 1 ||
        tokens_k > TF_MAX_M)
        return TF_ERR_SHAPE;
    // 256 threads for each head of 128 queries, the last of each sequence perhaps fewer
    if (too_many((tokens_q + 127 * (batch < tokens_q ? batch : tokens_q)) * 2 * q_heads)) return TF_ERR_SHAPE;
    return tf::prompt_attention_workspace_bytes(batch, tokens_q, tokens_k, q_heads, head_dim);
}

int tf_prompt_attention(int dtype, const void* Q, int64_t q_stride, const void* K, int64_t k_stride, const void* V,
                        int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int64_t batch, int64_t tokens_q,
                        int64_t tokens_k, int q_heads, int kv_heads, int head_dim, float scale, int causal, void* O,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!Q || !K || !V || !cu_q || !cu_k || !O) return TF_ERR_NULL;
    if (bad_dtype(dtype) || bad_scale(scale)) return TF_ERR_ARG;
    const int64_t need =
        tf_prompt_attention_workspace_bytes(batch, tokens_q, tokens_k, q_heads, kv_heads, head_dim);
    if (need < 0) return (int)need;
    if (bad_stride(q_stride, q_heads, head_dim) || bad_stride(k_stride, kv_heads, head_dim) ||
        bad_stride(v_stride, kv_heads, head_dim))
        return TF_ERR_SHAPE;
    if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(cu_q, 4) ||
        misaligned(cu_k, 4) || misaligned(workspace))
        return TF_ERR_ALIGN;
    if (workspace && (int64_t)workspace_bytes < need) return TF_ERR_ARG;
    const auto turn = tf::workspace_turn(need > 0 ? workspace : nullptr);
    return tf::launch_prompt_attention(dtype == TF_BF16, Q, q_stride, K, k_stride, V, v_stride, cu_q, cu_k, batch,
                                       tokens_q, tokens_k, q_heads, kv_heads, head_dim, scale, causal != 0, O,
                                       need > 0 ? workspace : nullptr, static_cast<hipStream_t>(stream));
}

}  // extern "C"
