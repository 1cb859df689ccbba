// halo_paged_prompt_mha: causal attention of packed chunks of new tokens over a paged K/V cache.
#include <math.h>

#include "prompt_line.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale);
long long paged_stride(const halo_paged_shape& s);
}  // namespace halo

using namespace halo;

extern "C" size_t halo_paged_prompt_mha_workspace_bytes(const halo_paged_shape* shape, int n_tok, int n_seq) {
    if (check_paged_shape(shape) != HALO_OK || n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES || n_tok <= 0 || n_tok > HALO_MAX_PROMPT_ROWS) return 0;
    return prompt::f32_workspace(*shape, n_tok, n_seq);
}

extern "C" halo_status halo_paged_prompt_mha(const halo_paged_shape* shape, int n_tok, int n_seq, const void* q, long long q_stride,
                                             const int32_t* q_start, const void* K_cache, const void* V_cache, const uint8_t* K_scale,
                                             const uint8_t* V_scale, const int32_t* block_table, const int32_t* seq_len,
                                             const uint8_t* keep, float scale, void* out, float* lse, void* workspace,
                                             size_t workspace_bytes, uint32_t* dev_status, void* stream) {
    halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!q || !q_start || !K_cache || !V_cache || !block_table || !seq_len || !out || q == out) return HALO_ERR_ARG;
    if (!isfinite(scale)) return HALO_ERR_ARG;
    if (n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES || n_tok <= 0 || n_tok > HALO_MAX_PROMPT_ROWS) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    if (q_stride < static_cast<long long>(shape->n_heads) * shape->head_dim) return HALO_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out) || q_stride * elem % 16 != 0) return HALO_ERR_ALIGN;
    rc = check_eight(*shape, K_scale, V_scale);
    if (rc != HALO_OK) return rc;
    const size_t need = halo_paged_prompt_mha_workspace_bytes(shape, n_tok, n_seq);
    if (!workspace || workspace_bytes < need) return HALO_ERR_WORKSPACE;
    if (!aligned16(workspace)) return HALO_ERR_ALIGN;
    prompt::Args a = {};
    a.n_tok = n_tok;
    a.n_seq = n_seq;
    a.H = shape->n_heads;
    a.Hk = shape->n_kv_heads;
    a.G = a.H / a.Hk;
    a.dh = shape->head_dim;
    a.page_size = shape->page_size;
    a.page_shift = -1;
    for (int b = 0; b < 31; ++b)
        if (shape->page_size == 1 << b) a.page_shift = b;
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.page_stride = paged_stride(*shape);
    a.q_stride = q_stride;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.q = q;
    a.K = K_cache;
    a.V = V_cache;
    a.K_scale = K_scale;
    a.V_scale = V_scale;
    a.q_start = q_start;
    a.table = block_table;
    a.seq_len = seq_len;
    a.keep = keep;
    a.out = out;
    a.lse = lse;
    a.status = dev_status;
    return prompt::f32_launch(a, *shape, workspace, static_cast<cudaStream_t>(stream));
}
