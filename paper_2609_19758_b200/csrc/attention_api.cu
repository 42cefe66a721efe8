// Argument checks of the attention operators and the entry points that only prepare.
#include "attention.cuh"

namespace fpsk {

bool elem_ok(int type) { return type == FPSK_ELEM_FP16 || type == FPSK_ELEM_BF16 || type == FPSK_ELEM_FP32; }
bool head_dim_ok(int dim) { return dim >= 8 && dim <= FPSK_MAX_HEAD_DIM && dim % 8 == 0; }

fpsk_status check_cache(const fpsk_paged_cache *c)
{
    if (!c || !c->k || !c->v) return FPSK_ERR_NULL;
    if (c->type != FPSK_ELEM_FP16 && c->type != FPSK_ELEM_BF16) return FPSK_ERR_DTYPE;
    if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFFLL || c->page_size < 1 || c->page_size > (1 << 20)) return FPSK_ERR_SHAPE;
    if (c->n_heads < 1 || c->n_heads > 65536 || !head_dim_ok(c->head_dim)) return FPSK_ERR_SHAPE;
    const int64_t s[] = {c->k_page_stride, c->k_token_stride, c->k_head_stride, c->v_page_stride, c->v_token_stride, c->v_head_stride};
    for (int64_t x : s)
        if (x < 0) return FPSK_ERR_SHAPE;
    // rows of different heads or tokens must not overlap
    if ((c->n_heads > 1 && (c->k_head_stride < c->head_dim || c->v_head_stride < c->head_dim)) ||
        (c->page_size > 1 && (c->k_token_stride < c->head_dim || c->v_token_stride < c->head_dim)) ||
        (c->n_pages > 1 && (c->k_page_stride < c->head_dim || c->v_page_stride < c->head_dim)))
        return FPSK_ERR_SHAPE;
    return FPSK_OK;
}

fpsk_status check_batch(const fpsk_paged_batch *b)
{
    if (!b) return FPSK_ERR_NULL;
    if (b->n_seqs < 0 || b->n_seqs > (1 << 20) || b->n_tokens < 0 || b->n_tokens > 0x7FFFFFFFLL || b->max_pages < 0) return FPSK_ERR_SHAPE;
    if (b->table_stride < b->max_pages) return FPSK_ERR_SHAPE;
    if (b->n_seqs == 0 && b->n_tokens > 0) return FPSK_ERR_SHAPE;
    if (b->n_seqs > 0 && (!b->cu_q || !b->kv_len || (b->max_pages > 0 && !b->block_table))) return FPSK_ERR_NULL;
    return FPSK_OK;
}

}  // namespace fpsk

extern "C" fpsk_status fpsk_attention_workspace_init(void *workspace, size_t ws_bytes, void *stream)
{
    if (!workspace) return FPSK_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return FPSK_ERR_ALIGN;
    if (ws_bytes < fpsk::kAttnSyncBytes) return FPSK_ERR_WORKSPACE;
    FPSK_CUDA_OK(cudaMemsetAsync(workspace, 0, fpsk::kAttnSyncBytes, static_cast<cudaStream_t>(stream)));
    return FPSK_OK;
}
