// Attention of a chunk of new tokens over a paged cache.
//
//   out_t = sum_j p_tj v_j,  p = softmax over the keys that token t may see of scale q_t . k_j
//
// in one pass over the keys: with the running maximum m, the running sum l and the running output o of the keys so far,
// a key with score s takes them to m' = max(m, s), l' = l e^(m - m') + e^(s - m'), o' likewise.
//
// This is the form for everything that the tensor-core kernel (paged_attention_tc.cu) does not take: heads of more than 128
// channels, more than 128 query heads to a key head, unaligned rows.  Every token and head reads its keys and values for
// itself, so it is bound by L2: 4096 tokens of 32 heads over 16384 keys take it 366 ms, the tensor-core kernel 0.85.
#include "attention.cuh"

#include <math.h>

namespace fpsk {

// One block per token and query head; its warps take every fourth key, a lane every 32nd channel.
constexpr int kPlainWarps = 4;
template <typename T>
__global__ void __launch_bounds__(32 * kPlainWarps) attention_rows_kernel(const __grid_constant__ AttnArgs g)
{
    constexpr int C = FPSK_MAX_HEAD_DIM / 32;
    __shared__ float sm[kPlainWarps], sl[kPlainWarps], so[kPlainWarps][FPSK_MAX_HEAD_DIM];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int tok = blockIdx.x, head = blockIdx.y;
    int seq = 0;
    for (int base = 0; base < g.n_seqs; base += blockDim.x) {
        const int i = base + threadIdx.x;
        const int before = __syncthreads_count(i < g.n_seqs && g.cu_q[i + 1] <= tok);
        seq += before;
        if (before < (int)blockDim.x) break;
    }
    if (seq >= g.n_seqs) return;
    int lo = 0, hi = 0;
    key_range(g, (long long)g.kv_len[seq] - (g.cu_q[seq + 1] - tok), g.kv_len[seq], lo, hi);
    const T *qp = static_cast<const T *>(g.q) + tok * g.qts + head * g.qhs;
    float q[C], o[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int c = lane + 32 * i;
        q[i] = c < g.dim ? Elem<T>::to_f(qp[c]) * g.scale_log2 : 0.f;
        o[i] = 0.f;
    }
    const int kvh = head / g.group;
    float m = -INFINITY, l = 0.f;
    for (int j = lo + warp; j < hi; j += kPlainWarps) {
        const int col = j / g.page_size, row = j - col * g.page_size;
        const long long page = col < g.max_pages ? g.table[seq * g.table_stride + col] : -1;
        const bool there = page >= 0 && page < g.n_pages;              // else zeros, as in the tensor-core kernel
        if (!there && lane == 0) report_status(g.status, FPSK_ERR_PARAM);
        const T *kp = static_cast<const T *>(g.k) + (there ? page * g.kps + row * g.kts + kvh * g.khs : 0);
        const T *vp = static_cast<const T *>(g.v) + (there ? page * g.vps + row * g.vts + kvh * g.vhs : 0);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = lane + 32 * i;
            if (there && c < g.dim) s = fmaf(q[i], Elem<T>::to_f(kp[c]), s);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        const float m2 = fmaxf(m, s), base = m2 == -INFINITY ? 0.f : m2;
        const float a = exp2f(m - base), p = exp2f(s - base);
        l = fmaf(l, a, p);
        m = m2;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = lane + 32 * i;
            if (c < g.dim) o[i] = fmaf(o[i], a, there ? p * Elem<T>::to_f(vp[c]) : 0.f);
        }
    }
    if (lane == 0) { sm[warp] = m; sl[warp] = l; }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int c = lane + 32 * i;
        if (c < g.dim) so[warp][c] = o[i];
    }
    __syncthreads();
    float top = -INFINITY, total = 0.f;
    for (int w = 0; w < kPlainWarps; ++w) top = fmaxf(top, sm[w]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < kPlainWarps; ++w) total += sl[w] * exp2f(sm[w] - base);
    for (int c = threadIdx.x; c < g.dim; c += blockDim.x) {
        float x = 0.f;
        for (int w = 0; w < kPlainWarps; ++w) x += so[w][c] * exp2f(sm[w] - base);
        static_cast<T *>(g.out)[tok * g.ots + head * g.ohs + c] = Elem<T>::from_f(total != 0.f ? x / total : 0.f);
    }
    if (g.lse && threadIdx.x == 0)
        g.lse[(long long)tok * g.hq + head] = total != 0.f ? (base + log2f(total)) * kLn2 : -INFINITY;
}

}  // namespace fpsk

using namespace fpsk;

extern "C" size_t fpsk_paged_attention_workspace_bytes(void) { return attention_tc_workspace_bytes(); }

extern "C" fpsk_status fpsk_paged_attention(const fpsk_paged_cache *cache, const fpsk_paged_batch *batch, const fpsk_attention *a,
                                            void *workspace, size_t ws_bytes, int32_t *d_status, void *stream)
{
    fpsk_status rc = check_cache(cache);
    if (rc != FPSK_OK) return rc;
    if ((rc = check_batch(batch)) != FPSK_OK) return rc;
    if (!a || !workspace) return FPSK_ERR_NULL;
    if (a->n_heads < 1 || a->n_heads > 65535 || a->n_heads % cache->n_heads || a->max_q_len < 0 || a->max_kv_len < 0) return FPSK_ERR_SHAPE;
    if ((a->causal != 0 && a->causal != 1) || a->window < -1 || !(a->scale >= 0.f) || isinf(a->scale)) return FPSK_ERR_PARAM;
    if (batch->n_tokens > 0 && (!a->q || !a->out)) return FPSK_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return FPSK_ERR_ALIGN;
    if (ws_bytes < fpsk_paged_attention_workspace_bytes()) return FPSK_ERR_WORKSPACE;
    if (batch->n_tokens == 0) return FPSK_OK;
    AttnArgs g = {};
    g.q = a->q; g.out = a->out; g.lse = a->lse; g.k = cache->k; g.v = cache->v;
    g.qts = a->q_token_stride; g.qhs = a->q_head_stride; g.ots = a->out_token_stride; g.ohs = a->out_head_stride;
    g.kps = cache->k_page_stride; g.kts = cache->k_token_stride; g.khs = cache->k_head_stride;
    g.vps = cache->v_page_stride; g.vts = cache->v_token_stride; g.vhs = cache->v_head_stride;
    g.cu_q = batch->cu_q; g.kv_len = batch->kv_len; g.table = batch->block_table;
    g.table_stride = batch->table_stride; g.n_pages = cache->n_pages;
    g.n_seqs = batch->n_seqs; g.max_pages = batch->max_pages; g.page_size = cache->page_size;
    g.n_tokens = (int)batch->n_tokens; g.hq = a->n_heads; g.hk = cache->n_heads; g.group = a->n_heads / cache->n_heads;
    g.dim = cache->head_dim;
    g.causal = a->causal; g.window = a->window;
    g.scale_log2 = (a->scale > 0.f ? a->scale : (float)(1.0 / sqrt((double)g.dim))) * 1.44269504088896341f;
    g.status = d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (attention_tc_takes(g))
        return attention_tc_launch(g, cache->type, a->max_q_len, a->max_kv_len, workspace, st);
    const dim3 grid((unsigned)g.n_tokens, (unsigned)g.hq);
    if (cache->type == FPSK_ELEM_FP16) attention_rows_kernel<__half><<<grid, 32 * kPlainWarps, 0, st>>>(g);
    else attention_rows_kernel<__nv_bfloat16><<<grid, 32 * kPlainWarps, 0, st>>>(g);
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
