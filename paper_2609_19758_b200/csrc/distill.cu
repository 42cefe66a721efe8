// The loss of rows of logits against a teacher's top logits, and its gradient.
//
// q = softmax(x / tau), p over the listed tokens; loss = sum_j p_j (log p_j - log q_j); d/dx_v = (m q_v - p_v) / tau, m = sum p.
// In powers of two: y = x c with c = log2(e) / tau, L = log2 sum 2^y, q = 2^(y - L).
//
// A cluster of blocks takes a row, each a slice of the vocabulary: one pass for L, the blocks' sums joined in their order, and one
// for the gradient.  The listed tokens' p are taken off at the end, by the block whose slice they lie in.
#include "decoder.cuh"

namespace fpsk {

struct DistillArgs {
    const void *x, *tok, *t;
    const float *weight;
    float *loss, *lse;
    void *dx;
    long long xs, toks, ts, dxs, rows;
    int vocab, top;
    int tok_bytes, t_type, grad_type;
    int normalize, backward;           // backward: lse is given
    float inv_tau, c;                  // 1 / tau, log2(e) / tau
    int blocks, slice;
};

__device__ __forceinline__ void store_grad(void *p, int type, long long at, float v)
{
    if (type == FPSK_ELEM_FP32) static_cast<float *>(p)[at] = v;
    else if (type == FPSK_ELEM_FP16) static_cast<__half *>(p)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v);
}

// Over the block, in a fixed order; `slots`: kRowWarps floats.
__device__ __forceinline__ float block_sum(float v, float *slots)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < kRowWarps; ++w) v += slots[w];
    return v;
}
__device__ __forceinline__ float block_max(float v, float *slots)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < kRowWarps; ++w) v = fmaxf(v, slots[w]);
    return v;
}

template <typename X> __global__ void __launch_bounds__(kRowThreads) distill_kernel(const __grid_constant__ DistillArgs g)
{
    constexpr int kEach = FPSK_MAX_TOP / kRowThreads;
    __shared__ int tok[FPSK_MAX_TOP];
    __shared__ float prob[FPSK_MAX_TOP];
    __shared__ float slots[kRowWarps], tops[kRowWarps];
    __shared__ float mine[4];                                          // largest, sum, loss: read by the other blocks
    const int tid = threadIdx.x;
    const unsigned int rank = cluster_rank();
    const int lo = (int)min((long long)g.vocab, (long long)rank * g.slice), hi = (int)min((long long)g.vocab, (long long)lo + g.slice);
    for (long long row = blockIdx.x / g.blocks; row < g.rows; row += gridDim.x / g.blocks) {
        const X *x = static_cast<const X *>(g.x) + row * g.xs;
        const float weight = g.weight ? g.weight[row] : 1.f;
        if (weight == 0.f) {
            if (g.dx)
                for (int v = lo + tid; v < hi; v += kRowThreads) store_grad(g.dx, g.grad_type, row * g.dxs + v, 0.f);
            if (!g.backward && rank == 0 && tid == 0) {
                g.loss[row] = 0.f;
                if (g.lse) g.lse[row] = 0.f;
            }
            continue;
        }
        // the teacher's probabilities
        float logp[kEach], xs[kEach];
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = tid + e * kRowThreads;
            logp[e] = -INFINITY;
            if (j < g.top) {
                const long long token = g.tok_bytes == 4 ? (long long)static_cast<const int *>(g.tok)[row * g.toks + j] : static_cast<const long long *>(g.tok)[row * g.toks + j];
                const bool in = token >= 0 && token < g.vocab;
                tok[j] = in ? (int)token : -1;
                if (in) {
                    const long long at = row * g.ts + j;
                    const float t = g.t_type == FPSK_ELEM_FP32 ? static_cast<const float *>(g.t)[at]
                                    : g.t_type == FPSK_ELEM_FP16 ? __half2float(static_cast<const __half *>(g.t)[at])
                                                                 : __bfloat162float(static_cast<const __nv_bfloat16 *>(g.t)[at]);
                    logp[e] = g.normalize ? t * g.inv_tau : t;
                }
            }
            most = fmaxf(most, logp[e]);
        }
        if (g.normalize) {
            most = block_max(most, slots);
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < kEach; ++e) s += logp[e] == -INFINITY ? 0.f : expf(logp[e] - most);
            s = block_sum(s, slots);
            const float off = most + logf(s);
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (logp[e] != -INFINITY) logp[e] -= off;
        }
        float mass = 0.f;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = tid + e * kRowThreads;
            const float p = logp[e] == -INFINITY ? 0.f : expf(logp[e]);
            if (j < g.top) prob[j] = p;
            mass += p;
        }
        mass = block_sum(mass, slots);

        float l2;                                                      // log2 of the sum
        if (g.backward) {
            l2 = g.lse[row] * kLog2e;
        } else {
            PowerSum p = {-INFINITY, 0.f};
            for (int v = lo + tid; v < hi; v += kRowThreads) p.add(Elem<X>::to_f(x[v]) * g.c);
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const float om = __shfl_xor_sync(0xFFFFFFFFu, p.m, o), os = __shfl_xor_sync(0xFFFFFFFFu, p.s, o);
                p.join(om, os);
            }
            __syncthreads();
            if ((tid & 31) == 0) {
                tops[tid >> 5] = p.m;
                slots[tid >> 5] = p.s;
            }
            __syncthreads();
            p = PowerSum{tops[0], slots[0]};
            for (int w = 1; w < kRowWarps; ++w) p.join(tops[w], slots[w]);
            if (tid == 0) {
                mine[0] = p.m;
                mine[1] = p.s;
            }
            cluster_sync();
            p = PowerSum{cluster_load(&mine[0], 0), cluster_load(&mine[1], 0)};
            for (int b = 1; b < g.blocks; ++b) p.join(cluster_load(&mine[0], b), cluster_load(&mine[1], b));
            l2 = log2_of(p);
        }
        // what the loss and the gradient want of the listed tokens, before the gradient is written (in the logits' place perhaps)
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = tid + e * kRowThreads;
            xs[e] = 0.f;
            if (j < g.top && tok[j] >= lo && tok[j] < hi) {
                xs[e] = Elem<X>::to_f(x[tok[j]]);
                if (logp[e] != -INFINITY) part = fmaf(prob[j], logp[e] - (xs[e] * g.inv_tau - l2 * kLn2), part);
            }
        }
        if (!g.backward) {
            part = block_sum(part, slots);
            if (tid == 0) mine[2] = part;
            cluster_sync();
            if (rank == 0 && tid == 0) {
                for (int b = 1; b < g.blocks; ++b) part += cluster_load(&mine[2], b);
                g.loss[row] = part;
                if (g.lse) g.lse[row] = l2 * kLn2;
            }
        } else {
            __syncthreads();
        }
        if (g.dx) {
            const float wt = weight * g.inv_tau, wm = wt * mass;
            for (int v = lo + tid; v < hi; v += kRowThreads)
                store_grad(g.dx, g.grad_type, row * g.dxs + v, mass == 0.f ? 0.f : wm * exp2_fast(fmaf(Elem<X>::to_f(x[v]), g.c, -l2)));
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int j = tid + e * kRowThreads;
                if (j < g.top && tok[j] >= lo && tok[j] < hi) {
                    // one of those that list a token writes it
                    float p = 0.f;
                    bool first = true;
                    for (int i = 0; i < g.top; ++i)
                        if (tok[i] == tok[j]) {
                            if (i < j) first = false;
                            p += prob[i];
                        }
                    if (first && mass != 0.f)
                        store_grad(g.dx, g.grad_type, row * g.dxs + tok[j], fmaf(wm, exp2_fast(fmaf(xs[e], g.c, -l2)), -wt * p));
                }
            }
        }
        if (!g.backward) cluster_sync();                               // (what the others read here is read)
        __syncthreads();
    }
}

template <typename X> static fpsk_status launch_distill(DistillArgs g, cudaStream_t st)
{
    constexpr int kGrain = 4096;
    const int grains = (g.vocab + kGrain - 1) / kGrain;
    g.blocks = 1;
    while (g.blocks < kRowMostBlocks && 2 * g.blocks <= grains && g.rows * g.blocks < 4 * kSms) g.blocks *= 2;
    g.slice = (grains + g.blocks - 1) / g.blocks * kGrain;
    const long long most = 1 << 20;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((g.rows < most ? g.rows : most) * g.blocks));
    cfg.blockDim = dim3(kRowThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = g.blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, distill_kernel<X>, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

}  // namespace fpsk

using namespace fpsk;

static fpsk_status distill(const fpsk_distill *a, bool backward, void *stream)
{
    if (!a) return FPSK_ERR_NULL;
    if (a->n_rows < 0 || a->n_rows > 0x7FFFFFFFLL || a->vocab < 1 || a->vocab > FPSK_MAX_VOCAB || a->top < 0 || a->top > FPSK_MAX_TOP) return FPSK_ERR_SHAPE;
    if (!elem_ok(a->logits_type) || !elem_ok(a->teacher_type) || (a->dlogits && !elem_ok(a->grad_type))) return FPSK_ERR_DTYPE;
    if (a->token_bytes != 4 && a->token_bytes != 8) return FPSK_ERR_DTYPE;
    if (!(a->temperature > 0.f) || a->temperature > 3.4e38f) return FPSK_ERR_PARAM;
    if (a->n_rows == 0) return FPSK_OK;
    if (!a->logits || (a->top > 0 && (!a->teacher_token || !a->teacher_logit))) return FPSK_ERR_NULL;
    if (backward ? !a->lse || !a->dlogits : !a->loss) return FPSK_ERR_NULL;
    if (a->logits_stride < 0 || a->token_stride < 0 || a->teacher_stride < 0 || (a->dlogits && a->n_rows > 1 && a->dlogits_stride < a->vocab)) return FPSK_ERR_SHAPE;
    const double inv = 1.0 / (double)a->temperature;
    if (inv > 3.4e38) return FPSK_ERR_PARAM;
    DistillArgs g = {};
    g.x = a->logits; g.tok = a->teacher_token; g.t = a->teacher_logit; g.weight = a->row_weight;
    g.loss = a->loss; g.lse = a->lse; g.dx = a->dlogits;
    g.xs = a->logits_stride; g.toks = a->token_stride; g.ts = a->teacher_stride; g.dxs = a->dlogits_stride;
    g.rows = a->n_rows; g.vocab = a->vocab; g.top = a->top;
    g.tok_bytes = a->token_bytes; g.t_type = a->teacher_type; g.grad_type = a->grad_type;
    g.normalize = a->normalize != 0; g.backward = backward;
    g.inv_tau = (float)inv;
    g.c = (float)(inv * 1.4426950408889634);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->logits_type == FPSK_ELEM_FP32) return launch_distill<float>(g, st);
    if (a->logits_type == FPSK_ELEM_FP16) return launch_distill<__half>(g, st);
    return launch_distill<__nv_bfloat16>(g, st);
}

extern "C" fpsk_status fpsk_distill_loss(const fpsk_distill *a, void *stream) { return distill(a, false, stream); }
extern "C" fpsk_status fpsk_distill_loss_backward(const fpsk_distill *a, void *stream) { return distill(a, true, stream); }
