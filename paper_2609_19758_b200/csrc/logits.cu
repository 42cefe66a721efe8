// Penalties, biases and grammar masks on rows of logits, with the greedy token and the log-sum-exp of what is left.
//
// For a token v of a row: z = l_v; seen: z > 0 ? z / rep : z rep; z -= freq c + pres where c > 0; z += biases; masked: -inf.
//
// A cluster of blocks takes a row, each a slice of the vocabulary.  Which of a chunk's tokens the history and the biases touch is
// gathered in shared memory first.
#include "decoder.cuh"

namespace fpsk {

struct LogitsArgs {
    const void *x;
    void *out;
    long long xs, os, rows;
    int vocab, out_type;
    const int *history, *history_len, *prompt_len;
    long long history_stride;
    int history_width;
    const float *rep, *freq, *pres;
    const int *bias_ptr, *bias_token;
    const float *bias_value;
    long long n_biases;
    const int *mask, *mask_row;
    long long mask_stride, n_masks;
    int *token;
    float *lse;
    int blocks;                        // of a row
    int slice;                         // tokens of a block, a multiple of the chunk
    int32_t *status;
};

constexpr int kChunk = 4096;
constexpr unsigned int kInPrompt = 0x80000000u;

// the order of argmax: a NaN above all, -0 like 0, the lowest token of equal ones
__device__ __forceinline__ unsigned long long pick_key(float z, int v)
{
    const unsigned int b = __float_as_uint(z + 0.f);
    const unsigned int k = z != z ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (unsigned long long)k << 32 | (0xFFFFFFFFu - (unsigned int)v);
}
constexpr unsigned int kKeyNothing = 0x007FFFFFu;                      // of -inf

__device__ __forceinline__ void store_elem(void *p, int type, long long at, float v)
{
    if (type == FPSK_ELEM_FP32) static_cast<float *>(p)[at] = v;
    else if (type == FPSK_ELEM_FP16) static_cast<__half *>(p)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v);
}

template <typename X> __global__ void __launch_bounds__(kRowThreads) adjust_logits_kernel(const __grid_constant__ LogitsArgs g)
{
    __shared__ unsigned int said[kChunk];                              // times behind the prompt, and whether in it
    __shared__ float bias[kChunk];
    __shared__ unsigned long long keys[kRowWarps];
    __shared__ float tops[kRowWarps], sums[kRowWarps];
    __shared__ float mine[4];                                          // key (two halves), largest, sum: read by the first block
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned int rank = cluster_rank();
    const int lo = (int)min((long long)g.vocab, (long long)rank * g.slice), hi = (int)min((long long)g.vocab, (long long)lo + g.slice);
    for (long long row = blockIdx.x / g.blocks; row < g.rows; row += gridDim.x / g.blocks) {
        const X *x = static_cast<const X *>(g.x) + row * g.xs;
        const int *history = g.history ? g.history + row * g.history_stride : nullptr;
        int n_hist = history ? g.history_width : 0;
        if (history && g.history_len) n_hist = max(0, min(n_hist, g.history_len[row]));
        const int n_prompt = history && g.prompt_len ? g.prompt_len[row] : 0;
        const float rep = g.rep ? g.rep[row] : 1.f, freq = g.freq ? g.freq[row] : 0.f, pres = g.pres ? g.pres[row] : 0.f;
        long long b0 = 0, b1 = 0;
        if (g.bias_ptr) {
            b0 = max(0LL, (long long)g.bias_ptr[row]);
            b1 = min(g.n_biases, (long long)g.bias_ptr[row + 1]);
        }
        const int *mask = nullptr;
        bool nothing = false;
        if (g.mask) {
            const long long m = g.mask_row ? (long long)g.mask_row[row] : row;
            if (m >= g.n_masks) {
                nothing = true;
                if (tid == 0) report_status(g.status, FPSK_ERR_PARAM);
            } else if (m >= 0) {
                mask = g.mask + m * g.mask_stride;
            }
        }
        unsigned long long best = 0;
        PowerSum p = {-INFINITY, 0.f};
        for (int c0 = lo; c0 < hi; c0 += kChunk) {
            const int n = min(kChunk, hi - c0);
            __syncthreads();
            for (int i = tid; i < kChunk; i += kRowThreads) {
                said[i] = 0;
                bias[i] = 0.f;
            }
            __syncthreads();
            for (int i = tid; i < n_hist; i += kRowThreads) {
                const unsigned int at = (unsigned int)history[i] - (unsigned int)c0;
                if (at < (unsigned int)n) {
                    if (i < n_prompt) atomicOr(&said[at], kInPrompt);
                    else atomicAdd(&said[at], 1u);
                }
            }
            if (warp == 0 && b0 < b1) {
                // in the list's order, whatever comes twice
                for (long long i0 = b0; i0 < b1; i0 += 32) {
                    const long long i = i0 + lane;
                    const unsigned int at = i < b1 ? (unsigned int)g.bias_token[i] - (unsigned int)c0 : 0xFFFFFFFFu;
                    const bool in = at < (unsigned int)n;
                    const float value = in ? g.bias_value[i] : 0.f;
                    const unsigned int same = __match_any_sync(0xFFFFFFFFu, in ? (int)at : -1 - lane);
                    if (__any_sync(0xFFFFFFFFu, __popc(same) > 1)) {
                        for (int l = 0; l < 32; ++l) {
                            if (l == lane && in) bias[at] += value;
                            __syncwarp();
                        }
                    } else if (in) {
                        bias[at] += value;
                    }
                    __syncwarp();
                }
            }
            __syncthreads();
            for (int i = tid; i < n; i += kRowThreads) {
                const int v = c0 + i;
                float z = Elem<X>::to_f(x[v]);
                const unsigned int c = said[i];
                if (c) z = z > 0.f ? __fdiv_rn(z, rep) : __fmul_rn(z, rep);
                if (c & ~kInPrompt) z = __fsub_rn(z, __fadd_rn(__fmul_rn((float)(c & ~kInPrompt), freq), pres));
                if (b0 < b1) z += bias[i];
                if (nothing || (mask && !(mask[v >> 5] >> (v & 31) & 1))) z = -INFINITY;
                if (g.out) store_elem(g.out, g.out_type, row * g.os + v, z);
                if (g.token || g.lse) {
                    best = max(best, pick_key(z, v));
                    p.add(z * kLog2e);
                }
            }
        }
        if (!g.token && !g.lse) continue;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
            const float om = __shfl_xor_sync(0xFFFFFFFFu, p.m, o), os = __shfl_xor_sync(0xFFFFFFFFu, p.s, o);
            p.join(om, os);
        }
        if (lane == 0) {
            keys[warp] = best;
            tops[warp] = p.m;
            sums[warp] = p.s;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kRowWarps; ++w) {
                best = max(best, keys[w]);
                p.join(tops[w], sums[w]);
            }
            mine[0] = __uint_as_float((unsigned int)(best >> 32));
            mine[1] = __uint_as_float((unsigned int)best);
            mine[2] = p.m;
            mine[3] = p.s;
        }
        cluster_sync();
        if (rank == 0 && tid == 0) {
            for (int b = 1; b < g.blocks; ++b) {
                const unsigned long long k = (unsigned long long)__float_as_uint(cluster_load(&mine[0], b)) << 32 | __float_as_uint(cluster_load(&mine[1], b));
                best = max(best, k);
                p.join(cluster_load(&mine[2], b), cluster_load(&mine[3], b));
            }
            if (g.token) g.token[row] = (unsigned int)(best >> 32) <= kKeyNothing ? -1 : (int)(0xFFFFFFFFu - (unsigned int)best);
            if (g.lse) g.lse[row] = log2_of(p) * kLn2;
        }
        cluster_sync();
    }
}

template <typename X> static fpsk_status launch_logits(LogitsArgs g, cudaStream_t st)
{
    const int chunks = (g.vocab + kChunk - 1) / kChunk;
    g.blocks = 1;
    while (g.blocks < kRowMostBlocks && 2 * g.blocks <= chunks && g.rows * g.blocks < 4 * kSms) g.blocks *= 2;
    g.slice = (chunks + g.blocks - 1) / g.blocks * kChunk;
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
    FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, adjust_logits_kernel<X>, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

}  // namespace fpsk

using namespace fpsk;

extern "C" fpsk_status fpsk_adjust_logits(const fpsk_logits *a, int32_t *d_status, void *stream)
{
    if (!a) return FPSK_ERR_NULL;
    if (a->n_rows < 0 || a->n_rows > 0x7FFFFFFFLL || a->vocab < 1 || a->vocab > FPSK_MAX_VOCAB) return FPSK_ERR_SHAPE;
    if (!elem_ok(a->logits_type) || (a->out && !elem_ok(a->out_type))) return FPSK_ERR_DTYPE;
    if (a->n_rows == 0) return FPSK_OK;
    if (!a->logits || (!a->out && !a->token && !a->lse)) return FPSK_ERR_NULL;
    if (a->logits_stride < 0 || (a->out && a->n_rows > 1 && a->out_stride < a->vocab)) return FPSK_ERR_SHAPE;
    if (a->history && (a->history_width < 0 || a->history_stride < 0)) return FPSK_ERR_SHAPE;
    if (!a->history && (a->history_len || a->prompt_len || a->repetition || a->frequency || a->presence)) return FPSK_ERR_NULL;
    if (a->bias_ptr && (a->n_biases < 0 || (a->n_biases > 0 && (!a->bias_token || !a->bias_value)))) return FPSK_ERR_NULL;
    if (a->mask && (a->n_masks < 0 || a->mask_stride < 0 || (!a->mask_row && a->n_masks < a->n_rows))) return FPSK_ERR_SHAPE;
    if (!a->mask && a->mask_row) return FPSK_ERR_NULL;
    LogitsArgs g = {};
    g.x = a->logits; g.out = a->out; g.xs = a->logits_stride; g.os = a->out_stride; g.rows = a->n_rows;
    g.vocab = a->vocab; g.out_type = a->out_type;
    g.history = a->history; g.history_len = a->history_len; g.prompt_len = a->prompt_len;
    g.history_stride = a->history_stride; g.history_width = a->history_width;
    g.rep = a->repetition; g.freq = a->frequency; g.pres = a->presence;
    g.bias_ptr = a->n_biases > 0 ? a->bias_ptr : nullptr; g.bias_token = a->bias_token; g.bias_value = a->bias_value; g.n_biases = a->n_biases;
    g.mask = a->mask; g.mask_row = a->mask_row; g.mask_stride = a->mask_stride; g.n_masks = a->n_masks;
    g.token = a->token; g.lse = a->lse; g.status = d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->logits_type == FPSK_ELEM_FP32) return launch_logits<float>(g, st);
    if (a->logits_type == FPSK_ELEM_FP16) return launch_logits<__half>(g, st);
    return launch_logits<__nv_bfloat16>(g, st);
}
