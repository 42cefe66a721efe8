// Residual addition and RMS norm, forward (16-bit, FP32 or e4m3 output) and backward.
//
// For a row: h = x + residual, r = (sum h^2 / d + eps)^-1/2, y = h r w; e4m3: s = max |y| / 448 over a group, y / s rounded.
// Backwards: n = h r, g = dy w, dx = r (g - n sum(g n) / d) + dh, dw = sum over the rows of dy n.
//
// The forms here read a row from memory again for what they computed its sums from (it is in L1 or L2 by then).  They take what the ring
// (add_norm_ring.cuh) does not: few rows, where one token of 4096 channels takes 3.6 us, the launch; up to 32 channels, or 512 in rows that start off
// 16 bytes; rows too long for two stages.
#include "add_norm.cuh"

namespace fpsk {

constexpr int kNormThreads = 256;      // of a block whose rows take at most eight warps

// Sums of two values over the warps of a row.  All threads of the block call it.
__device__ __forceinline__ float2 team_sum(float2 v, int warps, float2 *slots)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    if (warps == 1) return v;
    const int warp = threadIdx.x >> 5, first = warp / warps * warps;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[warp] = v;
    __syncthreads();
    float2 s = slots[first];
    for (int i = 1; i < warps; ++i) {
        s.x += slots[first + i].x;
        s.y += slots[first + i].y;
    }
    return s;
}
// Largest magnitude, as its bits: a NaN is larger than all.
__device__ __forceinline__ unsigned int team_max(unsigned int v, int warps, unsigned int *slots)
{
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if (warps == 1) return v;
    const int warp = threadIdx.x >> 5, first = warp / warps * warps;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[warp] = v;
    __syncthreads();
    unsigned int s = slots[first];
    for (int i = 1; i < warps; ++i) s = max(s, slots[first + i]);
    return s;
}
template <typename X, typename R, bool WIDE> __global__ void __launch_bounds__(1024) add_norm_kernel(const __grid_constant__ NormArgs g)
{
    __shared__ float2 sums[32];
    __shared__ unsigned int tops[32];
    let_the_next();
    behind_the_last();
    const int teams = (int)(blockDim.x >> 5) / g.warps, team = (int)(threadIdx.x >> 5) / g.warps;
    const int lanes = 32 * g.warps, lane = (int)threadIdx.x - team * lanes;
    for (long long row0 = (long long)blockIdx.x * teams; row0 < g.n; row0 += (long long)gridDim.x * teams) {
        const long long row = row0 + team;
        const bool live = row < g.n;
        const X *x = static_cast<const X *>(g.x) + (live ? row * g.xs : 0);
        const R *res = g.res ? static_cast<const R *>(g.res) + (live ? row * g.rs : 0) : nullptr;
        const int dim = live ? g.dim : 0;
        auto sum_of = [&](int c, float (&h)[8]) {
            load8<WIDE>(x + c, dim - c < 8 ? dim - c : 8, h);
            if (res) {
                float b[8];
                load8<WIDE>(res + c, dim - c < 8 ? dim - c : 8, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += b[i];
            }
        };
        float2 s = make_float2(0.f, 0.f);
        for (int c = 8 * lane; c < dim; c += 8 * lanes) {
            float h[8];
            sum_of(c, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) s.x = fmaf(h[i], h[i], s.x);
        }
        s = team_sum(s, g.warps, sums);
        const float r = rsqrtf(fmaf(s.x, g.inv_dim, g.eps));
        auto value_of = [&](int c, float (&h)[8], float (&y)[8]) {
            sum_of(c, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = h[i] * r;
            if (g.w) {
                float w[8];
                load8_any<WIDE>(g.w, g.wtype, c, dim - c < 8 ? dim - c : 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] *= w[i];
            }
        };
        float whole = 1.f;
        if (g.ytype == FPSK_ELEM_E4M3 && g.group == 0) {
            unsigned int top = 0;
            for (int c = 8 * lane; c < dim; c += 8 * lanes) {
                float h[8], y[8];
                value_of(c, h, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(y[i]));
            }
            whole = e4m3_scale(team_max(top, g.warps, tops));
            if (live && lane == 0) g.scale[row * g.ss] = whole;
        }
        // (whole warps walk together: groups of lanes share a scale)
        for (int c = 8 * lane; c - 8 * (lane & 31) < dim; c += 8 * lanes) {
            const int n = dim - c < 8 ? dim - c : 8;
            float h[8], y[8];
            value_of(c, h, y);
            if (n > 0 && g.hout) store8<WIDE>(static_cast<R *>(g.hout) + row * g.hs + c, n, h);
            if (g.ytype != FPSK_ELEM_E4M3) {
                if (n > 0) store8_any<WIDE>(g.y, g.ytype, row * g.ys + c, n, y);
                continue;
            }
            float scale = whole;
            if (g.group) {
                unsigned int top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(y[i]));
                for (int o = 1; o < g.group / 8; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                scale = e4m3_scale(top);
                if (n > 0 && c % g.group == 0) g.scale[row * g.ss + c / g.group] = scale;
            }
            const float by = over(scale);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= by;
            unsigned char *out = static_cast<unsigned char *>(g.y) + row * g.ys + c;
            const unsigned int lo = e4m3_pair(y[0], y[1]) | e4m3_pair(y[2], y[3]) << 16, hi = e4m3_pair(y[4], y[5]) | e4m3_pair(y[6], y[7]) << 16;
            if (WIDE && n == 8) *reinterpret_cast<uint2 *>(out) = make_uint2(lo, hi);
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) out[i] = (unsigned char)((i < 4 ? lo : hi) >> 8 * (i & 3));
            }
        }
    }
}

constexpr int kGradVecs = 4;           // of eight channels a thread adds up weight gradients for: 1024 threads hold the widest row

template <typename X, typename G, bool WIDE, int MOST> __global__ void __launch_bounds__(MOST) add_norm_grad_kernel(const __grid_constant__ NormGradArgs g)
{
    __shared__ float2 sums[32];
    const int teams = (int)(blockDim.x >> 5) / g.warps, team = (int)(threadIdx.x >> 5) / g.warps;
    const int lanes = 32 * g.warps, lane = (int)threadIdx.x - team * lanes;
    let_the_next();
    behind_the_last();
    float acc[kGradVecs][8] = {};
    for (long long row0 = (long long)blockIdx.x * teams; row0 < g.n; row0 += (long long)gridDim.x * teams) {
        const long long row = row0 + team;
        const bool live = row < g.n;
        const int dim = live ? g.dim : 0;
        const X *hp = static_cast<const X *>(g.h) + (live ? row * g.hs : 0);
        const G *dyp = static_cast<const G *>(g.dy) + (live ? row * g.dys : 0);
        auto grad_of = [&](int c, int n, float (&d)[8]) {              // d: dy -> dy w
            if (!g.w) return;
            float w[8];
            load8_any<WIDE>(g.w, g.wtype, c, n, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= w[i];
        };
        float2 s = make_float2(0.f, 0.f);
        for (int c = 8 * lane; c < dim; c += 8 * lanes) {
            const int n = dim - c < 8 ? dim - c : 8;
            float h[8], d[8];
            load8<WIDE>(hp + c, n, h);
            load8<WIDE>(dyp + c, n, d);
            grad_of(c, n, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s.x = fmaf(h[i], h[i], s.x);
                s.y = fmaf(h[i], d[i], s.y);
            }
        }
        s = team_sum(s, g.warps, sums);
        const float r = rsqrtf(fmaf(s.x, g.inv_dim, g.eps)), mean = s.y * r * g.inv_dim;
#pragma unroll
        for (int j = 0; j < kGradVecs; ++j) {
            const int c = 8 * (lane + j * lanes), n = dim - c < 8 ? dim - c : 8;
            if (n > 0) {
                float h[8], d[8];
                load8<WIDE>(hp + c, n, h);
                load8<WIDE>(dyp + c, n, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[i] *= r;
                    acc[j][i] = fmaf(d[i], h[i], acc[j][i]);
                }
                grad_of(c, n, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = __fmul_rn(r, fmaf(-h[i], mean, d[i]));
                if (g.dh) {
                    load8<WIDE>(static_cast<const G *>(g.dh) + row * g.dhs + c, n, h);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] += h[i];
                }
                store8<WIDE>(static_cast<G *>(g.dx) + row * g.dxs + c, n, d);
            }
        }
    }
    if (!g.part) return;
    float *part = g.part + ((long long)blockIdx.x * teams + team) * g.dim;
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
        const int c = 8 * (lane + j * lanes);
        if (c < g.dim) store8<false>(part + c, g.dim - c < 8 ? g.dim - c : 8, acc[j]);
    }
}

// dw[c] = sum of `rows` rows of partial gradients: a warp's lanes take neighbouring channels, the warps rows 32 apart, eight at a time.
__global__ void __launch_bounds__(1024) add_norm_sum_kernel(const float *part, int rows, int dim, float *dw)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    let_the_next();
    behind_the_last();
    if (c < dim)
        for (int r = warp; r < rows; r += 32 * 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r + 32 * i < rows ? part[(long long)(r + 32 * i) * dim + c] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
    sums[warp][lane] = s;
    __syncthreads();
    s = sums[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0 && blockIdx.x * 32 + warp < dim) dw[blockIdx.x * 32 + warp] = s;
}
static fpsk_status launch_sum(const float *part, int rows, int dim, float *dw, cudaStream_t st)
{
    Launch launch((unsigned)(dim + 31) / 32, 1024, 0, 1, st);
    FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg, add_norm_sum_kernel, part, rows, dim, dw));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

// warps of a row: a thread takes two vectors of eight channels, four where that would be more than 32 warps
static int warps_of(int dim)
{
    int w = 1;
    while (w < 32 && w * 512 < dim) w *= 2;
    return w;
}

template <typename X, typename R> static fpsk_status launch_norm(const NormArgs &g, bool wide, cudaStream_t st)
{
    const int threads = g.warps > 8 ? 32 * g.warps : kNormThreads, teams = threads / 32 / g.warps;
    const long long steps = (g.n + teams - 1) / teams, most = 1LL << 20;
    const unsigned blocks = (unsigned)(steps < most ? steps : most);
    Launch launch(blocks, threads, 0, 1, st);
    FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg, wide ? add_norm_kernel<X, R, true> : add_norm_kernel<X, R, false>, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

constexpr int kNormGradBlocks = 2 * kSms;
// partial rows of the weight gradient
static int grad_rows(int dim)
{
    const int w = warps_of(dim);
    return kNormGradBlocks * (w > 8 ? 1 : 8 / w);
}

template <typename X, typename G> static fpsk_status launch_norm_grad(const NormGradArgs &g, bool wide, float *dw, cudaStream_t st)
{
    const int threads = g.warps > 8 ? 32 * g.warps : kNormThreads, teams = threads / 32 / g.warps;
    const long long steps = (g.n + teams - 1) / teams;
    const unsigned blocks = (unsigned)(steps < kNormGradBlocks ? steps : kNormGradBlocks);
    if (blocks) {
        Launch launch(blocks, threads, 0, 1, st);
        FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg,
                                        threads > 512 ? (wide ? add_norm_grad_kernel<X, G, true, 1024> : add_norm_grad_kernel<X, G, false, 1024>)
                                                      : (wide ? add_norm_grad_kernel<X, G, true, 512> : add_norm_grad_kernel<X, G, false, 512>),
                                        g));
        FPSK_LAUNCH_CHECK();
    }
    return dw ? launch_sum(g.part, (int)blocks * teams, g.dim, dw, st) : FPSK_OK;
}

}  // namespace fpsk

using namespace fpsk;

static bool rows_ok(long long n, int dim, long long stride) { return n < 2 || stride >= dim; }

extern "C" fpsk_status fpsk_add_rms_norm(const fpsk_add_norm *a, int32_t *d_status, void *stream)
{
    if (!a) return FPSK_ERR_NULL;
    if (a->n_tokens < 0 || a->n_tokens > (1LL << 40) || a->dim < 1 || a->dim > FPSK_MAX_NORM_DIM) return FPSK_ERR_SHAPE;
    if (!elem_ok(a->x_type) || ((a->residual || a->residual_out) && !elem_ok(a->residual_type)) || (a->weight && !elem_ok(a->weight_type)))
        return FPSK_ERR_DTYPE;
    const bool e4m3 = a->y_type == FPSK_ELEM_E4M3;
    if (!e4m3 && !elem_ok(a->y_type)) return FPSK_ERR_DTYPE;
    if (!(a->eps >= 0.f) || a->eps > 3.4e38f) return FPSK_ERR_PARAM;
    if (e4m3 ? a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128 && a->group != 256 : a->group != 0) return FPSK_ERR_PARAM;
    if (a->n_tokens == 0) return FPSK_OK;
    if (!a->x || !a->y || (e4m3 && !a->scale)) return FPSK_ERR_NULL;
    // rows may be read again and again (a stride of 0), but not written over one another
    const int groups = a->group ? (a->dim + a->group - 1) / a->group : 1;
    if (a->x_stride < 0 || a->residual_stride < 0 || !rows_ok(a->n_tokens, a->dim, a->y_stride) ||
        (a->residual_out && !rows_ok(a->n_tokens, a->dim, a->residual_out_stride)) || (e4m3 && !rows_ok(a->n_tokens, groups, a->scale_stride)))
        return FPSK_ERR_SHAPE;
    if (!aligned(a->x, a->x_type) || !aligned(a->residual, a->residual_type) || !aligned(a->residual_out, a->residual_type) || !aligned(a->y, a->y_type) ||
        !aligned(a->weight, a->weight_type) || !aligned(a->scale, FPSK_ELEM_FP32))
        return FPSK_ERR_ALIGN;
    NormArgs g = {};
    g.x = a->x; g.res = a->residual; g.w = a->weight; g.hout = a->residual_out; g.y = a->y; g.scale = a->scale;
    g.xs = a->x_stride; g.rs = a->residual_stride; g.hs = a->residual_out_stride; g.ys = a->y_stride; g.ss = a->scale_stride;
    g.n = a->n_tokens; g.dim = a->dim; g.wtype = a->weight_type; g.ytype = a->y_type; g.group = a->group;
    g.warps = warps_of(a->dim);
    g.eps = a->eps;
    g.inv_dim = 1.f / (float)a->dim;
    const bool wide = row_wide(g.x, a->x_type, g.xs) && row_wide(g.res, a->residual_type, g.rs) && row_wide(g.hout, a->residual_type, g.hs) &&
                      row_wide(g.y, a->y_type, g.ys, e4m3 ? 8 : 16) && row_wide(g.w, a->weight_type, 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int rt = a->residual || a->residual_out ? a->residual_type : FPSK_ELEM_FP32;
    fpsk_status rc;
    if (norm_ring(g, wide, a->x_type, rt, d_status, st, &rc)) return rc;
#define FPSK_RES(X)                                                      \
    (rt == FPSK_ELEM_FP32 ? launch_norm<X, float>(g, wide, st)           \
                          : rt == FPSK_ELEM_FP16 ? launch_norm<X, __half>(g, wide, st) : launch_norm<X, __nv_bfloat16>(g, wide, st))
    if (a->x_type == FPSK_ELEM_FP32) return FPSK_RES(float);
    if (a->x_type == FPSK_ELEM_FP16) return FPSK_RES(__half);
    return FPSK_RES(__nv_bfloat16);
#undef FPSK_RES
}

extern "C" size_t fpsk_add_norm_workspace_bytes(int32_t dim)
{
    if (dim < 1 || dim > FPSK_MAX_NORM_DIM) return 0;
    return align_up((size_t)grad_rows(dim) * dim * sizeof(float), 256);
}

extern "C" fpsk_status fpsk_add_rms_norm_backward(const fpsk_add_norm_grad *a, void *workspace, size_t ws_bytes, int32_t *d_status, void *stream)
{
    if (!a) return FPSK_ERR_NULL;
    if (a->n_tokens < 0 || a->n_tokens > (1LL << 40) || a->dim < 1 || a->dim > FPSK_MAX_NORM_DIM) return FPSK_ERR_SHAPE;
    if (!elem_ok(a->h_type) || !elem_ok(a->grad_type) || (a->weight && !elem_ok(a->weight_type))) return FPSK_ERR_DTYPE;
    if (!(a->eps >= 0.f) || a->eps > 3.4e38f) return FPSK_ERR_PARAM;
    if (a->n_tokens > 0 && (!a->h || !a->dy || !a->dx)) return FPSK_ERR_NULL;
    if (a->h_stride < 0 || a->dy_stride < 0 || a->dh_stride < 0 || !rows_ok(a->n_tokens, a->dim, a->dx_stride)) return FPSK_ERR_SHAPE;
    if (a->dweight) {
        if (!workspace) return FPSK_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) % 256) return FPSK_ERR_ALIGN;
        if (ws_bytes < fpsk_add_norm_workspace_bytes(a->dim)) return FPSK_ERR_WORKSPACE;
    }
    if (!aligned(a->h, a->h_type) || !aligned(a->dy, a->grad_type) || !aligned(a->dh, a->grad_type) || !aligned(a->dx, a->grad_type) ||
        !aligned(a->weight, a->weight_type) || !aligned(a->dweight, FPSK_ELEM_FP32))
        return FPSK_ERR_ALIGN;
    NormGradArgs g = {};
    g.h = a->h; g.dy = a->dy; g.dh = a->dh; g.w = a->weight; g.dx = a->dx;
    g.part = a->dweight ? static_cast<float *>(workspace) : nullptr;
    g.hs = a->h_stride; g.dys = a->dy_stride; g.dhs = a->dh_stride; g.dxs = a->dx_stride;
    g.n = a->n_tokens; g.dim = a->dim; g.wtype = a->weight_type;
    g.warps = warps_of(a->dim);
    g.eps = a->eps;
    g.inv_dim = 1.f / (float)a->dim;
    const bool wide = row_wide(g.h, a->h_type, g.hs) && row_wide(g.dy, a->grad_type, g.dys) && row_wide(g.dh, a->grad_type, g.dhs) &&
                      row_wide(g.dx, a->grad_type, g.dxs) && row_wide(g.w, a->weight_type, 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    fpsk_status rc;
    int rows;
    if (norm_grad_ring(g, wide, a->h_type, a->grad_type, d_status, st, &rc, &rows)) return rc != FPSK_OK || !a->dweight ? rc : launch_sum(g.part, rows, g.dim, a->dweight, st);
#define FPSK_IN(G)                                                                              \
    (a->h_type == FPSK_ELEM_FP32 ? launch_norm_grad<float, G>(g, wide, a->dweight, st)          \
                                 : a->h_type == FPSK_ELEM_FP16 ? launch_norm_grad<__half, G>(g, wide, a->dweight, st)  \
                                                               : launch_norm_grad<__nv_bfloat16, G>(g, wide, a->dweight, st))
    if (a->grad_type == FPSK_ELEM_FP32) return FPSK_IN(float);
    if (a->grad_type == FPSK_ELEM_FP16) return FPSK_IN(__half);
    return FPSK_IN(__nv_bfloat16);
#undef FPSK_IN
}
