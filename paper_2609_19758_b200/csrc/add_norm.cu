// Residual addition and RMS norm, forward (16-bit, FP32 or e4m3 output) and backward.
//
// For a row: h = x + residual, r = (sum h^2 / d + eps)^-1/2, y = h r w; e4m3: s = max |y| / 448 over a group, y / s rounded.
// Backwards: n = h r, g = dy w, dx = r (g - n sum(g n) / d) + dh, dw = sum over the rows of dy n.
#include "decoder.cuh"

#include <cuda_fp8.h>

namespace fpsk {

struct NormArgs {
    const void *x, *res, *w;
    void *hout, *y;
    float *scale;
    long long xs, rs, hs, ys, ss;
    long long n;
    int dim, wtype, ytype, group;      // group: 0 or a power of two
    int warps;                         // of a row
    float eps, inv_dim;
};
struct NormGradArgs {
    const void *h, *dy, *dh, *w;
    void *dx;
    float *part;                       // [row teams][dim]
    long long hs, dys, dhs, dxs;
    long long n;
    int dim, wtype;
    int warps;
    float eps, inv_dim;
};

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
__device__ __forceinline__ unsigned int magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// The scale of a group whose largest magnitude has these bits, and one over it: a product and an approximate reciprocal (one unit), as
// two divisions for every eight channels took a fifth of the kernel.
__device__ __forceinline__ float e4m3_scale(unsigned int top)
{
    if (top == 0) return 1.f;
    const float s = __uint_as_float(top) * (1.f / 448.f);
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;                  // (a NaN stays)
}
__device__ __forceinline__ float over(float scale)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
    return r;
}
__device__ __forceinline__ unsigned int e4m3_pair(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
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

// ---------------------------------------------------------------- rows through a ring
// For many rows of 513 to 16384 channels: one warp of a block copies whole rows into a ring of stages, so that what is in flight does
// not depend on the other warps' registers, and those take a row each pass: sums over the row's threads, one barrier, the result.
// Rows that start off 16 bytes come as their aligned middles, and their first and last elements by plain loads a stage ahead.
// Above 8192 channels a row is divided among a cluster of blocks, which tell each other their sums.
struct RingRows {
    const char *base;
    long long stride;                  // bytes from row to row
    int size;                          // of an element
    int at;                            // in a row's part of a stage
};
struct RingArgs {
    NormArgs f;
    NormGradArgs b;
    RingRows in[3];
    int inputs;
    int row_bytes, stage_bytes, stages;
    int teams, log_teams;              // rows of a stage
    int blocks, slice;                 // a row's blocks, and how many channels each but the last has
    long long n, steps;
    int32_t *status;
};
constexpr int kRingMost = 8, kRingEdges = 6, kRingTeams = 8, kRingMostBlocks = 4;

// team of W warps: sums of two values, the same order everywhere; slots of the team alternate from row to row
__device__ __forceinline__ float2 ring_sum(float2 v, int warps, int team, float2 *slots)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    if (lane == 0) slots[(threadIdx.x >> 5) - team * warps] = v;
    if (warps == 1) return v;
    bar_sync(1 + team, 32 * warps);
    v = lane < warps ? slots[lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    return v;
}

// The copying warp.
template <bool WIDE>
__device__ __forceinline__ void ring_copy(const RingArgs &g, int c0, int dim, long long first, long long stride, uint32_t smem, unsigned long long *full, unsigned long long *empty)
{
    const int lane = threadIdx.x & 31;
    bool ok = true;
    int slot = 0;
    uint32_t phase = 0;
    unsigned int k = 0;
    const int mine = lane < g.teams * g.inputs ? lane : -1, my_row = mine >= 0 ? mine & (g.teams - 1) : 0, my_in = mine >= 0 ? mine >> g.log_teams : 0;
    // edge i of this lane: element e < 8 in front of the aligned middle, or e - 8 behind it
    unsigned int edge[kRingEdges];
    auto edge_of = [&](int i, long long step, const char *&from, uint32_t &to, int &size) {
        const int at = lane + 32 * i, e = at & 15, row = at >> 4 & (g.teams - 1), in = at >> (4 + g.log_teams);
        const long long r = (step << g.log_teams) + row;
        if (in >= g.inputs || step >= g.steps || r >= g.n) return false;
        const RingRows &p = g.in[in];
        size = p.size;
        const char *start = p.base + r * p.stride + (long long)c0 * p.size;
        const int all = dim * p.size, shift = (int)(reinterpret_cast<uintptr_t>(start) & 15), head = min(all, (16 - shift) & 15), tail = (all - head) & 15;
        const int off = e < 8 ? e * p.size : all - tail + (e - 8) * p.size;
        if (e < 8 ? off >= head : off >= all) return false;
        from = start + off;
        to = smem + row * g.row_bytes + p.at + shift + off;
        return true;
    };
    auto ask = [&](long long step) {
        if (WIDE) return;
#pragma unroll
        for (int i = 0; i < kRingEdges; ++i) {
            const char *from;
            uint32_t to;
            int size;
            edge[i] = 0;
            if (edge_of(i, step, from, to, size)) edge[i] = size == 4 ? *reinterpret_cast<const unsigned int *>(from) : *reinterpret_cast<const unsigned short *>(from);
        }
    };
    ask(first);
    for (long long step = first; step < g.steps; step += stride) {
        if (ok && !mbar_wait_bounded(smem_u32(&empty[slot]), phase ^ 1u)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        const uint32_t bar = smem_u32(&full[slot]), stage = slot * g.stage_bytes;
        int bytes = 0, shift = 0, head = 0;
        const char *start = nullptr;
        const RingRows &p = g.in[my_in];
        const long long r = (step << g.log_teams) + my_row;
        if (mine >= 0 && r < g.n) {
            start = p.base + r * p.stride + (long long)c0 * p.size;
            if (!WIDE) {
                shift = (int)(reinterpret_cast<uintptr_t>(start) & 15);
                head = min(dim * p.size, (16 - shift) & 15);
            }
            bytes = (dim * p.size - head) & ~15;
        }
        const int all = __reduce_add_sync(0xFFFFFFFFu, bytes);
        if (!WIDE) {
#pragma unroll
            for (int i = 0; i < kRingEdges; ++i) {
                const char *from;
                uint32_t to;
                int size;
                if (edge_of(i, step, from, to, size)) {
                    if (size == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + stage), "r"(edge[i]) : "memory");
                    else asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + stage), "h"((unsigned short)edge[i]) : "memory");
                }
            }
            __syncwarp();
        }
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)all);
        __syncwarp();
        if (bytes) bulk_g2s(smem + stage + my_row * g.row_bytes + p.at + shift + head, start + head, (uint32_t)bytes, bar);
        ask(step + stride);
        ++k;
        if (++slot == g.stages) {
            slot = 0;
            phase ^= 1u;
        }
    }
    let_the_next();
    // no copy is left in flight
    if (lane == 0)
        for (unsigned int back = min(k, (unsigned int)g.stages); back; --back) {
            const unsigned int piece = k - back;
            mbar_wait_bounded(smem_u32(&full[piece % g.stages]), piece / g.stages & 1u);
        }
}

// Vector j of a thread's channels: WIDE eight neighbours, j vectors of `lanes` threads on, else eight single ones, `lanes` apart.
template <bool WIDE> __device__ __forceinline__ int channel(int lane, int lanes, int j, int i) { return WIDE ? 8 * (lane + j * lanes) + i : lane + (8 * j + i) * lanes; }
// It from a row in shared memory, as pairs (0 behind the row).
template <bool WIDE> __device__ __forceinline__ void ring_load(const float *row, int lane, int lanes, int j, int dim, float2 (&v)[4])
{
    if (WIDE) {
        const int c = 8 * (lane + j * lanes);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (c < dim) {
            a = *reinterpret_cast<const float4 *>(row + c);
            b = *reinterpret_cast<const float4 *>(row + c + 4);
        }
        v[0] = make_float2(a.x, a.y); v[1] = make_float2(a.z, a.w);
        v[2] = make_float2(b.x, b.y); v[3] = make_float2(b.z, b.w);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = channel<false>(lane, lanes, j, 2 * i);
        v[i] = make_float2(c < dim ? row[c] : 0.f, c + lanes < dim ? row[c + lanes] : 0.f);
    }
}
template <bool WIDE, typename T> __device__ __forceinline__ void ring_load(const T *row, int lane, int lanes, int j, int dim, float2 (&v)[4])
{
    if (WIDE) {
        const int c = 8 * (lane + j * lanes);
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (c < dim) u = *reinterpret_cast<const uint4 *>(row + c);
        v[0] = HalfTraits<T>::unpack2(u.x); v[1] = HalfTraits<T>::unpack2(u.y);
        v[2] = HalfTraits<T>::unpack2(u.z); v[3] = HalfTraits<T>::unpack2(u.w);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = channel<false>(lane, lanes, j, 2 * i);
        v[i] = make_float2(c < dim ? Elem<T>::to_f(row[c]) : 0.f, c + lanes < dim ? Elem<T>::to_f(row[c + lanes]) : 0.f);
    }
}
template <bool WIDE> __device__ __forceinline__ void ring_weights(const void *w, int type, int lane, int lanes, int j, int dim, float2 (&v)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(1.f, 1.f);
    if (!w) return;
    float t[8];
    const int c = channel<WIDE>(lane, lanes, j, 0);
    if (WIDE) {
        if (c >= dim) return;
        load8_any<true>(w, type, c, 8, t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int ci = c + i * lanes;
            t[i] = ci >= dim ? 0.f
                   : type == FPSK_ELEM_FP32 ? static_cast<const float *>(w)[ci]
                   : type == FPSK_ELEM_FP16 ? __half2float(static_cast<const __half *>(w)[ci])
                                            : __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[ci]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(t[2 * i], t[2 * i + 1]);
}
template <bool WIDE, typename T> __device__ __forceinline__ void ring_store(T *row, int lane, int lanes, int j, int dim, const float2 (&v)[4])
{
    const int c = channel<WIDE>(lane, lanes, j, 0);
    if (WIDE) {
        if (c < dim) store_vec<T, 8>(row + c, true, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i * lanes < dim) row[c + i * lanes] = Elem<T>::from_f(i & 1 ? v[i / 2].y : v[i / 2].x);
}
template <bool WIDE> __device__ __forceinline__ void ring_store_any(void *p, int type, long long at, int lane, int lanes, int j, int dim, const float2 (&v)[4])
{
    if (type == FPSK_ELEM_FP32) ring_store<WIDE>(static_cast<float *>(p) + at, lane, lanes, j, dim, v);
    else if (type == FPSK_ELEM_FP16) ring_store<WIDE>(static_cast<__half *>(p) + at, lane, lanes, j, dim, v);
    else ring_store<WIDE>(static_cast<__nv_bfloat16 *>(p) + at, lane, lanes, j, dim, v);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Threads of a row's channels: J vectors of eight each; MOST: of the largest block.  The weights and their gradients stay in registers.
template <typename X, typename R, bool WIDE, bool GRAD, int MOST, int PER_SM>
__global__ void __launch_bounds__(MOST, PER_SM) add_norm_ring_kernel(const __grid_constant__ RingArgs g)
{
    constexpr int J = 2;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned long long full[kRingMost], empty[kRingMost], met[2];
    __shared__ float2 sums[2][kRingTeams][16];                         // of the teams' warps
    __shared__ unsigned int tops[2][kRingTeams][16];
    __shared__ float4 blocks_sum[2][kRingMostBlocks];                  // written by the row's blocks
    const int workers = (int)blockDim.x - 32, warps = workers / 32 >> g.log_teams;
    if (threadIdx.x == 0) {
        for (int s = 0; s < g.stages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), workers / 32);
        }
        mbar_init(smem_u32(&met[0]), 1);
        mbar_init(smem_u32(&met[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const bool shared_row = g.blocks > 1;
    if (shared_row) cluster_sync();
    behind_the_last();
    const int rank = shared_row ? (int)cluster_rank() : 0, c0 = rank * g.slice;
    const int row_dim = GRAD ? g.b.dim : g.f.dim, dim = min(g.slice, row_dim - c0);
    const long long first_step = blockIdx.x / g.blocks, step_stride = gridDim.x / g.blocks;
    if ((int)threadIdx.x >= workers) {
        ring_copy<WIDE>(g, c0, dim, first_step, step_stride, smem_u32(smem), full, empty);
        if (shared_row) cluster_sync();
        return;
    }
    const int team = (int)(threadIdx.x >> 5) / warps, lanes = 32 * warps, lane = (int)threadIdx.x - team * lanes;
    const float eps = GRAD ? g.b.eps : g.f.eps, inv_dim = GRAD ? g.b.inv_dim : g.f.inv_dim;
    float2 w[J][4], acc[GRAD ? J : 1][4] = {};
    {
        const void *weights = GRAD ? g.b.w : g.f.w;
        const int type = GRAD ? g.b.wtype : g.f.wtype;
        if (weights) weights = static_cast<const char *>(weights) + c0 * elem_bytes(type);
#pragma unroll
        for (int j = 0; j < J; ++j) ring_weights<WIDE>(weights, type, lane, lanes, j, dim, w[j]);
    }
    bool ok = true;
    int slot = 0, turn = 0;
    uint32_t phase = 0, meeting = 0;
    // this block's part of a row's sums (or largest), joined with the others' in their order
    auto meet = [&](float2 mine, unsigned int top) {
        float4 r = make_float4(mine.x, mine.y, __uint_as_float(top), 0.f);
        if (!shared_row) return r;
        const int at = meeting & 1;
        if ((int)threadIdx.x < g.blocks) {                             // (one row at a time: one team)
            if (threadIdx.x == 0) mbar_expect_tx(smem_u32(&met[at]), 16u * g.blocks);
            asm volatile(
                "{\n\t.reg .b32 a, m;\n\t"
                "mapa.shared::cluster.u32 a, %0, %2;\n\t"
                "mapa.shared::cluster.u32 m, %1, %2;\n\t"
                "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %5}, [m];\n\t}"
                ::"r"(smem_u32(&blocks_sum[at][rank])), "r"(smem_u32(&met[at])), "r"(threadIdx.x), "f"(r.x), "f"(r.y), "f"(r.z)
                : "memory");
        }
        if (ok && !mbar_wait_bounded(smem_u32(&met[at]), meeting >> 1 & 1u)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
        ++meeting;
        r = blocks_sum[at][0];
        for (int b = 1; b < g.blocks; ++b) {
            const float4 o = blocks_sum[at][b];
            r = make_float4(r.x + o.x, r.y + o.y, __uint_as_float(max(__float_as_uint(r.z), __float_as_uint(o.z))), 0.f);
        }
        return r;
    };
    const int log_group = GRAD ? 0 : 31 - __clz(max(g.f.group, 1));
    for (long long step = first_step; step < g.steps; step += step_stride, turn ^= 1) {
        const long long row = (step << g.log_teams) + team;
        const bool live = row < g.n;
        const int here = live ? dim : 0;
        if (ok && !mbar_wait_bounded(smem_u32(&full[slot]), phase)) ok = false;           // (the copying warp tells)
        auto input = [&](int i) {
            const int shift = WIDE ? 0 : (int)(reinterpret_cast<uintptr_t>(g.in[i].base + row * g.in[i].stride + (long long)c0 * g.in[i].size) & 15);
            return smem + slot * g.stage_bytes + team * g.row_bytes + g.in[i].at + shift;
        };
        auto release = [&] {
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&empty[slot]));
        };
        const X *first = reinterpret_cast<const X *>(input(0));
        const R *second = reinterpret_cast<const R *>(input(1));
        float2 sh = both(0.f), sg = both(0.f);
        if (GRAD) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float2 h[4], d[4];
                ring_load<WIDE>(first, lane, lanes, j, here, h);
                ring_load<WIDE>(second, lane, lanes, j, here, d);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sh = __ffma2_rn(h[i], h[i], sh);
                    sg = __ffma2_rn(h[i], __fmul2_rn(d[i], w[j][i]), sg);
                }
            }
            const float4 s = meet(ring_sum(make_float2(sh.x + sh.y, sg.x + sg.y), warps, team, sums[turn][team]), 0u);
            const float r = rsqrtf(fmaf(s.x, inv_dim, eps));
            // dx = (dy w - h r^2 mean(dy w h)) r + dh
            const float2 rr = both(r), off = both(-s.y * r * inv_dim * r);
            const R *third = g.b.dh ? reinterpret_cast<const R *>(input(2)) : nullptr;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float2 h[4], d[4];
                ring_load<WIDE>(first, lane, lanes, j, here, h);
                ring_load<WIDE>(second, lane, lanes, j, here, d);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[j][i] = __ffma2_rn(d[i], live ? __fmul2_rn(h[i], rr) : both(0.f), acc[j][i]);
                    d[i] = __fmul2_rn(rr, __ffma2_rn(h[i], off, __fmul2_rn(d[i], w[j][i])));
                }
                if (third) {
                    ring_load<WIDE>(third, lane, lanes, j, here, h);
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[i] = __fadd2_rn(d[i], h[i]);
                }
                if (j == J - 1) release();
                if (live) ring_store<WIDE>(static_cast<R *>(g.b.dx) + row * g.b.dxs + c0, lane, lanes, j, dim, d);
            }
        } else {
            float2 h[J][4];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                ring_load<WIDE>(first, lane, lanes, j, here, h[j]);
                if (g.f.res) {
                    float2 b[4];
                    ring_load<WIDE>(second, lane, lanes, j, here, b);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[j][i] = __fadd2_rn(h[j][i], b[i]);
                }
                if (j == J - 1) release();
                if (live && g.f.hout) ring_store<WIDE>(static_cast<R *>(g.f.hout) + row * g.f.hs + c0, lane, lanes, j, dim, h[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i) sh = __ffma2_rn(h[j][i], h[j][i], sh);
            }
            const float4 s = meet(ring_sum(make_float2(sh.x + sh.y, 0.f), warps, team, sums[turn][team]), 0u);
            const float2 rr = both(rsqrtf(fmaf(s.x, inv_dim, eps)));
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) h[j][i] = __fmul2_rn(__fmul2_rn(h[j][i], rr), w[j][i]);
            if (g.f.ytype != FPSK_ELEM_E4M3) {
                if (live) {
#pragma unroll
                    for (int j = 0; j < J; ++j) ring_store_any<WIDE>(g.f.y, g.f.ytype, row * g.f.ys + c0, lane, lanes, j, dim, h[j]);
                }
            } else if (WIDE) {
                // (a vector's eight channels are in one group, and a group's vectors in neighbouring lanes)
                unsigned int top[J], most = 0;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    top[j] = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) top[j] = max(top[j], max(magnitude(h[j][i].x), magnitude(h[j][i].y)));
                    if (8 * (lane + j * lanes) >= here) top[j] = 0;
                    most = max(most, top[j]);
                }
                float whole = 1.f;
                if (g.f.group) {
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1)
                        if (8 * o < g.f.group) {
#pragma unroll
                            for (int j = 0; j < J; ++j) top[j] = max(top[j], __shfl_xor_sync(0xFFFFFFFFu, top[j], o));
                        }
                } else {
                    most = __reduce_max_sync(0xFFFFFFFFu, most);
                    if (warps > 1) {
                        if ((threadIdx.x & 31) == 0) tops[turn][team][lane >> 5] = most;
                        bar_sync(1 + team, lanes);
                        most = __reduce_max_sync(0xFFFFFFFFu, (lane & 31) < warps ? tops[turn][team][lane & 31] : 0u);
                    }
                    whole = e4m3_scale(__float_as_uint(meet(both(0.f), most).z));
                    if (live && lane == 0 && rank == 0) g.f.scale[row * g.f.ss] = whole;
                }
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int c = 8 * (lane + j * lanes);
                    float scale = whole;
                    if (g.f.group) {
                        scale = e4m3_scale(top[j]);
                        if (c < here && (c & (g.f.group - 1)) == 0) g.f.scale[row * g.f.ss + (c0 + c >> log_group)] = scale;
                    }
                    const float2 by = both(over(scale));
                    unsigned int q[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 y = __fmul2_rn(h[j][i], by);
                        q[i] = e4m3_pair(y.x, y.y);
                    }
                    if (c < here) *reinterpret_cast<uint2 *>(static_cast<unsigned char *>(g.f.y) + row * g.f.ys + c0 + c) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
                }
            }
        }
        if (++slot == g.stages) {
            slot = 0;
            phase ^= 1u;
        }
    }
    if (GRAD && g.b.part) {
        float *part = g.b.part + ((first_step << g.log_teams) + team) * row_dim + c0;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = channel<WIDE>(lane, lanes, j, i);
                if (c < dim) part[c] = i & 1 ? acc[GRAD ? j : 0][i / 2].y : acc[GRAD ? j : 0][i / 2].x;
            }
    }
    if (shared_row) cluster_sync();                                    // no block leaves before what the others send it
}

// Whether the ring takes a call, and how.  A thread has sixteen channels and a block up to eight warps that work, two blocks to an SM:
// one row, or as many short ones as fill them.  Above 4096 channels a row has sixteen warps of a block that has its SM to itself, above 8192 two or
// four such blocks.  (Two blocks of eight warps for 8192 channels would leave each a ring of two stages.)
constexpr int kRingOne = 218 * 1024, kRingHalf = 108 * 1024;
static bool ring_plan(RingArgs &g, int dim, bool wide, int &threads)
{
    if (dim <= 128) return false;
    g.blocks = dim <= 8192 ? 1 : dim <= 16384 ? 2 : 4;
    // (a multiple of the largest group of channels with one scale)
    g.slice = g.blocks == 1 ? dim : ((dim + g.blocks - 1) / g.blocks + 255) / 256 * 256;
    const int warps = (g.slice + 511) / 512;
    if (warps == 1 && !wide) return false;                             // (eight rows' edges are too many for the copying warp)
    g.log_teams = warps > 4 ? 0 : warps > 2 ? 1 : warps > 1 ? 2 : 3;
    g.teams = 1 << g.log_teams;
    threads = 32 * (warps * g.teams + 1);
    g.row_bytes = 0;
    for (int i = 0; i < g.inputs; ++i) {
        g.in[i].at = g.row_bytes;
        g.row_bytes += (g.slice * g.in[i].size + 15) / 16 * 16 + (wide ? 0 : 16);
    }
    g.stage_bytes = (int)align_up((size_t)g.row_bytes * g.teams, 128);
    g.stages = (warps <= 8 ? kRingHalf : kRingOne) / g.stage_bytes;
    if (g.stages < 2) return false;
    if (g.stages > kRingMost) g.stages = kRingMost;
    g.steps = (g.n + g.teams - 1) >> g.log_teams;
    return g.steps * g.blocks >= 2 * kSms;
}
// rows of partial weight gradients at most
static int ring_most(const RingArgs &g, int threads) { return kSms * (threads > 288 ? 1 : 2) / g.blocks; }

template <typename X, typename R, bool GRAD> static fpsk_status launch_ring(const RingArgs &g, bool wide, int threads, int &rows, cudaStream_t st)
{
    Launch launch((unsigned)g.blocks, threads, (size_t)g.stages * g.stage_bytes, g.blocks, st);
    void (*kernel)(RingArgs) = threads <= 288 ? (wide ? add_norm_ring_kernel<X, R, true, GRAD, 288, 2> : add_norm_ring_kernel<X, R, false, GRAD, 288, 2>)
                                              : (wide ? add_norm_ring_kernel<X, R, true, GRAD, 544, 1> : add_norm_ring_kernel<X, R, false, GRAD, 544, 1>);
    int most = 1;
    FPSK_CUDA_OK(clusters_at_once(reinterpret_cast<const void *>(kernel), launch.cfg, &most));
    if (most > ring_most(g, threads)) most = ring_most(g, threads);
    if (most > g.steps) most = (int)g.steps;
    rows = most * g.teams;
    launch.cfg.gridDim = dim3((unsigned)(most * g.blocks));
    FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg, kernel, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
static RingRows ring_rows(const void *p, long long stride, int type)
{
    const int size = elem_bytes(type);
    return RingRows{static_cast<const char *>(p), stride * size, size, 0};
}

template <typename X, typename R> static fpsk_status launch_norm(const NormArgs &g, bool wide, int xtype, int rtype, int32_t *d_status, cudaStream_t st)
{
    if (wide || g.ytype != FPSK_ELEM_E4M3) {
        RingArgs r = {};
        const bool whole = wide && g.dim % 8 == 0;
        r.f = g;
        r.in[0] = ring_rows(g.x, g.xs, xtype);
        r.in[1] = ring_rows(g.res, g.rs, rtype);
        r.inputs = g.res ? 2 : 1;
        r.n = g.n;
        r.status = d_status;
        int threads, rows;
        if ((whole || g.ytype != FPSK_ELEM_E4M3) && ring_plan(r, g.dim, whole, threads)) return launch_ring<X, R, false>(r, whole, threads, rows, st);
    }
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

template <typename X, typename G> static fpsk_status launch_norm_grad(NormGradArgs g, bool wide, float *dw, int htype, int gtype, int32_t *d_status, cudaStream_t st)
{
    RingArgs r = {};
    const bool whole = wide && g.dim % 8 == 0;
    r.b = g;
    r.in[0] = ring_rows(g.h, g.hs, htype);
    r.in[1] = ring_rows(g.dy, g.dys, gtype);
    r.in[2] = ring_rows(g.dh, g.dhs, gtype);
    r.inputs = g.dh ? 3 : 2;
    r.n = g.n;
    r.status = d_status;
    int ring_threads, rows;
    if (ring_plan(r, g.dim, whole, ring_threads)) {
        const fpsk_status rc = launch_ring<X, G, true>(r, whole, ring_threads, rows, st);
        return rc != FPSK_OK || !dw ? rc : launch_sum(g.part, rows, g.dim, dw, st);
    }
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
#define FPSK_RES(X)                                                      \
    (rt == FPSK_ELEM_FP32 ? launch_norm<X, float>(g, wide, a->x_type, rt, d_status, st)           \
                          : rt == FPSK_ELEM_FP16 ? launch_norm<X, __half>(g, wide, a->x_type, rt, d_status, st) : launch_norm<X, __nv_bfloat16>(g, wide, a->x_type, rt, d_status, st))
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
#define FPSK_IN(G)                                                                              \
    (a->h_type == FPSK_ELEM_FP32 ? launch_norm_grad<float, G>(g, wide, a->dweight, a->h_type, a->grad_type, d_status, st)          \
                                 : a->h_type == FPSK_ELEM_FP16 ? launch_norm_grad<__half, G>(g, wide, a->dweight, a->h_type, a->grad_type, d_status, st)  \
                                                               : launch_norm_grad<__nv_bfloat16, G>(g, wide, a->dweight, a->h_type, a->grad_type, d_status, st))
    if (a->grad_type == FPSK_ELEM_FP32) return FPSK_IN(float);
    if (a->grad_type == FPSK_ELEM_FP16) return FPSK_IN(__half);
    return FPSK_IN(__nv_bfloat16);
#undef FPSK_IN
}
