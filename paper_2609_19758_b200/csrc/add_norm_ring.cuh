// Residual addition and RMS norm of many rows, forward and backward: whole rows through a ring of bulk copies.
//
// For a row: h = x + residual, r = (sum h^2 / d + eps)^-1/2, y = h r w; backwards dx = r (dy w) - h r^3 sum(dy w h) / d + dh and
// dw = sum over the rows of dy h r.
//
// What bounds it is memory, each input once and each output once.  One warp of a block copies rows into a ring of stages, so that what is
// in flight does not depend on the other warps' registers; those take a row each pass: its sums (a vector of eight channels after
// another, pairs in packed arithmetic), one barrier, the results.  A block keeps its shares of the weight's gradient in registers and
// leaves one row of them.  Rows that start off 16 bytes come as their aligned middles, and their first and last elements by plain loads a
// stage ahead.  Above 8192 channels a row is divided among a cluster of blocks, which tell each other their sums.
//
// Measured (a copy moves 6539 GB/s): 4096 tokens of 4096 channels, FP32 + BF16 to BF16, 31 us (5.4 TB/s; 8192 tokens at the rate
// of a copy: 5 us are the start and the end); 8192 x 8192 into e4m3 with groups of 128 99 us in a burst, 109 sustained (6.1, 5.6 TB/s);
// gradients of 4096 x 4096 BF16 33 us, 5 of them the sum of the blocks' rows, of 4096 x 8192 54, of 2048 x 16384 59, of 32768 channels
// 68 us for 1024 tokens.  With the rows held as floats between the two looks 46 us for 4096 x 4096, one element at a time instead of pairs.
#pragma once
#include "add_norm.cuh"

namespace fpsk {

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

// A thread has J vectors of eight of a row's channels; MOST: threads of the largest block.  The weights and their gradients stay in
// registers; what the backward pass's second look at a row wants is read from shared memory again.
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
        if (ok && !mbar_wait_bounded(smem_u32(&full[slot]), phase)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
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
// four such blocks.  (Two blocks of eight warps for 8192 channels would leave each a ring of two stages: 131 instead of 120 us for 8192 x
// 8192 into e4m3.)  Ring and plain form: 4096 channels, 100 tokens 5.0 and 5.1 us, 600 6.0 and 7.9, backward 11.3 and 11.5, 13.3 and 17.4;
// 60000 tokens of 128 channels 29 and 33, backward 49 and 70, 100000 of 64 46 and 51, 72 and 101.
constexpr int kRingOne = 218 * 1024, kRingHalf = 108 * 1024;
static bool ring_plan(RingArgs &g, int dim, bool wide, int &threads)
{
    if (dim <= 32) return false;
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
    return g.steps * g.blocks >= kSms / 2;
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
    count_ring();
    return FPSK_OK;
}
static RingRows ring_rows(const void *p, long long stride, int type)
{
    const int size = elem_bytes(type);
    return RingRows{static_cast<const char *>(p), stride * size, size, 0};
}

}  // namespace fpsk
