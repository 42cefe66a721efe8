// Norms of queries and keys with the position rotation in the same pass, their backward pass, and the writes of keys
// and values to a paged cache.
//
//   z = x r w,  r = rsqrt(mean(x^2) + eps);     (a, b) -> (a c - b s, b c + a s) over the channel pairs of a head
//   backward: u = R^T dy, n = x r, g = u w:     dx = r (g - n mean(g n)),   dw = sum over tokens and heads of u n
//
// All of it is bound by HBM: every input and output element moves once.  A head's channels sit in L = 8, 16 or 32 lanes
// so that the mean is a few shuffles, and a lane holds four channel PAIRS (two groups of four channels: i and
// i + rot/2, or eight neighbours when pairs are interleaved), so that the rotation needs no exchange.  The channels
// behind rot_dim are paired the same way, (i, i + (D - rot)/2), and not rotated, which keeps one mapping for all.
//
// This is the form for small calls and for any strides; large calls whose heads lie side by side go to norm_rope_ring.cu.  What
// bounds it is a launch's latency, and behind that the instructions it issues (some 350 for two heads and lanes, backward).
// Measured: one token of 32 + 8 heads of 128 3.4 us, a step of 64 requests into the cache 5.2 us, 1021 tokens of 28 + 4 heads
// of 96 backward 16.0 us, of which 1.6 pass before the first loads and 3.2 in the last block's sum over the blocks' rows.
#include "norm_rope.cuh"

namespace fpsk {

template <int L> static BlockMap block_map(int heads)
{
    constexpr int S = kRopeThreads / L;
    BlockMap m = {1, 1, 1};
    if (heads < S) {
        m.tokens = S / heads;
        m.step = kPer * m.tokens;
    } else {
        m.chunks = (heads + S * kPer - 1) / (S * kPer);
    }
    return m;
}
// The head and the offset in tokens of a slot's i-th vector; head >= heads: none.
struct SlotMap {
    int head0, token0, head_step, token_step;
    __device__ __forceinline__ SlotMap(const BlockMap &m, int heads, int slots, int slot, int chunk)
    {
        if (m.step == 1) {
            head0 = chunk * slots * kPer + slot;
            token0 = 0;
            head_step = slots;
            token_step = 0;
        } else {
            token0 = slot / heads;
            head0 = token0 < m.tokens ? slot - token0 * heads : heads;
            head_step = 0;
            token_step = m.tokens;
        }
    }
};

// WIDE: four elements at a time (all pointers and strides allow it), and 32-bit offsets into the tables.
template <typename X, typename Y, int L, bool APPEND, bool WIDE>
__global__ void __launch_bounds__(kRopeThreads, 3) norm_rope_kernel(const __grid_constant__ RopeArgs g)
{
    constexpr int S = kRopeThreads / L;
    const int lane = threadIdx.x % L;
    const LaneMap m(lane, g.dim, g.rot, g.interleaved);
    const SlotMap sm(g.map, g.n_all, S, threadIdx.x / L, blockIdx.y);
    // the slot's heads: what they are, where they lie (what the token adds comes with the token), their weights
    int kind[kPer];
    const X *src[kPer];
    Y *dst[kPer];
    float4 wa[kPer], wb[kPer];
    bool normed[kPer];
    const long long first = (long long)blockIdx.x * g.map.step, stride = (long long)gridDim.x * g.map.step;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        int h = sm.head0 + i * sm.head_step;
        kind[i] = 0;
        if (h >= g.h[0].n) { h -= g.h[0].n; kind[i] = 1; }
        if (kind[i] == 1 && h >= g.h[1].n) { h -= g.h[1].n; kind[i] = 2; }
        if (kind[i] == 2 && h >= g.h[2].n) kind[i] = -1;
        const HeadsArg &H = g.h[max(kind[i], 0)];
        const long long tok = first + sm.token0 + i * sm.token_step;
        src[i] = static_cast<const X *>(H.in) + tok * H.its + h * H.ihs;
        dst[i] = APPEND && kind[i] > 0 ? static_cast<Y *>(kind[i] == 1 ? g.at.k : g.at.v) + h * (kind[i] == 1 ? g.at.khs : g.at.vhs)
                                       : static_cast<Y *>(H.out) + tok * H.ots + h * H.ohs;
        normed[i] = H.w != nullptr && kind[i] != 2;
        wa[i] = wb[i] = splat4(1.f);
        if (normed[i] && m.on) {
            wa[i] = load4_any<WIDE>(H.w, H.wtype, m.ia);
            wb[i] = load4_any<WIDE>(H.w, H.wtype, m.ib);
        }
        if (!m.on) kind[i] = -1;                                       // lanes behind the last channel only take part in the sums
    }
    long long in_step[kPer], out_step[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        in_step[i] = stride * (kind[i] <= 0 ? g.h[0].its : kind[i] == 1 ? g.h[1].its : g.h[2].its);
        out_step[i] = APPEND && kind[i] > 0 ? 0 : stride * (kind[i] == 1 ? g.h[1].ots : g.h[0].ots);
    }
    float4 na[kPer], nb[kPer];                                         // the step ahead
    auto fetch = [&](long long tok) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            na[i] = nb[i] = splat4(0.f);
            if (kind[i] >= 0 && tok + sm.token0 + i * sm.token_step < g.n_tok) {
                na[i] = load4<WIDE>(src[i] + m.ia);
                nb[i] = load4<WIDE>(src[i] + m.ib);
            }
            src[i] += in_step[i];
        }
    };
    if (first < g.n_tok) fetch(first);
    int seq0 = 0;
    for (long long t0 = first; t0 < g.n_tok; t0 += stride) {
        float4 a[kPer], b[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) { a[i] = na[i]; b[i] = nb[i]; }
        if (t0 + stride < g.n_tok) fetch(t0 + stride);
        if (APPEND) {
            // how many sequences end at or before the step's first token (the tokens ascend)
            for (;;) {
                const int i = seq0 + (threadIdx.x & 31);
                const unsigned int before = __ballot_sync(0xFFFFFFFFu, i < g.at.n_seqs && __ldg(g.at.cu_q + i + 1) <= t0);
                seq0 += __popc(before);
                if (before != 0xFFFFFFFFu) break;
            }
        }
        long long place = -1, row_k = 0, row_v = 0;
        bool in_table = true, stored = true;
        float4 c = splat4(1.f), s = splat4(0.f);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const long long tok = t0 + sm.token0 + i * sm.token_step;
            const bool live = kind[i] >= 0 && tok < g.n_tok;
            if ((i == 0 || sm.token_step) && tok < g.n_tok) {          // what belongs to the token
                int pos = 0;
                if (APPEND) {
                    int seq = seq0;
                    if (sm.token_step || sm.token0)
                        while (seq < g.at.n_seqs && __ldg(g.at.cu_q + seq + 1) <= tok) ++seq;
                    place = -1;
                    stored = false;
                    if (seq < g.at.n_seqs) place = __ldg(g.at.kv_len + seq) - (__ldg(g.at.cu_q + seq + 1) - (int)tok);
                    pos = (int)place;
                    if (place >= 0) {
                        const unsigned int col = (unsigned int)place / (unsigned int)g.at.page_size;
                        const int row = (int)place - (int)(col * g.at.page_size);
                        const int page = col < (unsigned int)g.at.max_pages ? __ldg(g.at.table + seq * g.at.table_stride + col) : -1;
                        stored = page >= 0 && page < g.at.n_pages;
                        if (!stored && lane == 0) report_status(g.status, FPSK_ERR_PARAM);
                        row_k = page * g.at.kps + row * g.at.kts;
                        row_v = page * g.at.vps + row * g.at.vts;
                    }
                }
                if (g.positions) pos = __ldg(g.positions + tok);
                if (g.rot > 0) {
                    in_table = pos >= 0 && pos < g.n_pos;
                    if (in_table && m.on && m.rotated) {
                        if (WIDE) {
                            const int at = pos * (g.rot / 2) + m.cs;
                            c = load4<true>(g.cos + at);
                            s = load4<true>(g.sin + at);
                        } else {
                            const long long at = (long long)pos * (g.rot / 2) + m.cs;
                            c = load4<false>(g.cos + at);
                            s = load4<false>(g.sin + at);
                        }
                    }
                }
            }
            if (normed[i]) {
                const float ss = sum_lanes<L>(dot4(b[i], b[i], dot4(a[i], a[i], 0.f)));
                const float r = rsqrtf(fmaf(ss, g.inv_dim, g.eps));
                a[i] = mul4(scale4(a[i], r), wa[i]);
                b[i] = mul4(scale4(b[i], r), wb[i]);
            }
            if (m.rotated && kind[i] != 2) {
                if (g.interleaved) to_pairs(a[i], b[i]);
                rotate4(a[i], b[i], c, s);
                if (g.interleaved) from_pairs(a[i], b[i]);
            }
            if (!in_table && live && kind[i] != 2) {
                const bool no_place = APPEND && place < 0 && !g.positions;
                a[i] = b[i] = splat4(no_place ? 0.f : __int_as_float(0x7FC00000));
                if (!no_place && lane == 0) report_status(g.status, FPSK_ERR_PARAM);
            }
            Y *p = dst[i];
            if (APPEND && kind[i] > 0) p += kind[i] == 1 ? row_k : row_v;
            dst[i] += out_step[i];
            if (live && (!APPEND || kind[i] == 0 || stored)) {
                store4<WIDE>(p + m.ia, a[i]);
                store4<WIDE>(p + m.ib, b[i]);
            }
        }
    }
}

// ---------------------------------------------------------------- backward
// Persistent blocks, each on the heads of one kind, so that a lane keeps one set of eight weight-gradient sums.  They
// meet in shared memory, then in a partial row per block; the last block to arrive adds the rows in block order.
template <typename X, typename Y, int L, bool WIDE>
__global__ void __launch_bounds__(kRopeThreads, 2) norm_rope_grad_kernel(const __grid_constant__ RopeGradArgs g)
{
    constexpr int S = kRopeThreads / L;
    __shared__ __align__(16) float sums[kRopeThreads * 8];
    __shared__ int last;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    const LaneMap m(lane, g.dim, g.rot, g.interleaved);
    const int kind = (int)blockIdx.x >= g.blocks0;
    const HeadsGradArg &H = g.h[kind];
    const long long n_tok = H.n ? g.n_tok : 0;                         // a kind without heads only has its weight gradient of zero to write
    const int block = blockIdx.x - (kind ? g.blocks0 : 0), blocks = kind ? gridDim.x - g.blocks0 : g.blocks0;
    const int chunk = block % H.map.chunks, lanes_of_blocks = blocks / H.map.chunks;   // (blocks: a multiple of the chunks)
    const SlotMap sm(H.map, H.n, S, slot, chunk);
    const long long first = (long long)(block / H.map.chunks) * H.map.step, stride = (long long)lanes_of_blocks * H.map.step;
    float4 wa = splat4(1.f), wb = splat4(1.f), da = splat4(0.f), db = splat4(0.f);
    if (H.w && m.on) {
        wa = load4_any<WIDE>(H.w, H.wtype, m.ia);
        wb = load4_any<WIDE>(H.w, H.wtype, m.ib);
        if (g.interleaved) to_pairs(wa, wb);
    }
    const X *src[kPer];
    const Y *grad[kPer];
    Y *dst[kPer];
    bool there[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int h = sm.head0 + i * sm.head_step;
        const long long tok = first + sm.token0 + i * sm.token_step;
        there[i] = h < H.n && m.on;
        src[i] = static_cast<const X *>(H.in) + tok * H.its + h * H.ihs;
        grad[i] = static_cast<const Y *>(H.dout) + tok * H.dots + h * H.dohs;
        dst[i] = static_cast<Y *>(H.din) + tok * H.dits + h * H.dihs;
    }
    float4 na[kPer], nb[kPer], ga[kPer], gb[kPer];                     // the step ahead
    auto fetch = [&](long long tok) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            na[i] = nb[i] = ga[i] = gb[i] = splat4(0.f);
            if (there[i] && tok + sm.token0 + i * sm.token_step < n_tok) {
                na[i] = load4<WIDE>(src[i] + m.ia);
                nb[i] = load4<WIDE>(src[i] + m.ib);
                ga[i] = load4<WIDE>(grad[i] + m.ia);
                gb[i] = load4<WIDE>(grad[i] + m.ib);
            }
            src[i] += stride * H.its;
            grad[i] += stride * H.dots;
        }
    };
    if (first < n_tok) fetch(first);
    for (long long t0 = first; t0 < n_tok; t0 += stride) {
        float4 a[kPer], b[kPer], ua[kPer], ub[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) { a[i] = na[i]; b[i] = nb[i]; ua[i] = ga[i]; ub[i] = gb[i]; }
        if (t0 + stride < n_tok) fetch(t0 + stride);
        float4 c = splat4(1.f), s = splat4(0.f);
        bool in_table = true;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const long long tok = t0 + sm.token0 + i * sm.token_step;
            const bool live = there[i] && tok < n_tok;
            if (g.rot > 0 && (i == 0 || sm.token_step) && tok < n_tok) {
                const int pos = __ldg(g.positions + tok);
                in_table = pos >= 0 && pos < g.n_pos;
                if (in_table && m.on && m.rotated) {
                    const long long at = WIDE ? (long long)(pos * (g.rot / 2) + m.cs) : (long long)pos * (g.rot / 2) + m.cs;
                    c = load4<WIDE>(g.cos + at);
                    s = scale4(load4<WIDE>(g.sin + at), -1.f);
                }
            }
            if (g.interleaved) {
                to_pairs(a[i], b[i]);
                to_pairs(ua[i], ub[i]);
            }
            if (m.rotated) rotate4(ua[i], ub[i], c, s);
            if (!in_table && live) {
                ua[i] = ub[i] = splat4(__int_as_float(0x7FC00000));
                if (lane == 0) report_status(g.status, FPSK_ERR_PARAM);
            }
            if (H.w) {
                const float ss = sum_lanes<L>(dot4(b[i], b[i], dot4(a[i], a[i], 0.f)));
                // n; zero where there is no vector, so that it adds nothing (there the root is infinite when eps is 0)
                const float r = live ? rsqrtf(fmaf(ss, g.inv_dim, g.eps)) : 0.f;
                a[i] = scale4(a[i], r);
                b[i] = scale4(b[i], r);
                da = make_float4(fmaf(ua[i].x, a[i].x, da.x), fmaf(ua[i].y, a[i].y, da.y), fmaf(ua[i].z, a[i].z, da.z), fmaf(ua[i].w, a[i].w, da.w));
                db = make_float4(fmaf(ub[i].x, b[i].x, db.x), fmaf(ub[i].y, b[i].y, db.y), fmaf(ub[i].z, b[i].z, db.z), fmaf(ub[i].w, b[i].w, db.w));
                ua[i] = mul4(ua[i], wa);                            // g = u w
                ub[i] = mul4(ub[i], wb);
                const float dot = sum_lanes<L>(dot4(ub[i], b[i], dot4(ua[i], a[i], 0.f))) * g.inv_dim;
                ua[i] = norm_grad4(ua[i], a[i], dot, r);
                ub[i] = norm_grad4(ub[i], b[i], dot, r);
            }
            if (g.interleaved) from_pairs(ua[i], ub[i]);
            if (live) {
                store4<WIDE>(dst[i] + m.ia, ua[i]);
                store4<WIDE>(dst[i] + m.ib, ub[i]);
            }
            dst[i] += stride * H.dits;
        }
    }
    if (!g.h[0].dw && !g.h[1].dw) return;
    // the block's sums, in channel order
    const int dim = g.dim;
    if (g.interleaved) from_pairs(da, db);
    if (m.on) {
        store4<true>(sums + slot * dim + m.ia, da);
        store4<true>(sums + slot * dim + m.ib, db);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < dim; c += kRopeThreads) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < S; ++i) t += sums[i * dim + c];
        g.part[(size_t)blockIdx.x * dim + c] = t;
    }
    __syncthreads();
    if (threadIdx.x == 0) last = atom_acq_rel_add(g.count) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    for (int k = 0; k < 2; ++k)
        if (g.h[k].dw)
            sum_rows<kRopeThreads>(g.part + (size_t)(k ? g.blocks0 : 0) * dim, dim, k ? (int)gridDim.x - g.blocks0 : g.blocks0, dim, sums, g.h[k].dw);
    if (threadIdx.x == 0) *g.count = 0u;
}

// ---------------------------------------------------------------- host side
static bool wide(const void *p, int size, long long s0, long long s1)
{
    return reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && s0 % 4 == 0 && s1 % 4 == 0;
}

static fpsk_status check_rotary(const fpsk_rotary *r, int dim, bool positions)
{
    if (!r) return FPSK_OK;
    if (r->rot_dim < 0 || r->rot_dim > dim || r->rot_dim % 8 || (r->interleaved != 0 && r->interleaved != 1)) return FPSK_ERR_PARAM;
    if (r->rot_dim == 0) return FPSK_OK;
    if (!r->cos || !r->sin || (positions && !r->positions)) return FPSK_ERR_NULL;
    if (r->n_pos < 1) return FPSK_ERR_SHAPE;
    return FPSK_OK;
}
static fpsk_status check_heads(const fpsk_heads *h, int64_t n_tokens, bool out)
{
    if (h->n_heads < 0 || h->n_heads > 65536) return FPSK_ERR_SHAPE;
    if (h->n_heads == 0) return FPSK_OK;
    if (n_tokens > 0 && (!h->in || (out && !h->out))) return FPSK_ERR_NULL;
    if (h->weight && !elem_ok(h->weight_type)) return FPSK_ERR_DTYPE;
    return FPSK_OK;
}
static HeadsArg heads_arg(const fpsk_heads *h, int in_size, int out_size)
{
    HeadsArg a = {};
    if (!h || h->n_heads == 0) return a;
    a.in = h->in; a.out = h->out; a.w = h->weight;
    a.its = h->in_token_stride; a.ihs = h->in_head_stride; a.ots = h->out_token_stride; a.ohs = h->out_head_stride;
    a.n = h->n_heads; a.wtype = h->weight_type;
    a.wide_in = wide(h->in, in_size, a.its, a.ihs);
    a.wide_out = wide(h->out, out_size, a.ots, a.ohs);
    a.wide_w = wide(h->weight, elem_size(h->weight_type), 0, 0);
    return a;
}
template <typename G> static void rotary_arg(G &g, const fpsk_rotary *r)
{
    g.rot = r ? r->rot_dim : 0;
    g.interleaved = g.rot ? r->interleaved : 0;
    g.cos = g.rot ? r->cos : nullptr;
    g.sin = g.rot ? r->sin : nullptr;
    g.positions = g.rot ? r->positions : nullptr;
    g.n_pos = g.rot ? r->n_pos : 0;
    g.wide_tab = g.rot && wide(r->cos, 4, r->rot_dim / 2, 0) && wide(r->sin, 4, r->rot_dim / 2, 0);
}

// Three blocks a multiprocessor walk the tokens.
template <typename X, typename Y, int L, bool APPEND> static fpsk_status launch_rope_lanes(RopeArgs g, cudaStream_t st)
{
    g.map = block_map<L>(g.n_all);
    const long long steps = (g.n_tok + g.map.step - 1) / g.map.step, most = (148 * 3 + g.map.chunks - 1) / g.map.chunks;
    const dim3 grid((unsigned)(steps < most ? steps : most), (unsigned)g.map.chunks);
    bool all = g.rot == 0 || (g.wide_tab && g.n_pos * (g.rot / 2) <= 0x7FFFFFFFLL);
    for (int k = 0; k < 3; ++k)
        if (g.h[k].n) all = all && g.h[k].wide_in && (APPEND && k > 0 ? (k == 1 ? g.at.wide_k : g.at.wide_v) : g.h[k].wide_out) && (!g.h[k].w || g.h[k].wide_w);
    if (all) norm_rope_kernel<X, Y, L, APPEND, true><<<grid, kRopeThreads, 0, st>>>(g);
    else norm_rope_kernel<X, Y, L, APPEND, false><<<grid, kRopeThreads, 0, st>>>(g);
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
template <typename X, typename Y, bool APPEND> static fpsk_status launch_rope(const RopeArgs &g, cudaStream_t st)
{
    return g.dim <= 64 ? launch_rope_lanes<X, Y, 8, APPEND>(g, st) : g.dim <= 128 ? launch_rope_lanes<X, Y, 16, APPEND>(g, st)
                                                                                  : launch_rope_lanes<X, Y, 32, APPEND>(g, st);
}
template <bool APPEND> static fpsk_status launch_rope_typed(const RopeArgs &g, int in, int out, cudaStream_t st)
{
    if (g.n_tok == 0 || g.n_all == 0) return FPSK_OK;
    fpsk_status rc;
    if (rope_ring(g, in, out, APPEND, st, &rc)) return rc;
#define FPSK_IN(Y)                                                                        \
    (in == FPSK_ELEM_FP32 ? launch_rope<float, Y, APPEND>(g, st)                          \
                          : in == FPSK_ELEM_FP16 ? launch_rope<__half, Y, APPEND>(g, st)  \
                                                 : launch_rope<__nv_bfloat16, Y, APPEND>(g, st))
    if (out == FPSK_ELEM_FP16) return FPSK_IN(__half);
    if (out == FPSK_ELEM_BF16) return FPSK_IN(__nv_bfloat16);
    if constexpr (!APPEND) return FPSK_IN(float);
    return FPSK_ERR_DTYPE;
#undef FPSK_IN
}

constexpr int kGradBlocks = 148 * 2;
constexpr int kMostGradBlocks = kGradBlocks + 2 * (65536 / 16 + 1);   // (a kind has at least a block for each chunk of its heads)

template <typename X, typename Y, int L> static void launch_grad_lanes(const RopeGradArgs &g, unsigned blocks, cudaStream_t st)
{
    bool all = g.rot == 0 || (g.wide_tab && g.n_pos * (g.rot / 2) <= 0x7FFFFFFFLL);
    for (int k = 0; k < 2; ++k)
        if (g.h[k].n) all = all && g.h[k].wide_in && g.h[k].wide_dout && g.h[k].wide_din && (!g.h[k].w || g.h[k].wide_w);
    if (all) norm_rope_grad_kernel<X, Y, L, true><<<blocks, kRopeThreads, 0, st>>>(g);
    else norm_rope_grad_kernel<X, Y, L, false><<<blocks, kRopeThreads, 0, st>>>(g);
}
template <typename X, typename Y> static fpsk_status launch_grad(const RopeGradArgs &g, unsigned blocks, cudaStream_t st)
{
    if (g.dim <= 64) launch_grad_lanes<X, Y, 8>(g, blocks, st);
    else if (g.dim <= 128) launch_grad_lanes<X, Y, 16>(g, blocks, st);
    else launch_grad_lanes<X, Y, 32>(g, blocks, st);
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

}  // namespace fpsk

using namespace fpsk;

extern "C" fpsk_status fpsk_qk_norm_rope(const fpsk_heads *q, const fpsk_heads *k, int64_t n_tokens, int32_t head_dim,
                                         fpsk_elem in_type, fpsk_elem out_type, const fpsk_rotary *rot, float eps,
                                         int32_t *d_status, void *stream)
{
    if (n_tokens < 0 || !head_dim_ok(head_dim)) return FPSK_ERR_SHAPE;
    if (!elem_ok(in_type) || !elem_ok(out_type)) return FPSK_ERR_DTYPE;
    if (!(eps >= 0.f)) return FPSK_ERR_PARAM;
    for (const fpsk_heads *h : {q, k})
        if (h) {
            const fpsk_status rc = check_heads(h, n_tokens, true);
            if (rc != FPSK_OK) return rc;
        }
    const fpsk_status rc = check_rotary(rot, head_dim, n_tokens > 0);
    if (rc != FPSK_OK) return rc;
    RopeArgs g = {};
    g.h[0] = heads_arg(q, elem_size(in_type), elem_size(out_type));
    g.h[1] = heads_arg(k, elem_size(in_type), elem_size(out_type));
    g.n_all = g.h[0].n + g.h[1].n;
    if (n_tokens > (1LL << 40)) return FPSK_ERR_SHAPE;
    g.n_tok = n_tokens;
    g.dim = head_dim;
    g.eps = eps;
    g.inv_dim = 1.f / (float)head_dim;
    g.status = d_status;
    rotary_arg(g, rot);
    return launch_rope_typed<false>(g, in_type, out_type, static_cast<cudaStream_t>(stream));
}

extern "C" fpsk_status fpsk_paged_append(const fpsk_paged_cache *cache, const fpsk_paged_batch *batch, const fpsk_heads *k,
                                         const fpsk_heads *v, const fpsk_heads *q, fpsk_elem in_type,
                                         const fpsk_rotary *rot, float eps, int32_t *d_status, void *stream)
{
    fpsk_status rc = check_cache(cache);
    if (rc != FPSK_OK) return rc;
    rc = check_batch(batch);
    if (rc != FPSK_OK) return rc;
    if (!k || !v) return FPSK_ERR_NULL;
    if (!elem_ok(in_type)) return FPSK_ERR_DTYPE;
    if (!(eps >= 0.f)) return FPSK_ERR_PARAM;
    if (k->n_heads != cache->n_heads || v->n_heads != cache->n_heads) return FPSK_ERR_SHAPE;
    if ((rc = check_heads(k, batch->n_tokens, false)) != FPSK_OK || (rc = check_heads(v, batch->n_tokens, false)) != FPSK_OK) return rc;
    if (q && (rc = check_heads(q, batch->n_tokens, true)) != FPSK_OK) return rc;
    if ((rc = check_rotary(rot, cache->head_dim, false)) != FPSK_OK) return rc;
    const int size = elem_size(cache->type), in_size = elem_size(in_type);
    RopeArgs g = {};
    g.h[0] = heads_arg(q, in_size, size);
    g.h[1] = heads_arg(k, in_size, size);
    g.h[2] = heads_arg(v, in_size, size);
    g.n_all = g.h[0].n + g.h[1].n + g.h[2].n;
    g.n_tok = batch->n_tokens;
    g.dim = cache->head_dim;
    g.eps = eps;
    g.inv_dim = 1.f / (float)cache->head_dim;
    g.status = d_status;
    rotary_arg(g, rot);
    PlaceArg &p = g.at;
    p.cu_q = batch->cu_q; p.kv_len = batch->kv_len; p.table = batch->block_table;
    p.table_stride = batch->table_stride; p.n_pages = cache->n_pages;
    p.n_seqs = batch->n_seqs; p.max_pages = batch->max_pages; p.page_size = cache->page_size;
    p.kps = cache->k_page_stride; p.kts = cache->k_token_stride; p.khs = cache->k_head_stride;
    p.vps = cache->v_page_stride; p.vts = cache->v_token_stride; p.vhs = cache->v_head_stride;
    p.k = cache->k; p.v = cache->v;
    p.wide_k = wide(p.k, size, p.kps, p.kts) && p.khs % 4 == 0;
    p.wide_v = wide(p.v, size, p.vps, p.vts) && p.vhs % 4 == 0;
    return launch_rope_typed<true>(g, in_type, cache->type, static_cast<cudaStream_t>(stream));
}

extern "C" size_t fpsk_norm_rope_workspace_bytes(int32_t head_dim)
{
    if (!head_dim_ok(head_dim)) return 0;
    return kAttnSyncBytes + (size_t)kMostGradBlocks * head_dim * sizeof(float);
}

extern "C" fpsk_status fpsk_qk_norm_rope_backward(const fpsk_heads_grad *q, const fpsk_heads_grad *k, int64_t n_tokens,
                                                  int32_t head_dim, fpsk_elem in_type, fpsk_elem grad_type,
                                                  const fpsk_rotary *rot, float eps, void *workspace, size_t ws_bytes,
                                                  int32_t *d_status, void *stream)
{
    if (n_tokens < 0 || n_tokens > (1LL << 40) || !head_dim_ok(head_dim)) return FPSK_ERR_SHAPE;
    if (!elem_ok(in_type) || !elem_ok(grad_type)) return FPSK_ERR_DTYPE;
    if (!(eps >= 0.f)) return FPSK_ERR_PARAM;
    fpsk_status rc = check_rotary(rot, head_dim, n_tokens > 0);
    if (rc != FPSK_OK) return rc;
    RopeGradArgs g = {};
    const int in_size = elem_size(in_type), gsize = elem_size(grad_type);
    const fpsk_heads_grad *hs[2] = {q, k};
    for (int i = 0; i < 2; ++i) {
        const fpsk_heads_grad *h = hs[i];
        if (!h) continue;
        if (h->n_heads < 0 || h->n_heads > 65536) return FPSK_ERR_SHAPE;
        if (h->weight && !elem_ok(h->weight_type)) return FPSK_ERR_DTYPE;
        if (h->n_heads && n_tokens > 0 && (!h->in || !h->dout || !h->din)) return FPSK_ERR_NULL;
        if (h->weight && !h->dweight) return FPSK_ERR_NULL;
        HeadsGradArg &a = g.h[i];
        a.in = h->in; a.dout = h->dout; a.din = h->din; a.w = h->weight; a.dw = h->weight ? h->dweight : nullptr;
        a.its = h->in_token_stride; a.ihs = h->in_head_stride; a.dots = h->dout_token_stride; a.dohs = h->dout_head_stride;
        a.dits = h->din_token_stride; a.dihs = h->din_head_stride;
        a.n = h->n_heads; a.wtype = h->weight_type;
        a.wide_in = wide(a.in, in_size, a.its, a.ihs);
        a.wide_dout = wide(a.dout, gsize, a.dots, a.dohs);
        a.wide_din = wide(a.din, gsize, a.dits, a.dihs);
        a.wide_w = wide(a.w, elem_size(a.wtype), 0, 0);
    }
    if (!workspace) return FPSK_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return FPSK_ERR_ALIGN;
    if (ws_bytes < fpsk_norm_rope_workspace_bytes(head_dim)) return FPSK_ERR_WORKSPACE;
    g.n_tok = n_tokens;
    g.dim = head_dim;
    g.eps = eps;
    g.inv_dim = 1.f / (float)head_dim;
    g.status = d_status;
    rotary_arg(g, rot);
    g.count = static_cast<unsigned int *>(workspace);
    g.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + kAttnSyncBytes);
    // Blocks of each kind in proportion to its heads, a multiple of its chunks of heads, at least one where it has a weight
    // gradient to write.
    long long want[2];
    for (int i = 0; i < 2; ++i) {
        HeadsGradArg &a = g.h[i];
        a.map = head_dim <= 64 ? block_map<8>(a.n ? a.n : 1) : head_dim <= 128 ? block_map<16>(a.n ? a.n : 1) : block_map<32>(a.n ? a.n : 1);
        const long long steps = a.n ? (n_tokens + a.map.step - 1) / a.map.step : 0;
        const long long most = (long long)kGradBlocks * a.n / (g.h[0].n + g.h[1].n > 0 ? g.h[0].n + g.h[1].n : 1) / a.map.chunks;
        want[i] = (steps < most ? steps : most < 1 ? (steps < 1 ? steps : 1) : most) * a.map.chunks;
        if (want[i] == 0 && a.dw) want[i] = a.map.chunks;
    }
    g.blocks0 = (int)want[0];
    const unsigned blocks = (unsigned)(want[0] + want[1]);
    if (blocks == 0) return FPSK_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rope_grad_ring(g, in_type, grad_type, st, &rc)) return rc;
#define FPSK_IN(Y)                                                               \
    (in_type == FPSK_ELEM_FP32 ? launch_grad<float, Y>(g, blocks, st)            \
                               : in_type == FPSK_ELEM_FP16 ? launch_grad<__half, Y>(g, blocks, st) : launch_grad<__nv_bfloat16, Y>(g, blocks, st))
    if (grad_type == FPSK_ELEM_FP32) return FPSK_IN(float);
    if (grad_type == FPSK_ELEM_FP16) return FPSK_IN(__half);
    return FPSK_IN(__nv_bfloat16);
#undef FPSK_IN
}
