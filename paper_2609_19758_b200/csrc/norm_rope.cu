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
#include "attention.cuh"
#include "stream_pipe.cuh"

#include <mutex>

namespace fpsk {

struct HeadsArg {
    const void *in;
    void *out;
    const void *w;
    long long its, ihs, ots, ohs;      // strides of tokens and heads, input and output
    int n, wtype;
    int wide_in, wide_out, wide_w;
};

struct PlaceArg {                      // where the new tokens' keys and values go
    const int *cu_q, *kv_len, *table;
    long long table_stride, n_pages;
    int n_seqs, max_pages, page_size;
    long long kps, kts, khs, vps, vts, vhs;
    void *k, *v;
    int wide_k, wide_v;
};

struct RopeArgs {
    HeadsArg h[3];                     // queries, keys, values (values: append only, copied)
    int n_all;                         // heads of all kinds
    long long n_vec;                   // tokens x heads
    int dim, rot, interleaved;
    const float *cos, *sin;
    const int *positions;
    long long n_pos;
    float eps, inv_dim;
    int wide_tab;
    PlaceArg at;
    int32_t *status;
};

// What a lane of a head's L lanes holds: two groups of four channels.
struct LaneMap {
    int ia, ib, cs;
    bool on, rotated;
    __device__ __forceinline__ LaneMap(int lane, int dim, int rot, int interleaved)
    {
        const int p = 4 * lane;        // first of its four pairs
        on = p < dim / 2;
        rotated = p < rot / 2;
        cs = p;
        if (interleaved) {
            ia = 8 * lane;
            ib = ia + 4;
        } else if (rotated) {
            ia = p;
            ib = p + rot / 2;
        } else {
            ia = rot + (p - rot / 2);
            ib = ia + (dim - rot) / 2;
        }
    }
};
// eight neighbours (x0 x1 x2 x3)(x4 x5 x6 x7) <-> the four pairs' first and second members
__device__ __forceinline__ void to_pairs(float4 &a, float4 &b)
{
    const float4 x = a, y = b;
    a = make_float4(x.x, x.z, y.x, y.z);
    b = make_float4(x.y, x.w, y.y, y.w);
}
__device__ __forceinline__ void from_pairs(float4 &a, float4 &b)
{
    const float4 x = a, y = b;
    a = make_float4(x.x, y.x, x.y, y.y);
    b = make_float4(x.z, y.z, x.w, y.w);
}
__device__ __forceinline__ void rotate4(float4 &a, float4 &b, const float4 &c, const float4 &s)
{
    const float4 x = a, y = b;
    a = make_float4(x.x * c.x - y.x * s.x, x.y * c.y - y.y * s.y, x.z * c.z - y.z * s.z, x.w * c.w - y.w * s.w);
    b = make_float4(y.x * c.x + x.x * s.x, y.y * c.y + x.y * s.y, y.z * c.z + x.z * s.z, y.w * c.w + x.w * s.w);
}
__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 scale4(float4 a, float r) { return make_float4(a.x * r, a.y * r, a.z * r, a.w * r); }
__device__ __forceinline__ float dot4(float4 a, float4 b, float acc)
{
    return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, acc))));
}
__device__ __forceinline__ float4 splat4(float x) { return make_float4(x, x, x, x); }
template <int L> __device__ __forceinline__ float sum_lanes(float x)
{
#pragma unroll
    for (int o = L / 2; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

constexpr int kRopeThreads = 256;

// Block = 256 / L head slots, HPT consecutive rounds of them.  All loads of a thread's HPT heads are issued before the
// first is used.
template <typename X, typename Y, int L, int HPT, bool APPEND>
__global__ void __launch_bounds__(kRopeThreads) norm_rope_kernel(const __grid_constant__ RopeArgs g)
{
    constexpr int S = kRopeThreads / L;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    const LaneMap m(lane, g.dim, g.rot, g.interleaved);
    const long long v0 = (long long)blockIdx.x * (S * HPT);
    // (a 64-bit division takes longer than a head)
    const long long t0 = v0 < 0x7FFFFFFFLL ? (long long)((unsigned int)v0 / (unsigned int)g.n_all) : v0 / g.n_all;
    const int rem0 = (int)(v0 - t0 * g.n_all);

    int kind[HPT], head[HPT];
    long long tok[HPT];
    float4 a[HPT], b[HPT];
#pragma unroll
    for (int i = 0; i < HPT; ++i) {
        const int r = rem0 + slot + i * S;
        const int dt = r / g.n_all;
        int h = r - dt * g.n_all;
        tok[i] = t0 + dt;
        kind[i] = 0;
        if (h >= g.h[0].n) { h -= g.h[0].n; kind[i] = 1; }
        if (APPEND && kind[i] == 1 && h >= g.h[1].n) { h -= g.h[1].n; kind[i] = 2; }
        head[i] = h;
        a[i] = b[i] = splat4(0.f);
        if (v0 + slot + i * S >= g.n_vec) { kind[i] = -1; continue; }
        if (m.on) {
            const HeadsArg &H = g.h[kind[i]];
            const X *p = static_cast<const X *>(H.in) + tok[i] * H.its + h * H.ihs;
            a[i] = load4(p + m.ia, H.wide_in);
            b[i] = load4(p + m.ib, H.wide_in);
        }
    }

    // the weights of queries and of keys, once per thread
    float4 wa[2], wb[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        wa[k] = wb[k] = splat4(1.f);
        if (g.h[k].w && m.on) {
            wa[k] = load4_any(g.h[k].w, g.h[k].wtype, m.ia, g.h[k].wide_w);
            wb[k] = load4_any(g.h[k].w, g.h[k].wtype, m.ib, g.h[k].wide_w);
        }
    }

    // sequence of the block's first token: how many sequences end at or before it
    int seq0 = 0;
    if (APPEND) {
        const long long t_first = t0;
        for (int base = 0; base < g.at.n_seqs; base += kRopeThreads) {
            const int i = base + threadIdx.x;
            const int before = __syncthreads_count(i < g.at.n_seqs && g.at.cu_q[i + 1] <= t_first);
            seq0 += before;
            if (before < kRopeThreads) break;
        }
    }

#pragma unroll
    for (int i = 0; i < HPT; ++i) {
        long long pos = 0, place = 0;
        int seq = seq0;
        bool has_place = true;
        if (APPEND && kind[i] >= 0) {
            while (seq < g.at.n_seqs && g.at.cu_q[seq + 1] <= tok[i]) ++seq;
            has_place = seq < g.at.n_seqs;
            if (has_place) place = (long long)g.at.kv_len[seq] - (g.at.cu_q[seq + 1] - tok[i]);
            has_place = has_place && place >= 0;
            pos = place;
        }
        if (g.positions && kind[i] >= 0) pos = g.positions[tok[i]];
        const bool turn = kind[i] >= 0 && kind[i] != 2 && g.rot > 0;
        const bool in_table = pos >= 0 && pos < g.n_pos;
        float4 c = splat4(1.f), s = splat4(0.f);
        if (turn && in_table && m.on && m.rotated) {
            c = load4(g.cos + pos * (g.rot / 2) + m.cs, g.wide_tab);
            s = load4(g.sin + pos * (g.rot / 2) + m.cs, g.wide_tab);
        }
        const bool key = kind[i] == 1;
        const bool normed = kind[i] >= 0 && kind[i] != 2 && (key ? g.h[1].w : g.h[0].w) != nullptr;
        float ss = dot4(b[i], b[i], dot4(a[i], a[i], 0.f));
        ss = sum_lanes<L>(ss);
        if (kind[i] < 0) continue;
        if (normed) {
            const float r = rsqrtf(fmaf(ss, g.inv_dim, g.eps));
            a[i] = mul4(scale4(a[i], r), key ? wa[1] : wa[0]);
            b[i] = mul4(scale4(b[i], r), key ? wb[1] : wb[0]);
        }
        if (turn) {
            if (g.interleaved) to_pairs(a[i], b[i]);
            rotate4(a[i], b[i], c, s);
            if (g.interleaved) from_pairs(a[i], b[i]);
            if (!in_table) {
                if (APPEND && !has_place && !g.positions) a[i] = b[i] = splat4(0.f);
                else {
                    a[i] = b[i] = splat4(__int_as_float(0x7FC00000));
                    if (lane == 0) report_status(g.status, FPSK_ERR_PARAM);
                }
            }
        }
        if (!m.on) continue;
        if (!APPEND || kind[i] == 0) {
            const HeadsArg &H = g.h[kind[i]];
            Y *p = static_cast<Y *>(H.out) + tok[i] * H.ots + head[i] * H.ohs;
            store4(p + m.ia, a[i], H.wide_out);
            store4(p + m.ib, b[i], H.wide_out);
        } else if (has_place) {
            const long long col = place / g.at.page_size;
            const int row = (int)(place - col * g.at.page_size);
            const long long page = col < g.at.max_pages ? g.at.table[seq * g.at.table_stride + col] : -1;
            if (page < 0 || page >= g.at.n_pages) {
                if (lane == 0) report_status(g.status, FPSK_ERR_PARAM);
                continue;
            }
            const bool is_k = kind[i] == 1;
            Y *p = is_k ? static_cast<Y *>(g.at.k) + page * g.at.kps + row * g.at.kts + head[i] * g.at.khs
                        : static_cast<Y *>(g.at.v) + page * g.at.vps + row * g.at.vts + head[i] * g.at.vhs;
            store4(p + m.ia, a[i], is_k ? g.at.wide_k : g.at.wide_v);
            store4(p + m.ib, b[i], is_k ? g.at.wide_k : g.at.wide_v);
        }
    }
}

// ---------------------------------------------------------------- backward
struct HeadsGradArg {
    const void *in, *dout;
    void *din;
    const void *w;
    float *dw;
    long long its, ihs, dots, dohs, dits, dihs;
    int n, wtype;
    int wide_in, wide_dout, wide_din, wide_w;
};
struct RopeGradArgs {
    HeadsGradArg h[2];
    int blocks0;                       // the first blocks work on queries, the others on keys
    long long n_tok;
    int dim, rot, interleaved;
    const float *cos, *sin;
    const int *positions;
    long long n_pos;
    float eps, inv_dim;
    int wide_tab;
    float *part;                       // [blocks][dim]: every block's share of the weight gradient
    unsigned int *count;               // arrivals (returns to 0)
    int32_t *status;
};

// Persistent blocks, each on the heads of one kind, so that a lane keeps one set of eight weight-gradient sums.  They
// meet in shared memory, then in a partial row per block; the last block to arrive adds the rows in block order.
template <typename X, typename Y, int L>
__global__ void __launch_bounds__(kRopeThreads) norm_rope_grad_kernel(const __grid_constant__ RopeGradArgs g)
{
    constexpr int S = kRopeThreads / L, HPT = 2;
    __shared__ __align__(16) float sums[kRopeThreads * 8];
    __shared__ int last;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    const LaneMap m(lane, g.dim, g.rot, g.interleaved);
    const int kind = (int)blockIdx.x >= g.blocks0;
    const int block = blockIdx.x - (kind ? g.blocks0 : 0), blocks = kind ? gridDim.x - g.blocks0 : g.blocks0;
    const HeadsGradArg &H = g.h[kind];
    const long long n_vec = g.n_tok * H.n;
    float4 wa = splat4(1.f), wb = splat4(1.f), da = splat4(0.f), db = splat4(0.f);
    if (H.w && m.on) {
        wa = load4_any(H.w, H.wtype, m.ia, H.wide_w);
        wb = load4_any(H.w, H.wtype, m.ib, H.wide_w);
        if (g.interleaved) to_pairs(wa, wb);
    }
    for (long long v0 = (long long)block * (S * HPT); v0 < n_vec; v0 += (long long)blocks * (S * HPT)) {
        const long long t0 = v0 < 0x7FFFFFFFLL ? (long long)((unsigned int)v0 / (unsigned int)H.n) : v0 / H.n;
        const int rem0 = (int)(v0 - t0 * H.n);
        float4 a[HPT], b[HPT], ua[HPT], ub[HPT];
        long long tok[HPT];
        int head[HPT];
        bool live[HPT];
#pragma unroll
        for (int i = 0; i < HPT; ++i) {
            const int r = rem0 + slot + i * S, dt = r / H.n;
            head[i] = r - dt * H.n;
            tok[i] = t0 + dt;
            live[i] = v0 + slot + i * S < n_vec;
            a[i] = b[i] = ua[i] = ub[i] = splat4(0.f);
            if (live[i] && m.on) {
                const X *p = static_cast<const X *>(H.in) + tok[i] * H.its + head[i] * H.ihs;
                const Y *q = static_cast<const Y *>(H.dout) + tok[i] * H.dots + head[i] * H.dohs;
                a[i] = load4(p + m.ia, H.wide_in);
                b[i] = load4(p + m.ib, H.wide_in);
                ua[i] = load4(q + m.ia, H.wide_dout);
                ub[i] = load4(q + m.ib, H.wide_dout);
            }
        }
#pragma unroll
        for (int i = 0; i < HPT; ++i) {
            if (g.interleaved) {
                to_pairs(a[i], b[i]);
                to_pairs(ua[i], ub[i]);
            }
            if (g.rot > 0 && live[i]) {
                const long long pos = g.positions[tok[i]];
                const bool in_table = pos >= 0 && pos < g.n_pos;
                if (in_table && m.on && m.rotated) {
                    const float4 c = load4(g.cos + pos * (g.rot / 2) + m.cs, g.wide_tab);
                    const float4 s = load4(g.sin + pos * (g.rot / 2) + m.cs, g.wide_tab);
                    rotate4(ua[i], ub[i], c, scale4(s, -1.f));
                }
                if (!in_table) {
                    ua[i] = ub[i] = splat4(__int_as_float(0x7FC00000));
                    if (lane == 0) report_status(g.status, FPSK_ERR_PARAM);
                }
            }
            if (H.w) {
                const float ss = sum_lanes<L>(dot4(b[i], b[i], dot4(a[i], a[i], 0.f)));
                const float r = rsqrtf(fmaf(ss, g.inv_dim, g.eps));
                a[i] = scale4(a[i], r);                             // n
                b[i] = scale4(b[i], r);
                if (live[i] && m.on) {
                    da = make_float4(fmaf(ua[i].x, a[i].x, da.x), fmaf(ua[i].y, a[i].y, da.y), fmaf(ua[i].z, a[i].z, da.z), fmaf(ua[i].w, a[i].w, da.w));
                    db = make_float4(fmaf(ub[i].x, b[i].x, db.x), fmaf(ub[i].y, b[i].y, db.y), fmaf(ub[i].z, b[i].z, db.z), fmaf(ub[i].w, b[i].w, db.w));
                }
                ua[i] = mul4(ua[i], wa);                            // g = u w
                ub[i] = mul4(ub[i], wb);
                float dot = m.on ? dot4(ub[i], b[i], dot4(ua[i], a[i], 0.f)) : 0.f;
                dot = sum_lanes<L>(dot) * g.inv_dim;
                ua[i] = make_float4(r * (ua[i].x - a[i].x * dot), r * (ua[i].y - a[i].y * dot), r * (ua[i].z - a[i].z * dot), r * (ua[i].w - a[i].w * dot));
                ub[i] = make_float4(r * (ub[i].x - b[i].x * dot), r * (ub[i].y - b[i].y * dot), r * (ub[i].z - b[i].z * dot), r * (ub[i].w - b[i].w * dot));
            }
            if (g.interleaved) from_pairs(ua[i], ub[i]);
            if (live[i] && m.on) {
                Y *p = static_cast<Y *>(H.din) + tok[i] * H.dits + head[i] * H.dihs;
                store4(p + m.ia, ua[i], H.wide_din);
                store4(p + m.ib, ub[i], H.wide_din);
            }
        }
    }
    if (!g.h[0].dw && !g.h[1].dw) return;
    // the block's sums, in channel order
    const int dim = g.dim;
    if (g.interleaved) from_pairs(da, db);
    if (m.on) {
        store4(sums + slot * dim + m.ia, da, true);
        store4(sums + slot * dim + m.ib, db, true);
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
    // The rows of one kind, split over the threads of a channel group, eight loads in flight; then the threads' sums in order.
    for (int k = 0; k < 2; ++k) {
        if (!g.h[k].dw) continue;
        const int b0 = k ? g.blocks0 : 0, b1 = k ? gridDim.x : g.blocks0;
        const int groups = dim / 4, parts = kRopeThreads / groups;
        const int c = threadIdx.x % groups, p = threadIdx.x / groups;
        float4 t = splat4(0.f);
        if (p < parts) {
            for (int b = b0 + p; b < b1; b += 8 * parts) {
                float4 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = b + j * parts < b1 ? __ldcg(reinterpret_cast<const float4 *>(g.part + (size_t)(b + j * parts) * dim) + c) : splat4(0.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) t = make_float4(t.x + x[j].x, t.y + x[j].y, t.z + x[j].z, t.w + x[j].w);
            }
        }
        __syncthreads();
        if (p < parts) store4(sums + p * dim + 4 * c, t, true);
        __syncthreads();
        for (int ch = threadIdx.x; ch < dim; ch += kRopeThreads) {
            float s = 0.f;
            for (int i = 0; i < parts; ++i) s += sums[i * dim + ch];
            g.h[k].dw[ch] = s;
        }
    }
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

// Heads per thread: one while the call has fewer head slots than the card holds at once (latency), else four, whose loads
// are in flight together.
template <typename X, typename Y, bool APPEND> static fpsk_status launch_rope(const RopeArgs &g, cudaStream_t st)
{
    const int L = g.dim <= 64 ? 8 : g.dim <= 128 ? 16 : 32, S = kRopeThreads / L;
    const int hpt = g.n_vec > 148LL * 8 * S ? 4 : 1;
    const long long blocks = (g.n_vec + S * hpt - 1) / (S * hpt);
    if (blocks > 0x7FFFFFFFLL) return FPSK_ERR_SHAPE;
#define FPSK_ROPE(LL, HH) norm_rope_kernel<X, Y, LL, HH, APPEND><<<(unsigned)blocks, kRopeThreads, 0, st>>>(g)
    if (hpt == 1) {
        if (L == 8) FPSK_ROPE(8, 1);
        else if (L == 16) FPSK_ROPE(16, 1);
        else FPSK_ROPE(32, 1);
    } else {
        if (L == 8) FPSK_ROPE(8, 4);
        else if (L == 16) FPSK_ROPE(16, 4);
        else FPSK_ROPE(32, 4);
    }
#undef FPSK_ROPE
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
template <bool APPEND> static fpsk_status launch_rope_typed(const RopeArgs &g, int in, int out, cudaStream_t st)
{
    if (g.n_vec == 0) return FPSK_OK;
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

constexpr int kGradBlocks = 148 * 3;

template <typename X, typename Y> static fpsk_status launch_grad(const RopeGradArgs &g, unsigned blocks, cudaStream_t st)
{
    if (g.dim <= 64) norm_rope_grad_kernel<X, Y, 8><<<blocks, kRopeThreads, 0, st>>>(g);
    else if (g.dim <= 128) norm_rope_grad_kernel<X, Y, 16><<<blocks, kRopeThreads, 0, st>>>(g);
    else norm_rope_grad_kernel<X, Y, 32><<<blocks, kRopeThreads, 0, st>>>(g);
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
    g.n_vec = n_tokens * g.n_all;
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
    g.n_vec = batch->n_tokens * g.n_all;
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
    return kAttnSyncBytes + (size_t)kGradBlocks * head_dim * sizeof(float);
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
    // blocks of each kind in proportion to its heads, at least one where it has a weight gradient to write
    const int L = head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32, per = kRopeThreads / L * 2;
    long long want[2];
    for (int i = 0; i < 2; ++i) {
        want[i] = (n_tokens * g.h[i].n + per - 1) / per;
        if (want[i] == 0 && g.h[i].dw) want[i] = 1;
    }
    if (want[0] + want[1] > kGradBlocks) {
        const long long n0 = (long long)((double)kGradBlocks * (double)want[0] / (double)(want[0] + want[1]) + 0.5);
        want[0] = want[0] ? (n0 < 1 ? 1 : n0 > kGradBlocks - (want[1] ? 1 : 0) ? kGradBlocks - (want[1] ? 1 : 0) : n0) : 0;
        want[1] = want[1] ? kGradBlocks - want[0] : 0;
    }
    g.blocks0 = (int)want[0];
    const unsigned blocks = (unsigned)(want[0] + want[1]);
    if (blocks == 0) return FPSK_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define FPSK_IN(Y)                                                               \
    (in_type == FPSK_ELEM_FP32 ? launch_grad<float, Y>(g, blocks, st)            \
                               : in_type == FPSK_ELEM_FP16 ? launch_grad<__half, Y>(g, blocks, st) : launch_grad<__nv_bfloat16, Y>(g, blocks, st))
    if (grad_type == FPSK_ELEM_FP32) return FPSK_IN(float);
    if (grad_type == FPSK_ELEM_FP16) return FPSK_IN(__half);
    return FPSK_IN(__nv_bfloat16);
#undef FPSK_IN
}
