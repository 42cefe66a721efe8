// The norm and rotation kernels' form for large calls whose heads lie side by side: the rows of a token come by bulk copies.
//
// For a head x of d values with weights w, r = (sum x^2 / d + eps)^-1/2 and n = x r: y = R(n w), R turning the pairs by the
// token's angles.  Backwards, u = R^T dy: dw += u n, and dx = r (u w - n sum(u w n) / d).
//
// What kept the plain form (norm_rope.cu) from HBM's rate is what a thread has to hold and to compute to have enough loads in
// flight.  Here one warp copies whole tokens - every kind's heads, the rows of the rotation tables - into a ring of stages in
// shared memory, up to 200 KB in flight on every SM whatever the other warps do; the others read them from there.  Where the new
// tokens go in the cache is looked up by the copying warp as well, 32 tokens at a time, so that the chain of dependent loads
// (sequence, length, page) passes once for 32.
//
// Measured: 4096 tokens of 64 heads of 128, FP32 in and 16 bits out, 36.5 us (5.5 TB/s; 31.1 us at the rate of a copy), its
// backward pass 63.1 us (4.3 TB/s: the latency of two sums across lanes a head, one behind the other; 0.60 instructions are issued
// in a cycle of a scheduler, so that their number is not the bound); 11112 tokens with
// 96 heads of 128 into the cache 131 us (6.3 TB/s).
#include "norm_rope.cuh"

#include <atomic>

namespace fpsk {

enum { kOpRope = 0, kOpAppend = 1, kOpGrad = 2 };
// Threads of heads, and one warp that copies.  The backward pass (92 registers) takes 512; the others 512, 640 or 768, the fewest with
// which a stage takes the fewest rounds: 11112 tokens of 96 heads in 140 us with 512 (three rounds) and in 130 with 768 (two), 4096 tokens
// of 64 heads in 44 us with 512 and in 48 with 768 (two rounds both).
constexpr int kRingWorkers = 512, kRingMostWorkers = 768;
constexpr int kRingMost = 8;                     // stages
constexpr int kRingBytes = 200 * 1024, kRingStage = 32 * 1024;

struct RingPiece {
    const char *base;
    long long step;                    // bytes from token to token
    int bytes, at;                     // of a token, place in the token's block of a stage
};
struct RingArgs {
    RopeArgs r;
    RopeGradArgs d;
    RingPiece piece[4];
    int pieces;
    int token_bytes, row_bytes;        // a token's block, and what of it the pieces fill; behind: cos, sin
    int cos_at, table_bytes;           // bytes of a row of a table
    int log_tokens, stages, stage_bytes;
    int workers;
    unsigned int head_magic;           // ceil(2^32 / heads): a vector's token by a multiplication
    int n_all;
    long long n_tok, steps;
    int dim, rot, interleaved;
    const float *cos, *sin;
    const int *positions;
    long long n_pos;
    float eps, inv_dim;
    int32_t *status;
};
struct RingToken {                     // what the copying warp found out about a token
    long long row_k, row_v;            // its rows in the cache
    int flags;                         // 1: in the tables, 2: has a place, 4: that place is in the cache
    int pad;
};

template <typename X, typename Y, int L, int OP>
__global__ void __launch_bounds__((OP == kOpGrad ? kRingWorkers : kRingMostWorkers) + 32, 1) norm_rope_ring_kernel(const __grid_constant__ RingArgs g)
{
    const int workers = OP == kOpGrad ? kRingWorkers : g.workers, S = workers / L;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ unsigned long long full[kRingMost], empty[kRingMost];
    __shared__ RingToken info[kRingMost][32];
    __shared__ int last;
    const int tid = threadIdx.x, warp = tid >> 5, lane32 = tid & 31;
    const int tokens = 1 << g.log_tokens;
    if (tid == 0) {
        for (int s = 0; s < g.stages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), workers / 32);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    bool ok = true;

    if (warp == workers / 32) {
        // ------------------------------------------------------------ copies
        int slot = 0, in_batch = 32;
        uint32_t phase = 0;
        RingToken mine = {};
        int pos = 0;
        long long filled = 0;
        for (long long step = blockIdx.x; step < g.steps; step += gridDim.x) {
            if (in_batch == 32) {
                // the next 32 tokens of this block, a lane each
                in_batch = 0;
                const long long tok = ((step + (long long)(lane32 >> g.log_tokens) * gridDim.x) << g.log_tokens) + (lane32 & (tokens - 1));
                mine = RingToken{};
                pos = -1;
                if (tok < g.n_tok) {
                    if (OP == kOpAppend) {
                        const PlaceArg &at = g.r.at;
                        int lo = 0, hi = at.n_seqs;                    // how many sequences end at or before the token
                        while (lo < hi) {
                            const int mid = (lo + hi) >> 1;
                            if (__ldg(at.cu_q + mid + 1) <= tok) lo = mid + 1;
                            else hi = mid;
                        }
                        const int place = lo < at.n_seqs ? __ldg(at.kv_len + lo) - (__ldg(at.cu_q + lo + 1) - (int)tok) : -1;
                        if (place >= 0) {
                            const unsigned int col = (unsigned int)place / (unsigned int)at.page_size;
                            const int row = place - (int)(col * at.page_size);
                            const int page = col < (unsigned int)at.max_pages ? __ldg(at.table + lo * at.table_stride + col) : -1;
                            mine.flags = page >= 0 && page < at.n_pages ? 6 : 2;
                            mine.row_k = page * at.kps + row * at.kts;
                            mine.row_v = page * at.vps + row * at.vts;
                        }
                        pos = place;
                    }
                    if (g.positions) pos = __ldg(g.positions + tok);
                    if (g.rot == 0 || (pos >= 0 && pos < g.n_pos)) mine.flags |= 1;
                    if ((OP == kOpAppend && (mine.flags & 6) == 2) ||
                        (!(mine.flags & 1) && !(OP == kOpAppend && !(mine.flags & 2) && !g.positions)))
                        report_status(g.status, FPSK_ERR_PARAM);
                }
            }
            const long long t0 = step << g.log_tokens;
            const int n = (int)min((long long)tokens, g.n_tok - t0);
            if (ok && !mbar_wait_bounded(smem_u32(&empty[slot]), phase ^ 1u)) ok = false;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            // the token that lane j < n copies
            const int from = in_batch + (lane32 & (tokens - 1));
            RingToken t;
            t.row_k = __shfl_sync(0xFFFFFFFFu, mine.row_k, from);
            t.row_v = __shfl_sync(0xFFFFFFFFu, mine.row_v, from);
            t.flags = __shfl_sync(0xFFFFFFFFu, mine.flags, from);
            const int p = __shfl_sync(0xFFFFFFFFu, pos, from);
            const bool table = lane32 < n && g.rot > 0 && (t.flags & 1);
            const int tables = __popc(__ballot_sync(0xFFFFFFFFu, table));
            if (lane32 < n) info[slot][lane32] = t;
            __syncwarp();
            const uint32_t bar = smem_u32(&full[slot]), dst = smem_u32(smem) + slot * g.stage_bytes + lane32 * g.token_bytes;
            if (lane32 == 0) mbar_expect_tx(bar, (uint32_t)(n * g.row_bytes + tables * 2 * g.table_bytes));
            __syncwarp();
            if (lane32 < n)
                for (int k = 0; k < g.pieces; ++k)
                    if (g.piece[k].bytes) bulk_g2s(dst + g.piece[k].at, g.piece[k].base + (t0 + lane32) * g.piece[k].step, g.piece[k].bytes, bar);
            if (table) {
                bulk_g2s(dst + g.cos_at, g.cos + (long long)p * (g.rot / 2), g.table_bytes, bar);
                bulk_g2s(dst + g.cos_at + g.table_bytes, g.sin + (long long)p * (g.rot / 2), g.table_bytes, bar);
            }
            in_batch += tokens;
            ++filled;
            if (++slot == g.stages) { slot = 0; phase ^= 1u; }
        }
        // own copies still in flight, should the others' waits have given up
        for (int i = 0; i < g.stages && i < filled; ++i) {
            if (--slot < 0) { slot = g.stages - 1; phase ^= 1u; }
            if (!mbar_wait_bounded(smem_u32(&full[slot]), phase)) ok = false;
        }
    } else {
        // ------------------------------------------------------------ heads
        const int lane = tid % L, first = tid / L;
        const LaneMap m(lane, g.dim, g.rot, g.interleaved);
        float4 wa[2], wb[2], da[2], db[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const void *w = OP == kOpGrad ? g.d.h[k].w : g.r.h[k].w;
            const int type = OP == kOpGrad ? g.d.h[k].wtype : g.r.h[k].wtype;
            wa[k] = wb[k] = splat4(1.f);
            da[k] = db[k] = splat4(0.f);
            if (w && m.on) {
                wa[k] = load4_any<true>(w, type, m.ia);
                wb[k] = load4_any<true>(w, type, m.ib);
                if (OP == kOpGrad && g.interleaved) to_pairs(wa[k], wb[k]);
            }
        }
        const bool norm0 = (OP == kOpGrad ? g.d.h[0].w : g.r.h[0].w) != nullptr, norm1 = (OP == kOpGrad ? g.d.h[1].w : g.r.h[1].w) != nullptr;
        const int n0 = OP == kOpGrad ? g.d.h[0].n : g.r.h[0].n, n1 = OP == kOpGrad ? g.d.h[1].n : g.r.h[1].n;
        // One head: x (and the gradient y) from the stage, the result to `to`.
        auto head = [&](const X *x, const Y *y, const float4 &c, const float4 &s, int flags, int kind, Y *to, bool write) {
            float4 a = splat4(0.f), b = splat4(0.f), ua = splat4(0.f), ub = splat4(0.f);
            if (m.on) {
                a = lds4(x + m.ia);
                b = lds4(x + m.ib);
                if (OP == kOpGrad) {
                    ua = lds4(y + m.ia);
                    ub = lds4(y + m.ib);
                }
            }
            const bool second = kind == 1;
            if (OP == kOpGrad) {
                if (g.interleaved) {
                    to_pairs(a, b);
                    to_pairs(ua, ub);
                }
                if (m.rotated) rotate4(ua, ub, c, s);                  // (s comes negated)
                if (!(flags & 1)) ua = ub = splat4(__int_as_float(0x7FC00000));
                if (second ? norm1 : norm0) {
                    const float r = rsqrtf(fmaf(sum_lanes<L>(dot4(b, b, dot4(a, a, 0.f))), g.inv_dim, g.eps));
                    a = scale4(a, r);
                    b = scale4(b, r);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (k == kind) {
                            da[k] = make_float4(fmaf(ua.x, a.x, da[k].x), fmaf(ua.y, a.y, da[k].y), fmaf(ua.z, a.z, da[k].z), fmaf(ua.w, a.w, da[k].w));
                            db[k] = make_float4(fmaf(ub.x, b.x, db[k].x), fmaf(ub.y, b.y, db[k].y), fmaf(ub.z, b.z, db[k].z), fmaf(ub.w, b.w, db[k].w));
                            ua = mul4(ua, wa[k]);
                            ub = mul4(ub, wb[k]);
                        }
                    if (!m.on) ua = ub = splat4(0.f);
                    const float dot = sum_lanes<L>(dot4(ub, b, dot4(ua, a, 0.f))) * g.inv_dim;
                    ua = norm_grad4(ua, a, dot, r);
                    ub = norm_grad4(ub, b, dot, r);
                }
                if (g.interleaved) from_pairs(ua, ub);
                a = ua;
                b = ub;
            } else {
                if (kind == 0 ? norm0 : second && norm1) {
                    const float r = rsqrtf(fmaf(sum_lanes<L>(dot4(b, b, dot4(a, a, 0.f))), g.inv_dim, g.eps));
                    a = mul4(scale4(a, r), second ? wa[1] : wa[0]);
                    b = mul4(scale4(b, r), second ? wb[1] : wb[0]);
                }
                if (kind != 2) {
                    if (m.rotated) {
                        if (g.interleaved) to_pairs(a, b);
                        rotate4(a, b, c, s);
                        if (g.interleaved) from_pairs(a, b);
                    }
                    if (!(flags & 1)) a = b = splat4(OP == kOpAppend && !(flags & 2) && !g.positions ? 0.f : __int_as_float(0x7FC00000));
                }
            }
            if (write && m.on) {
                store4<true>(to + m.ia, a);
                store4<true>(to + m.ib, b);
            }
        };
        auto factors = [&](const unsigned char *block, int flags, float4 &c, float4 &s) {
            if (!m.on || !m.rotated || !(flags & 1)) return;
            const float *t = reinterpret_cast<const float *>(block + g.cos_at) + m.cs;
            c = lds4(t);
            s = lds4(t + g.rot / 2);
            if (OP == kOpGrad) s = scale4(s, -1.f);
        };
        auto place_of = [&](int v, int &kind) {                        // the kind of a token's v-th head; returns its number
            int h = v;
            kind = 0;
            if (h >= n0) { h -= n0; kind = 1; }
            if (OP == kOpAppend && kind == 1 && h >= n1) { h -= n1; kind = 2; }
            return h;
        };
        auto piece_at = [&](int kind) { return kind == 0 ? g.piece[0].at : kind == 1 ? g.piece[1].at : g.piece[2].at; };
        auto grad_at = [&](int kind) { return kind == 0 ? g.piece[2].at : g.piece[3].at; };
        // where a head goes, but for the token (and, for keys and values of the cache, for the token's row)
        auto out_of = [&](int kind, int h, long long &token_step) {
            if (OP == kOpGrad) {
                token_step = kind ? g.d.h[1].dits : g.d.h[0].dits;
                return static_cast<Y *>(kind ? g.d.h[1].din : g.d.h[0].din) + h * (kind ? g.d.h[1].dihs : g.d.h[0].dihs);
            }
            if (OP == kOpAppend && kind) {
                token_step = 0;
                return kind == 1 ? static_cast<Y *>(g.r.at.k) + h * g.r.at.khs : static_cast<Y *>(g.r.at.v) + h * g.r.at.vhs;
            }
            token_step = kind ? g.r.h[1].ots : g.r.h[0].ots;
            return static_cast<Y *>(kind ? g.r.h[1].out : g.r.h[0].out) + h * (kind ? g.r.h[1].ohs : g.r.h[0].ohs);
        };
        int slot = 0;
        uint32_t phase = 0;
        auto done = [&]() {
            __syncwarp();
            if (lane32 == 0) mbar_arrive(smem_u32(&empty[slot]));
            if (++slot == g.stages) { slot = 0; phase ^= 1u; }
        };
        if (tokens == 1 && g.n_all <= 2 * S) {
            // A token to a stage, at most two heads to a thread: always the same ones, so what addresses them is worked out once
            // (4096 tokens of 64 heads in 36.5 us; in the loop below, which holds for any number, 44.2).
            int kind[2], x_at[2], y_at[2];
            Y *to[2];
            long long next[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int h = place_of(first + i * S, kind[i]);
                if (first + i * S >= g.n_all) kind[i] = -1;
                x_at[i] = piece_at(kind[i]) + h * g.dim * (int)sizeof(X);
                y_at[i] = OP == kOpGrad ? grad_at(kind[i]) + h * g.dim * (int)sizeof(Y) : 0;
                to[i] = kind[i] < 0 ? nullptr : out_of(kind[i], h, next[i]);
                if (kind[i] >= 0) to[i] += blockIdx.x * next[i];
                else next[i] = 0;
                next[i] *= gridDim.x;
            }
            for (long long step = blockIdx.x; step < g.steps; step += gridDim.x) {
                if (ok) ok = mbar_wait_warp(smem_u32(&full[slot]), phase);
                const unsigned char *stage = smem + slot * g.stage_bytes;
                const RingToken &t = info[slot][0];
                const int flags = t.flags;
                float4 c = splat4(1.f), s = splat4(0.f);
                if (ok) factors(stage, flags, c, s);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (ok && kind[i] >= 0) {
                        Y *p = to[i];
                        if (OP == kOpAppend && kind[i]) p += kind[i] == 1 ? t.row_k : t.row_v;
                        head(reinterpret_cast<const X *>(stage + x_at[i]), reinterpret_cast<const Y *>(stage + y_at[i]), c, s, flags, kind[i], p,
                             OP != kOpAppend || kind[i] == 0 || (flags & 4));
                    }
                    to[i] += next[i];
                }
                done();
            }
        } else {
            for (long long step = blockIdx.x; step < g.steps; step += gridDim.x) {
                if (ok) ok = mbar_wait_warp(smem_u32(&full[slot]), phase);
                const long long t0 = step << g.log_tokens;
                const int vectors = ok ? (int)min((long long)tokens, g.n_tok - t0) * g.n_all : 0;
                const unsigned char *stage = smem + slot * g.stage_bytes;
                for (int v = first; v < vectors; v += S) {
                    const int j = tokens == 1 ? 0 : (int)__umulhi((unsigned int)v, g.head_magic);
                    int kind;
                    const int h = place_of(v - j * g.n_all, kind);
                    const unsigned char *block = stage + j * g.token_bytes;
                    const int flags = info[slot][j].flags;
                    float4 c = splat4(1.f), s = splat4(0.f);
                    factors(block, flags, c, s);
                    long long token_step;
                    Y *p = out_of(kind, h, token_step);
                    if (OP == kOpAppend && kind) p += kind == 1 ? info[slot][j].row_k : info[slot][j].row_v;
                    else p += (t0 + j) * token_step;
                    head(reinterpret_cast<const X *>(block + piece_at(kind)) + h * g.dim, reinterpret_cast<const Y *>(block + grad_at(kind)) + h * g.dim, c, s,
                         flags, kind, p, OP != kOpAppend || kind == 0 || (flags & 4));
                }
                done();
            }
        }
        if (OP == kOpGrad) {
            // the block's sums of both kinds; the stages are free when all workers are here
            asm volatile("bar.sync 1, 512;" ::: "memory");
            float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (g.interleaved) from_pairs(da[k], db[k]);
                if (m.on) {
                    store4<true>(sums + (k * S + first) * g.dim + m.ia, da[k]);
                    store4<true>(sums + (k * S + first) * g.dim + m.ib, db[k]);
                }
            }
            asm volatile("bar.sync 1, 512;" ::: "memory");
            for (int c = tid; c < 2 * g.dim; c += kRingWorkers) {
                const int k = c >= g.dim;
                const float *p = sums + k * S * g.dim + c - k * g.dim;
                float t = 0.f;
                for (int i = 0; i < S; ++i) t += p[i * g.dim];
                g.d.part[(size_t)blockIdx.x * 2 * g.dim + c] = t;
            }
        }
    }
    if (!ok && lane32 == 0) report_status(g.status, FPSK_ERR_TIMEOUT);
    if (OP != kOpGrad || (!g.d.h[0].dw && !g.d.h[1].dw)) return;
    __syncthreads();
    if (tid == 0) last = atom_acq_rel_add(g.d.count) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    float *sums = reinterpret_cast<float *>(smem);
    for (int k = 0; k < 2; ++k)
        if (g.d.h[k].dw) sum_rows<kRingWorkers + 32>(g.d.part + k * g.dim, 2 * g.dim, (int)gridDim.x, g.dim, sums, g.d.h[k].dw);
    if (tid == 0) *g.d.count = 0u;
}

// ---------------------------------------------------------------- host side
// A kind's heads of a token as one copy: side by side, everything in steps of 16 bytes.
static bool add_piece(RingArgs &g, const void *base, long long token_stride, long long head_stride, int heads, int size)
{
    RingPiece &p = g.piece[g.pieces++];
    p.base = static_cast<const char *>(base);
    p.step = token_stride * size;
    p.bytes = heads * g.dim * size;
    p.at = g.row_bytes;
    g.row_bytes += p.bytes;
    return (heads == 1 || head_stride == g.dim) && p.bytes % 16 == 0 && p.step % 16 == 0 && reinterpret_cast<uintptr_t>(base) % 16 == 0;
}
// Tokens of a stage and stages: as many tokens (a power of two) as 32 KB hold, as many stages as 200 KB hold.  Not taken: tokens of
// which less than two stages fit, and calls of less than six steps for every SM: there the plain form, whose start is shorter, is as
// fast or faster (backward, 64 heads of 128: 1024 tokens 20.8 against 22.3 us; 4096 tokens 65 against 86 us).
static bool plan_ring(RingArgs &g)
{
    g.table_bytes = g.rot * 2;
    g.cos_at = g.row_bytes;
    g.token_bytes = (int)align_up((size_t)g.row_bytes + 2 * g.table_bytes, 128);
    if (g.rot && (g.table_bytes % 16 || reinterpret_cast<uintptr_t>(g.cos) % 16 || reinterpret_cast<uintptr_t>(g.sin) % 16)) return false;
    for (g.log_tokens = 0; g.log_tokens < 5 && (g.token_bytes << (g.log_tokens + 1)) <= kRingStage;) ++g.log_tokens;
    g.stage_bytes = g.token_bytes << g.log_tokens;
    g.stages = kRingBytes / g.stage_bytes;
    if (g.stages > kRingMost) g.stages = kRingMost;
    g.steps = (g.n_tok + (1 << g.log_tokens) - 1) >> g.log_tokens;
    g.head_magic = (unsigned int)((0x100000000ULL + g.n_all - 1) / g.n_all);
    return g.stages >= 2 && g.n_all >= 2 && g.n_all <= 2048 && g.steps >= 6 * kRingBlocks;
}
template <typename X, typename Y, int L, int OP> static fpsk_status launch_ring(RingArgs &g, cudaStream_t st)
{
    static std::atomic<unsigned long long> prepared{0};               // one bit per device
    int dev = 0;
    FPSK_CUDA_OK(cudaGetDevice(&dev));
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(prepared.load(std::memory_order_acquire) & bit)) {
        FPSK_CUDA_OK(cudaFuncSetAttribute(norm_rope_ring_kernel<X, Y, L, OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes));
        prepared.fetch_or(bit, std::memory_order_release);
    }
    const int vectors = g.n_all << g.log_tokens;
    g.workers = kRingWorkers;
    for (int w = kRingWorkers; OP != kOpGrad && w <= kRingMostWorkers; w += 128)
        if ((vectors + w / L - 1) / (w / L) < (vectors + g.workers / L - 1) / (g.workers / L)) g.workers = w;
    norm_rope_ring_kernel<X, Y, L, OP><<<kRingBlocks, g.workers + 32, kRingBytes, st>>>(g);
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
template <typename X, typename Y, int OP> static fpsk_status launch_ring_dim(RingArgs &g, cudaStream_t st)
{
    return g.dim <= 64 ? launch_ring<X, Y, 8, OP>(g, st) : g.dim <= 128 ? launch_ring<X, Y, 16, OP>(g, st) : launch_ring<X, Y, 32, OP>(g, st);
}
template <int OP> static fpsk_status launch_ring_typed(RingArgs &g, int in, int out, cudaStream_t st)
{
#define FPSK_IN(Y)                                                                                                            \
    (in == FPSK_ELEM_FP32 ? launch_ring_dim<float, Y, OP>(g, st)                                                              \
                          : in == FPSK_ELEM_FP16 ? launch_ring_dim<__half, Y, OP>(g, st) : launch_ring_dim<__nv_bfloat16, Y, OP>(g, st))
    if (out == FPSK_ELEM_FP16) return FPSK_IN(__half);
    if (out == FPSK_ELEM_BF16) return FPSK_IN(__nv_bfloat16);
    if constexpr (OP != kOpAppend) return FPSK_IN(float);
    return FPSK_ERR_DTYPE;
#undef FPSK_IN
}
template <typename A> static void ring_common(RingArgs &g, const A &a, int heads)
{
    g.n_all = heads;
    g.n_tok = a.n_tok;
    g.dim = a.dim; g.rot = a.rot; g.interleaved = a.interleaved;
    g.cos = a.cos; g.sin = a.sin; g.positions = a.positions;
    g.n_pos = a.n_pos; g.eps = a.eps; g.inv_dim = a.inv_dim;
    g.status = a.status;
}

bool rope_ring(const RopeArgs &a, int in_type, int out_type, bool append, cudaStream_t st, fpsk_status *rc)
{
    if (append && !a.at.wide_k) return false;
    if (append && !a.at.wide_v) return false;
    RingArgs g = {};
    g.r = a;
    ring_common(g, a, a.n_all);
    for (int k = 0; k < (append ? 3 : 2); ++k) {
        const HeadsArg &h = a.h[k];
        if (h.n == 0) { ++g.pieces; continue; }                        // no bytes: no copy
        if (!add_piece(g, h.in, h.its, h.ihs, h.n, elem_size(in_type)) || (h.w && !h.wide_w)) return false;
        if (!(append && k > 0) && !h.wide_out) return false;
    }
    if (!plan_ring(g)) return false;
    *rc = append ? launch_ring_typed<kOpAppend>(g, in_type, out_type, st) : launch_ring_typed<kOpRope>(g, in_type, out_type, st);
    return true;
}

bool rope_grad_ring(const RopeGradArgs &a, int in_type, int grad_type, cudaStream_t st, fpsk_status *rc)
{
    RingArgs g = {};
    g.d = a;
    ring_common(g, a, a.h[0].n + a.h[1].n);
    if (g.n_all == 0) return false;
    for (int k = 0; k < 2; ++k) {
        const HeadsGradArg &h = a.h[k];
        if (h.n == 0) return false;
        if (!add_piece(g, h.in, h.its, h.ihs, h.n, elem_size(in_type)) || (h.w && !h.wide_w) || !h.wide_din) return false;
    }
    for (int k = 0; k < 2; ++k)
        if (!add_piece(g, a.h[k].dout, a.h[k].dots, a.h[k].dohs, a.h[k].n, elem_size(grad_type))) return false;
    if (!plan_ring(g)) return false;
    *rc = launch_ring_typed<kOpGrad>(g, in_type, grad_type, st);
    return true;
}

}  // namespace fpsk
