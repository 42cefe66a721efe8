// The loss of rows of logits against a teacher's top logits, and its gradient.
//
// q = softmax(x / tau), p over the listed tokens; loss = sum_j p_j (log p_j - log q_j); d/dx_v = (m q_v - p_v) / tau, m = sum p.
// In powers of two, with c = log2(e) / tau and a reference M near the row's largest logit: S = sum 2^((x - M) c), q_v = 2^((x_v - M) c) / S,
// log q_v = (x_v - M) / tau - ln S.  M and S stay apart to the end, and from the loss to a gradient that comes later, so that nothing is
// rounded at the size of the logarithm.
//
// What bounds it is memory: the logits once, the gradient once.  The gradient needs S first, so a row is looked at twice; the second look
// finds it in L2 as long as the rows at work at a time are not too many bytes, which a cluster of blocks to a row sees to.  One warp of a
// block copies pieces of 8 KB of its slice into a ring, once or twice over; four warps sum the slice up, exchange (M, S) through the
// cluster's shared memory, and write the gradient; one or three warps prepare the teacher's probabilities for the next row and take them off the
// gradient of the one before, so that neither is waited for.
//
// Measured: 4096 rows of 131072 FP32 logits with BF16 gradients 543 us in a burst (5.9 TB/s of logits and gradients, 0.91 of a copy),
// 636 sustained, at the power limit; losses of 2048 rows of 65536 BF16 52 us (0.79; the special function unit, which makes the powers, is busy
// for 66 %); loss, then gradient of 1500 x 50257 FP16 94 us; 5 rows of 131072 11 us.  (Without the
// largest listed logit as reference 521, 49 and 9 us.)  Rows held in shared memory between the two looks
// (eight slices of 64 KB, three blocks to an SM): 662 us, as fewer rows are at work at a time.  The gradient's factor folded into the
// exponent, a product fewer for two elements: no faster.
#include "decoder.cuh"

namespace fpsk {

enum { kLossOnly = 0, kLossAndGrad = 1, kGradOnly = 2 };

struct DistillArgs {
    const void *x, *tok, *t;
    const float *weight;
    float *loss, *lse, *sums;          // sums: M and S of each row, written by the loss, read by the gradient alone where they are given
    void *dx;
    long long xs, toks, ts, dxs, rows;
    int vocab, top;
    int tok_bytes, t_type;
    int normalize;
    float tau, inv_tau, c;             // c = log2(e) / tau
    int blocks;                        // of a row
    int teachers;                      // warps
    int teacher_at, map_at, map_words; // in shared memory: behind the ring the teacher's arrays, and the map of listed tokens
    int32_t *status;
};

constexpr int kWorkers = 128, kMostTeachers = 3;   // threads of the sums and gradients, warps of the teacher
constexpr int kDistillThreads = kWorkers + 32 + 32 * kMostTeachers;
constexpr int kPiece = 8192, kPieceVecs = kPiece / 16, kStages = 5;
constexpr int kTogether = 4;            // listed tokens of a lane at a time
constexpr float kMostPowers = 256.f;    // (a piece has 32 of a thread's at most: equal logits do not reach it)

template <typename X> __device__ __forceinline__ float vec_max(const uint4 &u)
{
    float2 e[Vec<X>::n / 2];
    Vec<X>::open(u, e);
    float top = fmaxf(e[0].x, e[0].y);
#pragma unroll
    for (int j = 1; j < Vec<X>::n / 2; ++j) top = fmaxf(top, fmaxf(e[j].x, e[j].y));
    return top;
}
// sum += 2^((x - M) c) of a vector's elements
template <typename X> __device__ __forceinline__ void add_powers(const uint4 &u, float2 minus, float2 cc, float2 &sum)
{
    float2 e[Vec<X>::n / 2];
    Vec<X>::open(u, e);
#pragma unroll
    for (int j = 0; j < Vec<X>::n / 2; ++j) {
        const float2 y = __fmul2_rn(__fadd2_rn(e[j], minus), cc);
        sum = __fadd2_rn(sum, make_float2(exp2_fast(y.x), exp2_fast(y.y)));
    }
}
// 2^((x - M) c) summed, joined over a warp's first LANES lanes like join_lanes, in 64 bits: what is rounded at the size of the whole sum is
// rounded once, so that the order of the additions, which goes by a row's alignment, rarely shows.
struct LongSum {
    float m;
    double s;
};
template <int LANES> __device__ __forceinline__ LongSum join_long(LongSum r, float c)
{
    float top = r.m;
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    double s = r.s * (double)exp2_fast((r.m - top) * c);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return LongSum{top, s};
}
// f 2^((x - M) c)
template <typename X> __device__ __forceinline__ void gradients(const uint4 &u, float2 minus, float2 cc, float2 ff, float2 (&e)[Vec<X>::n / 2])
{
    Vec<X>::open(u, e);
#pragma unroll
    for (int j = 0; j < Vec<X>::n / 2; ++j) {
        const float2 y = __fmul2_rn(__fadd2_rn(e[j], minus), cc);
        e[j] = __fmul2_rn(make_float2(exp2_fast(y.x), exp2_fast(y.y)), ff);
    }
}

template <typename X, typename G, int MODE> __global__ void __launch_bounds__(kDistillThreads, 4) distill_kernel(const __grid_constant__ DistillArgs g)
{
    constexpr int VEC = Vec<X>::n;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned long long full[kStages], empty[kStages], ready[2], met[2];
    __shared__ float4 blocks_sum[2][kRowMostBlocks];                   // written by the cluster's blocks: M, S, the teacher's two
    __shared__ LongSum warps_sum[2][kWorkers / 32];
    __shared__ float4 result[2], taught[2];                            // M, S, the teacher's two; K, xr, the teacher's two
    __shared__ float teams[6][kMostTeachers], highest[2];              // highest: of the block's listed logits
    __shared__ int teams_twice[kMostTeachers], counts[2][kMostTeachers];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)cluster_rank();
    const long long first_row = blockIdx.x / g.blocks, row_step = gridDim.x / g.blocks;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), kWorkers / 32);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&ready[b]), 1);
            mbar_init(smem_u32(&met[b]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < g.map_words; i += blockDim.x) reinterpret_cast<unsigned int *>(smem + g.map_at)[i] = 0;
    __syncthreads();
    cluster_sync();
    behind_the_last();
    // Every wait is bounded; once one has given up the others are passed over, and all roles still run to their ends.
    bool ok = true;
    // (asked for a row ahead: the answer takes a microsecond)
    auto weight_of = [&](long long row) { return g.weight && row < g.rows ? g.weight[row] : 1.f; };
    float weight_next = weight_of(first_row);
    auto wait = [&](unsigned long long &bar, uint32_t parity) {
        if (ok && !mbar_wait_bounded(smem_u32(&bar), parity)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
    };

    // A warp takes its powers with a reference that is no more than 2^8 below the largest of them, and not below the block's largest listed
    // logit: an exponent is rounded at its own size, so that the largest powers, which are most of the sum and of the gradient, want
    // exponents near 0.  (Errors of 1.2e-6 relative in an FP32 gradient and 4e-6 in a small loss of few rows without the listed logit, for
    // normal logits with larger ones listed; of 5e-6 in the gradient with a reference that moved at 2^100 only, for a logit that is not
    // listed 30 to 50 above the others.  It costs 1 % for 4096 x 131072 normal logits, 543 us, and 3, 7 and -13 % where they spread 2.5, 5 and 20
    // times as far; a reference for each thread, which moves in most rows, 6 to 23 %.)
    constexpr bool anchored = MODE != kGradOnly;
    // the teacher's mass, from what it says: normalized its largest logit and 1 / s, else the mass itself
    auto mass_of = [&](float a0, float a1) { return g.normalize ? (a1 == 0.f ? 0.f : 1.f) : a0; };

    if (warp == kWorkers / 32) {
        // ------------------------------------------------------------ copies
        if (lane == 0) {
            unsigned int k = 0;                                        // pieces so far
            int stage = 0;
            uint32_t phase = 0;
            for (long long row = first_row; row < g.rows && ok; row += row_step) {
                const float weight = weight_next;
                weight_next = weight_of(row + row_step);
                if (weight == 0.f) continue;
                const X *x = static_cast<const X *>(g.x) + row * g.xs;
                const Slice sl(x, g.vocab, g.blocks, rank, X());
                const char *from = reinterpret_cast<const char *>(x + sl.a);
                for (int pass = 0; pass < (MODE == kLossAndGrad ? 2 : 1); ++pass) {
                    for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                        wait(empty[stage], phase ^ 1u);
                        if (!ok) break;
                        const uint32_t bytes = 16u * (uint32_t)min(kPieceVecs, sl.v1 - v), bar = smem_u32(&full[stage]);
                        mbar_expect_tx(bar, bytes);
                        bulk_g2s(smem_u32(smem) + stage * kPiece, from + 16LL * v, bytes, bar);
                        ++k;
                        if (++stage == kStages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            }
            let_the_next();
            // no copy is left in flight
            for (unsigned int back = min(k, (unsigned int)kStages); back; --back) {
                const unsigned int piece = k - back;
                mbar_wait_bounded(smem_u32(&full[piece % kStages]), piece / kStages & 1u);
            }
        }
    } else if (warp > kWorkers / 32) {
        // ------------------------------------------------------------ the teacher
        const int me = tid - kWorkers - 32, all = 32 * g.teachers, my_warp = me >> 5;
        unsigned int *map = reinterpret_cast<unsigned int *>(smem + g.map_at);
        // Of two rows at a time, for each of the teacher's warps: the listed tokens that are this block's, their t and logit.
        const int room = (g.top + all - 1) / all * 32;
        auto list = [&](int which, int b, int w) { return reinterpret_cast<float *>(smem + g.teacher_at) + ((which * 2 + b) * g.teachers + w) * room; };
        // over the teacher's warps, in their order
        auto total = [&](float v, int slot) {
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
            if (g.teachers == 1) return v;
            if (lane == 0) teams[slot][my_warp] = v;
            bar_sync(4, all);
            v = teams[slot][0];
            for (int w = 1; w < g.teachers; ++w) v += teams[slot][w];
            return v;
        };
        auto largest = [&](float v, int slot) {
#pragma unroll
            for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
            if (g.teachers == 1) return v;
            if (lane == 0) teams[slot][my_warp] = v;
            bar_sync(4, all);
            v = teams[slot][0];
            for (int w = 1; w < g.teachers; ++w) v = fmaxf(v, teams[slot][w]);
            return v;
        };
        // a token's place among this block's of a row, or -1
        auto place = [&](const Slice &sl, int t) {
            if (t < 0) return -1;
            if (t < sl.a) return rank == 0 ? t : -1;
            if (t >= sl.tail) return rank == g.blocks - 1 ? 8 + t - sl.tail : -1;
            const int v = (t - sl.a) / VEC;
            return v >= sl.v0 && v < sl.v1 ? 16 + t - sl.a - sl.v0 * VEC : -1;
        };
        // The first kTogether listed tokens of each lane are asked for a row ahead, and their logits brought into L2 half a row
        // ahead: the chain weight, token, logit takes as long as a row otherwise.
        int token[kTogether];
        float t[kTogether];
        auto ask = [&](long long row, int j0) {
#pragma unroll
            for (int i = 0; i < kTogether; ++i) {
                const int j = j0 + all * i;
                token[i] = -1;
                t[i] = -INFINITY;
                if (row < g.rows && j < g.top) {
                    const long long v = g.tok_bytes == 4 ? (long long)static_cast<const int *>(g.tok)[row * g.toks + j]
                                                         : static_cast<const long long *>(g.tok)[row * g.toks + j];
                    if (v >= 0 && v < g.vocab) token[i] = (int)v;
                    const long long at = row * g.ts + j;
                    t[i] = g.t_type == FPSK_ELEM_FP32 ? static_cast<const float *>(g.t)[at]
                           : g.t_type == FPSK_ELEM_FP16 ? __half2float(static_cast<const __half *>(g.t)[at])
                                                        : __bfloat162float(static_cast<const __nv_bfloat16 *>(g.t)[at]);
                }
            }
        };
        // The sums over the list and the loss are the first block's, a token's gradient that of the block that has the token.  (Where
        // the blocks exchange nothing each sums for itself.)
        const bool sums = MODE == kGradOnly || rank == 0, losses = MODE != kGradOnly && rank == 0;
        const float ct = g.normalize ? g.c : kLog2e;
        auto bring = [&](long long row) {
            if (row >= g.rows) return;
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            const Slice sl(x, g.vocab, g.blocks, rank, X());
#pragma unroll
            for (int i = 0; i < kTogether; ++i)
                if (losses ? token[i] >= 0 : place(sl, token[i]) >= 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(x + token[i]));
        };
        // loss = sum p (log p - log q) = K + m ((M - xr) / tau + ln S), with the largest listed t as reference u, and the student's logit of
        // its token as xr; normalized, with e = 2^((t - u) c), s = sum e, m = 1:  K = sum e ((t - u) - (x - xr)) / (tau s) - ln s;
        // else with e = 2^(t log2(e)), m = sum e:                                 K = sum e (t - (x - xr) / tau).
        // (Another entry as reference may be one that a large negative number masks, there or in the student, and takes all precision
        // from the sums; the largest one has a share of p.)  Each lane has a reference of its own, which moves with its largest t.
        auto prepare = [&](long long row, int b) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            const Slice sl(x, g.vocab, g.blocks, rank, X());
            float u = kNoReference, xr = 0.f, s = 0.f, d = 0.f, high = kNoReference;
            auto refer = [&](float top, float x_top) {                 // the sums so far, with another reference
                const float f = g.normalize ? exp2_fast((u - top) * ct) : 1.f, more = g.normalize ? (u - top) + (x_top - xr) : (x_top - xr) * g.inv_tau;
                d = s == 0.f || f == 0.f ? 0.f : fmaf(s, more, d) * f;
                s *= f;
                u = top;
                xr = x_top;
            };
            int count = 0;
            for (int base = 0; base < g.top; base += all * kTogether) {            // (as often for each warp: there are barriers in it)
                if (base) ask(row, base + me);
                int at[kTogether];
                float l[kTogether];
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    at[i] = t[i] != -INFINITY ? place(sl, token[i]) : -1;
                    l[i] = at[i] >= 0 || (losses && token[i] >= 0) ? Elem<X>::to_f(x[token[i]]) : 0.f;
                }
                if (anchored) {
#pragma unroll
                    for (int i = 0; i < kTogether; ++i)
                        if (at[i] >= 0 && l[i] < 3e38f) high = fmaxf(high, l[i]);
                }
                if (MODE != kLossOnly) {
#pragma unroll
                    for (int i = 0; i < kTogether; ++i) {
                        const unsigned int own = __ballot_sync(0xFFFFFFFFu, at[i] >= 0);
                        if (at[i] >= 0) {
                            const int k = count + __popc(own & ((1u << lane) - 1u));
                            reinterpret_cast<int *>(list(0, b, my_warp))[k] = token[i];
                            list(1, b, my_warp)[k] = t[i];
                            list(2, b, my_warp)[k] = l[i];
                        }
                        count += __popc(own);
                    }
                }
                if (sums) {
                    float top = u, x_top = xr;
#pragma unroll
                    for (int i = 0; i < kTogether; ++i)
                        if (token[i] >= 0 && t[i] >= top) {
                            top = t[i];
                            x_top = fabsf(l[i]) <= kMostFloat ? l[i] : 0.f;
                        }
                    refer(top, x_top);
#pragma unroll
                    for (int i = 0; i < kTogether; ++i) {
                        if (token[i] < 0 || t[i] == -INFINITY) continue;
                        const float e = exp2_fast(g.normalize ? (t[i] - u) * ct : t[i] * ct);
                        s += e;
                        if (losses && e != 0.f) d = fmaf(e, g.normalize ? (t[i] - u) - (l[i] - xr) : t[i] - (l[i] - xr) * g.inv_tau, d);
                    }
                }
            }
            if (MODE != kLossOnly && lane == 0) counts[b][my_warp] = count;
            if (anchored) {
                high = largest(high, 5);
                if (me == 0) highest[b] = high;
            }
            if (sums) {
                // (the lowest lane of the largest t, and of the lowest warp)
                float top = u;
#pragma unroll
                for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                float x_top = __shfl_sync(0xFFFFFFFFu, xr, __ffs(__ballot_sync(0xFFFFFFFFu, u == top)) - 1);
                if (g.teachers > 1) {
                    if (lane == 0) {
                        teams[0][my_warp] = top;
                        teams[1][my_warp] = x_top;
                    }
                    bar_sync(4, all);
                    for (int w = g.teachers - 1; w >= 0; --w)
                        if (teams[0][w] >= top) {
                            top = teams[0][w];
                            x_top = teams[1][w];
                        }
                }
                refer(top, x_top);
                s = total(s, 3);
                if (losses) d = total(d, 4);
                if (me == 0) {
                    float4 v = make_float4(0.f, xr, 0.f, 0.f);
                    if (!g.normalize) v = make_float4(d, xr, s, 1.f);
                    else if (s != 0.f) v = make_float4(d / s * g.inv_tau - logf(s), xr, u, 1.f / s);
                    taught[b] = v;
                }
            }
            if (g.teachers == 1) __syncwarp();
            else bar_sync(4, all);
            if (me == 0) mbar_arrive(smem_u32(&ready[b]));
        };
        float weight_before = 1.f;
        auto finish = [&](long long row, float weight, int b) {
            bar_sync(2 + b, kWorkers + all);                           // the row's gradient is written
            const float M = result[b].x, S = result[b].y, u = g.normalize ? result[b].z : 0.f, over = result[b].w;
            const float m = mass_of(result[b].z, over);
            if (losses && me == 0) {
                const float ln = logf(S);
                g.loss[row] = m == 0.f ? 0.f : fmaf(m, fmaf(M - taught[b].y, g.inv_tau, ln), taught[b].x);
                if (g.lse) g.lse[row] = fmaf(M, g.inv_tau, ln);
                if (g.sums) {
                    g.sums[2 * row] = M;
                    g.sums[2 * row + 1] = S;
                }
            }
            if (MODE != kLossOnly && m != 0.f) {
                const Slice sl(static_cast<const X *>(g.x) + row * g.xs, g.vocab, g.blocks, rank, X());
                const int *tok = reinterpret_cast<const int *>(list(0, b, my_warp));
                const int count = counts[b][my_warp];
                bool twice = false;
                for (int j = lane; j < count; j += 32) {
                    const int at = place(sl, tok[j]);
                    if (atomicOr(&map[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u) twice = true;
                }
                twice = __any_sync(0xFFFFFFFFu, twice);
                if (g.teachers > 1) {
                    if (lane == 0) teams_twice[my_warp] = twice;
                    bar_sync(4, all);
                    for (int w = 0; w < g.teachers; ++w) twice |= teams_twice[w] != 0;
                }
                const float wt = weight * g.inv_tau, f = wt * m / S;
                G *dx = static_cast<G *>(g.dx) + row * g.dxs;
                for (int j = lane; j < count; j += 32) {
                    const int at = place(sl, tok[j]);
                    map[at >> 5] = 0;
                    float p = exp2_fast((list(1, b, my_warp)[j] - u) * ct) * over;
                    bool first = true;
                    if (twice) {                                       // the first of those that list a token writes it
                        p = 0.f;
                        for (int w = 0; w < g.teachers; ++w)
                            for (int i = 0; i < counts[b][w]; ++i)
                                if (reinterpret_cast<const int *>(list(0, b, w))[i] == tok[j]) {
                                    if (w < my_warp || (w == my_warp && i < j)) first = false;
                                    p += exp2_fast((list(1, b, w)[i] - u) * ct) * over;
                                }
                    }
                    if (first) dx[tok[j]] = Elem<G>::from_f(fmaf(f, exp2_fast((list(2, b, my_warp)[j] - M) * g.c), -wt * p));
                }
                if (g.teachers == 1) __syncwarp();
                else bar_sync(4, all);
            }
        };
        // one row ahead
        long long before = -1;
        unsigned int n = 0;
        ask(first_row, me);
        for (long long row = first_row; row < g.rows; row += row_step) {
            const float weight = weight_next;
            weight_next = weight_of(row + row_step);
            if (weight == 0.f) {
                if (MODE != kGradOnly && rank == 0 && me == 0) {
                    g.loss[row] = 0.f;
                    if (g.lse) g.lse[row] = 0.f;
                    if (g.sums) {
                        g.sums[2 * row] = 0.f;
                        g.sums[2 * row + 1] = 1.f;
                    }
                }
                ask(row + row_step, me);
                continue;
            }
            prepare(row, n & 1);
            ask(row + row_step, me);
            if (before >= 0) finish(before, weight_before, (n - 1) & 1);
            bring(row + row_step);
            before = row;
            weight_before = weight;
            ++n;
        }
        if (before >= 0) finish(before, weight_before, (n - 1) & 1);
    } else {
        // ------------------------------------------------------------ sums and gradients
        unsigned int n = 0;                                            // rows so far
        int stage = 0;
        uint32_t phase = 0;
        const float c = g.c;
        const float2 cc = make_float2(c, c);
        // what the loss kept of a row: M and S, or the log-sum-exp
        auto kept_of = [&](long long row) {
            if (MODE != kGradOnly || row >= g.rows) return make_float2(0.f, 0.f);
            return g.sums ? make_float2(g.sums[2 * row], g.sums[2 * row + 1]) : make_float2(g.lse[row], 0.f);
        };
        float2 kept_next = kept_of(first_row);
        for (long long row = first_row; row < g.rows; row += row_step) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            const float weight = weight_next;
            const float2 kept = kept_next;
            weight_next = weight_of(row + row_step);
            kept_next = kept_of(row + row_step);
            const Slice sl(x, g.vocab, g.blocks, rank, X());
            // the elements in front of the first vector and behind the last: the first block's and the last block's, one to a lane
            int loose = -1;
            if (warp == 0 && rank == 0 && lane < sl.a) loose = lane;
            if (warp == 0 && rank == g.blocks - 1 && lane >= 16 && sl.tail + lane - 16 < g.vocab) loose = sl.tail + lane - 16;
            G *dx = MODE != kLossOnly ? static_cast<G *>(g.dx) + row * g.dxs : nullptr;
            const bool wide = MODE != kLossOnly && reinterpret_cast<uintptr_t>(dx + sl.a) % (VEC * sizeof(G) < 16 ? VEC * sizeof(G) : 16) == 0;
            if (weight == 0.f) {
                if (MODE != kLossOnly) {
                    float2 zero[VEC / 2] = {};
                    for (int v = sl.v0 + tid; v < sl.v1; v += kWorkers) store_vec<G, VEC>(dx + sl.a + (long long)v * VEC, wide, zero);
                    if (loose >= 0) dx[loose] = Elem<G>::from_f(0.f);
                }
                continue;
            }
            const int b = n & 1;
            const float x_loose = loose >= 0 ? Elem<X>::to_f(x[loose]) : -INFINITY;
            float M, S;
            float2 said;                                               // by the teacher
            if (MODE != kGradOnly) {
                wait(ready[b], n >> 1 & 1u);
                const float first = fmaxf(highest[b], x_loose);
                float2 s2 = make_float2(loose >= 0 ? exp2_fast((x_loose - first) * c) : 0.f, 0.f), minus = make_float2(-first, -first);
                for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                    wait(full[stage], phase);
                    const uint4 *piece = reinterpret_cast<const uint4 *>(smem + stage * kPiece) + tid;
                    const int vecs = sl.v1 - v;
                    // A warp's reference is the largest of its first logits, and stays where it is unless a lane's powers of a piece add up to
                    // kMostPowers or more (an infinity, a NaN): then it moves to the piece's largest and the piece is summed anew.
                    auto refer = [&](float top) {
#pragma unroll
                        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                        const float f = exp2_fast((-minus.x - top) * c);
                        s2 = make_float2(s2.x * f, s2.y * f);
                        minus = make_float2(-top, -top);
                    };
                    if (v == sl.v0) refer(tid < vecs ? fmaxf(vec_max<X>(piece[0]), -minus.x) : -minus.x);
                    float2 sum = make_float2(0.f, 0.f);
                    if (vecs >= kPieceVecs) {
#pragma unroll
                        for (int i = 0; i < kPieceVecs / kWorkers; ++i) add_powers<X>(piece[i * kWorkers], minus, cc, sum);
                    } else {
                        for (int at = tid; at < vecs; at += kWorkers) add_powers<X>(piece[at - tid], minus, cc, sum);
                    }
                    if (__any_sync(0xFFFFFFFFu, !(sum.x + sum.y < kMostPowers))) {
                        float top = -minus.x;
                        for (int at = tid; at < min(vecs, kPieceVecs); at += kWorkers) top = fmaxf(top, vec_max<X>(piece[at - tid]));
                        refer(top);
                        sum = make_float2(0.f, 0.f);
                        for (int at = tid; at < min(vecs, kPieceVecs); at += kWorkers) add_powers<X>(piece[at - tid], minus, cc, sum);
                    }
                    s2 = __fadd2_rn(s2, sum);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                LongSum r = join_long<32>(LongSum{-minus.x, (double)s2.x + (double)s2.y}, c);
                if (lane == 0) warps_sum[b][warp] = r;
                bar_sync(1, kWorkers);
                r = join_long<kWorkers / 32>(warps_sum[b][lane % (kWorkers / 32)], c);
                // (the teacher's logits are read before any block goes on to write the gradient, perhaps in the logits' place)
                wait(ready[b], n >> 1 & 1u);
                said = make_float2(taught[b].z, taught[b].w);
                if (g.blocks > 1) {
                    if (tid < g.blocks) {
                        if (tid == 0) mbar_expect_tx(smem_u32(&met[b]), 16u * g.blocks);
                        const uint32_t at = smem_u32(&blocks_sum[b][rank]), bar = smem_u32(&met[b]);
                        asm volatile(
                            "{\n\t.reg .b32 a, m;\n\t"
                            "mapa.shared::cluster.u32 a, %0, %2;\n\t"
                            "mapa.shared::cluster.u32 m, %1, %2;\n\t"
                            "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %6}, [m];\n\t}"
                            ::"r"(at), "r"(bar), "r"(tid), "f"(r.m), "f"((float)r.s), "f"(said.x), "f"(said.y)
                            : "memory");
                    }
                    wait(met[b], n >> 1 & 1u);
                    const float4 theirs = lane < g.blocks ? blocks_sum[b][lane] : make_float4(kNoReference, 0.f, 0.f, 0.f);
                    said = make_float2(blocks_sum[b][0].z, blocks_sum[b][0].w);
                    r = join_long<kRowMostBlocks>(LongSum{theirs.x, theirs.y}, c);
                    r = LongSum{__shfl_sync(0xFFFFFFFFu, r.m, 0), __shfl_sync(0xFFFFFFFFu, r.s, 0)};
                }
                M = r.m;
                S = (float)r.s;
            } else {
                wait(ready[b], n >> 1 & 1u);
                said = make_float2(taught[b].z, taught[b].w);
                M = kept.x;
                S = kept.y;
                if (!g.sums) {
                    M = kept.x * g.tau;
                    if (fabsf(kept.x) <= kMostFloat) M = fminf(fmaxf(M, -kMostFloat), kMostFloat);     // (any M will do)
                    S = expf(fmaf(-M, g.inv_tau, kept.x));             // what M's rounding left of it
                }
            }
            if (tid == 0) result[b] = make_float4(M, S, said.x, said.y);
            if (MODE != kLossOnly) {
                // (a row without a teacher has zeros, whatever it holds)
                const float m = mass_of(said.x, said.y), f = m == 0.f ? 0.f : weight * g.inv_tau * m / S;
                const float2 ff = make_float2(f, f), minus = make_float2(-M, -M);
                G *out = dx + sl.a + ((long long)sl.v0 + tid) * VEC;
                for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                    wait(full[stage], phase);
                    const uint4 *piece = reinterpret_cast<const uint4 *>(smem + stage * kPiece) + tid;
                    const int vecs = sl.v1 - v;
                    if (vecs >= kPieceVecs && wide && m != 0.f) {
#pragma unroll
                        for (int i = 0; i < kPieceVecs / kWorkers; ++i) {
                            float2 e[VEC / 2];
                            gradients<X>(piece[i * kWorkers], minus, cc, ff, e);
                            store_vec<G, VEC>(out + i * kWorkers * VEC, true, e);
                        }
                    } else {
                        for (int at = tid; at < min(vecs, kPieceVecs); at += kWorkers) {
                            float2 e[VEC / 2] = {};
                            if (m != 0.f) gradients<X>(piece[at - tid], minus, cc, ff, e);
                            store_vec<G, VEC>(out + (at - tid) * VEC, wide, e);
                        }
                    }
                    out += kPieceVecs * VEC;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (loose >= 0) dx[loose] = Elem<G>::from_f(m == 0.f ? 0.f : f * exp2_fast((x_loose - M) * c));
            }
            bar_arrive(2 + b, kWorkers + 32 * g.teachers);
            ++n;
        }
    }
    __syncthreads();
    cluster_sync();                                                    // no block leaves before what the others send it
}

constexpr int kMostShared = 224 * 1024;         // dynamic, of a block (227 KB less what is static)
// (131072 FP32 logits, 512 KB a row: eight blocks to a row 513 us, four 700, one 846; 65536: eight 286, four 273, two 364; 32768: four 285,
// two 260, one 373; 8192: two 236, one 155.  262144, with all the clusters that fit 338 us, with 60 MB of rows 304; 400000: 414, 376.)
constexpr long long kRowsInL2 = 40LL << 20, kLongRowsInL2 = 60LL << 20;

template <typename X, typename G, int MODE> static fpsk_status launch_distill(DistillArgs g, cudaStream_t st)
{
    const int vecs = (g.vocab + Vec<X>::n - 1) / Vec<X>::n;
    auto slice_pieces = [&](int blocks) { return ((vecs + blocks - 1) / blocks + kPieceVecs - 1) / kPieceVecs; };
    // (one warp and three, 3000 rows of 100000: 340 and 373 us for 128 tokens listed, 468 and 404 for 256)
    g.teachers = g.top <= 160 ? 1 : kMostTeachers;
    const int teacher = MODE == kLossOnly ? 0 : (int)align_up((size_t)6 * (g.top + 32 * g.teachers) * sizeof(float), 128);
    auto map_bytes = [&](int blocks) { return MODE == kLossOnly ? 0 : (int)align_up((size_t)((vecs + blocks - 1) / blocks * Vec<X>::n + 16 + 31) / 32 * 4, 128); };
    g.teacher_at = kStages * kPiece;
    g.map_at = g.teacher_at + teacher;
    // One block to a row, unless there are too few rows for all SMs, or the rows at work at a time (four blocks to an SM) would take
    // more than kRowsInL2, so that the second look at them finds them gone from L2, or a block's map of its tokens has no room (from
    // 1.3 million tokens a block on; the most blocks always have it).
    const long long row_bytes = (long long)vecs * 16;
    g.blocks = 1;
    while (g.blocks < kRowMostBlocks && slice_pieces(g.blocks) > 1 &&
           (g.rows * g.blocks < 3 * kSms || (MODE == kLossAndGrad && 4 * kSms / g.blocks * row_bytes > kRowsInL2) || g.map_at + map_bytes(g.blocks) > kMostShared))
        g.blocks *= 2;
    g.map_words = map_bytes(g.blocks) / 4;
    Launch launch((unsigned)g.blocks, kWorkers + 32 + 32 * g.teachers, (size_t)g.map_at + map_bytes(g.blocks), g.blocks, st);
    auto kernel = distill_kernel<X, G, MODE>;
    int most = 1;
    FPSK_CUDA_OK(clusters_at_once(reinterpret_cast<const void *>(kernel), launch.cfg, &most));
    // (rows too long for that even with the most blocks each: fewer at a time)
    if (MODE == kLossAndGrad && g.blocks == kRowMostBlocks && most > kLongRowsInL2 / row_bytes) most = (int)(kLongRowsInL2 / row_bytes);
    if (most < 1) most = 1;
    launch.cfg.gridDim = dim3((unsigned)((g.rows < most ? g.rows : most) * g.blocks));
    FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg, kernel, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
template <typename X> static fpsk_status launch_distill_typed(const DistillArgs &g, int grad_type, bool backward, cudaStream_t st)
{
    if (!g.dx) return launch_distill<X, float, kLossOnly>(g, st);
#define FPSK_GRAD(G) (backward ? launch_distill<X, G, kGradOnly>(g, st) : launch_distill<X, G, kLossAndGrad>(g, st))
    if (grad_type == FPSK_ELEM_FP32) return FPSK_GRAD(float);
    if (grad_type == FPSK_ELEM_FP16) return FPSK_GRAD(__half);
    return FPSK_GRAD(__nv_bfloat16);
#undef FPSK_GRAD
}

}  // namespace fpsk

using namespace fpsk;

static fpsk_status distill(const fpsk_distill *a, float *sums, bool backward, int32_t *d_status, void *stream)
{
    if (!a) return FPSK_ERR_NULL;
    if (a->n_rows < 0 || a->n_rows > 0x7FFFFFFFLL || a->vocab < 1 || a->vocab > FPSK_MAX_VOCAB || a->top < 0 || a->top > FPSK_MAX_TOP) return FPSK_ERR_SHAPE;
    if (!elem_ok(a->logits_type) || !elem_ok(a->teacher_type) || (a->dlogits && !elem_ok(a->grad_type))) return FPSK_ERR_DTYPE;
    if (a->token_bytes != 4 && a->token_bytes != 8) return FPSK_ERR_DTYPE;
    if (!(a->temperature > 0.f) || a->temperature > 3.4e38f) return FPSK_ERR_PARAM;
    if (a->n_rows == 0) return FPSK_OK;
    if (!a->logits || (a->top > 0 && (!a->teacher_token || !a->teacher_logit))) return FPSK_ERR_NULL;
    if (backward ? (!a->lse && !sums) || !a->dlogits : !a->loss) return FPSK_ERR_NULL;
    if (a->logits_stride < 0 || a->token_stride < 0 || a->teacher_stride < 0 || (a->dlogits && a->n_rows > 1 && a->dlogits_stride < a->vocab)) return FPSK_ERR_SHAPE;
    if (!aligned(a->logits, a->logits_type) || (a->dlogits && !aligned(a->dlogits, a->grad_type)) || reinterpret_cast<uintptr_t>(a->teacher_token) % a->token_bytes ||
        !aligned(a->teacher_logit, a->teacher_type) || !aligned(a->row_weight, FPSK_ELEM_FP32) || !aligned(a->loss, FPSK_ELEM_FP32) || !aligned(a->lse, FPSK_ELEM_FP32) ||
        !aligned(sums, FPSK_ELEM_FP32))
        return FPSK_ERR_ALIGN;
    const double inv = 1.0 / (double)a->temperature;
    if (inv * 1.4426950408889634 > 3.4e38) return FPSK_ERR_PARAM;      // (c)
    DistillArgs g = {};
    g.x = a->logits; g.tok = a->teacher_token; g.t = a->teacher_logit; g.weight = a->row_weight;
    g.loss = a->loss; g.lse = a->lse; g.sums = sums; g.dx = a->dlogits;
    g.xs = a->logits_stride; g.toks = a->token_stride; g.ts = a->teacher_stride; g.dxs = a->dlogits_stride;
    g.rows = a->n_rows; g.vocab = a->vocab; g.top = a->top;
    g.tok_bytes = a->token_bytes; g.t_type = a->teacher_type;
    g.normalize = a->normalize != 0;
    g.tau = a->temperature;
    g.inv_tau = (float)inv;
    g.c = (float)(inv * 1.4426950408889634);
    g.status = d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->logits_type == FPSK_ELEM_FP32) return launch_distill_typed<float>(g, a->grad_type, backward, st);
    if (a->logits_type == FPSK_ELEM_FP16) return launch_distill_typed<__half>(g, a->grad_type, backward, st);
    return launch_distill_typed<__nv_bfloat16>(g, a->grad_type, backward, st);
}

extern "C" fpsk_status fpsk_distill_loss(const fpsk_distill *a, int32_t *d_status, void *stream) { return distill(a, nullptr, false, d_status, stream); }
extern "C" fpsk_status fpsk_distill_loss_backward(const fpsk_distill *a, int32_t *d_status, void *stream) { return distill(a, nullptr, true, d_status, stream); }
extern "C" fpsk_status fpsk_distill_loss_sums(const fpsk_distill *a, float *sums, int32_t *d_status, void *stream) { return distill(a, sums, false, d_status, stream); }
extern "C" fpsk_status fpsk_distill_loss_backward_sums(const fpsk_distill *a, const float *sums, int32_t *d_status, void *stream)
{
    return distill(a, const_cast<float *>(sums), true, d_status, stream);
}
