// The loss of rows of logits against a teacher's top logits, and its gradient.
//
// q = softmax(x / tau), p over the listed tokens; loss = sum_j p_j (log p_j - log q_j); d/dx_v = (m q_v - p_v) / tau, m = sum p.
// In powers of two, with c = log2(e) / tau and a reference M near the row's largest logit: S = sum 2^((x - M) c), q_v = 2^((x_v - M) c) / S,
// log q_v = (x_v - M) / tau - ln S.  M and S stay apart to the end, so that nothing is rounded at the size of the logarithm.
//
// What bounds it is memory: the logits once, the gradient once.  The gradient needs S first, so a row has to stay on the chip from the
// first look at it to the second: a cluster of blocks holds it in shared memory, each block a slice (131072 FP32 logits: eight times
// 64 KB, three blocks to an SM).  One warp of a block copies pieces of 8 KB into a ring; eight warps sum a slice up, exchange (M, S)
// through the cluster's shared memory, and write the gradient, freeing the pieces as they go for the next row's copies; one warp prepares the
// teacher's probabilities for the next row and takes them off the gradient of the one before, so that neither is waited for.
#include "decoder.cuh"
#include "stream_pipe.cuh"

#include <mutex>

namespace fpsk {

enum { kLossOnly = 0, kLossAndGrad = 1, kGradOnly = 2 };

struct DistillArgs {
    const void *x, *tok, *t;
    const float *weight;
    float *loss, *lse;
    void *dx;
    long long xs, toks, ts, dxs, rows;
    int vocab, top;
    int tok_bytes, t_type;
    int normalize;
    float tau, inv_tau, c;             // c = log2(e) / tau
    int blocks;                        // of a row
    int stages;                        // of the ring
    int resident;                      // a slice fits the ring: it is copied once for both passes
    int teacher_at, map_at, map_words; // in shared memory: behind the ring the teacher's arrays, and the map of listed tokens
    int32_t *status;
};

constexpr int kWorkers = 128, kDistillThreads = kWorkers + 64;
constexpr int kPiece = 8192, kPieceVecs = kPiece / 16, kMostStages = 27;
constexpr float kNoReference = -3.4e38f;

__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("barrier.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// 2^((x - M) c) summed
struct RefSum {
    float m, s;
};
// Joined over a warp's first LANES lanes (the others hold no reference), in a fixed order; every lane has the result.
template <int LANES> __device__ __forceinline__ RefSum join_lanes(RefSum r, float c)
{
    float top = r.m;
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    float s = r.s * exp2_fast((r.m - top) * c);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return RefSum{top, s};
}

// A vector of 16 bytes as pairs.
template <typename X> struct Vec;
template <> struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void open(const uint4 &u, float2 (&v)[2])
    {
        v[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        v[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
};
template <typename X> struct Vec16 {
    static constexpr int n = 8;
    static __device__ __forceinline__ void open(const uint4 &u, float2 (&v)[4])
    {
        v[0] = HalfTraits<X>::unpack2(u.x);
        v[1] = HalfTraits<X>::unpack2(u.y);
        v[2] = HalfTraits<X>::unpack2(u.z);
        v[3] = HalfTraits<X>::unpack2(u.w);
    }
};
template <> struct Vec<__half> : Vec16<__half> {};
template <> struct Vec<__nv_bfloat16> : Vec16<__nv_bfloat16> {};

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

// Where the 16-byte vectors of a row lie: `a` elements in front of the first, `n` vectors, of which a block has [v0, v1).
struct Slice {
    int a, n, v0, v1, tail;            // tail: first element behind the vectors
    template <typename X> __device__ __forceinline__ Slice(const X *row, int vocab, int blocks, int rank, X)
    {
        const int per = Vec<X>::n;
        a = min(vocab, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(X));
        n = (vocab - a) / per;
        tail = a + n * per;
        const int each = (n + blocks - 1) / blocks;
        v0 = min(n, rank * each);
        v1 = min(n, v0 + each);
    }
};

// Stores the gradients of one vector's elements.
template <typename G, int N> __device__ __forceinline__ void store_vec(G *p, bool wide, const float2 (&v)[N / 2])
{
    if (wide) {
        if (sizeof(G) == 4) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) reinterpret_cast<float4 *>(p)[i] = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
        } else if (N == 8) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = round_pair<typename std::conditional<sizeof(G) == 2, G, __half>::type>(v[i % (N / 2)].x, v[i % (N / 2)].y);
            *reinterpret_cast<uint4 *>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        } else {
            uint32_t u[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) u[i] = round_pair<typename std::conditional<sizeof(G) == 2, G, __half>::type>(v[i].x, v[i].y);
            *reinterpret_cast<uint2 *>(p) = make_uint2(u[0], u[1]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        p[2 * i] = Elem<G>::from_f(v[i].x);
        p[2 * i + 1] = Elem<G>::from_f(v[i].y);
    }
}

template <typename X, typename G, int MODE> __global__ void __launch_bounds__(kDistillThreads, 3) distill_kernel(const __grid_constant__ DistillArgs g)
{
    constexpr int VEC = Vec<X>::n;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned long long full[kMostStages], empty[kMostStages], ready[2], met[2];
    __shared__ float2 blocks_sum[2][kRowMostBlocks];                   // written by the cluster's blocks
    __shared__ float2 warps_sum[2][kWorkers / 32];
    __shared__ float2 result[2];
    __shared__ float mass[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)cluster_rank();
    const long long first_row = blockIdx.x / g.blocks, row_step = gridDim.x / g.blocks;
    if (tid == 0) {
        for (int s = 0; s < g.stages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), kWorkers / 32);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&ready[b]), 1);
            mbar_init(smem_u32(&met[b]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < g.map_words; i += kDistillThreads) reinterpret_cast<unsigned int *>(smem + g.map_at)[i] = 0;
    __syncthreads();
    cluster_sync();
    // Every wait is bounded; once one has given up the others are passed over, and all roles still run to their ends.
    bool ok = true;
    auto wait = [&](unsigned long long &bar, uint32_t parity) {
        if (ok && !mbar_wait_bounded(smem_u32(&bar), parity)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
    };

    if (warp == kWorkers / 32) {
        // ------------------------------------------------------------ copies
        if (lane == 0) {
            unsigned int k = 0;                                        // pieces so far
            int stage = 0;
            uint32_t phase = 0;
            for (long long row = first_row; row < g.rows && ok; row += row_step) {
                if (g.weight && g.weight[row] == 0.f) continue;
                const X *x = static_cast<const X *>(g.x) + row * g.xs;
                const Slice sl(x, g.vocab, g.blocks, rank, X());
                const char *from = reinterpret_cast<const char *>(x + sl.a);
                for (int pass = 0; pass < (MODE == kLossAndGrad && !g.resident ? 2 : 1); ++pass) {
                    for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                        wait(empty[stage], phase ^ 1u);
                        if (!ok) break;
                        const uint32_t bytes = 16u * (uint32_t)min(kPieceVecs, sl.v1 - v), bar = smem_u32(&full[stage]);
                        mbar_expect_tx(bar, bytes);
                        bulk_g2s(smem_u32(smem) + stage * kPiece, from + 16LL * v, bytes, bar);
                        ++k;
                        if (++stage == g.stages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            }
            // no copy is left in flight
            for (unsigned int back = min(k, (unsigned int)g.stages); back; --back) {
                const unsigned int piece = k - back;
                mbar_wait_bounded(smem_u32(&full[piece % g.stages]), piece / g.stages & 1u);
            }
        }
    } else if (warp == kWorkers / 32 + 1) {
        // ------------------------------------------------------------ the teacher
        float *arrays = reinterpret_cast<float *>(smem + g.teacher_at);
        unsigned int *map = reinterpret_cast<unsigned int *>(smem + g.map_at);
        // of two rows at a time: token, log p, p, logit
        auto array = [&](int which, int b) { return arrays + (which * 2 + b) * g.top; };
        auto prepare = [&](long long row, int b) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            int *tok = reinterpret_cast<int *>(array(0, b));
            float *logp = array(1, b), *prob = array(2, b), *xs = array(3, b);
            float most = -INFINITY;
            for (int j = lane; j < g.top; j += 32) {
                const long long token = g.tok_bytes == 4 ? (long long)static_cast<const int *>(g.tok)[row * g.toks + j]
                                                         : static_cast<const long long *>(g.tok)[row * g.toks + j];
                const bool in = token >= 0 && token < g.vocab;
                const long long at = row * g.ts + j;
                const float t = g.t_type == FPSK_ELEM_FP32 ? static_cast<const float *>(g.t)[at]
                                : g.t_type == FPSK_ELEM_FP16 ? __half2float(static_cast<const __half *>(g.t)[at])
                                                             : __bfloat162float(static_cast<const __nv_bfloat16 *>(g.t)[at]);
                const float l = !in ? -INFINITY : g.normalize ? t * g.inv_tau : t;
                tok[j] = in ? (int)token : -1;
                xs[j] = in ? Elem<X>::to_f(x[token]) : 0.f;
                logp[j] = l;
                most = fmaxf(most, l);
            }
            if (g.normalize) {
#pragma unroll
                for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
                float s = 0.f;
                for (int j = lane; j < g.top; j += 32) s += logp[j] == -INFINITY ? 0.f : expf(logp[j] - most);
#pragma unroll
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
                const float ln = logf(s);
                for (int j = lane; j < g.top; j += 32)
                    if (logp[j] != -INFINITY) logp[j] = logp[j] - most - ln;
            }
            float sum = 0.f;
            for (int j = lane; j < g.top; j += 32) {
                const float p = logp[j] == -INFINITY ? 0.f : expf(logp[j]);
                prob[j] = p;
                sum += p;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            if (lane == 0) mass[b] = sum;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ready[b]));
        };
        auto finish = [&](long long row, int b) {
            const int *tok = reinterpret_cast<const int *>(array(0, b));
            const float *logp = array(1, b), *prob = array(2, b), *xs = array(3, b);
            bar_sync(2 + b, kWorkers + 32);                            // the row's gradient is written
            const float M = result[b].x, S = result[b].y;
            if (MODE != kGradOnly && rank == 0) {
                const float ln = logf(S);
                float l = 0.f;
                for (int j = lane; j < g.top; j += 32)
                    if (logp[j] != -INFINITY) l = fmaf(prob[j], logp[j] - fmaf(xs[j] - M, g.inv_tau, -ln), l);
#pragma unroll
                for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
                if (lane == 0) {
                    g.loss[row] = l;
                    if (g.lse) g.lse[row] = fmaf(M, g.inv_tau, ln);
                }
            }
            if (MODE != kLossOnly && mass[b] != 0.f) {
                const X *x = static_cast<const X *>(g.x) + row * g.xs;
                const Slice sl(x, g.vocab, g.blocks, rank, X());
                // a listed token's place among this block's, or -1
                auto place = [&](int t) {
                    if (t < 0) return -1;
                    if (t < sl.a) return rank == 0 ? t : -1;
                    if (t >= sl.tail) return rank == g.blocks - 1 ? 8 + t - sl.tail : -1;
                    const int v = (t - sl.a) / VEC;
                    return v >= sl.v0 && v < sl.v1 ? 16 + t - sl.a - sl.v0 * VEC : -1;
                };
                bool twice = false;
                for (int j = lane; j < g.top; j += 32) {
                    const int at = place(tok[j]);
                    if (at >= 0 && atomicOr(&map[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u) twice = true;
                }
                twice = __any_sync(0xFFFFFFFFu, twice);
                __syncwarp();
                const float wt = (g.weight ? g.weight[row] : 1.f) * g.inv_tau, f = wt * mass[b] / S;
                G *dx = static_cast<G *>(g.dx) + row * g.dxs;
                for (int j = lane; j < g.top; j += 32) {
                    const int at = place(tok[j]);
                    if (at < 0) continue;
                    map[at >> 5] = 0;
                    float p = prob[j];
                    bool first = true;
                    if (twice) {                                       // the first of those that list a token writes it
                        p = 0.f;
                        for (int i = 0; i < g.top; ++i)
                            if (tok[i] == tok[j]) {
                                if (i < j) first = false;
                                p += prob[i];
                            }
                    }
                    if (first) dx[tok[j]] = Elem<G>::from_f(fmaf(f, exp2_fast((xs[j] - M) * g.c), -wt * p));
                }
                __syncwarp();
            }
        };
        // one row ahead
        long long before = -1;
        unsigned int n = 0;
        for (long long row = first_row; row < g.rows; row += row_step) {
            if (g.weight && g.weight[row] == 0.f) {
                if (MODE != kGradOnly && rank == 0 && lane == 0) {
                    g.loss[row] = 0.f;
                    if (g.lse) g.lse[row] = 0.f;
                }
                continue;
            }
            prepare(row, n & 1);
            if (before >= 0) finish(before, (n - 1) & 1);
            before = row;
            ++n;
        }
        if (before >= 0) finish(before, (n - 1) & 1);
    } else {
        // ------------------------------------------------------------ sums and gradients
        unsigned int n = 0;                                            // rows so far
        int stage = 0;
        uint32_t phase = 0;
        const float c = g.c;
        const float2 cc = make_float2(c, c);
        for (long long row = first_row; row < g.rows; row += row_step) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            const float weight = g.weight ? g.weight[row] : 1.f;
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
            const int stage0 = stage;
            if (MODE != kGradOnly) {
                RefSum r = {kNoReference, 0.f};
                if (loose >= 0 && x_loose != -INFINITY) r = RefSum{x_loose, x_loose == x_loose ? 1.f : x_loose};
                float2 s2 = make_float2(r.s, 0.f), minus = make_float2(-r.m, -r.m);
                for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                    wait(full[stage], phase);
                    const uint4 *piece = reinterpret_cast<const uint4 *>(smem + stage * kPiece) + tid;
                    const int vecs = sl.v1 - v;
                    // The reference is the largest of the thread's first logits, and stays where it is unless a piece's powers add up to
                    // 2^100 or more (an infinity, a NaN): then it moves to the piece's largest and the piece is summed anew.  A
                    // reference below the row's largest costs no precision.
                    if (v == sl.v0 && tid < vecs && loose < 0) {
                        const float top = vec_max<X>(piece[0]);
                        if (top != -INFINITY) minus = make_float2(-top, -top);
                    }
                    float2 sum = make_float2(0.f, 0.f);
                    if (vecs >= kPieceVecs) {
#pragma unroll
                        for (int i = 0; i < kPieceVecs / kWorkers; ++i) add_powers<X>(piece[i * kWorkers], minus, cc, sum);
                    } else {
                        for (int at = tid; at < vecs; at += kWorkers) add_powers<X>(piece[at - tid], minus, cc, sum);
                    }
                    if (!(sum.x + sum.y < 1.2676506e30f)) {
                        float top = -minus.x;
                        for (int at = tid; at < min(vecs, kPieceVecs); at += kWorkers) top = fmaxf(top, vec_max<X>(piece[at - tid]));
                        const float f = exp2_fast((-minus.x - top) * c);
                        s2 = make_float2(s2.x * f, s2.y * f);
                        minus = make_float2(-top, -top);
                        sum = make_float2(0.f, 0.f);
                        for (int at = tid; at < min(vecs, kPieceVecs); at += kWorkers) add_powers<X>(piece[at - tid], minus, cc, sum);
                    }
                    s2 = __fadd2_rn(s2, sum);
                    if (MODE == kLossOnly || !g.resident) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                    }
                    if (++stage == g.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                r = join_lanes<32>(RefSum{-minus.x, s2.x + s2.y}, c);
                if (lane == 0) warps_sum[b][warp] = make_float2(r.m, r.s);
                bar_sync(1, kWorkers);
                const float2 mine = warps_sum[b][lane % (kWorkers / 32)];
                r = join_lanes<kWorkers / 32>(RefSum{mine.x, mine.y}, c);
                // (the teacher's logits are read before any block goes on to write the gradient, perhaps in the logits' place)
                wait(ready[b], n >> 1 & 1u);
                if (g.blocks > 1) {
                    if (tid < g.blocks) {
                        if (tid == 0) mbar_expect_tx(smem_u32(&met[b]), 8u * g.blocks);
                        const uint32_t at = smem_u32(&blocks_sum[b][rank]), bar = smem_u32(&met[b]);
                        asm volatile(
                            "{\n\t.reg .b32 a, m;\n\t"
                            "mapa.shared::cluster.u32 a, %0, %2;\n\t"
                            "mapa.shared::cluster.u32 m, %1, %2;\n\t"
                            "st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [a], {%3, %4}, [m];\n\t}"
                            ::"r"(at), "r"(bar), "r"(tid), "f"(r.m), "f"(r.s)
                            : "memory");
                    }
                    wait(met[b], n >> 1 & 1u);
                    const float2 theirs = lane < g.blocks ? blocks_sum[b][lane] : make_float2(kNoReference, 0.f);
                    r = join_lanes<kRowMostBlocks>(RefSum{theirs.x, theirs.y}, c);
                    r = RefSum{__shfl_sync(0xFFFFFFFFu, r.m, 0), __shfl_sync(0xFFFFFFFFu, r.s, 0)};
                }
                M = r.m;
                S = r.s;
            } else {
                wait(ready[b], n >> 1 & 1u);
                const float lse = g.lse[row];
                M = lse * g.tau;
                S = expf(fmaf(-M, g.inv_tau, lse));                    // what M's rounding left of it
            }
            if (tid == 0) result[b] = make_float2(M, S);
            if (MODE != kLossOnly) {
                if (g.resident && MODE == kLossAndGrad) stage = stage0;
                // (a row without a teacher has zeros, whatever it holds)
                const float m = mass[b], f = m == 0.f ? 0.f : weight * g.inv_tau * m / S;
                const float2 ff = make_float2(f, f), minus = make_float2(-M, -M);
                G *out = dx + sl.a + ((long long)sl.v0 + tid) * VEC;
                for (int v = sl.v0; v < sl.v1; v += kPieceVecs) {
                    if (MODE == kGradOnly || !g.resident) wait(full[stage], phase);
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
                    if (++stage == g.stages) {
                        stage = 0;
                        if (MODE == kGradOnly || !g.resident) phase ^= 1u;
                    }
                }
                if (loose >= 0) dx[loose] = Elem<G>::from_f(m == 0.f ? 0.f : f * exp2_fast((x_loose - M) * c));
            }
            bar_arrive(2 + b, kWorkers + 32);
            ++n;
        }
    }
    __syncthreads();
    cluster_sync();                                                    // no block leaves before what the others send it
}

// Clusters of a launch that fit the device side by side, asked once for each shape of launch.
static int clusters_at_once(const void *kernel, const cudaLaunchConfig_t &cfg, int *out)
{
    struct Key {
        const void *kernel;
        int device, blocks;
        size_t bytes;
    };
    static std::mutex lock;
    static Key keys[64];
    static int values[64], used = 0;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int blocks = (int)cfg.attrs[0].val.clusterDim.x;
    std::lock_guard<std::mutex> hold(lock);
    for (int i = 0; i < (used < 64 ? used : 64); ++i)
        if (keys[i].kernel == kernel && keys[i].device == device && keys[i].blocks == blocks && keys[i].bytes == cfg.dynamicSmemBytes) {
            *out = values[i];
            return cudaSuccess;
        }
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 2048);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(out, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (*out < 1) *out = 1;
    keys[used % 64] = Key{kernel, device, blocks, cfg.dynamicSmemBytes};
    values[used % 64] = *out;
    ++used;
    return cudaSuccess;
}

constexpr int kMostBytes = 227 * 1024 - 2048, kThirdBytes = 74 * 1024;

template <typename X, typename G, int MODE> static fpsk_status launch_distill(DistillArgs g, cudaStream_t st)
{
    const int vecs = (g.vocab + Vec<X>::n - 1) / Vec<X>::n;
    auto slice_pieces = [&](int blocks) { return ((vecs + blocks - 1) / blocks + kPieceVecs - 1) / kPieceVecs; };
    const int teacher = (int)align_up((size_t)8 * g.top * sizeof(float), 128);
    auto map_bytes = [&](int blocks) { return MODE == kLossOnly ? 0 : (int)align_up((size_t)((vecs + blocks - 1) / blocks * Vec<X>::n + 16 + 31) / 32 * 4, 128); };
    // Slices of 64 KB at most, so that three blocks share an SM and one computes while another's copies arrive; smaller ones where there
    // are few rows.
    g.blocks = 1;
    while (g.blocks < kRowMostBlocks && (slice_pieces(g.blocks) > 8 || (g.rows * g.blocks < 3 * kSms && slice_pieces(g.blocks) > 1))) g.blocks *= 2;
    const int pieces = slice_pieces(g.blocks), fixed = teacher + map_bytes(g.blocks);
    int stages = (kThirdBytes - fixed) / kPiece;
    if (MODE == kLossAndGrad && stages < pieces) stages = (113 * 1024 - 2048 - fixed) / kPiece;
    if (MODE == kLossAndGrad && stages < pieces) stages = (kMostBytes - fixed) / kPiece;
    if (stages < 4) stages = 4;                                        // (a map of the largest vocabulary leaves room for them)
    if (stages > kMostStages) stages = kMostStages;
    g.stages = stages;
    g.resident = pieces <= stages;
    g.teacher_at = stages * kPiece;
    g.map_at = g.teacher_at + teacher;
    g.map_words = map_bytes(g.blocks) / 4;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)g.blocks);
    cfg.blockDim = dim3(kDistillThreads);
    cfg.dynamicSmemBytes = (size_t)g.map_at + map_bytes(g.blocks);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = g.blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    auto kernel = distill_kernel<X, G, MODE>;
    int most = 1;
    FPSK_CUDA_OK((cudaError_t)clusters_at_once(reinterpret_cast<const void *>(kernel), cfg, &most));
    cfg.gridDim = dim3((unsigned)((g.rows < most ? g.rows : most) * g.blocks));
    FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, g));
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

static fpsk_status distill(const fpsk_distill *a, bool backward, int32_t *d_status, void *stream)
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
    if (reinterpret_cast<uintptr_t>(a->logits) % elem_bytes(a->logits_type) || (a->dlogits && reinterpret_cast<uintptr_t>(a->dlogits) % elem_bytes(a->grad_type)))
        return FPSK_ERR_ALIGN;
    const double inv = 1.0 / (double)a->temperature;
    if (inv > 3.4e38) return FPSK_ERR_PARAM;
    DistillArgs g = {};
    g.x = a->logits; g.tok = a->teacher_token; g.t = a->teacher_logit; g.weight = a->row_weight;
    g.loss = a->loss; g.lse = a->lse; g.dx = a->dlogits;
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

extern "C" fpsk_status fpsk_distill_loss(const fpsk_distill *a, int32_t *d_status, void *stream) { return distill(a, false, d_status, stream); }
extern "C" fpsk_status fpsk_distill_loss_backward(const fpsk_distill *a, int32_t *d_status, void *stream) { return distill(a, true, d_status, stream); }
