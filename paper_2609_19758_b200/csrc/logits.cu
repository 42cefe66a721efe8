// Penalties, biases and grammar masks on rows of logits, with the greedy token and the log-sum-exp of what is left.
//
// For a token v of a row: z = l_v; seen: z > 0 ? z / rep : z rep; z -= freq c + pres where c > 0; z += biases; masked: -inf.
//
// What bounds it is memory, the logits once and the result once, where there is no history; with one it is the instructions and barriers
// of finding out what it touches.  A cluster of blocks takes a row, whose pieces of 8 KB go to the blocks in turn.  One warp of a block
// copies them into a ring, passing over those that a mask forbids as a whole; the others count in shared memory, a word to a token, how
// often the history has each, and then go through the pieces: touched tokens are adjusted in place, and the largest is looked for
// with one vote of a warp for all its tokens of a piece.  Tokens with biases are stored as they were and done behind the stream, one to a thread.
// An in-place call without token or lse copies nothing: only what changes is read or written.
//
// Measured: 2000 rows of 32000 FP32 logits without histories, token and log-sum-exp, 51 us (0.77 of a copy); 96 rows of 131072 with histories
// of 4096, biases and masks 43 us (17 without them, floor 8): a block's 16384 tokens take some 20 us, of which the history's counting is 4 and
// the words' looking through 3, three blocks to an SM; 640 rows of 50257 BF16 to FP32 93 us (46, floor 30); one row of 32000 with a history of
// 1000 7 us.  Tokens adjusted by divided threads of their own, in lists of 32, took 52 and 113 us, with a map of bits for the stream 60.
#include "decoder.cuh"

namespace fpsk {

struct LogitsArgs {
    const void *x;
    void *out;
    long long xs, os, rows;
    int vocab;
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
    int blocks, log_blocks;            // of a row
    int chunk;                         // vectors whose tokens have words at a time, a multiple of a piece
    int in_place;                      // and neither token nor lse wanted: what stays as it is is left alone
    int words_at;                      // in shared memory, behind the ring
    int32_t *status;
};

// Threads that work: the history's counting is bound by its latency (96 rows of 131072 with histories of 4096: 43 us with 256, 52 with 128).
template <bool WORDS> struct Workers {
    static constexpr int n = WORDS ? 256 : 128, threads = n + 32, stages = 4;       // (three blocks to an SM, or five)
};
constexpr int kRowPiece = 8192, kRowPieceVecs = kRowPiece / 16;
constexpr int kWordBytes = 32 * 1024;  // of the words of a chunk, at most
constexpr int kMostChunk = 32768;      // tokens of a chunk without words, at most

// What a block has of a row: `a` elements in front of the first 16-byte vector, `n` vectors, of whose pieces every blocks-th is the
// block's (what is frequent has low numbers in many vocabularies: a slice of its own would be most of the work).  Its own vectors
// and their tokens are numbered from 0, `mine` of them.
template <typename X> struct Share {
    static constexpr int N = Vec<X>::n, kTokens = kRowPieceVecs * N;
    int a, n, tail, mine, rank, log;   // tail: first element behind the vectors; log: of the blocks' number
    __device__ __forceinline__ Share(const X *row, int vocab, int log_blocks, int rank_) : rank(rank_), log(log_blocks)
    {
        a = min(vocab, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(X));
        n = (vocab - a) / N;
        tail = a + n * N;
        const int pieces = (n + kRowPieceVecs - 1) / kRowPieceVecs, own = (pieces - rank + (1 << log) - 1) >> log;
        mine = own <= 0 ? 0 : (own - 1) * kRowPieceVecs + min(kRowPieceVecs, n - (((own - 1) << log) + rank) * kRowPieceVecs);
    }
    // the vector of the row, the token, behind a number of the block's own
    __device__ __forceinline__ int vec(int own) const { return ((own / kRowPieceVecs) << log | rank) * kRowPieceVecs + own % kRowPieceVecs; }
    __device__ __forceinline__ int token(int own) const { return a + ((own / kTokens) << log | rank) * kTokens + own % kTokens; }
    // its own number of a token, or -1
    __device__ __forceinline__ int own_of(int v) const
    {
        const unsigned int t = (unsigned int)(v - a), piece = t / kTokens;
        if (t >= (unsigned int)(n * N) || (int)(piece & ((1u << log) - 1u)) != rank) return -1;
        return (int)((piece >> log) * kTokens + t % kTokens);
    }
};

// A token's word: how often it comes behind the prompt, and from the top whether it is in the prompt, has a bias, has several.  16 bits
// where the history is short enough.
template <typename W> struct Word {
    static constexpr unsigned int kInPrompt = 1u << (8 * sizeof(W) - 1), kBiased = kInPrompt >> 1, kBiasedTwice = kInPrompt >> 2, kTimes = kBiasedTwice - 1;
    static __device__ __forceinline__ int shift(int at) { return sizeof(W) == 2 ? 16 * (at & 1) : 0; }
    static __device__ __forceinline__ unsigned int *home(W *words, int at) { return reinterpret_cast<unsigned int *>(words) + (sizeof(W) == 2 ? at >> 1 : at); }
    static __device__ __forceinline__ void count(W *words, int at) { atomicAdd(home(words, at), 1u << shift(at)); }
    static __device__ __forceinline__ unsigned int mark(W *words, int at, unsigned int bits) { return atomicOr(home(words, at), bits << shift(at)) >> shift(at); }
    // whether any of N tokens has a word that is not 0; `at` is a multiple of N
    template <int N> static __device__ __forceinline__ bool any(const W *words, int at)
    {
        if (sizeof(W) * N == 8) {
            const uint2 u = *reinterpret_cast<const uint2 *>(words + at);
            return u.x | u.y;
        }
        unsigned int some = 0;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(W) * N / 16); ++i) {
            const uint4 u = reinterpret_cast<const uint4 *>(words + at)[i];
            some |= u.x | u.y | u.z | u.w;
        }
        return some;
    }
};

// the order of argmax: a NaN above all, the lowest token of equal ones
__device__ __forceinline__ unsigned long long pick_key(float z, int v)
{
    const unsigned int b = __float_as_uint(z + 0.f);                   // (-0 is 0)
    const unsigned int k = z != z ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (unsigned long long)k << 32 | (0xFFFFFFFFu - (unsigned int)v);
}
constexpr unsigned int kKeyNothing = 0x007FFFFFu, kKeyInfinity = 0xFF800000u, kKeyNan = 0xFFFFFFFFu;
__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

// A warp's largest so far and its token, the same in all lanes, and each lane's sum of powers with the largest as reference.  (One that
// followed it at a distance of 2^60 left log-sum-exps 3e-6 off: exponents are rounded at their own size.  It took as long.)
struct Picked {
    float best, m, s;
    int at;
    __device__ __forceinline__ void follow()
    {
        if (best > m) {
            s *= exp2_fast((m - best) * kLog2e);
            m = best;
        }
    }
    // K vectors of N values of each lane; the first values of a lane's vectors are the tokens v, v + step, ..  Tokens rise from lane to
    // lane, vector to vector and call to call.
    template <int K, int N> __device__ __forceinline__ void add(const float2 (&z)[K][N / 2], int v, int step, bool sum)
    {
        float tops[K], top;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            tops[k] = max_nan(z[k][0].x, z[k][0].y);
#pragma unroll
            for (int i = 1; i < N / 2; ++i) tops[k] = max_nan(tops[k], max_nan(z[k][i].x, z[k][i].y));
        }
        top = tops[0];
#pragma unroll
        for (int k = 1; k < K; ++k) top = max_nan(top, tops[k]);
        if (__any_sync(0xFFFFFFFFu, !(top <= best))) {
            float most = top;
#pragma unroll
            for (int o = 16; o; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
            const bool nan = most != most;
            if (nan ? best == best : most > best) {
                bool found = false;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const unsigned int who = __ballot_sync(0xFFFFFFFFu, nan ? tops[k] != tops[k] : tops[k] == most);
                    if (who && !found) {
                        found = true;
                        int first = 0;                                 // the place of the lane's first such value
#pragma unroll
                        for (int i = N - 1; i >= 0; --i) {
                            const float x = i & 1 ? z[k][i / 2].y : z[k][i / 2].x;
                            if (nan ? x != x : x == most) first = i;
                        }
                        at = __shfl_sync(0xFFFFFFFFu, v + k * step + first, __ffs(who) - 1);
                    }
                }
                best = most;
                follow();
            }
        }
        if (sum) {
            const float2 minus = make_float2(-m, -m), c = make_float2(kLog2e, kLog2e);
            float2 t = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const float2 y = __fmul2_rn(__fadd2_rn(z[k][i], minus), c);
                    t = __fadd2_rn(t, make_float2(exp2_fast(y.x), exp2_fast(y.y)));
                }
            s += t.x + t.y;
        }
    }
};

// The same of a lane's single tokens, in any order.
struct Single {
    float best, m, s;
    int at;
    __device__ __forceinline__ void add(float z, int v, bool sum)
    {
        if (z != z ? best == best : z > best) {
            best = z;
            at = v;
            if (best > m) {
                s *= exp2_fast((m - best) * kLog2e);
                m = best;
            }
        } else if (v < at && (z == best || z != z)) {
            at = v;
        }
        if (sum) s += exp2_fast((z - m) * kLog2e);
    }
};

// the bits of N tokens from `e` on
template <int N> __device__ __forceinline__ unsigned int mask_bits(const int *mask, int e)
{
    const int w = e >> 5, s = e & 31;
    unsigned int b = (unsigned int)mask[w] >> s;
    if (s + N > 32) b |= (unsigned int)mask[w + 1] << (32 - s);
    return b & ((1u << N) - 1u);
}
// O: the type of the result, or void.  W: of the words, void where there are neither histories nor biases.
template <typename X, typename O, typename W> __global__ void __launch_bounds__(Workers<!std::is_void<W>::value>::threads, std::is_void<W>::value ? 5 : 3) adjust_logits_kernel(const __grid_constant__ LogitsArgs g)
{
    constexpr int N = Vec<X>::n, kRowWorkers = Workers<!std::is_void<W>::value>::n, kRowWarps = kRowWorkers / 32, kEachVecs = kRowPieceVecs / kRowWorkers;
    constexpr int kRowStages = Workers<!std::is_void<W>::value>::stages;
    constexpr bool OUT = !std::is_void<O>::value, WORDS = !std::is_void<W>::value;
    constexpr unsigned int kAll = (1u << N) - 1u;
    using Out = typename std::conditional<OUT, O, float>::type;
    using Wd = typename std::conditional<WORDS, W, unsigned int>::type;
    using F = Word<Wd>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned long long full[kRowStages], empty[kRowStages], met[2];
    __shared__ unsigned long long keys[2][kRowWarps];
    __shared__ float2 sums[2][kRowWarps];
    __shared__ float4 blocks_sum[2][kRowMostBlocks];                   // written by the cluster's blocks: key (two halves), reference, sum
    Wd *words = reinterpret_cast<Wd *>(smem + g.words_at);             // of a chunk's tokens, of 8 in front of the row's vectors, 8 behind
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank();
    const bool pick = g.token || g.lse, sum = g.lse != nullptr;
    const long long first_row = blockIdx.x / g.blocks, row_step = gridDim.x / g.blocks;
    if (tid == 0) {
        for (int s = 0; s < kRowStages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), kRowWarps);
        }
        mbar_init(smem_u32(&met[0]), 1);
        mbar_init(smem_u32(&met[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cluster_sync();
    behind_the_last();
    // Every wait is bounded; once one has given up the others are passed over, and all roles still run to their ends.
    bool ok = true;
    auto wait = [&](unsigned long long &bar, uint32_t parity) {
        if (ok && !mbar_wait_bounded(smem_u32(&bar), parity)) {
            ok = false;
            report_status(g.status, FPSK_ERR_TIMEOUT);
        }
    };
    // a row's mask (NULL: none), and whether the one that it asks for is missing
    auto mask_of = [&](long long row, bool &missing) -> const int * {
        missing = false;
        if (!g.mask) return nullptr;
        const long long m = g.mask_row ? (long long)g.mask_row[row] : row;
        missing = m >= g.n_masks;
        return m >= 0 && !missing ? g.mask + m * g.mask_stride : nullptr;
    };

    if (warp == kRowWarps) {
        // ------------------------------------------------------------ copies
        unsigned int k = 0;                                            // pieces so far
        int stage = 0;
        uint32_t phase = 0;
        for (long long row = first_row; row < g.rows && !g.in_place; row += row_step) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            const Share<X> sl(x, g.vocab, g.log_blocks, rank);
            bool missing;
            const int *mask = mask_of(row, missing);
            const char *from = reinterpret_cast<const char *>(x + sl.a);
            for (int own = 0; own < sl.mine; own += kRowPieceVecs) {
                const int vecs = min(kRowPieceVecs, sl.mine - own), v = sl.vec(own);
                bool needed = !missing;
                if (mask) {
                    const int w0 = (sl.a + v * N) >> 5, w1 = (sl.a + (v + vecs) * N - 1) >> 5;
                    unsigned int any = 0;
                    for (int w = w0 + lane; w <= w1; w += 32) any |= (unsigned int)mask[w];
                    needed = __any_sync(0xFFFFFFFFu, any != 0);
                }
                if (lane == 0) {
                    wait(empty[stage], phase ^ 1u);
                    const uint32_t bar = smem_u32(&full[stage]);
                    if (ok && needed) {
                        mbar_expect_tx(bar, 16u * (uint32_t)vecs);
                        bulk_g2s(smem_u32(smem) + stage * kRowPiece, from + 16LL * v, 16u * (uint32_t)vecs, bar);
                    } else {
                        mbar_arrive(bar);
                    }
                }
                ++k;
                if (++stage == kRowStages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        let_the_next();
        // no copy is left in flight
        if (lane == 0)
            for (unsigned int back = min(k, (unsigned int)kRowStages); back; --back) {
                const unsigned int piece = k - back;
                mbar_wait_bounded(smem_u32(&full[piece % kRowStages]), piece / kRowStages & 1u);
            }
    } else {
        unsigned int n_rows = 0;
        int stage = 0;
        uint32_t phase = 0;
        const int chunk_tokens = g.chunk * N;
        for (long long row = first_row; row < g.rows; row += row_step, ++n_rows) {
            const X *x = static_cast<const X *>(g.x) + row * g.xs;
            Out *out = OUT ? static_cast<Out *>(g.out) + row * g.os : nullptr;
            const Share<X> sl(x, g.vocab, g.log_blocks, rank);
            const bool wide = OUT && reinterpret_cast<uintptr_t>(out + sl.a) % (N * sizeof(Out) < 16 ? N * sizeof(Out) : 16) == 0;
            const int buf = n_rows & 1;

            // the row's parameters, asked for together; the history's first tokens before their number is known
            const int *history = WORDS && g.history ? g.history + row * g.history_stride : nullptr;
            constexpr int kEarly = 4;
            int early[kEarly];
            auto first_of_history = [&] {
#pragma unroll
                for (int i = 0; i < kEarly; ++i) early[i] = history && tid + i * kRowWorkers < g.history_width ? history[tid + i * kRowWorkers] : -1;
            };
            first_of_history();
            int n_hist = history ? g.history_width : 0, n_prompt = 0;
            if (history && g.history_len) n_hist = max(0, min(n_hist, g.history_len[row]));
            if (history && g.prompt_len) n_prompt = g.prompt_len[row];
            const float rep = WORDS && g.rep ? g.rep[row] : 1.f, freq = WORDS && g.freq ? g.freq[row] : 0.f, pres = WORDS && g.pres ? g.pres[row] : 0.f;
            long long b0 = 0, b1 = 0;
            if (WORDS && g.bias_ptr) {
                b0 = max(0LL, (long long)g.bias_ptr[row]);
                b1 = min(g.n_biases, (long long)g.bias_ptr[row + 1]);
            }
            // the first biases and their logits as well
            int bias_v = -1;
            float bias_b = 0.f, bias_l = 0.f;
            if (WORDS && b0 + tid < b1) {
                bias_v = g.bias_token[b0 + tid];
                bias_b = g.bias_value[b0 + tid];
                if (sl.own_of(bias_v) >= 0) bias_l = Elem<X>::to_f(x[bias_v]);
            }
            bool nothing;
            const int *mask = mask_of(row, nothing);
            if (nothing && tid == 0) report_status(g.status, FPSK_ERR_PARAM);
            const bool masks = mask || nothing;
            auto allowed = [&](int e) { return nothing ? 0u : mask ? mask_bits<N>(mask, e) : kAll; };
            // z of a token, all but its biases and the mask; c: its word.  (By one over the repetition: a unit at most from the quotient.)
            const float inv_rep = 1.f / rep;
            auto adjusted = [&](float z, unsigned int c) {
                const float less = __fadd_rn(__fmul_rn((float)(c & F::kTimes), freq), pres);
                if (c & (F::kInPrompt | F::kTimes)) z = __fmul_rn(z, z > 0.f ? inv_rep : rep);
                return c & F::kTimes ? __fsub_rn(z, less) : z;
            };

            Picked p = {-INFINITY, kNoReference, 0.f, -1};
            Single own = {-INFINITY, kNoReference, 0.f, -1};
            auto single = [&](int v, float z) {
                if (masks && (nothing || !(mask[v >> 5] >> (v & 31) & 1))) z = -INFINITY;
                if (OUT) out[v] = Elem<Out>::from_f(z);
                if (pick) own.add(z, v, sum);
            };
            for (int c0 = 0; c0 < sl.mine || c0 == 0; c0 += g.chunk) {
                const int c1 = min(sl.mine, c0 + g.chunk);             // the chunk's vectors
                // The elements in front of the row's first vector and behind its last go with the first chunk of the first and the last block.
                const bool front = c0 == 0 && rank == 0, back = c0 == 0 && rank == g.blocks - 1;
                int loose = -1;
                if (warp == 0 && front && lane < sl.a) loose = lane;
                if (warp == 0 && back && lane >= 16 && sl.tail + lane - 16 < g.vocab) loose = sl.tail + lane - 16;
                // a token's word of this chunk, or -1
                const bool edges = sl.a > 0 || sl.tail < g.vocab;
                auto slot = [&](int v) {
                    const int own = sl.own_of(v);
                    if (own >= c0 * N && own < c1 * N) return own - c0 * N;
                    if (!edges) return -1;
                    if (front && v >= 0 && v < sl.a) return chunk_tokens + v;
                    if (back && v >= sl.tail && v < g.vocab) return chunk_tokens + 8 + v - sl.tail;
                    return -1;
                };
                if (WORDS) {
                    bar_sync(1, kRowWorkers);                          // the chunk in front is done with
                    if (c0) first_of_history();
                    for (int i = tid; i < (chunk_tokens + 16) * (int)sizeof(Wd) / 16; i += kRowWorkers) reinterpret_cast<uint4 *>(words)[i] = make_uint4(0u, 0u, 0u, 0u);
                    bar_sync(1, kRowWorkers);
                    auto count = [&](int i, int v) {
                        const int at = slot(v);
                        if (at < 0) return;
                        if (i < n_prompt) F::mark(words, at, F::kInPrompt);
                        else F::count(words, at);
                    };
                    for (int i0 = tid; i0 < n_hist; i0 += kEarly * kRowWorkers) {
                        int now[kEarly];
#pragma unroll
                        for (int i = 0; i < kEarly; ++i) {             // the next ones set out before these are counted
                            const int next = i0 + (kEarly + i) * kRowWorkers;
                            now[i] = early[i];
                            early[i] = next < n_hist ? history[next] : -1;
                        }
#pragma unroll
                        for (int i = 0; i < kEarly; ++i)
                            if (i0 + i * kRowWorkers < n_hist && now[i] >= 0) count(i0 + i * kRowWorkers, now[i]);
                    }
                    for (long long i = b0 + tid; i < b1; i += kRowWorkers) {
                        const int at = slot(i == b0 + tid ? bias_v : g.bias_token[i]);
                        if (at >= 0 && F::mark(words, at, F::kBiased) & F::kBiased) F::mark(words, at, F::kBiasedTwice);
                    }
                    bar_sync(1, kRowWorkers);
                }
                // A vector's touched tokens; which of them have biases and wait for those.
                auto adjust = [&](float2 (&z)[N / 2], int own_vec) {
                    const Wd *w = words + (own_vec - c0) * N;
                    unsigned int biased = 0;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const unsigned int c = w[j];
                        float &y = j & 1 ? z[j / 2].y : z[j / 2].x;
                        if (c & F::kBiased) biased |= 1u << j;
                        else y = adjusted(y, c);
                    }
                    return biased;
                };
                if (g.in_place) {
                    for (int v0 = c0; v0 < c1; v0 += kRowWorkers) {
                        const int v = v0 + tid, e = sl.token(v0 * N) + tid * N;
                        const bool here = v < c1;
                        const bool some = WORDS && here && F::template any<N>(words, (v - c0) * N);
                        const unsigned int bits = here ? allowed(e) : kAll;
                        if (OUT && (some || bits != kAll)) {
                            float2 z[N / 2];
                            Vec<X>::open(*reinterpret_cast<const uint4 *>(x + e), z);
                            if (WORDS && some) adjust(z, v);
#pragma unroll
                            for (int j = 0; j < N; ++j)
                                if (!(bits >> j & 1u)) (j & 1 ? z[j / 2].y : z[j / 2].x) = -INFINITY;
                            store_vec<Out, N>(out + e, wide, z);
                        }
                    }
                } else {
                    for (int v0 = c0; v0 < c1; v0 += kRowPieceVecs) {
                        wait(full[stage], phase);
                        const uint4 *piece = reinterpret_cast<const uint4 *>(smem + stage * kRowPiece) + tid;
                        const int v = v0 + tid, e = sl.token(v0 * N) + tid * N;
                        float2 z[kEachVecs][N / 2];
                        if (v0 + kRowPieceVecs <= c1 && !WORDS && !masks) {
#pragma unroll
                            for (int k = 0; k < kEachVecs; ++k) {
                                Vec<X>::open(piece[k * kRowWorkers], z[k]);
                                if (OUT) store_vec<Out, N>(out + e + k * kRowWorkers * N, wide, z[k]);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < kEachVecs; ++k) {
                                const int vk = v + k * kRowWorkers, ek = e + k * kRowWorkers * N;
                                const bool here = vk < c1;
                                Vec<X>::open(piece[k * kRowWorkers], z[k]);
                                unsigned int biased = 0;
                                if (WORDS && here && F::template any<N>(words, (vk - c0) * N)) biased = adjust(z[k], vk);
                                const unsigned int bits = !here ? 0u : masks ? allowed(ek) : kAll;
                                if (bits != kAll) {
#pragma unroll
                                    for (int j = 0; j < N; ++j)
                                        if (!(bits >> j & 1u)) (j & 1 ? z[k][j / 2].y : z[k][j / 2].x) = -INFINITY;
                                }
                                // (biased tokens as they are: their turn comes)
                                if (OUT && here) store_vec<Out, N>(out + ek, wide, z[k]);
                                if (WORDS && pick && biased) {
#pragma unroll
                                    for (int j = 0; j < N; ++j)
                                        if (biased >> j & 1u) (j & 1 ? z[k][j / 2].y : z[k][j / 2].x) = -INFINITY;
                                }
                            }
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                        if (++stage == kRowStages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                        if (pick) p.add<kEachVecs, N>(z, e, kRowWorkers * N, sum);
                    }
                }
                if (WORDS && b0 < b1) {
                    bar_sync(1, kRowWorkers);                          // (the stream has stored them as they were)
                    for (long long i = b0 + tid; i < b1; i += kRowWorkers) {
                        const bool known = i == b0 + tid;
                        const int v = known ? bias_v : g.bias_token[i], where = slot(v);
                        if (where < 0) continue;
                        float b = known ? bias_b : g.bias_value[i];
                        if (words[where] & F::kBiasedTwice) {          // the first of its entries does it, in the list's order
                            bool mine_to_do = true;
                            for (long long k = b0; k < i && mine_to_do; ++k) mine_to_do = g.bias_token[k] != v;
                            if (!mine_to_do) continue;
                            for (long long k = i + 1; k < b1; ++k)
                                if (g.bias_token[k] == v) b += g.bias_value[k];
                        }
                        single(v, adjusted(known && where < chunk_tokens ? bias_l : Elem<X>::to_f(x[v]), words[where]) + b);
                    }
                }
                if (loose >= 0) {
                    const unsigned int c = WORDS ? words[slot(loose)] : 0u;
                    if (!(c & F::kBiased)) single(loose, adjusted(Elem<X>::to_f(x[loose]), c));
                }
            }
            if (!pick) continue;
            unsigned long long key = max(p.at < 0 ? 0ull : pick_key(p.best, p.at), own.at < 0 ? 0ull : pick_key(own.best, own.at));
#pragma unroll
            for (int o = 16; o; o >>= 1) key = max(key, __shfl_xor_sync(0xFFFFFFFFu, key, o));
            const float top = fmaxf(p.m, own.m);
            RefSum r = join_lanes<32>(RefSum{top, p.s * exp2_fast((p.m - top) * kLog2e) + own.s * exp2_fast((own.m - top) * kLog2e)}, kLog2e);
            if (lane == 0) {
                keys[buf][warp] = key;
                sums[buf][warp] = make_float2(r.m, r.s);
            }
            bar_sync(1, kRowWorkers);
            if (warp == 0) {
                const float2 t = sums[buf][lane % kRowWarps];
                r = join_lanes<kRowWarps>(RefSum{t.x, t.y}, kLog2e);
                key = keys[buf][lane % kRowWarps];
#pragma unroll
                for (int o = kRowWarps / 2; o; o >>= 1) key = max(key, __shfl_xor_sync(0xFFFFFFFFu, key, o));
                if (g.blocks > 1) {
                    // (all hear of all, so that none is two rows ahead of another)
                    if (lane == 0) mbar_expect_tx(smem_u32(&met[buf]), 16u * g.blocks);
                    if (lane < g.blocks) {
                        asm volatile(
                            "{\n\t.reg .b32 a, m;\n\t"
                            "mapa.shared::cluster.u32 a, %0, %2;\n\t"
                            "mapa.shared::cluster.u32 m, %1, %2;\n\t"
                            "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %6}, [m];\n\t}"
                            ::"r"(smem_u32(&blocks_sum[buf][rank])), "r"(smem_u32(&met[buf])), "r"(lane), "f"(__uint_as_float((unsigned int)(key >> 32))),
                            "f"(__uint_as_float((unsigned int)key)), "f"(r.m), "f"(r.s)
                            : "memory");
                    }
                    wait(met[buf], n_rows >> 1 & 1u);
                    const float4 theirs = lane < g.blocks ? blocks_sum[buf][lane] : make_float4(0.f, 0.f, kNoReference, 0.f);
                    key = (unsigned long long)__float_as_uint(theirs.x) << 32 | __float_as_uint(theirs.y);
                    r = join_lanes<kRowMostBlocks>(RefSum{theirs.z, theirs.w}, kLog2e);
#pragma unroll
                    for (int o = kRowMostBlocks / 2; o; o >>= 1) key = max(key, __shfl_xor_sync(0xFFFFFFFFu, key, o));
                }
                if (rank == 0 && lane == 0) {
                    const unsigned int k = (unsigned int)(key >> 32);
                    if (g.token) g.token[row] = k <= kKeyNothing ? -1 : (int)(0xFFFFFFFFu - (unsigned int)key);
                    if (g.lse) g.lse[row] = k == kKeyNan ? __uint_as_float(0x7FC00000u) : k == kKeyInfinity ? INFINITY : r.m + logf(r.s);
                }
            }
        }
    }
    __syncthreads();
    cluster_sync();                                                    // no block leaves before what the others send it
}

template <typename X, typename O, typename W> static fpsk_status launch_logits(LogitsArgs g, cudaStream_t st)
{
    constexpr int N = Vec<X>::n;
    constexpr bool WORDS = !std::is_void<W>::value;
    using Wd = typename std::conditional<WORDS, W, char>::type;
    const int chunk_tokens = WORDS ? kWordBytes / (int)sizeof(Wd) : kMostChunk;
    // Blocks of a row: as many as make shares of one chunk, and more, down to 4096 tokens each, where there are too few rows for the SMs.
    g.blocks = 1;
    while (g.blocks < kRowMostBlocks && ((WORDS && g.vocab > g.blocks * chunk_tokens) || (g.rows * g.blocks < 3 * kSms && g.vocab > g.blocks * 4096))) {
        g.blocks *= 2;
        ++g.log_blocks;
    }
    const int vecs = (g.vocab + N - 1) / N, pieces = ((vecs + kRowPieceVecs - 1) / kRowPieceVecs + g.blocks - 1) / g.blocks;
    g.chunk = (pieces < chunk_tokens / N / kRowPieceVecs ? pieces : chunk_tokens / N / kRowPieceVecs) * kRowPieceVecs;
    g.words_at = g.in_place ? 0 : Workers<WORDS>::stages * kRowPiece;
    auto kernel = adjust_logits_kernel<X, O, W>;
    Launch launch((unsigned)g.blocks, Workers<WORDS>::threads, (size_t)g.words_at + (WORDS ? (g.chunk * N + 16) * sizeof(Wd) : 0), g.blocks, st);
    int most = 1;
    FPSK_CUDA_OK(clusters_at_once(reinterpret_cast<const void *>(kernel), launch.cfg, &most));
    launch.cfg.gridDim = dim3((unsigned)((g.rows < most ? g.rows : most) * g.blocks));
    FPSK_CUDA_OK(cudaLaunchKernelEx(&launch.cfg, kernel, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}
template <typename X> static fpsk_status launch_logits_typed(const LogitsArgs &g, int out_type, cudaStream_t st)
{
    // (16 bits: three of them flags.  96 rows of 131072 with histories of 4096 take 43 us with them and 52 with 32, 640 of 50257 93 and 140)
    const bool words = g.history || g.bias_ptr, narrow = !g.history || g.history_width < (int)Word<uint16_t>::kBiasedTwice;
#define FPSK_OUT(O) (!words ? launch_logits<X, O, void>(g, st) : narrow ? launch_logits<X, O, uint16_t>(g, st) : launch_logits<X, O, uint32_t>(g, st))
    if (!g.out) return FPSK_OUT(void);
    if (out_type == FPSK_ELEM_FP32) return FPSK_OUT(float);
    if (out_type == FPSK_ELEM_FP16) return FPSK_OUT(__half);
    return FPSK_OUT(__nv_bfloat16);
#undef FPSK_OUT
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
    if (!aligned(a->logits, a->logits_type) || (a->out && !aligned(a->out, a->out_type))) return FPSK_ERR_ALIGN;
    const void *values[] = {a->history, a->history_len, a->prompt_len, a->repetition, a->frequency, a->presence, a->bias_ptr, a->bias_token, a->bias_value,
                           a->mask, a->mask_row, a->token, a->lse};
    for (const void *p : values)
        if (!aligned(p, FPSK_ELEM_FP32)) return FPSK_ERR_ALIGN;
    if (a->history && (a->history_width < 0 || a->history_width > FPSK_MAX_HISTORY || a->history_stride < 0)) return FPSK_ERR_SHAPE;
    if (!a->history && (a->history_len || a->prompt_len || a->repetition || a->frequency || a->presence)) return FPSK_ERR_NULL;
    if (a->bias_ptr && (a->n_biases < 0 || (a->n_biases > 0 && (!a->bias_token || !a->bias_value)))) return FPSK_ERR_NULL;
    if (a->mask && (a->n_masks < 0 || a->mask_stride < 0 || (!a->mask_row && a->n_masks < a->n_rows))) return FPSK_ERR_SHAPE;
    if (!a->mask && a->mask_row) return FPSK_ERR_NULL;
    LogitsArgs g = {};
    g.x = a->logits; g.out = a->out; g.xs = a->logits_stride; g.os = a->out_stride; g.rows = a->n_rows;
    g.vocab = a->vocab;
    g.history = a->history; g.history_len = a->history_len; g.prompt_len = a->prompt_len;
    g.history_stride = a->history_stride; g.history_width = a->history_width;
    g.rep = a->repetition; g.freq = a->frequency; g.pres = a->presence;
    g.bias_ptr = a->n_biases > 0 ? a->bias_ptr : nullptr; g.bias_token = a->bias_token; g.bias_value = a->bias_value; g.n_biases = a->n_biases;
    g.mask = a->mask; g.mask_row = a->mask_row; g.mask_stride = a->mask_stride; g.n_masks = a->n_masks;
    g.token = a->token; g.lse = a->lse; g.status = d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    g.in_place = a->out == a->logits && a->out_type == a->logits_type && (a->n_rows == 1 || a->out_stride == a->logits_stride) && !g.token && !g.lse;
    if (a->logits_type == FPSK_ELEM_FP32) return launch_logits_typed<float>(g, a->out_type, st);
    if (a->logits_type == FPSK_ELEM_FP16) return launch_logits_typed<__half>(g, a->out_type, st);
    return launch_logits_typed<__nv_bfloat16>(g, a->out_type, st);
}
