// Attention over a paged cache on the 5th-generation tensor cores.
//
//   S = Q K^T (tcgen05, operands in shared memory) -> softmax weights P in registers -> O += P V (P from TMEM)
//
// Rows.  The queries of the G heads that share a key head meet the same keys, so a tile of 128 rows holds 128 / G tokens
// times G heads, and every key and value is read once for all of them.
// Items.  The work on one key head of one sequence is cut into items of one query tile (SPLIT: the sequences have at most one
// tile of queries, as in decoding) or two (PAIR: prompts), and measured in tiles of 128 keys.  All items lie on one
// axis, (sequence, key head, query tile) ordered, which is cut into equal ranges, one per CTA: every SM gets the same
// number of key tiles whatever the lengths are.  An item that a cut divides leaves partial results (running maximum, sum and
// output, FP32) that a second, small kernel joins; all others are finished where they are computed.
// Two workers per CTA, a warpgroup each, a thread per row, with accumulators S and O of their own in TMEM.  In
// a PAIR item they hold different query tiles and share every key tile; in a SPLIT item they hold the same queries and take
// alternate key tiles, and meet at the item's end.  While one computes its softmax, the tensor cores work for the other.
// A loader warp brings Q tiles and the pages of K and V by TMA into a ring of tiles, 128-byte swizzled; one warp issues
// the MMAs.  Maximum: the reference maximum of a row follows the true one only when that has grown by more than 2^8 (P then
// stays below 256, exact enough in 16 bits whatever its size), so O in TMEM is rescaled rarely.
// Every wait is bounded: a role whose wait gave up stops waiting and issuing, walks through its loops, reports
// FPSK_ERR_TIMEOUT and the CTA frees its TMEM and leaves.
#include "attention.cuh"
#include "tc_ops.cuh"

#include <cuda.h>
#include <math.h>
#include <atomic>

namespace fpsk {

constexpr int kRowsPerTile = 128, kKeysPerTile = 128;
constexpr int kTcaThreads = 384;                 // warps 0-3 and 4-7: workers, 8: MMA issue, 9: loader
constexpr int kHalfBytes = 128 * 128;            // 128 rows of one 64-channel half of a tile
constexpr int kTcaMaxSeqs = 16384;
constexpr float kLazy = 8.f;                     // growth of the maximum (in powers of two) that O is not rescaled for

// 32 consecutive columns of this thread's accumulator row; the values are there when the statement ends
__device__ __forceinline__ void tm_ld32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        :
        "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
// 128 consecutive columns of this thread's accumulator row; the values are there when the statement ends
__device__ __forceinline__ void tm_ld128(uint32_t taddr, uint32_t (&v)[128])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x128.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, "
        "%38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, "
        "%60, %61, %62, %63, %64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, %76, %77, %78, %79, %80, %81, "
        "%82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95, %96, %97, %98, %99, %100, %101, %102, "
        "%103, %104, %105, %106, %107, %108, %109, %110, %111, %112, %113, %114, %115, %116, %117, %118, %119, %120, "
        "%121, %122, %123, %124, %125, %126, %127}, [%128];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        :
        "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]), "=r"(v[32]),
        "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]), "=r"(v[40]),
        "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]), "=r"(v[48]),
        "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]), "=r"(v[56]),
        "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63]), "=r"(v[64]),
        "=r"(v[65]), "=r"(v[66]), "=r"(v[67]), "=r"(v[68]), "=r"(v[69]), "=r"(v[70]), "=r"(v[71]), "=r"(v[72]),
        "=r"(v[73]), "=r"(v[74]), "=r"(v[75]), "=r"(v[76]), "=r"(v[77]), "=r"(v[78]), "=r"(v[79]), "=r"(v[80]),
        "=r"(v[81]), "=r"(v[82]), "=r"(v[83]), "=r"(v[84]), "=r"(v[85]), "=r"(v[86]), "=r"(v[87]), "=r"(v[88]),
        "=r"(v[89]), "=r"(v[90]), "=r"(v[91]), "=r"(v[92]), "=r"(v[93]), "=r"(v[94]), "=r"(v[95]), "=r"(v[96]),
        "=r"(v[97]), "=r"(v[98]), "=r"(v[99]), "=r"(v[100]), "=r"(v[101]), "=r"(v[102]), "=r"(v[103]), "=r"(v[104]),
        "=r"(v[105]), "=r"(v[106]), "=r"(v[107]), "=r"(v[108]), "=r"(v[109]), "=r"(v[110]), "=r"(v[111]),
        "=r"(v[112]), "=r"(v[113]), "=r"(v[114]), "=r"(v[115]), "=r"(v[116]), "=r"(v[117]), "=r"(v[118]),
        "=r"(v[119]), "=r"(v[120]), "=r"(v[121]), "=r"(v[122]), "=r"(v[123]), "=r"(v[124]), "=r"(v[125]),
        "=r"(v[126]), "=r"(v[127])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t taddr, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        :
        : "r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
        "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
        "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem desc], 16-bit operands
__device__ __forceinline__ void tc_mma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate)
        : "memory");
}
// operand descriptors of tiles with 128-byte rows, 128-byte swizzle: eight rows are 1024 bytes.  K-major (Q, K): the
// rows are M or N, the row's channels the inner dimension.  MN-major (V): the rows are the inner dimension (keys), the
// row's 64 channels one block of N, and the next block lies kHalfBytes further.
__device__ __forceinline__ uint64_t sw128_desc(uint32_t saddr, uint32_t lbo_bytes)
{
    return tc_smem_desc(saddr, lbo_bytes, 1024) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void named_bar_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---------------------------------------------------------------- items
struct TcaArgs {
    AttnArgs a;
    int tile_tokens;                   // tokens of a 128-row tile: 128 / group
    int box_rows;                      // keys of one TMA box: the largest power of two that divides a page, at most 128
    float *part_o;                     // [2 slots per CTA][rows][DP]
    float2 *part_ml;                   // [2 slots per CTA][rows]: maximum (powers of two), sum
    struct SplitRecord *records;       // [CTA]
};
// A divided item, written by its second CTA: what the joining kernel needs.
struct SplitRecord {
    int parts;                         // 0: none
    int first_cta, token0, n_tok, kvh;
    int pad[3];
};

struct Item {
    int token0, n_tok;                 // first token (packed axis), tokens of the item
    int p0, kv_len;                    // position of the first token
    int lo, hi;                        // keys that some token of the item may see
    int tile0, units;                  // first key tile, key tiles (at least 1: an item without keys writes its zeros)
};

__device__ __forceinline__ void seq_lengths(const AttnArgs &g, int b, int &cu, int &q_len, int &kv_len)
{
    const int c0 = __ldg(g.cu_q + b), c1 = __ldg(g.cu_q + b + 1);
    cu = min(max(c0, 0), g.n_tokens);
    q_len = max(min(c1, g.n_tokens) - cu, 0);
    kv_len = max(__ldg(g.kv_len + b), 0);
}
__device__ __forceinline__ Item make_item(const AttnArgs &g, int cu, int q_len, int kv_len, int qi, int item_tokens)
{
    Item it;
    const int t0 = qi * item_tokens;
    it.token0 = cu + t0;
    it.n_tok = min(q_len - t0, item_tokens);
    it.p0 = kv_len - q_len + t0;
    it.kv_len = kv_len;
    int skip;
    key_range(g, it.p0 + it.n_tok - 1, kv_len, skip, it.hi);
    key_range(g, max(it.p0, 0), kv_len, it.lo, skip);
    if (it.hi <= it.lo) it.lo = it.hi = 0;
    it.tile0 = it.lo / kKeysPerTile;
    it.units = max(1, (it.hi + kKeysPerTile - 1) / kKeysPerTile - it.tile0);
    return it;
}

// PAIR: the key tiles of [tile_a, tile_b) that worker w's own tokens may see, [a, b).
__device__ __forceinline__ void worker_tiles(const AttnArgs &g, const Item &it, int w, int tile_tokens, int tile_a, int tile_b, int &a, int &b)
{
    const int t0 = w * tile_tokens, n = min(it.n_tok - t0, tile_tokens);
    a = b = tile_a;
    if (n <= 0) return;
    int lo, hi, skip;
    key_range(g, it.p0 + t0 + n - 1, it.kv_len, skip, hi);
    key_range(g, max(it.p0 + t0, 0), it.kv_len, lo, skip);
    if (hi <= lo) return;
    a = max(tile_a, lo / kKeysPerTile);
    b = max(a, min(tile_b, (hi + kKeysPerTile - 1) / kKeysPerTile));
}

// Walks the items of a CTA's range; every role walks for itself.
struct Walk {
    int b, kvh, qi, n_items;
    int cu, q_len, kv_len;
    __device__ __forceinline__ void open(const AttnArgs &g, int item_tokens)
    {
        seq_lengths(g, b, cu, q_len, kv_len);
        n_items = (q_len + item_tokens - 1) / item_tokens;
    }
    __device__ __forceinline__ void next(const AttnArgs &g, int item_tokens)
    {
        if (++qi < n_items) return;
        qi = 0;
        if (++kvh < g.hk) return;
        kvh = 0;
        do {
            ++b;
            if (b >= g.n_seqs) { n_items = 0; return; }
            open(g, item_tokens);
        } while (n_items == 0);
    }
};

template <int DP, bool PAIR> struct Tca {
    static constexpr int kTile = kRowsPerTile * DP * 2;
    static constexpr int kHalves = DP / 64;
    static constexpr int kQTiles = PAIR ? 2 : 1;
    static constexpr int kSlots = DP == 128 ? (PAIR ? 5 : 6) : 8;
    static constexpr int kBars = (kQTiles + kSlots) * kTile;           // barriers, start state, SPLIT: row statistics
    static constexpr int kSmem = kBars + 3072;
    static constexpr int kRows = kQTiles * kRowsPerTile;               // of a partial result
};

struct TcaBars {                       // shared memory, after the tiles
    unsigned long long q_full, q_empty, done, s_full[2], p_ready[2], o_done[2], kv_full[8], kv_empty[8];
    uint32_t tmem;
    int b, kvh, qi, u, left;
    long long totals[kTcaThreads / 32];
};
static_assert(sizeof(TcaBars) <= 1024, "barriers fit before the row statistics");

template <typename T, int DP, bool PAIR>
__global__ void __launch_bounds__(kTcaThreads, 1)
attention_tc_kernel(const __grid_constant__ TcaArgs ga, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v)
{
    using Cfg = Tca<DP, PAIR>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const AttnArgs &g = ga.a;
    TcaBars *sh = reinterpret_cast<TcaBars *>(smem + Cfg::kBars);
    float2 *row_ml = reinterpret_cast<float2 *>(smem + Cfg::kBars + 1024);     // [2][128], SPLIT only
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + Cfg::kQTiles * Cfg::kTile;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tile_tokens = ga.tile_tokens, item_tokens = tile_tokens * Cfg::kQTiles;

    if (tid == 0) {
        mbar_init(smem_u32(&sh->q_full), 1);
        mbar_init(smem_u32(&sh->q_empty), 1);
        mbar_init(smem_u32(&sh->done), 1);
        for (int w = 0; w < 2; ++w) {
            mbar_init(smem_u32(&sh->s_full[w]), 1);
            mbar_init(smem_u32(&sh->p_ready[w]), 4);
            mbar_init(smem_u32(&sh->o_done[w]), 1);
        }
        for (int s = 0; s < Cfg::kSlots; ++s) {
            mbar_init(smem_u32(&sh->kv_full[s]), 1);
            mbar_init(smem_u32(&sh->kv_empty[s]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) {
        tc_alloc(smem_u32(&sh->tmem), 512);
        tc_relinquish();
    }

    // ---- this CTA's range: key tiles of every sequence (in the ring, before it is used), their total, the first item
    unsigned int *seq_units = reinterpret_cast<unsigned int *>(smem + Cfg::kQTiles * Cfg::kTile);
    long long mine = 0;
    for (int base = 0; base < g.n_seqs; base += kTcaThreads) {
        const int b = base + tid;
        int cu = 0, q_len = 0, kv_len = 0, n = 0;
        if (b < g.n_seqs) {
            seq_lengths(g, b, cu, q_len, kv_len);
            n = (q_len + item_tokens - 1) / item_tokens;
        }
        unsigned int units = 0;
        if (n <= 4)
            for (int i = 0; i < n; ++i) units += make_item(g, cu, q_len, kv_len, i, item_tokens).units;
        for (unsigned int many = __ballot_sync(0xFFFFFFFFu, n > 4); many; many &= many - 1) {
            const int src = __ffs(many) - 1;                           // long prompts: the whole warp
            const int ql = __shfl_sync(0xFFFFFFFFu, q_len, src), kl = __shfl_sync(0xFFFFFFFFu, kv_len, src);
            const int ni = __shfl_sync(0xFFFFFFFFu, n, src);
            unsigned int t = 0;
            for (int i = lane; i < ni; i += 32) t += make_item(g, 0, ql, kl, i, item_tokens).units;
            t = __reduce_add_sync(0xFFFFFFFFu, t);
            if (lane == src) units = t;
        }
        if (b < g.n_seqs) seq_units[b] = units;
        mine += units;
    }
    for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    if (lane == 0) sh->totals[warp] = mine;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    long long total = 0;
    for (int w = 0; w < kTcaThreads / 32; ++w) total += sh->totals[w];
    total *= g.hk;
    const long long per = (total + gridDim.x - 1) / gridDim.x, start = per * blockIdx.x;
    if (warp == 0) {
        if (lane == 0) sh->left = (int)(start < total ? (total - start < per ? total - start : per) : 0);
        long long before = 0;
        bool found = start >= total;
        for (int base = 0; base < g.n_seqs && !found; base += 32) {
            const long long u = base + lane < g.n_seqs ? (long long)seq_units[base + lane] * g.hk : 0;
            long long incl = u;
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned int hit = __ballot_sync(0xFFFFFFFFu, before + incl > start);
            if (hit) {
                const int src = __ffs(hit) - 1;
                const long long rest = start - before - __shfl_sync(0xFFFFFFFFu, incl - u, src);
                const int b = base + src, per_head = (int)seq_units[b];
                const int kvh = (int)(rest / per_head);
                int u_in = (int)(rest - (long long)kvh * per_head), qi = 0;
                int cu, q_len, kv_len;
                seq_lengths(g, b, cu, q_len, kv_len);
                const int n = (q_len + item_tokens - 1) / item_tokens;
                for (int i0 = 0; i0 < n; i0 += 32) {
                    const int un = i0 + lane < n ? make_item(g, cu, q_len, kv_len, i0 + lane, item_tokens).units : 0;
                    int in = un;
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xFFFFFFFFu, in, o);
                        if (lane >= o) in += x;
                    }
                    const unsigned int at = __ballot_sync(0xFFFFFFFFu, in > u_in);
                    if (at) {
                        const int s2 = __ffs(at) - 1;
                        qi = i0 + s2;
                        u_in -= __shfl_sync(0xFFFFFFFFu, in - un, s2);
                        break;
                    }
                    u_in -= __shfl_sync(0xFFFFFFFFu, in, 31);
                }
                if (lane == 0) { sh->b = b; sh->kvh = kvh; sh->qi = qi; sh->u = u_in; }
                found = true;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    __syncthreads();
    int left = sh->left, u = sh->u;
    Walk walk;
    walk.b = sh->b; walk.kvh = sh->kvh; walk.qi = sh->qi;
    if (left > 0) walk.open(g, item_tokens);
    bool ok = true;                    // of this role
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !mbar_wait_bounded(bar, parity)) ok = false;
        __syncwarp();                  // the tcgen05 instructions behind it want the warp together
    };

    if (tid == 0) {
        // the record of a divided item: written by the CTA behind its first
        SplitRecord r = {};
        if (left > 0 && u > 0) {
            const long long item0 = start - u;
            if (item0 >= start - per) {
                const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
                r.first_cta = blockIdx.x - 1;
                r.parts = (int)((item0 + it.units - 1) / per) - r.first_cta + 1;
                r.token0 = it.token0; r.n_tok = it.n_tok; r.kvh = walk.kvh;
            }
        }
        ga.records[blockIdx.x] = r;
    }

    if (warp == 9) {
        // ------------------------------------------------------------ loader
        fence_proxy_async();
        const int page_size = g.page_size, R = ga.box_rows;
        int slot = 0, fills = 0;
        uint32_t phase = 0, q_phase = 0;
        bool q_used = false;
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            const int n = min(left, it.units - u);
            if (it.hi > it.lo) {
                wait(smem_u32(&sh->q_empty), q_phase ^ 1u);
                if (ok && lane == 0) {
                    mbar_expect_tx(smem_u32(&sh->q_full), (uint32_t)(Cfg::kQTiles * Cfg::kHalves * tile_tokens * g.group * 128));
                    for (int w = 0; w < Cfg::kQTiles; ++w)
                        for (int h = 0; h < Cfg::kHalves; ++h)
                            tma_load_3d(q_smem + w * Cfg::kTile + h * kHalfBytes, &map_q, h * 64, walk.kvh * g.group, it.token0 + w * tile_tokens,
                                        smem_u32(&sh->q_full));
                }
                q_phase ^= 1u;
                q_used = true;
                const int *row = g.table + (long long)walk.b * g.table_stride;
                const int tile_a = it.tile0 + u, tile_b = tile_a + n;
                // a tile of K or V: its boxes that hold a visible key
                auto load = [&](int tile, const CUtensorMap *map) {
                    const int k0 = tile * kKeysPerTile;
                    const int r0 = max(0, it.lo - k0) / R, r1 = (min(kKeysPerTile, it.hi - k0) + R - 1) / R;
                    const uint32_t full = smem_u32(&sh->kv_full[slot]), dst = ring + slot * Cfg::kTile;
                    wait(smem_u32(&sh->kv_empty[slot]), phase ^ 1u);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) return;
                    if (lane == 0) mbar_expect_tx(full, (uint32_t)((r1 - r0) * R * 128 * Cfg::kHalves));
                    __syncwarp();
                    for (int i = lane; i < (r1 - r0) * Cfg::kHalves; i += 32) {
                        const int box = r0 + i / Cfg::kHalves, h = i % Cfg::kHalves;
                        const int key = k0 + box * R, col = key / page_size;
                        long long page = col < g.max_pages ? __ldg(row + col) : -1;
                        if (page < 0 || page >= g.n_pages) {
                            report_status(g.status, FPSK_ERR_PARAM);
                            page = g.n_pages;                          // outside the tensor map: zeros
                        }
                        tma_load_4d(dst + h * kHalfBytes + box * R * 128, map, h * 64, key - col * page_size, walk.kvh, (int)page, full);
                    }
                    ++fills;
                    if (++slot == Cfg::kSlots) { slot = 0; phase ^= 1u; }
                };
                if constexpr (PAIR) {
                    for (int t = tile_a; t < tile_b; ++t) {
                        load(t, &map_k);
                        load(t, &map_v);
                    }
                } else {
                    load(tile_a, &map_k);
                    if (n > 1) load(tile_a + 1, &map_k);
                    for (int t = tile_a; t < tile_b; ++t) {
                        load(t, &map_v);
                        if (t + 2 < tile_b) load(t + 2, &map_k);
                    }
                }
            }
            left -= n;
            u = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
        // own copies still in flight (only after a wait that gave up)
        const int own = min(fills, Cfg::kSlots);
        for (int i = 0; i < own; ++i) {
            if (--slot < 0) { slot = Cfg::kSlots - 1; phase ^= 1u; }
            if (!mbar_wait_bounded(smem_u32(&sh->kv_full[slot]), phase)) ok = false;
        }
        if (q_used && !mbar_wait_bounded(smem_u32(&sh->q_full), q_phase ^ 1u)) ok = false;
    } else if (warp == 8) {
        // ------------------------------------------------------------ MMA issue
        const uint32_t fmt = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t base_desc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(kRowsPerTile >> 4) << 24);
        const uint32_t idesc_s = base_desc | ((uint32_t)(kKeysPerTile >> 3) << 17);
        const uint32_t idesc_o = base_desc | (1u << 16) | ((uint32_t)(DP >> 3) << 17);
        int slot = 0;
        uint32_t phase = 0, q_phase = 0, p_phase[2] = {0, 0};
        auto next_slot = [&]() {
            if (++slot == Cfg::kSlots) { slot = 0; phase ^= 1u; }
        };
        auto issue_s = [&](int w, uint32_t k_addr) {
            if (ok && lane == 0) {
                const uint32_t qa = q_smem + (PAIR ? w * Cfg::kTile : 0);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = (k / 4) * kHalfBytes + (k % 4) * 32;
                    tc_mma(tmem + w * 128, sw128_desc(qa + off, 16), sw128_desc(k_addr + off, 16), idesc_s, k > 0);
                }
                tc_commit(smem_u32(&sh->s_full[w]));
            }
        };
        auto issue_o = [&](int w, uint32_t v_addr, bool accumulate) {
            wait(smem_u32(&sh->p_ready[w]), p_phase[w]);
            p_phase[w] ^= 1u;
            tc_fence_after();
            if (ok && lane == 0) {
#pragma unroll
                for (int k = 0; k < kKeysPerTile / 16; ++k)
                    tc_mma_ts(tmem + 256 + w * 128, tmem + w * 128 + k * 8, sw128_desc(v_addr + k * 2048, kHalfBytes), idesc_o,
                              accumulate || k > 0);
                tc_commit(smem_u32(&sh->o_done[w]));
            }
        };
        auto release = [&](int s) {
            if (ok && lane == 0) tc_commit(smem_u32(&sh->kv_empty[s]));
        };
        // rows of a V tile that no token of the item may see: zeros, for 0 * (what lies there) must not be NaN
        auto clean_v = [&](const Item &it, int tile, uint32_t v_addr) {
            const int k0 = tile * kKeysPerTile, r0 = max(0, it.lo - k0), r1 = min(kKeysPerTile, it.hi - k0);
            if (r0 == 0 && r1 == kKeysPerTile) return;
            for (int i = lane; i < kKeysPerTile * 8 * Cfg::kHalves; i += 32) {
                const int r = (i >> 3) & (kKeysPerTile - 1);
                if (r < r0 || r >= r1)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_addr + i * 16), "r"(0) : "memory");
            }
            fence_proxy_async();
            __syncwarp();
        };
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            const int n = min(left, it.units - u);
            if (it.hi > it.lo) {
                const int tile_a = it.tile0 + u, tile_b = tile_a + n;
                wait(smem_u32(&sh->q_full), q_phase);
                q_phase ^= 1u;
                auto wait_full = [&]() {
                    wait(smem_u32(&sh->kv_full[slot]), phase);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    tc_fence_after();
                };
                if constexpr (PAIR) {
                    int wa[2], wb[2];
                    for (int w = 0; w < 2; ++w) worker_tiles(g, it, w, tile_tokens, tile_a, tile_b, wa[w], wb[w]);
                    wait_full();
                    for (int w = 0; w < 2; ++w)
                        if (tile_a >= wa[w] && tile_a < wb[w]) issue_s(w, ring + slot * Cfg::kTile);
                    release(slot);
                    next_slot();
                    for (int t = tile_a; t < tile_b; ++t) {
                        const int v_slot = slot;
                        wait_full();
                        next_slot();
                        const uint32_t v_addr = ring + v_slot * Cfg::kTile;
                        if (ok) clean_v(it, t, v_addr);
                        if (t + 1 < tile_b) wait_full();
                        for (int w = 0; w < 2; ++w) {
                            if (t >= wa[w] && t < wb[w]) issue_o(w, v_addr, t > wa[w]);
                            if (t + 1 >= wa[w] && t + 1 < wb[w]) issue_s(w, ring + slot * Cfg::kTile);
                        }
                        release(v_slot);
                        if (t + 1 < tile_b) {
                            release(slot);
                            next_slot();
                        }
                    }
                } else {
                    for (int i = 0; i < 2 && i < n; ++i) {
                        wait_full();
                        issue_s(i, ring + slot * Cfg::kTile);
                        release(slot);
                        next_slot();
                    }
                    for (int i = 0; i < n; ++i) {
                        wait_full();
                        const uint32_t v_addr = ring + slot * Cfg::kTile;
                        if (ok) clean_v(it, tile_a + i, v_addr);
                        issue_o(i & 1, v_addr, i > 1);
                        release(slot);
                        next_slot();
                        if (i + 2 < n) {
                            wait_full();
                            issue_s(i & 1, ring + slot * Cfg::kTile);
                            release(slot);
                            next_slot();
                        }
                    }
                }
                if (ok && lane == 0) tc_commit(smem_u32(&sh->q_empty));
            }
            left -= n;
            u = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
        if (lane == 0) {
            tc_commit(smem_u32(&sh->done));
            if (!mbar_wait_bounded(smem_u32(&sh->done), 0)) ok = false;
        }
        __syncwarp();
    } else if (warp < 8) {
        // ------------------------------------------------------------ workers: a thread per row
        const int w = warp >> 2, rloc = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + lanes + w * 128, to = tmem + lanes + 256 + w * 128;
        const int tok_in_tile = rloc / g.group, head_in_group = rloc - tok_in_tile * g.group;
        const float sl2 = g.scale_log2;
        uint32_t s_phase = 0, o_count = 0;
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            const int n = min(left, it.units - u);
            const int t_in_item = (PAIR ? w * tile_tokens : 0) + tok_in_tile;
            const bool valid = tok_in_tile < tile_tokens && t_in_item < it.n_tok;
            const bool warp_on = __any_sync(0xFFFFFFFFu, valid);
            int lo = 0, hi = 0x7FFFFFFF;                               // rows without a token compute what nobody reads
            if (valid) key_range(g, it.p0 + t_in_item, it.kv_len, lo, hi);
            int ta = 0, tb = 0, step = 1;
            if (it.hi > it.lo) {
                const int tile_a = it.tile0 + u, tile_b = tile_a + n;
                if constexpr (PAIR) worker_tiles(g, it, w, tile_tokens, tile_a, tile_b, ta, tb);
                else { ta = tile_a + w; tb = tile_b; step = 2; }
            }
            float m = -INFINITY, l = 0.f;
            bool have_o = false;
            for (int t = ta; t < tb; t += step) {
                wait(smem_u32(&sh->s_full[w]), s_phase);
                s_phase ^= 1u;
                tc_fence_after();
                if (warp_on) {
                    uint32_t s[128];
                    tm_ld128(ts, s);
                    const int k0 = t * kKeysPerTile;
                    if (__any_sync(0xFFFFFFFFu, k0 < lo || k0 + kKeysPerTile > hi)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (k0 + i < lo || k0 + i >= hi) s[i] = 0xFF800000u;
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 128; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(s[i]));
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
                    if (!have_o) {
                        m = top;
                    } else {
                        const bool grow = valid && top > m + kLazy;
                        if (__any_sync(0xFFFFFFFFu, grow)) {
                            const float alpha = grow ? ex2(m - top) : 1.f;
                            if (grow) m = top;
                            l *= alpha;
                            wait(smem_u32(&sh->o_done[w]), (o_count - 1u) & 1u);
                            tc_fence_after();
#pragma unroll
                            for (int c = 0; c < DP / 32; ++c) {
                                uint32_t o[32];
                                tm_ld32(to + c * 32, o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tm_st32(to + c * 32, o);
                            }
                            tm_wait_st();
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    const float2 sc = make_float2(sl2, sl2), nb = make_float2(-base, -base);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t p[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float2 x = make_float2(__uint_as_float(s[64 * h + 2 * i]), __uint_as_float(s[64 * h + 2 * i + 1]));
                            x = __ffma2_rn(x, sc, nb);
                            x = make_float2(ex2(x.x), ex2(x.y));
                            sum[i & 1] = __fadd2_rn(sum[i & 1], x);
                            p[i] = pack_pair<T>(x.x, x.y);
                        }
                        tm_st32(ts + 32 * h, p);
                    }
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    tm_wait_st();
                }
                have_o = true;
                ++o_count;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[w]));
            }
            if (have_o) {
                wait(smem_u32(&sh->o_done[w]), (o_count - 1u) & 1u);
                tc_fence_after();
            }
            // ---- the item's end: finished here, or a partial result
            const bool whole = u == 0 && n == it.units;
            float wt0 = 1.f, wt1 = 0.f;                               // SPLIT: weights of the two workers' outputs
            bool have1 = false;
            if constexpr (!PAIR) {
                row_ml[w * 128 + rloc] = make_float2(m, l);
                tc_fence_before();
                named_bar_sync(1, 256);                               // both outputs are complete
                tc_fence_after();
                const float2 a = row_ml[rloc], b = row_ml[128 + rloc];
                have1 = n > 1 && it.hi > it.lo;
                m = fmaxf(a.x, b.x);
                const float base = m == -INFINITY ? 0.f : m;
                wt0 = ex2(a.x - base);
                wt1 = ex2(b.x - base);
                l = a.y * wt0 + b.y * wt1;
            }
            const bool have0 = PAIR ? have_o : it.hi > it.lo;
            if (warp_on) {
                const int row = (PAIR ? w * 128 : 0) + rloc;
                const int pslot = 2 * blockIdx.x + (u == 0 ? 1 : 0);
                const float inv = l != 0.f ? 1.f / l : 0.f;
                const long long head = walk.kvh * g.group + head_in_group;
                T *dst = static_cast<T *>(g.out) + (long long)(it.token0 + t_in_item) * g.ots + head * g.ohs;
                float *pdst = ga.part_o + ((long long)pslot * Cfg::kRows + row) * DP;
                if (valid && (PAIR || w == 0)) {
                    if (whole) {
                        if (g.lse)
                            g.lse[(long long)(it.token0 + t_in_item) * g.hq + head] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                    } else {
                        ga.part_ml[(long long)pslot * Cfg::kRows + row] = make_float2(m, l);
                    }
                }
                // SPLIT: each worker brings one half of the channels of both outputs
                const int c0 = PAIR ? 0 : w * (DP / 64), c1 = PAIR ? DP / 32 : c0 + DP / 64;
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    if (c < c0 || c >= c1) continue;
                    float o[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
                    const uint32_t tc = tmem + lanes + 256 + (PAIR ? w * 128 : 0) + c * 32;
                    if (have0) {
                        uint32_t x[32];
                        tm_ld32(tc, x);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(x[i]) * wt0;
                    }
                    if (!PAIR && have1) {
                        uint32_t x[32];
                        tm_ld32(tc + 128, x);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = fmaf(__uint_as_float(x[i]), wt1, o[i]);
                    }
                    if (!valid) {
                    } else if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            if (c * 32 + i < g.dim)
                                *reinterpret_cast<uint4 *>(dst + c * 32 + i) =
                                    make_uint4(pack_pair<T>(o[i] * inv, o[i + 1] * inv), pack_pair<T>(o[i + 2] * inv, o[i + 3] * inv),
                                               pack_pair<T>(o[i + 4] * inv, o[i + 5] * inv), pack_pair<T>(o[i + 6] * inv, o[i + 7] * inv));
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4 *>(pdst + c * 32 + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                    __syncwarp();
                }
                tc_fence_before();
            }
            if constexpr (!PAIR) named_bar_sync(2, 256);
            left -= n;
            u = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
    }
    if (!ok && lane == 0) report_status(g.status, FPSK_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tc_dealloc(tmem, 512);
}

// Joins the parts of the divided items: a warp per row, four channels per lane.
template <typename T, int DP, bool PAIR>
__global__ void __launch_bounds__(256) attention_join_kernel(const __grid_constant__ TcaArgs ga)
{
    constexpr int kRows = Tca<DP, PAIR>::kRows;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttnArgs &g = ga.a;
    const SplitRecord r = ga.records[blockIdx.x];
    if (r.parts == 0) return;
    const int lane = threadIdx.x & 31;
    for (int i = blockIdx.y * 8 + (threadIdx.x >> 5); i < r.n_tok * g.group; i += gridDim.y * 8) {
        const int t = i / g.group, h = i - t * g.group, w = t / ga.tile_tokens;
        const int row = w * 128 + (t - w * ga.tile_tokens) * g.group + h;
        auto at = [&](int part) { return (long long)(2 * (r.first_cta + part) + (part == 0 ? 1 : 0)) * kRows + row; };
        float m = -INFINITY;
        for (int p = lane; p < r.parts; p += 32) m = fmaxf(m, ga.part_ml[at(p)].x);
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = 0; p0 < r.parts; p0 += 32) {
            float wt = 0.f, lp = 0.f;
            if (p0 + lane < r.parts) {
                const float2 ml = ga.part_ml[at(p0 + lane)];
                wt = ex2(ml.x - base);
                lp = ml.y * wt;
            }
            for (int o = 16; o; o >>= 1) lp += __shfl_xor_sync(0xFFFFFFFFu, lp, o);
            l += lp;
            const int np = min(32, r.parts - p0);
            for (int p = 0; p < np; ++p) {
                const float x = __shfl_sync(0xFFFFFFFFu, wt, p);
                if (lane * 4 < DP) {
                    const float4 o = *reinterpret_cast<const float4 *>(ga.part_o + at(p0 + p) * DP + lane * 4);
                    acc = make_float4(fmaf(o.x, x, acc.x), fmaf(o.y, x, acc.y), fmaf(o.z, x, acc.z), fmaf(o.w, x, acc.w));
                }
            }
        }
        const float inv = l != 0.f ? 1.f / l : 0.f;
        const long long head = r.kvh * g.group + h, tok = r.token0 + t;
        if (lane * 4 < g.dim)
            *reinterpret_cast<uint2 *>(static_cast<T *>(g.out) + tok * g.ots + head * g.ohs + lane * 4) =
                make_uint2(pack_pair<T>(acc.x * inv, acc.y * inv), pack_pair<T>(acc.z * inv, acc.w * inv));
        if (g.lse && lane == 0) g.lse[tok * g.hq + head] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
}

// ---------------------------------------------------------------- host side
using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
static EncodeFn encode_fn()
{
    static const EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            return (EncodeFn) nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}
static bool encode(CUtensorMap *map, int type, int rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    static const cuuint32_t ones[4] = {1, 1, 1, 1};
    const EncodeFn fn = encode_fn();
    return fn && fn(map, type == FPSK_ELEM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                    const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_count()
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

constexpr int kMaxPartRows = 2 * kRowsPerTile, kMaxDP = 128;
size_t attention_tc_workspace_bytes()
{
    const size_t ctas = (size_t)sm_count();
    return align_up(ctas * sizeof(SplitRecord), 256) + 2 * ctas * kMaxPartRows * (kMaxDP * sizeof(float) + sizeof(float2));
}

static bool aligned16(const void *p, long long s0, long long s1, long long s2)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 % 8 == 0 && s1 % 8 == 0 && s2 % 8 == 0;
}
// What the tensor-core kernel takes: heads of up to 128 channels, at most 128 query heads to a key head, whole eight-row
// groups of a page, and 16-byte aligned rows (TMA).  The rest is the row kernel's.
bool attention_tc_takes(const AttnArgs &g)
{
    return g.dim <= 128 && g.group <= 128 && g.page_size % 8 == 0 && g.n_seqs <= kTcaMaxSeqs && aligned16(g.q, g.qts, g.qhs, 0) &&
           aligned16(g.out, g.ots, g.ohs, 0) && aligned16(g.k, g.kps, g.kts, g.khs) && aligned16(g.v, g.vps, g.vts, g.vhs);
}

template <typename T, int DP, bool PAIR> static fpsk_status launch_tc(const AttnArgs &a, int type, void *ws, cudaStream_t st)
{
    using Cfg = Tca<DP, PAIR>;
    const int ctas = sm_count();
    if (ctas < 1) return FPSK_ERR_CUDA;
    TcaArgs g;
    g.a = a;
    g.tile_tokens = kRowsPerTile / a.group;
    g.box_rows = a.page_size & -a.page_size;
    if (g.box_rows > kKeysPerTile) g.box_rows = kKeysPerTile;
    char *p = static_cast<char *>(ws);
    g.records = reinterpret_cast<SplitRecord *>(p);
    p += align_up((size_t)ctas * sizeof(SplitRecord), 256);
    g.part_o = reinterpret_cast<float *>(p);
    p += (size_t)2 * ctas * kMaxPartRows * kMaxDP * sizeof(float);
    g.part_ml = reinterpret_cast<float2 *>(p);
    // strides of dimensions of one element are never used, but the encoder wants them valid
    auto bytes = [](long long s, long long n) { return (cuuint64_t)(n > 1 && s > 0 ? s * 2 : 16); };
    CUtensorMap mq, mk, mv;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)a.dim, (cuuint64_t)a.hq, (cuuint64_t)a.n_tokens};
        const cuuint64_t str[2] = {bytes(a.qhs, a.hq), bytes(a.qts, a.n_tokens)};
        const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)g.tile_tokens};
        if (!encode(&mq, type, 3, a.q, dims, str, box)) return FPSK_ERR_CUDA;
    }
    const cuuint64_t dims[4] = {(cuuint64_t)a.dim, (cuuint64_t)a.page_size, (cuuint64_t)a.hk, (cuuint64_t)a.n_pages};
    const cuuint32_t box[4] = {64, (cuuint32_t)g.box_rows, 1, 1};
    const cuuint64_t ks[3] = {bytes(a.kts, a.page_size), bytes(a.khs, a.hk), bytes(a.kps, a.n_pages)};
    const cuuint64_t vs[3] = {bytes(a.vts, a.page_size), bytes(a.vhs, a.hk), bytes(a.vps, a.n_pages)};
    if (!encode(&mk, type, 4, a.k, dims, ks, box) || !encode(&mv, type, 4, a.v, dims, vs, box)) return FPSK_ERR_CUDA;

    static std::atomic<unsigned long long> prepared{0};               // one bit per device
    int dev = 0;
    FPSK_CUDA_OK(cudaGetDevice(&dev));
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(prepared.load(std::memory_order_acquire) & bit)) {
        FPSK_CUDA_OK(cudaFuncSetAttribute(attention_tc_kernel<T, DP, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem));
        prepared.fetch_or(bit, std::memory_order_release);
    }
    attention_tc_kernel<T, DP, PAIR><<<ctas, kTcaThreads, Cfg::kSmem, st>>>(g, mq, mk, mv);
    FPSK_LAUNCH_CHECK();
    // the join's launch overlaps the end of the kernel before it
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, PAIR ? 8 : 4);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, attention_join_kernel<T, DP, PAIR>, g));
    FPSK_LAUNCH_CHECK();
    return FPSK_OK;
}

// PAIR where a sequence may have more tokens than one tile holds.
fpsk_status attention_tc_launch(const AttnArgs &a, int type, int max_q_len, void *ws, cudaStream_t st)
{
    const bool pair = max_q_len > kRowsPerTile / a.group;
#define FPSK_TCA(TT)                                                                                                              \
    (a.dim <= 64 ? (pair ? launch_tc<TT, 64, true>(a, type, ws, st) : launch_tc<TT, 64, false>(a, type, ws, st))                  \
                 : (pair ? launch_tc<TT, 128, true>(a, type, ws, st) : launch_tc<TT, 128, false>(a, type, ws, st)))
    return type == FPSK_ELEM_FP16 ? FPSK_TCA(__half) : FPSK_TCA(__nv_bfloat16);
#undef FPSK_TCA
}

}  // namespace fpsk
