// Attention over a paged cache on the 5th-generation tensor cores.
//
//   S = Q K^T (tcgen05, operands in shared memory) -> softmax weights P in registers -> O += P V (P from TMEM)
//
// Rows.  The queries of the G heads that share a key head meet the same keys, so a tile of 128 rows holds 128 / G tokens
// times G heads, and every key and value is read once for all of them.
// Items.  The work on one key head of one sequence is cut into items of one query tile (SPLIT, COPIES: a few tokens, as in
// decoding) or two (PAIR: prompts), and measured in tiles of 128 keys.  All items lie on one axis, ordered by sequence, key head and query tile, which is cut into equal ranges, one per CTA: every SM gets the same
// number of key tiles whatever the lengths are.  An item that a cut divides leaves partial results (running maximum, sum and
// output, FP32), joined in the order of the parts; all others are finished where they are computed.  (COPIES, a few rows: joined in the
// launch by the CTA whose part comes last; the others by a second launch, for in the first its code would be cold: 78 against 59 us
// for windows.)
// Two workers per CTA, a warpgroup each, a thread per row, with accumulators S and O of their own in TMEM.  In
// a PAIR item they hold different query tiles and share every key tile; in a SPLIT item they hold the same queries and take
// alternate key tiles, and meet at the item's end.  While one computes its softmax, the tensor cores work for the other.
// Two loader warps bring Q and K tiles and V tiles, page by page, by TMA into a ring of tiles, 128-byte swizzled; a warp for
// each worker issues its MMAs.  Maximum: the reference of a row follows its maximum only when the weights of a step outgrow it (see
// Reference), so O in TMEM is rescaled rarely and most steps take no maximum at all.
// Roundings.  Weights meet the values as 16-bit numbers, which the tensor cores want: each is off by half a unit of the type at most,
// the sum that divides them is not rounded.  Sums, maxima and outputs are FP32 up to the one rounding at the end.
// What bounds it.  Many rows: the tensor cores and the exponentials, about equally.  A step of 64 keys takes a worker 1277 cycles (two
// warps on a scheduler; 1024 of them their exponentials, four lanes a cycle), the two workers' four products about 1150, where
// S = Q K^T is held up by shared memory (48 cycles for 128 x 64 x 16: 128 bytes a cycle; O += P V has P in TMEM and is not).
// Few rows: HBM, and the latency from the launch to the first scores (6 us), of which a short context is all.
// Measured, sustained: 4096 new tokens of 32 heads over 16384 keys of 8 heads of 128, 882 us (1.09 PFLOP/s, 0.66 of a library's large
// product); 4 tokens over 262144 keys 213 us (5.0 TB/s, 0.77 of a copy); 96 requests of one token, 98296 keys, 98 us (4.1 TB/s).
// In a burst of up to a hundred launches they take 850, 177 and 84 us: within some 0.1 s the load brings the chip to its power
// limit, and the SM clock from 1965 to 1590 - 1740 MHz.  The other times in this file, both sides of a choice, are of bursts.
// Every wait is bounded: a role whose wait gave up stops waiting and issuing, walks through its loops, reports
// FPSK_ERR_TIMEOUT and the CTA frees its TMEM and leaves.
#include "attention.cuh"
#include "tc_ops.cuh"

#include <cuda.h>
#include <math.h>
#include <atomic>

namespace fpsk {

constexpr int kRowsPerTile = 128, kKeysPerTile = 128;
constexpr int kPairKeys = 64;                    // keys of a PAIR worker's step: two S accumulators fit its TMEM columns
constexpr int kTcaThreads = 384;                 // warps 0-3 and 4-7: workers, 8 and 11: their MMAs, 9 and 10: loaders
constexpr int kHalfBytes = 128 * 128;            // 128 rows of one 64-channel half of a tile
constexpr int kTcaMaxSeqs = 16384;
// An item's beginning and end, in key tiles.  96 requests of uneven length take 84 us with 2, 91 with 1, 89 with 3; windows of 1000 keys
// 34, 35, 45; 64 requests of 8 tokens 72, 68, 78.
constexpr int kItemCost = 2;
// Weights are powers of two over a row's reference, which lies kBelow binary digits under its maximum when it is set, and is renewed
// when the sum of a step's weights passes kMost.  BF16 has the exponents of FP32: any reference will do.  FP16 rounds weights below
// 2^-14 to multiples of 2^-24, and a long tail of such weights counts (131071 keys at 2^-24.4 of a dominant one are 0.006 of
// it, and would be off by a third of that): with the reference eight digits down that is 2^-33 of the largest weight each, 2^-13 of it for 2^20 keys.
// 128 weights of 2^8 stay within kMost, so that equal scores take no maximum either, and no weight passes the largest FP16 number.
template <typename T> struct Reference {
    static constexpr float kBelow = 0.f, kMost = 4096.f;
};
template <> struct Reference<__half> {
    static constexpr float kBelow = 8.f, kMost = 60000.f;
};

// 32 consecutive columns of this thread's accumulator row; valid after tm_wait32 on the same array
__device__ __forceinline__ void tm_load32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        :
        "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
// all loads of this thread are complete (the array goes through, so that no use of it can move in front)
__device__ __forceinline__ void tm_wait32(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        :
        "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
        "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
        "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
        "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
        :
        : "memory");
}
__device__ __forceinline__ void tm_ld16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tm_ld32(uint32_t taddr, uint32_t (&v)[32])
{
    tm_load32(taddr, v);
    tm_wait32(v);
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
__device__ __forceinline__ void tm_st16(uint32_t taddr, const uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16};"
        :
        : "r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D[tmem] (+)= A * B, 16-bit operands, A in shared memory or in TMEM.  Descriptors come as low words (address, leading offset)
// next to one high word: with everything uniform over the warp the steps of a tile are additions in uniform registers, and
// a step takes a few cycles to issue instead of about a hundred.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
// a value that all lanes hold, told to the compiler
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
// Operand descriptors of tiles with 128-byte rows, 128-byte swizzle.  K-major (Q, K): the rows are M or N, the row's channels the
// inner dimension.  MN-major (V): the rows are the inner dimension (keys), the row's 64 channels one block of N.  Low word:
// address and the offset between blocks of 64 channels (MN-major); high word: the offset between groups of eight rows.
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t block_bytes) { return (saddr >> 4) | ((block_bytes >> 4) << 16); }
__device__ __forceinline__ uint32_t desc_hi(uint32_t group_bytes) { return (group_bytes >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, int v, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// Bounded wait on an mbarrier phase, without a call (a call's register conventions would spill the rows that the workers hold)
// and without the clock: the limit counts polls, each of which sleeps in hardware for a while.
constexpr int kMostPolls = 1 << 22;
__device__ __forceinline__ bool bar_wait_inline(uint32_t bar, uint32_t parity)
{
#pragma unroll 1
    for (int i = 0; i < kMostPolls; ++i)
        if (mbar_try(bar, parity)) return true;
    return false;
}
__device__ __forceinline__ void named_bar_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// 16 bytes, or (n = 0) zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// maxima that pass a NaN on
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float max2(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// a whole 32-byte sector
__device__ __forceinline__ void store8(void *p, const uint32_t (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// ---------------------------------------------------------------- items
// How a K or V tile lies in shared memory, and by which tensor map it comes.  Both halves of a row (64 channels each) in one
// load: groups of eight rows, [group][half][8 rows][128 bytes].  Half by half: [half][128 rows][128 bytes].  kByRows: the same places,
// but copied row by row (cp.async, 16 bytes a lane), for pages that are not whole groups of eight rows.
enum { kByHalves = 0, kGroupsOfAllPages = 1, kHeadsOfAllPages = 2, kByRows = 3 };
struct TileLayout {
    int map;                           // one of the four above
    uint32_t half_bytes, group_bytes;  // offsets of the second half, of the next eight rows
};
struct TcaArgs {
    AttnArgs a;
    int tile_tokens;                   // tokens of a query tile: its rows / group
    int box_log;                       // keys of one TMA box, 2^box_log: the largest power of two that divides a page, at most 128
    int tile_pages, tile_rest;         // a tile further: so many pages and rows
    TileLayout kl, vl;
    int wide_out;                      // rows of the output are whole 32-byte sectors
    float *part_o;                     // [2 slots per CTA][rows][DP]
    float2 *part_ml;                   // [2 slots per CTA][rows]: maximum (powers of two), sum
    unsigned int *arrived;             // [CTA]: parts that are there of the divided item that begins in this CTA (returns to 0)
    struct SplitRecord *records;       // [CTA]
};
// A divided item of more than 32 rows, written by its second CTA: what the joining kernel needs.
struct SplitRecord {
    int parts;                         // 0: none
    int first, token0, rows, kvh;
    int pad[3];
};

struct Item {
    int token0, n_tok;                 // first token (packed axis), tokens of the item
    int p0, kv_len;                    // position of the first token
    int lo, hi;                        // keys that some token of the item may see
    int tile0, units;                  // first key tile, key tiles (at least 1: an item without keys writes its zeros)
    // on the axis an item takes some places for its beginning and end (kItemCost) and one for every key tile
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

// PAIR: the steps (64 keys) of [step_a, step_b) that worker w's own tokens may see, [a, b).
__device__ __forceinline__ void worker_steps(const AttnArgs &g, const Item &it, int w, int tile_tokens, int step_a, int step_b, int &a, int &b)
{
    const int t0 = w * tile_tokens, n = min(it.n_tok - t0, tile_tokens);
    a = b = step_a;
    if (n <= 0) return;
    int lo, hi, skip;
    key_range(g, it.p0 + t0 + n - 1, it.kv_len, skip, hi);
    key_range(g, max(it.p0 + t0, 0), it.kv_len, lo, skip);
    if (hi <= lo) return;
    a = max(step_a, lo / kPairKeys);
    b = max(a, min(step_b, (hi + kPairKeys - 1) / kPairKeys));
}

// Walks the items of a CTA's range; every role walks for itself.
struct Walk {
    int b, kvh, qi, n_items;
    int cu, q_len, kv_len;
    // the CTA's key tiles [a, b) of the item at hand: `in` places of it lie before the CTA's range, `left` places are left of that
    __device__ __forceinline__ static void share(const Item &it, int cost, int in, int left, int &a, int &b)
    {
        a = max(0, in - cost);
        b = min(it.units, max(0, in + left - cost));
    }
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

// Kinds of items: see above.  COPIES: a SPLIT item of at most 32 rows with its queries four times in the tile, once for each
// quarter of the TMEM lanes.
enum Mode { kPair = 0, kSplit = 1, kCopies = 4 };

template <int DP, int MODE> struct Tca {
    static constexpr bool kIsPair = MODE == kPair;
    static constexpr int kTileRows = MODE == kCopies ? 32 : kRowsPerTile;      // rows of a query tile
    static constexpr int kTile = kRowsPerTile * DP * 2;
    static constexpr int kHalves = DP / 64;
    static constexpr int kQTiles = kIsPair ? 2 : 1;
    static constexpr int kSlots = DP == 128 ? 5 : 8;
    static constexpr int kStage = MODE == kCopies ? 4 * 8 * (DP + 4) * 4 : 0;  // eight rows of the four copies' outputs
    static constexpr int kBars = (kQTiles + kSlots) * kTile + kStage;          // barriers, start state, SPLIT: row statistics
    static constexpr int kSmem = kBars + 3072;
    static constexpr int kRows = kQTiles * kTileRows;                          // of a partial result
};

struct TcaBars {                       // shared memory, after the tiles
    unsigned long long q_full, q_empty, done, s_full[4], p_ready[4], o_done[4], kv_full[8], kv_empty[8];
    uint32_t tmem;
    int b, kvh, qi, in, left, last;
    long long totals[kTcaThreads / 32], items[kTcaThreads / 32];
};
static_assert(sizeof(TcaBars) <= 1024, "barriers fit before the row statistics");

// Joins the parts of one row of a divided item: a warp, four channels per lane, four parts in flight.  Little code, because it runs
// once in a launch, straight from L2.
template <typename T, int DP, int MODE>
__device__ __forceinline__ void join_row(const TcaArgs &ga, int first, int parts, int token0, int kvh, int i)
{
    constexpr int kRows = Tca<DP, MODE>::kRows, kTileRows = Tca<DP, MODE>::kTileRows;
    const AttnArgs &g = ga.a;
    const int lane = threadIdx.x & 31, t = i / g.group, h = i - t * g.group, tile = MODE == kPair && t >= ga.tile_tokens;
    const int row = tile * kTileRows + i - tile * ga.tile_tokens * g.group;
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        // the first part lies in the second slot of its CTA, the others in the first of theirs
        const long long at = (long long)(2 * (first + p) + (p == 0 ? 1 : 0)) * kRows + row;
        const float2 ml = __ldcg(ga.part_ml + at);
        const float4 o = lane * 4 < DP ? __ldcg(reinterpret_cast<const float4 *>(ga.part_o + at * DP) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float m2 = fmaxf(m, ml.x), base = m2 == -INFINITY ? 0.f : m2, x = ex2(m - base), y = ex2(ml.x - base);
        m = m2;
        l = fmaf(l, x, ml.y * y);
        acc = make_float4(fmaf(acc.x, x, o.x * y), fmaf(acc.y, x, o.y * y), fmaf(acc.z, x, o.z * y), fmaf(acc.w, x, o.w * y));
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    const long long tok = token0 + t, head = kvh * g.group + h;
    if (lane * 4 < g.dim)
        *reinterpret_cast<uint2 *>(static_cast<T *>(g.out) + tok * g.ots + head * g.ohs + lane * 4) =
            make_uint2(round_pair<T>(acc.x * inv, acc.y * inv), round_pair<T>(acc.z * inv, acc.w * inv));
    if (g.lse && lane == 0) g.lse[tok * g.hq + head] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
}

// BY_ROWS: K and V come by kByRows (a template, not a branch: a branch in the loaders cost 96 requests' step 84 -> 89 us).
template <typename T, int DP, int MODE, bool BY_ROWS>
__global__ void __launch_bounds__(kTcaThreads, 1)
attention_tc_kernel(const __grid_constant__ TcaArgs ga, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v)
{
    using Cfg = Tca<DP, MODE>;
    constexpr bool PAIR = MODE == kPair;
    extern __shared__ __align__(1024) unsigned char smem[];
    const AttnArgs &g = ga.a;
    TcaBars *sh = reinterpret_cast<TcaBars *>(smem + Cfg::kBars);
    float2 *row_ml = reinterpret_cast<float2 *>(smem + Cfg::kBars + 1024);     // [2][128], SPLIT only
    const uint32_t q_smem = smem_u32(smem), ring = q_smem + Cfg::kQTiles * Cfg::kTile;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tile_tokens = ga.tile_tokens, item_tokens = tile_tokens * Cfg::kQTiles;

    if (tid == 0) {
        mbar_init(smem_u32(&sh->q_full), 1);
        mbar_init(smem_u32(&sh->q_empty), 2);
        mbar_init(smem_u32(&sh->done), 2);
        for (int w = 0; w < 4; ++w) {                                  // worker w & 1, even and odd steps
            mbar_init(smem_u32(&sh->s_full[w]), 1);
            mbar_init(smem_u32(&sh->p_ready[w]), 4);
            mbar_init(smem_u32(&sh->o_done[w]), 1);
        }
        for (int s = 0; s < Cfg::kSlots; ++s) {
            mbar_init(smem_u32(&sh->kv_full[s]), 1);
            mbar_init(smem_u32(&sh->kv_empty[s]), 2);                  // both MMA warps pass every tile
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) {
        tc_alloc(smem_u32(&sh->tmem), 512);
        tc_relinquish();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");                 // what is above touches no global memory
    if (MODE != kCopies && tid == 351) ga.records[blockIdx.x].parts = 0;
    if (tid >= 352 && tid < 355)
        asm volatile("prefetch.tensormap [%0];" ::"l"(tid == 352 ? &map_q : tid == 353 ? &map_k : &map_v) : "memory");

    // ---- this CTA's range: key tiles of every sequence (in the ring, before it is used), their total, the first item
    uint2 *seq_work = reinterpret_cast<uint2 *>(smem + Cfg::kQTiles * Cfg::kTile);    // key tiles and items of one key head
    long long mine = 0, mine_items = 0;
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
        if (b < g.n_seqs) seq_work[b] = make_uint2(units, (unsigned int)n);
        mine += units;
        mine_items += n;
    }
    if (warp * 32 < g.n_seqs) {
        for (int o = 16; o; o >>= 1) {
            mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
            mine_items += __shfl_xor_sync(0xFFFFFFFFu, mine_items, o);
        }
    }
    if (lane == 0) { sh->totals[warp] = mine; sh->items[warp] = mine_items; }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;
    long long total = 0, items = 0;
    for (int w = 0; w < kTcaThreads / 32 && w * 32 < g.n_seqs; ++w) {
        total += sh->totals[w];
        items += sh->items[w];
    }
    total *= g.hk;
    items *= g.hk;
    // A small call is cut finely, a key tile for each worker; else an item's beginning and end count as well.
    const bool small = total <= 2 * gridDim.x;
    const int item_cost = small ? 0 : kItemCost;
    const bool narrow = total + items * kItemCost < 0x40000000LL;      // (divisions of 64 bits cost hundreds of cycles)
    long long per;
    if (small) {
        per = (total <= gridDim.x ? 1 : 2) * (!PAIR && total <= gridDim.x && total >= 2 * items ? 2 : 1);
    } else {
        total += items * kItemCost;
        per = narrow ? (long long)(((unsigned int)total + gridDim.x - 1) / gridDim.x) : (total + gridDim.x - 1) / gridDim.x;
    }
    const long long start = per * blockIdx.x;
    if (warp == 0) {
        if (lane == 0) sh->left = (int)(start < total ? (total - start < per ? total - start : per) : 0);
        long long before = 0;
        bool found = start >= total;
        for (int base = 0; base < g.n_seqs && !found; base += 32) {
            const uint2 sw = base + lane < g.n_seqs ? seq_work[base + lane] : make_uint2(0u, 0u);
            const int head_places = (int)(sw.x + sw.y * item_cost);
            const long long u = (long long)head_places * g.hk;
            long long incl = u;
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned int hit = __ballot_sync(0xFFFFFFFFu, before + incl > start);
            if (hit) {
                const int src = __ffs(hit) - 1;
                const long long rest = start - before - __shfl_sync(0xFFFFFFFFu, incl - u, src);
                const int b = base + src, per_head = __shfl_sync(0xFFFFFFFFu, head_places, src), n = __shfl_sync(0xFFFFFFFFu, (int)sw.y, src);
                const int kvh = narrow ? (int)((unsigned int)rest / (unsigned int)per_head) : (int)(rest / per_head);
                int in = (int)(rest - (long long)kvh * per_head), qi = 0;
                int cu = 0, q_len = 0, kv_len = 0;
                if (n > 1) seq_lengths(g, b, cu, q_len, kv_len);
                for (int i0 = 0; n > 1 && i0 < n; i0 += 32) {
                    const int un = i0 + lane < n ? make_item(g, cu, q_len, kv_len, i0 + lane, item_tokens).units + item_cost : 0;
                    int sum = un;
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                        if (lane >= o) sum += x;
                    }
                    const unsigned int at = __ballot_sync(0xFFFFFFFFu, sum > in);
                    if (at) {
                        const int s2 = __ffs(at) - 1;
                        qi = i0 + s2;
                        in -= __shfl_sync(0xFFFFFFFFu, sum - un, s2);
                        break;
                    }
                    in -= __shfl_sync(0xFFFFFFFFu, sum, 31);
                }
                if (lane == 0) { sh->b = b; sh->kvh = kvh; sh->qi = qi; sh->in = in; }
                found = true;
            }
            before += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    __syncthreads();
    int left = sh->left, in = sh->in;
    Walk walk;
    walk.b = sh->b; walk.kvh = sh->kvh; walk.qi = sh->qi;
    if (left > 0) walk.open(g, item_tokens);
    bool ok = true;                    // of this role
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !bar_wait_inline(bar, parity)) ok = false;
        __syncwarp();                  // the tcgen05 instructions behind it want the warp together
    };

    // Registers: 384 threads x 168 at launch = 64512; afterwards 256 x 192 + 128 x 112 = 63488.  (Each role's instruction stands
    // in its own branch: the compiler takes the smaller number behind a join.)
    auto load_q = [&](int kvh, int token0) {
        constexpr int kLoads = MODE == kCopies ? 4 : Cfg::kQTiles;
        mbar_expect_tx(smem_u32(&sh->q_full), (uint32_t)(kLoads * Cfg::kHalves * tile_tokens * g.group * 128));
        for (int w = 0; w < kLoads; ++w)
            for (int h = 0; h < Cfg::kHalves; ++h)
                tma_load_3d(q_smem + (PAIR ? w * Cfg::kTile : w * 32 * 128) + h * kHalfBytes, &map_q, h * 64, kvh * g.group,
                            token0 + (PAIR ? w * tile_tokens : 0), smem_u32(&sh->q_full));
    };
    if (warp == 9 || warp == 10) {
        // ------------------------------------------------------------ loaders: Q and K tiles, V tiles
        asm volatile("setmaxnreg.dec.sync.aligned.u32 112;");
        fence_proxy_async();
        const bool is_v = warp == 10;
        const CUtensorMap *map = is_v ? &map_v : &map_k;
        const TileLayout tl = is_v ? ga.vl : ga.kl;
        const int page_size = g.page_size, R = 1 << ga.box_log;
        const int halves = tl.map == kByHalves ? Cfg::kHalves : 1;
        const uint32_t box_bytes = (uint32_t)(R * 128 * Cfg::kHalves) / halves;
        left = uniform(left);
        in = uniform(in);
        int seq = 0;                                                   // tiles of K and V that went before this item
        int last = -1;                                                 // this warp's last one
        uint32_t q_phase = 0;
        bool q_used = false;
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            int ua, ub;
            Walk::share(it, item_cost, in, left, ua, ub);
            ua = uniform(ua);
            const int lo = uniform(it.lo), hi = uniform(it.hi), n = uniform(ub) - ua;
            if (hi > lo && n > 0) {
                const int kvh = uniform(walk.kvh), tile_a = uniform(it.tile0) + ua;
                const int token0 = uniform(it.token0);
                if (is_v) {                                            // (K tiles may come before the last item is through with its Q)
                    if (q_used) {
                        wait(smem_u32(&sh->q_empty), q_phase ^ 1u);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (ok && elect_one()) load_q(kvh, token0);
                    }
                    q_phase ^= 1u;
                    q_used = true;
                }
                const int *table = g.table + (long long)walk.b * g.table_stride;
                // A tile's boxes (up to 16), one per lane: column of the table and row of the page.  They are carried from tile to tile;
                // a division here would wait for the special-function unit, which the workers keep busy.
                int key = tile_a * kKeysPerTile + lane * R;
                int col = key / page_size, row = key - col * page_size;
                auto fetch = [&]() {
                    const bool wanted = key + R > lo && key < hi && lane * R < kKeysPerTile;
                    return !wanted ? 0 : col < g.max_pages ? __ldg(table + col) : -1;
                };
                if constexpr (BY_ROWS) {
                    // A lane looks up the rows lane, lane + 32, ..; half a warp (a quarter, for heads of 64) copies a row.
                    constexpr int kChunks = DP / 8, kRowsAtOnce = 32 / kChunks;
                    const T *base = static_cast<const T *>(is_v ? g.v : g.k) + (long long)kvh * (is_v ? g.vhs : g.khs);
                    const long long ps = is_v ? g.vps : g.kps, ts = is_v ? g.vts : g.kts;
                    const int chunk = lane % kChunks, half = chunk / 8, size = chunk * 8 < g.dim ? 16 : 0;
                    int c[4], r[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at_key = tile_a * kKeysPerTile + lane + 32 * j;
                        c[j] = at_key / page_size;
                        r[j] = at_key - c[j] * page_size;
                    }
                    int pages[4];
                    auto look_up = [&](int k0) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int key = k0 + lane + 32 * j;
                            pages[j] = key < lo || key >= hi ? 0 : c[j] < g.max_pages ? __ldg(table + c[j]) : -1;
                        }
                    };
                    look_up(tile_a * kKeysPerTile);
                    int in_flight = -1;                                // this item's tile whose copies are not known to have landed
                    auto landed = [&](int behind) {
                        if (behind) asm volatile("cp.async.wait_group 1;" ::: "memory");
                        else asm volatile("cp.async.wait_group 0;" ::: "memory");
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh->kv_full[in_flight % Cfg::kSlots]));
                        in_flight = -1;
                    };
                    for (int i = 0; i < n && ok; ++i) {
                        const int k0 = (tile_a + i) * kKeysPerTile;
                        const int at = seq + (PAIR ? 2 * i + is_v : is_v ? min(2 * i + 2, 2 * n - 1) : max(2 * i - 1, 0));
                        const int slot = at % Cfg::kSlots;
                        const uint32_t phase = (uint32_t)(at / Cfg::kSlots) & 1u, empty = smem_u32(&sh->kv_empty[slot]);
                        long long row_at[4];                           // -1: not wanted, -2: no such page
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int key = k0 + lane + 32 * j;
                            row_at[j] = -1;
                            if (key >= lo && key < hi) {
                                row_at[j] = pages[j] >= 0 && pages[j] < g.n_pages ? pages[j] * ps + r[j] * ts : -2;
                                if (row_at[j] == -2) report_status(g.status, FPSK_ERR_PARAM);
                            }
                            c[j] += ga.tile_pages;
                            r[j] += ga.tile_rest;
                            if (r[j] >= page_size) { r[j] -= page_size; ++c[j]; }
                        }
                        if (i + 1 < n) look_up(k0 + kKeysPerTile);     // its latency passes behind the copies
                        // (a tile in flight is handed on before a wait that may be long)
                        if (in_flight >= 0 && !__all_sync(0xFFFFFFFFu, mbar_try(empty, phase ^ 1u))) landed(0);
                        wait(empty, phase ^ 1u);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        const uint32_t dst = ring + slot * Cfg::kTile + half * kHalfBytes;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll 8                                                       // (1.63 ms; 4: 1.79, 16: 1.97)
                            for (int x = 0; x < 32; x += kRowsAtOnce) {
                                const int src_lane = x + lane / kChunks, row = 32 * j + src_lane;
                                const long long from = __shfl_sync(0xFFFFFFFFu, row_at[j], src_lane);
                                if (from != -1)
                                    copy16(dst + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), from >= 0 && size ? base + from + chunk * 8 : base,
                                           from >= 0 ? size : 0);
                            }
                        asm volatile("cp.async.commit_group;" ::: "memory");
                        if (in_flight >= 0) landed(1);
                        in_flight = at;
                        last = at;
                    }
                    if (in_flight >= 0) landed(0);
                    if (ok) seq += 2 * n;
                } else {
                int next = fetch();
                for (int i = 0; i < n; ++i) {
                    const int tile = tile_a + i, k0 = tile * kKeysPerTile;
                    int page = next;
                    const int page_row = row;
                    key += kKeysPerTile;
                    col += ga.tile_pages;
                    row += ga.tile_rest;
                    if (row >= page_size) { row -= page_size; ++col; }
                    if (i + 1 < n) next = fetch();                     // its latency passes behind the wait
                    // this tile's place in the order in which the MMAs use the ring
                    const int at = seq + (PAIR ? 2 * i + is_v : is_v ? min(2 * i + 2, 2 * n - 1) : max(2 * i - 1, 0));
                    const int slot = at % Cfg::kSlots;
                    const uint32_t phase = (uint32_t)(at / Cfg::kSlots) & 1u;
                    const uint32_t full = smem_u32(&sh->kv_full[slot]), dst = ring + slot * Cfg::kTile;
                    const int b0 = max(0, lo - k0) >> ga.box_log, b1 = (min(kKeysPerTile, hi - k0) + R - 1) >> ga.box_log;
                    wait(smem_u32(&sh->kv_empty[slot]), phase ^ 1u);
                    if (page < 0 || page >= g.n_pages) {
                        report_status(g.status, FPSK_ERR_PARAM);
                        page = (int)g.n_pages;                         // outside the tensor map: zeros
                    }
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (ok) {
                        if (elect_one()) mbar_expect_tx(full, (uint32_t)((b1 - b0) * halves) * box_bytes);
                        __syncwarp();
                        for (int box = b0; box < b1; ++box) {
                            const int pg = __shfl_sync(0xFFFFFFFFu, page, box), at_row = __shfl_sync(0xFFFFFFFFu, page_row, box);
                            if (elect_one()) {
                                if (tl.map == kGroupsOfAllPages)
                                    tma_load_5d(dst + box * box_bytes, map, 0, 0, 0, kvh, pg * (page_size >> 3) + (at_row >> 3), full);
                                else if (tl.map == kHeadsOfAllPages)
                                    tma_load_5d(dst + box * box_bytes, map, 0, 0, 0, at_row >> 3, pg * g.hk + kvh, full);
                                else
                                    for (int h = 0; h < Cfg::kHalves; ++h)
                                        tma_load_4d(dst + h * kHalfBytes + box * box_bytes, map, h * 64, at_row, kvh, pg, full);
                            }
                            __syncwarp();
                        }
                        last = at;
                    }
                }
                if (ok) seq += 2 * n;
                }
            }
            left -= uniform(it.units) + item_cost - in;
            in = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
        // The last fill of every slot: in flight still only if the MMA warp's waits gave up.
        for (int at = last; at >= 0 && at >= seq - Cfg::kSlots; --at)
            if (!bar_wait_inline(smem_u32(&sh->kv_full[at % Cfg::kSlots]), (uint32_t)(at / Cfg::kSlots) & 1u)) ok = false;
        if (q_used && !bar_wait_inline(smem_u32(&sh->q_full), q_phase ^ 1u)) ok = false;
    } else if (warp == 8 || warp == 11) {
        // ------------------------------------------------------------ MMA issue, a warp for each worker: while one waits for its
        // worker or works through its barriers, the tensor core has the other's
        asm volatile("setmaxnreg.dec.sync.aligned.u32 112;");
        const int w = warp == 11;
        const uint32_t fmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t base_desc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(kRowsPerTile >> 4) << 24);
        constexpr int kStepKeys = PAIR ? kPairKeys : kKeysPerTile;
        const uint32_t idesc_s = base_desc | ((uint32_t)(kStepKeys >> 3) << 17);
        const uint32_t idesc_o = base_desc | (1u << 16) | ((uint32_t)(DP >> 3) << 17);
        const uint32_t tm = (uint32_t)uniform((int)tmem);
        const uint32_t q_hi = desc_hi(1024), k_hi = desc_hi(ga.kl.group_bytes), v_hi = desc_hi(ga.vl.group_bytes);
        left = uniform(left);
        in = uniform(in);
        int seq = 0;                                                   // tiles of K and V that went before this item
        uint32_t q_phase = 0, s_count = 0, o_count = 0;                // steps issued so far
        bool first_item = true;
        auto all_wait = [&](uint32_t bar, uint32_t parity) {
            wait(bar, parity);
            ok = __all_sync(0xFFFFFFFFu, ok);
            tc_fence_after();
        };
        // TMEM columns of the worker's S (and P) in a step
        auto s_col = [&](uint32_t count) { return tm + w * 128 + (PAIR ? (count & 1u) * kPairKeys : 0u); };
        auto issue_s = [&](uint32_t k_addr) {
            const uint32_t c = s_count++;
            if (ok && elect_one()) {
                const uint32_t qa = desc_lo(q_smem + (PAIR ? w * Cfg::kTile : 0), 16), kb = desc_lo(k_addr, 16);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
                    mma_ss(s_col(c), qa + ((k / 4) * kHalfBytes + (k % 4) * 32) / 16, q_hi,
                           kb + (k / 4) * (ga.kl.half_bytes / 16) + (k % 4) * 2, k_hi, idesc_s, k > 0);
                tc_commit(smem_u32(&sh->s_full[w + 2 * (c & 1u)]));
            }
            __syncwarp();
        };
        auto issue_o = [&](uint32_t v_addr, bool accumulate) {
            const uint32_t c = o_count++;
            all_wait(smem_u32(&sh->p_ready[w + 2 * (c & 1u)]), (c >> 1) & 1u);
            if (ok && elect_one()) {
                const uint32_t vb = desc_lo(v_addr, ga.vl.half_bytes), step = ga.vl.group_bytes / 8;
#pragma unroll
                for (int k = 0; k < kStepKeys / 16; ++k)
                    mma_ts(tm + 256 + w * 128, s_col(c) + k * 8, vb + k * step, v_hi, idesc_o, accumulate || k > 0);
                tc_commit(smem_u32(&sh->o_done[w + 2 * (c & 1u)]));
            }
            __syncwarp();
        };
        // a tile by its place in the ring's order
        auto tile_addr = [&](int at) { return ring + (uint32_t)(at % Cfg::kSlots) * Cfg::kTile; };
        auto wait_tile = [&](int at) { all_wait(smem_u32(&sh->kv_full[at % Cfg::kSlots]), (uint32_t)(at / Cfg::kSlots) & 1u); };
        auto release = [&](unsigned long long *bar) {
            if (ok && elect_one()) tc_commit(smem_u32(bar));
            __syncwarp();
        };
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            int ua, ub;
            Walk::share(it, item_cost, in, left, ua, ub);
            ua = uniform(ua);
            const int lo = uniform(it.lo), hi = uniform(it.hi), n = uniform(ub) - ua;
            if (hi > lo && n > 0) {
                const int tile_a = uniform(it.tile0) + ua, tile_b = tile_a + n;
                // rows of a V tile that no token of the item may see: zeros, for 0 * (what lies there) must not be NaN (in a PAIR
                // item both warps write them, each before its own MMAs)
                auto clean_v = [&](int tile, uint32_t v_addr) {
                    const int k0 = tile * kKeysPerTile, r0 = max(0, lo - k0), r1 = min(kKeysPerTile, hi - k0);
                    if (r0 == 0 && r1 == kKeysPerTile) return;
                    for (int i = lane; i < kKeysPerTile * 8 * Cfg::kHalves; i += 32) {
                        const int r = i >> (2 + Cfg::kHalves), h = Cfg::kHalves == 2 ? (i >> 3) & 1 : 0;
                        if (r < r0 || r >= r1)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_addr + (r >> 3) * ga.vl.group_bytes + h * ga.vl.half_bytes + (r & 7) * 128 + (i & 7) * 16), "r"(0) : "memory");
                    }
                    fence_proxy_async();
                    __syncwarp();
                };
                if (w == 1 && first_item) {                            // (the loader of V, which brings the others, has V to bring)
                    fence_proxy_async();
                    const int kvh = uniform(walk.kvh), token0 = uniform(it.token0);
                    if (ok && elect_one()) load_q(kvh, token0);
                    __syncwarp();
                }
                first_item = false;
                all_wait(smem_u32(&sh->q_full), q_phase);
                q_phase ^= 1u;
                // The tile of queries is free behind the item's last S: the next item's comes (and its V tiles behind it) while this
                // one's weights, outputs and end are still to be done.
                if constexpr (PAIR) {
                    // S is two steps ahead of P V, so that a softmax never waits for its scores
                    int sa, sb;
                    worker_steps(g, it, w, tile_tokens, 2 * tile_a, 2 * tile_b, sa, sb);
                    sa = uniform(sa);
                    sb = uniform(sb);
                    if (sa >= sb) release(&sh->q_empty);
                    auto next_s = [&](int st, uint32_t k_addr) {
                        if (st < sa || st >= sb) return;
                        issue_s(k_addr);
                        if (st == sb - 1) release(&sh->q_empty);
                    };
                    const uint32_t k_half = 8 * ga.kl.group_bytes, v_half = 8 * ga.vl.group_bytes;   // the tile's second 64 keys
                    wait_tile(seq);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        next_s(2 * tile_a + h, tile_addr(seq) + h * k_half);
                    release(&sh->kv_empty[seq % Cfg::kSlots]);
                    for (int t = tile_a; t < tile_b; ++t) {
                        const int vt = seq + 1, kt = seq + 2;
                        const bool more = t + 1 < tile_b;
                        wait_tile(vt);
                        if (ok) clean_v(t, tile_addr(vt));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int st = 2 * t + h;
                            if (st >= sa && st < sb) issue_o(tile_addr(vt) + h * v_half, st > sa);
                            if (h == 1) release(&sh->kv_empty[vt % Cfg::kSlots]);
                            if (more && h == 0) wait_tile(kt);
                            if (more) next_s(st + 2, tile_addr(kt) + h * k_half);
                        }
                        if (more) release(&sh->kv_empty[kt % Cfg::kSlots]);
                        seq += 2;
                    }
                } else {
                    // Every other tile is this worker's.  Both warps go through the ring in its order and pass every tile on, their own
                    // or not: a warp that waited for its own alone could take the parity of an older fill of a slot for the one it wants.
                    auto step = [&](bool is_v, int i) {
                        const int at = seq++;
                        wait_tile(at);
                        if ((i & 1) != w) {
                            if (ok && elect_one()) mbar_arrive(smem_u32(&sh->kv_empty[at % Cfg::kSlots]));
                            __syncwarp();
                            return;
                        }
                        if (is_v) {
                            if (ok) clean_v(tile_a + i, tile_addr(at));
                            issue_o(tile_addr(at), i > w);
                        } else {
                            issue_s(tile_addr(at));
                            if (i + 2 >= n) release(&sh->q_empty);
                        }
                        release(&sh->kv_empty[at % Cfg::kSlots]);
                    };
                    if (n <= w) release(&sh->q_empty);
                    step(false, 0);
                    if (n > 1) step(false, 1);
                    for (int i = 0; i < n; ++i) {
                        step(true, i);
                        if (i + 2 < n) step(false, i + 2);
                    }
                }
            }
            left -= uniform(it.units) + item_cost - in;
            in = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
        if (elect_one()) tc_commit(smem_u32(&sh->done));
        __syncwarp();
        if (!bar_wait_inline(smem_u32(&sh->done), 0)) ok = false;
        __syncwarp();
    } else {
        // ------------------------------------------------------------ workers: a thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        constexpr int kCols = MODE == kCopies ? 32 : PAIR ? kPairKeys : 128;   // keys of a step that a thread weighs
        const int w = warp >> 2, rloc = tid & 127, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t to = tmem + lanes + 256 + w * 128;
        const int row = MODE == kCopies ? lane : rloc;                 // in the query tile
        const int tok_in_tile = row / g.group, head_in_group = row - tok_in_tile * g.group;
        const int col0 = MODE == kCopies ? quarter * 32 : 0;
        const float sl2 = g.scale_log2;
        uint32_t count = 0;                                            // steps so far
        long long pos = start - in;                                    // the item's place on the axis
        // the barrier (of its four) and the parity of step c
        auto step_bar = [&](unsigned long long *bars, uint32_t c) { return smem_u32(&bars[w + 2 * (c & 1u)]); };
        while (left > 0) {
            const Item it = make_item(g, walk.cu, walk.q_len, walk.kv_len, walk.qi, item_tokens);
            int ua, ub;
            Walk::share(it, item_cost, in, left, ua, ub);
            const int n = ub - ua;
            if (n > 0) {
            const int t_in_item = (PAIR ? w * tile_tokens : 0) + tok_in_tile;
            const bool valid = tok_in_tile < tile_tokens && t_in_item < it.n_tok;
            const bool warp_on = __any_sync(0xFFFFFFFFu, valid);
            int lo = 0, hi = 0x7FFFFFFF;                               // rows without a token compute what nobody reads
            if (valid) key_range(g, it.p0 + t_in_item, it.kv_len, lo, hi);
            int ta = 0, tb = 0, step = 1;
            if (it.hi > it.lo) {
                const int tile_a = it.tile0 + ua, tile_b = tile_a + n;
                if constexpr (PAIR) worker_steps(g, it, w, tile_tokens, 2 * tile_a, 2 * tile_b, ta, tb);
                else { ta = tile_a + w; tb = tile_b; step = 2; }
            }
            float m = -INFINITY, l = 0.f;
            bool have_o = false;
            bool open = true;                                          // some row of the warp may have no reference maximum yet
            for (int t = ta; t < tb; t += step) {
                const int k0 = t * (PAIR ? kPairKeys : kKeysPerTile) + col0;
                const uint32_t ts = tmem + lanes + w * 128 + (PAIR ? (count & 1u) * kPairKeys : 0u);
                const bool masked = __any_sync(0xFFFFFFFFu, k0 < lo || k0 + kCols > hi);
                wait(step_bar(sh->s_full, count), (count >> 1) & 1u);
                tc_fence_after();
                if (warp_on) {
                    constexpr int kChunks = kCols / 32;
                    auto load_scores = [&](uint32_t (&s)[kChunks][32]) {
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) tm_load32(ts + col0 + c * 32, s[c]);
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) tm_wait32(s[c]);
                        if (masked) {
#pragma unroll
                            for (int i = 0; i < kCols; ++i)
                                if (k0 + i < lo || k0 + i >= hi) s[i / 32][i % 32] = 0xFF800000u;
                        }
                    };
                    auto top32 = [&](const uint32_t (&s)[32], float top) {
                        float a = top, b = __uint_as_float(s[0]);
#pragma unroll
                        for (int i = 1; i < 29; i += 4) {
                            a = max3(a, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
                            b = max3(b, __uint_as_float(s[i + 2]), __uint_as_float(s[i + 3]));
                        }
                        return max2(max3(a, __uint_as_float(s[29]), __uint_as_float(s[30])), max2(b, __uint_as_float(s[31])));
                    };
                    // a row that has met NaN or +inf is NaN, whatever its other scores are
                    auto reference = [](float top) { return top < INFINITY ? top : __int_as_float(0x7FC00000); };
                    auto top_score = [&](uint32_t (&s)[kChunks][32]) {
                        float top = -INFINITY;
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) top = top32(s[c], top);
                        return top * sl2 - Reference<T>::kBelow;
                    };
                    // Weights against the reference maximum, which the first step that a row sees sets (with a window that need not be
                    // the item's first; weights against anything else could all be zero).  The sum of a step's weights tells whether
                    // a score has outgrown it: while the sum is at most kMost no weight is larger, and no maximum is taken.  Else
                    // (rare) the reference follows, O is rescaled and the weights are computed once more.
                    uint32_t p[kCols / 2];
                    float step_sum;
                    bool again = !have_o || (open && __any_sync(0xFFFFFFFFu, valid && m == -INFINITY && max(k0, lo) < min(k0 + kCols, hi)));
#pragma unroll 1
                    for (;;) {
                        uint32_t s[kChunks][32];
                        load_scores(s);
                        if (again) {
                            const float top = top_score(s);
                            const bool grow = valid && !(top <= m);
                            const float m2 = grow ? reference(top) : m, alpha = grow ? ex2(m - m2) : 1.f;
                            m = m2;
                            l *= alpha;
                            open = __any_sync(0xFFFFFFFFu, valid && m == -INFINITY);
                            if (have_o) {
                                wait(step_bar(sh->o_done, count - 1u), ((count - 1u) >> 1) & 1u);
                                tc_fence_after();
#pragma unroll 1
                                for (int c = 0; c < DP / 16; ++c) {
                                    uint32_t o[16];
                                    tm_ld16(to + c * 16, o);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                    tm_st16(to + c * 16, o);
                                }
                                tm_wait_st();
                            }
                        }
                        const float base = m == -INFINITY ? 0.f : m;
                        const float2 sc = make_float2(sl2, sl2), nb = make_float2(-base, -base);
                        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                float2 x = make_float2(__uint_as_float(s[c][2 * i]), __uint_as_float(s[c][2 * i + 1]));
                                x = __ffma2_rn(x, sc, nb);
                                x = make_float2(ex2(x.x), ex2(x.y));
                                sum[i & 1] = __fadd2_rn(sum[i & 1], x);
                                p[c * 16 + i] = round_pair<T>(x.x, x.y);
                            }
                        }
                        step_sum = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                        // (a row without a reference has seen no key, or scores of -inf alone: weights of zero)
                        if (again || __all_sync(0xFFFFFFFFu, !valid || step_sum <= Reference<T>::kMost)) break;
                        again = true;
                    }
                    l += step_sum;
                    if constexpr (MODE == kCopies) {
                        // zeros for the other quarters' keys
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t x[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = q == quarter ? p[i] : 0u;
                            tm_st16(ts + q * 16, x);
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < kCols / 64; ++h) {
                            uint32_t x[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = p[h * 32 + i];
                            tm_st32(ts + h * 32, x);
                        }
                    }
                    tm_wait_st();
                }
                have_o = true;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(step_bar(sh->p_ready, count));
                ++count;
            }
            if (have_o) {
                wait(step_bar(sh->o_done, count - 1u), ((count - 1u) >> 1) & 1u);
                tc_fence_after();
            }
            // ---- the item's end: finished here, or a partial result
            const bool whole = n == it.units;
            const bool any = it.hi > it.lo, have1 = any && n > 1;     // SPLIT: outputs of the two workers
            float wt0 = 1.f, wt1 = 0.f;                               // and their weights
            if constexpr (!PAIR) {
                row_ml[w * 128 + rloc] = make_float2(m, l);
                tc_fence_before();
                named_bar_sync(1, 256);                               // both outputs are complete
                tc_fence_after();
                const float2 a = row_ml[rloc], b = row_ml[128 + rloc];
                m = fmaxf(a.x, b.x);
                if constexpr (MODE == kCopies) {
                    for (int q = 0; q < 4; ++q) m = max3(m, row_ml[q * 32 + lane].x, row_ml[128 + q * 32 + lane].x);
                }
                const float base = m == -INFINITY ? 0.f : m;
                wt0 = ex2(a.x - base);
                wt1 = ex2(b.x - base);
                l = a.y * wt0 + b.y * wt1;
                if constexpr (MODE == kCopies) {
                    l = 0.f;
                    for (int q = 0; q < 4; ++q) {
                        const float2 x = row_ml[q * 32 + lane], y = row_ml[128 + q * 32 + lane];
                        l += x.y * ex2(x.x - base) + y.y * ex2(y.x - base);
                    }
                }
            }
            const bool have0 = PAIR ? have_o : any;
            const int pslot = 2 * blockIdx.x + (ua == 0 ? 1 : 0);        // divided: the part of the CTA where the item begins, or a later one
            // 32 channels of this row: the worker's own (PAIR) or both workers'
            auto outputs = [&](int c, float (&o)[32]) {
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
            };
            const float inv = l != 0.f ? 1.f / l : 0.f;
            if (warp_on && valid && (PAIR || w == 0) && (MODE != kCopies || quarter == 0)) {
                if (!whole) ga.part_ml[(long long)pslot * Cfg::kRows + (PAIR ? w * 128 : 0) + row] = make_float2(m, l);
                else if (g.lse)
                    g.lse[(long long)(it.token0 + t_in_item) * g.hq + walk.kvh * g.group + head_in_group] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
            }
            if constexpr (MODE == kCopies) {
                // The four copies' shares meet in shared memory, eight rows at a time; then a thread per four channels writes.
                float *stage = reinterpret_cast<float *>(smem + (Cfg::kQTiles + Cfg::kSlots) * Cfg::kTile);
                constexpr int kLine = DP + 4;
                const int rows = it.n_tok * g.group;
                for (int r0 = 0; r0 < rows; r0 += 8) {
                    const bool mine = row >= r0 && row < r0 + 8 && valid;
#pragma unroll 1
                    for (int cc = 0; cc < DP / 64; ++cc) {
                        const int c = w * (DP / 64) + cc;             // each worker brings one half of the channels
                        float o[32];
                        outputs(c, o);
                        if (mine) {
                            float *dst = stage + (quarter * 8 + row - r0) * kLine + c * 32;
                            const float f = whole ? inv : 1.f;
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<float4 *>(dst + i) = make_float4(o[i] * f, o[i + 1] * f, o[i + 2] * f, o[i + 3] * f);
                        }
                        __syncwarp();
                    }
                    named_bar_sync(3, 256);
                    const int wtid = tid & 255, r = wtid / (DP / 4), ch = wtid % (DP / 4) * 4;
                    if (r < 8 && r0 + r < rows) {
                        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float4 y = *reinterpret_cast<const float4 *>(stage + (q * 8 + r) * kLine + ch);
                            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                        }
                        const int rr = r0 + r, tk = rr / g.group;
                        if (!whole)
                            *reinterpret_cast<float4 *>(ga.part_o + ((long long)pslot * Cfg::kRows + rr) * DP + ch) = x;
                        else if (ch < g.dim)
                            *reinterpret_cast<uint2 *>(static_cast<T *>(g.out) + (long long)(it.token0 + tk) * g.ots +
                                                       (walk.kvh * g.group + rr - tk * g.group) * g.ohs + ch) =
                                make_uint2(round_pair<T>(x.x, x.y), round_pair<T>(x.z, x.w));
                    }
                    named_bar_sync(2, 256);
                }
            } else if (warp_on) {
                T *dst = static_cast<T *>(g.out) + (long long)(it.token0 + t_in_item) * g.ots + (walk.kvh * g.group + head_in_group) * g.ohs;
                float *pdst = ga.part_o + ((long long)pslot * Cfg::kRows + (PAIR ? w * 128 : 0) + row) * DP;
#pragma unroll 1
                for (int cc = 0; cc < (PAIR ? DP / 32 : DP / 64); ++cc) {
                    const int c = PAIR ? cc : w * (DP / 64) + cc;     // SPLIT: each worker brings one half of the channels
                    float o[32];
                    outputs(c, o);
                    if (!valid) {
                    } else if (whole && ga.wide_out) {
#pragma unroll
                        for (int i = 0; i < 32; i += 16)
                            if (c * 32 + i < g.dim) {
                                uint32_t x[8];
#pragma unroll
                                for (int k = 0; k < 8; ++k) x[k] = round_pair<T>(o[i + 2 * k] * inv, o[i + 2 * k + 1] * inv);
                                store8(dst + c * 32 + i, x);
                            }
                    } else if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            if (c * 32 + i < g.dim)
                                *reinterpret_cast<uint4 *>(dst + c * 32 + i) =
                                    make_uint4(round_pair<T>(o[i] * inv, o[i + 1] * inv), round_pair<T>(o[i + 2] * inv, o[i + 3] * inv),
                                               round_pair<T>(o[i + 4] * inv, o[i + 5] * inv), round_pair<T>(o[i + 6] * inv, o[i + 7] * inv));
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint32_t x[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) x[k] = __float_as_uint(o[i + k]);
                            store8(pdst + c * 32 + i, x);
                        }
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if constexpr (MODE == kSplit) named_bar_sync(2, 256);
            if (!whole) {
                // COPIES: joined by the CTA whose part is the last to arrive, in the order of the parts.  Else by the kernel behind.
                auto cta_of = [&](long long at) { return narrow ? (int)((unsigned int)at / (unsigned int)per) : (int)(at / per); };
                const int first = cta_of(pos + item_cost), parts = cta_of(pos + item_cost + it.units - 1) - first + 1;
                if constexpr (MODE == kCopies) {
                named_bar_sync(4, 256);
                if (tid == 0) {
                    const bool last = atom_acq_rel_add(ga.arrived + first) == (unsigned int)(parts - 1);
                    if (last) ga.arrived[first] = 0u;
                    sh->last = last;
                }
                named_bar_sync(4, 256);
                if (sh->last)
                    for (int i = warp; i < it.n_tok * g.group; i += 8) join_row<T, DP, MODE>(ga, first, parts, it.token0, walk.kvh, i);
                } else if (tid == 0 && blockIdx.x == first + 1) {
                    const SplitRecord r = {parts, first, it.token0, it.n_tok * g.group, walk.kvh, {0, 0, 0}};
                    ga.records[blockIdx.x] = r;
                }
            }
            }
            pos += it.units + item_cost;
            left -= it.units + item_cost - in;
            in = 0;
            if (left > 0) walk.next(g, item_tokens);
        }
    }
    if (!ok && lane == 0) report_status(g.status, FPSK_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tc_dealloc(tmem, 512);
}

// A block for eight rows of a divided item.
template <typename T, int DP, int MODE> __global__ void __launch_bounds__(256) attention_join_kernel(const __grid_constant__ TcaArgs ga)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const SplitRecord *r = ga.records + blockIdx.x;
    const int i = blockIdx.y * 8 + (threadIdx.x >> 5), parts = __ldcg(&r->parts);
    if (parts == 0 || i >= __ldcg(&r->rows)) return;
    join_row<T, DP, MODE>(ga, __ldcg(&r->first), parts, __ldcg(&r->token0), __ldcg(&r->kvh), i);
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
    static const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
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
    return kAttnSyncBytes + align_up(ctas * sizeof(SplitRecord), 256) + 2 * ctas * kMaxPartRows * (kMaxDP * sizeof(float) + sizeof(float2));
}

static bool aligned16(const void *p, long long s0, long long s1, long long s2)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 % 8 == 0 && s1 % 8 == 0 && s2 % 8 == 0;
}
// What the tensor-core kernel takes: heads of up to 128 channels, at most 128 query heads to a key head, rows at 16-byte
// boundaries, and no expanded query dimension (TMA wants strides; a cache has none of 0).  The rest is the row kernel's.
bool attention_tc_takes(const AttnArgs &g)
{
    return g.dim <= 128 && g.group <= 128 && g.n_seqs <= kTcaMaxSeqs && aligned16(g.q, g.qts, g.qhs, 0) &&
           aligned16(g.out, g.ots, g.ohs, 0) && aligned16(g.k, g.kps, g.kts, g.khs) && aligned16(g.v, g.vps, g.vts, g.vhs) &&
           (g.n_tokens == 1 || g.qts > 0) && (g.hq == 1 || g.qhs > 0);
}

template <typename T, int DP, int MODE, bool BY_ROWS> static fpsk_status launch_tc(const AttnArgs &a, int type, int max_q_len, int max_kv_len, void *ws, cudaStream_t st)
{
    using Cfg = Tca<DP, MODE>;
    const int sms = sm_count();
    if (sms < 1) return FPSK_CUDA_FAILED(cudaErrorInvalidDevice, "the number of multiprocessors");
    if (sms > (int)(kAttnSyncBytes / sizeof(unsigned int))) return FPSK_ERR_PARAM;
    TcaArgs g;
    g.a = a;
    g.tile_tokens = Cfg::kTileRows / a.group;
    // a CTA on every SM, or for every key tile where the lengths promise fewer
    const int item_tokens = g.tile_tokens * Cfg::kQTiles;
    auto pieces = [](int n, int of) { return (double)(((long long)n + of - 1) / of); };
    const double tiles = (double)a.n_seqs * a.hk * pieces(max_q_len, item_tokens) * pieces(max_kv_len, kKeysPerTile);
    const int ctas = tiles < 1.0 ? 1 : tiles < sms ? (int)tiles : sms;
    for (g.box_log = 3; g.box_log < 7 && a.page_size % (2 << g.box_log) == 0;) ++g.box_log;
    g.wide_out = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && a.ots % 16 == 0 && a.ohs % 16 == 0 && a.dim % 16 == 0;
    g.tile_pages = kKeysPerTile / a.page_size;
    g.tile_rest = kKeysPerTile % a.page_size;
    char *p = static_cast<char *>(ws);
    g.arrived = reinterpret_cast<unsigned int *>(p);
    p += kAttnSyncBytes;
    g.records = reinterpret_cast<SplitRecord *>(p);
    p += align_up((size_t)sms * sizeof(SplitRecord), 256);
    g.part_o = reinterpret_cast<float *>(p);
    p += (size_t)2 * sms * kMaxPartRows * kMaxDP * sizeof(float);
    g.part_ml = reinterpret_cast<float2 *>(p);
    // strides of dimensions of one element are never used, but the encoder wants them valid
    auto bytes = [](long long s, long long n) { return (cuuint64_t)(n > 1 && s > 0 ? s * 2 : 16); };
    CUtensorMap mq, mk, mv;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)a.dim, (cuuint64_t)a.hq, (cuuint64_t)a.n_tokens};
        const cuuint64_t str[2] = {bytes(a.qhs, a.hq), bytes(a.qts, a.n_tokens)};
        const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)g.tile_tokens};
        if (!encode(&mq, type, 3, a.q, dims, str, box)) return FPSK_CUDA_FAILED(cudaErrorInvalidValue, "the tensor map of the queries");
    }
    // A box of K or V holds the rows of one head and page.  Heads of 128 channels come with both halves in one load where two of
    // the outer dimensions merge into one: the eight-row groups of all pages (a page is page_size rows long), or the heads of all
    // pages (a page is its heads long).
    auto kv_map = [&](CUtensorMap *m, TileLayout &tl, const void *base, long long ps, long long ts, long long hs) {
        const cuuint32_t R = 1u << g.box_log;
        tl.map = BY_ROWS ? kByRows : kByHalves;
        if (BY_ROWS) {
            tl.half_bytes = kHalfBytes;
            tl.group_bytes = 1024;
            *m = mq;                                                   // (never loaded by)
            return true;
        }
        if (a.dim == 128 && (a.n_pages == 1 || ps == a.page_size * ts) && a.n_pages * (a.page_size / 8) <= 0x7FFFFFFFLL) tl.map = kGroupsOfAllPages;
        else if (a.dim == 128 && (a.n_pages == 1 || ps == a.hk * hs) && a.n_pages * a.hk <= 0x7FFFFFFFLL) tl.map = kHeadsOfAllPages;
        if (tl.map == kByHalves) {
            tl.half_bytes = kHalfBytes;
            tl.group_bytes = 1024;
            const cuuint64_t dims[4] = {(cuuint64_t)a.dim, (cuuint64_t)a.page_size, (cuuint64_t)a.hk, (cuuint64_t)a.n_pages};
            const cuuint64_t str[3] = {bytes(ts, a.page_size), bytes(hs, a.hk), bytes(ps, a.n_pages)};
            const cuuint32_t box[4] = {64, R, 1, 1};
            return encode(m, type, 4, base, dims, str, box);
        }
        tl.half_bytes = 1024;
        tl.group_bytes = 2048;
        const bool groups = tl.map == kGroupsOfAllPages;
        const cuuint64_t n_groups = (cuuint64_t)(a.page_size / 8);
        const cuuint64_t dims[5] = {64, 8, 2, groups ? (cuuint64_t)a.hk : n_groups, groups ? n_groups * (cuuint64_t)a.n_pages : (cuuint64_t)(a.n_pages * a.hk)};
        const cuuint64_t str[4] = {bytes(ts, 8), 128, groups ? bytes(hs, a.hk) : bytes(8 * ts, n_groups), groups ? bytes(8 * ts, dims[4]) : bytes(hs, dims[4])};
        const cuuint32_t box[5] = {64, 8, 2, groups ? 1 : R / 8, groups ? R / 8 : 1};
        return encode(m, type, 5, base, dims, str, box);
    };
    if (!kv_map(&mk, g.kl, a.k, a.kps, a.kts, a.khs) || !kv_map(&mv, g.vl, a.v, a.vps, a.vts, a.vhs))
        return FPSK_CUDA_FAILED(cudaErrorInvalidValue, "the tensor maps of the cache");

    static std::atomic<unsigned long long> prepared{0};               // one bit per device
    int dev = 0;
    FPSK_CUDA_OK(cudaGetDevice(&dev));
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(prepared.load(std::memory_order_acquire) & bit)) {
        FPSK_CUDA_OK(cudaFuncSetAttribute(attention_tc_kernel<T, DP, MODE, BY_ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem));
        prepared.fetch_or(bit, std::memory_order_release);
    }
    // Both launches may begin before the kernel in front has ended (they wait for it before they read): what a launch costs passes
    // behind it.
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kTcaThreads);
    cfg.dynamicSmemBytes = Cfg::kSmem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, attention_tc_kernel<T, DP, MODE, BY_ROWS>, g, mq, mk, mv));
    FPSK_LAUNCH_CHECK();
    if constexpr (MODE != kCopies) {
        cfg.gridDim = dim3((unsigned)ctas, Cfg::kRows / 8);
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        FPSK_CUDA_OK(cudaLaunchKernelEx(&cfg, attention_join_kernel<T, DP, MODE>, g));
        FPSK_LAUNCH_CHECK();
    }
    return FPSK_OK;
}

// COPIES for a few rows of new tokens a sequence (its end goes by eight rows, and holds at most 32); then, for heads of up to 64
// channels, SPLIT while they fit one tile; else PAIR.  In us, this rule first:
//   4 rows: one token, 1001 keys 12.1, SPLIT and PAIR 13.5; 96 requests, up to 8192 keys 88, SPLIT 99, PAIR 98
//   24 rows, heads of 128: 64 requests of 4096 keys 48, PAIR 51; 8 of 500 16.2, 15.1; one of 65536 62, 60
//   32 rows, heads of 128: the same PAIR 58, 15.0, 60, COPIES 60, 17.6, 65; 262144 keys 181, 179
//   32 rows, heads of 64: 49, 15.6, 58, SPLIT 57, 14.8, 53
//   33 to 128 rows, heads of 128: 64 rows, 131072 keys PAIR 100, SPLIT 108; 32 requests of 4096 keys 33.7, 35.6; 8 of 1024 16.7, 20.8
//   33 to 128 rows, heads of 64: 128 rows, 262144 keys SPLIT 144, PAIR 176 (the softmax of one tile takes longer than its
//   keys, half as many bytes, take to come); 64 requests of 7 tokens 22.0, 23.2; but 64 of 32 tokens 61.5, 55
// Pages that are not whole groups of eight rows: copied by rows, bound by the copying warps (each a tile of 128 keys of K or V
// in some 8000 cycles): 4096 tokens over 16384 keys in pages of 12 in 1.63 ms, 96 requests of one token in 0.23 ms (pages of 16: 0.84 and
// 0.084); pages of 1 take no longer.
fpsk_status attention_tc_launch(const AttnArgs &a, int type, int max_q_len, int max_kv_len, void *ws, cudaStream_t st)
{
    if (max_q_len < 1) max_q_len = 1;
    if (max_kv_len < 1) max_kv_len = 1;
    const long long rows = (long long)max_q_len * a.group;
    const bool by_rows = a.page_size % 8 != 0, copies = rows <= (a.dim > 64 ? 24 : 32);
#define FPSK_TCA(TT, DD, MM, RR) launch_tc<TT, DD, MM, RR>(a, type, max_q_len, max_kv_len, ws, st)
#define FPSK_TCA_ROWS(TT, DD) (copies ? FPSK_TCA(TT, DD, kCopies, true) : FPSK_TCA(TT, DD, kPair, true))
#define FPSK_TCA_DIM(TT)                                                                                  \
    (by_rows       ? a.dim > 64 ? FPSK_TCA_ROWS(TT, 128) : FPSK_TCA_ROWS(TT, 64)                          \
     : a.dim > 64  ? copies ? FPSK_TCA(TT, 128, kCopies, false) : FPSK_TCA(TT, 128, kPair, false)         \
     : copies      ? FPSK_TCA(TT, 64, kCopies, false)                                                     \
     : rows <= kRowsPerTile ? FPSK_TCA(TT, 64, kSplit, false) : FPSK_TCA(TT, 64, kPair, false))
    return type == FPSK_ELEM_FP16 ? FPSK_TCA_DIM(__half) : FPSK_TCA_DIM(__nv_bfloat16);
#undef FPSK_TCA_ROWS
#undef FPSK_TCA_DIM
#undef FPSK_TCA
}

}  // namespace fpsk
