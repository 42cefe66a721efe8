// Shared by the two forms of the norm and rotation kernels (norm_rope.cu, norm_rope_ring.cu): their arguments, how a head's channels
// lie in lanes, and the last sum of the weight gradients.
#pragma once
#include "attention.cuh"
#include "stream_pipe.cuh"

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

// How a block walks tokens and heads.  A block has S = 256 / L head slots; a slot has kPer heads at a time: of one token (`tokens`
// = 1: head, head + S, ..), or, where a token has fewer heads than slots, one head of kPer tokens, `tokens` apart.  What differs from
// one step to the next is a pointer increment; with the addresses computed anew for every head the kernel was bound by them
// (390 instructions for two heads, 0.8 issued per cycle, at half the memory's rate).
constexpr int kRopeThreads = 256, kPer = 2;
struct BlockMap {
    int tokens;                        // of a block at a time, in the sense above
    int step;                          // tokens a block covers in one step: 1 or kPer * tokens
    int chunks;                        // of S * kPer heads (grid y)
};
struct RopeArgs {
    HeadsArg h[3];                     // queries, keys, values (values: append only, copied)
    int n_all;                         // heads of all kinds
    long long n_tok;
    BlockMap map;
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
// (roundings spelled out, so that both forms of the kernels give the same bits)
__device__ __forceinline__ float turn(float x, float c, float y, float s) { return fmaf(x, c, __fmul_rn(y, s)); }
__device__ __forceinline__ void rotate4(float4 &a, float4 &b, const float4 &c, const float4 &s)
{
    const float4 x = a, y = b;
    a = make_float4(turn(x.x, c.x, -y.x, s.x), turn(x.y, c.y, -y.y, s.y), turn(x.z, c.z, -y.z, s.z), turn(x.w, c.w, -y.w, s.w));
    b = make_float4(turn(y.x, c.x, x.x, s.x), turn(y.y, c.y, x.y, s.y), turn(y.z, c.z, x.z, s.z), turn(y.w, c.w, x.w, s.w));
}
// r (g - n mean(g n)) of four channels
__device__ __forceinline__ float4 norm_grad4(float4 g, float4 n, float mean, float r)
{
    return make_float4(__fmul_rn(r, fmaf(-n.x, mean, g.x)), __fmul_rn(r, fmaf(-n.y, mean, g.y)), __fmul_rn(r, fmaf(-n.z, mean, g.z)),
                       __fmul_rn(r, fmaf(-n.w, mean, g.w)));
}
__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 scale4(float4 a, float r) { return make_float4(a.x * r, a.y * r, a.z * r, a.w * r); }
__device__ __forceinline__ float dot4(float4 a, float4 b, float acc)
{
    return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, acc))));
}
__device__ __forceinline__ float4 splat4(float x) { return make_float4(x, x, x, x); }
// over the L lanes of a slot (whole slots take a branch, not whole warps)
template <int L> __device__ __forceinline__ float sum_lanes(float x)
{
    const unsigned int mask = L == 32 ? 0xFFFFFFFFu : ((1u << L) - 1u) << (threadIdx.x & (32 - L) & 31);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) x += __shfl_xor_sync(mask, x, o);
    return x;
}

struct HeadsGradArg {
    const void *in, *dout;
    void *din;
    const void *w;
    float *dw;
    long long its, ihs, dots, dohs, dits, dihs;
    int n, wtype;
    int wide_in, wide_dout, wide_din, wide_w;
    BlockMap map;
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


// Sums `rows` rows of `dim` floats, `pitch` apart, in a fixed order: over the threads of a channel group with eight loads in flight,
// then the threads' sums in order.  All THREADS threads call it; sums: shared, 4 * THREADS floats.
template <int THREADS>
__device__ __forceinline__ void sum_rows(const float *part, int pitch, int rows, int dim, float *sums, float *out)
{
    const int groups = dim / 4, parts = THREADS / groups, c = threadIdx.x % groups, p = threadIdx.x / groups;
    float4 t = splat4(0.f);
    if (p < parts) {
        for (int b = p; b < rows; b += 8 * parts) {
            float4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = b + j * parts < rows ? __ldcg(reinterpret_cast<const float4 *>(part + (size_t)(b + j * parts) * pitch) + c) : splat4(0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) t = make_float4(t.x + x[j].x, t.y + x[j].y, t.z + x[j].z, t.w + x[j].w);
        }
    }
    __syncthreads();
    if (p < parts) store4<true>(sums + p * dim + 4 * c, t);
    __syncthreads();
    for (int ch = threadIdx.x; ch < dim; ch += THREADS) {
        float s = 0.f;
        for (int i = 0; i < parts; ++i) s += sums[i * dim + ch];
        out[ch] = s;
    }
    __syncthreads();
}

// norm_rope_ring.cu: true where it takes the call (and *rc is its status)
bool rope_ring(const RopeArgs &g, int in_type, int out_type, bool append, cudaStream_t st, fpsk_status *rc);
bool rope_grad_ring(const RopeGradArgs &g, int in_type, int grad_type, cudaStream_t st, fpsk_status *rc);
constexpr int kRingBlocks = 148;       // at most, of the ring form (rows of its weight-gradient partials)

}  // namespace fpsk
