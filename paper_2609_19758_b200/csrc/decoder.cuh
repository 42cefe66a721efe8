// Shared by the decoder's operators (add_norm.cu, logits.cu, distill.cu): eight-element loads and stores of rows that start anywhere,
// and reductions whose order is fixed.
#pragma once
#include "attention.cuh"
#include "fpsk_decoder.h"
#include "stream_pipe.cuh"

#include <type_traits>

namespace fpsk {

constexpr int kSms = 148;

// Eight consecutive elements as FP32; WIDE: the address is a multiple of 16 bytes and all eight are there, otherwise the first n of them,
// one by one (the rest: 0).
template <bool WIDE> __device__ __forceinline__ void load8(const float *p, int n, float (&v)[8])
{
    if (WIDE && n == 8) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
}
template <bool WIDE, typename T> __device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (WIDE && n == 8) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        const float2 a = HalfTraits<T>::unpack2(u.x), b = HalfTraits<T>::unpack2(u.y), c = HalfTraits<T>::unpack2(u.z), d = HalfTraits<T>::unpack2(u.w);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
        v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? Elem<T>::to_f(p[i]) : 0.f;
}
template <bool WIDE> __device__ __forceinline__ void store8(float *p, int n, const float (&v)[8])
{
    if (WIDE && n == 8) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
}
template <bool WIDE, typename T> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (WIDE && n == 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(round_pair<T>(v[0], v[1]), round_pair<T>(v[2], v[3]), round_pair<T>(v[4], v[5]), round_pair<T>(v[6], v[7]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = Elem<T>::from_f(v[i]);
}
// the same of a run-time type
template <bool WIDE> __device__ __forceinline__ void load8_any(const void *p, int type, long long at, int n, float (&v)[8])
{
    if (type == FPSK_ELEM_FP32) load8<WIDE>(static_cast<const float *>(p) + at, n, v);
    else if (type == FPSK_ELEM_FP16) load8<WIDE>(static_cast<const __half *>(p) + at, n, v);
    else load8<WIDE>(static_cast<const __nv_bfloat16 *>(p) + at, n, v);
}
template <bool WIDE> __device__ __forceinline__ void store8_any(void *p, int type, long long at, int n, const float (&v)[8])
{
    if (type == FPSK_ELEM_FP32) store8<WIDE>(static_cast<float *>(p) + at, n, v);
    else if (type == FPSK_ELEM_FP16) store8<WIDE>(static_cast<__half *>(p) + at, n, v);
    else store8<WIDE>(static_cast<__nv_bfloat16 *>(p) + at, n, v);
}

__host__ __device__ __forceinline__ int elem_bytes(int type) { return type == FPSK_ELEM_FP32 ? 4 : type == FPSK_ELEM_E4M3 ? 1 : 2; }
inline bool aligned(const void *p, int type) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(type) == 0; }
// rows of 16-byte vectors: the base and the stride
inline bool row_wide(const void *p, int type, long long stride, int bytes = 16)
{
    return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride * elem_bytes(type) % bytes == 0);
}

// ---------------------------------------------------------------- rows of a vocabulary: a cluster of blocks to a row
constexpr int kRowMostBlocks = 8;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("barrier.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ unsigned int cluster_rank()
{
    unsigned int r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
constexpr float kMostFloat = 3.402823466e38f, kNoReference = -kMostFloat;      // (a row may hold nothing but the lowest number: its powers are 1)
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

// A launch that overlaps the end of the kernel in front: its blocks start where that one's have left, and touch no global memory before
// behind_the_last().  Every kernel that is launched so waits, so that a call sees all that was queued before it.
struct Launch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attrs[2] = {};
    Launch(unsigned blocks, unsigned threads, size_t bytes, unsigned cluster, cudaStream_t st)
    {
        cfg.gridDim = dim3(blocks);
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = bytes;
        cfg.stream = st;
        attrs[0].id = cudaLaunchAttributeClusterDimension;
        attrs[0].val.clusterDim.x = cluster;
        attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
        attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attrs;
        cfg.numAttrs = 2;
    }
    Launch(const Launch &) = delete;
};
__device__ __forceinline__ void behind_the_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Kernels whose blocks stay call it when their last copies are under way: blocks of the next call that come sooner take what places are
// left, and lie unevenly on the SMs for the rest of their lives (4096 x 131072 logits in 616 instead of 522 us).
__device__ __forceinline__ void let_the_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// How many clusters of a launch fit the device side by side (decoder.cu: asked once for each shape of launch).
cudaError_t clusters_at_once(const void *kernel, const cudaLaunchConfig_t &cfg, int *out);

}  // namespace fpsk
