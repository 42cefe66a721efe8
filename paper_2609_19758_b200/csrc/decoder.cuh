// Shared by the decoder's operators (add_norm.cu, logits.cu, distill.cu): eight-element loads and stores of rows that start anywhere,
// and reductions whose order is fixed.
#pragma once
#include "attention.cuh"
#include "fpsk_decoder.h"

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
// rows of 16-byte vectors: the base and the stride
inline bool row_wide(const void *p, int type, long long stride, int bytes = 16)
{
    return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride * elem_bytes(type) % bytes == 0);
}

// ---------------------------------------------------------------- rows of a vocabulary: a cluster of blocks to a row
constexpr int kRowThreads = 512, kRowWarps = kRowThreads / 32, kRowMostBlocks = 8;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
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
// a value of another block's shared memory, at the place that it has in this one's
__device__ __forceinline__ float cluster_load(const float *p, unsigned int rank)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p);
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(at), "r"(rank) : "memory");
    return v;
}

// The sum of 2^(y - m) over some y, m the largest of them (0 where that is -inf).
struct PowerSum {
    float m, s;                        // m may be -inf: nothing yet
    __device__ __forceinline__ void add(float y)
    {
        if (y > m) {
            s = s * exp2_fast(m - y) + 1.f;                            // (m = -inf, s = 0: 0 + 1)
            m = y;
        } else {
            s += y == m ? (m == -INFINITY ? 0.f : 1.f) : exp2_fast(y - m);     // (a NaN reaches s)
        }
    }
    __device__ __forceinline__ void join(float om, float os)
    {
        const float top = fmaxf(m, om), ref = top == -INFINITY ? 0.f : top;
        s = s * (m == ref ? 1.f : exp2_fast(m - ref)) + os * (om == ref ? 1.f : exp2_fast(om - ref));       // (infinities alike)
        m = top;
    }
};
__device__ __forceinline__ float log2_of(const PowerSum &p) { return p.m == -INFINITY && p.s == 0.f ? -INFINITY : p.m + log2f(p.s); }

}  // namespace fpsk
