// Shared by the attention operators (norm_rope.cu, paged_attention.cu): element types, four-element loads and stores,
// and the place of a token in a paged cache.
#pragma once
#include "fpsk_common.cuh"
#include "fpsk_attention.h"

namespace fpsk {

constexpr size_t kAttnSyncBytes = 4096;        // synchronisation words at the start of a workspace

__host__ __device__ __forceinline__ int elem_size(int type) { return type == FPSK_ELEM_FP32 ? 4 : 2; }

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float to_f(float x) { return x; }
    static __device__ __forceinline__ float from_f(float x) { return x; }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
};

// two values rounded to a pair
template <typename T> __device__ __forceinline__ uint32_t round_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t round_pair<__half>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t round_pair<__nv_bfloat16>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Four consecutive elements as FP32; WIDE: the address is a multiple of four elements.
template <bool WIDE> __device__ __forceinline__ float4 load4(const float *p)
{
    if (WIDE) return __ldg(reinterpret_cast<const float4 *>(p));
    return make_float4(__ldg(p), __ldg(p + 1), __ldg(p + 2), __ldg(p + 3));
}
template <bool WIDE, typename T> __device__ __forceinline__ float4 load4(const T *p)
{
    if (WIDE) {
        const uint2 u = __ldg(reinterpret_cast<const uint2 *>(p));
        const float2 a = HalfTraits<T>::unpack2(u.x), b = HalfTraits<T>::unpack2(u.y);
        return make_float4(a.x, a.y, b.x, b.y);
    }
    return make_float4(Elem<T>::to_f(p[0]), Elem<T>::to_f(p[1]), Elem<T>::to_f(p[2]), Elem<T>::to_f(p[3]));
}
// the same from shared memory
__device__ __forceinline__ float4 lds4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
template <typename T> __device__ __forceinline__ float4 lds4(const T *p)
{
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    const float2 a = HalfTraits<T>::unpack2(u.x), b = HalfTraits<T>::unpack2(u.y);
    return make_float4(a.x, a.y, b.x, b.y);
}
template <bool WIDE> __device__ __forceinline__ void store4(float *p, float4 x)
{
    if (WIDE) { *reinterpret_cast<float4 *>(p) = x; return; }
    p[0] = x.x; p[1] = x.y; p[2] = x.z; p[3] = x.w;
}
template <bool WIDE, typename T> __device__ __forceinline__ void store4(T *p, float4 x)
{
    if (WIDE) { *reinterpret_cast<uint2 *>(p) = make_uint2(round_pair<T>(x.x, x.y), round_pair<T>(x.z, x.w)); return; }
    p[0] = Elem<T>::from_f(x.x); p[1] = Elem<T>::from_f(x.y); p[2] = Elem<T>::from_f(x.z); p[3] = Elem<T>::from_f(x.w);
}
// four weights of a run-time type (they are read once per thread)
template <bool WIDE> __device__ __forceinline__ float4 load4_any(const void *p, int type, int at)
{
    if (type == FPSK_ELEM_FP32) return load4<WIDE>(static_cast<const float *>(p) + at);
    if (type == FPSK_ELEM_FP16) return load4<WIDE>(static_cast<const __half *>(p) + at);
    return load4<WIDE>(static_cast<const __nv_bfloat16 *>(p) + at);
}

__device__ __forceinline__ void report_status(int32_t *d_status, int code)
{
    if (d_status) atomicMax(d_status, code);
}

struct AttnArgs {
    const void *q, *k, *v;
    void *out;
    float *lse;
    long long qts, qhs, ots, ohs;
    long long kps, kts, khs, vps, vts, vhs;
    const int *cu_q, *kv_len, *table;
    long long table_stride, n_pages;
    int n_seqs, max_pages, page_size;
    int n_tokens, hq, hk, group, dim;
    int causal, window;
    float scale_log2;                  // scores in units of ln 2: exponentials are powers of two
    int32_t *status;
};

constexpr float kLn2 = 0.693147180559945309f;

// The keys [lo, hi) that the token at position p may see.
__device__ __forceinline__ void key_range(const AttnArgs &g, long long p, int kv_len, int &lo, int &hi)
{
    hi = g.causal ? (int)(p + 1 < kv_len ? p + 1 : kv_len) : kv_len;
    lo = g.window >= 0 && p > g.window ? (int)(p - g.window) : 0;
    if (hi < 0 || p < 0) hi = 0;
}

// paged_attention_tc.cu
bool attention_tc_takes(const AttnArgs &g);
size_t attention_tc_workspace_bytes();
fpsk_status attention_tc_launch(const AttnArgs &g, int type, int max_q_len, int max_kv_len, void *ws, cudaStream_t st);

// Checks shared by the entry points (attention_api.cu).
bool elem_ok(int type);
bool head_dim_ok(int dim);
fpsk_status check_cache(const fpsk_paged_cache *c);
fpsk_status check_batch(const fpsk_paged_batch *b);

}  // namespace fpsk
