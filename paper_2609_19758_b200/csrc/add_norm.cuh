// Shared by the forms of the residual addition and norm (add_norm.cu, add_norm_ring.cuh): their arguments, and the scales of 8-bit outputs.
#pragma once
#include "decoder.cuh"

#include <cuda_fp8.h>

namespace fpsk {

struct NormArgs {
    const void *x, *res, *w;
    void *hout, *y;
    float *scale;
    long long xs, rs, hs, ys, ss;
    long long n;
    int dim, wtype, ytype, group;      // group: 0 or a power of two
    int warps;                         // of a row
    float eps, inv_dim;
};
struct NormGradArgs {
    const void *h, *dy, *dh, *w;
    void *dx;
    float *part;                       // [row teams][dim]
    long long hs, dys, dhs, dxs;
    long long n;
    int dim, wtype;
    int warps;
    float eps, inv_dim;
};

__device__ __forceinline__ unsigned int magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// The scale of a group whose largest magnitude has these bits, and one over it: a product and an approximate reciprocal (one unit), as
// two divisions for every eight channels took a fifth of the kernel.
__device__ __forceinline__ float e4m3_scale(unsigned int top)
{
    if (top == 0) return 1.f;
    const float s = __uint_as_float(top) * (1.f / 448.f);
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;                  // (a NaN stays)
}
__device__ __forceinline__ float over(float scale)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
    return r;
}
__device__ __forceinline__ unsigned int e4m3_pair(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// add_norm_ring.cu, add_norm_ring_grad.cu: true where the ring takes the call (*rc is its status then); `rows` of partial weight gradients
// are left in g.part.
void count_ring();
bool norm_ring(const NormArgs &g, bool wide, int x_type, int res_type, int32_t *d_status, cudaStream_t st, fpsk_status *rc);
bool norm_grad_ring(const NormGradArgs &g, bool wide, int h_type, int grad_type, int32_t *d_status, cudaStream_t st, fpsk_status *rc, int *rows);

}  // namespace fpsk
