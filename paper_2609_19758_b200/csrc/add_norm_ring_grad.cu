// The backward pass of residual addition and norm through the ring.
#include "add_norm_ring.cuh"

namespace fpsk {

bool norm_grad_ring(const NormGradArgs &g, bool wide, int h_type, int grad_type, int32_t *d_status, cudaStream_t st, fpsk_status *rc, int *rows)
{
    RingArgs r = {};
    const bool whole = wide && g.dim % 8 == 0;
    r.b = g;
    r.in[0] = ring_rows(g.h, g.hs, h_type);
    r.in[1] = ring_rows(g.dy, g.dys, grad_type);
    r.in[2] = ring_rows(g.dh, g.dhs, grad_type);
    r.inputs = g.dh ? 3 : 2;
    r.n = g.n;
    r.status = d_status;
    int threads;
    if (!ring_plan(r, g.dim, whole, threads)) return false;
#define FPSK_IN(G)                                                                             \
    (h_type == FPSK_ELEM_FP32 ? launch_ring<float, G, true>(r, whole, threads, *rows, st)      \
                              : h_type == FPSK_ELEM_FP16 ? launch_ring<__half, G, true>(r, whole, threads, *rows, st) : launch_ring<__nv_bfloat16, G, true>(r, whole, threads, *rows, st))
    *rc = grad_type == FPSK_ELEM_FP32 ? FPSK_IN(float) : grad_type == FPSK_ELEM_FP16 ? FPSK_IN(__half) : FPSK_IN(__nv_bfloat16);
#undef FPSK_IN
    return true;
}

}  // namespace fpsk
