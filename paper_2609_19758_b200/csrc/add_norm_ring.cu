// The forward pass of residual addition and norm through the ring.
#include "add_norm_ring.cuh"

namespace fpsk {

bool norm_ring(const NormArgs &g, bool wide, int x_type, int res_type, int32_t *d_status, cudaStream_t st, fpsk_status *rc)
{
    RingArgs r = {};
    const bool whole = wide && g.dim % 8 == 0;
    if (g.ytype == FPSK_ELEM_E4M3 && !whole) return false;             // (a group's channels lie in neighbouring lanes)
    r.f = g;
    r.in[0] = ring_rows(g.x, g.xs, x_type);
    r.in[1] = ring_rows(g.res, g.rs, res_type);
    r.inputs = g.res ? 2 : 1;
    r.n = g.n;
    r.status = d_status;
    int threads, rows;
    if (!ring_plan(r, g.dim, whole, threads)) return false;
#define FPSK_RES(X)                                                                           \
    (res_type == FPSK_ELEM_FP32 ? launch_ring<X, float, false>(r, whole, threads, rows, st)   \
                                : res_type == FPSK_ELEM_FP16 ? launch_ring<X, __half, false>(r, whole, threads, rows, st) : launch_ring<X, __nv_bfloat16, false>(r, whole, threads, rows, st))
    *rc = x_type == FPSK_ELEM_FP32 ? FPSK_RES(float) : x_type == FPSK_ELEM_FP16 ? FPSK_RES(__half) : FPSK_RES(__nv_bfloat16);
#undef FPSK_RES
    return true;
}

}  // namespace fpsk
