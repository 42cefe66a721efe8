// What the decoder's operators ask the device for on the host, and what they count for their tests.
#include "add_norm.cuh"
#include "fpsk_test.h"

#include <atomic>
#include <mutex>

namespace fpsk {

cudaError_t clusters_at_once(const void *kernel, const cudaLaunchConfig_t &cfg, int *out)
{
    struct Key {
        const void *kernel;
        int device, blocks, threads;
        size_t bytes;
    };
    static std::mutex lock;
    static Key keys[64];
    static int values[64], used = 0;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int blocks = (int)cfg.attrs[0].val.clusterDim.x;
    std::lock_guard<std::mutex> hold(lock);
    for (int i = 0; i < (used < 64 ? used : 64); ++i)
        if (keys[i].kernel == kernel && keys[i].device == device && keys[i].blocks == blocks && keys[i].threads == (int)cfg.blockDim.x && keys[i].bytes == cfg.dynamicSmemBytes) {
            *out = values[i];
            return cudaSuccess;
        }
    cudaFuncAttributes a;
    e = cudaFuncGetAttributes(&a, kernel);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)a.sharedSizeBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(out, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (*out < 1) *out = 1;
    keys[used % 64] = Key{kernel, device, blocks, (int)cfg.blockDim.x, cfg.dynamicSmemBytes};
    values[used % 64] = *out;
    ++used;
    return cudaSuccess;
}

static std::atomic<uint64_t> g_rings{0};
void count_ring() { g_rings.fetch_add(1, std::memory_order_relaxed); }

}  // namespace fpsk

extern "C" uint64_t fpsk_norm_ring_count(void) { return fpsk::g_rings.load(); }
