#include "us_ops.h"

#include <cstdlib>
#include <mutex>
#include <new>
#include <set>
#include <utility>

namespace us {

namespace {
// programmatic dependent launch: environment US_PDL, read once per process, as for the other kernels
bool pdl()
{
    static const bool on = [] { const char* v = std::getenv("US_PDL"); return !(v && *v) || std::atoi(v) != 0; }();
    return on;
}
std::mutex g_lock;
std::set<std::pair<int, const void*>> g_allowed;
int g_sms[kMaxDevices];
}  // namespace

cudaError_t ops_launch(const void* kernel, dim3 grid, int block, int64_t smem, cudaStream_t st, void** args, unsigned cluster)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    forget_last_call();
    return cudaLaunchKernelExC(&cfg, kernel, args);
}

cudaError_t ops_kernel_allow(const void* kernel, int most)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> hold(g_lock);
    if (g_allowed.count({dev, kernel})) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    try {
        g_allowed.insert({dev, kernel});
    } catch (const std::bad_alloc&) {   // (the next call sets the attributes again)
    }
    return e;
}

cudaError_t ops_symbol(void** kept, const void* symbol, void** address)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaGetSymbolAddress(address, symbol);
    std::lock_guard<std::mutex> hold(g_lock);
    if (!kept[dev]) e = cudaGetSymbolAddress(&kept[dev], symbol);
    *address = kept[dev];
    return e;
}

int ops_sms()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return 148; }
    std::lock_guard<std::mutex> hold(g_lock);
    if (!g_sms[dev] && cudaDeviceGetAttribute(&g_sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 148; }
    return g_sms[dev];
}

}  // namespace us
