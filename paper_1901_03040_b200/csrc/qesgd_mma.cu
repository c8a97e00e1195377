// Host side of the tensor-core units: the driver's encoder of tensor maps, how many clusters a device runs at once.
#include <mutex>

#include "qesgd_mma.cuh"

QesgdEncodeTiledFn qesgd_encode_tiled()
{
    static std::mutex mutex;
    static QesgdEncodeTiledFn encode = nullptr;
    std::lock_guard<std::mutex> lock(mutex);
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            encode = (QesgdEncodeTiledFn)fn;
        else
            cudaGetLastError();
    }
    return encode;
}

uint32_t qesgd_active_clusters(QesgdClusters &known, const void *kernel, uint32_t threads, uint32_t smem, uint32_t cluster)
{
    static std::mutex mutex;
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64 || cluster < 1 || cluster > 16) return 1;
    std::lock_guard<std::mutex> lock(mutex);
    int &n = known.count[device][cluster];
    if (n == 0) {
        cudaLaunchConfig_t c = {};
        c.gridDim = dim3(cluster);
        c.blockDim = dim3(threads);
        c.dynamicSmemBytes = smem;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = cluster;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        c.attrs = at;
        c.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &c) != cudaSuccess || n < 1) {
            cudaGetLastError();
            n = 1;
        }
    }
    return (uint32_t)n;
}
