// Host side of the tensor-core units: the driver's encoder of tensor maps.
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
