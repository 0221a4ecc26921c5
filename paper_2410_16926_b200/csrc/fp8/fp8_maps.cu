// Host side of the tensor-core kernels: maps of matrices for tiled copies, shared memory limits.
#include <dlfcn.h>

#include <map>
#include <mutex>
#include <utility>

#include "fp8_mma.cuh"

namespace pvq {
namespace fp8 {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's function, looked up by name: the library links with no driver, so that it loads where there is none.
static EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* driver = dlopen("libcuda.so.1", RTLD_NOW | RTLD_LOCAL);
        return driver ? reinterpret_cast<EncodeTiled>(dlsym(driver, "cuTensorMapEncodeTiled")) : nullptr;
    }();
    return f;
}

int tile_map(CUtensorMap* map, const void* p, Element type, int64_t rows, int64_t cols, int64_t ld, int box_x, int box_y) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return set_cuda_error(cudaErrorInitializationError);
    const int size = type == Element::kByte ? 1 : (type == Element::kBf16 ? 2 : 4);
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld) * size};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_x), static_cast<cuuint32_t>(box_y)}, steps[2] = {1, 1};
    const CUtensorMapDataType t = type == Element::kByte ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                                         : (type == Element::kBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32);
    const CUresult r = encode(map, t, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PVQ_OK : set_cuda_error(cudaErrorInvalidValue);
}

int allow_shared(const void* kernel, size_t bytes) {
    static std::mutex mu;
    static std::map<std::pair<const void*, int>, size_t> allowed;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return set_cuda_error(e);
    std::lock_guard<std::mutex> lock(mu);
    size_t& most = allowed[{kernel, dev}];
    if (bytes <= most) return PVQ_OK;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e != cudaSuccess) return set_cuda_error(e);
    most = bytes;
    return PVQ_OK;
}

int registers_of(const void* kernel, int* registers) {
    static std::mutex mu;
    static std::map<std::pair<const void*, int>, int> memo;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return set_cuda_error(e);
    std::lock_guard<std::mutex> lock(mu);
    int& known = memo[{kernel, dev}];
    if (known == 0) {
        cudaFuncAttributes a;
        e = cudaFuncGetAttributes(&a, kernel);
        if (e != cudaSuccess) return set_cuda_error(e);
        known = a.numRegs;
    }
    *registers = known;
    return PVQ_OK;
}

int clusters_of(const void* kernel, unsigned threads, size_t shared, unsigned size, int* clusters) {
    static std::mutex mu;
    static std::map<std::pair<const void*, int>, int> memo;  // (threads and shared memory are a kernel's own)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return set_cuda_error(e);
    std::lock_guard<std::mutex> lock(mu);
    int& known = memo[{kernel, dev * 16 + static_cast<int>(size)}];
    if (known == 0) {
        cudaLaunchConfig_t config = {};
        config.gridDim = dim3(size);
        config.blockDim = dim3(threads);
        config.dynamicSmemBytes = shared;
        cudaLaunchAttribute cluster;
        cluster.id = cudaLaunchAttributeClusterDimension;
        cluster.val.clusterDim.x = size, cluster.val.clusterDim.y = 1, cluster.val.clusterDim.z = 1;
        config.attrs = &cluster;
        config.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&known, kernel, &config);
        if (e != cudaSuccess) {
            known = 0;
            return set_cuda_error(e);
        }
        if (known < 1) known = 1;
    }
    *clusters = known;
    return PVQ_OK;
}

}  // namespace fp8
}  // namespace pvq
