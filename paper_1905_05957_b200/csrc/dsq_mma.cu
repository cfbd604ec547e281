// Host side of the tensor-core products: tensor maps and the device's number of SMs.
#include "dsq_mma.cuh"

namespace dsq {

namespace {
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, asked for by name so that the library links against the runtime alone.
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}
}  // namespace

int sm_count() {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 148;
  n = known[dev].load(std::memory_order_relaxed);
  if (!n) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 148;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

namespace {
constexpr size_t kProbeSmem = 226 * 1024;     // about what the kernels take: one CTA an SM
__global__ void __launch_bounds__(kMmaThreads, 1) k_cluster_probe() {}   // never launched: asked about
}

int cluster_count(uint32_t size) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices][9];
  int dev = 0, n = 0;
  if (size < 2 || size > 8 || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  n = known[dev][size].load(std::memory_order_relaxed);
  if (!n) {
    (void)cudaFuncSetAttribute(k_cluster_probe, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProbeSmem);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(size * (sm_count() / size));
    cfg.blockDim = dim3(kMmaThreads);
    cfg.dynamicSmemBytes = kProbeSmem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = size;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, k_cluster_probe, &cfg) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      n = sm_count() / (int)size;
    }
    known[dev][size].store(n, std::memory_order_relaxed);
  }
  return n;
}

cudaError_t make_tensor_map(CUtensorMap* map, int kind, const void* base, uint64_t cols, uint64_t rows, uint64_t batch, uint64_t ld,
                            uint64_t batch_stride, uint32_t box_cols, uint32_t box_rows, bool block) {
  const EncodeFn fn = encoder();
  if (!fn) return cudaErrorNotSupported;
  const uint64_t size = kind != kMmaI8 ? 2 : 1;
  const cuuint64_t dims[3] = {cols, rows, batch};
  const cuuint64_t strides[2] = {ld * size, batch_stride * size};   // bytes, of the second and the third dimension
  const cuuint32_t box[3] = {box_cols, box_rows, 1};
  const cuuint32_t step[3] = {1, 1, 1};
  const CUresult r = fn(map, kind != kMmaI8 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 3,
                        const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        block ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace dsq
