// Host side of the tensor-core products: tensor maps, launches, the SM count.
#pragma once

#include <atomic>
#include <utility>

#include "host_common.cuh"
#include "tensor_core.cuh"

namespace fopd {

using TensorMapEncode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                     const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                     CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// (the driver's entry point by way of the runtime: the library links against no driver library)
inline TensorMapEncode tensor_map_encode() {
  static std::atomic<void *> entry{nullptr};
  void *fn = entry.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return nullptr;
    }
    entry.store(fn, std::memory_order_release);
  }
  return reinterpret_cast<TensorMapEncode>(fn);
}

// [rows, cols] elements at a pitch in bytes (a multiple of 16, base 16-byte aligned); boxes of box_rows x 128 bytes, swizzled.
inline int make_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t cols, int64_t rows, int64_t pitch_bytes,
                    int box_cols, int box_rows) {
  TensorMapEncode encode = tensor_map_encode();
  if (!encode) return FOPD_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, unit[2] = {1, 1};
  return encode(map, type, 2, const_cast<void *>(base), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? FOPD_OK
             : FOPD_ERR_CUDA;
}

inline int current_sms(int *sms) {
  static std::atomic<int> known[kMaxDevices];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return FOPD_ERR_CUDA;
  *sms = known[dev].load(std::memory_order_relaxed);
  if (*sms == 0) {
    if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return FOPD_ERR_CUDA;
    known[dev].store(*sms, std::memory_order_relaxed);
  }
  return FOPD_OK;
}

// Launches a job on up to one CTA (pair) per SM (pair); most_tiles: at least as many as the job will have.
template <int kCtas, int kN, class Job>
int launch_product(const typename Job::Params &params, int64_t most_tiles, int sms, cudaStream_t st) {
  using Shape = ProductShape<kCtas, kN>;
  auto *kernel = product_kernel<kCtas, kN, Job>;
  static std::atomic<bool> ready[kMaxDevices];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return FOPD_ERR_CUDA;
  if (!ready[dev].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem) != cudaSuccess) {
      (void)cudaGetLastError();
      return FOPD_ERR_CUDA;
    }
    ready[dev].store(true, std::memory_order_relaxed);
  }
  if (most_tiles <= 0) return FOPD_OK;
  const int64_t groups = most_tiles < sms / kCtas ? most_tiles : sms / kCtas;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * kCtas));
  cfg.blockDim = dim3(kProductThreads);
  cfg.dynamicSmemBytes = Shape::kSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = kCtas > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, params) != cudaSuccess) {
    (void)cudaGetLastError();
    return FOPD_ERR_CUDA;
  }
  return FOPD_OK;
}

// Any other kernel of a call, launched early as well (it begins with grid_wait).
template <class... Params, class... Args>
int launch_early(void (*kernel)(Params...), dim3 grid, int threads, cudaStream_t st, Args &&...args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) != cudaSuccess) {
    (void)cudaGetLastError();
    return FOPD_ERR_CUDA;
  }
  return FOPD_OK;
}

static inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Parts of one temporary, each 256-byte aligned.
struct Layout {
  int64_t bytes = 0;
  int64_t take(int64_t n) {
    const int64_t at = bytes;
    bytes += round_up(n, 256);
    return at;
  }
};

}  // namespace fopd
