// Host-side helpers shared by the training operators: device check, tensor-map encoding, launches.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "adacons.h"
#include "adacons_common.cuh"
#include "adacons_status.cuh"

namespace adacons {

// What the operators need to know of the current device; looked up once per device.
struct DeviceInfo { int device = -1, sms = 0; TensorMapEncoder encode; };

inline int query_device(DeviceInfo* info) {
  int dev = 0, major = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return ADACONS_ECUDA;
  }
  if (major != 10) return ADACONS_EARCH;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess) {
    cudaGetLastError();
    return ADACONS_ECUDA;
  }
  info->device = dev;
  info->sms = sms;
  info->encode.fn = reinterpret_cast<TensorMapEncodeFn>(fn);
  return ADACONS_OK;
}

// The multiprocessors of the current device, for operators that need no more of it.
inline int device_sms(int* sms) {
  static std::mutex mutex;
  static int known[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  if (dev < 0 || dev >= 64) return ADACONS_ELIMIT;
  std::lock_guard<std::mutex> lock(mutex);
  if (known[dev] == 0) {
    DeviceInfo info;
    const int rc = query_device(&info);
    if (rc != ADACONS_OK) return rc;
    known[dev] = info.sms;
  }
  *sms = known[dev];
  return ADACONS_OK;
}

inline bool encode_map(const DeviceInfo& info, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims,
                       const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
  return info.encode(map, type, static_cast<cuuint32_t>(rank), const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

enum LaunchKind { kLaunchPlain = 0, kLaunchOverlap = 1, kLaunchCooperative = 2 };   // overlap: programmatic stream serialisation
template <typename... Params, typename... Args>
inline bool launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, LaunchKind kind, int cluster, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  if (kind == kLaunchOverlap) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (kind == kLaunchCooperative) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeCooperative;
    attr[cfg.numAttrs++].val.cooperative = 1;
  }
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[cfg.numAttrs].val.clusterDim.y = 1;
    attr[cfg.numAttrs++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return true;
  cudaGetLastError();
  return false;
}

}  // namespace adacons
