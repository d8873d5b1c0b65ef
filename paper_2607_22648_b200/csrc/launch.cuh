// Host side of the attention kernels: the current GPU, shared-memory limits, tensor maps.
#pragma once
#include <atomic>

#include <cuda.h>

#include "attend_split.cuh"

namespace ptk {

struct Gpu { int dev, sms; };
inline int current_gpu(Gpu* g) {
  if (cudaGetDevice(&g->dev) != cudaSuccess || cudaDeviceGetAttribute(&g->sms, cudaDevAttrMultiProcessorCount, g->dev) != cudaSuccess || g->sms <= 0) {
    (void)cudaGetLastError();
    return PTSTORE_E_CUDA;
  }
  if (g->sms > MAX_SMS) g->sms = MAX_SMS;    // a B200 has 148; the workspace does not depend on the device
  return PTSTORE_OK;
}

// Lets a kernel use its shared memory, once per device (the setting belongs to the device; concurrent first calls set it twice).
template <typename F>
int allow_smem(F* kernel, int bytes, std::atomic<u64>& devices, int dev) {
  const u64 bit = 1ull << (dev & 63);
  if (dev < 64 && (devices.load(std::memory_order_acquire) & bit)) return PTSTORE_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    (void)cudaGetLastError();
    return PTSTORE_E_CUDA;
  }
  if (dev < 64) devices.fetch_or(bit, std::memory_order_release);
  return PTSTORE_OK;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {                 // null where the driver has none
  static std::atomic<void*> entry{nullptr};
  void* fn = entry.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &got) != cudaSuccess || got != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return nullptr;
    }
    entry.store(fn, std::memory_order_release);
  }
  return reinterpret_cast<EncodeTiled>(fn);
}
inline bool encode(CUtensorMap* map, bool half, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* boxes) {
  const EncodeTiled fn = encode_tiled();
  const cuuint32_t steps[5] = {1, 1, 1, 1, 1};
  return fn && fn(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace ptk
