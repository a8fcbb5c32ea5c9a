// What the host sides of the single layers' calls share.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/iodf.h"

namespace iodf {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline int status_of(cudaError_t e) {
  return e == cudaSuccess ? IODF_OK : e == cudaErrorMemoryAllocation ? IODF_ENOMEM : IODF_ECUDA;
}

// Makes the handle's device current for the duration of a call.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    err_ = cudaGetDevice(&prev_);
    if (err_ == cudaSuccess && prev_ != device) {
      err_ = cudaSetDevice(device);
      restore_ = err_ == cudaSuccess;
    }
  }
  ~OnDevice() { if (restore_) cudaSetDevice(prev_); }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  cudaError_t error() const { return err_; }

 private:
  int prev_ = -1;
  bool restore_ = false;
  cudaError_t err_;
};

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline size_t up_to(size_t n, size_t m) { return (n + m - 1) / m * m; }

// The driver's cuTensorMapEncodeTiled, NULL if it has none.
inline EncodeTiled tensor_map_encoder() {
  cudaDriverEntryPointQueryResult found;
  void* entry = nullptr;
  const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &entry, 12000, cudaEnableDefault, &found);
  return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(entry) : nullptr;
}

}  // namespace iodf
