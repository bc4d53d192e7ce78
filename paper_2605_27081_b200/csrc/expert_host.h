// Host side shared by the operators on tokens sorted by expert: argument checks and entry points of the driver.
#pragma once

#include <cuda.h>

#include <atomic>
#include <initializer_list>

#include "logit_rows_host.h"

namespace remoe {
namespace sorted {

// A matrix of `n` rows: its address, the distance of its rows, and the alignment that its type asks for.  One without rows may be null.
inline bool bad_matrix(const void* p, int64_t stride, int64_t n, int64_t columns, int size) {
  return (!p && n > 0) || rows::misaligned(p, size) || (n > 1 && stride < columns);
}

// Widest access (16 bytes at most) that every row of a matrix starts on.
inline int access_width(const void* p, int64_t stride, int64_t n, int size) {
  const uint64_t bits = reinterpret_cast<uintptr_t>(p) | (n > 1 ? (uint64_t)stride * size : 0) | 16;
  return (int)(bits & (~bits + 1));
}

// An entry point of the driver, looked up once.
template <typename Fn>
inline cudaError_t driver_entry(const char* name, std::atomic<void*>* known, Fn* out) {
  void* fn = known->load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint(name, &fn, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (!fn) return cudaErrorNotSupported;
    known->store(fn, std::memory_order_release);
  }
  *out = reinterpret_cast<Fn>(fn);
  return cudaSuccess;
}

// Refuses buffers (null: none) in memory of the host, which a kernel would fault on, or read over the bus where it is page-locked.  45 ns each; the
// runtime's query, which tells the device as well, takes 68.
inline int check_device_memory(std::initializer_list<const void*> buffers) {
  static std::atomic<void*> known{nullptr};
  CUresult (*attribute)(void*, CUpointer_attribute, CUdeviceptr);
  if (driver_entry("cuPointerGetAttribute", &known, &attribute) != cudaSuccess) return REMOE_E_CUDA;
  for (const void* p : buffers) {
    CUmemorytype type;
    if (p && (attribute(&type, CU_POINTER_ATTRIBUTE_MEMORY_TYPE, reinterpret_cast<CUdeviceptr>(p)) != CUDA_SUCCESS || type == CU_MEMORYTYPE_HOST)) return REMOE_E_ARG;
  }
  return REMOE_OK;
}

}  // namespace sorted
}  // namespace remoe
