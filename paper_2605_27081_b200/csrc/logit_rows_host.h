// Host side shared by the operators on rows of logits: argument checks, the device of a call, launches.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "remoe.h"
#include "remoe_internal.cuh"

namespace remoe {
namespace rows {

// Makes the device of `ptr` current for the call and puts the caller's back; err_code() tells a pointer that is no
// device memory (REMOE_E_ARG) from a failing runtime call (REMOE_E_CUDA).
class PointerDevice {
 public:
  explicit PointerDevice(const void* ptr) {
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, ptr) != cudaSuccess) {
      cudaGetLastError();
      code_ = REMOE_E_CUDA;
      return;
    }
    if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) {
      code_ = REMOE_E_ARG;
      return;
    }
    if (cudaGetDevice(&prev_) != cudaSuccess) { code_ = REMOE_E_CUDA; return; }
    device_ = at.device;
    if (prev_ != device_) {
      if (cudaSetDevice(device_) != cudaSuccess) { code_ = REMOE_E_CUDA; return; }
      switched_ = true;
    }
  }
  ~PointerDevice() {
    if (switched_) cudaSetDevice(prev_);
  }
  PointerDevice(const PointerDevice&) = delete;
  PointerDevice& operator=(const PointerDevice&) = delete;
  int err_code() const { return code_; }

 private:
  int prev_ = -1, device_ = -1, code_ = REMOE_OK;
  bool switched_ = false;
};

constexpr int64_t kSliceBytes = 52 * 1024;     // of a row in one block, where eight blocks are enough for that
constexpr size_t kSmemLimit = 220 * 1024;      // dynamic shared memory of a block; the longest float32 row needs 216 KB in eight

// Range of the inverse temperature.  Above, its product with log2(e) leaves float32 from 2.36e38 on (0 * inf for the largest element); below,
// a difference of logits beyond float32 may still be a distance that counts, where it reads as -inf (from about 3e-37 on).
constexpr float kLeastInverse = 0x1p-100f, kLargestInverse = 0x1p100f;

inline int element_size(int32_t dtype) { return dtype == REMOE_F32 ? 4 : dtype == REMOE_BF16 || dtype == REMOE_F16 ? 2 : 0; }
inline bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// More blocks than a grid holds (cudaErrorInvalidConfiguration) is a shape that the kernels are not built for.
inline int status(cudaError_t e) { return e == cudaSuccess ? REMOE_OK : e == cudaErrorInvalidConfiguration ? REMOE_E_UNSUPPORTED : REMOE_E_CUDA; }

// What every operator asks of its rows.
inline int check_rows(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t row_stride, float inv_temperature) {
  if (n_rows < 0 || vocab < 1 || !logits) return REMOE_E_ARG;
  if (dtype == REMOE_FP8_E4M3 || dtype == REMOE_INT4_G32) return REMOE_E_UNSUPPORTED;
  if (!element_size(dtype)) return REMOE_E_ARG;
  if (vocab > REMOE_ROWS_MAX_VOCAB) return REMOE_E_UNSUPPORTED;
  if (row_stride < vocab && n_rows > 1) return REMOE_E_ARG;
  if (!(inv_temperature >= kLeastInverse && inv_temperature <= kLargestInverse)) return REMOE_E_ARG;      // NaN, too
  if (misaligned(logits, element_size(dtype))) return REMOE_E_ARG;
  return REMOE_OK;
}

// Blocks that share a row, one part of it in the shared memory of each: a power of two up to eight, so that four blocks
// of 256 threads lie on an SM with 52 KB each (three where the selection's lists, 19 KB, lie behind the part); more where there are few
// rows, down to 8 KB.
inline int parts_of_row(int32_t n_rows, int32_t vocab, int size) {
  int parts = 1;
  while (parts < 8 && (int64_t)vocab * size > (int64_t)parts * kSliceBytes) parts *= 2;
  while (parts < 8 && (int64_t)n_rows * parts < 296 && (int64_t)vocab * size > (int64_t)parts * 16384) parts *= 2;
  return parts;
}
// Shared memory of a part: whole units of eight elements, whatever the row's alignment.
inline int slice_bytes(int32_t vocab, int size, int parts) { return ((vocab + 14) / 8 + parts - 1) / parts * 8 * size; }

// One launch in clusters of `parts` blocks.  Its status is the launch's own, whatever an earlier call has left in the runtime's error state.
template <auto Kernel, typename Args>
inline cudaError_t launch(const Args& args, int64_t blocks, int parts, int threads, size_t smem, cudaStream_t stream) {
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)parts;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, Kernel, args);
}

// One launch of `Kernel`, a cluster of args.parts blocks for each row.
template <auto Kernel, int NT, typename Args>
inline cudaError_t launch_resident(const Args& args, size_t more_smem, cudaStream_t stream) {
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(Kernel, kSmemLimit, ready);
  if (e != cudaSuccess) return e;
  return launch<Kernel>(args, (int64_t)args.n_rows * args.parts, args.parts, NT, (size_t)args.slice_bytes + more_smem, stream);
}

// Rows enough for persistent blocks that take whole rows: one for each SM.  (257 rows of 50257 fp16 with 5 alternatives: 16 us this
// way, one row a block, 19 with a cluster a row; 2048 of 131072 bf16 with 64: 135 against 568, since each of a row's blocks selects as
// much as one for the whole row would.)  Shorter rows are over before such a block's warps have handed them on.
inline bool many_rows(int32_t n_rows, int32_t vocab) { return vocab >= 8192 && n_rows >= 148; }

// One launch of persistent blocks.
template <auto Kernel, typename Shape, typename Args>
inline cudaError_t launch_pipe(const Args& args, cudaStream_t stream) {
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(Kernel, Shape::kSmem, ready);
  if (e != cudaSuccess) return e;
  const int most = 148 * Shape::kBlocks;
  return launch<Kernel>(args, args.n_rows < most ? args.n_rows : most, 1, Shape::kThreads, Shape::kSmem, stream);
}

// Blocks a row for the element-wise passes: of about `piece` bytes each.  (The distillation's gradient with 128 entries a row, 2048 x
// 131072 bf16: 402 us in pieces of 16 KB, each of which reads the list, 264 of 32, 212 of 128.)
inline int pieces_of_row(int32_t vocab, int size, int piece) {
  const int64_t bytes = (int64_t)vocab * size;
  return (int)(bytes <= piece ? 1 : (bytes + piece / 2) / piece);
}

}  // namespace rows
}  // namespace remoe
