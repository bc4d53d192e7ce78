// Tokens sorted by expert and back: the order of the selections, rows out to their experts, the weighted sum of a
// token's rows, and its backward pass.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "expert_host.h"

namespace cg = cooperative_groups;

namespace remoe {
namespace {

// ------------------------------------------------------------------------------------------------------------ sort
// Row of selection s = (selections of lower experts) + (earlier selections of its own).  One cluster: every warp takes a run of
// consecutive selections and counts them by expert (lanes with the same expert find one another with match.any, so a
// counter has one writer at a time), the counts are summed over the warps and, through distributed shared memory, over
// the blocks, and a second walk over the same selections hands out the rows.  Integers only, the same order every time.
struct SortArgs {
  const int* ids;
  int* rows;
  int* offsets;
  int n, n_experts, run;                 // selections, experts, selections of one warp (a multiple of 32)
};

constexpr int kSortWarps = 32;

__global__ void __launch_bounds__(kSortWarps * 32) sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ int sort_smem[];
  const int N = a.n_experts, W = blockDim.x >> 5;
  int* total = sort_smem;                // [N] of this block
  int* base = total + N;                 // [N] first row of an expert's selections in this block
  int* every = base + N;                 // [N] of all blocks, then the first row of the expert
  int* count = every + N;                // [W][N]
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t begin = ((int64_t)rank * W + warp) * a.run;
  const int64_t end = begin + a.run < a.n ? begin + a.run : a.n;
  int* mine = count + warp * N;

  for (int i = threadIdx.x; i < W * N; i += blockDim.x) count[i] = 0;
  __syncthreads();
  for (int64_t s0 = begin; s0 < end; s0 += 32) {
    const int id = s0 + lane < end ? __ldg(a.ids + s0 + lane) : -1;
    const bool valid = (unsigned)id < (unsigned)N;
    const unsigned peers = __match_any_sync(0xffffffffu, valid ? id : -1);
    if (valid && lane == __ffs(peers) - 1) mine[id] += __popc(peers);
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < N; e += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < W; ++w) {
      const int c = count[w * N + e];
      count[w * N + e] = sum;
      sum += c;
    }
    total[e] = sum;
  }
  cluster.sync();
  for (int e = threadIdx.x; e < N; e += blockDim.x) {
    int before = 0, all = 0;
    for (int b = 0; b < blocks; ++b) {
      const int c = *cluster.map_shared_rank(total + e, b);
      before += b < rank ? c : 0;
      all += c;
    }
    base[e] = before;
    every[e] = all;
  }
  cluster.sync();                        // no block leaves while another reads its counts
  if (warp == 0) {                       // running sum over the experts, a piece for each lane
    const int per = (N + 31) / 32, e0 = min(N, lane * per), e1 = min(N, e0 + per);
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += every[e];
    int upto = sum;
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    int first = upto - sum;
    for (int e = e0; e < e1; ++e) {
      const int c = every[e];
      every[e] = first;
      if (rank == 0) a.offsets[e] = first;
      first += c;
    }
    if (rank == 0 && lane == 31) a.offsets[N] = upto;
  }
  __syncthreads();
  for (int64_t s0 = begin; s0 < end; s0 += 32) {
    const bool there = s0 + lane < end;
    const int id = there ? __ldg(a.ids + s0 + lane) : -1;
    const bool valid = (unsigned)id < (unsigned)N;
    const unsigned peers = __match_any_sync(0xffffffffu, valid ? id : -1);
    int row = -1;
    if (valid) row = every[id] + base[id] + mine[id] + __popc(peers & ((1u << lane) - 1));
    __syncwarp();
    if (valid && lane == __ffs(peers) - 1) mine[id] += __popc(peers);
    __syncwarp();
    if (there) a.rows[s0 + lane] = row;
  }
}

// ------------------------------------------------------------------------------------------- rows out, rows back
template <int BYTES> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = unsigned; };
template <> struct Word<2> { using type = unsigned short; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// V consecutive elements of a row as one access.
template <typename T, int V>
struct Vec {
  using W = typename Word<V * (int)sizeof(T)>::type;
  union {
    W word;
    T e[V];
  };
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ void load(const T* p) { word = *reinterpret_cast<const W*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<W*>(p) = word; }
};

struct RowArgs {
  const void* a;                         // dispatch: x; combine: the experts' rows; its backward pass: the experts' rows
  int64_t a_stride;
  const void* b;                         // combine: base or null; backward pass: gradient of the sum
  int64_t b_stride;
  void* out;                             // dispatch: the experts' rows; combine: the sum; backward pass: gradient of the rows or null
  int64_t out_stride;
  const int* rows;                       // [tokens, K]
  const float* gates;                    // [tokens, K] or null
  float* d_gates;                        // [tokens, K] or null
  int K, H, n_rows;
};

constexpr int kGroup = 8;                // rows of a token whose loads are under way together

// One block a token: its row is read once and written to the places of its selections.
template <typename T, int V>
__global__ void __launch_bounds__(256) dispatch_kernel(const __grid_constant__ RowArgs a) {
  const int64_t t = blockIdx.x;
  const int* rows = a.rows + t * a.K;
  const T* x = static_cast<const T*>(a.a) + t * a.a_stride;
  T* out = static_cast<T*>(a.out);
  const int body = a.H / V;
  for (int i = threadIdx.x; i < body; i += blockDim.x) {
    Vec<T, V> v;
    v.load(x + i * V);
    for (int k = 0; k < a.K; ++k) {
      const int r = __ldg(rows + k);
      if ((unsigned)r < (unsigned)a.n_rows) v.store(out + r * a.out_stride + i * V);
    }
  }
  for (int i = body * V + threadIdx.x; i < a.H; i += blockDim.x) {
    const T v = x[i];
    for (int k = 0; k < a.K; ++k) {
      const int r = __ldg(rows + k);
      if ((unsigned)r < (unsigned)a.n_rows) out[r * a.out_stride + i] = v;
    }
  }
}

template <typename T, int V>
__device__ __forceinline__ void combine_piece(const RowArgs& a, int64_t t, int i) {
  const int* rows = a.rows + t * a.K;
  const float* gates = a.gates ? a.gates + t * a.K : nullptr;
  const T* ys = static_cast<const T*>(a.a) + i;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  for (int k0 = 0; k0 < a.K; k0 += kGroup) {
    Vec<T, V> v[kGroup];
    float g[kGroup];
    bool there[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const int r = k0 + k < a.K ? __ldg(rows + k0 + k) : -1;
      there[k] = (unsigned)r < (unsigned)a.n_rows;
      if (there[k]) {
        v[k].load(ys + r * a.a_stride);
        g[k] = gates ? __ldg(gates + k0 + k) : 1.f;
      }
    }
#pragma unroll
    for (int k = 0; k < kGroup; ++k)
      if (there[k]) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = fmaf(g[k], to_float(v[k].e[j]), sum[j]);
      }
  }
  Vec<T, V> o;
  if (a.b) {
    o.load(static_cast<const T*>(a.b) + t * a.b_stride + i);
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += to_float(o.e[j]);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) o.e[j] = from_float<T>(sum[j]);
  o.store(static_cast<T*>(a.out) + t * a.out_stride + i);
}

// One block a token; the rows are added in the order of the selections, in float32.
template <typename T, int V>
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ RowArgs a) {
  const int body = a.H / V;
  for (int i = threadIdx.x; i < body; i += blockDim.x) combine_piece<T, V>(a, blockIdx.x, i * V);
  for (int i = body * V + threadIdx.x; i < a.H; i += blockDim.x) combine_piece<T, 1>(a, blockIdx.x, i);
}

template <typename T, int V>
__device__ __forceinline__ void combine_backward_piece(const RowArgs& a, int64_t t, int k0, int i, float (&dot)[kGroup]) {
  const int* rows = a.rows + t * a.K;
  Vec<T, V> d, v[kGroup];
  int r[kGroup];
  d.load(static_cast<const T*>(a.b) + t * a.b_stride + i);
#pragma unroll
  for (int k = 0; k < kGroup; ++k) {
    r[k] = k0 + k < a.K ? __ldg(rows + k0 + k) : -1;
    if ((unsigned)r[k] >= (unsigned)a.n_rows) r[k] = -1;
    if (a.d_gates && r[k] >= 0) v[k].load(static_cast<const T*>(a.a) + r[k] * a.a_stride + i);
  }
#pragma unroll
  for (int k = 0; k < kGroup; ++k) {
    if (r[k] < 0) continue;
    if (a.d_gates) {
#pragma unroll
      for (int j = 0; j < V; ++j) dot[k] = fmaf(to_float(v[k].e[j]), to_float(d.e[j]), dot[k]);
    }
    if (a.out) {
      const float g = a.gates ? __ldg(a.gates + t * a.K + k0 + k) : 1.f;
      Vec<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.e[j] = from_float<T>(g * to_float(d.e[j]));
      o.store(static_cast<T*>(a.out) + r[k] * a.out_stride + i);
    }
  }
}

// One block a token: the gradient of the sum is read once for up to eight of its rows; each row's scalar product with
// it is summed over the block in a fixed order.
template <typename T, int V>
__global__ void __launch_bounds__(256) combine_backward_kernel(const __grid_constant__ RowArgs a) {
  __shared__ float part[8][kGroup];
  const int64_t t = blockIdx.x;
  const int body = a.H / V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int k0 = 0; k0 < a.K; k0 += kGroup) {
    float dot[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; ++k) dot[k] = 0.f;
    for (int i = threadIdx.x; i < body; i += blockDim.x) combine_backward_piece<T, V>(a, t, k0, i * V, dot);
    for (int i = body * V + threadIdx.x; i < a.H; i += blockDim.x) combine_backward_piece<T, 1>(a, t, k0, i, dot);
    if (!a.d_gates) continue;
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
#pragma unroll
      for (int d = 16; d; d >>= 1) dot[k] += __shfl_xor_sync(0xffffffffu, dot[k], d);
      if (lane == 0) part[warp][k] = dot[k];
    }
    __syncthreads();
    if (threadIdx.x < kGroup && k0 + threadIdx.x < a.K) {
      float sum = 0.f;
      for (int w = 0; w < (int)(blockDim.x >> 5); ++w) sum += part[w][threadIdx.x];
      a.d_gates[t * a.K + k0 + threadIdx.x] = sum;
    }
    __syncthreads();
  }
}

enum Op { kDispatch, kCombine, kCombineBackward };

template <Op OP, typename T, int V>
cudaError_t launch_rows(const RowArgs& a, int n_tokens, cudaStream_t stream) {
  const int pieces = (a.H + V - 1) / V;
  int threads = (pieces + 31) / 32 * 32;
  if (threads > 256) threads = 256;
  if constexpr (OP == kDispatch) return rows::launch<dispatch_kernel<T, V>>(a, n_tokens, 1, threads, 0, stream);
  if constexpr (OP == kCombine) return rows::launch<combine_kernel<T, V>>(a, n_tokens, 1, threads, 0, stream);
  if constexpr (OP == kCombineBackward) return rows::launch<combine_backward_kernel<T, V>>(a, n_tokens, 1, threads, 0, stream);
}

template <Op OP>
int launch_rows(const RowArgs& a, int n_tokens, int32_t dtype, int width, cudaStream_t stream) {
  cudaError_t e = cudaErrorInvalidValue;
  if (dtype == REMOE_F32) {
    switch (width) {
      case 16: e = launch_rows<OP, float, 4>(a, n_tokens, stream); break;
      case 8: e = launch_rows<OP, float, 2>(a, n_tokens, stream); break;
      case 4: e = launch_rows<OP, float, 1>(a, n_tokens, stream); break;
    }
  } else if (dtype == REMOE_BF16) {
    switch (width) {
      case 16: e = launch_rows<OP, __nv_bfloat16, 8>(a, n_tokens, stream); break;
      case 8: e = launch_rows<OP, __nv_bfloat16, 4>(a, n_tokens, stream); break;
      case 4: e = launch_rows<OP, __nv_bfloat16, 2>(a, n_tokens, stream); break;
      case 2: e = launch_rows<OP, __nv_bfloat16, 1>(a, n_tokens, stream); break;
    }
  } else {
    switch (width) {
      case 16: e = launch_rows<OP, __half, 8>(a, n_tokens, stream); break;
      case 8: e = launch_rows<OP, __half, 4>(a, n_tokens, stream); break;
      case 4: e = launch_rows<OP, __half, 2>(a, n_tokens, stream); break;
      case 2: e = launch_rows<OP, __half, 1>(a, n_tokens, stream); break;
    }
  }
  return rows::status(e);
}

int check_rows_call(int32_t n_tokens, int32_t top_k, int32_t hidden, int32_t dtype, const int32_t* rows_dev, int32_t n_rows) {
  if (n_tokens < 0 || top_k < 1 || hidden < 1 || n_rows < 0 || (!rows_dev && n_tokens > 0) || rows::misaligned(rows_dev, 4)) return REMOE_E_ARG;
  if (dtype == REMOE_FP8_E4M3 || dtype == REMOE_INT4_G32) return REMOE_E_UNSUPPORTED;
  if (!rows::element_size(dtype)) return REMOE_E_ARG;
  if ((int64_t)n_tokens * top_k > 0x7fffffff) return REMOE_E_UNSUPPORTED;
  return REMOE_OK;
}

}  // namespace
}  // namespace remoe

using namespace remoe;

extern "C" int remoe_expert_sort(int32_t n_tokens, int32_t top_k, int32_t n_experts, const int32_t* ids_dev, int32_t* rows_dev,
                                 int32_t* offsets_dev, void* cuda_stream) {
  if (n_tokens < 0 || top_k < 1 || n_experts < 1 || !offsets_dev || ((!ids_dev || !rows_dev) && n_tokens > 0)) return REMOE_E_ARG;
  if (rows::misaligned(ids_dev, 4) || rows::misaligned(rows_dev, 4) || rows::misaligned(offsets_dev, 4)) return REMOE_E_ARG;
  if (n_experts > REMOE_SORT_MAX_EXPERTS || (int64_t)n_tokens * top_k > 0x7fffffff) return REMOE_E_UNSUPPORTED;
  rows::PointerDevice device(offsets_dev);
  if (device.err_code()) return device.err_code();
  SortArgs a{ids_dev, rows_dev, offsets_dev, n_tokens * top_k, n_experts, 0};
  const int strips = (a.n + 31) / 32;
  int blocks = 1;
  while (blocks < 8 && strips > blocks * kSortWarps * 4) blocks *= 2;
  int warps = (strips + blocks - 1) / blocks;
  warps = warps < 4 ? 4 : warps > kSortWarps ? kSortWarps : warps;
  a.run = (int)(((int64_t)strips + warps * blocks - 1) / (warps * blocks)) * 32;
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(sort_kernel, (size_t)(kSortWarps + 3) * REMOE_SORT_MAX_EXPERTS * 4, ready);
  if (e != cudaSuccess) return REMOE_E_CUDA;
  return rows::status(rows::launch<sort_kernel>(a, blocks, blocks, warps * 32, (size_t)(warps + 3) * n_experts * 4,
                                                static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" int remoe_expert_dispatch(int32_t n_tokens, int32_t top_k, int32_t hidden, int32_t dtype, const void* x_dev, int64_t x_stride,
                                     const int32_t* rows_dev, int32_t n_rows, void* xs_dev, int64_t xs_stride, void* cuda_stream) {
  const int bad = check_rows_call(n_tokens, top_k, hidden, dtype, rows_dev, n_rows);
  if (bad) return bad;
  const int size = rows::element_size(dtype);
  if (sorted::bad_matrix(x_dev, x_stride, n_tokens, hidden, size) || sorted::bad_matrix(xs_dev, xs_stride, n_rows, hidden, size))
    return REMOE_E_ARG;
  if (n_tokens == 0 || n_rows == 0) return REMOE_OK;
  rows::PointerDevice device(x_dev);
  if (device.err_code()) return device.err_code();
  const RowArgs a{x_dev, x_stride, nullptr, 0, xs_dev, xs_stride, rows_dev, nullptr, nullptr, top_k, hidden, n_rows};
  const int width = std::min(sorted::access_width(x_dev, x_stride, n_tokens, size), sorted::access_width(xs_dev, xs_stride, n_rows, size));
  return launch_rows<kDispatch>(a, n_tokens, dtype, width, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int remoe_expert_combine(int32_t n_tokens, int32_t top_k, int32_t hidden, int32_t dtype, int32_t n_rows, const void* ys_dev,
                                    int64_t ys_stride, const int32_t* rows_dev, const float* gates_dev, const void* base_dev,
                                    int64_t base_stride, void* out_dev, int64_t out_stride, void* cuda_stream) {
  const int bad = check_rows_call(n_tokens, top_k, hidden, dtype, rows_dev, n_rows);
  if (bad) return bad;
  const int size = rows::element_size(dtype);
  if (sorted::bad_matrix(ys_dev, ys_stride, n_rows, hidden, size) || sorted::bad_matrix(out_dev, out_stride, n_tokens, hidden, size))
    return REMOE_E_ARG;
  if (base_dev && sorted::bad_matrix(base_dev, base_stride, n_tokens, hidden, size)) return REMOE_E_ARG;
  if (base_dev == out_dev && base_stride != out_stride && n_tokens > 1) return REMOE_E_ARG;
  if (gates_dev && rows::misaligned(gates_dev, 4)) return REMOE_E_ARG;
  if (n_tokens == 0) return REMOE_OK;
  rows::PointerDevice device(out_dev);
  if (device.err_code()) return device.err_code();
  const RowArgs a{ys_dev, ys_stride, base_dev, base_stride, out_dev, out_stride, rows_dev, gates_dev, nullptr, top_k, hidden, n_rows};
  int width = std::min(sorted::access_width(ys_dev, ys_stride, n_rows, size), sorted::access_width(out_dev, out_stride, n_tokens, size));
  if (base_dev) width = std::min(width, sorted::access_width(base_dev, base_stride, n_tokens, size));
  return launch_rows<kCombine>(a, n_tokens, dtype, width, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int remoe_expert_combine_backward(int32_t n_tokens, int32_t top_k, int32_t hidden, int32_t dtype, const void* d_out_dev,
                                             int64_t d_out_stride, int32_t n_rows, const void* ys_dev, int64_t ys_stride,
                                             const int32_t* rows_dev, const float* gates_dev, void* d_ys_dev, int64_t d_ys_stride,
                                             float* d_gates_dev, void* cuda_stream) {
  const int bad = check_rows_call(n_tokens, top_k, hidden, dtype, rows_dev, n_rows);
  if (bad) return bad;
  const int size = rows::element_size(dtype);
  if (!d_ys_dev && !d_gates_dev) return REMOE_E_ARG;
  if (sorted::bad_matrix(d_out_dev, d_out_stride, n_tokens, hidden, size)) return REMOE_E_ARG;
  if (d_gates_dev && (sorted::bad_matrix(ys_dev, ys_stride, n_rows, hidden, size) || rows::misaligned(d_gates_dev, 4))) return REMOE_E_ARG;
  if (d_ys_dev && sorted::bad_matrix(d_ys_dev, d_ys_stride, n_rows, hidden, size)) return REMOE_E_ARG;
  if (d_ys_dev && d_ys_dev == ys_dev && d_ys_stride != ys_stride && n_rows > 1) return REMOE_E_ARG;
  if (gates_dev && rows::misaligned(gates_dev, 4)) return REMOE_E_ARG;
  if (n_tokens == 0) return REMOE_OK;
  rows::PointerDevice device(d_out_dev);
  if (device.err_code()) return device.err_code();
  const RowArgs a{ys_dev, ys_stride, d_out_dev, d_out_stride, d_ys_dev, d_ys_stride, rows_dev, gates_dev, d_gates_dev, top_k, hidden, n_rows};
  int width = sorted::access_width(d_out_dev, d_out_stride, n_tokens, size);
  if (d_gates_dev) width = std::min(width, sorted::access_width(ys_dev, ys_stride, n_rows, size));
  if (d_ys_dev) width = std::min(width, sorted::access_width(d_ys_dev, d_ys_stride, n_rows, size));
  return launch_rows<kCombineBackward>(a, n_tokens, dtype, width, static_cast<cudaStream_t>(cuda_stream));
}
