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
// consecutive selections and counts them by expert (lanes with the same expert find one another by a vote for each bit of the id, so a
// counter has one writer at a time); the counts before a selection within its run are its rank there.  The counts are summed over the warps
// and, through distributed shared memory, over the blocks, and every rank becomes a row.  Integers only, the same order every time.
struct SortArgs {
  const int* ids;
  int* rows;
  int* offsets;
  int n, n_experts, run;                 // selections, experts, selections of one warp (a multiple of 32)
};

constexpr int kSortWarps = 32;
constexpr int kSortBlocks = 16;          // most blocks of the cluster
constexpr int kStrips = 8;               // of 32 selections whose loads are under way together

// ONCE: a run is at most kStrips strips, whose experts and ranks stay in registers; longer ones are read a second time.
template <bool ONCE>
__global__ void __launch_bounds__(kSortWarps * 32) sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ int sort_smem[];
  const int N = a.n_experts, W = blockDim.x >> 5;
  int* total = sort_smem;                // [N] of this block
  int* base = total + N;                 // [N] selections in lower blocks, then the first row of an expert's selections in this block
  int* every = base + N;                 // [N] of all blocks
  int* count = every + N;                // [W][N]
  int* theirs = count + W * N;           // [blocks][N] counts of every block
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned below = (1u << lane) - 1;
  const int bits = 32 - __clz(N - 1);
  const int64_t begin = ((int64_t)rank * W + warp) * a.run;
  const int64_t end = begin + a.run < a.n ? begin + a.run : a.n;
  int* mine = count + warp * N;

  int id[kStrips], at[kStrips];          // expert (-1: none) and rank among the run's selections of it so far
  auto load = [&](int64_t s0) {
#pragma unroll
    for (int i = 0; i < kStrips; ++i) {
      const int64_t s = s0 + i * 32 + lane;
      id[i] = s < end ? a.ids[s] : -1;   // (a coherent load: `rows` may be the same memory)
    }
  };
  auto take = [&](int64_t s0) {          // hands out places from the warp's counters
    unsigned peers[kStrips];
#pragma unroll
    for (int i = 0; i < kStrips; ++i)
      if ((unsigned)id[i] >= (unsigned)N) id[i] = -1;
    if (s0 + 32 * (kStrips / 2) < end) {  // many strips: their votes between one another
#pragma unroll
      for (int i = 0; i < kStrips; ++i) peers[i] = __ballot_sync(0xffffffffu, id[i] >= 0);
      for (int b = 0; b < bits; ++b) {
#pragma unroll
        for (int i = 0; i < kStrips; ++i) {
          const bool set = (id[i] >> b) & 1;
          const unsigned with = __ballot_sync(0xffffffffu, set);
          peers[i] &= set ? with : ~with;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kStrips / 2; ++i) {
        if (s0 + i * 32 >= end) break;
        peers[i] = __ballot_sync(0xffffffffu, id[i] >= 0);
        for (int b = 0; b < bits; ++b) {
          const bool set = (id[i] >> b) & 1;
          const unsigned with = __ballot_sync(0xffffffffu, set);
          peers[i] &= set ? with : ~with;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kStrips; ++i) {
      if (s0 + i * 32 >= end) break;
      const int old = id[i] >= 0 ? mine[id[i]] : 0;
      __syncwarp();
      if (id[i] >= 0 && !(peers[i] & below)) mine[id[i]] = old + __popc(peers[i]);
      __syncwarp();
      at[i] = old + __popc(peers[i] & below);
    }
  };
  load(begin);
  for (int i = threadIdx.x; i < W * N; i += blockDim.x) count[i] = 0;
  __syncthreads();
  take(begin);
  if constexpr (!ONCE)
    for (int64_t s0 = begin + 32 * kStrips; s0 < end; s0 += 32 * kStrips) {
      load(s0);
      take(s0);
    }
  __syncthreads();
  for (int e = threadIdx.x; e < N; e += blockDim.x) {
    int sum = 0;
#pragma unroll 8
    for (int w = 0; w < W; ++w) {
      const int c = count[w * N + e];
      count[w * N + e] = sum;
      sum += c;
    }
    total[e] = sum;
  }
  cluster.sync();
  // a thread for each block and expert: one trip to another block's memory, not one behind the other
  for (int i = threadIdx.x; i < blocks * N; i += blockDim.x) theirs[i] = *cluster.map_shared_rank(total + i % N, i / N);
  __syncthreads();
  cluster.barrier_arrive();              // (no block leaves while another reads its counts)
  for (int e = threadIdx.x; e < N; e += blockDim.x) {
    int before = 0, all = 0;
    for (int b = 0; b < blocks; ++b) {
      const int c = theirs[b * N + e];
      before += b < rank ? c : 0;
      all += c;
    }
    base[e] = before;
    every[e] = all;
  }
  __syncthreads();
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
      base[e] += first;
      if (rank == 0) a.offsets[e] = first;
      first += every[e];
    }
    if (rank == 0 && lane == 31) a.offsets[N] = upto;
  }
  __syncthreads();
  for (int64_t s0 = begin; s0 < end; s0 += 32 * kStrips) {
    if constexpr (!ONCE) {
      load(s0);
      take(s0);                          // (the counters have become the run's first places)
    }
#pragma unroll
    for (int i = 0; i < kStrips; ++i) {
      const int64_t s = s0 + i * 32 + lane;
      int row = -1;
      if (id[i] >= 0) row = base[id[i]] + at[i] + (ONCE ? mine[id[i]] : 0);
      if (s < end) a.rows[s] = row;
    }
  }
  cluster.barrier_wait();
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

// A load under a predicate, zero without it: no branch, so that a group's loads are issued one behind the other.  (With an if around each,
// the compiler finished one row before it asked for the next: 50 instead of 30 us for the sum of 4096 x 6 rows of 2048 bf16.)  It reads memory that the same
// thread may write afterwards (a gradient over the rows themselves), so it names memory to the compiler, too.
__device__ __forceinline__ void load_word_if(uint4& w, const void* p, bool yes) {
  w = make_uint4(0, 0, 0, 0);
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "+r"(w.x), "+r"(w.y), "+r"(w.z), "+r"(w.w)
               : "l"(p), "r"((int)yes)
               : "memory");
}
__device__ __forceinline__ void load_word_if(uint2& w, const void* p, bool yes) {
  w = make_uint2(0, 0);
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %3, 0;\n\t@p ld.global.v2.u32 {%0, %1}, [%2];\n\t}" : "+r"(w.x), "+r"(w.y) : "l"(p), "r"((int)yes) : "memory");
}
__device__ __forceinline__ void load_word_if(unsigned& w, const void* p, bool yes) {
  w = 0;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(w) : "l"(p), "r"((int)yes) : "memory");
}
__device__ __forceinline__ void load_word_if(unsigned short& w, const void* p, bool yes) {
  w = 0;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p ld.global.u16 %0, [%1];\n\t}" : "+h"(w) : "l"(p), "r"((int)yes) : "memory");
}

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
  __device__ __forceinline__ void load_if(const T* p, bool yes) { load_word_if(word, p, yes); }
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
  int K, H, n_rows, n_tokens;
  int threads, parts;                    // threads of an item (whole warps), items of a token
};

constexpr int kGroup = 8;                // rows of a token whose loads are under way together

// One block a token: its row is read once, kUnroll pieces under way together, and written to the places of its selections.
template <typename T, int V>
__global__ void __launch_bounds__(256) dispatch_kernel(const __grid_constant__ RowArgs a) {
  constexpr int kUnroll = 4;
  const int64_t t = blockIdx.x;
  const int* rows = a.rows + t * a.K;
  const T* x = static_cast<const T*>(a.a) + t * a.a_stride;
  T* out = static_cast<T*>(a.out);
  const int body = a.H / V;
  for (int i0 = threadIdx.x; i0 < body; i0 += kUnroll * blockDim.x) {
    Vec<T, V> v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * (int)blockDim.x < body) v[u].load(x + (i0 + u * (int)blockDim.x) * V);
    for (int k = 0; k < a.K; ++k) {
      const int r = __ldg(rows + k);
      if ((unsigned)r >= (unsigned)a.n_rows) continue;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (i0 + u * (int)blockDim.x < body) v[u].store(out + r * a.out_stride + (i0 + u * (int)blockDim.x) * V);
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

// Blocks of 256 threads that lie on an SM together: what a group's rows take in registers decides.
template <typename T, int V, bool TAIL>
constexpr int resident_blocks() { return V * sizeof(T) < 8 ? 4 : TAIL ? 2 : 3; }

// The rows and gates of a token, a lane each (up to 32 of them), loaded an item ahead of their use.
struct Picks {
  int row;
  float gate;
  __device__ __forceinline__ void load(const RowArgs& a, int64_t t, int k0, int lane) {
    row = -1;
    gate = 1.f;
    if (k0 + lane < a.K) {
      row = __ldg(a.rows + t * a.K + k0 + lane);
      if (a.gates) gate = __ldg(a.gates + t * a.K + k0 + lane);
    }
  }
  // Of one selection, for all lanes.  (Looked over here, not where it is loaded, so that nothing waits for the load.)
  __device__ __forceinline__ int row_of(const RowArgs& a, int k) const {
    const int r = __shfl_sync(0xffffffffu, row, k);
    return (unsigned)r < (unsigned)a.n_rows ? r : -1;
  }
  __device__ __forceinline__ float gate_of(int k) const { return __shfl_sync(0xffffffffu, gate, k); }
};

// Adds a token's rows to `sum` in the order of the selections.
template <typename T, int V>
__device__ __forceinline__ void add_rows(const RowArgs& a, int64_t t, Picks p, int i, bool here, int lane, float (&sum)[V]) {
  for (int kb = 0; kb < a.K; kb += 32) {
    if (kb) p.load(a, t, kb, lane);
    for (int k0 = 0; k0 < 32 && kb + k0 < a.K; k0 += kGroup) {
      Vec<T, V> v[kGroup];
      float g[kGroup];
      int r[kGroup];
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        r[k] = p.row_of(a, k0 + k);
        g[k] = p.gate_of(k0 + k);
        v[k].load_if(static_cast<const T*>(a.a) + r[k] * a.a_stride + i, r[k] >= 0 && here);
      }
#pragma unroll
      for (int k = 0; k < kGroup; ++k)
        if (r[k] >= 0) {
#pragma unroll
          for (int j = 0; j < V; ++j) sum[j] = fmaf(g[k], to_float(v[k].e[j]), sum[j]);
        }
    }
  }
}

// Items of the combine, dealt to the groups of threads in turn, in steps of mixed digits (no division an item).
struct Item {
  int64_t token, by;
  int part, part_by;
  __device__ __forceinline__ Item(const RowArgs& a, int step) {
    const int64_t first = (int64_t)blockIdx.x * step + threadIdx.x / a.threads;
    const int stride = (int)gridDim.x * step;
    token = first / a.parts;
    part = (int)(first - token * a.parts);
    by = stride / a.parts;
    part_by = stride % a.parts;
  }
  __device__ __forceinline__ void next(const RowArgs& a) {
    token += by;
    part += part_by;
    if (part >= a.parts) { part -= a.parts; ++token; }
  }
};

// An item is a piece of a token's row for a.threads threads (whole warps), V elements each, in float32; the elements behind the last whole V
// are pieces of one.  Persistent: the next item's rows and gates are on their way while this one's data is.
template <typename T, int V, bool TAIL>
__global__ void __launch_bounds__(256, resident_blocks<T, V, TAIL>()) combine_kernel(const __grid_constant__ RowArgs a) {
  const int lane = threadIdx.x & 31, body = a.H / V, pieces = body + a.H % V, step = (int)blockDim.x / a.threads;
  Picks next;
  Item item(a, step);
  if (item.token < a.n_tokens) next.load(a, item.token, 0, lane);
  while (item.token < a.n_tokens) {
    const int64_t t = item.token;
    const int piece = item.part * a.threads + (int)threadIdx.x % a.threads;
    const Picks p = next;
    const bool whole = piece < body, here = piece < pieces;
    const int i = whole ? piece * V : body * V + piece - body;
    item.next(a);
    if (item.token < a.n_tokens) next.load(a, item.token, 0, lane);
    T* out = static_cast<T*>(a.out) + t * a.out_stride + i;
    const T* base = a.b ? static_cast<const T*>(a.b) + t * a.b_stride + i : nullptr;
    if (!TAIL || __any_sync(0xffffffffu, whole)) {
      float sum[V];
      Vec<T, V> o;
      if (base && whole) o.load(base);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = 0.f;
      add_rows<T, V>(a, t, p, i, whole, lane, sum);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (base) sum[j] += to_float(o.e[j]);
        o.e[j] = from_float<T>(sum[j]);
      }
      if (whole) o.store(out);
    }
    if (TAIL && __any_sync(0xffffffffu, here && !whole)) {
      const bool single = here && !whole;
      float sum[1] = {0.f};
      const float first = base && single ? to_float(*base) : 0.f;
      add_rows<T, 1>(a, t, p, i, single, lane, sum);
      if (single) *out = from_float<T>(base ? sum[0] + first : sum[0]);
    }
  }
}

// The same sum for rows that are whole numbers of accesses of 4 bytes or more: copies to shared memory, a few units (up to G rows of an
// item's piece, and the base) ahead of the sums.  A thread reads nothing but what it copied, so there is no barrier, and what is under way costs
// no registers.  Taken where there are more items than fit at once: 4096 x 6 rows of 2048 bf16 and a base take 24.0 us, with the loads in registers,
// one item at a time, 33; one token 3.7 against 2.7 (of which either has a launch).  G is the least of 2, 4, 6 and 8 that takes a token's rows at
// once, since the instructions of a unit are for G rows: 4096 x 4 of them take 16.6 us, in groups of eight 21.4, 4096 x 2 of 4096 24.5 and 40.
// Units ahead and blocks of an SM by what measured best: for G = 8 one ahead and three blocks (25.7 us for 4096 x 6 then), two blocks 29.5, two
// ahead 29.8; with accesses of 8 bytes four blocks (4096 x 6 of 1028: 21.1 us; three: 23.3), which for those of 16 are slower (26.4).
__host__ __device__ constexpr int copy_depth(int group) { return group <= 2 ? 4 : group <= 4 ? 3 : 2; }
constexpr int kCopyThreads = 256;
__host__ __device__ constexpr int copy_blocks(int bytes) { return bytes == 16 ? 3 : 4; }         // of an SM, by the width of an access

template <int BYTES>
__device__ __forceinline__ void copy_if(uint32_t dst, const void* src, bool yes) {
  if constexpr (BYTES == 16)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src), "r"((int)yes) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %3, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], %2;\n\t}" ::"r"(dst), "l"(src), "n"(BYTES), "r"((int)yes)
                 : "memory");
}

template <typename T, int V, int G>
__global__ void __launch_bounds__(kCopyThreads) combine_copy_kernel(const __grid_constant__ RowArgs a) {
  using W = typename Word<V * (int)sizeof(T)>::type;
  extern __shared__ __align__(16) unsigned char copy_smem[];
  W* mine = reinterpret_cast<W*>(copy_smem) + threadIdx.x;               // [D][group, base][blockDim.x]
  constexpr int D = copy_depth(G);
  const int per = (G + (a.b ? 1 : 0)) * (int)blockDim.x;
  const int lane = threadIdx.x & 31, pieces = a.H / V, step = (int)blockDim.x / a.threads;
  const int in_item = (int)threadIdx.x % a.threads;
  Item item(a, step);
  struct Unit {                          // an item, and the first of its selections
    Item at;
    int k0;
    __device__ __forceinline__ void next(const RowArgs& a) {
      k0 += G;
      if (k0 >= a.K) { k0 = 0; at.next(a); }
    }
  };
  Unit now{item, 0}, ahead = now;
  Picks picks[D + 1];                // of the units from `now` on; the last one's is on its way
  auto look = [&](Picks& p, const Unit& u) {
    p.row = -1;
    p.gate = 1.f;
    if (u.at.token < a.n_tokens && lane < G && u.k0 + lane < a.K) {
      const int64_t at = u.at.token * a.K + u.k0 + lane;
      p.row = __ldg(a.rows + at);
      if (a.gates) p.gate = __ldg(a.gates + at);
    }
  };
  auto send = [&](const Picks& p, const Unit& u, int slot) {
    const int piece = u.at.part * a.threads + in_item;
    const bool here = u.at.token < a.n_tokens && piece < pieces;
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(mine + slot * per);
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const int r = p.row_of(a, k);
      copy_if<(int)sizeof(W)>(dst + k * blockDim.x * (int)sizeof(W), static_cast<const T*>(a.a) + r * a.a_stride + piece * V, here && r >= 0);
    }
    if (a.b) copy_if<(int)sizeof(W)>(dst + G * blockDim.x * (int)sizeof(W), static_cast<const T*>(a.b) + u.at.token * a.b_stride + piece * V, here && u.k0 == 0);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look(picks[0], ahead);
#pragma unroll
  for (int i = 0; i < D - 1; ++i) {
    const Unit u = ahead;
    ahead.next(a);
    look(picks[i + 1], ahead);
    send(picks[i], u, i);
  }
  float sum[V];
  int slot = 0;
  while (now.at.token < a.n_tokens) {
    const Unit u = ahead;
    ahead.next(a);
    look(picks[D], ahead);
    send(picks[D - 1], u, slot == 0 ? D - 1 : slot - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(D - 1) : "memory");
    const W* from = mine + slot * per;
    if (now.k0 == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = 0.f;
    }
    Vec<T, V> v;
    const int piece = now.at.part * a.threads + in_item;
    const bool here = piece < pieces;
#pragma unroll
    for (int k = 0; k < G; ++k)
      if (picks[0].row_of(a, k) >= 0) {
        const float g = picks[0].gate_of(k);
        v.word = from[k * blockDim.x];
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = fmaf(g, to_float(v.e[j]), sum[j]);
      }
    if (now.k0 + G >= a.K && here) {
      const int64_t t = now.at.token;
      if (a.b) {
        if (now.k0 == 0) v.word = from[G * blockDim.x];
        else v.load(static_cast<const T*>(a.b) + t * a.b_stride + piece * V);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += to_float(v.e[j]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) v.e[j] = from_float<T>(sum[j]);
      v.store(static_cast<T*>(a.out) + t * a.out_stride + piece * V);
    }
#pragma unroll
    for (int i = 0; i < D; ++i) picks[i] = picks[i + 1];
    now.next(a);
    slot = slot == D - 1 ? 0 : slot + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int V, int G>
__device__ __forceinline__ void backward_piece(const RowArgs& a, int64_t t, const int (&r)[G], const float (&g)[G], int i, float (&dot)[G]) {
  Vec<T, V> d, v[G];
  d.load(static_cast<const T*>(a.b) + t * a.b_stride + i);
  if (a.d_gates) {
#pragma unroll
    for (int k = 0; k < G; ++k) v[k].load_if(static_cast<const T*>(a.a) + r[k] * a.a_stride + i, r[k] >= 0);
  }
#pragma unroll
  for (int k = 0; k < G; ++k) {
    if (r[k] < 0) continue;
    if (a.d_gates) {
#pragma unroll
      for (int j = 0; j < V; ++j) dot[k] = fmaf(to_float(v[k].e[j]), to_float(d.e[j]), dot[k]);
    }
    if (a.out) {
      Vec<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.e[j] = from_float<T>(g[k] * to_float(d.e[j]));
      o.store(static_cast<T*>(a.out) + r[k] * a.out_stride + i);
    }
  }
}

// Eight or four values a lane, summed over the warp: lane l ends with the sum of value l / (32 / G) of all lanes.
template <int G>
__device__ __forceinline__ float reduce_group(float (&x)[G], int lane) {
  float s = 0.f;
#pragma unroll
  for (int n = G / 2, by = 16; by; n /= 2, by /= 2) {
    if (n) {                             // half of the values for each half of the lanes
      const bool high = lane & by;
#pragma unroll
      for (int k = 0; k < G / 2; ++k)
        if (k < n) {
          const float keep = high ? x[k + n] : x[k], give = high ? x[k] : x[k + n];
          x[k] = keep + __shfl_xor_sync(0xffffffffu, give, by);
        }
      s = x[0];
    } else {
      s += __shfl_xor_sync(0xffffffffu, s, by);
    }
  }
  return s;
}

// A token for a.threads threads, one warp (several tokens a block) or the whole block: the gradient of the sum is read once for up to eight of
// its rows, whose scalar products with it are summed in a fixed order.  Persistent as above.
template <typename T, int V, bool TAIL, int G>
constexpr int backward_blocks() { return G == 4 && V * sizeof(T) >= 8 ? 4 : resident_blocks<T, V, TAIL>(); }

template <typename T, int V, bool TAIL, int G>
__global__ void __launch_bounds__(256, backward_blocks<T, V, TAIL, G>()) combine_backward_kernel(const __grid_constant__ RowArgs a) {
  __shared__ float part[2][8][G];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, body = a.H / V, pieces = body + a.H % V, step = (int)blockDim.x / a.threads;
  const int64_t stride = (int64_t)gridDim.x * step;
  const int first = threadIdx.x % a.threads;
  int64_t t = (int64_t)blockIdx.x * step + threadIdx.x / a.threads;
  int turn = 0;
  Picks next;
  if (t < a.n_tokens) next.load(a, t, 0, lane);
  for (; t < a.n_tokens; t += stride) {
    Picks p = next;
    if (t + stride < a.n_tokens) next.load(a, t + stride, 0, lane);
    for (int kb = 0; kb < a.K; kb += G) {
      if (kb && kb % 32 == 0) p.load(a, t, kb, lane);
      int r[G];
      float g[G], dot[G];
#pragma unroll
      for (int k = 0; k < G; ++k) {
        r[k] = p.row_of(a, kb % 32 + k);
        g[k] = p.gate_of(kb % 32 + k);
        dot[k] = 0.f;
      }
      for (int i = first; i < pieces; i += a.threads) {
        if (!TAIL || i < body) backward_piece<T, V, G>(a, t, r, g, i * V, dot);
        else backward_piece<T, 1, G>(a, t, r, g, body * V + i - body, dot);
      }
      if (!a.d_gates) continue;
      const float s = reduce_group<G>(dot, lane);
      float* d_gates = a.d_gates + t * a.K + kb;
      if (a.threads == 32) {
        if (lane % (32 / G) == 0 && kb + lane / (32 / G) < a.K) d_gates[lane / (32 / G)] = s;
        continue;
      }
      if (lane % (32 / G) == 0) part[turn][warp][lane / (32 / G)] = s;
      __syncthreads();                   // (two sets of sums: the next one's writers do not have to wait for these readers)
      if (threadIdx.x < G && kb + threadIdx.x < a.K) {
        float sum = 0.f;
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) sum += part[turn][w][threadIdx.x];
        d_gates[threadIdx.x] = sum;
      }
      turn ^= 1;
    }
  }
}

enum Op { kDispatch, kCombine, kCombineBackward };

template <typename T, int V, int G>
cudaError_t launch_copies(const RowArgs& a, int threads, cudaStream_t stream) {
  constexpr size_t kPiece = copy_depth(G) * V * sizeof(T);
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(combine_copy_kernel<T, V, G>, kPiece * (G + 1) * kCopyThreads, ready);
  if (e != cudaSuccess) return e;
  return rows::launch<combine_copy_kernel<T, V, G>>(a, 148 * copy_blocks(V * sizeof(T)), 1, threads, kPiece * (G + (a.b ? 1 : 0)) * threads, stream);
}

template <Op OP, typename T, int V, bool TAIL>
cudaError_t launch_rows_as(const RowArgs& args, cudaStream_t stream) {
  RowArgs a = args;
  const int pieces = a.H / V + a.H % V;
  a.threads = pieces >= 256 ? 256 : (pieces + 31) / 32 * 32;
  a.parts = 1;
  if constexpr (OP == kDispatch) return rows::launch<dispatch_kernel<T, V>>(a, a.n_tokens, 1, a.threads, 0, stream);
  if constexpr (OP == kCombine) {
    a.parts = (pieces + a.threads - 1) / a.threads;
    a.threads = ((pieces + a.parts - 1) / a.parts + 31) / 32 * 32;         // (257 pieces: twice 160 threads)
    const int step = 256 / a.threads;
    const int64_t blocks = ((int64_t)a.n_tokens * a.parts + step - 1) / step;
    if constexpr (!TAIL && V * sizeof(T) >= 4)
      if (blocks > 148 * copy_blocks(V * sizeof(T))) {
        if (a.K <= 2) return launch_copies<T, V, 2>(a, step * a.threads, stream);
        if (a.K <= 4) return launch_copies<T, V, 4>(a, step * a.threads, stream);
        if (a.K <= 6) return launch_copies<T, V, 6>(a, step * a.threads, stream);
        return launch_copies<T, V, 8>(a, step * a.threads, stream);
      }
    return rows::launch<combine_kernel<T, V, TAIL>>(a, std::min<int64_t>(blocks, 148 * resident_blocks<T, V, TAIL>()), 1, step * a.threads, 0, stream);
  }
  if constexpr (OP == kCombineBackward) {
    const int step = a.threads == 32 ? 8 : 1, threads = step * a.threads;
    const int64_t blocks = ((int64_t)a.n_tokens + step - 1) / step;
    if (a.K <= 4)
      return rows::launch<combine_backward_kernel<T, V, TAIL, 4>>(a, std::min<int64_t>(blocks, 148 * (backward_blocks<T, V, TAIL, 4>() * 256 / threads)), 1, threads, 0, stream);
    return rows::launch<combine_backward_kernel<T, V, TAIL, 8>>(a, std::min<int64_t>(blocks, 148 * (backward_blocks<T, V, TAIL, 8>() * 256 / threads)), 1, threads, 0, stream);
  }
}

// TAIL: a row is not a whole number of accesses.
template <Op OP, typename T, int V>
cudaError_t launch_rows(const RowArgs& a, cudaStream_t stream) {
  if constexpr (V > 1 && OP != kDispatch)
    if (a.H % V) return launch_rows_as<OP, T, V, true>(a, stream);
  return launch_rows_as<OP, T, V, false>(a, stream);
}

template <Op OP>
int launch_rows(const RowArgs& a, int32_t dtype, int width, cudaStream_t stream) {
  cudaError_t e = cudaErrorInvalidValue;
  if (dtype == REMOE_F32) {
    switch (width) {
      case 16: e = launch_rows<OP, float, 4>(a, stream); break;
      case 8: e = launch_rows<OP, float, 2>(a, stream); break;
      case 4: e = launch_rows<OP, float, 1>(a, stream); break;
    }
  } else if (dtype == REMOE_BF16) {
    switch (width) {
      case 16: e = launch_rows<OP, __nv_bfloat16, 8>(a, stream); break;
      case 8: e = launch_rows<OP, __nv_bfloat16, 4>(a, stream); break;
      case 4: e = launch_rows<OP, __nv_bfloat16, 2>(a, stream); break;
      case 2: e = launch_rows<OP, __nv_bfloat16, 1>(a, stream); break;
    }
  } else {
    switch (width) {
      case 16: e = launch_rows<OP, __half, 8>(a, stream); break;
      case 8: e = launch_rows<OP, __half, 4>(a, stream); break;
      case 4: e = launch_rows<OP, __half, 2>(a, stream); break;
      case 2: e = launch_rows<OP, __half, 1>(a, stream); break;
    }
  }
  return rows::status(e);
}

template <bool ONCE>
cudaError_t launch_sort(const SortArgs& a, int blocks, int warps, cudaStream_t stream) {
  static std::atomic<bool> ready[kMaxDevices];
  if (blocks > 8) {
    const cudaError_t e = cudaFuncSetAttribute(sort_kernel<ONCE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = allow_dynamic_smem(sort_kernel<ONCE>, (size_t)(kSortWarps + 3 + kSortBlocks) * REMOE_SORT_MAX_EXPERTS * 4, ready);
  if (e != cudaSuccess) return e;
  return rows::launch<sort_kernel<ONCE>>(a, blocks, blocks, warps * 32, (size_t)(warps + 3 + blocks) * a.n_experts * 4, stream);
}

int check_rows_call(int32_t n_tokens, int32_t top_k, int32_t hidden, int32_t dtype, const int32_t* rows_dev, int32_t n_rows) {
  if (n_tokens < 0 || top_k < 1 || hidden < 1 || n_rows < 0 || (!rows_dev && n_tokens > 0) || rows::misaligned(rows_dev, 4)) return REMOE_E_ARG;
  if (dtype == REMOE_FP8_E4M3 || dtype == REMOE_INT4_G32) return REMOE_E_UNSUPPORTED;
  if (!rows::element_size(dtype)) return REMOE_E_ARG;
  if ((int64_t)n_tokens * top_k > 0x7fffffff || hidden > REMOE_EXPERT_MAX_HIDDEN) return REMOE_E_UNSUPPORTED;
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
  if (const int host = n_tokens > 0 ? sorted::check_device_memory({ids_dev, rows_dev}) : REMOE_OK) return host;
  SortArgs a{ids_dev, rows_dev, offsets_dev, n_tokens * top_k, n_experts, 0};
  const int strips = (int)(((int64_t)a.n + 31) / 32);
  int blocks = 1;
  // One block for up to 4096 selections (2048: 5.2 us, shared between two blocks 7.8; 8192: 9.5 and, between eight, 8.1), else the eight that any
  // cluster may have, and from 16384 on the sixteen that this GPU can give (8192: 5.8 us with either; 24576: 6.8 with eight, 6.4 with sixteen;
  // 65536: 9.8 and 8.2; 262144: 41 and 25).
  if (strips > kSortWarps * kStrips / 2) blocks = strips > 2 * kSortWarps * kStrips ? kSortBlocks : 8;
  int warps = (strips + blocks - 1) / blocks;
  warps = warps < 4 ? 4 : warps > kSortWarps ? kSortWarps : warps;
  a.run = (int)(((int64_t)strips + warps * blocks - 1) / (warps * blocks)) * 32;
  return rows::status(a.run <= 32 * kStrips ? launch_sort<true>(a, blocks, warps, static_cast<cudaStream_t>(cuda_stream))
                                            : launch_sort<false>(a, blocks, warps, static_cast<cudaStream_t>(cuda_stream)));
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
  if (const int host = sorted::check_device_memory({rows_dev, xs_dev})) return host;
  const RowArgs a{x_dev, x_stride, nullptr, 0, xs_dev, xs_stride, rows_dev, nullptr, nullptr, top_k, hidden, n_rows, n_tokens, 0, 0};
  const int width = std::min(sorted::access_width(x_dev, x_stride, n_tokens, size), sorted::access_width(xs_dev, xs_stride, n_rows, size));
  return launch_rows<kDispatch>(a, dtype, width, static_cast<cudaStream_t>(cuda_stream));
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
  if (const int host = sorted::check_device_memory({n_rows > 0 ? ys_dev : nullptr, rows_dev, gates_dev, base_dev == out_dev ? nullptr : base_dev})) return host;
  const RowArgs a{ys_dev, ys_stride, base_dev, base_stride, out_dev, out_stride, rows_dev, gates_dev, nullptr, top_k, hidden, n_rows, n_tokens, 0, 0};
  int width = std::min(sorted::access_width(ys_dev, ys_stride, n_rows, size), sorted::access_width(out_dev, out_stride, n_tokens, size));
  if (base_dev) width = std::min(width, sorted::access_width(base_dev, base_stride, n_tokens, size));
  return launch_rows<kCombine>(a, dtype, width, static_cast<cudaStream_t>(cuda_stream));
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
  if (const int host = sorted::check_device_memory({n_rows > 0 && d_gates_dev ? ys_dev : nullptr, rows_dev, gates_dev, n_rows > 0 ? d_ys_dev : nullptr, d_gates_dev})) return host;
  const RowArgs a{ys_dev, ys_stride, d_out_dev, d_out_stride, d_ys_dev, d_ys_stride, rows_dev, gates_dev, d_gates_dev, top_k, hidden, n_rows, n_tokens, 0, 0};
  int width = sorted::access_width(d_out_dev, d_out_stride, n_tokens, size);
  if (d_gates_dev) width = std::min(width, sorted::access_width(ys_dev, ys_stride, n_rows, size));
  if (d_ys_dev) width = std::min(width, sorted::access_width(d_ys_dev, d_ys_stride, n_rows, size));
  return launch_rows<kCombineBackward>(a, dtype, width, static_cast<cudaStream_t>(cuda_stream));
}
