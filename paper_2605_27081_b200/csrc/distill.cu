// remoe_distill_topk / remoe_distill_topk_backward: divergence of rows of logits from a teacher that is known by its
// top log probabilities, and its gradient.
//
// S: the ids of the list.  q = softmax of the list's values, or (tail) their exp with q_r = 1 - sum q as one more
// class for all that is not listed; p_r = the student's mass outside S.
//   loss = sum_S q (ln q - ln p) + q_r (ln q_r - ln p_r)
//   dx_v = s w (Q p_v - q_v)                            v in S
//          s w (Q p_r - q_r) e^{s x_v} / sum_{not S}    v not in S
// Q is the sum of the q and of the q_r that is in the loss.  It is 1 for most lists; with tail it is not where q_r is left out (no live
// element outside S) or cut to 0 (values that sum to more than one).  The second line is p_v (Q - q_r / p_r), written so that
// it holds where the student leaves nearly nothing outside S: the sum outside S is taken over those elements alone, not as a
// difference.
#include <type_traits>

#include "logit_rows.cuh"
#include "logit_rows_host.h"
#include "remoe_internal.cuh"

namespace remoe {
namespace rows {

constexpr int kSmallVocab = 256;        // up to here a row is held by a group of lanes, one unit per lane
constexpr int kMaxList = REMOE_ROWS_MAX_TOP;

struct DistillArgs {
  const void* logits;
  void* d_logits;
  int64_t stride, d_stride;
  int V, n_rows, parts, slice_bytes, K, tail;
  float s;
  const int32_t* ids;
  const float *y, *weight;
  float *loss, *stats;
  const float* stats_in;
};

// What the block shares of a row between its two passes.
struct RowShared {
  float m_rest, coef;              // outside the list: coef * 2^((x - m_rest) c)
  double of_e, of_q, weight;       // in the list: weight * (of_e * e - of_q * q)
  int kind;                        // 0: left out (zeros), 1: takes part
};

// Gradient in the list from the row_stats: weight * (Q e^{(x - m) s - ln Z} - sum of e^{y - ln_q} over the entries of its id, in order),
// with `over` = Q - 1.
// In 64 bits for float32 results, whose rounding a difference of float32 exponentials would exceed; in float32 for the others.
template <typename T>
__device__ __forceinline__ float entry_gradient(float m, float ln_z, float ln_q, float over, float s, float weight, const int* id, const float* y, int K, int k,
                                                float x, bool twice) {
  typedef typename std::conditional<sizeof(T) == 4, double, float>::type R;
  auto e = [](R v) {
    if constexpr (sizeof(T) == 4) return exp(v);
    else return ex2(v * kLog2e);
  };
  R q = 0;
  for (int j = k; j < (twice ? K : k + 1); ++j)
    if (id[j] == id[k]) q += e((R)y[j] - ln_q);
  const R p = e(((R)x - m) * s - ln_z);
  return (float)((R)s * weight * (p - q + (R)over * p));
}

// Gradient outside the list, of one unit.
template <typename T>
__device__ __forceinline__ void rest_grad_unit(Unit<T>& q, float m, float c, float coef) {
  const f2 nm = pack2(-m, -m), cc = pack2(c, c), k2 = pack2(coef, coef);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f2 d = mul2(add2(Elem<T>::widen(q.w[j]), nm), cc);
    float d0, d1;
    unpack2(d, d0, d1);
    q.w[j] = Elem<T>::narrow(mul2(pack2(ex2(d0), ex2(d1)), k2));
  }
}

// Elements [e0, e1) of a row that lies at any address: whole units in one store each, the ends element by element.
template <typename T, typename F>
__device__ __forceinline__ void write_elements(T* out, int e0, int e1, int n_threads, int tid, F value) {
  const int pad = row_pad(out), u0 = (e0 + pad + 7) >> 3, u1 = (e1 + pad) >> 3;
  for (int u = u0 + tid; u < u1; u += n_threads) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = value(8 * u + j - pad);
    Unit<T> q;
    q.set(v);
    store_unit(out - pad + 8 * (int64_t)u, q);
  }
  const int head = min(8 * u0 - pad, e1), tail = max(8 * u1 - pad, head);
  if (tid < 8) {
    if (e0 + tid < head) Elem<T>::put(out + e0 + tid, value(e0 + tid));
  } else if (tid < 16) {
    const int i = tail + tid - 8;
    if (i < e1) Elem<T>::put(out + i, value(i));
  }
}

template <typename T>
__device__ __forceinline__ void fill_unit(Unit<T>& q, float x) {
  const float v[8] = {x, x, x, x, x, x, x, x};
  q.set(v);
}

struct ListSums {
  double z, q, qy, qx;             // sum over the list of e^{(x - m_list) s} (each id once), q, q (y - shift), q (x - m_list) s
};
__device__ __forceinline__ ListSums warp_sum(ListSums v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
    v.q += __shfl_xor_sync(0xffffffffu, v.q, o);
    v.qy += __shfl_xor_sync(0xffffffffu, v.qy, o);
    v.qx += __shfl_xor_sync(0xffffffffu, v.qx, o);
  }
  return v;
}

// What a row's list comes to, before its row is known.
struct ListSide {
  ListSums sums;
  float m_list;                    // largest logit of the list
  double shift;                    // of the list's values: the largest (tail = 0), or 0
  bool some, bad;                  // an entry with a probability; an entry that makes the row NaN
};

// Joins list and rest of a row; writes its loss and row_stats (`out`), and what its gradient needs to rs (`share`).
__device__ __forceinline__ void finish_row(const DistillArgs& a, int64_t r, float weight, const State& rest, const ListSide& l, bool share, bool out,
                                           RowShared& rs) {
  const double s = a.s;
  const ListSums& v = l.sums;
  const float m = max_nan(rest.m, l.m_list);
  const bool alive = m != -kInf, others = rest.m > -kInf;        // a NaN is alive
  const double x_shift = l.m_list != -kInf ? (double)l.m_list : 0.0;
  const double grow = 1.0 + (double)rest.R;
  // one of the two is 1, or both are
  const bool list_on_top = l.m_list >= rest.m;
  const double lesser = others && l.m_list != -kInf ? exp(((double)(list_on_top ? rest.m : l.m_list) - m) * s) : 1.0;
  const double of_rest = !others ? 0.0 : list_on_top ? lesser : 1.0, of_list = l.m_list == -kInf ? 0.0 : list_on_top ? 1.0 : lesser;
  const double z = of_rest * grow + of_list * v.z, inv_z = 1.0 / z, ln_z = ln_wide(z), ln_rest = ln_wide(grow);
  const double of_q = a.tail || !l.some ? 1.0 : 1.0 / v.q, ln_q = a.tail || !l.some ? 0.0 : l.shift + ln_wide(v.q);
  const double q_all = v.q * of_q, q_rest = a.tail && others ? fmax(0.0, 1.0 - v.q) : 0.0;
  const double over = !a.tail || !l.some ? 0.0 : others ? fmax(0.0, v.q - 1.0) : v.q - 1.0;        // Q - 1
  const double ln_p_rest = ((double)rest.m - m) * s + ln_rest - ln_z;
  double loss = (v.qy - v.qx) * of_q + (((double)m - x_shift) * s + ln_z - (ln_q - l.shift)) * q_all;
  if (q_rest > 0.0) loss += q_rest * (ln_wide(q_rest) - ln_p_rest);
  const double p_rest = others ? of_rest * grow * inv_z : 0.0, c_rest = p_rest - q_rest + over * p_rest;
  const bool in = l.some && alive;
  const float poison = l.bad ? nan_value() : 0.f;
  if (share) {
    rs.kind = l.bad || in;
    rs.m_rest = others ? rest.m : 0.f;
    rs.coef = (others ? (float)(s * weight * c_rest) / (float)grow : 0.f) + poison;
    rs.of_e = (1.0 + over) * of_list * inv_z + poison;
    rs.of_q = of_q;
    rs.weight = s * weight;
  }
  if (out) {
    if (a.loss) a.loss[r] = (in ? (float)loss : 0.f) + poison;
    if (a.stats) {
      float* o = a.stats + 8 * r;
      o[0] = m; o[1] = (float)ln_z; o[2] = rest.m; o[3] = others ? (float)ln_rest : -kInf;
      o[4] = (float)c_rest; o[5] = (float)ln_q; o[6] = (in ? 1.f : 0.f) + poison; o[7] = (float)over;
    }
  }
}

// Few rows, and the gradient at any number of them: one row per cluster of `parts` blocks, each block's slice of it in shared
// memory; at most one entry of the list a thread.
//
// While the slice is on its way, the list's side is computed: a few numbers, in 64 bits, since the loss is a small
// difference of large terms.  Its sums are taken relative to the list's own largest element, so they wait for nothing.
// Then the list's elements are taken out of the slice (set to -inf where they lie in shared memory), the rest is summed in one
// pass, blocks and list are joined, and the gradient is computed from the slice and written.
//
// With the gradient, 4096 rows of 102400 bf16 take 386 us, 0.67 of the copy rate.  A block lives 14 us, four of them on an SM: 3.2
// until slice and list are there, 2.5 for the first pass, 6 until the cluster's slowest block has joined and the figures are
// there, 2.2 for the second pass; the exponentials, two an element at 16 a cycle, take 0.7 of the memory time by themselves.
// Slower, measured: persistent blocks that take a row twice through a ring, the second time out of L2 (388 us); the same with
// other warps for the second pass, fed by a ring of their own (480); slices of two rows at a time in the shared memory of a
// pair of blocks, one group of warps for each pass (565); slices of 26 KB (645) or 104 KB (406).
template <typename T, int NT, bool GRAD>
__global__ void __launch_bounds__(NT, 1024 / NT) distill_rows_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int W = NT / 32;
  __shared__ State per_warp[W];
  __shared__ State mine;
  __shared__ uint64_t bar;
  __shared__ __align__(16) int s_id[NT];
  __shared__ float s_y[NT];
  __shared__ float warp_m[W], warp_y[W];
  __shared__ ListSums warp_sums[W];
  __shared__ int s_bad, s_twice;
  __shared__ RowShared rs;
  extern __shared__ __align__(16) unsigned char units[];
  const int part = a.parts > 1 ? (int)cluster_rank() : 0;
  const int64_t r = blockIdx.x / a.parts;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  const int V = a.V, K = a.K, tid = threadIdx.x;
  const float c = a.s * kLog2e;
  const float weight = a.weight ? a.weight[r] : 1.f;
  const Slice sl(V, row_pad(row), part, a.parts);
  const int n_units = sl.last - sl.first;
  const int e0 = max(0, 8 * sl.first - sl.pad), e1 = min(V, 8 * sl.last - sl.pad);      // the elements of the slice
  T* out = GRAD ? static_cast<T*>(a.d_logits) + r * a.d_stride : nullptr;
  const bool leader = part == 0 && tid == 0;

  if (weight == 0.f) {                                    // the whole cluster
    if (leader) {
      if (a.loss) a.loss[r] = 0.f;
      if (a.stats)
        for (int i = 0; i < 8; ++i) a.stats[8 * r + i] = 0.f;
    }
    if (GRAD) write_elements(out, e0, e1, NT, tid, [](int) { return 0.f; });
    return;
  }

  if (tid == 0) s_bad = s_twice = 0;
  start_slice(row, V, sl, units, &bar);
  const double s = a.s;
  int id = -1;
  float y = -kInf, x = -kInf;
  bool bad = false;
  if (tid < K) {
    id = a.ids[r * K + tid];
    y = a.y[r * K + tid];
    bad = id < -1 || id >= V || (id >= 0 && !(y < kInf));
    if (id < 0 || id >= V) { id = -1; y = -kInf; }
    else x = Elem<T>::get(row + id);
  }
  s_id[tid] = id;
  s_y[tid] = y;
  float m_list = x, y_top = y;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    m_list = max_nan(m_list, __shfl_xor_sync(0xffffffffu, m_list, o));
    y_top = fmaxf(y_top, __shfl_xor_sync(0xffffffffu, y_top, o));
  }
  if ((tid & 31) == 0) { warp_m[tid >> 5] = m_list; warp_y[tid >> 5] = y_top; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) {
    m_list = max_nan(m_list, warp_m[w]);
    y_top = fmaxf(y_top, warp_y[w]);
  }
  const bool some = y_top > -kInf;
  const double shift = a.tail || !some ? 0.0 : (double)y_top;
  bool first = id >= 0;                                   // no entry before this one has its id
  if (first) {
    const int4* ids4 = reinterpret_cast<const int4*>(s_id);
    for (int j = 0; j < (tid >> 2); ++j) {
      const int4 v = ids4[j];
      first = first && v.x != id && v.y != id && v.z != id && v.w != id;
    }
    for (int j = tid & ~3; j < tid; ++j) first = first && s_id[j] != id;
    if (!first) s_twice = 1;
  }
  if (bad) s_bad = 1;
  const double x_shift = m_list != -kInf ? (double)m_list : 0.0;
  double e = 0.0, q = 0.0;
  if (first && m_list != -kInf) e = exp(((double)x - m_list) * s);
  if (y > -kInf) q = exp((double)y - shift);
  {
    ListSums v{e, q, 0.0, 0.0};
    if (q != 0.0) { v.qy = q * ((double)y - shift); v.qx = q * (((double)x - x_shift) * s); }
    v = warp_sum(v);
    if ((tid & 31) == 0) warp_sums[tid >> 5] = v;
  }

  const bool arrived = wait_slice(&bar);
  if (id >= e0 && id < e1) reinterpret_cast<T*>(units)[id + sl.pad - 8 * sl.first] = Elem<T>::masked();
  __syncthreads();
  constexpr int N = sizeof(T) == 2 ? 4 : 2;
  Stream<T, false, false> st(c);
  {
    int u = tid;
    for (; u + (N - 1) * NT < n_units; u += N * NT) {
      Unit<T> v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) load_shared_unit(units, u + i * NT, v[i]);
      st.add(v);
    }
    for (; u < n_units; u += NT) {
      Unit<T> v[1];
      load_shared_unit(units, u, v[0]);
      st.add(v);
    }
  }
  join_block<NT>(arrived ? st.finish() : State{0.f, nan_value(), nan_value()}, c, per_warp, &mine);
  if (a.parts > 1) {
    cluster_sync();
  }
  if (tid < 32) {
    __syncwarp();
    const State rest = a.parts > 1 ? join_cluster(&mine, a.parts, c) : mine;
    ListSums v = warp_sums[0];
    for (int w = 1; w < W; ++w) { v.z += warp_sums[w].z; v.q += warp_sums[w].q; v.qy += warp_sums[w].qy; v.qx += warp_sums[w].qx; }
    const ListSide list{v, m_list, shift, some, s_bad != 0};
    finish_row(a, r, weight, rest, list, tid == 0, leader, rs);
  }
  if (a.parts > 1) {
    __syncwarp();
    cluster_arrive();                                     // this block has read what it needs of the others
  }
  if (GRAD) {
    __syncthreads();
    if (rs.kind == 0) {
      write_elements(out, e0, e1, NT, tid, [](int) { return 0.f; });
    } else {
      const float m_rest = rs.m_rest, coef = rs.coef;
      if (row_pad(out) == sl.pad) {
        for (int u = tid; u < n_units; u += NT) {
          Unit<T> v;
          load_shared_unit(units, u, v);
          rest_grad_unit(v, m_rest, c, coef);
          const int g = sl.first + u;
          if (g >= sl.full0 && g < sl.full1) store_unit(out - sl.pad + 8 * (int64_t)g, v);
          else store_ragged(out, V, sl.pad, g, v);
        }
      } else {
        const T* own = reinterpret_cast<const T*>(units) + sl.pad - 8 * sl.first;
        write_elements(out, e0, e1, NT, tid, [&](int i) { return coef * ex2((Elem<T>::get(own + i) - m_rest) * c); });
      }
      __syncthreads();                                    // the list's elements go over what was just written there
      if (first && id >= e0 && id < e1) {
        double of_id = q;
        if (s_twice)
          for (int j = tid + 1; j < K; ++j)
            if (s_id[j] == id && s_y[j] > -kInf) of_id += exp((double)s_y[j] - shift);
        Elem<T>::put(out + id, (float)(rs.weight * (e * rs.of_e - of_id * rs.of_q)));
      }
    }
  }
  if (a.parts > 1) cluster_wait();                        // no block leaves while another reads its shared memory
}

// ---- many rows ---------------------------------------------------------------------------------------------------
// Persistent blocks (logit_rows.cuh).  The list's elements are taken out of each chunk that arrives (-inf in shared memory)
// by a warp between the copies and the consumers, so their loop knows nothing of lists.
struct alignas(16) ListShared {
  int id[kMaxList];                // -1: unused entry
  unsigned char first[kMaxList];   // no entry before it has its id
  ListSide side;
  unsigned loose[2];               // bits of the slice's ragged units that are listed
};
constexpr int kHash = 2 * kMaxList, kLists = kMaxList / 32;      // table in which ids that come twice are looked for; entries a lane

// One warp's registers for the list of a row: entries lane, lane + 32, ...
template <typename T>
struct ListFetch {
  int id[kLists];
  float y[kLists];
  T x[kLists];                     // as loaded: a conversion would wait for it
  __device__ __forceinline__ void entries(const DistillArgs& a, int64_t r) {
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
      const int k = (threadIdx.x & 31) + 32 * i;
      id[i] = -1;
      y[i] = -kInf;
      if (k < a.K && r < a.n_rows) { id[i] = a.ids[r * a.K + k]; y[i] = a.y[r * a.K + k]; }
    }
  }
  __device__ __forceinline__ void logits(const DistillArgs& a, int64_t r) {
#pragma unroll
    for (int i = 0; i < kLists; ++i)
      x[i] = id[i] >= 0 && id[i] < a.V ? static_cast<const T*>(a.logits)[r * a.stride + id[i]] : Elem<T>::masked();
  }
};

// One warp: brings a fetched list into l and computes its sums.  `ids_out` is called when ids and loose are in place, the rest follows.
template <typename T, typename Ids>
__device__ __forceinline__ void lay_list(const DistillArgs& a, ListFetch<T>& f, const Slice& sl, ListShared& l, int* seen, Ids ids_out) {
  const int lane = threadIdx.x & 31, V = a.V, K = a.K;
  const double s = a.s;
  int (&id)[kLists] = f.id;
  float (&y)[kLists] = f.y;
  T (&x)[kLists] = f.x;
#pragma unroll
  for (int i = 0; i < kHash / 128; ++i) reinterpret_cast<int4*>(seen)[lane + 32 * i] = make_int4(-1, -1, -1, -1);
  bool bad = false, twice = false;
  float m_list = -kInf, y_top = -kInf;
  unsigned loose = 0;
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    const int k = lane + 32 * i;
    bad = bad || id[i] < -1 || id[i] >= V || (id[i] >= 0 && !(y[i] < kInf));
    if (id[i] < 0 || id[i] >= V) { id[i] = -1; y[i] = -kInf; }
    if (k < K) { l.id[k] = id[i]; l.first[k] = id[i] >= 0; }
    y_top = fmaxf(y_top, y[i]);
    const int u = (id[i] + sl.pad) >> 3;
    if (id[i] >= 0 && sl.holds(id[i]) && !(u >= sl.full0 && u < sl.full1)) loose |= 1u << ((id[i] + sl.pad) & 7) << (u == sl.ragged(0) ? 0 : 8);
  }
  loose = __reduce_or_sync(0xffffffffu, loose);
  if (lane == 0) { l.loose[0] = loose & 0xffu; l.loose[1] = loose >> 8; }
  __syncwarp();
  ids_out();
  // an id that is in the table already stands in the list twice: rare, and worked out entry by entry
#pragma unroll
  for (int i = 0; i < kLists; ++i)
    if (id[i] >= 0)
      for (int h = (int)((unsigned)id[i] * 2654435761u >> 16) & (kHash - 1);; h = (h + 1) & (kHash - 1)) {
        const int was = atomicCAS(&seen[h], -1, id[i]);
        if (was == -1) break;
        if (was == id[i]) { twice = true; break; }
      }
  twice = __any_sync(0xffffffffu, twice);
  if (twice)
    for (int k = lane; k < K; k += 32)
      for (int j = 0; j < k; ++j)
        if (l.id[j] == l.id[k]) l.first[k] = 0;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kLists; ++i) m_list = max_nan(m_list, Elem<T>::get(&x[i]));
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    m_list = max_nan(m_list, __shfl_xor_sync(0xffffffffu, m_list, o));
    y_top = fmaxf(y_top, __shfl_xor_sync(0xffffffffu, y_top, o));
  }
  const bool some = y_top > -kInf;
  const double shift = a.tail || !some ? 0.0 : (double)y_top, x_shift = m_list != -kInf ? (double)m_list : 0.0;
  ListSums sums{0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    if (32 * i >= K) continue;
    const int k = lane + 32 * i;
    const double xi = Elem<T>::get(&x[i]);
    if (k < K && l.first[k] && m_list != -kInf) sums.z += exp((xi - m_list) * s);
    if (y[i] > -kInf) {
      const double q = exp((double)y[i] - shift);
      if (q != 0.0) {
        sums.q += q;
        sums.qy += q * ((double)y[i] - shift);
        sums.qx += q * ((xi - x_shift) * s);
      }
    }
  }
  sums = warp_sum(sums);
  bad = __any_sync(0xffffffffu, bad);
  if (lane == 0) l.side = ListSide{sums, m_list, shift, some, bad};
  __syncwarp();
}

// One warp: takes the listed elements of a slice out of its chunks and passes them on.
template <typename T, int NB, int CHUNK>
__device__ __forceinline__ void pass_chunks(const Slice& sl, const ListShared& l, int K, unsigned char* buf, RingPlace<NB>& in, uint64_t* full, uint64_t* passed) {
  typedef Chunks<T, CHUNK> C;
  const int lane = threadIdx.x & 31;
  int id[kLists], at[kLists];              // entries lane, lane + 32, ...; chunk of each (-1: in none)
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    id[i] = lane + 32 * i < K ? l.id[lane + 32 * i] : -1;
    const int u = (id[i] + sl.pad) >> 3;
    at[i] = id[i] >= 0 && u >= sl.full0 && u < sl.full1 ? (u - sl.full0) / C::kUnits : -1;
  }
  const int n = C::count(sl);
  for (int ch = 0; ch < n; ++ch) {
    in.wait(full);
    T* const chunk = reinterpret_cast<T*>(buf + in.slot * CHUNK) + sl.pad - 8 * (sl.full0 + ch * C::kUnits);
    bool wrote = false;
#pragma unroll
    for (int i = 0; i < kLists; ++i)
      if (at[i] == ch) { chunk[id[i]] = Elem<T>::masked(); wrote = true; }
    if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // before a later copy goes over it
    in.pass(passed, wrote);
  }
}

// Sums of what is left of a slice, by NT threads (tid: 0 .. NT - 1).
template <typename T, int NT, int NB, int CHUNK>
__device__ __forceinline__ State sum_slice(const T* row, int V, const Slice& sl, const ListShared& l, const unsigned char* buf, float c, int tid,
                                           RingPlace<NB>& in, uint64_t* passed, uint64_t* empty) {
  typedef Chunks<T, CHUNK> C;
  constexpr int N = C::kUnits / NT;
  static_assert(C::kUnits % NT == 0, "whole units for every thread");
  Unit<T> loose[1];
  const bool has_loose = tid < 2 && sl.ragged(tid) >= 0;
  if (has_loose) load_ragged(row, V, sl.pad, sl.ragged(tid), loose[0]);
  Stream<T, false, false> st(c);
  const int chunks = C::count(sl);
  for (int ch = 0; ch < chunks; ++ch) {
    const int n = C::units(sl, ch);
    in.wait(passed);
    const unsigned char* units = buf + in.slot * CHUNK;
    if (n == C::kUnits) {
      Unit<T> q[N];
#pragma unroll
      for (int i = 0; i < N; ++i) load_shared_unit(units, tid + i * NT, q[i]);
      st.add(q);
    } else {
#pragma unroll 1
      for (int u = tid; u < n; u += NT) {
        Unit<T> q[1];
        load_shared_unit(units, u, q[0]);
        st.add(q);
      }
    }
    in.pass(empty, st.top() == 1.f);
  }
  if (has_loose) {                         // those are not in the ring; the chunks' barriers have made the list visible
    const unsigned bits = l.loose[tid];
    float v[8];
    loose[0].values(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = bits >> j & 1u ? -kInf : v[j];
    loose[0].set(v);
    st.add(loose);
  }
  return in.ok ? st.finish() : State{0.f, nan_value(), nan_value()};
}

// The loss alone (1024 rows of 151936 bf16: 65 us, 0.73 of the copy rate; 10 us of them until the first lists are there and
// behind the last row).  Warps of a block, each at its own pace:
//   producer   issues the copies;
//   listers    two, for every second row each, up to two rows ahead: read the lists and compute their sums (two dependent loads
//              behind the copies on their way take 5 us each);
//   passer     takes the list's elements out of the chunks;
//   consumers  sum what is left;
//   finisher   joins sums and list and writes the loss.
template <typename T>
struct LossShape {
  static constexpr int kConsumers = 128, kBlocks = 4, kSlots = 3;
  static constexpr int kChunk = kConsumers * 16 * (sizeof(T) == 2 ? 6 : 4);
  static constexpr int kThreads = kConsumers + 160;
  static constexpr size_t kSmem = (size_t)kChunk * kSlots;
};

template <typename T>
__global__ void __launch_bounds__(LossShape<T>::kThreads, LossShape<T>::kBlocks) distill_loss_kernel(const __grid_constant__ DistillArgs a) {
  typedef LossShape<T> Shape;
  constexpr int NT = Shape::kConsumers, NB = Shape::kSlots, CHUNK = Shape::kChunk, PAIR = NT + 32;
  __shared__ PipeShared<NB> ps;
  __shared__ uint64_t passed[NB];              // chunks that the passer is done with
  __shared__ State per_warp[2][NT / 32];
  __shared__ ListShared lists[2];
  __shared__ __align__(16) int seen[2][kHash];
  __shared__ RowShared unused;
  extern __shared__ __align__(128) unsigned char ring_buffer[];
  const int V = a.V, tid = threadIdx.x, lane = tid & 31;
  const T* logits = static_cast<const T*>(a.logits);
  const float c = a.s * kLog2e;
  RowWeights weights(a.weight, a.n_rows, blockIdx.x, gridDim.x);
  if (tid == 0) {
    init_pipe(ps, NT / 32);
    for (int i = 0; i < NB; ++i) ring::mbar_init(&passed[i], 1);
    ring::mbar_fence_init();
  }
  __syncthreads();
  const int role = tid < NT ? 0 : (tid - NT) / 32 + 1;
  auto slice_of = [&](int64_t r) { return Slice(V, row_pad(logits + r * a.stride), 0, 1); };

  if (role == 5) {
    produce<T, NB, CHUNK>(ps, ring_buffer, weights, logits, a.stride, V);
  } else if (role >= 3) {                      // listers
    const int par = role - 3;
    int i_row = weights.next(0);
    if (par) i_row = weights.next(i_row + 1);
    for (bool again = false; weights.row(i_row) < a.n_rows; i_row = weights.next(weights.next(i_row + 1) + 1), again = true) {
      const int64_t r = weights.row(i_row);
      ListFetch<T> f;
      f.entries(a, r);
      f.logits(a, r);
      if (again) bar_sync<kBarListFree, 64>(par);
      lay_list<T>(a, f, slice_of(r), lists[par], seen[par], [&] { bar_arrive<kBarIds, 64>(par); });
      bar_arrive<kBarList, 64>(par);
    }
  } else if (role == 2) {                      // passer
    RingPlace<NB> in;
    int par = 0;
    for (int i_row = weights.next(0); weights.row(i_row) < a.n_rows; i_row = weights.next(i_row + 1), par ^= 1) {
      bar_sync<kBarIds, 64>(par);
      pass_chunks<T, NB, CHUNK>(slice_of(weights.row(i_row)), lists[par], a.K, ring_buffer, in, ps.full, passed);
    }
  } else if (role == 1) {                      // finisher
    int par = 0;
    for (int i_row = 0; weights.row(i_row) < a.n_rows; ++i_row) {
      const int64_t r = weights.row(i_row);
      const float weight = weights.at(i_row);
      if (weight == 0.f) {
        if (lane == 0 && a.loss) a.loss[r] = 0.f;
        if (lane < 8 && a.stats) a.stats[8 * r + lane] = 0.f;
        continue;
      }
      const bool later = weights.row(weights.next(weights.next(i_row + 1) + 1)) < a.n_rows;      // a row will wait for this one's buffers
      bar_sync<kBarList, 64>(par);
      bar_sync<kBarReady, PAIR>(par);
      finish_row(a, r, weight, join_warps<NT>(per_warp[par], c), lists[par].side, false, lane == 0, unused);
      __syncwarp();
      if (later) {
        bar_arrive<kBarListFree, 64>(par);
        bar_arrive<kBarFree, PAIR>(par);
      }
      par ^= 1;
    }
  } else {                                     // consumers
    RingPlace<NB> in;
    int par = 0, done = 0;
    for (int i_row = weights.next(0); weights.row(i_row) < a.n_rows; i_row = weights.next(i_row + 1), par ^= 1, ++done) {
      const T* row = logits + weights.row(i_row) * a.stride;
      if (done >= 2) bar_sync<kBarFree, PAIR>(par);
      join_warp(sum_slice<T, NT, NB, CHUNK>(row, V, slice_of(weights.row(i_row)), lists[par], ring_buffer, c, tid, in, passed, ps.empty), c, per_warp[par]);
      bar_arrive<kBarReady, PAIR>(par);
    }
  }
}

__device__ __forceinline__ float exp32(double x) { return ex2((float)x * kLog2e); }
constexpr double kFaintLog = -745.0;            // e^x of less is 0 in 64 bits as well

// Rows of up to 256 elements: LPR lanes a row, eight elements a lane, the list laid out over the row's elements in shared
// memory.  BACKWARD takes what rows share from row_stats instead of computing it.  Exponentials are float32, sums and
// the loss's logarithms 64 bits: the terms' own errors are relative (2e-7) and do not grow where list and row nearly agree,
// while 64-bit exponentials took a third of the time (13312 rows of 64: 12 us with float32 ones, 18 with 64-bit ones).  The list's sum is one where it is
// subtracted from one (tail), and so are probabilities that a float32 exponential flushes to zero, in a walk of their own.
template <typename T, int LPR, bool GRAD, bool BACKWARD>
__global__ void __launch_bounds__(256) distill_small_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int G = 256 / LPR, W = 8 * LPR;       // rows a block; entries and elements a row at most
  __shared__ int s_id[G][W], s_owner[G][W];
  __shared__ float s_y[G][W];
  __shared__ float s_q[G][W];                     // by element: the list's probability
  const int lane = threadIdx.x & (LPR - 1), gi = threadIdx.x / LPR;
  const int64_t r = (int64_t)blockIdx.x * G + gi;
  const bool there = r < a.n_rows;
  const int64_t rr = there ? r : 0;
  const int V = a.V, K = a.K;
  const T* row = static_cast<const T*>(a.logits) + rr * a.stride;
  const float c = a.s * kLog2e, weight = a.weight ? a.weight[rr] : 1.f;
  const double s = a.s;
  auto group_sum = [](double v) {
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o, LPR);
    return v;
  };
  auto group_max = [](float v) {
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o, LPR));
    return v;
  };
  const unsigned group_bits = (LPR == 32 ? 0xffffffffu : ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1)));
  auto group_any = [&](bool p) { return (__ballot_sync(0xffffffffu, p) & group_bits) != 0; };

  Unit<T> q;
  if (row_pad(row) == 0 && 8 * lane + 8 <= V) load_unit(row + 8 * lane, q);
  else load_ragged(row, V, 0, lane, q);
  for (int v = lane; v < W; v += LPR) { s_owner[gi][v] = -1; s_q[gi][v] = 0.f; }
  __syncwarp();
  bool bad = false;
  float ytop = -kInf;
#pragma unroll 4
  for (int k = lane; k < K; k += LPR) {
    const int id = a.ids[rr * K + k];
    const float y = a.y[rr * K + k];
    const bool used = id >= 0 && id < V;
    bad = bad || id < -1 || id >= V || (id >= 0 && !(y < kInf));
    s_id[gi][k] = used ? id : -1;
    s_y[gi][k] = used ? y : -kInf;
    ytop = fmaxf(ytop, used ? y : -kInf);
    if (used) s_owner[gi][id] = k;               // of entries with one id, any
  }
  __syncwarp();
  bad = group_any(bad);
  ytop = group_max(ytop);
  const bool some = ytop > -kInf;
  bool twice = false;
#pragma unroll 4
  for (int k = lane; k < K; k += LPR) twice = twice || (s_id[gi][k] >= 0 && s_owner[gi][s_id[gi][k]] != k);
  twice = group_any(twice);
  double ln_q = 0.0, qs = 0.0, entropy = 0.0;     // entropy: sum of q ln q over the list
  bool faint = false;                             // q that is 0 as float32 (but may be infinitely or greatly far from p)
  if (BACKWARD) {
    ln_q = a.stats_in[8 * rr + 5];
  } else if (some) {
    const double shift = a.tail ? 0.0 : (double)ytop;
#pragma unroll 4
    for (int k = lane; k < K; k += LPR) qs += a.tail ? exp((double)s_y[gi][k]) : (double)exp32((double)s_y[gi][k] - shift);
  }
  if (!BACKWARD) {
    qs = group_sum(qs);
    ln_q = a.tail || !some ? 0.0 : (double)ytop + ln_wide(qs);
  }
#pragma unroll 4
  for (int k = lane; k < K; k += LPR) {
    const int id = s_id[gi][k];
    if (id < 0) continue;
    const double ln = (double)s_y[gi][k] - ln_q;
    float p = exp32(ln);
    if (p != 0.f) entropy += p * ln;
    else faint = faint || ln > kFaintLog;
    if (twice) {
      for (int j = 0; j < k; ++j)
        if (s_id[gi][j] == id) p = -1.f;          // the first entry of the id has summed it
      if (p >= 0.f)
        for (int j = k + 1; j < K; ++j)
          if (s_id[gi][j] == id) p += exp32((double)s_y[gi][j] - ln_q);
    }
    if (p >= 0.f) s_q[gi][id] = p;
  }
  __syncwarp();
  float v[8];
  q.values(v);
  unsigned listed = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) listed |= s_owner[gi][8 * lane + j] >= 0 ? 1u << j : 0u;

  float m, m_rest, coef, flag, inv_z;             // inv_z: Q / Z
  double ln_z;
  if (BACKWARD) {
    const float* o = a.stats_in + 8 * rr;
    m = o[0]; ln_z = o[1]; flag = o[6];
    inv_z = (1.f + o[7]) * ex2(-(float)ln_z * kLog2e);
    const bool others = o[2] > -kInf;
    m_rest = others ? o[2] : 0.f;
    coef = others ? a.s * weight * o[4] * ex2(-o[3] * kLog2e) : 0.f;
  } else {
    float top = -kInf;
    Unit<T> w[1];
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = listed >> j & 1u ? -kInf : v[j];
      top = max_nan(top, listed >> j & 1u ? v[j] : -kInf);
    }
    w[0].set(x);
    Stream<T, false, false> st(c);
    st.add(w);
    State rest = st.finish();
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) rest = merge(rest, shuffle_down(rest, o, LPR), c);
    rest.m = __shfl_sync(0xffffffffu, rest.m, 0, LPR);
    rest.R = __shfl_sync(0xffffffffu, rest.R, 0, LPR);
    m = max_nan(rest.m, group_max(top));
    const bool alive = m != -kInf, others = rest.m > -kInf;
    double z = 0.0;
    if (alive) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (listed >> j & 1u) z += ex2((v[j] - m) * c);
    }
    const double of_rest = others ? (double)ex2((rest.m - m) * c) * (1.0 + (double)rest.R) : 0.0;
    z = group_sum(z) + of_rest;
    ln_z = ln_wide(z);
    const double q_rest = a.tail && others ? fmax(0.0, 1.0 - qs) : 0.0;
    const double ln_rest = ln_wide(1.0 + (double)rest.R), ln_p_rest = ((double)rest.m - m) * s + ln_rest - ln_z;
    double loss = entropy;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (listed >> j & 1u) {
        const float p = s_q[gi][8 * lane + j];
        if (p != 0.f) loss -= p * (((double)v[j] - m) * s - ln_z);
      }
    if (group_any(faint))
      for (int k = lane; k < K; k += LPR) {
        const int id = s_id[gi][k];
        const double ln = id >= 0 ? (double)s_y[gi][k] - ln_q : 0.0;
        if (ln > kFaintLog && exp32(ln) == 0.f) loss += exp(ln) * (ln - (((double)Elem<T>::get(row + id) - m) * s - ln_z));
      }
    loss = group_sum(loss);
    if (q_rest > 0.0) loss += q_rest * (ln_wide(q_rest) - ln_p_rest);
    inv_z = (float)(1.0 / z);
    double c_rest = others ? of_rest / z - q_rest : 0.0;
    float over = 0.f;                               // Q - 1
    if (a.tail && some && (!others || qs > 1.0)) {
      over = (float)(qs - 1.0);
      inv_z += over * inv_z;
      if (others) c_rest += (qs - 1.0) * (of_rest / z);
    }
    const bool in = some && alive;
    flag = bad ? nan_value() : in ? 1.f : 0.f;
    m_rest = others ? rest.m : 0.f;
    coef = others ? (float)(s * weight * c_rest) / (1.f + rest.R) : 0.f;
    if (there && lane == 0) {
      const bool counts = weight != 0.f;
      if (a.loss) a.loss[r] = !counts ? 0.f : bad ? nan_value() : in ? (float)loss : 0.f;
      if (a.stats) {
        float* o = a.stats + 8 * r;
        o[0] = m; o[1] = (float)ln_z; o[2] = rest.m; o[3] = others ? (float)ln_rest : -kInf;
        o[4] = (float)c_rest; o[5] = (float)ln_q; o[6] = counts ? flag : 0.f; o[7] = over;
      }
    }
  }
  if (GRAD && there && 8 * lane < V) {
    T* out = static_cast<T*>(a.d_logits) + r * a.d_stride;
    float d[8];
    if (weight == 0.f || flag == 0.f) {
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = 0.f;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (listed >> j & 1u) d[j] = a.s * weight * (ex2((v[j] - m) * c) * inv_z - s_q[gi][8 * lane + j]);
        else d[j] = coef * ex2((v[j] - m_rest) * c);
        if (!(flag == flag)) d[j] = flag;
      }
    }
    q.set(d);
    if (row_pad(out) == 0 && 8 * lane + 8 <= V) store_unit(out + 8 * lane, q);
    else store_ragged(out, V, 0, lane, q);
  }
}

// Element-wise from the row_stats, `parts` blocks a row, at most one entry of the list a thread.
template <typename T>
__global__ void __launch_bounds__(kPieceThreads, 6) distill_backward_kernel(const __grid_constant__ DistillArgs a) {
  static_assert(kMaxList <= kPieceThreads, "one entry a thread");
  __shared__ int s_id[kMaxList];
  __shared__ float s_y[kMaxList];
  const int tid = threadIdx.x, V = a.V, K = a.K;
  const int64_t r = blockIdx.x / a.parts;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* out = static_cast<T*>(a.d_logits) + r * a.d_stride;
  const Piece<T> piece(row, out, V, (int)(blockIdx.x - (unsigned)r * (unsigned)a.parts), a.parts);
  Unit<T> q[Piece<T>::kUnits];
  piece.load_batch(piece.u0 + tid, q);
  int id = -1;
  float y = -kInf;
  if (tid < K) {
    id = a.ids[r * K + tid];
    y = a.y[r * K + tid];
  }
  const float* o = a.stats_in + 8 * r;
  const float m = o[0], ln_z = o[1], m_out = o[2], ln_z_out = o[3], c_rest = o[4], ln_q = o[5], flag = o[6], weight = a.weight[r], c = a.s * kLog2e;
  if (weight == 0.f || flag == 0.f || !(flag == flag)) {
    piece.fill(weight == 0.f || flag == 0.f ? 0.f : flag);
    return;
  }
  const bool others = m_out > -kInf;
  const float m_rest = others ? m_out : 0.f, coef = others ? a.s * weight * c_rest * ex2(-ln_z_out * kLog2e) : 0.f;
  // the entries of this piece: their logits before anything is written over
  const int at = (id + piece.pad) >> 3;
  bool mine = id >= 0 && id < V && at >= piece.u0 && at < piece.u1, twice = false;
  T x = Elem<T>::masked();
  if (mine) x = row[id];
  if (tid < K) {
    s_id[tid] = id >= 0 && id < V ? id : -1;
    s_y[tid] = y;
  }
  __syncthreads();
  piece.run(q, [&](int, Unit<T>& v) { rest_grad_unit(v, m_rest, c, coef); });
  __syncthreads();                               // the list's elements go over what was just written there
  if (mine) {
    for (int j = 0; j < K; ++j)
      if (j != tid && s_id[j] == id) {
        twice = true;
        if (j < tid) mine = false;
      }
    if (mine) Elem<T>::put(out + id, entry_gradient<T>(m, ln_z, ln_q, a.stats_in[8 * r + 7], a.s, weight, s_id, s_y, K, tid, Elem<T>::get(&x), twice));
  }
}

template <typename T, int LPR>
cudaError_t launch_small(const DistillArgs& a, bool backward, cudaStream_t st) {
  const int64_t blocks = ((int64_t)a.n_rows + 256 / LPR - 1) / (256 / LPR);
  return backward     ? launch<distill_small_kernel<T, LPR, true, true>>(a, blocks, 1, 256, 0, st)
         : a.d_logits ? launch<distill_small_kernel<T, LPR, true, false>>(a, blocks, 1, 256, 0, st)
                      : launch<distill_small_kernel<T, LPR, false, false>>(a, blocks, 1, 256, 0, st);
}

template <typename T>
cudaError_t launch_distill(DistillArgs a, bool backward, cudaStream_t st) {
  if (a.V <= kSmallVocab)
    return a.V <= 64    ? launch_small<T, 8>(a, backward, st)
           : a.V <= 128 ? launch_small<T, 16>(a, backward, st)
                        : launch_small<T, 32>(a, backward, st);
  if (backward) {
    a.parts = pieces_of_row(a.V, sizeof(T), 128 * 1024);
    return launch<distill_backward_kernel<T>>(a, (int64_t)a.n_rows * a.parts, 1, kPieceThreads, 0, st);
  }
  if (!a.d_logits && many_rows(a.n_rows, a.V)) return launch_pipe<distill_loss_kernel<T>, LossShape<T>>(a, st);
  a.parts = parts_of_row(a.n_rows, a.V, sizeof(T));
  a.slice_bytes = slice_bytes(a.V, sizeof(T), a.parts);
  if (a.V >= 8192 || a.K > 128)
    return a.d_logits ? launch_resident<distill_rows_kernel<T, 256, true>, 256>(a, 0, st)
                      : launch_resident<distill_rows_kernel<T, 256, false>, 256>(a, 0, st);
  return a.d_logits ? launch_resident<distill_rows_kernel<T, 128, true>, 128>(a, 0, st)
                    : launch_resident<distill_rows_kernel<T, 128, false>, 128>(a, 0, st);
}

int run_distill(const DistillArgs& a, int32_t dtype, bool backward, void* cuda_stream) {
  if (a.n_rows == 0) return REMOE_OK;
  PointerDevice dev(a.logits);
  if (dev.err_code() != REMOE_OK) return dev.err_code();
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == REMOE_F32 ? launch_distill<float>(a, backward, st)
                        : dtype == REMOE_BF16 ? launch_distill<__nv_bfloat16>(a, backward, st) : launch_distill<__half>(a, backward, st);
  return status(e);
}

int check_distill(const DistillArgs& a, int32_t dtype) {
  const int rc = check_rows(a.n_rows, a.V, dtype, a.logits, a.stride, a.s);
  if (rc != REMOE_OK) return rc;
  if (a.K < 1 || a.K > a.V) return REMOE_E_ARG;
  if (a.K > REMOE_ROWS_MAX_TOP) return REMOE_E_UNSUPPORTED;
  if (!a.ids || !a.y) return REMOE_E_ARG;
  if (a.d_logits && ((a.d_stride < a.V && a.n_rows > 1) || misaligned(a.d_logits, element_size(dtype)))) return REMOE_E_ARG;
  if (a.d_logits == a.logits && a.d_stride != a.stride && a.n_rows > 1) return REMOE_E_ARG;
  if (misaligned(a.ids, 4) || misaligned(a.y, 4) || misaligned(a.weight, 4) || misaligned(a.loss, 4) || misaligned(a.stats, 4) ||
      misaligned(a.stats_in, 4))
    return REMOE_E_ARG;
  return REMOE_OK;
}

}  // namespace rows
}  // namespace remoe

extern "C" int remoe_distill_topk(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits_dev, int64_t row_stride,
                                  float inv_temperature, int32_t n_top, const int32_t* teacher_ids_dev,
                                  const float* teacher_logprobs_dev, int32_t tail, const float* row_weight_dev, float* loss_dev,
                                  float* row_stats_dev, void* d_logits_dev, int64_t d_row_stride, void* cuda_stream) {
  using namespace remoe::rows;
  DistillArgs a{logits_dev, d_logits_dev, row_stride, d_row_stride, vocab, n_rows, 1, 0, n_top, tail, inv_temperature,
                teacher_ids_dev, teacher_logprobs_dev, row_weight_dev, loss_dev, row_stats_dev, nullptr};
  const int rc = check_distill(a, dtype);
  if (rc != REMOE_OK) return rc;
  if ((tail != 0 && tail != 1) || (!loss_dev && !row_stats_dev && !d_logits_dev)) return REMOE_E_ARG;
  return run_distill(a, dtype, false, cuda_stream);
}

extern "C" int remoe_distill_topk_backward(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits_dev,
                                           int64_t row_stride, float inv_temperature, int32_t n_top,
                                           const int32_t* teacher_ids_dev, const float* teacher_logprobs_dev,
                                           const float* row_stats_dev, const float* grad_loss_dev, void* d_logits_dev,
                                           int64_t d_row_stride, void* cuda_stream) {
  using namespace remoe::rows;
  DistillArgs a{logits_dev, d_logits_dev, row_stride, d_row_stride, vocab, n_rows, 1, 0, n_top, 0, inv_temperature,
                teacher_ids_dev, teacher_logprobs_dev, grad_loss_dev, nullptr, nullptr, row_stats_dev};
  const int rc = check_distill(a, dtype);
  if (rc != REMOE_OK) return rc;
  if (!row_stats_dev || !grad_loss_dev || !d_logits_dev) return REMOE_E_ARG;
  return run_distill(a, dtype, true, cuda_stream);
}
