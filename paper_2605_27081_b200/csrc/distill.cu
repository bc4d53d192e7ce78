// remoe_distill_topk / remoe_distill_topk_backward: divergence of rows of logits from a teacher that is known by its
// top log probabilities, and its gradient.
//
// S: the ids of the list.  q = softmax of the list's values, or (tail) their exp with q_r = 1 - sum q as one more
// class for all that is not listed; p_r = the student's mass outside S.
//   loss = sum_S q (ln q - ln p) + q_r (ln q_r - ln p_r)
//   dx_v = s w (p_v - q_v)                            v in S
//          s w (p_r - q_r) e^{s x_v} / sum_{not S}    v not in S
// The second line is p_v (1 - q_r / p_r), written so that it holds where the student leaves nearly nothing outside S:
// the sum outside S is taken over those elements alone, not as a difference.
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
  int V, n_rows, parts, K, tail;
  float s;
  const int32_t* ids;
  const float *y, *weight;
  float *loss, *stats;
  const float* stats_in;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What the gradient of a row needs.
struct RowGrad {
  float m_rest, coef;        // outside the list: coef * 2^((x - m_rest) c)
  float m;
  double ln_z, ln_q, weight; // in the list: weight * (e^{(x - m) s - ln_z} - e^{y - ln_q})
  int kind;                  // 0: left out (zeros), 1: takes part
};

struct EntryShared {
  int id[kMaxList];          // -1: unused entry
  float y[kMaxList];
  float x[kMaxList];
  int first[kMaxList];       // no entry before it has its id
  int bad, twice;
  RowGrad g;
};

// Gradient at entry k, for the first entry of its id: the list's probabilities of that id summed in order.
__device__ __forceinline__ float entry_gradient(const RowGrad& g, double s, const int* id, const float* y, int K, int k, float x, bool twice) {
  double q = 0.0;
  if (twice) {
    for (int j = k; j < K; ++j)
      if (id[j] == id[k]) q += exp((double)y[j] - g.ln_q);
  } else {
    q = exp((double)y[k] - g.ln_q);
  }
  return (float)(g.weight * (exp(((double)x - g.m) * s - g.ln_z) - q));
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

template <typename T>
__device__ __forceinline__ void fill_unit(Unit<T>& q, float x) {
  const float v[8] = {x, x, x, x, x, x, x, x};
  q.set(v);
}

// One row per cluster of `parts` blocks.
template <typename T, int NT, bool GRAD>
__global__ void __launch_bounds__(NT) distill_rows_kernel(const __grid_constant__ DistillArgs a) {
  __shared__ State per_warp[NT / 32];
  __shared__ State mine;
  __shared__ EntryShared en;
  extern __shared__ __align__(16) unsigned listed_words[];     // one byte per unit of the slice: which elements are in the list
  const unsigned char* listed = reinterpret_cast<const unsigned char*>(listed_words);
  const int part = a.parts > 1 ? (int)cluster_rank() : 0;
  const int64_t r = blockIdx.x / a.parts;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  const int V = a.V, K = a.K, tid = threadIdx.x;
  const float c = a.s * kLog2e;
  const float weight = a.weight ? a.weight[r] : 1.f;
  T* out = GRAD ? static_cast<T*>(a.d_logits) + r * a.d_stride : nullptr;
  const int out_pad = GRAD ? row_pad(out) : 0;
  const Slice so(V, out_pad, part, a.parts);                   // the part of the gradient that this block writes
  const bool leader = part == 0 && tid == 0;

  if (weight != 0.f) {
    const Slice sl(V, row_pad(row), part, a.parts);
    for (int i = tid; i < (sl.last - sl.first + 3) / 4; i += NT) listed_words[i] = 0;
    if (tid == 0) en.bad = en.twice = 0;
    __syncthreads();
    for (int k = tid; k < K; k += NT) {
      const int id = a.ids[r * K + k];
      const float y = a.y[r * K + k];
      const bool used = id >= 0 && id < V;
      if (id < -1 || id >= V || (id >= 0 && !(y < kInf))) en.bad = 1;
      en.id[k] = used ? id : -1;
      en.y[k] = used ? y : -kInf;
      en.x[k] = used ? Elem<T>::get(row + id) : -kInf;
      if (used && sl.holds(id)) {
        const int p = id + sl.pad - 8 * sl.first;
        atomicOr(&listed_words[p >> 5], 1u << (p & 31));
      }
    }
    __syncthreads();
    for (int k = tid; k < K; k += NT) {
      bool first = true;
      for (int j = 0; j < k; ++j) first = first && en.id[j] != en.id[k];
      en.first[k] = first && en.id[k] >= 0;
      if (!first && en.id[k] >= 0) en.twice = 1;
    }

    // the sums of what is not listed
    constexpr int N = sizeof(T) == 2 ? 4 : 2;
    Stream<T> st(c);
    const T* base = row - sl.pad;
    auto without_listed = [&](Unit<T>& q, int u) {
      const unsigned bits = listed[u - sl.first];
      if (bits) {
        float v[8];
        q.values(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = bits >> j & 1u ? -kInf : v[j];
        q.set(v);
      }
    };
    int u = sl.full0 + tid;
    for (; u + (N - 1) * NT < sl.full1; u += N * NT) {
      Unit<T> q[N];
#pragma unroll
      for (int i = 0; i < N; ++i) load_unit(base + 8 * (int64_t)(u + i * NT), q[i]);
#pragma unroll
      for (int i = 0; i < N; ++i) without_listed(q[i], u + i * NT);
      st.add(q);
    }
    for (; u < sl.full1; u += NT) {
      Unit<T> q[1];
      load_unit(base + 8 * (int64_t)u, q[0]);
      without_listed(q[0], u);
      st.add(q);
    }
    if (tid < 2 && sl.ragged(tid) >= 0) {
      Unit<T> q[1];
      load_ragged(row, V, sl.pad, sl.ragged(tid), q[0]);
      without_listed(q[0], sl.ragged(tid));
      st.add(q);
    }
    join_block<NT>(st.finish(), c, per_warp, &mine);
    __syncthreads();
    if (a.parts > 1) cluster_sync();

    // The list's side: a few numbers, in 64 bits, since the loss is a small difference of its terms.
    if (tid < 32) {
      const State rest = a.parts > 1 ? join_cluster(&mine, a.parts, c) : mine;
      const double s = a.s;
      float m = rest.m, ytop = -kInf;
      for (int k = tid; k < K; k += 32) {
        m = max_nan(m, en.x[k]);
        ytop = fmaxf(ytop, en.y[k]);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
        ytop = fmaxf(ytop, __shfl_xor_sync(0xffffffffu, ytop, o));
      }
      const bool some = ytop > -kInf, alive = m != -kInf, others = rest.m > -kInf;   // NaN: alive
      double z = 0.0, qs = 0.0;
      if (alive) {
        for (int k = tid; k < K; k += 32) {
          if (en.first[k]) z += exp(((double)en.x[k] - m) * s);
          if (some) qs += exp((double)en.y[k] - (a.tail ? 0.0 : (double)ytop));
        }
      }
      z = warp_sum(z) + (others ? exp(((double)rest.m - m) * s) * (1.0 + (double)rest.R) : 0.0);
      qs = warp_sum(qs);
      const double ln_z = log(z), ln_q = a.tail || !some ? 0.0 : (double)ytop + log(qs);
      const double q_rest = a.tail && others ? fmax(0.0, 1.0 - qs) : 0.0;
      const double ln_p_rest = ((double)rest.m - m) * s + log1p((double)rest.R) - ln_z;
      double loss = 0.0;
      for (int k = tid; k < K; k += 32) {
        const double ln = (double)en.y[k] - ln_q, q = exp(ln);
        if (q != 0.0) loss += q * (ln - (((double)en.x[k] - m) * s - ln_z));
      }
      loss = warp_sum(loss);
      if (q_rest > 0.0) loss += q_rest * (log(q_rest) - ln_p_rest);
      if (tid == 0) {
        const bool in = some && alive;
        const float poison = en.bad ? nan_value() : 0.f;
        const double c_rest = others ? exp(ln_p_rest) - q_rest : 0.0;
        RowGrad& g = en.g;
        g.kind = en.bad || in;
        g.m_rest = others ? rest.m : 0.f;
        g.coef = (others ? (float)((double)a.s * weight * c_rest / (1.0 + (double)rest.R)) : 0.f) + poison;
        g.m = m;
        g.ln_z = ln_z + poison;
        g.ln_q = ln_q;
        g.weight = (double)a.s * weight;
        if (leader) {
          if (a.loss) a.loss[r] = (in ? (float)loss : 0.f) + poison;
          if (a.stats) {
            float* o = a.stats + 8 * r;
            o[0] = m; o[1] = (float)ln_z; o[2] = rest.m; o[3] = others ? log1pf(rest.R) : -kInf;
            o[4] = (float)c_rest; o[5] = (float)ln_q; o[6] = (in ? 1.f : 0.f) + poison; o[7] = 0.f;
          }
        }
      }
    }
    __syncthreads();
  } else if (leader) {
    if (a.loss) a.loss[r] = 0.f;
    if (a.stats)
      for (int i = 0; i < 8; ++i) a.stats[8 * r + i] = 0.f;
  }

  if (GRAD) {
    const bool zero = weight == 0.f || en.g.kind == 0;
    const bool alike = row_pad(row) == out_pad;
    float m_rest = 0.f, coef = 0.f;
    if (!zero) { m_rest = en.g.m_rest; coef = en.g.coef; }
    constexpr int N = sizeof(T) == 2 ? 4 : 2;
    const T* in_base = row - out_pad;
    T* out_base = out - out_pad;
    if (alike) {
      int u = so.full0 + tid;
      for (; u < so.full1; u += N * NT) {
        Unit<T> q[N];
        if (!zero) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (u + i * NT < so.full1) load_unit(in_base + 8 * (int64_t)(u + i * NT), q[i]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (u + i * NT < so.full1) {
            if (zero) fill_unit(q[i], 0.f);
            else rest_grad_unit(q[i], m_rest, c, coef);
            store_unit(out_base + 8 * (int64_t)(u + i * NT), q[i]);
          }
      }
    } else {
      for (int u = so.full0 + tid; u < so.full1; u += NT) {
        Unit<T> q;
        if (zero) {
          fill_unit(q, 0.f);
        } else {
          load_ragged(row, V, out_pad, u, q);
          rest_grad_unit(q, m_rest, c, coef);
        }
        store_unit(out_base + 8 * (int64_t)u, q);
      }
    }
    if (tid < 2 && so.ragged(tid) >= 0) {
      Unit<T> q;
      if (zero) {
        fill_unit(q, 0.f);
      } else {
        load_ragged(row, V, out_pad, so.ragged(tid), q);
        rest_grad_unit(q, m_rest, c, coef);
      }
      store_ragged(out, V, out_pad, so.ragged(tid), q);
    }
    if (!zero) {
      __syncthreads();                        // the list's elements go over what was just written there
      for (int k = tid; k < K; k += NT)
        if (en.first[k] && so.holds(en.id[k]))
          Elem<T>::put(out + en.id[k], entry_gradient(en.g, a.s, en.id, en.y, K, k, en.x[k], en.twice));
    }
  }
  if (a.parts > 1) cluster_sync();            // no block leaves while another reads its shared memory
}

// Rows of up to 256 elements: LPR lanes a row, eight elements a lane, the list laid out over the row's elements in shared
// memory.  BACKWARD takes what rows share from row_stats instead of computing it.
template <typename T, int LPR, bool GRAD, bool BACKWARD>
__global__ void __launch_bounds__(256) distill_small_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int G = 256 / LPR, W = 8 * LPR;       // rows a block; entries and elements a row at most
  __shared__ int s_id[G][W], s_owner[G][W];
  __shared__ float s_y[G][W];
  __shared__ double s_q[G][W];                    // by element: the list's probability
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
  for (int v = lane; v < W; v += LPR) { s_owner[gi][v] = -1; s_q[gi][v] = 0.0; }
  __syncwarp();
  bool bad = false;
  float ytop = -kInf;
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
  for (int k = lane; k < K; k += LPR) twice = twice || (s_id[gi][k] >= 0 && s_owner[gi][s_id[gi][k]] != k);
  twice = group_any(twice);
  double ln_q = 0.0, qs = 0.0, entropy = 0.0;     // entropy: sum of q ln q over the list
  if (BACKWARD) {
    ln_q = a.stats_in[8 * rr + 5];
  } else if (some) {
    const double shift = a.tail ? 0.0 : (double)ytop;
    for (int k = lane; k < K; k += LPR) qs += exp((double)s_y[gi][k] - shift);
  }
  if (!BACKWARD) {
    qs = group_sum(qs);
    ln_q = a.tail || !some ? 0.0 : (double)ytop + log(qs);
  }
  for (int k = lane; k < K; k += LPR) {
    const int id = s_id[gi][k];
    if (id < 0) continue;
    double p = exp((double)s_y[gi][k] - ln_q);
    if (p != 0.0) entropy += p * ((double)s_y[gi][k] - ln_q);
    if (twice) {
      for (int j = 0; j < k; ++j)
        if (s_id[gi][j] == id) p = -1.0;          // the first entry of the id has summed it
      if (p >= 0.0)
        for (int j = k + 1; j < K; ++j)
          if (s_id[gi][j] == id) p += exp((double)s_y[gi][j] - ln_q);
    }
    if (p >= 0.0) s_q[gi][id] = p;
  }
  __syncwarp();
  float v[8];
  q.values(v);
  unsigned listed = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) listed |= s_owner[gi][8 * lane + j] >= 0 ? 1u << j : 0u;

  float m, m_rest, coef, flag;
  double ln_z;
  if (BACKWARD) {
    const float* o = a.stats_in + 8 * rr;
    m = o[0]; ln_z = o[1]; flag = o[6];
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
    Stream<T> st(c);
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
        if (listed >> j & 1u) z += exp(((double)v[j] - m) * s);
    }
    z = group_sum(z) + (others ? exp(((double)rest.m - m) * s) * (1.0 + (double)rest.R) : 0.0);
    ln_z = log(z);
    const double q_rest = a.tail && others ? fmax(0.0, 1.0 - qs) : 0.0;
    const double ln_p_rest = ((double)rest.m - m) * s + log1p((double)rest.R) - ln_z;
    double loss = entropy;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (listed >> j & 1u) {
        const double p = s_q[gi][8 * lane + j];
        if (p != 0.0) loss -= p * (((double)v[j] - m) * s - ln_z);
      }
    loss = group_sum(loss);
    if (q_rest > 0.0) loss += q_rest * (log(q_rest) - ln_p_rest);
    const double c_rest = others ? exp(ln_p_rest) - q_rest : 0.0;
    const bool in = some && alive;
    flag = bad ? nan_value() : in ? 1.f : 0.f;
    m_rest = others ? rest.m : 0.f;
    coef = others ? (float)(s * weight * c_rest / (1.0 + (double)rest.R)) : 0.f;
    if (there && lane == 0) {
      const bool counts = weight != 0.f;
      if (a.loss) a.loss[r] = !counts ? 0.f : bad ? nan_value() : in ? (float)loss : 0.f;
      if (a.stats) {
        float* o = a.stats + 8 * r;
        o[0] = m; o[1] = (float)ln_z; o[2] = rest.m; o[3] = others ? log1pf(rest.R) : -kInf;
        o[4] = (float)c_rest; o[5] = (float)ln_q; o[6] = counts ? flag : 0.f; o[7] = 0.f;
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
        if (listed >> j & 1u) d[j] = (float)(s * weight * (exp(((double)v[j] - m) * s - ln_z) - s_q[gi][8 * lane + j]));
        else d[j] = coef * ex2((v[j] - m_rest) * c);
        if (!(flag == flag)) d[j] = flag;
      }
    }
    q.set(d);
    if (row_pad(out) == 0 && 8 * lane + 8 <= V) store_unit(out + 8 * lane, q);
    else store_ragged(out, V, 0, lane, q);
  }
}

constexpr int kBackThreads = 256, kBackUnits = 4;

// `parts` blocks a row, each thread four units and at most one entry of the list.
template <typename T>
__global__ void __launch_bounds__(kBackThreads) distill_backward_kernel(const __grid_constant__ DistillArgs a) {
  static_assert(kMaxList <= kBackThreads, "one entry a thread");
  __shared__ int s_id[kMaxList];
  __shared__ float s_y[kMaxList];
  const int tid = threadIdx.x, V = a.V, K = a.K;
  const int64_t r = blockIdx.x / a.parts;
  const int lo = (int)(blockIdx.x - (unsigned)r * (unsigned)a.parts) * kBackThreads * kBackUnits;     // first unit
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* out = static_cast<T*>(a.d_logits) + r * a.d_stride;
  const int pad = row_pad(out), units = (V + pad + 7) >> 3, full0 = pad > 0 ? 1 : 0, full1 = (V + pad) >> 3;
  const bool alike = row_pad(row) == pad;
  const float* o = a.stats_in + 8 * r;
  const float weight = a.weight[r], flag = o[6], c = a.s * kLog2e;
  const bool zero = weight == 0.f || flag == 0.f;
  Unit<T> q[kBackUnits];
  float x = 0.f;
  if (!zero) {
#pragma unroll
    for (int i = 0; i < kBackUnits; ++i) {
      const int u = lo + i * kBackThreads + tid;
      if (u >= units) continue;
      if (alike && u >= full0 && u < full1) load_unit(row - pad + 8 * (int64_t)u, q[i]);
      else load_ragged(row, V, pad, u, q[i]);
    }
    if (tid < K) {
      const int id = a.ids[r * K + tid];
      s_id[tid] = id >= 0 && id < V ? id : -1;
      s_y[tid] = a.y[r * K + tid];
      if (s_id[tid] >= 0) x = Elem<T>::get(row + id);         // before anything of the row may be written over
    }
  }
  const bool others = o[2] > -kInf;
  const float m_rest = others ? o[2] : 0.f;
  const float coef = flag == flag ? (others ? a.s * weight * o[4] * ex2(-o[3] * kLog2e) : 0.f) : flag;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBackUnits; ++i) {
    const int u = lo + i * kBackThreads + tid;
    if (u >= units) continue;
    if (zero) fill_unit(q[i], 0.f);
    else rest_grad_unit(q[i], m_rest, c, coef);
    if (u >= full0 && u < full1) store_unit(out - pad + 8 * (int64_t)u, q[i]);
    else store_ragged(out, V, pad, u, q[i]);
  }
  if (zero || !(flag == flag)) return;
  const int id = tid < K ? s_id[tid] : -1, u = (id + pad) >> 3;
  bool mine = id >= 0 && u >= lo && u < lo + kBackThreads * kBackUnits, twice = false;
  if (mine)
    for (int j = 0; j < K; ++j) {
      if (j != tid && s_id[j] == id) {
        twice = true;
        if (j < tid) mine = false;
      }
    }
  __syncthreads();
  if (mine) {
    RowGrad g;
    g.m = o[0]; g.ln_z = o[1]; g.ln_q = o[5]; g.weight = (double)a.s * weight;
    Elem<T>::put(out + id, entry_gradient(g, a.s, s_id, s_y, K, tid, x, twice));
  }
}

template <typename T>
cudaError_t launch_small(const DistillArgs& a, bool backward, cudaStream_t st) {
  const bool narrow = a.V <= 64;
  const unsigned blocks = narrow ? ((unsigned)a.n_rows + 31) / 32 : ((unsigned)a.n_rows + 7) / 8;
  if (backward) {
    if (narrow) distill_small_kernel<T, 8, true, true><<<blocks, 256, 0, st>>>(a);
    else distill_small_kernel<T, 32, true, true><<<blocks, 256, 0, st>>>(a);
  } else if (a.d_logits) {
    if (narrow) distill_small_kernel<T, 8, true, false><<<blocks, 256, 0, st>>>(a);
    else distill_small_kernel<T, 32, true, false><<<blocks, 256, 0, st>>>(a);
  } else {
    if (narrow) distill_small_kernel<T, 8, false, false><<<blocks, 256, 0, st>>>(a);
    else distill_small_kernel<T, 32, false, false><<<blocks, 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}

template <typename T, int NT, bool GRAD>
cudaError_t launch_distill_rows(const DistillArgs& a, cudaStream_t st) {
  static std::atomic<bool> allowed[kMaxDevices];
  const size_t smem = (((size_t)(a.V + 14) / 8 + a.parts - 1) / a.parts + 3) / 4 * 4;
  if (smem > 40 * 1024) {
    const cudaError_t e = allow_dynamic_smem(distill_rows_kernel<T, NT, GRAD>, REMOE_ROWS_MAX_VOCAB / 8 + 64, allowed);
    if (e != cudaSuccess) return e;
  }
  return launch_rows(distill_rows_kernel<T, NT, GRAD>, a.n_rows, a.parts, NT, smem, st, a);
}

template <typename T>
cudaError_t launch_distill(DistillArgs a, bool backward, cudaStream_t st) {
  if (a.V <= kSmallVocab) return launch_small<T>(a, backward, st);
  if (backward) {
    const int units = (a.V + 15) >> 3;
    a.parts = (units + kBackThreads * kBackUnits - 1) / (kBackThreads * kBackUnits);
    const int64_t blocks = (int64_t)a.n_rows * a.parts;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    distill_backward_kernel<T><<<(unsigned)blocks, kBackThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  a.parts = parts_of_row(a.n_rows, a.V, 512);
  if (a.V >= 8192) return a.d_logits ? launch_distill_rows<T, 512, true>(a, st) : launch_distill_rows<T, 512, false>(a, st);
  return a.d_logits ? launch_distill_rows<T, 128, true>(a, st) : launch_distill_rows<T, 128, false>(a, st);
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
  DistillArgs a{logits_dev, d_logits_dev, row_stride, d_row_stride, vocab, n_rows, 1, n_top, tail, inv_temperature,
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
  DistillArgs a{logits_dev, d_logits_dev, row_stride, d_row_stride, vocab, n_rows, 1, n_top, 0, inv_temperature,
                teacher_ids_dev, teacher_logprobs_dev, grad_loss_dev, nullptr, nullptr, row_stats_dev};
  const int rc = check_distill(a, dtype);
  if (rc != REMOE_OK) return rc;
  if (!row_stats_dev || !grad_loss_dev || !d_logits_dev) return REMOE_E_ARG;
  return run_distill(a, dtype, true, cuda_stream);
}
