// remoe_token_logprobs / remoe_token_logprobs_backward: log probabilities of given tokens, entropy and top
// alternatives of rows of logits, and the gradient.
//
//   p = softmax(s x), lp = s (x_token - m) - ln Z, H = ln Z - (1/Z) sum s (x - m) e^{s (x - m)}
//   dx = s [ g_lp (1[v = token] - p) - g_H p (ln p + H) ]
#include "logit_rows.cuh"
#include "logit_rows_host.h"

namespace remoe {
namespace rows {

constexpr int kCandidates = 1536;       // elements above the threshold that one block can hold
constexpr int kTies = 512;              // elements equal to it
constexpr int kSmallVocab = 256;        // up to here a row is held by a group of lanes, one unit per lane

struct LogprobArgs {
  const void* logits;
  int64_t stride;
  int V, n_rows, parts, slice_bytes, top_k;
  float s;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob, *stats;
  int32_t* top_ids;
};

// Shared memory of the selection.  Keys hold (value, then lowest index first): all distinct.
template <int NT>
struct TopShared {
  static_assert(kCandidates + kTies >= 8 * REMOE_ROWS_MAX_TOP, "the lists of eight blocks");
  unsigned long long above[kCandidates + kTies];      // the ties' list lies behind it; both hold the lists of a join later
  unsigned long long sorted[REMOE_ROWS_MAX_TOP];
  int columns[NT];
  int n_columns, n_above, n_ties;
  int warp_count[NT / 32];
};

__device__ __forceinline__ unsigned long long full_key(uint32_t k, int id) { return ((unsigned long long)k << 32) | (0xffffffffu - (uint32_t)id); }

// A block's slice in shared memory, as the selection looks at it: calls f(key, id) for the elements of unit i.
template <typename T, typename F>
__device__ __forceinline__ void each_element(const unsigned char* units, const Slice& sl, int V, int i, F f) {
  Unit<T> q;
  load_shared_unit(units, i, q);
  float v[8];
  q.values(v);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int id = 8 * (sl.first + i) + j - sl.pad;
    if (id >= 0 && id < V) f(order_key(v[j]), id);
  }
}

// Elements of the slice at or above `t`.
template <typename T, int NT>
__device__ int count_keys(const unsigned char* units, const Slice& sl, int V, uint32_t t, int* warp_count) {
  int n = 0;
  for (int i = threadIdx.x; i < sl.last - sl.first; i += NT) each_element<T>(units, sl, V, i, [&](uint32_t k, int) { n += k >= t; });
  n = __reduce_add_sync(0xffffffffu, n);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_count[threadIdx.x >> 5] = n;
  __syncthreads();
  int all = 0;
  for (int w = 0; w < NT / 32; ++w) all += warp_count[w];
  return all;
}

// The `want` largest elements of the slice, sorted, to sh.sorted.
//
// A thread has kept the largest of its elements (units tid, tid + NT, ...).  The want-th largest of these NT numbers is a
// lower bound t for the want-th largest element, and only threads whose largest reaches t hold such elements: their
// units (a few per cent of the slice) are looked at again, and what is above t is sorted by counting for each
// the keys above it.  t may be rounded down to fewer bits, which adds candidates and never loses one.
// Elements equal to t matter only where too few are above it.  Where few threads hold t they are listed with the others;
// in masked rows nearly all elements are equal, and those of the lowest indices are taken in one ordered scan that
// stops as soon as there are enough.  Rows whose large elements sit in few threads overflow the list: then the
// want-th largest value is found by its bits, with a count over the slice for each.
template <typename T, int NT>
__device__ void select_top(const unsigned char* units, const Slice& sl, int V, float mine, int want, TopShared<NT>& sh) {
  const int tid = threadIdx.x, n_units = sl.last - sl.first;
  unsigned long long* const ties = sh.above + kCandidates;
  uint32_t t = 0;
  const uint32_t key = mine == mine && tid < n_units ? order_key(mine) : 0;   // no unit: below all values
  if (tid == 0) sh.n_columns = sh.n_above = sh.n_ties = 0;
  constexpr int kLow = Elem<T>::kUnusedBits;          // the key's bits that say nothing for a 16-bit type
  int holders = NT;                                   // threads whose largest is at least t
  for (int b = 31; b >= kLow; --b) {
    const uint32_t cand = t | (1u << b);
    const int n = __syncthreads_count(key >= cand);
    if (n >= want) {
      t = cand;
      holders = n;
      if (n <= want + want / 4 + 4) break;
    }
  }
  if (!(t & 0x80000000u)) t |= (1u << kLow) - 1u;      // they are ones in a negative value's key
  const bool list_ties = holders <= 2 * want + 32;
  __syncthreads();
  if (key > t || (list_ties && key == t)) sh.columns[atomicAdd(&sh.n_columns, 1)] = tid;
  __syncthreads();
  const int nc = sh.n_columns, rounds = (n_units + NT - 1) / NT;
  auto push = [&](uint32_t k, int id) {
    if (k > t) {
      const int i = atomicAdd(&sh.n_above, 1);
      if (i < kCandidates) sh.above[i] = full_key(k, id);
    } else if (list_ties && k == t) {
      const int i = atomicAdd(&sh.n_ties, 1);
      if (i < kTies) ties[i] = full_key(k, id);
    }
  };
  for (int w = tid; w < nc * rounds; w += NT) {
    const int i = (w / nc) * NT + sh.columns[w % nc];
    if (i < n_units) each_element<T>(units, sl, V, i, push);
  }
  __syncthreads();
  int na = sh.n_above, nt = list_ties ? sh.n_ties : kTies + 1;
  if (na > kCandidates) {
    __syncthreads();
    uint32_t v = 0;
    for (int b = 31; b >= 0; --b)
      if (count_keys<T, NT>(units, sl, V, v | (1u << b), sh.warp_count) >= want) v |= 1u << b;
    t = v;
    __syncthreads();
    if (tid == 0) sh.n_above = 0;
    __syncthreads();
    for (int i = tid; i < n_units; i += NT)
      each_element<T>(units, sl, V, i, [&](uint32_t k, int id) {
        if (k > t) sh.above[atomicAdd(&sh.n_above, 1)] = full_key(k, id);      // fewer than `want`
      });
    __syncthreads();
    na = sh.n_above;
    nt = kTies + 1;
  }
  int used_ties = 0;
  if (na < want) {
    used_ties = nt;
    if (nt > kTies) {
      const int need = want - na;
      int have = 0;
      for (int base = 0; base < n_units && have < need; base += NT) {
        unsigned hits = 0;
        if (base + tid < n_units)
          each_element<T>(units, sl, V, base + tid, [&](uint32_t k, int id) { hits |= k == t ? 1u << ((id + sl.pad) & 7) : 0u; });
        int upto = __popc(hits);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, upto, o);
          if ((tid & 31) >= o) upto += up;
        }
        __syncthreads();
        if ((tid & 31) == 31) sh.warp_count[tid >> 5] = upto;
        __syncthreads();
        int at = have + upto - __popc(hits), all = 0;
        for (int w = 0; w < NT / 32; ++w) {
          if (w < (tid >> 5)) at += sh.warp_count[w];
          all += sh.warp_count[w];
        }
        for (; hits && at < need; hits &= hits - 1, ++at)
          ties[at] = full_key(t, 8 * (sl.first + base + tid) + __ffs(hits) - 1 - sl.pad);
        have += all;
      }
      used_ties = min(need, have);
      __syncthreads();
    }
  }
  // four neighbouring lanes count for one key
  const int n = na + used_ties;
  for (int b = 0; b < 4 * n; b += NT) {
    const int i = (b + tid) >> 2;
    const unsigned long long k = i < na ? sh.above[i] : i < n ? ties[i - na] : 0ull;
    int rank = 0;
    for (int j = tid & 3; j < na; j += 4) rank += sh.above[j] > k;
    for (int j = tid & 3; j < used_ties; j += 4) rank += ties[j] > k;
    rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    rank += __shfl_xor_sync(0xffffffffu, rank, 2);
    if (i < n && (tid & 3) == 0 && rank < want) sh.sorted[rank] = k;
  }
  __syncthreads();
}

// One row per cluster of `parts` blocks, each block's slice of it in shared memory.
template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT) logprob_rows_kernel(const __grid_constant__ LogprobArgs a) {
  __shared__ State per_warp[NT / 32];
  __shared__ State mine;
  __shared__ uint64_t bar;
  extern __shared__ __align__(16) unsigned char units[];       // the slice; the selection's lists behind it
  const int part = a.parts > 1 ? (int)cluster_rank() : 0;
  const int64_t r = blockIdx.x / a.parts;
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  const int V = a.V, tid = threadIdx.x;
  const Slice sl(V, row_pad(row), part, a.parts);
  const float c = a.s * kLog2e;
  const bool leader = part == 0 && tid == 0;
  start_slice(row, V, sl, units, &bar);

  int token = -1;
  float x_token = 0.f;
  if (leader && a.tokens) {
    token = a.tokens[r];
    if (token >= 0 && token < V) x_token = Elem<T>::get(row + token);
  }
  __syncthreads();
  const bool arrived = wait_slice(&bar);

  constexpr int N = sizeof(T) == 2 ? 4 : 2;
  const int n_units = sl.last - sl.first;
  Stream<T, true, true> st(c);
  int u = tid;
  for (; u + (N - 1) * NT < n_units; u += N * NT) {
    Unit<T> q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) load_shared_unit(units, u + i * NT, q[i]);
    st.add(q);
  }
  for (; u < n_units; u += NT) {
    Unit<T> q[1];
    load_shared_unit(units, u, q[0]);
    st.add(q);
  }
  join_block<NT>(arrived ? st.finish() : State{0.f, nan_value(), nan_value()}, c, per_warp, &mine);
  TopShared<NT>& sh = *reinterpret_cast<TopShared<NT>*>(units + a.slice_bytes);
  if (TOP) {
    const int want = min(a.top_k, sl.length(V));
    if (want > 0) select_top<T, NT>(units, sl, V, st.top(), want, sh);
  }
  __syncthreads();
  State all = mine;
  if (a.parts > 1) {
    cluster_sync();
    if (part == 0) all = join_cluster(&mine, a.parts, c);
  }
  const float ln_z = all.m == -kInf ? -kInf : log1pf(all.R);
  if (leader) {
    const bool none = all.m == -kInf;
    const float h = none ? 0.f : ln_z - kLn2 * all.U / (1.f + all.R);
    float lp = 0.f;
    if (token >= 0 && token < V) lp = none ? -kInf : (x_token - all.m) * a.s - ln_z;
    else if (token != -1) lp = nan_value();
    if (a.logprob) a.logprob[r] = lp;
    if (a.entropy) a.entropy[r] = h;
    if (a.stats) {
      float* o = a.stats + 4 * r;
      o[0] = all.m; o[1] = ln_z; o[2] = h; o[3] = lp;
    }
  }
  if (TOP && part == 0) {
    int32_t* ids = a.top_ids + r * a.top_k;
    float* lps = a.top_logprob + r * a.top_k;
    auto write = [&](int rank, unsigned long long k) {
      const float x = key_value((uint32_t)(k >> 32));
      ids[rank] = (int32_t)(0xffffffffu - (uint32_t)k);
      lps[rank] = all.m == -kInf ? -kInf : (x - all.m) * a.s - ln_z;
    };
    if (!(all.R == all.R)) {
      for (int i = tid; i < a.top_k; i += NT) {
        ids[i] = -1;
        lps[i] = nan_value();
      }
    } else if (a.parts == 1) {
      for (int i = tid; i < a.top_k; i += NT) write(i, sh.sorted[i]);
    } else {
      // the blocks' sorted lists, one behind the other in the candidates' place; a key's rank is its place in its
      // own list plus, for each other list, the number of keys above it there
      unsigned long long* lists = sh.above;
      const int K = a.top_k;
      for (int i = tid; i < a.parts * K; i += NT) {
        const int p = i / K, j = i - p * K;
        lists[i] = j < Slice(V, sl.pad, p, a.parts).length(V) ? load_remote64(remote_shared(&sh.sorted[j], p)) : 0ull;
      }
      __syncthreads();
      for (int i = tid; i < a.parts * K; i += NT) {
        const unsigned long long k = lists[i];
        if (k == 0ull) continue;
        const int p = i / K;
        int rank = i - p * K;
        for (int o = 0; o < a.parts && rank < K; ++o) {
          if (o == p) continue;
          int lo = 0, hi = K;
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (lists[o * K + mid] > k) lo = mid + 1;
            else hi = mid;
          }
          rank += lo;
        }
        if (rank < K) write(rank, k);
      }
    }
  }
  if (a.parts > 1) cluster_sync();       // no block leaves while another reads its shared memory
}

// Rows of up to 256 elements: LPR lanes a row, eight elements a lane, all in registers.
template <typename T, int LPR>
__global__ void __launch_bounds__(256) logprob_small_kernel(const __grid_constant__ LogprobArgs a) {
  const int lane = threadIdx.x & (LPR - 1);
  const int64_t r = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const bool there = r < a.n_rows;
  const T* row = static_cast<const T*>(a.logits) + (there ? r : 0) * a.stride;
  const float c = a.s * kLog2e;
  Unit<T> q[1];
  if (row_pad(row) == 0 && 8 * lane + 8 <= a.V) load_unit(row + 8 * lane, q[0]);
  else load_ragged(row, a.V, 0, lane, q[0]);
  float v[8];
  q[0].values(v);
  Stream<T, true, true> st(c);
  st.add(q);
  State all = st.finish();
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) all = merge(all, shuffle_down(all, o, LPR), c);
  all = State{__shfl_sync(0xffffffffu, all.m, 0, LPR), __shfl_sync(0xffffffffu, all.R, 0, LPR), __shfl_sync(0xffffffffu, all.U, 0, LPR)};
  const bool none = all.m == -kInf, bad = !(all.R == all.R);
  const float ln_z = none ? -kInf : log1pf(all.R);
  if (there && lane == 0) {
    const int token = a.tokens ? a.tokens[r] : -1;
    const float h = none ? 0.f : ln_z - kLn2 * all.U / (1.f + all.R);
    float lp = 0.f;
    if (token >= 0 && token < a.V) lp = none ? -kInf : (Elem<T>::get(row + token) - all.m) * a.s - ln_z;
    else if (token != -1) lp = nan_value();
    if (a.logprob) a.logprob[r] = lp;
    if (a.entropy) a.entropy[r] = h;
    if (a.stats) {
      float* o = a.stats + 4 * r;
      o[0] = all.m; o[1] = ln_z; o[2] = h; o[3] = lp;
    }
  }
  // the alternatives one by one: the largest key of each lane's elements that are not taken yet, then of the group
  uint32_t key[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) key[j] = order_key(v[j]);
  unsigned left = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) left |= 8 * lane + j < a.V ? 1u << j : 0u;
  for (int k = 0; k < a.top_k; ++k) {
    uint32_t best = 0;
    int at = -1;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if ((left >> j & 1u) && (at < 0 || key[j] > best)) { best = key[j]; at = j; }
    const unsigned long long own = at < 0 ? 0ull : full_key(best, 8 * lane + at);
    unsigned long long top = own;
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, top, o, LPR);
      top = other > top ? other : top;
    }
    if (at >= 0 && own == top) left &= ~(1u << at);
    if (there && lane == 0) {
      const float x = key_value((uint32_t)(top >> 32));
      a.top_ids[r * a.top_k + k] = bad ? -1 : (int32_t)(0xffffffffu - (uint32_t)top);
      a.top_logprob[r * a.top_k + k] = bad ? nan_value() : none ? -kInf : (x - all.m) * a.s - ln_z;
    }
  }
}

struct LogprobGradArgs {
  const void* logits;
  void* d_logits;
  int64_t stride, d_stride;
  int V, n_rows, tiles;
  float s;
  const int32_t* tokens;
  const float *stats, *g_logprob, *g_entropy;
};

// Gradient of one unit: dx = e (A + B d) with d = (x - m) log2(e) s, e = 2^d, A = -s (g_lp + g_H (H - ln Z)) / Z and
// B = -s g_H ln 2 / Z.
template <typename T>
__device__ __forceinline__ void logprob_grad_unit(Unit<T>& q, float m, float c, float A, float B) {
  const f2 nm = pack2(-m, -m), cc = pack2(c, c), A2 = pack2(A, A), B2 = pack2(B, B);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f2 d = mul2(add2(Elem<T>::widen(q.w[j]), nm), cc);
    float d0, d1;
    unpack2(d, d0, d1);
    d0 = max_nan(d0, -200.f);                 // 2^-200 is 0 in float32; -inf would give 0 * inf
    d1 = max_nan(d1, -200.f);
    q.w[j] = Elem<T>::narrow(mul2(pack2(ex2(d0), ex2(d1)), fma2(B2, pack2(d0, d1), A2)));
  }
}

constexpr int kGradThreads = 256, kGradUnits = 4;

// Element-wise: what a row's gradient shares is in its row_stats.  Long rows: `tiles` blocks a row, each thread four
// units.  Short rows (SMALL): one unit a thread over all rows' units.
template <typename T, bool SMALL>
__global__ void __launch_bounds__(kGradThreads) logprob_grad_kernel(const __grid_constant__ LogprobGradArgs a) {
  constexpr int N = SMALL ? 1 : kGradUnits;
  int64_t r;
  int u0;
  if (SMALL) {
    const int64_t i = (int64_t)blockIdx.x * kGradThreads + threadIdx.x;
    r = i / a.tiles;                          // tiles: units a row
    u0 = (int)(i - r * a.tiles);
    if (r >= a.n_rows) return;
  } else {
    r = blockIdx.x / a.tiles;
    u0 = (int)(blockIdx.x - (unsigned)r * (unsigned)a.tiles) * kGradThreads * N + threadIdx.x;
  }
  const T* row = static_cast<const T*>(a.logits) + r * a.stride;
  T* out = static_cast<T*>(a.d_logits) + r * a.d_stride;
  const int V = a.V, pad = row_pad(out);      // stores are whole units; loads are where both rows lie alike
  const bool alike = row_pad(row) == pad;
  const int full0 = pad > 0 ? 1 : 0, full1 = (V + pad) >> 3, units = (V + pad + 7) >> 3;

  const float m = a.stats[4 * r], ln_z = a.stats[4 * r + 1], h = a.stats[4 * r + 2];
  const int token = a.tokens ? a.tokens[r] : -1;
  const float g = a.g_logprob && token != -1 ? a.g_logprob[r] : 0.f;
  const float gh = a.g_entropy ? a.g_entropy[r] : 0.f;
  const bool zero = (g == 0.f && gh == 0.f) || m == -kInf;
  const bool bad = !zero && (token < -1 || token >= V);
  const float inv_z = ex2(-ln_z * kLog2e), c = a.s * kLog2e;
  const float A = -a.s * (g + gh * (h - ln_z)) * inv_z, B = -a.s * gh * kLn2 * inv_z;
  Unit<T> q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = u0 + i * kGradThreads;
    if (u >= units || zero) continue;
    if (alike && u >= full0 && u < full1) load_unit(row - pad + 8 * (int64_t)u, q[i]);
    else load_ragged(row, V, pad, u, q[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = u0 + i * kGradThreads;
    if (u >= units) continue;
    if (zero || bad) {
      const float x = bad ? nan_value() : 0.f;
      const float v[8] = {x, x, x, x, x, x, x, x};
      q[i].set(v);
    } else {
      float at_token = 0.f;
      const bool here = token >= 0 && (token + pad) >> 3 == u;
      if (here) {
        // 1 - p without cancellation where p is nearly one
        float v[8];
        q[i].values(v);
        float x = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) x = 8 * u + j - pad == token ? v[j] : x;
        const float lp = max_nan((x - m) * a.s - ln_z, -200.f);
        at_token = a.s * (-g * expm1f(lp) - gh * ex2(lp * kLog2e) * (lp + h));
      }
      logprob_grad_unit(q[i], m, c, A, B);
      if (here) {
        float v[8];
        q[i].values(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 8 * u + j - pad == token ? at_token : v[j];
        q[i].set(v);
      }
    }
    if (u >= full0 && u < full1) store_unit(out - pad + 8 * (int64_t)u, q[i]);
    else store_ragged(out, V, pad, u, q[i]);
  }
}

template <typename T>
cudaError_t launch_logprobs(LogprobArgs a, cudaStream_t st) {
  const bool top = a.top_k > 0;
  if (a.V <= kSmallVocab) {
    if (a.V <= 64) logprob_small_kernel<T, 8><<<((unsigned)a.n_rows + 31) / 32, 256, 0, st>>>(a);
    else logprob_small_kernel<T, 32><<<((unsigned)a.n_rows + 7) / 8, 256, 0, st>>>(a);
    return cudaGetLastError();
  }
  const bool wide = a.V >= 8192 || a.top_k > 64;
  a.parts = parts_of_row(a.n_rows, a.V, sizeof(T));
  a.slice_bytes = slice_bytes(a.V, sizeof(T), a.parts);
  if (wide) return top ? launch_resident<logprob_rows_kernel<T, 256, true>, 256>(a, sizeof(TopShared<256>), st)
                       : launch_resident<logprob_rows_kernel<T, 256, false>, 256>(a, 0, st);
  return top ? launch_resident<logprob_rows_kernel<T, 128, true>, 128>(a, sizeof(TopShared<128>), st)
             : launch_resident<logprob_rows_kernel<T, 128, false>, 128>(a, 0, st);
}

template <typename T>
cudaError_t launch_logprobs_grad(LogprobGradArgs a, cudaStream_t st) {
  const int units = (a.V + 15) >> 3;                       // any alignment
  int64_t blocks;
  const bool small = units <= kGradThreads;
  if (small) {
    a.tiles = units;
    blocks = ((int64_t)a.n_rows * units + kGradThreads - 1) / kGradThreads;
  } else {
    a.tiles = (units + kGradThreads * kGradUnits - 1) / (kGradThreads * kGradUnits);
    blocks = (int64_t)a.n_rows * a.tiles;
  }
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  if (small) logprob_grad_kernel<T, true><<<(unsigned)blocks, kGradThreads, 0, st>>>(a);
  else logprob_grad_kernel<T, false><<<(unsigned)blocks, kGradThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace rows
}  // namespace remoe

extern "C" int remoe_token_logprobs(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits_dev, int64_t row_stride,
                                    float inv_temperature, const int32_t* tokens_dev, int32_t top_k, float* logprob_dev,
                                    float* entropy_dev, int32_t* top_ids_dev, float* top_logprob_dev, float* row_stats_dev,
                                    void* cuda_stream) {
  using namespace remoe::rows;
  int rc = check_rows(n_rows, vocab, dtype, logits_dev, row_stride, inv_temperature);
  if (rc != REMOE_OK) return rc;
  if (top_k < 0 || top_k > vocab) return REMOE_E_ARG;
  if (top_k > REMOE_ROWS_MAX_TOP) return REMOE_E_UNSUPPORTED;
  if (top_k > 0 && (!top_ids_dev || !top_logprob_dev)) return REMOE_E_ARG;
  if (logprob_dev && !tokens_dev) return REMOE_E_ARG;
  if (!logprob_dev && !entropy_dev && !row_stats_dev && top_k == 0) return REMOE_E_ARG;
  if (misaligned(tokens_dev, 4) || misaligned(logprob_dev, 4) || misaligned(entropy_dev, 4) || misaligned(top_ids_dev, 4) ||
      misaligned(top_logprob_dev, 4) || misaligned(row_stats_dev, 4))
    return REMOE_E_ARG;
  if (n_rows == 0) return REMOE_OK;
  PointerDevice dev(logits_dev);
  if (dev.err_code() != REMOE_OK) return dev.err_code();
  const LogprobArgs a{logits_dev, row_stride, vocab, n_rows, 1, 0, top_k, inv_temperature, tokens_dev,
                      logprob_dev, entropy_dev, top_logprob_dev, row_stats_dev, top_ids_dev};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = dtype == REMOE_F32 ? launch_logprobs<float>(a, st)
                  : dtype == REMOE_BF16 ? launch_logprobs<__nv_bfloat16>(a, st) : launch_logprobs<__half>(a, st);
  return status(e);
}

extern "C" int remoe_token_logprobs_backward(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits_dev,
                                             int64_t row_stride, float inv_temperature, const int32_t* tokens_dev,
                                             const float* row_stats_dev, const float* grad_logprob_dev,
                                             const float* grad_entropy_dev, void* d_logits_dev, int64_t d_row_stride,
                                             void* cuda_stream) {
  using namespace remoe::rows;
  int rc = check_rows(n_rows, vocab, dtype, logits_dev, row_stride, inv_temperature);
  if (rc != REMOE_OK) return rc;
  if (!row_stats_dev || !d_logits_dev || (d_row_stride < vocab && n_rows > 1) || (grad_logprob_dev && !tokens_dev)) return REMOE_E_ARG;
  if (!grad_logprob_dev && !grad_entropy_dev) return REMOE_E_ARG;
  if (d_logits_dev == logits_dev && d_row_stride != row_stride && n_rows > 1) return REMOE_E_ARG;
  if (misaligned(tokens_dev, 4) || misaligned(row_stats_dev, 4) || misaligned(grad_logprob_dev, 4) ||
      misaligned(grad_entropy_dev, 4) || misaligned(d_logits_dev, element_size(dtype)))
    return REMOE_E_ARG;
  if (n_rows == 0) return REMOE_OK;
  PointerDevice dev(logits_dev);
  if (dev.err_code() != REMOE_OK) return dev.err_code();
  const LogprobGradArgs a{logits_dev, d_logits_dev, row_stride, d_row_stride, vocab, n_rows, 1, inv_temperature,
                          tokens_dev, row_stats_dev, grad_logprob_dev, grad_entropy_dev};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = dtype == REMOE_F32 ? launch_logprobs_grad<float>(a, st)
                  : dtype == REMOE_BF16 ? launch_logprobs_grad<__nv_bfloat16>(a, st) : launch_logprobs_grad<__half>(a, st);
  return status(e);
}
