// remoe_token_logprobs / remoe_token_logprobs_backward: log probabilities of given tokens, entropy and top
// alternatives of rows of logits, and the gradient.
//
//   p = softmax(s x), lp = s (x_token - m) - ln Z, H = ln Z - (1/Z) sum s (x - m) e^{s (x - m)}
//   dx = s [ g_lp (1[v = token] - p) - g_H p (ln p + H) ]
#include "logit_rows.cuh"
#include "logit_rows_host.h"

namespace remoe {
namespace rows {

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

// Shared memory of the selection: room for CAND keys, COLUMNS groups to look at again.  Keys hold (value, then lowest index
// first): all distinct, none zero.
template <int CAND, int COLUMNS>
struct alignas(16) TopShared {
  static constexpr int kCand = CAND, kColumns = COLUMNS;
  static_assert(CAND >= 2 * REMOE_ROWS_MAX_TOP && CAND % 8 == 0, "");
  unsigned long long cand[CAND + 8];
  unsigned long long sorted[REMOE_ROWS_MAX_TOP];
  unsigned short columns[COLUMNS];
  int n_columns, n_cand;
  int warp_count[16];
};

__device__ __forceinline__ unsigned long long full_key(uint32_t k, int id) { return ((unsigned long long)k << 32) | (0xffffffffu - (uint32_t)id); }

// What the selection looks at: units 0 .. n_units - 1, unit i holding the elements from 8 i + id0 on, those of [0, V) valid.
// NT threads have each seen some of them; key(i): of the largest element that thread i has seen (0: none).  A column is a
// group of units whose largest element is known; bit g of columns(i, t): column(i, g) of thread i may reach t; reach(i, t): how
// many of them do, for a t whose bits below kReachLow are zero.
//
// A block's slice in shared memory; column t: units t, t + NT, ...
template <typename T, int NT>
struct SharedSource {
  static constexpr int kKeys = NT, kAtOnce = 4, kReachLow = 0;
  const unsigned char* units;
  int n_units, id0, V;
  const uint32_t* keys;
  __device__ __forceinline__ uint32_t key(int i) const { return keys[i]; }
  __device__ __forceinline__ int reach(int i, uint32_t t) const { return keys[i] >= t; }
  __device__ __forceinline__ void load(int i, Unit<T>& q) const { load_shared_unit(units, i, q); }
  __device__ __forceinline__ int per_column() const { return (n_units + NT - 1) / NT; }
  __device__ __forceinline__ int loose() const { return 0; }           // units in no column
  __device__ __forceinline__ int loose_unit(int) const { return -1; }
  __device__ __forceinline__ int unit(int column, int k) const {
    const int i = column + k * NT;
    return i < n_units ? i : -1;
  }
  __device__ __forceinline__ unsigned columns(int, uint32_t) const { return 1u; }
  __device__ __forceinline__ int column(int i, int) const { return i; }
};
// A row in memory that passed through a pipe; column (segment, t): thread t's units of the segment's chunks.
constexpr int kSegments = 16;
template <typename T, int NT, int UNITS>
struct RowSource {
  static constexpr int kKeys = NT, kAtOnce = 6, kReachLow = 16;
  const T* row;
  int n_units, id0, V, full0, full1, pad;
  const uint32_t* keys;
  const unsigned short* seg;                       // [segment][NT] upper halves of the keys of the largest elements
  int segments, seg_chunks;
  __device__ __forceinline__ uint32_t key(int i) const { return keys[i]; }
  __device__ __forceinline__ int reach(int i, uint32_t t) const { return __popc(columns(i, t)); }
  __device__ __forceinline__ void load(int i, Unit<T>& q) const {
    if (i >= full0 && i < full1) load_unit(row - pad + 8 * (int64_t)i, q);
    else load_ragged(row, V, pad, i, q);
  }
  __device__ __forceinline__ int per_column() const { return seg_chunks * (UNITS / NT); }
  __device__ __forceinline__ int loose() const { return 2; }
  __device__ __forceinline__ int loose_unit(int i) const { return i == 0 ? (full0 > 0 ? 0 : -1) : (full1 < n_units && n_units - 1 >= full0 ? n_units - 1 : -1); }
  __device__ __forceinline__ int unit(int column, int k) const {
    const int i = full0 + (column / NT) * seg_chunks * UNITS + k * NT + column % NT;
    return i < full1 ? i : -1;
  }
  __device__ __forceinline__ unsigned columns(int i, uint32_t t) const {
    unsigned hits = 0;
#pragma unroll
    for (int g = 0; g < kSegments; ++g) hits |= seg[g * NT + i] >= t >> 16 ? 1u << g : 0u;
    return hits & ((1u << segments) - 1u);
  }
  __device__ __forceinline__ int column(int i, int g) const { return g * NT + i; }
};

// Bit j: element j of unit i, held in q, is valid and above `least` (or equal to it, where `equal`).
template <typename T, typename Source>
__device__ __forceinline__ unsigned hits_of(const Source& src, int i, const Unit<T>& q, float least, bool equal) {
  float v[8];
  q.values(v);
  unsigned hits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) hits |= v[j] > least || (equal && v[j] == least) ? 1u << j : 0u;
  const int lo = -(8 * i + src.id0), hi = src.V - (8 * i + src.id0);
  return hits & (lo > 0 ? 0xffu << lo : 0xffu) & (hi < 8 ? (1u << max(hi, 0)) - 1u : 0xffu);
}
template <typename T>
__device__ __forceinline__ float element_of(const Unit<T>& q, int j) {
  float v[8];
  q.values(v);
  float x = v[0];
#pragma unroll
  for (int m = 1; m < 8; ++m) x = j == m ? v[m] : x;
  return x;
}
__device__ __forceinline__ int scan_warp(int n) {        // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, n, o);
    if ((threadIdx.x & 31) >= o) n += up;
  }
  return n;
}

// Sum over the group's threads, in every one.
template <typename Group>
__device__ __forceinline__ int group_sum(const Group& group, int tid, int n, int* warp_count) {
  n = __reduce_add_sync(0xffffffffu, n);
  if ((tid & 31) == 0) warp_count[tid >> 5] = n;
  group.sync();
  int all = 0;
#pragma unroll
  for (int w = 0; w < Group::kThreads / 32; ++w) all += warp_count[w];
  group.sync();
  return all;
}

// The `want` largest elements of the source, sorted, to sh.sorted, by a group of FT threads (tid: 0 .. FT - 1).
//
// If t is such that `want` of the source's keys reach it, it is a lower bound of the want-th largest element, and only
// columns whose largest reaches t hold such elements: their units (a few per cent) are looked at again, what reaches t is
// listed, and the list is sorted by counting for each key the keys above it.  A lower t adds candidates and never
// loses an element.
// First t: each warp finds the value that its share of `want` of its part of the keys reach, by bits, and the least of these is
// taken; one barrier.  Where that lets too much through, or a warp's share is large, t is found from the columns' largest
// elements over the whole group, a barrier for each bit.
// In masked rows nearly all elements are equal and t is their value.  Then only what is above t is listed, and what is missing
// are the elements equal to t of the lowest indices, found in one ordered scan that stops as soon as there are enough.
// Rows whose large elements sit in few columns overflow the list all the same: there the want-th largest value is found by
// its bits, with a count over the source for each.
// Lists are filled with one addition per warp, the places within it from a scan: an addition for each entry, one behind
// the other, took 140 cycles an entry.
template <typename T, typename Group, typename Source, typename Shared>
__device__ void select_top(const Group& group, const Source& src, int tid, int want, Shared& sh) {
  constexpr int FT = Group::kThreads, kLow = Elem<T>::kUnusedBits, W = FT / 32, KPT = Source::kKeys / FT;   // kLow: the key's bits that say nothing
  constexpr uint32_t kMasked = 0x007fffffu;                                           // key of -inf, the least there is
  static_assert(Source::kKeys % FT == 0, "");
  const int n_units = src.n_units, lane = tid & 31;
  uint32_t key[KPT];
#pragma unroll
  for (int i = 0; i < KPT; ++i) key[i] = src.key(tid + i * FT);
  auto reach = [&](uint32_t x) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) n += key[i] >= x;
    return n;
  };
  // Places for n entries of each lane in a list whose length is *length.
  auto places = [&](int n, int* length) {
    const int upto = scan_warp(n);
    int at = 0;
    if (lane == 31 && upto) at = atomicAdd(length, upto);
    return __shfl_sync(0xffffffffu, at, 31) + upto - n;
  };
  uint32_t t = 0;
  bool equal = true;                                      // elements equal to t are listed, too
  int n_cand = Shared::kCand + 1;
  for (int attempt = 4 * want <= Source::kKeys && n_units >= Source::kKeys ? 0 : 1; attempt < 2 && n_cand > Shared::kCand; ++attempt) {
    t = 0;
    if (tid == 0) sh.n_columns = sh.n_cand = 0;
    if (attempt == 0) {
      const int share = (want + W - 1) / W;
      static_assert(Source::kKeys / W < 1024, "three counts in one word");
      for (int b = 30; b >= (kLow & ~1); b -= 2) {         // two bits at a time
        const uint32_t one = 1u << b;
        const unsigned n = __reduce_add_sync(0xffffffffu, (unsigned)reach(t + one) | (unsigned)reach(t + 2 * one) << 10 | (unsigned)reach(t + 3 * one) << 20);
        const int n1 = n & 1023u, n2 = n >> 10 & 1023u, n3 = n >> 20;
        const int m = n3 >= share ? 3 : n2 >= share ? 2 : n1 >= share ? 1 : 0;
        t += m * one;
        const int got = m == 3 ? n3 : m == 2 ? n2 : n1;
        if (m && got <= share + share / 8 + 1) break;
      }
      if (lane == 0) sh.warp_count[tid >> 5] = (int)t;
      group.sync();
#pragma unroll
      for (int w = 0; w < W; ++w) t = min(t, (uint32_t)sh.warp_count[w]);
      group.sync();
    } else {
      for (int b = 31; b >= (kLow > Source::kReachLow ? kLow : Source::kReachLow); --b) {
        const uint32_t cand = t | (1u << b);
        int n = 0;
        for (int i = tid; i < Source::kKeys; i += FT) n += src.reach(i, cand);
        n = group_sum(group, tid, n, sh.warp_count);
        if (n >= want) {
          t = cand;
          if (n <= want + want / 4 + 4) break;
        }
      }
    }
    if (!(t & 0x80000000u)) t |= (1u << kLow) - 1u;      // ones in a negative value's key
    t = max(t, kMasked);
    equal = group_sum(group, tid, reach(t), sh.warp_count) <= 2 * want + 32;
    unsigned mine[KPT];
    int n_mine = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      mine[i] = key[i] > t || (equal && key[i] == t) ? src.columns(tid + i * FT, t) : 0u;
      n_mine += __popc(mine[i]);
    }
    int at = places(n_mine, &sh.n_columns);
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      for (; mine[i]; mine[i] &= mine[i] - 1, ++at)
        if (at < Shared::kColumns) sh.columns[at] = (unsigned short)src.column(tid + i * FT, __ffs(mine[i]) - 1);
    group.sync();
    const int nc = sh.n_columns;
    if (nc <= Shared::kColumns) {
      const float least = key_value(t);
      const int per = src.per_column(), groups = nc + (src.loose() ? 1 : 0);
      // eight lanes a column, kAtOnce columns at once; the loose units as one more column
      constexpr int kAtOnce = Source::kAtOnce;
      for (int k0 = 0; k0 < per; k0 += 8)
        for (int g0 = tid >> 3; g0 - (tid >> 3 & 3) < groups; g0 += FT / 8 * kAtOnce) {
          Unit<T> q[kAtOnce];
          int unit[kAtOnce];
          const int k = k0 + (tid & 7);
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            const int g = g0 + i * (FT / 8);
            unit[i] = -1;
            if (g < nc) unit[i] = k < per ? src.unit(sh.columns[g], k) : -1;
            else if (g == nc && k < src.loose()) unit[i] = src.loose_unit(k);
            if (unit[i] >= 0) src.load(unit[i], q[i]);
          }
          unsigned long long hits = 0;
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i)
            if (unit[i] >= 0) hits |= (unsigned long long)hits_of<T>(src, unit[i], q[i], least, equal) << 8 * i;
          int place = places(__popcll(hits), &sh.n_cand);
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i)
            for (unsigned h = (unsigned)(hits >> 8 * i) & 0xffu; h; h &= h - 1, ++place) {
              const int m = __ffs(h) - 1;
              if (place < Shared::kCand) sh.cand[place] = full_key(order_key(element_of<T>(q[i], m)), 8 * unit[i] + m + src.id0);
            }
        }
    }
    group.sync();
    n_cand = nc <= Shared::kColumns ? sh.n_cand : Shared::kCand + 1;
    group.sync();
  }
  if (n_cand > Shared::kCand) {
    uint32_t v = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t cand = v | 1u << b;
      int n = 0;
      if (cand > kMasked) {
        const float least = key_value(cand);
        for (int i = tid; i < n_units; i += FT) {
          Unit<T> q;
          src.load(i, q);
          n += __popc(hits_of<T>(src, i, q, least, true));
        }
      } else {
        n = tid == 0 ? src.V : 0;                         // all of them
      }
      if (group_sum(group, tid, n, sh.warp_count) >= want) v = cand;
    }
    t = max(v, kMasked);
    equal = false;
    if (tid == 0) sh.n_cand = 0;
    group.sync();
    for (int i = tid; i < n_units; i += FT) {             // fewer than `want` elements in all
      Unit<T> q;
      src.load(i, q);
      for (unsigned h = hits_of<T>(src, i, q, key_value(t), false); h; h &= h - 1) {
        const int m = __ffs(h) - 1, place = atomicAdd(&sh.n_cand, 1);
        if (place < Shared::kCand) sh.cand[place] = full_key(order_key(element_of<T>(q, m)), 8 * i + m + src.id0);
      }
    }
    group.sync();
    n_cand = min(sh.n_cand, want);
  }
  if (n_cand < want && !equal) {
    const float least = key_value(t);
    for (int base = 0; base < n_units && n_cand < want; base += FT) {
      unsigned hits = 0;
      if (base + tid < n_units) {
        Unit<T> q;
        src.load(base + tid, q);
        hits = hits_of<T>(src, base + tid, q, least, true) & ~hits_of<T>(src, base + tid, q, least, false);
      }
      const int upto = scan_warp(__popc(hits));
      if (lane == 31) sh.warp_count[tid >> 5] = upto;
      group.sync();
      int at = n_cand + upto - __popc(hits), all = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (w < (tid >> 5)) at += sh.warp_count[w];
        all += sh.warp_count[w];
      }
      group.sync();
      for (; hits && at < want; hits &= hits - 1, ++at) sh.cand[at] = full_key(t, 8 * (base + tid) + __ffs(hits) - 1 + src.id0);
      n_cand = min(want, n_cand + all);
    }
  }
  if (tid < 8) sh.cand[n_cand + tid] = 0ull;              // the counts below take eight keys at a time
  group.sync();
  for (int i = tid; i < n_cand; i += FT) {
    const unsigned long long k = sh.cand[i];
    int rank = 0;
    for (int j = 0; j < n_cand; j += 8) {
      ulonglong2 o[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) o[m] = *reinterpret_cast<const ulonglong2*>(&sh.cand[j + 2 * m]);
#pragma unroll
      for (int m = 0; m < 4; ++m) rank += (o[m].x > k) + (o[m].y > k);
    }
    if (rank < want) sh.sorted[rank] = k;
  }
  group.sync();
}

__device__ __forceinline__ uint32_t top_key(float top) { return top == top ? order_key(top) : 0u; }

// (x - m) s, where x - m may lie beyond float32 and the product within.  Halving and doubling are exact.
__device__ __forceinline__ float scaled_distance(float x, float m, float s) { return 2.f * ((0.5f * x - 0.5f * m) * s); }

// What a row's outputs come from, once it is joined.
struct RowResult {
  State all;
  float ln_z;
};
__device__ __forceinline__ RowResult row_result(const State& all) { return RowResult{all, all.m == -kInf ? -kInf : log1pf(all.R)}; }
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t r, const RowResult& w, int token, float x_token) {
  const bool none = w.all.m == -kInf;
  const float h = none ? 0.f : w.ln_z - kLn2 * w.all.U / (1.f + w.all.R);
  float lp = 0.f;
  if (token >= 0 && token < a.V) lp = none ? -kInf : scaled_distance(x_token, w.all.m, a.s) - w.ln_z;
  else if (token != -1) lp = nan_value();
  if (a.logprob) a.logprob[r] = lp;
  if (a.entropy) a.entropy[r] = h;
  if (a.stats) {
    float* o = a.stats + 4 * r;
    o[0] = w.all.m; o[1] = w.ln_z; o[2] = h; o[3] = lp;
  }
}
__device__ __forceinline__ void write_alternative(const LogprobArgs& a, int64_t r, const RowResult& w, int rank, unsigned long long key) {
  const float x = key_value((uint32_t)(key >> 32));
  const bool bad = !(w.all.R == w.all.R);
  a.top_ids[r * a.top_k + rank] = bad ? -1 : (int32_t)(0xffffffffu - (uint32_t)key);
  a.top_logprob[r * a.top_k + rank] = bad ? nan_value() : w.all.m == -kInf ? -kInf : scaled_distance(x, w.all.m, a.s) - w.ln_z;
}

typedef TopShared<8 * REMOE_ROWS_MAX_TOP, 256> FewShared;   // room for the lists of a cluster's eight blocks

// Few rows: one row per cluster of `parts` blocks, each block's slice of it in shared memory.  One row of 102400 bf16 with 20
// alternatives takes 11.0 us, one of twenty calls in a captured graph: a copy, one pass, the selection (2.3 us) and the cluster's join, one
// behind the other.  32 rows of 151936 float32 with 8: 14.9 us, slices of 76 KB, two blocks on an SM.
template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT) logprob_rows_kernel(const __grid_constant__ LogprobArgs a) {
  __shared__ State per_warp[NT / 32];
  __shared__ State mine;
  __shared__ uint64_t bar;
  __shared__ uint32_t keys[TOP ? NT : 1];                      // each thread reads its own
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
  FewShared& sh = *reinterpret_cast<FewShared*>(units + a.slice_bytes);
  if (TOP) {
    const int want = min(a.top_k, sl.length(V));
    const SharedSource<T, NT> src{units, n_units, 8 * sl.first - sl.pad, V, keys};
    keys[tid] = tid < n_units ? top_key(st.top()) : 0u;
    if (want > 0) select_top<T>(WholeGroup<NT>{}, src, tid, want, sh);
  }
  __syncthreads();
  State all = mine;
  if (a.parts > 1) {
    cluster_sync();
    if (part == 0) all = join_cluster(&mine, a.parts, c);
  }
  const RowResult res = row_result(all);
  if (leader) write_row(a, r, res, token, x_token);
  if (TOP && part == 0) {
    if (a.parts == 1 || !(all.R == all.R)) {
      for (int i = tid; i < a.top_k; i += NT) write_alternative(a, r, res, i, sh.sorted[i]);
    } else {
      // the blocks' sorted lists, one behind the other in the candidates' place; a key's rank is its place in its
      // own list plus, for each other list, the number of keys above it there
      unsigned long long* lists = sh.cand;
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
        if (rank < K) write_alternative(a, r, res, rank, k);
      }
    }
  }
  if (a.parts > 1) cluster_sync();       // no block leaves while another reads its shared memory
}

typedef TopShared<768, 1024> ManyShared;

// Shape of the persistent blocks: threads that consume, threads that finish rows, blocks an SM, units of a chunk for each
// consumer, chunks in the ring.
template <typename T, bool TOP>
struct ManyShape {
  static constexpr int kConsumers = TOP ? 256 : 128, kFinishers = TOP ? 128 : 32, kBlocks = TOP ? 2 : 5;
  static constexpr int kChunk = kConsumers * 16 * (sizeof(T) == 2 ? 6 : 4), kSlots = TOP ? 2 : 3;
  static constexpr int kThreads = kConsumers + 32 + kFinishers;
  static constexpr size_t kSegBytes = (size_t)kSegments * kConsumers * sizeof(short);
  static constexpr size_t kSmem = (size_t)kChunk * kSlots + (TOP ? sizeof(ManyShared) + 2 * kSegBytes : 0);
};

// What the consumers hand over at the end of a row, twice.
template <int NT, bool TOP>
struct Handover {
  State per_warp[NT / 32];
  uint32_t keys[TOP ? NT : 1];
};

// Many rows: persistent blocks, each takes row after row through its ring of chunks.  One warp issues the copies, the
// consumers sum, and the finishers join a row's sums, select its top elements and write while the consumers are at the next
// row already (two ahead at most).  What bounds it: without alternatives the memory (4096 x 102400 bf16, calls back to back: 135 us, 0.95
// of the copy rate; 158 behind a kernel that has just written 256 MB); with them the finishers, 15 us a row, since their loads queue for 3
// to 5 us behind the copies on their way to the SM (2048 x 131072 bf16, 64 alternatives: 137 us; 110 without the selection).  The float32
// form with alternatives spills 328 bytes a thread (the 16-bit ones 56 and 8).  With fewer rows than blocks a block has one row, and
// its selection overlaps nothing (257 x 50257 fp16, 5 alternatives: 14.8 us).
template <typename T, bool TOP>
__global__ void __launch_bounds__(ManyShape<T, TOP>::kThreads, ManyShape<T, TOP>::kBlocks) logprob_pipe_kernel(const __grid_constant__ LogprobArgs a) {
  typedef ManyShape<T, TOP> Shape;
  constexpr int NT = Shape::kConsumers, FT = Shape::kFinishers, NB = Shape::kSlots, CHUNK = Shape::kChunk, ALL = NT + FT;          // of a handover
  typedef Chunks<T, CHUNK> C;
  constexpr int N = C::kUnits / NT;
  static_assert(C::kUnits % NT == 0, "whole units for every thread");
  __shared__ PipeShared<NB> ps;
  __shared__ Handover<NT, TOP> over[2];
  extern __shared__ __align__(128) unsigned char ring_buffer[];
  const int V = a.V, tid = threadIdx.x;
  const T* logits = static_cast<const T*>(a.logits);
  const float c = a.s * kLog2e;
  if (tid == 0) init_pipe(ps, NT / 32);
  __syncthreads();

  if (tid >= NT + FT) {                        // the last warp
    produce<T, NB, CHUNK>(ps, ring_buffer, RowWeights(nullptr, a.n_rows, blockIdx.x, gridDim.x), logits, a.stride, V);
    return;
  }
  unsigned char* const lists = ring_buffer + NB * CHUNK;
  auto segments_of = [&](int parity) { return reinterpret_cast<unsigned short*>(lists + sizeof(ManyShared) + parity * Shape::kSegBytes); };
  if (tid >= NT) {
    const int ft = tid - NT;
    ManyShared& sh = *reinterpret_cast<ManyShared*>(lists);
    const FinishGroup<FT> group;
    int par = 0;                               // parity of the block's row
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x, par ^= 1) {
      const T* row = logits + r * a.stride;
      const Slice sl(V, row_pad(row), 0, 1);
      int token = -1;
      T x_token = Elem<T>::masked();
      if (ft == 0 && a.tokens) {
        token = a.tokens[r];
        if (token >= 0 && token < V) x_token = row[token];
      }
      bar_sync<kBarReady, ALL>(par);
      const Handover<NT, TOP>& o = over[par];
      const RowResult res = row_result(join_warps<NT>(o.per_warp, c));
      if (ft == 0) write_row(a, r, res, token, Elem<T>::get(&x_token));
      if (TOP) {
        const int chunks = C::count(sl), seg_chunks = (chunks + kSegments - 1) / kSegments;
        const RowSource<T, NT, C::kUnits> src{row, sl.last, -sl.pad, V, sl.full0, sl.full1, sl.pad, o.keys, segments_of(par), (chunks + seg_chunks - 1) / seg_chunks, seg_chunks};
        select_top<T>(group, src, ft, a.top_k, sh);
        for (int i = ft; i < a.top_k; i += FT) write_alternative(a, r, res, i, sh.sorted[i]);
        group.sync();                          // the lists are free again
      }
      if (r + 2 * (int64_t)gridDim.x < a.n_rows) bar_arrive<kBarFree, ALL>(par);
    }
    return;
  }

  int par = 0;                                 // parity of the block's row
  RingPlace<NB> in;
  for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x, par ^= 1) {
    const T* row = logits + r * a.stride;
    const Slice sl(V, row_pad(row), 0, 1);
    const int chunks = C::count(sl), seg_chunks = (chunks + kSegments - 1) / kSegments;
    unsigned short* const seg = segments_of(par);
    Unit<T> loose[1];
    const bool has_loose = tid < 2 && sl.ragged(tid) >= 0;
    if (has_loose) load_ragged(row, V, sl.pad, sl.ragged(tid), loose[0]);
    if (r >= 2 * (int64_t)gridDim.x) bar_sync<kBarFree, ALL>(par);
    Stream<T, true, true> st(c);
    typename Elem<T>::Word all = Elem<T>::lowest();
    for (int ch = 0, in_seg = 0, g = 0; ch < chunks; ++ch) {
      const int n = C::units(sl, ch);
      in.wait(ps.full);
      const unsigned char* units = ring_buffer + in.slot * CHUNK;
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
      in.pass(ps.empty, st.top() == 1.f);
      if (TOP && (++in_seg == seg_chunks || ch + 1 == chunks)) {
        seg[g * NT + tid] = (unsigned short)(top_key(st.top()) >> 16);
        st.close_segment(all);
        in_seg = 0;
        ++g;
      }
    }
    if (has_loose) st.add(loose);
    if (TOP) {
      st.close_segment(all);
      st.M = all;
      over[par].keys[tid] = top_key(st.top());
    }
    join_warp(in.ok ? st.finish() : State{0.f, nan_value(), nan_value()}, c, over[par].per_warp);
    bar_arrive<kBarReady, ALL>(par);
  }
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
    if (token >= 0 && token < a.V) lp = none ? -kInf : scaled_distance(Elem<T>::get(row + token), all.m, a.s) - ln_z;
    else if (token != -1) lp = nan_value();
    if (a.logprob) a.logprob[r] = lp;
    if (a.entropy) a.entropy[r] = h;
    if (a.stats) {
      float* o = a.stats + 4 * r;
      o[0] = all.m; o[1] = ln_z; o[2] = h; o[3] = lp;
    }
  }
  if (a.top_k == 0) return;                        // the same for all threads
  // The alternatives one by one: each lane's keys are sorted, the group's largest head is taken and its lane moves on.
  // (2785 rows of 200 bf16, 22 alternatives: 8 us; 17.8 with a search through the lane's keys and shuffles in each round.)
  unsigned long long key[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) key[j] = 8 * lane + j < a.V ? full_key(order_key(v[j]), 8 * lane + j) : 0ull;
#pragma unroll
  for (int round = 0; round < 8; ++round)          // odd-even transposition, descending
#pragma unroll
    for (int j = round & 1; j < 7; j += 2) {
      const unsigned long long x = key[j], y = key[j + 1];
      key[j] = x > y ? x : y;
      key[j + 1] = x > y ? y : x;
    }
  const unsigned group = LPR == 32 ? 0xffffffffu : ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  unsigned long long mine = 0ull;                  // of every LPR alternatives, this lane writes one
  for (int k = 0; k < a.top_k; ++k) {
    const unsigned hi = __reduce_max_sync(group, (unsigned)(key[0] >> 32));
    const unsigned lo = __reduce_max_sync(group, (unsigned)(key[0] >> 32) == hi ? (unsigned)key[0] : 0u);
    const unsigned long long top = (unsigned long long)hi << 32 | lo;
    if (key[0] == top) {
#pragma unroll
      for (int j = 0; j < 7; ++j) key[j] = key[j + 1];
      key[7] = 0ull;
    }
    if ((k & (LPR - 1)) == lane) mine = top;
    if ((k & (LPR - 1)) == LPR - 1 || k + 1 == a.top_k) {
      const int at = (k & ~(LPR - 1)) + lane;
      if (there && at <= k) {
        const float x = key_value((uint32_t)(mine >> 32));
        a.top_ids[r * a.top_k + at] = bad ? -1 : (int32_t)(0xffffffffu - (uint32_t)mine);
        a.top_logprob[r * a.top_k + at] = bad ? nan_value() : none ? -kInf : scaled_distance(x, all.m, a.s) - ln_z;
      }
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

constexpr int kGradThreads = 256;
template <typename T>
constexpr int kGradUnits = sizeof(T) == 2 ? 4 : 1;

// 4096 rows of 102400 bf16, a fifth of them padding: 249 us, 6.1 TB/s, 0.93 of the copy rate on the bytes that are moved (273 behind kernels that
// leave writes in L2).
// Element-wise: what a row's gradient shares is in its row_stats.  Long rows: `tiles` blocks a row, each thread 64 bytes
// (32 of float32: twice the registers a byte).  Short rows (SMALL): one unit a thread over all rows' units.
template <typename T, bool SMALL>
__global__ void __launch_bounds__(kGradThreads) logprob_grad_kernel(const __grid_constant__ LogprobGradArgs a) {
  constexpr int N = SMALL ? 1 : kGradUnits<T>;
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
  int token = a.tokens ? a.tokens[r] : -1;
  const bool outside = token < -1 || token >= V;
  const float g = a.g_logprob && token != -1 ? a.g_logprob[r] : 0.f;
  if (outside) token = -1;                    // the entropy's gradient knows no token
  const float gh = a.g_entropy ? a.g_entropy[r] : 0.f;
  const bool zero = (g == 0.f && gh == 0.f) || m == -kInf;
  const bool bad = !zero && outside && g != 0.f;
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
    const int64_t n = a.n_rows;
    return a.V <= 64    ? launch<logprob_small_kernel<T, 8>>(a, (n + 31) / 32, 1, 256, 0, st)
           : a.V <= 128 ? launch<logprob_small_kernel<T, 16>>(a, (n + 15) / 16, 1, 256, 0, st)
                        : launch<logprob_small_kernel<T, 32>>(a, (n + 7) / 8, 1, 256, 0, st);
  }
  if (many_rows(a.n_rows, a.V) && (!top || a.V >= 32768)) {
    return top ? launch_pipe<logprob_pipe_kernel<T, true>, ManyShape<T, true>>(a, st)
               : launch_pipe<logprob_pipe_kernel<T, false>, ManyShape<T, false>>(a, st);
  }
  // 256 threads a block for long rows and for many alternatives; with few of those the selection's fixed steps weigh more than the
  // pass, and more blocks of 128 lie beside one another.  (5000 rows of 9000 bf16, 20 alternatives: 64 us with 128 threads, 81 with
  // 256; of 16000: 91 and 94, with 64 alternatives 135 and 118.)
  const bool few = a.top_k > 0 && a.top_k <= 32;
  const bool wide = a.V >= (few ? 32768 : 8192) || a.top_k > 64;
  a.parts = parts_of_row(a.n_rows, a.V, sizeof(T));
  a.slice_bytes = slice_bytes(a.V, sizeof(T), a.parts);
  if (wide) return top ? launch_resident<logprob_rows_kernel<T, 256, true>, 256>(a, sizeof(FewShared), st)
                       : launch_resident<logprob_rows_kernel<T, 256, false>, 256>(a, 0, st);
  return top ? launch_resident<logprob_rows_kernel<T, 128, true>, 128>(a, sizeof(FewShared), st)
             : launch_resident<logprob_rows_kernel<T, 128, false>, 128>(a, 0, st);
}

template <typename T>
cudaError_t launch_logprobs_grad(LogprobGradArgs a, cudaStream_t st) {
  const int units = (a.V + 14) >> 3;                       // any alignment
  if (units <= kGradThreads) {
    a.tiles = units;
    return launch<logprob_grad_kernel<T, true>>(a, ((int64_t)a.n_rows * units + kGradThreads - 1) / kGradThreads, 1, kGradThreads, 0, st);
  }
  a.tiles = (units + kGradThreads * kGradUnits<T> - 1) / (kGradThreads * kGradUnits<T>);
  return launch<logprob_grad_kernel<T, false>>(a, (int64_t)a.n_rows * a.tiles, 1, kGradThreads, 0, st);
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
